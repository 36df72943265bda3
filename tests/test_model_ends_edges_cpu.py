"""Checks of the model-end operators' host side and sources that need no GPU."""
import os
import re

from paper_2609_37842_gb300 import build as B


def test_an_expired_wait_is_answered():
    """A bounded wait that runs out must change what the kernel does next: a CTA that went on would use stale data,
    and might leave while another still stores to its shared memory. Only the drain after an expired wait, which has
    a shorter limit of its own, may drop the result."""
    waits = 0
    for name in ("k_embed.cu", "k_loss.cu", "k_norm.cu"):
        with open(os.path.join(B.CSRC, name)) as fh:
            for line in fh:
                if re.search(r"\bmbar_wait(_cluster)?\(", line):
                    waits += 1
                    dropped = re.match(r"\s*mbar_wait(_cluster)?\(", line)
                    assert not dropped or "EOGP_WAIT_CYCLES /" in line, (name, line)
    assert waits
