"""Checks of the model-end operators' host side and sources that need no GPU."""
import os
import re
import shutil
import subprocess
from types import SimpleNamespace

import pytest

from paper_2609_37842_gb300 import build as B
from paper_2609_37842_gb300 import eogp as E

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()
    E.lib()


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


SORT_PLAN_CHECK = r"""
#include "sort_plan.h"
#include <initializer_list>
#include <cstdio>
int main() {
  const long long most = 1ll << 30;
  for (int V : {1, 2, 511, 512, 513, 50000, 262143, 262144, 1 << 30})
    for (long long M : {0ll, 1ll, 4095ll, 4096ll, 4097ll, 32768ll, 32769ll, 1048576ll, 1048577ll, most - 1, most}) {
      const SortPlan p = sort_plan(V, M);
      const bool keys = p.bits <= kMaxSortBits && p.bins == 1 << p.bits && (1ll << (p.passes * p.bits)) > V;
      const bool all = p.blocks <= kMaxSortBlocks && static_cast<long long>(p.blocks) * p.per_block >= M;
      const bool used = M == 0 ? p.blocks == 0 : static_cast<long long>(p.blocks - 1) * p.per_block < M;
      if (!keys || !all || !used) {
        std::printf("V %d M %lld: %d passes of %d bits, %d blocks of %d\n", V, M, p.passes, p.bits, p.blocks,
                    p.per_block);
        return 1;
      }
    }
  return 0;
}
"""


def test_sort_plan(tmp_path):
    """The plan of the embedding gradient's sort, compiled without optimisation and with undefined arithmetic trapped:
    it covers all positions and keys, and a batch without positions needs no block."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(SORT_PLAN_CHECK)
    subprocess.run([gxx, "-std=c++17", "-O0", "-fsanitize=undefined", "-fsanitize-undefined-trap-on-error",
                    "-I", B.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stdout)


def test_tensors_of_a_device_that_is_not_current(monkeypatch):
    """The library launches on the current device, whose kernels could not read another device's memory."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    t = SimpleNamespace(device=torch.device("cuda", 1))
    for f in (lambda: E.norm(t), lambda: E.embed(t, t), lambda: E.embed_grad(t, t, 4), lambda: E.cross_entropy(t, t),
              lambda: E.norm_grad(t, t, t, t)):
        with pytest.raises(ValueError, match="current CUDA device"):
            f()


def test_sizes_beyond_a_c_int(monkeypatch):
    """A call whose size a C int does not hold is refused, not made on the size's lowest 32 bits. The tensors are
    views of a few elements."""
    monkeypatch.setattr(E, "_device_of", lambda *t: torch.device("cpu"))
    n = 2 ** 32 + 2
    rows, tok = torch.zeros(1, 1, 8), torch.zeros((1, 1), dtype=torch.int64)
    many, toks = rows.expand(n, 1, 8), tok.expand(n, 1)
    stat = torch.zeros(1, 1).expand(n, 1)
    small = torch.zeros(2, 1, 8)
    for f in (lambda: E.norm(many, out=many), lambda: E.norm_grad(many, many, stat, stat),
              lambda: E.embed(toks, torch.zeros(4, 8), out=many), lambda: E.embed(tok, torch.zeros(1, 8).expand(n, 8)),
              lambda: E.embed_grad(toks, many, 4), lambda: E.embed_grad(tok.expand(2, 1), small, n),
              lambda: E.cross_entropy(many, toks, dlogits=many)):
        with pytest.raises(E.EOGPError) as e:
            f()
        assert e.value.code == E.EUNSUPPORTED
