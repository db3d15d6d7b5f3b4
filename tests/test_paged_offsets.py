"""CPU tests of what a ragged batch's numbers are taken to say (csrc/paged.h), whatever they are: the same code that the
kernels run, compiled for the host."""
import itertools
import os
import shutil
import subprocess

import pytest

from paper_2606_24033_amd import build

PROGRAM = r"""
#include <cstdio>
#include "paged.h"
int main() {
  bgtq::PagedBatch b = {};
  int c0, c1, len;
  while (std::scanf("%d %d %d %d %d %d", &b.n_tokens, &b.max_new, &b.max_ctx, &c0, &c1, &len) == 6) {
    const bgtq::paged::Seq s = bgtq::paged::make_seq(b, c0, c1, len);
    std::printf("%d %d %d %d\n", s.first, s.n, s.len, s.ok ? 1 : 0);
  }
  return 0;
}
"""
LO, HI = -2 ** 31, 2 ** 31 - 1


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which(build.HIPCC) is None:
        pytest.skip("no hipcc")
    d = tmp_path_factory.mktemp("paged_offsets")
    (d / "main.hip").write_text(PROGRAM)
    # (signed overflow wraps, as on the device: a host compiler may do anything with it)
    subprocess.run([build.HIPCC, "-x", "hip", "--offload-host-only", "-O2", "-std=c++17", "-fwrapv", "-I", build.CSRC, "-I",
                    os.path.join(build.ROOT, "include"), str(d / "main.hip"), "-o", str(d / "main")], check=True)

    def run(rows):
        text = "\n".join(" ".join(map(str, r)) for r in rows)
        out = subprocess.run([str(d / "main")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def test_any_offsets_stay_inside_the_inputs(program):
    """A sequence's tokens lie inside the inputs whatever its offsets are, and it is taken as it stands only where they
    and its length contradict neither each other nor the host's bounds."""
    offsets = [LO, LO + 1, LO + 5, -20, -1, 0, 1, 5, 6, 19, 20, 21, 25, 2 ** 30, HI - 5, HI - 1, HI]
    lengths = [LO, -1, 0, 1, 14, 15, 20, 99, 100, 101, HI]
    rows = [(n, new, 100, c0, c1, length) for n, new in ((20, 20), (20, 15), (0, 0), (1, 1), (HI, HI))
            for c0, c1, length in itertools.product(offsets, offsets, lengths)]
    got = program(rows)
    assert len(got) == len(rows)
    for (n, new, ctx, c0, c1, length), (first, count, seen, ok) in zip(rows, got):
        case = (n, new, c0, c1, length)
        assert 0 <= first <= n and 0 <= count and first + count <= n, case
        valid = 0 <= c0 <= c1 <= n and c1 - c0 <= new and c1 - c0 <= length <= ctx
        assert bool(ok) == valid, case
        if valid:
            assert (first, count, seen) == (c0, c1 - c0, length), case
