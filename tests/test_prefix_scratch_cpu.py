"""The prefix attention's scratch holds the partial results of every call that a context accepts."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "prefix_scratch.h"
// argv: CTAs, then pairs (row dims of a context, hd of a call); prints allocated and needed floats
int main(int n, char** v) {
  const int ctas = std::atoi(v[1]);
  for (int i = 2; i + 1 < n; i += 2) {
    const size_t dims = std::strtoull(v[i], nullptr, 10), hd = std::strtoull(v[i + 1], nullptr, 10);
    std::printf("%zu %zu\n", sdsat::prefix_attention_scratch(dims, ctas), sdsat::px_scratch_floats(dims / hd, (int)hd, ctas));
  }
}
"""


@pytest.fixture(scope="module")
def sizes(tmp_path_factory):
    at = tmp_path_factory.mktemp("scratch")
    (at / "main.cpp").write_text(PROGRAM)
    exe = str(at / "main")
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2403_18647_gb300", "csrc"), str(at / "main.cpp"), "-o", exe],
                   check=True)
    return lambda ctas, pairs: [tuple(map(int, line.split())) for line in subprocess.run(
        [exe, str(ctas)] + [str(x) for p in pairs for x in p], check=True, capture_output=True, text=True).stdout.splitlines()]


@pytest.mark.parametrize("ctas", [1, 148, 152])
def test_every_accepted_call_fits(sizes, ctas):
    """Contexts of 1 to 4000 heads of 64 and 128 dimensions, calls with heads of either size."""
    contexts = [64 * h * hd for hd in (64, 128) for h in (2, 4, 20, 32, 40, 64, 972, 974, 1000, 4000)]
    got = sizes(ctas, [(c, hd) for c in contexts for hd in (64, 128)])
    assert len(got) == 2 * len(contexts)
    for (have, need), c, hd in zip(got, [c for c in contexts for _ in (0, 1)], [64, 128] * len(contexts)):
        assert have >= need, (c, hd)
        # two rows of partial results for each row and head, and 64 of each CTA, of hd values, a reference and four sums
        assert need >= (2 * (c // hd) + 64 * ctas) * (hd + 5)
