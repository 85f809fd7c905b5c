"""Block attention over shared pages where calls are rare: sizes at the ends of the allowed ranges (against 64 bits, with
the tolerances of test_gpu_prefix_attention.py)."""
import pytest
import torch

import synth
from test_gpu_prefix_attention import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import paper_2403_18647_gb300 as sd
    return sd


def test_heads_of_half_the_size_on_a_context_of_many(sd):
    """2000 heads of 64 dimensions with 64 rows each, as many as a context of 1000 heads of 128 takes (one head in 40 is
    compared)."""
    ctx = sd.Context(synth.ModelShape("wide", 1, 128, 1000, 128, 256, 256, 0), None, max_position=64)
    c = Case(18, 4, 16, 2000, 2000, 64, [3, 60, 64, 130], 0)
    some = lambda x: x.view(64, 2000, 64)[:, 7::40].reshape(64, -1)  # noqa: E731
    out = c.run(ctx)
    assert torch.isfinite(out).all()
    c.dims, c.x, c.k, c.v = (4, 16, 50, 50, 64), some(c.x), c.k[:, 7::40], c.v[:, 7::40]
    c.check(some(out))
    assert ctx.get_error() == 0
