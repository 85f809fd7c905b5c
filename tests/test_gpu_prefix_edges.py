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


def test_cache_heads_of_more_queries_than_a_reciprocal_divides_are_refused(sd):
    """Rows of a cache head are divided by its query heads with 32-bit reciprocals: their number times G < 2^32."""
    ctx = sd.Context(synth.ModelShape("wide", 1, 128, 1000, 128, 256, 256, 0), None, max_position=64)

    def call(H, Hk=1):
        c = Case(19, 1, 1, H, Hk, 64, [2], 0)
        return c, c.run(ctx)

    for H, Hk in ((65536, 1), (128000, 1), (128000, 2)):
        with pytest.raises(sd.SdsatError) as e:
            call(H, Hk)
        assert e.value.status == 1
    c, out = call(65535)
    some = lambda x: x.view(1, 65535, 64)[:, 65500:].reshape(1, -1)  # noqa: E731
    c.dims, c.x = (1, 1, 35, 1, 64), some(c.x)
    c.check(some(out))
    assert ctx.get_error() == 0


@pytest.mark.parametrize("H,hd,type", [(40, 128, torch.float32), (64, 64, torch.float32), (40, 128, torch.bfloat16)])
def test_many_short_segments_on_every_sm(sd, H, hd, type):
    """Some twenty items of one unit for each CTA, so that the segments' descriptions go round several times: every
    call gives the same bits."""
    ctx = sd.Context(synth.SHAPES["13b"], None, max_position=64)
    c = Case(20, 64, 1, H, H, hd, [s % 5 for s in range(64)], 0, type)
    out = c.run(ctx)
    c.check(out)
    for _ in range(100):
        assert torch.equal(c.run(ctx), out)
    assert ctx.get_error() == 0
