"""What the parts, the totals and the joins of the chunk attention leave of an error.

fp32: queries and probabilities hold 24 bits, a score is an fp32 sum of 3 * hd / 16 products of 16 (truncated, 2^-23 each, small
parts first, so hd / 16 of them count), a step's O one of 3 * 4 products, the total is rounded: relative to sum p |v| a row is off by
2^-23 (hd / 16 + 4 + steps / 2 ...) at the worst and by about the root of that.  The root mean square of the error against the
root mean square of the result stays below 2^-20 (1e-6) whatever the length.
bf16: P and the result are rounded to 8 bits, 2^-9 / sqrt(3) each in the mean; of the P's roundings the row's mean is
taken with the same weights as its values: sqrt(2) 2^-9 / sqrt(3) = 1.6e-3 in all for values of mean 0, 2.5e-3 with room."""
import pytest
import torch

import synth
from ragged import Pages, attention, generator

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_2403_18647_gb300 as sd
    return sd.Context(synth.SHAPES["tiny"], None, max_position=64)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new,held", [([1], [31000]), ([40, 3], [9000, 17000]), ([2500], [0]), ([130, 130, 130], [0, 64, 2000])])
def test_errors_in_the_mean(ctx, hd, new, held):
    for type, most in ((torch.float32, 2 ** -20), (torch.bfloat16, 2.5e-3)):
        g = generator(len(new) + hd)
        H, Hk = 8, 2
        p = Pages(g, Hk, hd, new, held)
        q = (torch.randn(p.rows, H * hd, generator=g, device="cuda") * 1.5).to(type)
        out = torch.empty_like(q)
        ctx.op_chunk_attention(q, p.k, p.v, p.table, p.lens, p.starts, H, Hk, hd, out)
        ref, _ = attention(p, q, H, Hk, hd)
        rel = ((out.double().view(ref.shape) - ref).norm() / ref.norm()).item()
        assert rel <= most, rel


@pytest.mark.parametrize("type", [torch.float32, torch.bfloat16])
def test_growing_maxima(ctx, type):
    """Scores that grow from step to step, so that every reference moves: O and the total are rescaled each time."""
    g = generator(9)
    H, hd = 4, 128
    p = Pages(g, 1, hd, [150], [1500])
    q = torch.randn(p.rows, H * hd, generator=g, device="cuda").to(type)
    lead = torch.randn(hd, generator=g, device="cuda")
    q.view(-1, hd).add_(lead.to(type))
    for j, page in enumerate(p.table[0].tolist()):
        if page >= 0:
            p.k[page] = (p.k[page].float() * 0.1 + lead * (j * 0.2)).bfloat16()   # q k / sqrt(hd) grows by 2 and more a page
    out = torch.empty_like(q)
    ctx.op_chunk_attention(q, p.k, p.v, p.table, p.lens, p.starts, H, 1, hd, out)
    ref, size = attention(p, q, H, 1, hd)
    err = (out.double().view(ref.shape) - ref).abs()
    # scores reach 60: an fp32 score is 60 * hd / 16 * 2^-23 off at the worst, which the weights are in proportion
    slack = size * 60 * 8 * 2 ** -22 + 2e-5
    if type == torch.bfloat16:
        slack = slack + 2 ** -8 * (ref.abs() + size)
    assert (err - slack).max().item() <= 0
