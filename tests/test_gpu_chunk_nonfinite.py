"""NaN and infinities that rows see stay visible in the chunk attention's results, however the batch is divided.

Tolerances of the other rows as in test_gpu_chunk_attention.py."""
import math

import pytest
import torch

import synth
from ragged import PAGE, Pages, attention, generator

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16

# H, Hk, hd, new rows, committed slots: items cut along their keys with a thread for each row at the join (the first two: 130
# and 100 rows), with a warp for each (few rows), and not cut
CASES = [(2, 2, 128, 130, 1500), (4, 2, 64, 50, 3000), (2, 1, 128, 3, 5000), (4, 4, 64, 40, 30)]


@pytest.fixture(scope="module")
def ctx():
    import paper_2403_18647_gb300 as sd
    return sd.Context(synth.SHAPES["tiny"], None, max_position=64)


def check(ctx, p, q, H, Hk, hd):
    out = torch.empty_like(q)
    ctx.op_chunk_attention(q, p.k, p.v, p.table, p.lens, p.starts, H, Hk, hd, out)
    ref, size = attention(p, q, H, Hk, hd)
    got = out.double().view(ref.shape)
    assert torch.equal(got.isnan(), ref.isnan())
    err = (got - ref).abs()
    if q.dtype == BF16:
        err = err - 2 ** -8 * (ref.abs() + size)
    fine = ~ref.isnan()
    assert fine.any() and not fine.all() and err[fine].max().item() <= 2e-5
    assert ctx.get_error() == 0


def batch(seed, type, H, Hk, hd, new, held):
    g = generator(seed)
    p = Pages(g, Hk, hd, [new], [held])
    return p, (torch.randn(new, H * hd, generator=g, device="cuda") * 1.5).to(type)


@pytest.mark.parametrize("H,Hk,hd,new,held", CASES)
@pytest.mark.parametrize("type", [F32, BF16])
def test_a_query(ctx, type, H, Hk, hd, new, held):
    p, q = batch(1, type, H, Hk, hd, new, held)
    for row in {0, new // 2, new - 1}:
        q[row, hd + 5] = math.nan                          # of head 1 alone
        check(ctx, p, q, H, Hk, hd)


@pytest.mark.parametrize("H,Hk,hd,new,held", CASES)
@pytest.mark.parametrize("type", [F32, BF16])
def test_a_key_and_a_value(ctx, type, H, Hk, hd, new, held):
    """That only the last rows see, and that all rows of a cache head see."""
    for slot in (held + new // 2, held + new - 1, held // 2):
        p, q = batch(2, type, H, Hk, hd, new, held)
        p.k[p.table[0, slot // PAGE].long(), 0, slot % PAGE, 3] = math.nan
        if Hk == 1 and slot < held:                        # (no row of another head is finite)
            q = q[:, :hd].contiguous().repeat(1, H)
            out = torch.zeros_like(q)
            ctx.op_chunk_attention(q, p.k, p.v, p.table, p.lens, p.starts, H, Hk, hd, out)
            assert out.isnan().all()
        else:
            check(ctx, p, q, H, Hk, hd)
    p, q = batch(3, type, H, Hk, hd, new, held)
    p.v[p.table[0, held // 2 // PAGE].long(), 0, held // 2 % PAGE, 3] = math.nan
    check(ctx, p, q, H, Hk, hd)


@pytest.mark.parametrize("H,Hk,hd,new,held", CASES)
def test_infinite_scores(ctx, H, Hk, hd, new, held):
    """A score of -inf has no weight, one of inf leaves a row no value."""
    p, q = batch(4, BF16, H, Hk, hd, new, held)
    p.k[p.table[0, held // 2 // PAGE].long(), 0, held // 2 % PAGE, 3] = math.inf
    check(ctx, p, q, H, Hk, hd)
