"""Sequences with many more rows than their table holds, whose items are cut, and what the context computes after them.

Tolerances as in test_gpu_chunk_attention.py."""
import math

import pytest
import torch

import synth
from ragged import PAGE, Pages, attention, generator

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def sd():
    import paper_2403_18647_gb300 as sd
    return sd


def call(ctx, p, q, H, Hk, hd):
    out = torch.full_like(q, math.nan)
    ctx.op_chunk_attention(q, p.k, p.v, p.table, p.lens, p.starts, H, Hk, hd, out)
    return out


def check(p, q, out, H, Hk, hd):
    ref, size = attention(p, q, H, Hk, hd)
    err = (out.double().view(ref.shape) - ref).abs()
    if out.dtype == BF16:
        err = err - 2 ** -8 * (ref.abs() + size)
    assert err.max().item() <= 2e-5


@pytest.mark.parametrize("type,H,hd,columns,new,held", [(BF16, 1, 128, 8, [3840], [0]), (F32, 1, 128, 8, [3785], [0]), (BF16, 2, 64, 8, [3175], [0]),
                                                        (F32, 2, 64, 30, [5000, 3], [100, 1900]), (BF16, 4, 128, 12, [1, 2900, 700], [767, 500, 0])])
def test_cut_items_past_the_table(sd, type, H, hd, columns, new, held):
    ctx = sd.Context(synth.SHAPES["tiny"], None, max_position=64)
    g = generator(sum(new))
    valid = Pages(g, 4, 128, [200], [6000])
    x = (torch.randn(200, 4 * 128, generator=g, device="cuda") * 1.5).to(type)
    p = Pages(g, H, hd, new, [min(m, columns * PAGE) for m in held])
    p.table = p.table[:, :columns].contiguous()
    q = (torch.randn(p.rows, H * hd, generator=g, device="cuda") * 1.5).to(type)
    for _ in range(2):
        out = call(ctx, p, q, H, H, hd)
        assert ctx.get_error() == sd.DEV_PAGE
        check(p, q, out, H, H, hd)
        out = call(ctx, valid, x, 4, 4, 128)              # its items are cut, too: the counts of their parts began at zero
        assert ctx.get_error() == 0
        check(valid, x, out, 4, 4, 128)
