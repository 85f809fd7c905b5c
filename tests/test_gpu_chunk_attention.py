"""Attention of a ragged batch's new rows over pages, against 64 bits.

Tolerances.  fp32: queries and probabilities in parts that hold 24 bits, fp32 sums, exps 2^-22 off; outputs are O(1):
2e-5 absolute, as for the other attention kernels.  bf16: the result is rounded once (2^-8 |ref|) and so is every
probability (2^-8 of sum p |v|), beside that 2e-5.
"""
import math

import pytest
import torch

import synth
from ragged import PAGE, Pages, attention, generator, ints

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def sd():
    import paper_2403_18647_gb300 as sd
    return sd


@pytest.fixture(scope="module")
def ctx(sd):
    return sd.Context(synth.SHAPES["tiny"], None, max_position=64)


def queries(g, rows, H, hd, type, scale=1.5):
    return (torch.randn(rows, H * hd, generator=g, device="cuda") * scale).to(type)


def run(ctx, p, q, H, Hk, hd, out=None):
    out = torch.full_like(q, math.nan) if out is None else out
    ctx.op_chunk_attention(q, p.k, p.v, p.table, p.lens, p.starts, H, Hk, hd, out)
    return out


def check(p, q, out, H, Hk, hd):
    ref, size = attention(p, q, H, Hk, hd)
    mine = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    for at, n in zip(p.first, p.new):
        mine[at:at + n] = True
    err = (out.double().view(ref.shape) - ref).abs()[mine]
    if out.dtype == BF16:
        err = err - (ref.abs() + size)[mine] * 2 ** -8
    assert err.numel() == 0 or err.max().item() <= 2e-5, err.max().item()


SIZES = [
    # H, Hk, hd, new rows, committed slots
    (1, 1, 64, [1], [0]), (2, 2, 128, [1], [1]), (4, 4, 64, [6, 3], [64, 63]), (4, 4, 128, [127], [0]), (4, 2, 128, [128, 1], [0, 127]),
    (4, 4, 128, [129], [0]), (2, 2, 64, [255, 256, 257], [0, 1, 0]), (4, 4, 128, [64, 64], [64, 128]), (32, 8, 128, [1] * 9, list(range(60, 69))),
    (8, 1, 64, [16, 17, 33], [100, 0, 300]), (14, 2, 64, [5, 40], [90, 1000]), (20, 4, 128, [25, 26, 52, 53], [7, 0, 200, 511]),
    (40, 40, 128, [300], [777]), (32, 4, 128, [700, 1, 30], [50, 2500, 129]), (128, 1, 64, [3, 1], [200, 0]), (15, 5, 128, [43, 86, 200], [1, 2, 3]),
    (6, 2, 64, [0, 5, 0, 0, 130, 0], [9, 0, 64, 0, 70, 128]), (4, 4, 64, [1500], [0]), (2, 1, 128, [1], [20000]), (2, 2, 64, [2, 130], [9000, 12000]),
    (64, 64, 64, [1, 2, 3], [0, 5, 129]), (1, 1, 128, [640], [5000]),
]


@pytest.mark.parametrize("H,Hk,hd,new,held", SIZES)
@pytest.mark.parametrize("type", [F32, BF16])
def test_sizes(ctx, H, Hk, hd, new, held, type):
    g = generator(sum(new) + H)
    p = Pages(g, Hk, hd, new, held).spoil(math.nan)
    q = queries(g, p.rows, H, hd, type)
    check(p, q, run(ctx, p, q, H, Hk, hd), H, Hk, hd)
    assert ctx.get_error() == 0


@pytest.mark.parametrize("type", [F32, BF16])
def test_many_sequences(ctx, type):
    """More sequences than threads of a block, most of them of a row, some of none."""
    g = generator(1)
    new = [(7 * s) % 3 for s in range(1024)]
    held = [(s * 37) % 200 for s in range(1024)]
    p = Pages(g, 2, 64, new, held).spoil(math.inf)
    q = queries(g, p.rows, 4, 64, type)
    check(p, q, run(ctx, p, q, 4, 2, 64), 4, 2, 64)
    assert ctx.get_error() == 0


@pytest.mark.parametrize("type", [F32, BF16])
@pytest.mark.parametrize("scale", [0.0, 30.0])
def test_flat_and_peaked_scores(ctx, type, scale):
    """All slots alike, and one slot that takes everything, late ones among them (the running maximum grows)."""
    g = generator(2)
    p = Pages(g, 2, 128, [200, 3], [900, 40])
    p.k *= 3
    q = queries(g, p.rows, 4, 128, type, scale)
    out = run(ctx, p, q, 4, 2, 128)
    ref, size = attention(p, q, 4, 2, 128)
    err = (out.double().view(ref.shape) - ref).abs()
    # scores reach 30 * 3 * sqrt(128) / 8.. a thousand: an fp32 product of 128 terms is 128 * 2^-24 * sum |q k| / sqrt(hd) off
    slack = 2e-5 + 2 * size * (128 * 2 ** -24 * scale * 3 * 128 ** 0.5)
    if type == BF16:
        slack = slack + (ref.abs() + size) * 2 ** -8
    assert (err - slack).max().item() <= 0
    assert ctx.get_error() == 0


@pytest.mark.parametrize("type", [F32, BF16])
def test_rows_of_no_sequence_and_strides(ctx, type):
    """Rows before the first sequence and behind the last stay as they are; rows any distance apart."""
    g = generator(3)
    H, Hk, hd = 4, 2, 64
    p = Pages(g, Hk, hd, [20, 150], [100, 3], before=5)
    rows = p.rows + 9
    wide = torch.randn(rows, H * hd + 72, generator=g, device="cuda").to(type)
    q = wide[:, 8:8 + H * hd]
    hold = torch.full((rows, H * hd + 40), 7.0, dtype=type, device="cuda")
    out = run(ctx, p, q, H, Hk, hd, hold[:, 16:16 + H * hd])
    check(p, q.contiguous(), out.contiguous(), H, Hk, hd)
    assert (hold[:5] == 7).all() and (hold[p.rows:] == 7).all() and (hold[:, :16] == 7).all() and (hold[:, 16 + H * hd:] == 7).all()
    assert ctx.get_error() == 0


@pytest.mark.parametrize("type", [F32, BF16])
def test_the_result_may_replace_the_queries(ctx, type):
    g = generator(4)
    p = Pages(g, 4, 128, [70, 1, 300], [700, 90, 0])
    q = queries(g, p.rows, 8, 128, type)
    out = run(ctx, p, q, 8, 4, 128)
    again = q.clone()
    run(ctx, p, again, 8, 4, 128, again)
    assert torch.equal(out, again)


@pytest.mark.parametrize("type", [F32, BF16])
def test_missing_pages(sd, ctx, type):
    """Slots without a page are reported and left out; a row that sees none is 0."""
    g = generator(5)
    p = Pages(g, 2, 64, [40, 3, 200], [300, 0, 500], columns=1)
    p.spoil(math.nan)
    p.table[0, 1] = -1
    p.table[0, 3] = p.k.shape[0]
    p.table[1, 0] = 1 << 30
    p.table[2, 0:5] = -7
    q = queries(g, p.rows, 4, 64, type)
    out = run(ctx, p, q, 4, 2, 64)
    assert ctx.get_error() == sd.DEV_PAGE
    check(p, q, out, 4, 2, 64)
    assert (out[40:43] == 0).all()


@pytest.mark.parametrize("type", [F32, BF16])
def test_slots_past_the_table(sd, ctx, type):
    """Lengths that reach past the table's columns, and absurd ones: what the table holds is attended to."""
    g = generator(6)
    p = Pages(g, 2, 64, [10, 4, 70], [128 - 4, 100, 60])
    p.table = p.table[:, :2].contiguous()
    q = queries(g, p.rows, 2, 64, type)
    out = run(ctx, p, q, 2, 2, 64)
    assert ctx.get_error() == sd.DEV_PAGE
    check(p, q, out, 2, 2, 64)
    p.lens = ints([2 ** 31 - 1, -5, 2 ** 30])
    out = run(ctx, p, q, 2, 2, 64)
    assert ctx.get_error() == sd.DEV_PAGE
    # all 128 slots for the first and the last, slots 0 .. i of the second (its length counts as 0)
    p.ctx = [128, 0, 128]
    p.table = torch.cat([p.table, torch.full((3, 9), -1, dtype=torch.int32, device="cuda")], 1)
    check(p, q, out, 2, 2, 64)


def test_starts_that_do_not_ascend(sd, ctx):
    g = generator(7)
    p = Pages(g, 2, 64, [10, 4, 70], [100, 9, 60])
    q = queries(g, p.rows, 2, 64, F32)
    for starts in ([0, 10, 5, 84], [-1, 10, 14, 84], [0, 10, 14, 85], [3, 2, 1, 0], [0, 10, 14, 2 ** 31 - 1], [-2 ** 31, 0, 0, 0]):
        p.starts = ints(starts)
        out = run(ctx, p, q, 2, 2, 64, torch.full_like(q, 7.0))
        assert ctx.get_error() == sd.DEV_CAPACITY and (out == 7).all()
    p.starts = ints([20, 20, 20, 20])
    out = run(ctx, p, q, 2, 2, 64, torch.full_like(q, 7.0))
    assert ctx.get_error() == 0 and (out == 7).all()


def test_results_do_not_change_from_call_to_call(ctx):
    g = generator(8)
    for new, held in (([1, 1, 40], [9000, 300, 100]), ([600], [3000])):
        p = Pages(g, 8, 128, new, held)
        q = queries(g, p.rows, 32, 128, BF16)
        first = run(ctx, p, q, 32, 8, 128)
        for _ in range(5):
            assert torch.equal(first, run(ctx, p, q, 32, 8, 128))


def test_streams_and_graphs(ctx):
    """On a side stream, and captured: a replay reads the lengths, starts and pages of its time."""
    g = generator(9)
    H, Hk, hd = 8, 2, 128
    p = Pages(g, Hk, hd, [60, 1, 33], [500, 2000, 0])
    q = queries(g, p.rows, H, hd, BF16)
    out = run(ctx, p, q, H, Hk, hd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run(ctx, p, q, H, Hk, hd)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, again)
    graph = torch.cuda.CUDAGraph()
    hold = torch.zeros_like(q)
    with torch.cuda.graph(graph):
        run(ctx, p, q, H, Hk, hd, hold)
    graph.replay()
    assert torch.equal(hold, out)
    p.new, p.ctx, p.first = [10, 80, 2], [300, 1900, 40], [1, 11, 91]
    p.starts.copy_(ints([1, 11, 91, 93]))
    p.lens.copy_(ints(p.ctx))
    hold.fill_(7.0)
    graph.replay()
    check(p, q, hold, H, Hk, hd)
    assert (hold[0] == 7).all() and (hold[93:] == 7).all()
    assert ctx.get_error() == 0


def test_offsets_past_32_bits(ctx):
    """A pool and rows of more than 2^31 values: the last pages and rows are reached."""
    g = generator(10)
    H, Hk, hd, pages = 64, 64, 128, 4200                       # 4200 * 64 * 64 * 128 = 2.2e9 values
    k = torch.zeros(pages, Hk, PAGE, hd, dtype=BF16, device="cuda")
    v = torch.zeros_like(k)
    p = Pages(g, Hk, hd, [3, 65], [100, 70])
    p.table += pages - p.k.shape[0]
    k[-p.k.shape[0]:], v[-p.k.shape[0]:] = p.k, p.v
    p.table.masked_fill_(p.table < pages - p.k.shape[0], -1)
    ld, rows = 1 << 25, p.rows                                  # 68 rows of 2^25 values: 2^31.1
    q = torch.empty((rows - 1) * ld + H * hd, dtype=BF16, device="cuda").as_strided((rows, H * hd), (ld, 1))
    q.copy_(queries(g, rows, H, hd, BF16))
    out = torch.empty(rows, H * hd, dtype=BF16, device="cuda")
    ctx.op_chunk_attention(q, k, v, p.table, p.lens, p.starts, H, Hk, hd, out)
    p.k, p.v = k, v
    check(p, q.contiguous(), out, H, Hk, hd)
    run(ctx, p, q, H, Hk, hd, q)
    assert torch.equal(q.contiguous(), out)


def base(type=F32):
    g = generator(11)
    p = Pages(g, 2, 64, [2, 4], [70, 80])
    return dict(q=queries(g, p.rows, 4, 64, type), k_pages=p.k, v_pages=p.v, table=p.table, lens=p.lens, starts=p.starts, H=4, Hk=2, hd=64,
                out=torch.full((6, 256), 7.0, dtype=type, device="cuda"))


WRONG = {
    "q": [lambda t: t.half(), lambda t: t.bfloat16(), lambda t: t[:, :192], lambda t: t.t(), lambda t: t.cpu(), lambda t: t[0]],
    "out": [lambda t: t.bfloat16(), lambda t: t[:5], lambda t: t[:, :192], lambda t: t.cpu()],
    "k_pages": [lambda t: t.float(), lambda t: t[:, :1].contiguous(), lambda t: t[:4], lambda t: t[..., :32].contiguous(), lambda t: t.cpu()],
    "v_pages": [lambda t: t.float(), lambda t: t[:4], lambda t: t.transpose(0, 1)],
    "table": [lambda t: t.long(), lambda t: t.t(), lambda t: t.cpu(), lambda t: t[0]],
    "lens": [lambda t: t.long(), lambda t: t[:1], lambda t: t.cpu()],
    "starts": [lambda t: t.long(), lambda t: t[:2], lambda t: t.float()],
}


@pytest.mark.parametrize("name", WRONG)
def test_wrong_tensors_are_refused(ctx, name):
    for wrong in WRONG[name]:
        a = base()
        a[name] = wrong(a[name])
        with pytest.raises(ValueError):
            ctx.op_chunk_attention(**a)
    assert ctx.get_error() == 0


def test_wrong_sizes_are_refused(sd, ctx):
    for status, change in ((1, dict(H=3)), (1, dict(hd=32)), (1, dict(H=0)), (1, dict(Hk=0))):
        a = {**base(), **change}
        if "hd" in change or "Hk" in change:
            with pytest.raises((ValueError, sd.SdsatError)):
                ctx.op_chunk_attention(**a)
            continue
        with pytest.raises(sd.SdsatError) as e:
            ctx.op_chunk_attention(**a)
        assert e.value.status == status
    a = base()
    hold = torch.zeros(6, 257, device="cuda")
    for q, out in ((hold[:, 1:], a["out"]), (a["q"], hold[:, :256]), (hold.flatten()[1:1537].view(6, 256), a["out"])):
        with pytest.raises(sd.SdsatError) as e:
            ctx.op_chunk_attention(**{**a, "q": q, "out": out})
        assert e.value.status == 1
    many = torch.zeros(1, 129 * 64, device="cuda")
    pages = torch.zeros(1, 1, PAGE, 64, dtype=BF16, device="cuda")
    one = dict(k_pages=pages, v_pages=pages, table=ints([[0]]), lens=ints([0]), starts=ints([0, 1]), hd=64, Hk=1)
    with pytest.raises(sd.SdsatError) as e:
        ctx.op_chunk_attention(q=many, H=129, out=many.clone(), **one)
    assert e.value.status == 6
    few = torch.zeros(1, 64, device="cuda")
    with pytest.raises(sd.SdsatError) as e:
        ctx.op_chunk_attention(q=few, H=1, out=few.clone(), **{**one, "table": torch.zeros(1025, 1, dtype=torch.int32, device="cuda"),
                                                              "lens": torch.zeros(1025, dtype=torch.int32, device="cuda"),
                                                              "starts": torch.zeros(1026, dtype=torch.int32, device="cuda")})
    assert e.value.status == 6
    none = torch.zeros(0, 256, device="cuda")
    ctx.op_chunk_attention(**{**base(), "q": none, "out": none})   # no rows: nothing to do
    assert ctx.get_error() == 0


def test_rows_over_one_anothers_are_refused(sd, ctx):
    p = Pages(generator(31), 2, 64, [3], [5])
    hold = torch.ones(6, 256, device="cuda")
    with pytest.raises(sd.SdsatError) as e:
        run(ctx, p, hold[::2], 4, 2, 64, hold[:3])
    assert e.value.status == 1 and ctx.get_error() == 0
