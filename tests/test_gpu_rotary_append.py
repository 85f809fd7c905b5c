"""Head norms, rotation and append of a ragged batch's rows, against 64 bits.

Tolerances.  A rotated value is a c + z s with a and z normed.  fp32 roundings of 2^-24: one of the cosine or sine, one of
the product, one of the sum, times |a c| + |z s|: 4 * 2^-24 (|a| + |z|) at magnitude 1.  A norm: squares and their sum 10 of
them, halved by the root; rsqrt 2 ulp (4 of them), mean and eps 1, two products 2: 12 in all.  2^-20 (|a| + |z|) holds
both.  bf16 results are rounded once beside that: 2^-8 |ref|."""
import math

import pytest
import torch

import synth
from ragged import PAGE, Pages, generator, ints

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def sd():
    import paper_2403_18647_gb300 as sd
    return sd


@pytest.fixture(scope="module")
def ctx(sd):
    return sd.Context(synth.SHAPES["tiny"], None, max_position=64)


def frequencies(dims, theta=1e4, scaling=None, factor=1.0, low=1.0, high=32.0, original=0, magnitude=1.0):
    f = []
    for i in range(dims // 2):
        w = theta ** (-2 * i / dims)
        keep = 1.0 if scaling is None else 0.0
        if scaling == "parts":
            keep = min(1.0, max(0.0, (original * w / (2 * math.pi) - low) / (high - low)))
        f.append(w * (keep + (1 - keep) / factor))
    return torch.tensor(f, dtype=torch.float64, device="cuda")


def turned(x, gain, eps, position, dims, interleaved, f, magnitude):
    """x (rows, heads, hd) in 64 bits -> the rotated rows and |a| + |z| of each place."""
    x = x.double()
    if gain is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * gain.double()
    angle = position.double()[:, None] * f
    c, s = angle.cos()[:, None] * magnitude, angle.sin()[:, None] * magnitude
    i = torch.arange(dims // 2, device="cuda")
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + dims // 2)
    y, size = x.clone(), x.abs()
    a, z = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - z * s, a * s + z * c
    size[..., first] = size[..., second] = (a.abs() + z.abs()) * magnitude
    return y, size


class Batch:
    def __init__(self, seed, H, Hk, hd, new, held, type, norm=True, before=0, behind=0):
        g = generator(seed)
        self.p = p = Pages(g, Hk, hd, new, held, before=before)
        self.dims = H, Hk, hd
        rows = p.rows + behind
        x = (torch.randn(rows, (H + 2 * Hk) * hd + 8, generator=g, device="cuda") * 2).to(type)
        self.q, self.k, self.v = x[:, :H * hd], x[:, H * hd:(H + Hk) * hd], x[:, (H + Hk) * hd:(H + 2 * Hk) * hd]
        self.gains = [(1 + 0.3 * torch.randn(hd, generator=g, device="cuda")).bfloat16() if norm else None for _ in range(2)]
        self.out = torch.full((rows, H * hd), 7.0, dtype=type, device="cuda")
        self.positions = None

    def run(self, ctx, rope, eps=1e-5, refs=None):
        H, Hk, hd = self.dims
        p = self.p
        ctx.op_rotary_append(rope, self.q, self.k, self.v, self.out, p.k, p.v, p.table, p.lens, p.starts, H, Hk, hd,
                             positions=self.positions, q_gain=self.gains[0], k_gain=self.gains[1], eps=eps, refs=refs)

    def check(self, ctx, rope, dims, interleaved, eps=1e-5, **scaling):
        H, Hk, hd = self.dims
        p = self.p
        was = p.k.clone(), p.v.clone()
        self.run(ctx, rope, eps)
        f, magnitude = frequencies(dims, **scaling), scaling.get("magnitude", 1.0)
        k, v = was
        near = torch.zeros(k.shape, dtype=torch.float64, device="cuda")
        k = k.double()
        mine = torch.zeros(self.out.shape[0], dtype=torch.bool, device="cuda")
        for s, n in enumerate(p.new):
            r = slice(p.first[s], p.first[s] + n)
            mine[r] = True
            pos = torch.arange(p.ctx[s], p.ctx[s] + n, device="cuda") if self.positions is None else self.positions[r].long()
            ref, size = turned(self.q[r].reshape(n, H, hd), self.gains[0], eps, pos, dims, interleaved, f, magnitude)
            slack = 2 ** -20 * size + (2 ** -8 * ref.abs() if self.out.dtype == BF16 else 0)
            assert ((self.out[r].double().view(n, H, hd) - ref).abs() <= slack).all()
            page, place = p.slots(s)
            ref, size = turned(self.k[r].reshape(n, Hk, hd), self.gains[1], eps, pos, dims, interleaved, f, magnitude)
            k[page, :, place] = ref
            near[page, :, place] = 2 ** -20 * size + 2 ** -8 * ref.abs()
            v[page, :, place] = self.v[r].reshape(n, Hk, hd).bfloat16()
        assert ((p.k.double() - k).abs() <= near).all()                 # (all other slots as they were)
        assert torch.equal(p.v, v)
        assert (self.out[~mine] == 7).all()
        assert ctx.get_error() == 0


SIZES = [(1, 1, 64, [1], [0]), (1, 1, 128, [3], [63]), (4, 4, 64, [6, 1], [70, 0]), (32, 8, 128, [1] * 40, list(range(40, 80))),
         (14, 2, 64, [5, 200, 1], [64, 0, 999]), (5, 5, 128, [130], [1]), (3, 1, 64, [0, 7, 0, 9], [5, 0, 64, 100]), (40, 40, 128, [33], [20000])]


@pytest.mark.parametrize("H,Hk,hd,new,held", SIZES)
@pytest.mark.parametrize("type", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_sizes(ctx, H, Hk, hd, new, held, type, interleaved):
    for norm in (False, True):
        b = Batch(H + hd, H, Hk, hd, new, held, type, norm, before=2, behind=3)
        b.check(ctx, ctx.rope(hd, 32768, interleaved=interleaved), hd, interleaved)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_parts_of_a_head(ctx, hd, interleaved):
    """Every even number of rotated dimensions, whatever lane and place a pair's second value has."""
    b = Batch(3, 3, 3, hd, [9, 2], [60, 5], F32)
    for dims in range(2, hd + 1, 2):
        b.out.fill_(7.0)
        b.check(ctx, ctx.rope(dims, 4096, interleaved=interleaved), dims, interleaved)


SCALING = [dict(scaling="linear", factor=4.0), dict(scaling="parts", factor=8.0, low=1.0, high=4.0, original=8192),
           dict(scaling="parts", factor=16.0, low=1.0, high=32.0, original=2048, magnitude=1.277), dict(theta=5e5), dict(theta=1e6, magnitude=0.5)]


@pytest.mark.parametrize("scaling", SCALING)
def test_scaled_frequencies_at_far_positions(ctx, scaling):
    b = Batch(4, 4, 2, 128, [70, 1], [20000, 131000], BF16)
    b.check(ctx, ctx.rope(128, 131072, **scaling), 128, False, **scaling)


def test_norms_of_queries_or_keys_alone_and_small_rows(ctx):
    rope = ctx.rope(64, 4096)
    for which in (0, 1):
        b = Batch(5, 4, 2, 64, [12], [3], F32)
        b.gains[which] = None
        b.q[3] = 0
        b.k[4] = 0
        b.q[5] *= 1e-4
        b.check(ctx, rope, 64, False, eps=1e-6)


def test_positions(sd, ctx):
    b = Batch(6, 4, 2, 64, [12, 4], [3, 90], F32)
    b.positions = ints([5, 5, 5, 0, 4095] + list(range(11)))
    rope = ctx.rope(64, 4096)
    b.check(ctx, rope, 64, False)
    far = b.positions.clone()
    far[0], far[1], far[4] = -1, 2 ** 31 - 1, 4096
    kept = b.positions.clone()
    kept[0], kept[1], kept[4] = 0, 4095, 4095
    b.positions = kept
    b.run(ctx, rope)
    out, k = b.out.clone(), b.p.k.clone()
    b.positions = far
    b.run(ctx, rope)
    assert ctx.get_error() == sd.DEV_POSITION
    assert torch.equal(b.out, out) and torch.equal(b.p.k, k)


@pytest.mark.parametrize("type", [F32, BF16])
def test_the_queries_may_be_replaced(ctx, type):
    rope = ctx.rope(128, 4096)
    b = Batch(7, 8, 2, 128, [30, 1], [100, 7], type)
    b.run(ctx, rope)
    out = b.out.clone()
    b.out = b.q
    b.run(ctx, rope)
    assert torch.equal(b.q, out)


def test_rows_that_are_not_written(sd, ctx):
    """Without a page, past the table, on another sequence's page: CAPACITY, and nothing of the cache changes."""
    rope = ctx.rope(64, 4096)
    b = Batch(8, 4, 2, 64, [10, 3, 4, 2], [60, 0, 128, 64], F32)
    p = b.p
    refs = torch.ones(p.k.shape[0], dtype=torch.int32, device="cuda")
    want = Batch(8, 4, 2, 64, [10, 3, 4, 2], [60, 0, 128, 64], F32)
    want.run(ctx, rope, refs=refs)
    assert ctx.get_error() == 0
    refs[p.table[1, 0].long()] = 2
    page = p.table[2, 2].item()
    p.table[2, 2] = p.k.shape[0]
    p.table[0, 1] = -1
    k, v = p.k.clone(), p.v.clone()
    b.run(ctx, rope, refs=refs)
    assert ctx.get_error() == sd.DEV_CAPACITY
    assert torch.equal(b.out, want.out)
    at, place = p.table[0, 0].long(), slice(60, 64)                     # the first four rows of sequence 0, and sequence 3
    k[at, :, place], v[at, :, place] = want.p.k[at, :, place], want.p.v[at, :, place]
    at = p.table[3, 1].long()
    k[at, :, :2], v[at, :, :2] = want.p.k[at, :, :2], want.p.v[at, :, :2]
    assert torch.equal(p.k, k) and torch.equal(p.v, v) and page >= 0
    # lengths past the table, and negative ones
    p.lens = ints([2 ** 31 - 1, -5, 64 * p.table.shape[1], -2 ** 31])
    k, v = p.k.clone(), p.v.clone()
    b.run(ctx, rope)
    assert ctx.get_error() & sd.DEV_CAPACITY
    assert torch.equal(p.k, k) and torch.equal(p.v, v)


def test_starts_that_do_not_ascend_reach_no_other_memory(sd, ctx):
    rope = ctx.rope(64, 4096)
    for b_ in (4, 40):
        b = Batch(9, 4, 2, 64, [3] * b_, [5] * b_, F32)
        for starts in (list(range(3 * b_, -1, -3)), [-2 ** 31] * (b_ + 1), [2 ** 31 - 1] * (b_ + 1), [0] + [2 ** 31 - 1, -2 ** 31] * (b_ // 2)):
            b.p.starts = ints(starts)
            k, v = b.p.k.clone(), b.p.v.clone()
            b.run(ctx, rope)
            torch.cuda.synchronize()
            ctx.get_error()
            free = torch.ones(k.shape[0], dtype=torch.bool, device="cuda")
            free[b.p.table[b.p.table >= 0].long()] = False
            assert torch.equal(b.p.k[free], k[free]) and torch.equal(b.p.v[free], v[free])


@pytest.mark.parametrize("b_", [31, 32, 33, 1000, 5000])
def test_many_sequences(ctx, b_):
    """The search for a row's sequence, sequences without rows among them."""
    b = Batch(10, 1, 1, 64, [(5 * s) % 3 for s in range(b_)], [s % 70 for s in range(b_)], F32, norm=False)
    b.check(ctx, ctx.rope(64, 4096), 64, False)


def test_streams_and_graphs(ctx):
    rope = ctx.rope(128, 4096)
    b = Batch(11, 8, 2, 128, [30, 1], [100, 7], BF16)
    k, v = b.p.k.clone(), b.p.v.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.run(ctx, rope)
    torch.cuda.current_stream().wait_stream(side)
    out, ko, vo = b.out.clone(), b.p.k.clone(), b.p.v.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run(ctx, rope)
    for t, w in ((b.p.k, k), (b.p.v, v)):
        t.copy_(w)
    b.out.zero_()
    graph.replay()
    assert torch.equal(b.out, out) and torch.equal(b.p.k, ko) and torch.equal(b.p.v, vo)
    b.p.lens.copy_(ints([90, 20]))
    b.p.ctx = [90, 20]
    graph.replay()
    hold = b.out.clone()
    b.check(ctx, rope, 128, False)
    assert torch.equal(hold, b.out)


def test_a_rotation_outlives_its_context(sd):
    other = sd.Context(synth.SHAPES["tiny"], None, max_position=64)
    rope = other.rope(64, 128)
    other.close()
    rope.close()


WRONG_ROPE = [dict(dims=0), dict(dims=3), dict(dims=130), dict(max_position=0), dict(max_position=(1 << 24) + 1), dict(theta=0.0), dict(theta=math.nan),
              dict(theta=math.inf), dict(magnitude=0.0), dict(magnitude=-1.0), dict(scaling="linear", factor=0.0),
              dict(scaling="parts", factor=2.0), dict(scaling="parts", factor=2.0, original=64, low=3.0, high=3.0),
              dict(scaling="parts", factor=math.inf, original=64)]


@pytest.mark.parametrize("wrong", WRONG_ROPE)
def test_wrong_rotations_are_refused(sd, ctx, wrong):
    with pytest.raises(sd.SdsatError) as e:
        ctx.rope(**{**dict(dims=64, max_position=128), **wrong})
    assert e.value.status == 1
    with pytest.raises(ValueError):
        ctx.rope(64, 128, scaling="other")


WRONG = {
    "q": [lambda t: t.half(), lambda t: t.bfloat16(), lambda t: t[:, :192], lambda t: t.cpu()],
    "k": [lambda t: t.bfloat16(), lambda t: t[:5], lambda t: t[:, :64], lambda t: t.t()],
    "v": [lambda t: t.bfloat16(), lambda t: t[:5], lambda t: t[:, :64]],
    "q_out": [lambda t: t.bfloat16(), lambda t: t[:5], lambda t: t[:, :192]],
    "k_pages": [lambda t: t.float(), lambda t: t[:1], lambda t: t[:, :1].contiguous()],
    "v_pages": [lambda t: t.float(), lambda t: t[..., :32].contiguous()],
    "table": [lambda t: t.long(), lambda t: t[0], lambda t: t.t()],
    "lens": [lambda t: t.long(), lambda t: t[:1]], "starts": [lambda t: t.long(), lambda t: t[:2]],
    "positions": [lambda t: t.long(), lambda t: t[:5]], "refs": [lambda t: t.long(), lambda t: t[:2]],
    "q_gain": [lambda t: t.float(), lambda t: t[:63]], "k_gain": [lambda t: t.float(), lambda t: t[:63]],
}


@pytest.mark.parametrize("name", WRONG)
def test_wrong_tensors_are_refused(ctx, name):
    b = Batch(12, 4, 2, 64, [2, 4], [70, 80], F32)
    p = b.p
    whole = dict(q=b.q, k=b.k, v=b.v, q_out=b.out, k_pages=p.k, v_pages=p.v, table=p.table, lens=p.lens, starts=p.starts,
                 positions=ints([0] * 6), q_gain=b.gains[0], k_gain=b.gains[1], refs=torch.ones(p.k.shape[0], dtype=torch.int32, device="cuda"))
    rope = ctx.rope(64, 128)
    for wrong in WRONG[name]:
        with pytest.raises(ValueError):
            ctx.op_rotary_append(rope, H=4, Hk=2, hd=64, **{**whole, name: wrong(whole[name])})
    ctx.op_rotary_append(rope, H=4, Hk=2, hd=64, **whole)
    assert ctx.get_error() == 0


def test_wrong_sizes_are_refused(sd, ctx):
    b = Batch(13, 4, 2, 64, [2, 4], [70, 80], F32)
    rope = ctx.rope(64, 128)

    def refused(status=1, rope=rope, eps=1e-5, **change):
        a = dict(q=b.q, k=b.k, v=b.v, q_out=b.out, k_pages=b.p.k, v_pages=b.p.v, table=b.p.table, lens=b.p.lens, starts=b.p.starts, H=4, Hk=2, hd=64)
        with pytest.raises(sd.SdsatError) as e:
            ctx.op_rotary_append(rope, **{**a, **change}, eps=eps)
        assert e.value.status == status

    refused(rope=ctx.rope(66, 128))                     # more dimensions than a head has
    refused(rope=sd.Context(synth.SHAPES["tiny"], None, max_position=64).rope(64, 128))
    refused(eps=-1.0)
    refused(eps=math.nan)
    refused(H=3)
    hold = torch.zeros(6, 257, device="cuda")
    refused(q=hold[:, 1:])
    refused(q_out=hold[:, :256])
    refused(k=hold[:, :128])
    none = b.q[:0]
    ctx.op_rotary_append(rope, none, b.k[:0], b.v[:0], b.out[:0], b.p.k, b.p.v, b.p.table, b.p.lens, b.p.starts, 4, 2, 64)
    assert ctx.get_error() == 0


def test_offsets_past_32_bits(ctx):
    """A pool and rows of more than 2^31 values: the last pages and rows are reached."""
    H, Hk, hd, pages = 64, 64, 128, 4200
    b = Batch(14, H, Hk, hd, [3, 65], [100, 70], BF16)
    p = b.p
    small = p.k.shape[0]
    want = Batch(14, H, Hk, hd, [3, 65], [100, 70], BF16)
    rope = ctx.rope(hd, 4096)
    want.run(ctx, rope)
    k = torch.zeros(pages, Hk, PAGE, hd, dtype=BF16, device="cuda")
    v = torch.zeros_like(k)
    k[-small:], v[-small:] = p.k, p.v
    p.k, p.v = k, v
    p.table = torch.where(p.table >= 0, p.table + (pages - small), -1)
    ld = 1 << 25
    q = torch.empty((p.rows - 1) * ld + H * hd, dtype=BF16, device="cuda").as_strided((p.rows, H * hd), (ld, 1))
    q.copy_(b.q)
    b.q = b.out = q
    b.run(ctx, rope)
    assert torch.equal(b.out.contiguous(), want.out)
    assert torch.equal(k[-small:], want.p.k) and torch.equal(v[-small:], want.p.v)
    assert ctx.get_error() == 0


def test_rows_over_one_anothers_are_refused(sd, ctx):
    b = Batch(15, 4, 2, 64, [2, 4], [70, 80], F32)
    hold = torch.ones(12, 256, device="cuda")
    with pytest.raises(sd.SdsatError) as e:
        ctx.op_rotary_append(ctx.rope(64, 128), hold[::2], b.k, b.v, hold[:6], b.p.k, b.p.v, b.p.table, b.p.lens, b.p.starts, 4, 2, 64)
    assert e.value.status == 1 and (hold == 1).all() and ctx.get_error() == 0
