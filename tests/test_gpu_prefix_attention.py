"""Block attention over pages that the sequences share, against 64 bits.

Tolerances.  fp32: products of bf16 keys and values with queries and probabilities in parts whose
remainder is below 2^-16 of them, fp32 sums, exps 2^-22 off; outputs are O(1): 2e-5 absolute, as for
the other attention kernels.  bf16: one rounding of the output, 2^-9 |ref|, beside that; 2^-8 |ref| + 1e-4.
"""
import math

import pytest
import torch

import synth

pytestmark = pytest.mark.gpu

PAGE = 64


@pytest.fixture(scope="module")
def sd():
    import paper_2403_18647_gb300 as sd
    return sd


@pytest.fixture(scope="module")
def ctx(sd):
    return sd.Context(synth.SHAPES["13b"], None, max_position=64)


class Case:
    """Sequences of `lens` committed slots whose first `shared` pages are the same, on pages in random order."""

    def __init__(self, seed, b, q, H, Hk, hd, lens, shared, type=torch.float32, scale=1.5):
        g = torch.Generator(device="cuda").manual_seed(seed)
        need = [-(-(n + q) // PAGE) for n in lens]
        assert all(n >= shared for n in need)
        pages = shared + sum(n - shared for n in need) + 3
        order = torch.randperm(pages, generator=g, device="cuda").int()
        table = torch.full((b, max(need)), -1, dtype=torch.int32, device="cuda")
        table[:, :shared] = order[:shared]
        at = shared
        for s, n in enumerate(need):
            table[s, shared:n] = order[at:at + n - shared]
            at += n - shared
        self.dims = (b, q, H, Hk, hd)
        self.x = (torch.randn(b * q, H * hd, generator=g, device="cuda") * scale).to(type)
        self.k = torch.randn(pages, Hk, PAGE, hd, generator=g, device="cuda").bfloat16()
        self.v = torch.randn(pages, Hk, PAGE, hd, generator=g, device="cuda").bfloat16()
        self.table, self.lens = table, list(lens)
        self.shared = torch.full((b,), shared, dtype=torch.int32, device="cuda")
        self.anc = None

    def spoil(self, value):
        """What no row may see: unused pages, and the slots past each sequence's block."""
        b, q = self.dims[:2]
        free = torch.ones(self.k.shape[0], dtype=torch.bool, device="cuda")
        free[self.table[self.table >= 0].long()] = False
        for t in (self.k, self.v):
            t[free] = value
            for s in range(b):
                end = self.lens[s] + q
                if end % PAGE:
                    t[self.table[s, end // PAGE].long(), :, end % PAGE:] = value
        return self

    def run(self, ctx, out=None, shared=True, x=None):
        b, q, H, Hk, hd = self.dims
        x = self.x if x is None else x
        out = torch.full((b * q, H * hd), math.nan, dtype=x.dtype, device="cuda") if out is None else out
        ctx.op_prefix_attention(x, self.k, self.v, self.table, self.shared if shared else None,
                                torch.tensor(self.lens, dtype=torch.int32, device="cuda"), b, q, H, Hk, hd, out, anc=self.anc)
        return out

    def reference(self):
        b, q, H, Hk, hd = self.dims
        out = torch.zeros(b, q, H, hd, dtype=torch.float64, device="cuda")
        x = self.x.double().view(b, q, H, hd)
        for s, n in enumerate(self.lens):
            at = self.table[s, :-(-(n + q) // PAGE)].long()
            bad = (at < 0) | (at >= self.k.shape[0])
            k = self.k[at.masked_fill(bad, 0)].transpose(0, 1).reshape(Hk, -1, hd)[:, :n + q].double()
            v = self.v[at.masked_fill(bad, 0)].transpose(0, 1).reshape(Hk, -1, hd)[:, :n + q].double()
            seen = torch.ones(q, n + q, dtype=torch.bool, device="cuda").tril(n)
            if self.anc is not None:
                bits = (self.anc.view(b, q)[s].long()[:, None] >> torch.arange(q, device="cuda")) & 1
                seen[:, n:] = bits.bool()
            seen &= ~bad.repeat_interleave(PAGE)[:n + q]
            for h in range(H):
                hk = h // (H // Hk)
                p = (x[s, :, h] @ k[hk].t() / math.sqrt(hd)).masked_fill(~seen, -math.inf)
                p = torch.nan_to_num(p.softmax(-1), nan=0.0) if not seen.any(-1).all() else p.softmax(-1)
                some = seen.any(0)
                out[s, :, h] = p[:, some] @ v[hk][some]
        return out.view(b * q, H * hd)

    def check(self, out):
        ref = self.reference()
        err = (out.double() - ref).abs()
        if out.dtype == torch.float32:
            assert err.max().item() <= 2e-5, err.max().item()
        else:
            assert (err - ref.abs() * 2 ** -8).max().item() <= 1e-4, err.max().item()


SIZES = [
    # b, q, H, Hk, hd, lens, shared pages
    (1, 1, 1, 1, 64, [0], 0), (1, 1, 2, 2, 128, [1], 0), (1, 16, 4, 4, 64, [63], 0), (2, 1, 4, 4, 64, [64, 64], 1),
    (2, 6, 4, 4, 64, [128, 191], 2), (3, 5, 4, 4, 128, [130, 190, 517], 2), (4, 16, 2, 2, 128, [300, 256, 319, 1000], 4),
    (8, 6, 32, 32, 128, [2048, 2049, 2111, 2112, 2175, 2200, 2060, 2300], 32), (16, 4, 8, 8, 64, [70 + 13 * i for i in range(16)], 1),
    (64, 1, 4, 4, 128, [640 + i for i in range(64)], 10), (64, 1, 8, 2, 64, [130] * 64, 2), (5, 3, 16, 2, 128, [64, 65, 66, 700, 127], 1),
    (7, 9, 16, 1, 64, [200, 210, 220, 230, 240, 250, 260], 3), (2, 16, 40, 40, 128, [4095, 4200], 63), (64, 1, 32, 4, 128, [900 + 7 * i for i in range(64)], 14),
    (3, 1, 64, 64, 64, [0, 5, 129], 0), (4, 16, 40, 40, 128, [0, 1, 2, 3], 0), (2, 1, 1, 1, 128, [9000, 8960], 140),
]


@pytest.mark.parametrize("b,q,H,Hk,hd,lens,shared", SIZES)
@pytest.mark.parametrize("type", [torch.float32, torch.bfloat16])
def test_sizes(ctx, b, q, H, Hk, hd, lens, shared, type):
    c = Case(b + q + H, b, q, H, Hk, hd, lens, shared, type)
    c.check(c.run(ctx))
    assert ctx.get_error() == 0


@pytest.mark.parametrize("b,q,H,Hk,hd,lens,shared", SIZES[4:9])
def test_sharing_changes_no_result(ctx, b, q, H, Hk, hd, lens, shared):
    """The same pages, said to be shared or not, or shared by fewer columns."""
    c = Case(3, b, q, H, Hk, hd, lens, shared)
    c.check(c.run(ctx, shared=False))
    c.shared[-1] = 1
    c.check(c.run(ctx))


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 3e38])
@pytest.mark.parametrize("hd", [64, 128])
def test_what_no_row_sees_does_not_matter(ctx, hd, value):
    """NaN and infinities in unwritten slots, in unused pages and past a page's end."""
    c = Case(5, 5, 3, 4, 4, hd, [128, 140, 190, 253, 61 + 128], 2).spoil(value)
    c.check(c.run(ctx))
    c = Case(6, 1, 1, 4, 4, hd, [0], 0).spoil(value)
    c.check(c.run(ctx))


@pytest.mark.parametrize("lens", [[200, 260, 383], [128, 128, 128], [126, 254, 382]])
def test_tree_masks_and_rows_that_see_nothing(ctx, lens):
    g = torch.Generator().manual_seed(7)
    c = Case(7, 3, 11, 4, 2, 128, lens, 1)
    anc = torch.randint(0, 1 << 11, (33,), generator=g, dtype=torch.int32)
    anc[::5] = 0                      # rows that see the committed slots alone
    c.anc = anc.cuda()
    c.check(c.run(ctx))
    c = Case(8, 3, 11, 4, 2, 64, [0, 0, 0], 0)   # nothing committed: those rows see nothing at all
    c.anc = anc.cuda()
    out = c.run(ctx)
    assert (out.view(33, -1)[::5] == 0).all()
    c.check(out)


def test_shared_pages_that_are_not_all_committed(ctx):
    """A sequence whose committed slots end inside the shared pages: the rest of them are read as its own."""
    c = Case(9, 3, 4, 4, 4, 128, [512, 600, 640], 8)
    c.lens[1] = 300
    c.check(c.run(ctx))
    c.lens[0] = 0
    c.check(c.run(ctx))


def test_large_scores_and_one_key_that_wins(ctx):
    """Scores up to 50, growing along the sequence, so that every running maximum moves (a score is off
    by a few 2^-24 of itself, a probability relatively by as much: 1e-5)."""
    c = Case(10, 4, 6, 4, 4, 128, [1000, 1024, 1100, 1500], 15, scale=0.0)
    c.x += torch.linspace(-6, 6, 128, device="cuda").repeat(4)
    ramp = torch.zeros(c.k.shape[0], device="cuda")
    for s in range(4):
        for j, page in enumerate(c.table[s].tolist()):
            if page >= 0:
                ramp[page] = j
    c.k = (c.k.float() * 0.2 + ramp[:, None, None, None] * torch.linspace(-0.1, 0.1, 128, device="cuda")).bfloat16()
    c.check(c.run(ctx))
    c.x.neg_()
    c.check(c.run(ctx))


@pytest.mark.parametrize("b,q,H,Hk,hd,lens,shared", [
    (1, 1, 40, 40, 128, [9000], 0), (2, 16, 40, 40, 128, [9001, 8950], 139), (1, 3, 64, 64, 64, [12345], 0), (2, 4, 40, 40, 64, [7000, 6990], 0),
])
@pytest.mark.parametrize("type", [torch.float32, torch.bfloat16])
def test_long_shares(ctx, b, q, H, Hk, hd, lens, shared, type):
    """More than 16 units of 128 slots for every SM, so that sums are added up in several runs."""
    c = Case(16, b, q, H, Hk, hd, lens, shared, type)
    c.check(c.run(ctx))
    assert ctx.get_error() == 0


def test_maxima_that_move_from_run_to_run(ctx):
    """Scores that grow along 9000 slots by 30 and more (a probability is off by some 2^-24 of its exponent)."""
    c = Case(17, 1, 4, 40, 40, 128, [9000], 0, scale=0.0)
    c.x += torch.linspace(-1, 1, 128, device="cuda").repeat(40)
    at = torch.zeros(c.k.shape[0], device="cuda")
    at[c.table[0].long()] = torch.arange(c.table.shape[1], device="cuda", dtype=torch.float32)
    c.k = (c.k.float() * 0.2 + at[:, None, None, None] * torch.linspace(-0.06, 0.06, 128, device="cuda")).bfloat16()
    for _ in range(2):
        c.check(c.run(ctx))
        c.x.neg_()


def test_strides_and_other_streams(ctx):
    """q as a slice of a wider row, out into one; on a stream of its own."""
    c = Case(11, 3, 5, 4, 4, 64, [100, 130, 150], 1)
    wide = torch.full((15, 3 * 256), math.nan, device="cuda")
    wide[:, 256:512] = c.x
    out = torch.full((15, 1024), 7.0, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        q = wide * 1.0
        c.run(ctx, out=out[:, 512:768], x=q[:, 256:512])
    side.synchronize()
    c.check(out[:, 512:768])
    assert (out[:, :512] == 7).all() and (out[:, 768:] == 7).all()


def test_the_last_pages_of_a_large_pool(ctx):
    """Rows whose byte offsets pass 2^31 (K of 4.3 GB)."""
    b, q, H, hd, pages = 2, 3, 32, 128, 8192
    c = Case(12, b, q, H, H, hd, [150, 180], 1)
    k = torch.zeros(pages, H, PAGE, hd, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    n = c.k.shape[0]
    k[-n:], v[-n:] = c.k, c.v
    c.k, c.v = k, v
    c.table = torch.where(c.table >= 0, c.table + (pages - n), c.table)
    c.check(c.run(ctx))


def test_pages_outside_the_pool_are_reported_and_skipped(sd, ctx):
    c = Case(13, 3, 2, 4, 4, 128, [130, 200, 250], 1)
    c.table[1, 2] = -1
    c.table[2, 1] = c.k.shape[0]
    c.check(c.run(ctx))
    assert ctx.get_error() == sd.DEV_PAGE
    c.table[:, 0] = -5                # a shared page
    c.check(c.run(ctx))
    assert ctx.get_error() == sd.DEV_PAGE


def test_calls_repeat_their_bits_and_replay_from_a_graph(ctx):
    c = Case(14, 8, 6, 32, 32, 128, [1024 + 20 * i for i in range(8)], 16)
    a, z = c.run(ctx).clone(), c.run(ctx).clone()
    assert torch.equal(a, z)
    lens, out = torch.tensor(c.lens, dtype=torch.int32, device="cuda"), torch.zeros_like(a)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.op_prefix_attention(c.x, c.k, c.v, c.table, c.shared, lens, 8, 6, 32, 32, 128, out)
    for _ in range(3):
        out.zero_()
        g.replay()
        assert torch.equal(out, a)


def test_refusals(sd, ctx):
    c = Case(15, 2, 4, 4, 4, 64, [100, 120], 1)
    lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    out = torch.empty_like(c.x)

    def call(b=2, q=4, H=4, Hk=4, hd=64, x=c.x, o=out):
        ctx.op_prefix_attention(x, c.k, c.v, c.table, c.shared, lens, b, q, H, Hk, hd, o)

    for kw in (dict(b=0), dict(q=0), dict(hd=32), dict(hd=96), dict(H=0), dict(Hk=0), dict(H=3, Hk=2), dict(Hk=3)):
        with pytest.raises(sd.SdsatError) as e:
            call(**kw)
        assert e.value.status == 1, kw
    lib = sd.lib()
    args = lambda **k: [ctx.handle, k.get("q", c.x.data_ptr()), k.get("q_ld", 256), c.k.data_ptr(), c.v.data_ptr(), k.get("pages", 5),  # noqa: E731
                        c.table.data_ptr(), k.get("ld", 2), None, lens.data_ptr(), None, k.get("b", 2), k.get("n", 4), 4, 4, 64,
                        out.data_ptr(), k.get("out_ld", 256), k.get("type", 0)]
    for kw in (dict(q=None), dict(q=c.x.data_ptr() + 4), dict(q_ld=255), dict(q_ld=258), dict(out_ld=252), dict(pages=0),
               dict(ld=0), dict(b=65, n=1), dict(b=5, n=16), dict(n=17), dict(type=2), dict(type=1, q_ld=260)):
        assert lib.sdsat_op_prefix_attention(*args(**kw)) == 1, kw
    with pytest.raises(ValueError):
        call(o=out.bfloat16())
    with pytest.raises(ValueError):
        call(x=c.x[:3])
    assert ctx.get_error() == 0
