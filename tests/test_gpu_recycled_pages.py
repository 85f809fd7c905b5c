"""Prompts and blocks on cache slots that hold NaN and infinities of earlier owners: the same bits as on a clean cache
(what no row sees adds 0 either way)."""
import math

import pytest
import torch

import synth

pytestmark = pytest.mark.gpu

PAGE = 64
SHAPES = {
    "64": synth.SHAPES["tiny"],
    # heads of 128, and enough of them for two tiles of 128 positions a CTA
    "128": synth.ModelShape("wide", 2, 256, 40, 128, 688, 4104, 4096),
}


@pytest.fixture(scope="module", params=["64", "128"])
def model(request):
    import paper_2403_18647_gb300 as sd
    shape = SHAPES[request.param]
    return shape, sd.Context(shape, synth.make_model(shape, seed=0, device="cuda", gain_std=0.1), max_position=2048)


def prompts(n, seed=0):
    return synth.prompt_ids(seed, 40, n, 4096).cuda()


def rows(ctx, shape, kv, seq, n):
    return torch.stack([x for layer in range(shape.n_layers) for x in ctx.kv_read(kv, layer, seq, 0, n)])


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("n", [1, 15, 17, 65, 127, 129, 200, 333, 1001])
def test_a_prompt_into_recycled_pages(model, n, value):
    """In two parts (the second after committed slots), then a block; pages of a pool that others left non-finite."""
    shape, ctx = model
    ids, toks = prompts(n + 30), prompts(6, 1)
    got = []
    for fill in (0.0, value):
        kv = ctx.kv_paged(2, n + 64, 2 * (n // PAGE + 3))
        kv.k.fill_(fill), kv.v.fill_(fill)
        lg = torch.empty(6, shape.vocab, device="cuda")
        for part in (ids[:n], ids[n:]):
            ctx.kv_reserve(kv, 1, part.numel())
            ctx.prefill(kv, 0, part)
        ctx.kv_reserve(kv, 1, 6)
        ctx.block_forward(kv, toks, lg, 1, 6)
        got.append((rows(ctx, shape, kv, 0, n + 36), lg))
        assert ctx.get_error() == 0
    assert torch.isfinite(got[1][1]).all()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("n", [17, 65, 200, 1001])
def test_a_prompt_into_slots_that_were_rolled_back(model, n, value):
    """The same on contiguous caches: a sequence begins anew where another answer became non-finite."""
    shape, ctx = model
    ids = prompts(n)
    got = []
    for fill in (0.0, value):
        kv = ctx.kv(2, n + 20)
        x = torch.full((shape.n_heads, n + 20, shape.head_dim), fill, dtype=torch.bfloat16, device="cuda")
        for layer in range(shape.n_layers):
            for seq in range(2):
                ctx.kv_write(kv, layer, seq, 0, x, x)
        ctx.prefill(kv, 0, ids)
        got.append(rows(ctx, shape, kv, 0, n))
        assert ctx.get_error() == 0
    assert torch.isfinite(got[1].float()).all()
    assert torch.equal(got[0], got[1])


# bf16 rows of the caches move by one place between a tiled GEMM's and a skinny one's sums
NEAR = 3e-2


@pytest.mark.parametrize("holes", [(0,), (1,), (0, 1), (2, 3), (0, 1, 2, 3), (3,), (1, 2)])
def test_slots_without_a_page_are_not_attended_to(model, holes):
    """Committed slots whose page is gone are reported and left out, by a prompt's positions as by a block's (the same
    positions in blocks of 13); the pool's other pages hold NaN."""
    import paper_2403_18647_gb300 as sd
    shape, ctx = model
    n, more = 310, 39
    ids, got = prompts(n + more), []
    for part in (more, 13):
        kv = ctx.kv_paged(1, 512, 12)
        kv.k.fill_(math.nan), kv.v.fill_(math.nan)
        ctx.kv_reserve(kv, 1, n + more)
        ctx.prefill(kv, 0, ids[:n])
        for j in holes:
            page = kv.table[0, j].item()
            kv.k[:, page], kv.v[:, page] = math.nan, math.nan
            kv.table[0, j] = -1
        assert ctx.get_error() == 0
        for at in range(n, n + more, part):
            ctx.prefill(kv, 0, ids[at:at + part])
        assert ctx.get_error() == sd.DEV_PAGE
        got.append(torch.stack([x for layer in range(shape.n_layers) for x in ctx.kv_read(kv, layer, 0, n, more)]))
        assert ctx.get_error() == 0
    assert torch.isfinite(got[0].float()).all()
    assert (got[0].float() - got[1].float()).abs().max().item() <= NEAR


def test_a_prompt_without_any_page(model):
    """No slot of the prompt has a page: its rows are reported, and every result is finite."""
    import paper_2403_18647_gb300 as sd
    shape, ctx = model
    kv = ctx.kv_paged(1, 512, 4)
    kv.k.fill_(math.nan), kv.v.fill_(math.nan)
    ctx.prefill(kv, 0, prompts(200))
    assert ctx.get_error() == sd.DEV_PAGE | sd.DEV_CAPACITY
    assert kv.k.isnan().all()
