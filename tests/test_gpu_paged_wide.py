"""Paged caches of heads of 128 dimensions (16 KB blocks, two boxes of a page and head) and pools whose offsets pass 2^31
values: copies are exact; the decode step against contiguous caches."""
import pytest
import torch

import synth

pytestmark = pytest.mark.gpu

PAGE = 64
SHAPE = synth.ModelShape("wide", 2, 256, 40, 128, 688, 4104, 4096)
NEAR = 3e-2   # bf16 rows of the caches move by one place between a tiled GEMM's and a skinny one's sums


@pytest.fixture(scope="module")
def ctx():
    import paper_2403_18647_gb300 as sd
    return sd.Context(SHAPE, synth.make_model(SHAPE, seed=0, device="cuda", gain_std=0.1), max_position=2048)


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def prompts(n, seed=0):
    return synth.prompt_ids(seed, 40, n, 4096).cuda()


def pair(ctx, b, n, pages):
    """A contiguous and a paged cache of b sequences after the same prompt of n tokens, shared by the paged ones."""
    flat, kv = ctx.kv(b, n + 200), ctx.kv_paged(b + 1, n + 200, pages)
    ctx.kv_reserve(kv, 1, n, seq=b)
    ctx.prefill(kv, b, prompts(n))
    ctx.kv_fork(kv, i32([b] * b))
    for s in range(b):
        ctx.prefill(flat, s, prompts(n))
    return flat, kv


@pytest.mark.parametrize("b,q,n", [(1, 6, 333), (2, 6, 127), (4, 16, 700), (8, 6, 150), (64, 1, 200), (5, 12, 64)])
def test_blocks_after_a_shared_prompt(ctx, b, q, n):
    flat, kv = pair(ctx, b, n, -(-n // PAGE) + 5 * b)
    lg = [torch.empty(b * q, SHAPE.vocab, device="cuda") for _ in range(2)]
    acc, out = i32([0] * b), i32([0] * b * q)
    for step in range(3):
        toks = prompts(b * q, 5 + step)
        ctx.kv_reserve(kv, b, q)
        for i, c in enumerate((flat, kv)):
            ctx.block_forward(c, toks, lg[i], b, q)
        assert (lg[0] - lg[1]).abs().max().item() <= NEAR
        ctx.accept_greedy(flat, lg[0], toks, b, q, 0, acc, out)
        ctx.kv_commit(kv, ctx.kv_lengths(flat), b)
    for layer in range(2):
        for s in (0, b - 1):
            m = kv.lens[s].item()
            for a, z in zip(ctx.kv_read(flat, layer, s, 0, m), ctx.kv_read(kv, layer, s, 0, m)):
                assert (a.float() - z.float()).abs().max().item() <= NEAR
    assert ctx.get_error() == 0


def test_a_tree_block(ctx):
    b, q, n = 3, 7, 125
    flat, kv = pair(ctx, b, n, 20)
    parent, toks = i32([-1, 0, 0, 1, 2, 4, 4] * b), prompts(b * q, 3)
    lg = torch.empty(b * q, SHAPE.vocab, device="cuda")
    ctx.kv_reserve(kv, b, q)
    ctx.block_forward_tree(flat, toks, parent, lg, b, q)
    best, t = lg.argmax(-1).view(b, q), toks.view(b, q).clone()
    for j, p in ((2, 0), (4, 2), (6, 4)):
        t[:, j] = best[:, p]
    got = []
    for c in (flat, kv):
        ctx.block_forward_tree(c, t, parent, lg, b, q)
        acc, out, path = i32([0] * b), i32([0] * b * q), i32([0] * b * q)
        ctx.accept_tree(c, lg, t, parent, b, q, acc, out, path)
        got.append((acc.tolist(), path.tolist(), ctx.kv_lengths(c).tolist()[:b], lg.clone()))
    assert got[0][:3] == got[1][:3] and (got[0][3] - got[1][3]).abs().max().item() <= NEAR
    for s in range(b):
        m = got[0][2][s]
        for a, z in zip(ctx.kv_read(flat, 1, s, 0, m), ctx.kv_read(kv, 1, s, 0, m)):
            assert (a.float() - z.float()).abs().max().item() <= NEAR
    assert ctx.get_error() == 0


@pytest.mark.parametrize("pages", [40, 3400])
def test_copies_are_exact(ctx, pages):
    """Fork, reserve and compact at both ends of a pool; of 3400 pages K alone has 2.2e9 values."""
    kv = ctx.kv_paged(5, 512, pages)
    kv.k.normal_(), kv.v.normal_()
    last = [pages - 1, pages - 7, pages - 2]
    kv.table[0, :3], kv.refs[last], kv.lens[0] = i32(last), 1, 150
    taken = list(range(3, pages - 12))           # nothing is free but 0, 1, 2 and the last twelve
    kv.refs[taken] = 1
    before = {p: (kv.k[:, p].clone(), kv.v[:, p].clone()) for p in last}
    ctx.kv_fork(kv, i32([0, 0, 0, 0, 0]))
    ctx.kv_reserve(kv, 5, 6)                     # copies to 0, 1, 2 and into the end of the pool
    assert ctx.get_error() == 0
    want = [[last[0], last[1], p] for p in (0, 1, 2, pages - 12, last[2])]
    assert kv.table[:, :3].tolist() == want
    for p in (0, 1, 2, pages - 12):
        for pool, src in zip((kv.k, kv.v), before[last[2]]):
            assert torch.equal(pool[:, p, :, :22], src[:, :, :22])
    ctx.kv_free(kv, 0)
    ctx.kv_free(kv, 1)                           # two holes, 0 and 1
    ends = sorted(set(last + [pages - 12]))
    ctx.kv_compact(kv)
    assert ctx.get_error() == 0
    used = 1 + len(taken) + len(ends)
    moved = [p for p in ends if p >= used]
    holes = [p for p in range(used) if p in (0, 1) or (p >= pages - 12 and p not in ends)]
    to = dict(zip(moved, holes))
    assert len(moved) == len(holes) and kv.table[2:, :3].tolist() == [[to.get(p, p) for p in row] for row in want[2:]]
    for p in (last[0], last[1]):
        for pool, src in zip((kv.k, kv.v), before[p]):
            assert torch.equal(pool[:, to.get(p, p)], src)
    for p in (pages - 12, last[2]):
        for pool, src in zip((kv.k, kv.v), before[last[2]]):
            assert torch.equal(pool[:, to.get(p, p), :, :22], src[:, :, :22])
    rows = ctx.kv_read(kv, 1, 4, 0, 150)
    for row, src in zip(rows, range(2)):
        whole = torch.cat([before[p][src][1] for p in last], 1)[:, :150]
        assert torch.equal(row, whole)


def test_blocks_at_the_end_of_a_large_pool(ctx):
    """The same block on the first and on the last pages of 3400."""
    kv = ctx.kv_paged(1, 512, 3400)
    got = []
    for taken in (0, 3390):
        kv.refs[:taken] = 1
        ctx.kv_reserve(kv, 1, 300)
        assert kv.table[0, 0].item() == taken
        ctx.prefill(kv, 0, prompts(280))
        lg = torch.empty(6, SHAPE.vocab, device="cuda")
        ctx.block_forward(kv, prompts(6, 1), lg, 1, 6)
        got.append((lg, *ctx.kv_read(kv, 1, 0, 0, 286)))
        ctx.kv_free(kv, 0)
    assert all(torch.equal(a, z) for a, z in zip(*got))
    assert ctx.get_error() == 0
