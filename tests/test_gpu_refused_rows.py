"""Rows that a paged cache refuses (no page, or one that other sequences hold too) are not committed."""
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
def model(sd):
    shape = synth.SHAPES["tiny"]
    return shape, sd.Context(shape, synth.make_model(shape, seed=0, device="cuda", gain_std=0.1), max_position=8192)


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def prompts(n, seed=0):
    return synth.prompt_ids(seed, 40, n, 4096).cuda()


@pytest.mark.parametrize("committed", [0, 30])
@pytest.mark.parametrize("pages,n", [(0, 1), (0, 16), (0, 200), (1, 70), (2, 600), (35, 2400), (33, 4200), (65, 4200), (70, 4200)])
def test_a_prompt_with_too_few_pages(sd, model, committed, pages, n):
    """One block's, one chunk's and two chunks' rows (the second of 4200 alone would find 33 pages enough): the length
    stays, and the prompt goes in when there are pages."""
    shape, ctx = model
    kv = ctx.kv_paged(2, 6000, 100)
    ids = prompts(committed + n)
    if committed:
        ctx.kv_reserve(kv, 1, committed, seq=1)
        ctx.prefill(kv, 1, ids[:committed])
    if pages:
        ctx.kv_reserve(kv, 1, pages * PAGE - committed, seq=1)
    have = max(pages, -(-committed // PAGE)) * PAGE
    short = committed + n > have
    assert ctx.get_error() == 0
    ctx.prefill(kv, 1, ids[committed:])
    assert ctx.get_error() & ~sd.DEV_PAGE == (sd.DEV_CAPACITY if short else 0)
    assert kv.lens.tolist() == [0, committed if short else committed + n]
    if short:
        ctx.kv_reserve(kv, 1, n, seq=1)
        ctx.prefill(kv, 1, ids[committed:])
        assert ctx.get_error() == 0
        assert kv.lens.tolist() == [0, committed + n]


def test_a_prompt_into_shared_pages(sd, model):
    shape, ctx = model
    kv = ctx.kv_paged(2, 300, 12)
    ctx.kv_reserve(kv, 1, 200)
    ctx.prefill(kv, 0, prompts(100))
    ctx.kv_fork(kv, i32([0, 0]))
    before = kv.k.clone()
    ctx.prefill(kv, 1, prompts(40, 1))
    assert ctx.get_error() == sd.DEV_CAPACITY
    assert kv.lens.tolist() == [100, 100] and torch.equal(kv.k, before)


@pytest.mark.parametrize("call", ["greedy", "nucleus", "tree", "pipelined"])
def test_a_block_whose_rows_were_refused(sd, model, call):
    """Sequence 0 has pages, 1 shares its last one with 2, 3 has none behind a page's end."""
    shape, ctx = model
    kv = ctx.kv_paged(4, 300, 12)
    for s, n in ((0, 100), (1, 70), (3, 128)):
        ctx.kv_reserve(kv, 1, n, seq=s)
        ctx.prefill(kv, s, prompts(n, s))
    ctx.kv_fork(kv, i32([0, 1, 1, 3]))
    assert ctx.get_error() == 0
    q = 5
    toks, lg = prompts(4 * q, 7), torch.empty(4 * q, shape.vocab, device="cuda")
    acc, out = i32([0] * 4), i32([0] * 4 * q)
    parent = i32([-1, 0, 0, 1, 2] * 4)
    before = kv.k.clone()

    def step():
        if call == "tree":
            ctx.block_forward_tree(kv, toks, parent, lg, 4, q)
            ctx.accept_tree(kv, lg, toks, parent, 4, q, acc, out)
        else:
            ctx.block_forward(kv, toks, lg, 4, q)
            if call == "greedy":
                ctx.accept_greedy(kv, lg, toks, 4, q, q - 1, acc, out)
            elif call == "nucleus":
                ctx.accept_nucleus(kv, lg, toks, 4, q, q - 1, 0.95, 0.8, 3, acc, out)
            else:
                ctx.accept_pipelined(kv, lg, toks, i32([q - 1] * 4), 4, q, acc, out)

    step()
    assert ctx.get_error() & sd.DEV_CAPACITY
    assert kv.lens.tolist() == [100 + acc[0].item(), 70, 70, 128]
    rest = [i for i in range(12) if i != kv.table[0, 1].item()]
    assert torch.equal(kv.k[:, rest], before[:, rest])
    lens = kv.lens.tolist()
    ctx.kv_reserve(kv, 4, q)
    step()
    assert ctx.get_error() == 0
    assert kv.lens.tolist() == [n + a for n, a in zip(lens, acc.tolist())]
