"""Paged caches whose tables and lengths, which are handed out as writable memory, hold numbers that no call wrote: reported,
counted as none, and nothing beside them changes."""
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
    return shape, sd.Context(shape, synth.make_model(shape, seed=0, device="cuda", gain_std=0.1), max_position=1024)


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def cache(ctx):
    """Three sequences of 2, 1 and 3 pages, in this order, of a pool of 10."""
    kv = ctx.kv_paged(3, 256, 10)
    for s, n in ((0, 100), (1, 20), (2, 190)):
        ctx.kv_reserve(kv, 1, n, seq=s)
    ctx.kv_commit(kv, i32([100, 20, 190]), 3)
    assert kv.table.tolist() == [[0, 1, -1, -1], [2, -1, -1, -1], [3, 4, 5, -1]]
    return kv


OUTSIDE = [10, 11, 5000, 2 ** 31 - 1, -2, -2 ** 31]


@pytest.mark.parametrize("page", OUTSIDE)
def test_fork_and_free_drop_pages_outside_the_pool(sd, model, page):
    _, ctx = model
    kv = cache(ctx)
    kv.table[2, 1] = page
    ctx.kv_fork(kv, i32([2, 1]))
    assert ctx.get_error() == sd.DEV_PAGE
    assert kv.table.tolist() == [[3, -1, 5, -1], [2, -1, -1, -1], [3, page, 5, -1]]
    assert kv.refs.tolist() == [0, 0, 1, 2, 1, 2, 0, 0, 0, 0]
    ctx.kv_free(kv, 2)
    assert ctx.get_error() == sd.DEV_PAGE
    assert kv.table.tolist() == [[3, -1, 5, -1], [2, -1, -1, -1], [-1] * 4]
    assert kv.refs.tolist() == [0, 0, 1, 1, 1, 1, 0, 0, 0, 0]
    assert kv.lens.tolist() == [190, 20, 0]


@pytest.mark.parametrize("page", OUTSIDE)
def test_reserve_gives_a_page_in_their_place(sd, model, page):
    _, ctx = model
    kv = cache(ctx)
    kv.table[2, 2] = page
    ctx.kv_reserve(kv, 3, 6)
    assert ctx.get_error() == sd.DEV_PAGE
    assert kv.table.tolist() == [[0, 1, -1, -1], [2, -1, -1, -1], [3, 4, 6, 7]]
    assert kv.refs.tolist() == [1] * 8 + [0, 0]


@pytest.mark.parametrize("page", OUTSIDE)
def test_compact_leaves_them(sd, model, page):
    _, ctx = model
    kv = cache(ctx)
    ctx.kv_free(kv, 0)
    kv.table[1, 3] = page
    used = i32([0])
    ctx.kv_compact(kv, used)
    assert ctx.get_error() == sd.DEV_PAGE
    assert used.item() == 4
    assert kv.table.tolist() == [[-1] * 4, [2, -1, -1, page], [3, 0, 1, -1]]
    assert kv.refs.tolist() == [1] * 4 + [0] * 6


@pytest.mark.parametrize("src", [-2, -100, 3, 2 ** 31 - 1])
def test_sequences_outside_the_batch_are_not_forked_from(sd, model, src):
    """-1 alone empties a sequence."""
    _, ctx = model
    kv = cache(ctx)
    before = kv.table.tolist(), kv.refs.tolist(), kv.lens.tolist()
    ctx.kv_fork(kv, i32([0, src, 2]))
    assert ctx.get_error() == sd.DEV_PAGE
    assert (kv.table.tolist(), kv.refs.tolist(), kv.lens.tolist()) == before


@pytest.mark.parametrize("n", [-1, -70, -2 ** 31, 257, 10 ** 6, 2 ** 31 - 100])
def test_lengths_outside_the_capacity(sd, model, n):
    """Pages from slot 0 on, or none; a block's rows outside the capacity are not written."""
    shape, ctx = model
    kv = cache(ctx)
    kv.lens[1] = n
    ctx.kv_reserve(kv, 1, 70, seq=1)
    assert ctx.get_error() == sd.DEV_CAPACITY
    assert kv.table.tolist() == [[0, 1, -1, -1], [2, 6, -1, -1] if n < 0 else [2, -1, -1, -1], [3, 4, 5, -1]]
    assert kv.refs.tolist() == [1] * 6 + [1 if n < 0 else 0] + [0] * 3
    kv.lens[1] = n if n != -1 else -7            # (a block of six rows ends below 0)
    ctx.kv_reserve(kv, 1, 6, seq=2)
    ctx.get_error()
    kv.k.fill_(1.0), kv.v.fill_(1.0)
    lg = torch.empty(18, shape.vocab, device="cuda")
    ctx.block_forward(kv, synth.prompt_ids(0, 41, 18, 4096).cuda(), lg, 3, 6)
    assert ctx.get_error() & sd.DEV_CAPACITY
    written = kv.table[0, 1].item(), kv.table[2, 2].item(), kv.table[2, 3].item()    # the rows of the others
    rest = [i for i in range(10) if i not in written]
    assert (kv.k[:, rest] == 1).all() and (kv.v[:, rest] == 1).all()
    assert all((kv.k[:, i] != 1).any() for i in written)


@pytest.mark.parametrize("b", [1, 63, 64, 65, 200, 256])
def test_lengths_of_every_sequence_are_committed_and_rolled_back(sd, model, b):
    """A paged cache takes up to 256 sequences; so does a commit, and a contiguous cache's takes as many as it has."""
    _, ctx = model
    for kv in (ctx.kv_paged(256, 128, 600), ctx.kv(256, 128)):
        if isinstance(kv, sd.PagedKV):
            ctx.kv_reserve(kv, 256, 100)
        new = torch.tensor([(37 * s) % 101 for s in range(256)], dtype=torch.int32, device="cuda")
        ctx.kv_commit(kv, new, b)
        assert ctx.kv_lengths(kv).tolist() == new.tolist()[:b] + [0] * (256 - b)
        back = new // 2
        ctx.kv_commit(kv, back, b)
        assert ctx.kv_lengths(kv).tolist() == back.tolist()[:b] + [0] * (256 - b)
        assert ctx.get_error() == 0
        with pytest.raises(sd.SdsatError) as e:
            ctx.kv_commit(kv, new, 257)
        assert e.value.status == 1


@pytest.mark.parametrize("offset", [0, 1, 3, 7, 8])
@pytest.mark.parametrize("slot0,n", [(0, 1), (60, 70), (0, 200)])
def test_rows_to_and_from_buffers_of_any_alignment(sd, model, offset, slot0, n):
    """Buffers that start anywhere, as contiguous caches take them, beside values that must stay."""
    shape, ctx = model
    kv = ctx.kv_paged(2, 256, 9)
    ctx.kv_reserve(kv, 2, 256)
    size = shape.n_heads * n * shape.head_dim
    x = [torch.randn(size + 20, device="cuda").bfloat16() for _ in range(2)]
    at = lambda t: t[offset:offset + size].view(shape.n_heads, n, shape.head_dim)  # noqa: E731
    ctx.kv_write(kv, 1, 1, slot0, at(x[0]), at(x[1]))
    got = ctx.kv_read(kv, 1, 1, slot0, n)
    assert torch.equal(got[0], at(x[0])) and torch.equal(got[1], at(x[1]))
    back = [torch.full_like(t, 9.0) for t in x]
    assert sd.lib().sdsat_kv_read(ctx.handle, kv.handle, 1, 1, slot0, n, at(back[0]).data_ptr(), at(back[1]).data_ptr()) == 0
    for b, t in zip(back, x):
        assert torch.equal(b[offset:offset + size], t[offset:offset + size])
        assert (b[:offset] == 9).all() and (b[offset + size:] == 9).all()
    assert ctx.get_error() == 0
    ctx.kv_free(kv, 1)
    ctx.kv_write(kv, 1, 1, slot0, at(x[0]), at(x[1]))
    assert ctx.get_error() == sd.DEV_CAPACITY
    assert sd.lib().sdsat_kv_read(ctx.handle, kv.handle, 1, 1, slot0, n, at(back[0]).data_ptr(), at(back[1]).data_ptr()) == 0
    assert (at(back[0]) == 0).all() and (at(back[1]) == 0).all()
    assert ctx.get_error() == sd.DEV_CAPACITY


@pytest.mark.parametrize("slot0,n", [(256, 1), (255, 2), (2 ** 31 - 1, 1), (2 ** 31 - 100, 200), (1, 2 ** 31 - 1), (-1, 1), (0, -1)])
def test_rows_outside_the_capacity_are_refused(sd, model, slot0, n):
    """Slots whose sum with the number of rows does not fit 32 bits, too."""
    _, ctx = model
    x = torch.zeros(64, dtype=torch.bfloat16, device="cuda").data_ptr()
    for kv in (ctx.kv(2, 256), ctx.kv_paged(2, 256, 9)):
        for f in (sd.lib().sdsat_kv_write, sd.lib().sdsat_kv_read):
            assert f(ctx.handle, kv.handle, 0, 0, slot0, n, x, x) == 1
    assert ctx.get_error() == 0


def test_pools_of_more_rows_than_the_kernels_count(sd, model):
    """2 layers, 4 heads: 2^31 rows of K are 2^22 pages."""
    _, ctx = model
    for pages in (2 ** 22, 2 ** 22 + 1, 2 ** 31 - 1):
        with pytest.raises(sd.SdsatError) as e:
            ctx.kv_paged(1, 64, pages)
        assert e.value.status == 6, pages
