"""Paged caches: forking, reserving (copy on write), freeing and packing pages against a model of the
rules on the host, and the block decode step on them against contiguous caches.  Tables, counts and
copied rows are exact."""
import random

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
def bare(sd):
    return sd.Context(synth.SHAPES["tiny"], None, max_position=4096)


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


class Model:
    """The rules one sequence and one page at a time."""

    def __init__(self, batch, max_len, n_pages):
        self.cap, self.ld = max_len, -(-max_len // PAGE)
        self.table = [[-1] * self.ld for _ in range(batch)]
        self.len, self.refs = [0] * batch, [0] * n_pages
        self.rows = {}               # (page, slot) -> content
        self.short = False

    def fork(self, src):
        was, lens = [list(r) for r in self.table], list(self.len)
        for s, a in enumerate(src):
            self._set(s, list(was[a]) if a >= 0 else [-1] * self.ld, lens[a] if a >= 0 else 0)

    def _set(self, s, row, n):
        for p in self.table[s]:
            if p >= 0:
                self.refs[p] -= 1
        for p in row:
            if p >= 0:
                self.refs[p] += 1
        self.table[s], self.len[s] = row, n

    def free(self, s):
        self._set(s, [-1] * self.ld, 0)

    def wanted(self, s, n):
        return range(self.len[s] // PAGE, max(self.len[s] // PAGE, -(-min(self.len[s] + n, self.cap) // PAGE)))

    def reserve(self, seq, b, n):
        refs, need = list(self.refs), 0
        for s in range(seq, seq + b):
            self.short |= self.len[s] + n > self.cap
            for j in self.wanted(s, n):
                p = self.table[s][j]
                if p < 0 or refs[p] > 1:
                    need += 1
                    if p >= 0:
                        refs[p] -= 1
        if need > self.refs.count(0):
            self.short = True
            return
        for s in range(seq, seq + b):
            for j in self.wanted(s, n):
                p = self.table[s][j]
                if p >= 0 and self.refs[p] == 1:
                    continue
                new = self.refs.index(0)
                self.refs[new], self.table[s][j] = 1, new
                if p >= 0:
                    self.refs[p] -= 1
                    for r in range(max(0, min(PAGE, self.len[s] - j * PAGE))):
                        self.rows[new, r] = self.rows[p, r]

    def compact(self):
        used = sum(r > 0 for r in self.refs)
        moves = list(zip([p for p in range(used, len(self.refs)) if self.refs[p]], [p for p in range(used) if not self.refs[p]]))
        for a, z in moves:
            for s, row in enumerate(self.table):
                for j, p in enumerate(row):
                    for r in range(max(0, min(PAGE, self.len[s] - j * PAGE)) if p == a else 0):
                        self.rows[z, r] = self.rows[a, r]
            self.refs[z], self.refs[a] = self.refs[a], 0
            self.table = [[z if p == a else p for p in row] for row in self.table]
        return used

    def slot(self, s, t):
        return self.table[s][t // PAGE], t % PAGE


def compare(m, kv):
    assert kv.table.tolist() == m.table
    assert kv.refs.tolist() == m.refs
    assert kv.lens.tolist() == m.len


def contents(m, kv, ctx):
    """Every committed slot of every sequence holds what the model says (a number per row)."""
    for s, n in enumerate(m.len):
        if n == 0:
            continue
        want = torch.tensor([m.rows[m.slot(s, t)] for t in range(n)], device="cuda")
        for layer in (0, 1):
            k, v = ctx.kv_read(kv, layer, s, 0, n)
            assert torch.equal(k.float(), (want % 251)[None, :, None].float().expand_as(k)), (s, layer)
            assert torch.equal(v.float(), (want // 251 + layer)[None, :, None].float().expand_as(v)), (s, layer)


def write(m, kv, ctx, s, n, stamp):
    """n more committed slots of sequence s, each with a number of its own."""
    shape = synth.SHAPES["tiny"]
    at = m.len[s]
    ids = torch.arange(stamp, stamp + n, device="cuda")
    for layer in (0, 1):
        k = (ids % 251)[None, :, None].expand(shape.n_heads, n, shape.head_dim).bfloat16().contiguous()
        v = (ids // 251 + layer)[None, :, None].expand(shape.n_heads, n, shape.head_dim).bfloat16().contiguous()
        ctx.kv_write(kv, layer, s, at, k, v)
    for i in range(n):
        m.rows[m.slot(s, at + i)] = stamp + i
    m.len[s] += n
    ctx.kv_commit(kv, i32(m.len), len(m.len))


@pytest.mark.parametrize("seed", range(6))
def test_random_sequences_of_calls(sd, bare, seed):
    rng = random.Random(seed)
    batch, max_len, pages = rng.choice([(5, 300, 24), (9, 1000, 60), (33, 200, 90), (3, 64, 5)])
    kv, m, stamp = bare.kv_paged(batch, max_len, pages), Model(batch, max_len, pages), 0
    compare(m, kv)
    for _ in range(40):
        act = rng.choice(["grow", "grow", "grow", "fork", "back", "free", "compact"])
        m.short = False
        if act == "grow":
            seq = rng.randrange(batch)
            b, n = rng.randint(1, batch - seq), rng.choice([1, 3, 16, 64, 65, 150])
            bare.kv_reserve(kv, b, n, seq=seq)
            m.reserve(seq, b, n)
            assert bare.get_error() == (sd.DEV_CAPACITY if m.short else 0)
            compare(m, kv)
            if not m.short:
                for s in range(seq, seq + b):
                    k = rng.randint(0, n)
                    if k:
                        write(m, kv, bare, s, k, stamp)
                        stamp += k
        elif act == "fork":
            b = rng.randint(1, batch)
            src = [rng.choice([s, rng.randrange(batch), rng.randrange(batch), -1]) for s in range(b)]
            bare.kv_fork(kv, i32(src))
            m.fork(src)
        elif act == "back":                      # a rollback into pages that others may hold
            m.len = [rng.randint(0, n) if rng.random() < 0.3 else n for n in m.len]
            bare.kv_commit(kv, i32(m.len), batch)
        elif act == "free":
            s = rng.randrange(batch)
            bare.kv_free(kv, s)
            m.free(s)
        else:
            used = torch.zeros(1, dtype=torch.int32, device="cuda")
            bare.kv_compact(kv, used)
            assert used.item() == m.compact()
        compare(m, kv)
        assert bare.get_error() == 0
    contents(m, kv, bare)


def test_the_copy_takes_the_committed_slots_alone(bare):
    """A fork's first reserve copies len % 64 slots of every layer and head, whole pages stay shared."""
    kv, m = bare.kv_paged(3, 400, 12), Model(3, 400, 12)
    bare.kv_reserve(kv, 1, 150)
    m.reserve(0, 1, 150)
    write(m, kv, bare, 0, 150, 0)
    k, v = kv.k, kv.v
    k[:, 3:], v[:, 3:] = 7.0, 7.0
    bare.kv_fork(kv, i32([0, 0, 0]))
    m.fork([0, 0, 0])
    bare.kv_reserve(kv, 3, 6)
    m.reserve(0, 3, 6)
    compare(m, kv)
    assert kv.table[:, :3].tolist() == [[0, 1, 3], [0, 1, 4], [0, 1, 2]]
    contents(m, kv, bare)
    assert (k[:, 3:5, :, 22:] == 7).all() and (k[:, 5:] == 7).all() and (v[:, 3:5, :, 22:] == 7).all()
    bare.kv_reserve(kv, 3, 6)                    # nothing left to do
    compare(m, kv)


def test_a_full_pool_changes_nothing(sd, bare):
    kv, m = bare.kv_paged(4, 256, 5), Model(4, 256, 5)
    bare.kv_reserve(kv, 1, 256)
    m.reserve(0, 1, 256)
    write(m, kv, bare, 0, 200, 0)
    bare.kv_fork(kv, i32([0, 0, 0, 0]))
    m.fork([0, 0, 0, 0])
    bare.kv_reserve(kv, 4, 6)                    # wants three pages, one is free
    m.reserve(0, 4, 6)
    assert bare.get_error() == sd.DEV_CAPACITY
    compare(m, kv)
    contents(m, kv, bare)
    # shared pages are not written: the rows are refused, and the others' stay
    before = kv.k.clone()
    one = torch.ones(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    bare.kv_write(kv, 0, 1, 199, one, one)
    assert bare.get_error() == sd.DEV_CAPACITY
    assert torch.equal(kv.k, before)
    bare.kv_free(kv, 3)
    bare.kv_free(kv, 2)
    m.free(3), m.free(2)
    bare.kv_reserve(kv, 2, 6)
    m.reserve(0, 2, 6)
    assert bare.get_error() == 0
    compare(m, kv)


def test_long_tables_and_many_sequences(bare):
    """More table entries and pages than the table kernels have threads."""
    kv, m = bare.kv_paged(200, 4096, 3000), Model(200, 4096, 3000)
    bare.kv_reserve(kv, 1, 4000)
    m.reserve(0, 1, 4000)
    m.len[0] = 4000
    m.rows = {(p, r): p for p in range(3000) for r in range(PAGE)}
    bare.kv_commit(kv, i32(m.len[:1]), 1)
    src = [0] * 200
    bare.kv_fork(kv, i32(src))
    m.fork(src)
    bare.kv_reserve(kv, 200, 96)
    m.reserve(0, 200, 96)
    assert bare.get_error() == 0
    compare(m, kv)
    src = [(7 * s) % 200 if s % 3 else -1 for s in range(200)]
    bare.kv_fork(kv, i32(src))
    m.fork(src)
    compare(m, kv)
    bare.kv_compact(kv)
    m.compact()
    compare(m, kv)


def test_a_fork_from_outside_the_batch_is_reported(sd, bare):
    kv, m = bare.kv_paged(3, 128, 8), Model(3, 128, 8)
    bare.kv_reserve(kv, 3, 20)
    m.reserve(0, 3, 20)
    bare.kv_fork(kv, i32([1, 3, 99]))
    m.fork([1, 1, 2])
    assert bare.get_error() == sd.DEV_PAGE
    compare(m, kv)


def test_refusals(sd, bare):
    kv, flat = bare.kv_paged(3, 128, 8), bare.kv(3, 128)
    src = i32([0, 0, 0])
    for call in (lambda: bare.kv_fork(kv, src, 4), lambda: bare.kv_fork(kv, src, 0), lambda: bare.kv_free(kv, 3),
                 lambda: bare.kv_free(kv, -1), lambda: bare.kv_reserve(kv, 4, 1), lambda: bare.kv_reserve(kv, 1, 1, seq=3),
                 lambda: bare.kv_reserve(kv, 0, 1), lambda: bare.kv_reserve(kv, 1, -1), lambda: bare.kv_fork(flat, src),
                 lambda: bare.kv_free(flat, 0), lambda: bare.kv_reserve(flat, 1, 1), lambda: bare.kv_compact(flat),
                 lambda: bare.kv_paged(0, 64, 4), lambda: bare.kv_paged(257, 64, 4), lambda: bare.kv_paged(1, 64, 0),
                 lambda: bare.kv_paged(1, 0, 4)):
        with pytest.raises(sd.SdsatError) as e:
            call()
        assert e.value.status == 1
    with pytest.raises(sd.SdsatError) as e:
        bare.kv_paged(1, 5000, 4)
    assert e.value.status == 3
    bare.kv_reserve(kv, 3, 0)
    assert bare.get_error() == 0 and kv.refs.sum().item() == 0


# ---- the block decode step ------------------------------------------------------------------------


@pytest.fixture(scope="module")
def model(sd):
    shape = synth.SHAPES["tiny"]
    return shape, sd.Context(shape, synth.make_model(shape, seed=0, device="cuda", gain_std=0.1), max_position=1024)


def prompts(n, seed=0):
    return synth.prompt_ids(seed, 40, n, 4096).cuda()


# bf16 rows of the caches move by one place between a tiled GEMM's and a skinny one's sums
NEAR = 3e-2


@pytest.mark.parametrize("n", [1, 9, 16, 17, 63, 64, 65, 200, 513])
def test_prefill_into_pages(sd, model, n):
    """The same prompt into a contiguous and into a paged cache, in two parts, then a block."""
    shape, ctx = model
    flat, kv = ctx.kv(2, 700), ctx.kv_paged(2, 700, 40)
    ids = prompts(n + 30)
    for seq in (1, 0):                           # pages in another order than the sequences
        ctx.kv_reserve(kv, 1, n, seq=seq)
        for c in (flat, kv):
            ctx.prefill(c, seq, ids[:n])
        ctx.kv_reserve(kv, 1, 30, seq=seq)
        for c in (flat, kv):
            ctx.prefill(c, seq, ids[n:])
    assert kv.lens.tolist() == [n + 30] * 2
    for layer in range(shape.n_layers):
        for seq in range(2):
            for a, z in zip(ctx.kv_read(flat, layer, seq, 0, n + 30), ctx.kv_read(kv, layer, seq, 0, n + 30)):
                assert (a.float() - z.float()).abs().max().item() <= NEAR
    toks = prompts(12, 1)
    la, lz = torch.empty(12, shape.vocab, device="cuda"), torch.empty(12, shape.vocab, device="cuda")
    ctx.block_forward(flat, toks, la, 2, 6)
    ctx.kv_reserve(kv, 2, 6)
    ctx.block_forward(kv, toks, lz, 2, 6)
    assert (la - lz).abs().max().item() <= NEAR
    assert ctx.get_error() == 0


@pytest.mark.parametrize("b,q", [(2, 6), (4, 6), (5, 5), (10, 6), (64, 1), (4, 16)])
def test_samples_of_one_prompt_decode_as_sequences_of_their_own(sd, model, b, q):
    """b nucleus samples from pages that share the prompt, and from b contiguous copies of it: the same
    tokens, block by block (every block starts from the contiguous side's, so that a logit that rounds
    another way ends in one place)."""
    shape, ctx = model
    n = 150
    ids = prompts(n + 1)
    flat, kv = ctx.kv(b, 400), ctx.kv_paged(b + 1, 400, 3 + 5 * b)
    ctx.kv_reserve(kv, 1, n, seq=b)
    ctx.prefill(kv, b, ids[:n])
    ctx.kv_fork(kv, i32([b] * b))
    for s in range(b):
        ctx.prefill(flat, s, ids[:n])
    toks = torch.empty(b, q, dtype=torch.int32, device="cuda")
    toks[:, 0], toks[:, 1:] = ids[n], shape.adaptive_id
    lg = [torch.empty(b * q, shape.vocab, device="cuda") for _ in range(2)]
    acc = [torch.empty(b, dtype=torch.int32, device="cuda") for _ in range(2)]
    out = [torch.empty(b, q, dtype=torch.int32, device="cuda") for _ in range(2)]
    same = 0
    for step in range(6):
        ctx.kv_reserve(kv, b, q)
        for i, c in enumerate((flat, kv)):
            ctx.block_forward(c, toks, lg[i], b, q)
            ctx.accept_nucleus(c, lg[i], toks, b, q, q - 1 if step % 2 else 0, 0.95, 0.8, 5, acc[i], out[i])
        assert (lg[0] - lg[1]).abs().max().item() <= NEAR
        same += (out[0] == out[1]).float().mean().item() / 6
        ctx.kv_commit(kv, ctx.kv_lengths(flat), b)
        last = out[0].gather(1, (acc[0] - 1).long()[:, None])[:, 0]
        toks = toks.clone()
        toks[:, 0] = last if step % 2 else out[0][:, 0]
        toks[:, 1:] = shape.adaptive_id if step % 2 else out[0][:, 1:]
    assert same >= 0.97, same
    assert ctx.get_error() == 0
    if b > 1:
        assert kv.refs.max().item() == b + 1     # the prompt's whole pages are still shared


def test_tree_blocks_on_pages(sd, model):
    shape, ctx = model
    n, b = 125, 3                                # the block crosses a page's end
    ids = prompts(n)
    flat, kv = ctx.kv(b, 300), ctx.kv_paged(b, 300, 20)
    ctx.kv_reserve(kv, 1, n)
    ctx.prefill(kv, 0, ids)
    ctx.kv_fork(kv, i32([0] * b))
    for s in range(b):
        ctx.prefill(flat, s, ids)
    parent = i32([-1, 0, 0, 1, 2, 4, 4] * b)
    toks = prompts(7 * b, 3)
    lg = [torch.empty(7 * b, shape.vocab, device="cuda") for _ in range(2)]
    ctx.kv_reserve(kv, b, 7)
    ctx.block_forward_tree(flat, toks, parent, lg[0], b, 7)
    ctx.block_forward_tree(kv, toks, parent, lg[1], b, 7)
    assert (lg[0] - lg[1]).abs().max().item() <= NEAR
    # a path that is accepted whole: its rows move across the page's end
    best = lg[0].argmax(-1).view(b, 7)
    t = toks.view(b, 7).clone()
    for j, p in ((2, 0), (4, 2), (6, 4)):
        t[:, j] = best[:, p]
    out = []
    for c in (flat, kv):
        ctx.block_forward_tree(c, t, parent, lg[0], b, 7)
        best = lg[0].argmax(-1).view(b, 7)
        acc, o, path = torch.empty(b, dtype=torch.int32, device="cuda"), torch.empty(b, 7, dtype=torch.int32, device="cuda"), torch.empty(b, 7, dtype=torch.int32, device="cuda")
        ctx.accept_tree(c, lg[0], t, parent, b, 7, acc, o, path)
        out.append((acc.tolist(), o.tolist(), path.tolist(), ctx.kv_lengths(c).tolist()))
    assert out[0] == out[1]
    for layer in range(shape.n_layers):
        for s in range(b):
            m = out[0][3][s]
            for a, z in zip(ctx.kv_read(flat, layer, s, 0, m), ctx.kv_read(kv, layer, s, 0, m)):
                assert (a.float() - z.float()).abs().max().item() <= NEAR
    assert ctx.get_error() == 0


def test_a_block_without_pages_of_its_own_is_not_written(sd, model):
    shape, ctx = model
    kv = ctx.kv_paged(2, 300, 20)
    ctx.kv_reserve(kv, 1, 100)
    ctx.prefill(kv, 0, prompts(100))
    ctx.kv_fork(kv, i32([0, 0]))
    before = kv.k.clone()
    lg = torch.empty(12, shape.vocab, device="cuda")
    ctx.block_forward(kv, prompts(12, 1), lg, 2, 6)   # shared by both, nothing reserved
    assert ctx.get_error() & sd.DEV_CAPACITY
    assert torch.equal(before, kv.k)
    ctx.kv_reserve(kv, 2, 6)
    ctx.block_forward(kv, prompts(12, 1), lg, 2, 6)
    assert ctx.get_error() == 0 and torch.isfinite(lg).all()
