"""The operators of ragged batches together, as a decoder layer and its sampling would use them: heads rotated and appended to
a paged cache, attention over it, logits under rules, tokens selected and scored; prompts of different lengths, forked
samples, single tokens behind them."""
import math

import pytest
import torch

import synth
from ragged import generator, ints

pytestmark = pytest.mark.gpu

PAGE = 64


@pytest.fixture(scope="module")
def sd():
    import paper_2403_18647_gb300 as sd
    return sd


class Layer:
    """A reference in 64 bits that keeps every sequence's rotated keys and its values as the cache rounds them."""

    def __init__(self, ctx, kv, layer, type):
        self.ctx, self.kv, self.layer, self.type = ctx, kv, layer, type
        s = ctx.shape
        self.H, self.hd = s.n_heads, s.head_dim
        self.rope = ctx.rope(self.hd, 4096, theta=1e4)
        self.k, self.v = {}, {}
        self.gains = [(1 + 0.2 * torch.randn(self.hd, generator=generator(i), device="cuda")).bfloat16() for i in (1, 2)]

    def turned(self, x, gain, pos):
        x = x.double().view(x.shape[0], self.H, self.hd)
        x = x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt() * gain.double()
        half = self.hd // 2
        f = 1e4 ** (-torch.arange(half, dtype=torch.float64, device="cuda") * 2 / self.hd)
        c, s = (pos.double()[:, None] * f).cos()[:, None], (pos.double()[:, None] * f).sin()[:, None]
        a, z = x[..., :half], x[..., half:]
        return torch.cat((a * c - z * s, a * s + z * c), -1)

    def step(self, g, new):
        """new rows for sequences 0 .. b-1 through the operators, checked; the lengths are committed."""
        ctx, kv, H, hd = self.ctx, self.kv, self.H, self.hd
        b = len(new)
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        rows = starts[-1]
        x = (torch.randn(rows, 3 * H * hd, generator=g, device="cuda") * 1.5).to(self.type)
        q, k, v = x[:, :H * hd], x[:, H * hd:2 * H * hd], x[:, 2 * H * hd:]
        turned, out = torch.empty(rows, H * hd, dtype=self.type, device="cuda"), torch.empty(rows, H * hd, dtype=self.type, device="cuda")
        at, table, lens = ints(starts), kv.table[:b], kv.lens[:b]
        ctx.kv_reserve(kv, b, max(new))
        ctx.op_rotary_append(self.rope, q, k, v, turned, kv.k[self.layer], kv.v[self.layer], table, lens, at, H, H, hd,
                             q_gain=self.gains[0], k_gain=self.gains[1], refs=kv.refs)
        ctx.op_chunk_attention(turned, kv.k[self.layer], kv.v[self.layer], table, lens, at, H, H, hd, out)
        was = lens.tolist()
        for s, n in enumerate(new):
            if not n:
                continue
            r = slice(starts[s], starts[s + 1])
            pos = torch.arange(was[s], was[s] + n, device="cuda")
            # a key is rounded once to bf16; before that it is 2^-20 (|a| + |z|) off at most, and |a| + |z| below 16
            got_k, got_v = ctx.kv_read(kv, self.layer, s, 0, was[s] + n)
            ref = self.turned(k[r], self.gains[1], pos).transpose(0, 1)
            assert ((got_k[:, was[s]:].double() - ref).abs() <= 2 ** -8 * ref.abs() + 2 ** -16).all()
            assert torch.equal(got_v[:, was[s]:], v[r].reshape(n, H, hd).transpose(0, 1).bfloat16())
            if was[s]:
                assert torch.equal(got_k[:, :was[s]], self.k[s]) and torch.equal(got_v[:, :was[s]], self.v[s])
            self.k[s], self.v[s] = got_k, got_v
            y = turned[r].double().view(n, H, hd).transpose(0, 1)
            seen = torch.ones(n, was[s] + n, dtype=torch.bool, device="cuda").tril(was[s])
            w = (y @ got_k.double().transpose(1, 2) / math.sqrt(hd)).masked_fill(~seen, -math.inf).softmax(-1)
            ref, size = w @ got_v.double(), w @ got_v.double().abs()
            err = (out[r].double().view(n, H, hd).transpose(0, 1) - ref).abs()
            if self.type == torch.bfloat16:
                err = err - 2 ** -8 * (ref.abs() + size)
            assert err.max().item() <= 2e-5
        ctx.kv_commit(kv, ints([m + n for m, n in zip(was, new)]), b)
        return out

    def fork(self, src):
        self.ctx.kv_fork(self.kv, ints(src))
        k, v = dict(self.k), dict(self.v)
        for s, f in enumerate(src):
            if f >= 0:
                self.k[s], self.v[s] = k[f], v[f]


@pytest.mark.parametrize("type", [torch.float32, torch.bfloat16])
def test_prompts_forks_and_single_tokens(sd, type):
    ctx = sd.Context(synth.SHAPES["tiny"], None, max_position=4096)
    kv = ctx.kv_paged(6, 700, 60)
    layer = Layer(ctx, kv, 1, type)
    g = generator(3)
    layer.step(g, [130, 7, 300, 64])                 # prompts
    layer.step(g, [1, 200, 0, 65])                   # one decodes, one goes on, one waits
    layer.fork([0, 1, 2, 3, 1, 2])                   # samples of two of them
    layer.step(g, [1, 1, 1, 1, 1, 1])                # pages that were shared are copied before they are written
    layer.step(g, [3, 0, 17, 1, 6, 16])
    assert ctx.get_error() == 0
    kv.refs[kv.table[2, 0].long()] += 1              # a page that somebody else holds too is not written
    before = kv.k[1][kv.table[2, 0].long()].clone()
    kv.lens[2] = 5
    x = torch.randn(1, 3 * 256, device="cuda").to(type)
    out = torch.empty(1, 256, dtype=type, device="cuda")
    ctx.op_rotary_append(layer.rope, x[:, :256], x[:, 256:512], x[:, 512:], out, kv.k[1], kv.v[1], kv.table[2:3], kv.lens[2:3], ints([0, 1]),
                         4, 4, 64, refs=kv.refs)
    assert ctx.get_error() == sd.DEV_CAPACITY and torch.equal(kv.k[1][kv.table[2, 0].long()], before)


def test_rules_before_tokens_are_selected(sd):
    """Drafts verified against logits under rules: every emitted token is allowed, a forbidden draft is rejected, and the scores
    are those of the rows that the selection saw."""
    shape = synth.SHAPES["tiny"]
    ctx = sd.Context(shape, None, max_position=128)
    kv = ctx.kv(3, 100)
    g = generator(4)
    b, q, V = 3, 6, shape.vocab
    logits = torch.randn(b * q, V, generator=g, device="cuda") * 3
    drafts = logits.view(b, q, V).argmax(-1).int()
    tokens = torch.cat([ints([[5], [6], [7]]), drafts[:, :-1]], 1).contiguous()       # drafts that plain logits would accept
    allowed = torch.full((b * q, -(-V // 32)), -1, dtype=torch.int32, device="cuda")
    t = drafts[1, 2].item()
    allowed[1 * q + 2, t // 32] &= ~(1 << (t % 32)) if t % 32 < 31 else 0x7FFFFFFF       # sequence 1's third target is forbidden
    acc, out = torch.empty(b, dtype=torch.int32, device="cuda"), torch.empty(b * q, dtype=torch.int32, device="cuda")
    ruled = torch.empty_like(logits)
    ctx.op_adjust_logits(logits, ruled, q, tokens=tokens.view(-1), repetition=torch.ones(b, device="cuda"), allowed=allowed)
    ctx.accept_greedy(kv, ruled, tokens.view(-1), b, q, q - 1, acc, out)
    assert acc.tolist() == [q, 3, q]
    assert out.view(b, q)[1, 2].item() != t
    # a penalty that outweighs everything: no target repeats a token of the block before it
    ctx.op_adjust_logits(logits, ruled, q, tokens=tokens.view(-1), presence=torch.full((b,), 100.0, device="cuda"))
    ctx.accept_greedy(kv, ruled, tokens.view(-1), b, q, q - 1, acc, out)
    for s in range(b):
        for j in range(q):
            assert out.view(b, q)[s, j].item() not in tokens[s, :j + 1].tolist()
    logp, rank = torch.empty(b * q, device="cuda"), torch.empty(b * q, dtype=torch.int32, device="cuda")
    ctx.op_logprobs(ruled, tokens=out, logp=logp, rank=rank)
    assert (rank == 1).all()
    want = ruled.double().log_softmax(-1).gather(1, out.long()[:, None])[:, 0]
    assert (logp.double() - want).abs().max().item() <= 1e-5
    assert ctx.get_error() == 0


def test_the_chain_in_a_graph(sd):
    """Append, attention and rules captured once and replayed while the cache grows."""
    ctx = sd.Context(synth.SHAPES["tiny"], None, max_position=512)
    H, hd, b = 4, 64, 3
    kv = ctx.kv_paged(b, 300, 20)
    ctx.kv_reserve(kv, b, 300)
    rope = ctx.rope(hd, 512)
    g = generator(6)
    x = torch.zeros(b, 3 * H * hd, dtype=torch.bfloat16, device="cuda")
    turned, out = torch.zeros(b, H * hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(b, H * hd, dtype=torch.bfloat16, device="cuda")
    starts, grown, one = ints([0, 1, 2, 3]), torch.zeros(b, dtype=torch.int32, device="cuda"), ints([1, 1, 1])

    def step():
        ctx.op_rotary_append(rope, x[:, :256], x[:, 256:512], x[:, 512:], turned, kv.k[0], kv.v[0], kv.table, kv.lens, starts, H, H, hd, refs=kv.refs)
        ctx.op_chunk_attention(turned, kv.k[0], kv.v[0], kv.table, kv.lens, starts, H, H, hd, out)
        torch.add(kv.lens, one, out=grown)
        ctx.kv_commit(kv, grown, b)

    inputs = [torch.randn(b, 3 * H * hd, generator=g, device="cuda").bfloat16() for _ in range(140)]
    want = []
    for t in inputs:
        x.copy_(t)
        step()
        want.append(out.clone())
    ctx.kv_commit(kv, torch.zeros(b, dtype=torch.int32, device="cuda"), b)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for t, w in zip(inputs, want):
        x.copy_(t)
        graph.replay()
        assert torch.equal(out, w)
    assert kv.lens.tolist() == [140] * 3 and ctx.get_error() == 0
