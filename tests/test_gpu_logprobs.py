"""Log probabilities, ranks, entropies and alternatives against 64 bits.

Tolerance.  d = (l - m) / T and the sums are fp32: |d| is off by at most 2 units of 2^-24 |d|, an
exp by 2^-22 and by what its argument is off, and so is log S by 2^-22 + 2^-23 sum p |d| <= 1e-6 for
the entropies here (below 13); the result rounds once.  Allowed: 3e-6 + 4e-7 |ref|.  Ranks and ids are
exact: they follow from comparisons of the logits themselves.
"""
import math

import pytest
import torch

import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    import paper_2403_18647_gb300 as sd
    return sd


@pytest.fixture(scope="module")
def ctx(sd):
    return sd.Context(synth.SHAPES["tiny"], None, max_position=64)


def reference(x, tokens, n, temperature):
    """x [rows, V] of any type; float64 results, ids by (logit descending, id ascending)."""
    x = x.double()
    x = torch.where(x.isnan(), -math.inf, x)
    m = x.amax(-1, keepdim=True)
    dead = m == -math.inf
    d = torch.where(x == m, 0.0, (x - m) / temperature)
    e = torch.where(dead, 0.0, d.exp())
    s = e.sum(-1, keepdim=True)
    logz = torch.where(dead, math.inf, s.log())
    entropy = torch.where(dead, 0.0, s.log() - torch.where(e > 0, e * d, 0.0).sum(-1, keepdim=True) / s)[:, 0]
    t = tokens.long().clamp(min=0)[:, None]
    t = torch.where(t < x.shape[1], t, 0)
    lt = x.gather(1, t)
    ids = torch.arange(x.shape[1])
    none = tokens == -1
    rank = 1 + (x > lt).sum(-1) + ((x == lt) & (ids < t)).sum(-1)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :n]
    return dict(logp=torch.where(none, 0.0, (d.gather(1, t) - logz)[:, 0]), entropy=entropy,
                rank=torch.where(none, 0, rank).int(), top_ids=order.int(), top_logp=d.gather(1, order) - logz)


def run(ctx, logits, tokens, n, temperature=1.0):
    rows = logits.shape[0]
    out = dict(logp=torch.full((rows,), math.nan), entropy=torch.full((rows,), math.nan), rank=torch.full((rows,), -7, dtype=torch.int32),
               top_ids=torch.full((rows, n), -7, dtype=torch.int32), top_logp=torch.full((rows, n), math.nan))
    out = {k: v.cuda() for k, v in out.items()}
    ctx.op_logprobs(logits, tokens.cuda(), out["logp"], out["entropy"], out["rank"], out["top_ids"] if n else None,
                    out["top_logp"] if n else None, temperature=temperature)
    return {k: v.cpu() for k, v in out.items()}


def check(got, ref):
    for k in ("rank", "top_ids"):
        assert torch.equal(got[k], ref[k]), (k, got[k], ref[k])
    for k in ("logp", "entropy", "top_logp"):
        a, b = got[k].double(), ref[k]
        fine = b.isfinite()
        assert torch.equal(fine, a.isfinite()) and torch.equal(a[~fine], b[~fine]), (k, a, b)
        off = (a - b).abs()[fine] - 4e-7 * b.abs()[fine]
        assert off.numel() == 0 or off.max().item() <= 3e-6, (k, off.max().item())


def logits(seed, rows, vocab, std=2.5):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g) * std
    t = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    return x, t


@pytest.mark.parametrize("rows,vocab,n", [(1, 1, 1), (1, 2, 2), (3, 31, 31), (2, 33, 32), (7, 511, 5), (1, 4096, 20), (6, 4104, 0),
                                          (5, 4097, 1), (64, 32016, 10), (3, 32017, 32), (2, 65537, 20), (1, 262144, 32),
                                          (2, 131071, 7), (700, 1000, 3), (330, 9001, 2)])
@pytest.mark.parametrize("type", [torch.float32, torch.bfloat16])
def test_sizes(ctx, rows, vocab, n, type):
    x, t = logits(rows + vocab, rows, vocab)
    x = x.to(type)
    got = run(ctx, x.cuda(), t, n)
    check(got, reference(x, t, n, 1.0))
    assert ctx.get_error() == 0


@pytest.mark.parametrize("temperature", [0.05, 0.7, 1.0, 3.0])
def test_temperatures(ctx, temperature):
    x, t = logits(5, 9, 5003)
    check(run(ctx, x.cuda(), t, 20, temperature), reference(x, t, 20, float(torch.tensor(temperature))))


@pytest.mark.parametrize("type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("first,pad", [(0, 1), (0, 3), (1, 0), (2, 5), (3, 2), (5, 8)])
def test_rows_of_any_distance_and_alignment(ctx, type, first, pad):
    """A view into wider rows; what lies beside the vocabulary is not read as a logit."""
    x, t = logits(8, 11, 2501)
    wide = torch.full((11, first + 2501 + pad), math.nan).to(type)
    wide[:, first:first + 2501] = x.to(type)
    view = wide.cuda()[:, first:first + 2501]
    check(run(ctx, view, t, 12), reference(x.to(type), t, 12, 1.0))
    assert ctx.get_error() == 0


def test_ties_go_to_the_lowest_id(ctx):
    """All equal; two values; a long plateau at the edge of the alternatives; -0 beside +0."""
    V = 40007
    x = torch.zeros(5, V)
    x[1, ::2] = 1.0
    x[2, :] = torch.arange(V) // 9000
    x[3, 100:30000] = 3.0
    x[3, 35000] = 4.0
    x[4, 5::7] = -0.0
    x[4, 2] = 1.0
    t = torch.tensor([0, 1, V - 1, 29999, 5], dtype=torch.int32)
    check(run(ctx, x.cuda(), t, 32), reference(x, t, 32, 1.0))


@pytest.mark.parametrize("type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [19, 4099, 40003])
def test_ranks_among_neighbouring_values(ctx, type, vocab):
    """Tokens of every value of a set of zeros, smallest ones and values next to one another."""
    one = torch.tensor([0.0, 1.0, -1.0, 3.5, -0.25]).to(type)
    near = torch.cat([one, torch.nextafter(one, torch.full_like(one, math.inf)), torch.nextafter(one, torch.full_like(one, -math.inf)),
                      torch.tensor([-0.0, -math.inf, 2.0, -2.0]).to(type)])
    g = torch.Generator().manual_seed(11)
    x = near[torch.randint(0, near.numel(), (2 * near.numel(), vocab), generator=g)]
    t = torch.randint(0, vocab, (2 * near.numel(),), generator=g, dtype=torch.int32)
    x[torch.arange(t.numel()), t.long()] = near.repeat(2)
    check(run(ctx, x.cuda(), t, 5), reference(x, t, 5, 1.0))
    assert ctx.get_error() == 0


def test_masked_and_infinite_logits(ctx):
    """Banned ids, the type's lowest value, rows with fewer ids left than alternatives, rows with none, +inf."""
    V = 9000
    x, t = logits(3, 8, V)
    low = torch.finfo(torch.float32).min
    x[0, 100:] = -math.inf
    x[1, 7:] = -math.inf          # seven ids for twenty places
    x[2, :] = -math.inf
    x[3, 50:] = low
    x[4, :] = low
    x[5, 17] = math.inf
    x[6, [3, 8000]] = math.inf
    x[7, 1:] = -math.inf
    t[:] = torch.tensor([50, 8, 4, 60, 7, 3, 8000, 0])
    check(run(ctx, x.cuda(), t, 20), reference(x, t, 20, 1.0))
    assert ctx.get_error() == 0


def test_nan_counts_as_minus_infinity(sd, ctx):
    x, t = logits(4, 3, 6001)
    x[1, [0, 77, 6000]] = math.nan
    t[1] = 77
    check(run(ctx, x.cuda(), t, 9), reference(x, t, 9, 1.0))
    assert ctx.get_error() == sd.DEV_NAN_LOGITS
    x[1, :] = math.nan
    check(run(ctx, x.cuda(), t, 9), reference(x, t, 9, 1.0))
    assert ctx.get_error() == sd.DEV_NAN_LOGITS


def test_rows_without_a_token_and_tokens_outside(sd, ctx):
    x, t = logits(6, 6, 777)
    t[[1, 4]] = -1
    check(run(ctx, x.cuda(), t, 3), reference(x, t, 3, 1.0))
    assert ctx.get_error() == 0
    for bad in (777, -2, 2 ** 31 - 1):
        t[2] = bad
        at0 = t.clone()
        at0[2] = 0
        check(run(ctx, x.cuda(), t, 3), reference(x, at0, 3, 1.0))
        assert ctx.get_error() == sd.DEV_TOKEN


def test_offsets_past_32_bits(ctx):
    """Rows so far apart that the last one starts past 2^31 values."""
    V, ld = 1003, 1 << 30
    wide = torch.empty(3 * ld, dtype=torch.bfloat16, device="cuda")
    x, t = logits(9, 3, V)
    x = x.bfloat16()
    view = wide.as_strided((3, V), (ld, 1))
    view.copy_(x)
    check(run(ctx, view, t, 4), reference(x, t, 4, 1.0))


def test_outputs_are_optional_and_other_streams_are_followed(ctx):
    x, t = logits(10, 40, 32016)
    ref = reference(x, t, 5, 1.0)
    side = torch.cuda.Stream()
    xd, entropy = x.cuda(), torch.empty(40, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        y = xd * 1.0
        ctx.op_logprobs(y, entropy=entropy)
        got = run(ctx, y, t, 5)
    side.synchronize()
    check(got, ref)
    assert (entropy.cpu().double() - ref["entropy"]).abs().max().item() <= 1e-5
    ids, lp = torch.empty(40, 5, dtype=torch.int32, device="cuda"), torch.empty(40, 5, device="cuda")
    ctx.op_logprobs(xd, top_ids=ids, top_logp=lp)
    assert torch.equal(ids.cpu(), ref["top_ids"])


def test_calls_in_a_row_repeat_their_bits_and_replay_from_a_graph(ctx):
    x, t = logits(11, 48, 32016)
    xd, td = x.cuda(), t.cuda()
    a = run(ctx, xd, t, 10)
    b = run(ctx, xd, t, 10)
    assert all(torch.equal(a[k], b[k]) for k in a)
    lp = torch.zeros(48, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.op_logprobs(xd, td, logp=lp)
    lp.zero_()
    g.replay()
    assert torch.equal(lp.cpu(), a["logp"])


def test_refusals(sd, ctx):
    x, t = logits(12, 2, 100)
    x, t = x.cuda(), t.cuda()
    lp, ids = torch.empty(2, device="cuda"), torch.empty(2, 33, dtype=torch.int32, device="cuda")
    top = torch.empty(2, 33, device="cuda")
    for kw in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf),
               dict(top_ids=ids, top_logp=top), dict(top_ids=ids[:, :5].contiguous())):
        with pytest.raises(sd.SdsatError) as e:
            ctx.op_logprobs(x, t, lp, **kw)
        assert e.value.status == 1
    with pytest.raises(sd.SdsatError):
        ctx.op_logprobs(x, None, lp)                                  # logp of no token
    with pytest.raises(sd.SdsatError):
        ctx.op_logprobs(x[:, :4], t, lp, top_ids=ids[:, :5].contiguous(), top_logp=top[:, :5].contiguous())
    with pytest.raises(sd.SdsatError) as e:
        ctx.op_logprobs(torch.empty(1, 262145, device="cuda"), entropy=lp)
    assert e.value.status == 6
    with pytest.raises(ValueError):
        ctx.op_logprobs(x.t(), t, lp)
    with pytest.raises(ValueError):
        ctx.op_logprobs(x.double(), t, lp)
    ctx.op_logprobs(x[:0], t[:0], lp[:0])                             # no rows: nothing to do
    assert ctx.get_error() == 0
