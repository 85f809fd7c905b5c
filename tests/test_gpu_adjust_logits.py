"""Penalties, biases and masks of logits.  Every step is one fp32 operation that is rounded to nearest, so results are those
of the same steps on the host, bit for bit (bf16: rounded once more)."""
import math

import pytest
import torch

import synth
from ragged import generator, ints

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def sd():
    import paper_2403_18647_gb300 as sd
    return sd


@pytest.fixture(scope="module")
def ctx(sd):
    return sd.Context(synth.SHAPES["tiny"], None, max_position=64)


def make(seed, b, q, V, type, history=200, bias=10, masked=True, tokens=True, anc=False, pad=0):
    g = generator(seed)
    rows = b * q
    u = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    a = dict(logits=(torch.randn(rows, V + pad, generator=g, device="cuda") * 4).to(type)[:, :V], q=q)
    often = lambda *s: (u(*s) ** 4 * V).int().clamp_(max=V - 1)  # noqa: E731
    if history:
        a.update(history=often(b, history), history_lens=(u(b) * (history + 1)).int())
        a["prompt_lens"] = (a["history_lens"] * u(b) * 1.2).int()
    if tokens:
        a["tokens"] = often(rows)
    if anc:
        a["anc"] = torch.randint(0, 1 << q, (rows,), generator=g, device="cuda").int()
    a.update(repetition=0.7 + u(b), frequency=u(b) - 0.3, presence=u(b) - 0.5)
    if bias:
        a.update(bias_ids=often(b, bias), bias=torch.randn(b, bias, generator=g, device="cuda"))
    if masked:
        a["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (rows, -(-V // 32) + 1), generator=g, device="cuda", dtype=torch.int64).int()
    return a


def reference(a):
    """The rules one entry at a time, in fp32 on the host."""
    x = a["logits"].float().cpu()
    rows, V = x.shape
    q = a["q"]
    get = lambda n: a[n].cpu() if a.get(n) is not None else None  # noqa: E731
    history, lens, prompt, tokens, anc = (get(n) for n in ("history", "history_lens", "prompt_lens", "tokens", "anc"))
    bias_ids, bias, allowed = get("bias_ids"), get("bias"), get("allowed")
    one = lambda n, s, d: get(n)[s] if get(n) is not None else torch.tensor(d)  # noqa: E731
    for r in range(rows):
        s, j = divmod(r, q)
        made, seen = {}, set()
        if history is not None:
            n = min(max(int(lens[s]), 0), history.shape[1])
            for i, t in enumerate(history[s, :n].tolist()):
                if 0 <= t < V:
                    seen.add(t)
                    if prompt is None or i >= int(prompt[s]):
                        made[t] = made.get(t, 0) + 1
        if tokens is not None:
            for i in range(q):
                if (int(anc[r]) >> i & 1) if anc is not None else i <= j:
                    t = int(tokens[s * q + i])
                    if 0 <= t < V:
                        seen.add(t)
                        made[t] = made.get(t, 0) + 1
        at = torch.tensor(sorted(seen), dtype=torch.long)
        if at.numel():
            rep, freq, pres = one("repetition", s, 1.0), one("frequency", s, 0.0), one("presence", s, 0.0)
            l = x[r, at]
            l = torch.where(l > 0, l / rep, l * rep)
            c = torch.tensor([float(made.get(t, 0)) for t in at.tolist()])
            x[r, at] = torch.where(c > 0, (l - freq * c) - pres, l)
        if bias is not None:
            first = {}
            for t, v in zip(bias_ids[s].tolist(), bias[s]):
                if 0 <= t < V:
                    first.setdefault(t, v)
            for t, v in first.items():
                x[r, t] = x[r, t] + v
        if allowed is not None:
            bits = (allowed[r][:, None] >> torch.arange(32)) & 1
            x[r][bits.flatten()[:V] == 0] = -math.inf
    return x.to(a["logits"].dtype)


def same(x, y):
    return torch.equal(x.cpu().nan_to_num(nan=1e30), y.nan_to_num(nan=1e30)) and torch.equal(x.cpu().isnan(), y.isnan())


def run(ctx, a, out=None):
    out = torch.full(a["logits"].shape, math.nan, dtype=a["logits"].dtype, device="cuda") if out is None else out
    ctx.op_adjust_logits(out=out, **a)
    return out


SIZES = [(1, 1, 1), (1, 1, 31), (2, 1, 32), (1, 6, 33), (3, 2, 100), (1, 16, 4104), (8, 6, 2049), (64, 1, 1000), (2, 7, 32016), (1, 1, 128003),
         (5, 3, 16384), (2, 2, 16391), (300, 1, 5000), (40, 6, 20000)]


@pytest.mark.parametrize("b,q,V", SIZES)
@pytest.mark.parametrize("type", [F32, BF16])
def test_sizes(sd, ctx, b, q, V, type):
    a = make(b + q + V, b, q, V, type)
    assert same(run(ctx, a), reference(a))
    assert ctx.get_error() == 0


@pytest.mark.parametrize("type", [F32, BF16])
@pytest.mark.parametrize("without", ["history", "tokens", "bias", "allowed", "rules", "prompt_lens", "all"])
def test_parts_may_be_missing(ctx, type, without):
    a = make(1, 4, 3, 3001, type)
    gone = {"history": ["history", "history_lens", "prompt_lens"], "bias": ["bias", "bias_ids"], "rules": ["repetition", "frequency", "presence"],
            "all": [n for n in a if n not in ("logits", "q")]}.get(without, [without])
    for n in gone:
        a[n] = None
    out = run(ctx, a)
    assert same(out, reference(a))
    if without == "all":
        assert torch.equal(out, a["logits"])


@pytest.mark.parametrize("type", [F32, BF16])
def test_rows_of_a_tree(ctx, type):
    for q, V in ((5, 777), (16, 4104), (7, 40000)):
        a = make(q, 3, q, V, type, anc=True)
        assert same(run(ctx, a), reference(a))


@pytest.mark.parametrize("type", [F32, BF16])
def test_every_alignment(ctx, type):
    """Input and output rows at every offset from 16 bytes, what lies beside them untouched."""
    V, rows = 333, 3
    for i in range(0, 9):
        for o in range(0, 9):
            a = make(10 * i + o, rows, 1, V, type, history=40)
            wide = torch.full((rows, V + 11), 5.0, dtype=type, device="cuda")
            wide[:, i:i + V] = a["logits"]
            a["logits"] = wide[:, i:i + V]
            hold = torch.full((rows, V + 13), 7.0, dtype=type, device="cuda")
            run(ctx, a, hold[:, o:o + V])
            assert same(hold[:, o:o + V].contiguous(), reference(a))
            assert (hold[:, :o] == 7).all() and (hold[:, o + V:] == 7).all()


@pytest.mark.parametrize("type", [F32, BF16])
@pytest.mark.parametrize("b,q,V,pad", [(2, 6, 32016, 0), (1, 1, 4104, 3), (70, 1, 9001, 1)])
def test_in_place(ctx, type, b, q, V, pad):
    a = make(3, b, q, V, type, pad=pad)
    ref = reference(a)
    run(ctx, a, a["logits"])
    assert same(a["logits"], ref)


@pytest.mark.parametrize("type", [F32, BF16])
@pytest.mark.parametrize("b,q,V", [(320, 4, 700), (320, 16, 300), (2, 16, 300), (700, 16, 64)])
def test_trees_in_place(ctx, type, b, q, V):
    """A token that is on several branches, but not on the one between them, counts once in each row."""
    a = make(14, b, q, V, type, anc=True)
    ref = reference(a)
    run(ctx, a, a["logits"])
    assert same(a["logits"], ref) and ctx.get_error() == 0


@pytest.mark.parametrize("type", [F32, BF16])
def test_infinities_nan_and_rows_without_a_token(ctx, type):
    a = make(4, 4, 2, 1000, type)
    x = a["logits"]
    x[0, ::3], x[1, ::2], x[2, 5::7], x[3] = -math.inf, math.inf, math.nan, -math.inf
    a["allowed"][4] = 0
    a["allowed"][5] = -1
    out = run(ctx, a)
    assert same(out, reference(a))
    assert (out[4] == -math.inf).all()


def test_ids_that_are_no_tokens(sd, ctx):
    a = make(5, 3, 4, 500, F32)
    for n in ("history", "tokens", "bias_ids"):
        a[n].view(-1)[::3] = -1
        a[n].view(-1)[::7] = -2 ** 31
    assert same(run(ctx, a), reference(a)) and ctx.get_error() == 0
    for n, at in (("history", (1, 0)), ("tokens", (3,)), ("bias_ids", (2, 1))):
        c = {k: t.clone() if torch.is_tensor(t) else t for k, t in a.items()}
        c["history_lens"][:] = 200
        for far in (500, 2 ** 31 - 1):
            c[n][at] = far
            assert same(run(ctx, c), reference(c)) and ctx.get_error() == sd.DEV_TOKEN


def test_lengths_outside_the_history(ctx):
    a = make(6, 4, 1, 500, F32, history=37)
    a["history_lens"] = ints([-1, 38, 2 ** 31 - 1, 0])
    a["prompt_lens"] = ints([5, -3, 2 ** 31 - 1, 2])
    assert same(run(ctx, a), reference(a)) and ctx.get_error() == 0


@pytest.mark.parametrize("type", [F32, BF16])
def test_long_histories_of_few_tokens(ctx, type):
    """A count above what 16 bits hold, the most biases, the same ones again."""
    b, V = 2, 300
    a = make(7, b, 1, V, type, history=100000, bias=1024)
    a["history"][0] = 17
    a["history_lens"][:] = ints([100000, 99999])
    a["prompt_lens"][:] = 3
    a["frequency"][:] = 1e-4
    assert same(run(ctx, a), reference(a)) and ctx.get_error() == 0


def test_streams_and_graphs(ctx):
    a = make(8, 8, 6, 32016, F32)
    out = run(ctx, a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run(ctx, a)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, again)
    hold = torch.zeros_like(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(ctx, a, hold)
    graph.replay()
    assert torch.equal(hold, out)
    c = make(9, 8, 6, 32016, F32)
    for n, t in a.items():
        if torch.is_tensor(t):
            t.copy_(c[n])
    graph.replay()
    assert torch.equal(hold, run(ctx, c)) and ctx.get_error() == 0


WRONG = {
    "logits": [lambda t: t.half(), lambda t: t.bfloat16(), lambda t: t[:5], lambda t: t.cpu(), lambda t: t[0]],
    "out": [lambda t: t.bfloat16(), lambda t: t[:5], lambda t: t[:, :99], lambda t: t.cpu()],
    "history": [lambda t: t.long(), lambda t: t[:1], lambda t: t.cpu()], "history_lens": [lambda t: t.long(), lambda t: t[:1]],
    "prompt_lens": [lambda t: t.long(), lambda t: t[:1]], "tokens": [lambda t: t.long(), lambda t: t[:5]], "anc": [lambda t: t.long(), lambda t: t[:5]],
    "repetition": [lambda t: t.double(), lambda t: t[:1]], "frequency": [lambda t: t.double(), lambda t: t[:1]], "presence": [lambda t: t.bfloat16(), lambda t: t[:1]],
    "bias_ids": [lambda t: t.long(), lambda t: t[:1], lambda t: t[:, :3].contiguous(), lambda t: None],
    "bias": [lambda t: t.double(), lambda t: t[:1], lambda t: t[:, :3].contiguous(), lambda t: None],
    "allowed": [lambda t: t.long(), lambda t: t[:5], lambda t: t[:, :3].contiguous()], "q": [lambda q: 0, lambda q: 4, lambda q: -3],
}


@pytest.mark.parametrize("name", WRONG)
def test_wrong_tensors_are_refused(ctx, name):
    a = make(11, 2, 3, 100, F32, anc=True)
    a["out"] = torch.full((6, 100), 7.0, device="cuda")
    for wrong in WRONG[name]:
        with pytest.raises(ValueError):
            ctx.op_adjust_logits(**{**a, name: wrong(a[name])})
    assert (a["out"] == 7).all() and ctx.get_error() == 0


def test_wrong_sizes_are_refused(sd, ctx):
    def refused(status, **a):
        with pytest.raises(sd.SdsatError) as e:
            ctx.op_adjust_logits(**a)
        assert e.value.status == status

    x = torch.zeros(34, 100, device="cuda")
    refused(1, logits=x, out=x.clone(), q=17)
    refused(1, logits=x, out=x.clone(), history=torch.zeros(34, 5, dtype=torch.int32, device="cuda"))
    refused(6, logits=x[:1], out=x[:1].clone(), bias_ids=torch.zeros(1, 1025, dtype=torch.int32, device="cuda"), bias=torch.zeros(1, 1025, device="cuda"))
    refused(6, logits=x[:1], out=x[:1].clone(), history=torch.zeros(1, 1 << 19, dtype=torch.int32, device="cuda"), history_lens=ints([1]))
    wide = torch.zeros(1, (1 << 20) + 1, device="cuda")
    refused(6, logits=wide, out=wide.clone())
    ctx.op_adjust_logits(x[:0], x[:0])
    a = make(12, 1, 1, 1 << 20, F32)                    # the widest there is
    assert same(run(ctx, a), reference(a)) and ctx.get_error() == 0


def test_offsets_past_32_bits(ctx):
    """More than 2^31 logits: the last rows are reached."""
    b, V = 2150, 1000003
    x = torch.zeros(b, V, dtype=BF16, device="cuda")
    a = make(13, 2, 1, V, BF16)
    x[-2:] = a["logits"]
    ids = torch.full((b, 10), -1, dtype=torch.int32, device="cuda")
    ids[-2:] = a["bias_ids"]
    bias = torch.zeros(b, 10, device="cuda")
    bias[-2:] = a["bias"]
    ctx.op_adjust_logits(x, x, bias_ids=ids, bias=bias)
    for n in list(a):
        if n not in ("logits", "q", "bias_ids", "bias"):
            a[n] = None
    assert same(x[-2:], reference(a)) and (x[:-2] == 0).all()
    assert ctx.get_error() == 0


def test_rows_over_one_anothers_are_refused(sd, ctx):
    hold = torch.zeros(12, 100, device="cuda")
    with pytest.raises(sd.SdsatError) as e:
        ctx.op_adjust_logits(hold[::2], hold[:6])
    assert e.value.status == 1
    ctx.op_adjust_logits(hold[::2], hold[::2])
    assert ctx.get_error() == 0
