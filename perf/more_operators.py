"""The measured cases of the operators for ragged batches on a paged cache: new tokens' queries and keys are
normalised and rotated and their rows appended to the pages, every sequence's new tokens attend to what it holds, and
logits are adjusted by penalties, biases and a grammar's mask before a token is selected.

Kinds of cases:

  append     queries, keys and values of the new rows of b sequences: RMS norm of each head (optional), rotation of the
             first `dims` dimensions, keys and values to the sequences' pages of 64 slots
  attention  the new rows of b sequences, each sequence with a number of its own, over their pages
  adjust     repetition, frequency and presence penalties by a token history and the block's drafts, sparse biases,
             a mask of allowed tokens

With `own` false every operator is computed by elementary torch operations in 32 bits (angles in 64); with `own` true
by the library.
"""
import math
from types import SimpleNamespace

import torch

own = False

PAGE = 64          # slots of a page
F32, BF16 = "fp32", "bf16"
TYPES = {F32: torch.float32, BF16: torch.bfloat16}


def listed():
    return [
        # the drafts of two short sequences of a small decoder: launches and latency
        dict(name="tiny append", kind="append", heads=4, kv_heads=4, hd=64, b=2, chunks=2, new=6, ctx=70, dims=64, interleaved=False,
             norm=False, scaling="", type=F32),
        # a step of 64 sequences that decode a token each, four query heads to a cache head
        dict(name="decode append", kind="append", heads=32, kv_heads=8, hd=128, b=64, chunks=0, new=1, ctx=8200, dims=128,
             interleaved=False, norm=True, scaling="", type=BF16),
        # chunks of a dozen long prompts, frequencies scaled by parts
        dict(name="ragged append", kind="append", heads=32, kv_heads=8, hd=128, b=12, chunks=12, new=1100, ctx=30000, dims=128,
             interleaved=False, norm=True, scaling="parts", type=BF16),
        # a whole prompt of the 13B shape in 32 bits, pairs side by side, half of each head rotated
        dict(name="13b append", kind="append", heads=40, kv_heads=40, hd=128, b=1, chunks=1, new=4095, ctx=0, dims=64, interleaved=True,
             norm=False, scaling="linear", type=F32),
        # the drafts of two short sequences of a small decoder
        dict(name="tiny attention", kind="attention", heads=4, kv_heads=4, hd=64, b=2, chunks=2, new=6, ctx=70, type=F32),
        # a whole prompt of the 7B shape
        dict(name="7b prompt 4095", kind="attention", heads=32, kv_heads=32, hd=128, b=1, chunks=1, new=4095, ctx=0, type=BF16),
        # chunks of eight long prompts, four query heads to a cache head
        dict(name="ragged chunks", kind="attention", heads=32, kv_heads=8, hd=128, b=8, chunks=8, new=1100, ctx=16500, type=BF16),
        # most sequences decode a token, two bring the start of a prompt
        dict(name="mixed batch", kind="attention", heads=32, kv_heads=8, hd=128, b=48, chunks=2, new=100, ctx=8200, type=BF16),
        # the next chunk of one prompt, activations in 32 bits (13B heads)
        dict(name="13b chunk in 32 bits", kind="attention", heads=40, kv_heads=40, hd=128, b=1, chunks=1, new=777, ctx=2048, type=F32),
        # a block of a small decoder
        dict(name="tiny adjust", kind="adjust", b=1, q=6, vocab=4104, pad=0, history=100, bias=4, masked=True, type=F32),
        # eight samples of six rows, as the acceptance step sees them
        dict(name="block adjust", kind="adjust", b=8, q=6, vocab=32016, pad=0, history=2300, bias=20, masked=True, type=F32),
        # a large decoding batch with long histories, logits in 16 bits over a vocabulary of odd size
        dict(name="batch adjust", kind="adjust", b=256, q=1, vocab=128003, pad=5, history=9000, bias=100, masked=True, type=BF16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(4, 4, 64), (32, 32, 128), (40, 40, 128), (32, 8, 128), (16, 2, 64), (20, 4, 128), (14, 2, 64)]


def draw(rng):
    kind = rng.choice(["append", "append", "attention", "attention", "attention", "adjust", "adjust"])
    t = rng.choice([F32, BF16, BF16])
    if kind == "adjust":
        vocab = _log(rng, 1000, 200000)
        q = rng.choice([1, 1, 2, 6, 7, 16])
        b = _log(rng, 1, max(1, min(256, 256 * 128003 // (2 * vocab)) // q))
        return dict(kind=kind, b=b, q=q, vocab=vocab, pad=rng.choice([0, 0, 1, 8]), history=_log(rng, 1, 9000),
                    bias=rng.choice([0, 1, 10, 100, 300]), masked=rng.choice([True, True, False]), type=t)
    most = {"append": work(listed()[3])["bytes"], "attention": work(listed()[6])["flops"]}[kind]
    while True:
        heads, kv_heads, hd = rng.choice(HEADS)
        b = _log(rng, 1, 64)
        chunks = rng.choice([b, b, min(b, 2), 0])
        case = dict(kind=kind, heads=heads, kv_heads=kv_heads, hd=hd, b=b, chunks=chunks, new=_log(rng, 1, 4095) if chunks else 1,
                    ctx=_log(rng, 1, 16500), type=t)
        if kind == "append":
            case.update(dims=rng.choice([hd, hd, hd // 2, hd // 4, 20]), interleaved=rng.choice([False, False, True]),
                        norm=rng.choice([True, False]), scaling=rng.choice(["", "linear", "parts"]))
            if work(case)["bytes"] <= most:
                return case
        # (what the plain form holds is padded to the longest of the batch)
        elif work(case)["flops"] <= most and b * heads * case["new"] * (case["ctx"] + case["new"]) <= 6e9 and (
                b * kv_heads * hd * (case["ctx"] + case["new"]) <= 6e8):
            return case


# ---- inputs --------------------------------------------------------------------------------------


def _gen(seed, stream=0):
    return torch.Generator(device="cuda").manual_seed(seed * 1000003 + stream)


def _spread(i, k):
    return (0.37 + 0.6180339887 * i + 0.29 * k) % 1.0


def _batch(case):
    """Every sequence's new rows and committed slots (given by the case alone)."""
    b = case["b"]
    new = [(case["new"] if b == 1 else max(1, int(case["new"] * (0.3 + 0.7 * _spread(s, 0))))) if s < case["chunks"] else 1 for s in range(b)]
    ctx = [case["ctx"] if b == 1 else int(case["ctx"] * (0.05 + 0.95 * _spread(s, 1))) for s in range(b)]
    return new, ctx


SCALING = {"": {}, "linear": dict(scaling="linear", factor=4.0),
           "parts": dict(scaling="parts", factor=8.0, low=1.0, high=4.0, original=8192, magnitude=1.2)}
THETA, MAX_POSITION, EPS = 1e4, 32768, 1e-5
_handles = {}


def _context():
    """The library's context: a program keeps one for its lifetime."""
    if "ctx" not in _handles:
        import paper_2403_18647_gb300 as sd
        shape = SimpleNamespace(n_layers=1, d_model=5120, n_heads=40, head_dim=128, ffn_dim=688, vocab=4104, rms_eps=1e-5,
                                rope_theta=1e4, adaptive_id=4096)
        _handles["ctx"] = sd.Context(shape, None, max_position=4096)
    return _handles["ctx"]


def _rope(case):
    """The rotation of a model: made once, like its weights."""
    key = (case["dims"], case["interleaved"], case["scaling"])
    if key not in _handles:
        _handles[key] = _context().rope(case["dims"], MAX_POSITION, theta=THETA, interleaved=case["interleaved"], **SCALING[case["scaling"]])
    return _handles[key]


def _pages_state(case, g):
    """Pages of a ragged batch, handed out in any order."""
    new, ctx = _batch(case)
    need = [-(-(n + m) // PAGE) for n, m in zip(new, ctx)]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=g, device="cuda", dtype=torch.int32)
    table = torch.full((case["b"], max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    whole = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pool = lambda: torch.empty(pages, case["kv_heads"], PAGE, case["hd"], dtype=torch.bfloat16, device="cuda").normal_(generator=g)  # noqa: E731
    return dict(table=table, lens=whole(ctx), starts=whole(starts), rows=starts[-1], longest=max(new), k_pages=pool(), v_pages=pool())


def _append_state(case, seed):
    g = _gen(seed)
    s = _pages_state(case, g)
    H, Hk, hd, t = case["heads"], case["kv_heads"], case["hd"], TYPES[case["type"]]
    # queries, keys and values side by side, as one projection leaves them
    qkv = (torch.randn(s["rows"], (H + 2 * Hk) * hd, generator=g, device="cuda") * 1.5).to(t)
    s.update(q=qkv[:, :H * hd], k=qkv[:, H * hd:(H + Hk) * hd], v=qkv[:, (H + Hk) * hd:])
    s["q_out"] = torch.empty(s["rows"], H * hd, dtype=t, device="cuda")
    gain = lambda: (1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).bfloat16() if case["norm"] else None  # noqa: E731
    s.update(q_gain=gain(), k_gain=gain())
    return s


def _attention_state(case, seed):
    g = _gen(seed)
    s = _pages_state(case, g)
    x = torch.randn(s["rows"], case["heads"] * case["hd"], generator=g, device="cuda") * 1.5
    s["q"] = x.to(TYPES[case["type"]])
    s["out"] = torch.empty_like(s["q"])
    return s


def _adjust_state(case, seed):
    g = _gen(seed)
    b, q, V, n, m = case["b"], case["q"], case["vocab"], case["history"], case["bias"]
    rows = b * q
    u = lambda *shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
    x = (torch.randn(rows, V + case["pad"], generator=g, device="cuda") * 3).to(TYPES[case["type"]])
    often = lambda *shape: (u(*shape) ** 3 * V).int().clamp_(max=V - 1)  # noqa: E731   (few tokens make most of a text)
    lens = (n * (0.4 + 0.6 * u(b))).int().clamp_(min=1)
    s = dict(logits=x[:, :V], out=torch.empty(rows, V, dtype=x.dtype, device="cuda"), history=often(b, n), history_lens=lens,
             prompt_lens=(lens * u(b)).int(), tokens=often(rows), repetition=1 + 0.3 * u(b), frequency=0.5 * u(b), presence=u(b) - 0.3,
             bias_ids=None, bias=None, allowed=None)
    s["history"][torch.arange(n, device="cuda") >= lens[:, None]] = -1
    if m:
        first = torch.randint(0, V, (b, 1), generator=g, device="cuda")
        s["bias_ids"] = ((first + torch.arange(m, device="cuda") * (V // m)) % V).int()
        s["bias"] = torch.randn(b, m, generator=g, device="cuda") * 4
    if case["masked"]:
        # after some rows most tokens are allowed, after others one in sixteen
        words = torch.randint(-2 ** 31, 2 ** 31, (4, rows, -(-V // 32)), generator=g, device="cuda", dtype=torch.int64).int()
        many, few = words[0] | words[1] | words[2], words[0] & words[1] & words[2] & words[3]
        s["allowed"] = torch.where(u(rows, 1) < 0.5, many, few).contiguous()
    return s


STATES = {"append": _append_state, "attention": _attention_state, "adjust": _adjust_state}


def prepare(case, seed):
    s = STATES[case["kind"]](case, seed)
    s["case"] = case
    if own:
        s["ctx"] = _context()
        if case["kind"] == "append":
            s["rope"] = _rope(case)
    return s


# ---- the plain forms -------------------------------------------------------------------------------


def _rows_of(s):
    """(sequence, place among its new rows) of every row."""
    at = torch.arange(s["rows"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["starts"], at, right=True) - 1
    return seq, at - s["starts"][seq]


def _frequencies(case):
    """Radians a position, in 64 bits."""
    sc, dims = SCALING[case["scaling"]], case["dims"]
    f = THETA ** (-2 * torch.arange(dims // 2, dtype=torch.float64, device="cuda") / dims)
    if sc.get("scaling") == "linear":
        f = f / sc["factor"]
    if sc.get("scaling") == "parts":
        turns = sc["original"] * f / (2 * math.pi)
        keep = ((turns - sc["low"]) / (sc["high"] - sc["low"])).clamp(0, 1)
        f = f / sc["factor"] * (1 - keep) + f * keep
    return f, sc.get("magnitude", 1.0)


def _plain_append(s):
    c = s["case"]
    hd, dims, rows = c["hd"], c["dims"], s["rows"]
    seq, at = _rows_of(s)
    slot = s["lens"][seq] + at
    f, magnitude = _frequencies(c)
    angle = slot.double()[:, None] * f
    cos, sin = (angle.cos() * magnitude).float()[:, None], (angle.sin() * magnitude).float()[:, None]

    def turned(x, gain):
        x = x.float().view(rows, -1, hd)
        if gain is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
        pairs = x[..., :dims]
        pairs = pairs.unflatten(-1, (dims // 2, 2)) if c["interleaved"] else pairs.unflatten(-1, (2, dims // 2)).transpose(-1, -2)
        a, z = pairs[..., 0], pairs[..., 1]
        pairs = torch.stack((a * cos - z * sin, a * sin + z * cos), -1)
        pairs = pairs.flatten(-2) if c["interleaved"] else pairs.transpose(-1, -2).flatten(-2)
        return torch.cat((pairs, x[..., dims:]), -1)

    page, off = s["table"][seq, (slot // PAGE).long()].long()[:, None], (slot % PAGE).long()[:, None]
    head = torch.arange(c["kv_heads"], device="cuda")
    s["k_pages"][page, head, off] = turned(s["k"], s["k_gain"]).bfloat16()
    s["v_pages"][page, head, off] = s["v"].reshape(rows, -1, hd).bfloat16()
    return dict(q=turned(s["q"], s["q_gain"]).to(s["q"].dtype).view(rows, -1), k_pages=s["k_pages"], v_pages=s["v_pages"])


def _plain_attention(s):
    c = s["case"]
    b, H, Hk, hd = c["b"], c["heads"], c["kv_heads"], c["hd"]
    G, m = H // Hk, s["longest"]
    table = s["table"].long().clamp(min=0)
    n = table.shape[1] * PAGE
    k = s["k_pages"][table].permute(0, 2, 1, 3, 4).reshape(b, Hk, n, hd).float()
    v = s["v_pages"][table].permute(0, 2, 1, 3, 4).reshape(b, Hk, n, hd).float()
    local = torch.arange(m, device="cuda")
    row = (s["starts"][:-1, None] + local).clamp(max=s["rows"] - 1).long()          # sequences padded to the longest
    x = s["q"][row].float().view(b, m, Hk, G, hd).permute(0, 2, 1, 3, 4).reshape(b, Hk, m * G, hd)
    p = torch.matmul(x, k.transpose(2, 3)).mul_(1 / math.sqrt(hd)).view(b, Hk, m, G, n)
    last = s["lens"].long()[:, None] + local                                        # the last slot that a row sees
    hidden = torch.arange(n, device="cuda") > last[:, None, :, None, None]
    p = p.masked_fill_(hidden, -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1).view(b, Hk, m * G, 1)
    o = torch.matmul(p.view(b, Hk, m * G, n), v) / total
    o = o.view(b, Hk, m, G, hd).permute(0, 2, 1, 3, 4).reshape(b, m, H * hd)
    seq, at = _rows_of(s)
    return o[seq, at.long()].to(s["q"].dtype)


def _plain_adjust(s):
    c = s["case"]
    b, q, V = c["b"], c["q"], c["vocab"]
    rows = b * q
    each = lambda t: t.repeat_interleave(q, 0, output_size=rows)  # noqa: E731
    x = s["logits"].float()
    history = s["history"].long()
    place = torch.arange(history.shape[1], device="cuda")
    held = place < s["history_lens"][:, None]
    seen = torch.zeros(b, V + 1, device="cuda")                                     # (column V: nothing)
    ones = torch.ones((), device="cuda").expand(history.shape)
    seen.scatter_add_(1, torch.where(held, history, V), ones)
    made = torch.zeros(b, V + 1, device="cuda")
    made.scatter_add_(1, torch.where(held & (place >= s["prompt_lens"][:, None]), history, V), ones)
    # row j of a sequence comes after the block's tokens 0 .. j
    block = s["tokens"].long().view(b, 1, q).expand(b, q, q)
    block = torch.where(torch.ones(q, q, dtype=torch.bool, device="cuda").tril(), block, V).reshape(rows, q)
    made = each(made).scatter_add_(1, block, torch.ones((), device="cuda").expand(rows, q))[:, :V]
    seen = (each(seen)[:, :V] > 0) | (made > 0)
    r = each(s["repetition"])[:, None]
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - each(s["frequency"])[:, None] * made - each(s["presence"])[:, None] * (made > 0)
    if s["bias"] is not None:
        x = x.scatter_add(1, each(s["bias_ids"].long()), each(s["bias"]))
    if s["allowed"] is not None:
        ids = torch.arange(V, device="cuda")
        x = x.masked_fill(((s["allowed"][:, ids // 32] >> (ids % 32).int()) & 1) == 0, -math.inf)
    return x.to(s["logits"].dtype)


# ---- one pass ------------------------------------------------------------------------------------------


def run(s):
    c = s["case"]
    if c["kind"] == "append":
        if not own:
            return _plain_append(s)
        s["ctx"].op_rotary_append(s["rope"], s["q"], s["k"], s["v"], s["q_out"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["starts"],
                                  c["heads"], c["kv_heads"], c["hd"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS)
        return dict(q=s["q_out"], k_pages=s["k_pages"], v_pages=s["v_pages"])
    if c["kind"] == "attention":
        if not own:
            return _plain_attention(s)
        s["ctx"].op_chunk_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["starts"], c["heads"], c["kv_heads"],
                                    c["hd"], s["out"])
        return s["out"]
    if not own:
        return _plain_adjust(s)
    s["ctx"].op_adjust_logits(s["logits"], s["out"], c["q"], history=s["history"], history_lens=s["history_lens"],
                              prompt_lens=s["prompt_lens"], tokens=s["tokens"], repetition=s["repetition"], frequency=s["frequency"],
                              presence=s["presence"], bias_ids=s["bias_ids"], bias=s["bias"], allowed=s["allowed"])
    return s["out"]


# ---- what a pass cannot do without ------------------------------------------------------------------


def work(case):
    size = TYPES[case["type"]].itemsize
    if case["kind"] == "adjust":
        rows, V = case["b"] * case["q"], case["vocab"]
        return dict(bytes=2 * rows * V * size + (rows * V // 8 if case["masked"] else 0) + case["b"] * (4 * case["history"] * 7 // 10 + 8 * case["bias"]),
                    flops=6 * rows * V)
    H, Hk, hd = case["heads"], case["kv_heads"], case["hd"]
    new, ctx = _batch(case)
    rows = sum(new)
    if case["kind"] == "append":
        # rows read and written once, a position's cosines and sines read once
        return dict(bytes=rows * hd * (size * (2 * H + 2 * Hk) + 4 * Hk) + 4 * case["dims"] * rows, flops=rows * hd * 8 * (H + Hk))
    pairs = sum(n * m + n * (n + 1) // 2 for n, m in zip(new, ctx))
    return dict(bytes=4 * Hk * hd * sum(n + m for n, m in zip(new, ctx)) + 2 * size * rows * H * hd, flops=4 * H * hd * pairs)


# ---- 64 bits -------------------------------------------------------------------------------------------


def _exact_append(case, seed):
    s = _append_state(case, seed)
    hd, dims, half = case["hd"], case["dims"], case["dims"] // 2
    new, ctx = _batch(case)
    f = [THETA ** (-2 * i / dims) for i in range(half)]
    sc = SCALING[case["scaling"]]
    for i in range(half):
        keep = 0.0
        if sc.get("scaling") == "parts":
            keep = min(1.0, max(0.0, (sc["original"] * f[i] / (2 * math.pi) - sc["low"]) / (sc["high"] - sc["low"])))
        f[i] = f[i] * (keep + (1 - keep) / sc.get("factor", 1.0))
    first = [2 * i if case["interleaved"] else i for i in range(half)]
    second = [2 * i + 1 if case["interleaved"] else i + half for i in range(half)]
    whole = torch.tensor(f, dtype=torch.float64, device="cuda")
    out = {"q": torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), "k_pages": s["k_pages"].double(), "v_pages": s["v_pages"].double()}
    at = 0
    for i, (n, m) in enumerate(zip(new, ctx)):
        place = torch.arange(m, m + n, device="cuda")
        turn = torch.polar(torch.full((), sc.get("magnitude", 1.0), dtype=torch.float64, device="cuda").expand(n, half), place[:, None] * whole)
        for name, gain in (("q", s["q_gain"]), ("k", s["k_gain"]), ("v", None)):
            x = s[name][at:at + n].double().reshape(n, -1, hd)
            if gain is not None:
                x = x / (x.square().sum(-1, keepdim=True) / hd + EPS).sqrt() * gain.double()
            if name != "v":
                y = torch.complex(x[..., first], x[..., second]) * turn[:, None]
                x = x.clone()
                x[..., first], x[..., second] = y.real, y.imag
            if name == "q":
                out["q"][at:at + n] = x.flatten(1)
            else:
                page = s["table"][i].long()[place // PAGE]
                for h in range(case["kv_heads"]):
                    out[name + "_pages"][page, h, place % PAGE] = x[:, h]
        at += n
    return out


def _exact_attention(case, seed):
    s = _attention_state(case, seed)
    H, Hk, hd = case["heads"], case["kv_heads"], case["hd"]
    new, ctx = _batch(case)
    if sum(n * (n + m) for n, m in zip(new, ctx)) * H * hd > 6e11:
        return None
    out = torch.empty(s["rows"], H, hd, dtype=torch.float64, device="cuda")
    at = 0
    for i, (n, m) in enumerate(zip(new, ctx)):
        x = s["q"][at:at + n].double().view(n, H, hd)
        pages = s["table"][i, :-(-(n + m) // PAGE)].long()
        seen = torch.ones(n, n + m, dtype=torch.bool, device="cuda").tril(m)
        for h in range(Hk):
            k = s["k_pages"][pages, h].reshape(-1, hd)[:n + m].double()
            v = s["v_pages"][pages, h].reshape(-1, hd)[:n + m].double()
            for g in range(h * (H // Hk), (h + 1) * (H // Hk)):
                out[at:at + n, g] = (x[:, g] @ k.t() / math.sqrt(hd)).masked_fill(~seen, -math.inf).softmax(-1) @ v
        at += n
    return out.view(s["rows"], H * hd)


def _exact_adjust(case, seed):
    """Row by row on the host's numbers, only the entries that a rule names touched."""
    s = _adjust_state(case, seed)
    V, q = case["vocab"], case["q"]
    out = s["logits"].double()
    host = {n: s[n].tolist() for n in ("history", "history_lens", "prompt_lens", "tokens")}
    rule = {n: s[n].double().tolist() for n in ("repetition", "frequency", "presence")}
    bit = torch.arange(32, device="cuda", dtype=torch.int32)
    for r in range(case["b"] * q):
        i, j = divmod(r, q)
        text = host["history"][i][:host["history_lens"][i]]
        made = {}
        for t in text[host["prompt_lens"][i]:] + host["tokens"][i * q:r + 1]:
            made[t] = made.get(t, 0) + 1
        ids = sorted(set(text) | set(made))
        c = torch.tensor([made.get(t, 0) for t in ids], dtype=torch.float64, device="cuda")
        at = torch.tensor(ids, device="cuda")
        x = out[r, at]
        x = torch.where(x > 0, x / rule["repetition"][i], x * rule["repetition"][i])
        out[r, at] = x - rule["frequency"][i] * c - rule["presence"][i] * c.clamp(max=1)
        if s["bias"] is not None:
            out[r].index_add_(0, s["bias_ids"][i].long(), s["bias"][i].double())
        if s["allowed"] is not None:
            out[r][((s["allowed"][r][:, None] >> bit) & 1).flatten()[:V] == 0] = -math.inf
    return out


EXACT = {"append": _exact_append, "attention": _exact_attention, "adjust": _exact_adjust}


def exact(case, seed):
    return EXACT[case["kind"]](case, seed)
