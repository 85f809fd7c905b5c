"""The measured cases of the operators for many samples of one prompt: a paged KV cache whose
sequences share the prompt's pages, block attention that reads the shared pages once for all of
them, and the log probabilities that rank the samples.

Kinds of cases:

  attention  block-causal attention of b sequences of q rows over pages of 64 slots, the leading
             pages of the page table the same for every sequence
  branch     b sequences become copies of a parked prompt and get room for their next block: pages
             are shared, the prompt's partly filled page is copied for each
  round      a whole round of sampling on the cache: branch, grow by n slots, keep one sequence,
             pack the pages that are left at the front of the pool
  logprobs   log probability and rank of given tokens, entropy and the n best alternatives of
             rows of logits

With `own` false every operator is computed by elementary torch operations in 32 bits; with `own`
true by the library.
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
        # a small decoder drafting for two samples of a short prompt: launches and latency
        dict(name="tiny 2x6 after 64", kind="attention", heads=4, kv_heads=4, hd=64, b=2, q=6, prompt=64, grown=20, type=F32),
        # eight samples of a 2048-token prompt, 5 drafts each, some way into their answers (7B heads)
        dict(name="7b 8x6 after 2048", kind="attention", heads=32, kv_heads=32, hd=128, b=8, q=6, prompt=2048, grown=256, type=F32),
        # the largest block for four samples, 13B heads, a prompt that ends inside a page
        dict(name="13b 4x16 after 4095", kind="attention", heads=40, kv_heads=40, hd=128, b=4, q=16, prompt=4095, grown=100, type=F32),
        # many samples of a long document
        dict(name="7b 16x4 after 16500", kind="attention", heads=32, kv_heads=32, hd=128, b=16, q=4, prompt=16500, grown=500, type=F32),
        # plain decoding of 64 samples with four query heads to a cache head, activations in 16 bits
        dict(name="grouped 64x1 after 8200", kind="attention", heads=32, kv_heads=8, hd=128, b=64, q=1, prompt=8200, grown=300, type=BF16),
        # the cache of a small decoder branches into four samples
        dict(name="tiny branch", kind="branch", layers=2, heads=4, hd=64, b=4, prompt=100, n=6, pages=24),
        # the whole 7B-shaped cache branches into eight samples; 61 slots of the last page are filled
        dict(name="7b branch", kind="branch", layers=32, heads=32, hd=128, b=8, prompt=2045, n=6, pages=60),
        # a round of ten samples of up to 200 tokens on the 13B-shaped cache
        dict(name="13b round", kind="round", layers=40, heads=40, hd=128, b=10, prompt=1130, n=200, pages=90),
        # one block of a small decoder, five alternatives
        dict(name="tiny logprobs", kind="logprobs", rows=6, vocab=4104, pad=0, top=5, temperature=1.0, type=F32),
        # eight samples of six rows, as the acceptance step sees them
        dict(name="block logprobs", kind="logprobs", rows=48, vocab=32016, pad=0, top=10, temperature=0.8, type=F32),
        # scoring a batch of answers, the chosen token and its best rival
        dict(name="scoring", kind="logprobs", rows=4096, vocab=32016, pad=0, top=2, temperature=1.0, type=F32),
        # logits in 16 bits over a larger vocabulary of odd size, twenty alternatives
        dict(name="16 bits, odd vocabulary", kind="logprobs", rows=1000, vocab=128003, pad=0, top=20, temperature=1.0, type=BF16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "logprobs", "logprobs", "branch", "round"])
    if kind == "attention":
        heads, kv_heads, hd = rng.choice([(4, 4, 64), (32, 32, 128), (40, 40, 128), (32, 8, 128), (16, 2, 64), (20, 20, 64)])
        q = _log(rng, 1, 16)
        b = _log(rng, 1, 64 // q)
        grown = _log(rng, 1, 600)
        most = 17000 * 32 * 128 // (kv_heads * hd) if kv_heads * hd > 4096 else 17000
        while True:
            case = dict(kind=kind, heads=heads, kv_heads=kv_heads, hd=hd, b=b, q=q, prompt=_log(rng, 16, most), grown=grown,
                        type=rng.choice([F32, F32, BF16]))
            if work(case)["bytes"] <= work(listed()[3])["bytes"] and work(case)["flops"] <= work(listed()[3])["flops"]:
                return case
            grown = max(1, grown // 2)
    if kind == "logprobs":
        t = rng.choice([F32, F32, BF16])
        vocab = _log(rng, 1000, 200000)
        rows = _log(rng, 1, min(4096, 4096 * 32016 // vocab))
        return dict(kind=kind, rows=rows, vocab=vocab, pad=rng.choice([0, 0, 1, 8]), top=rng.choice([1, 2, 5, 10, 20, 32]),
                    temperature=rng.choice([1.0, 1.0, 0.2, 0.8, 1.5]), type=t)
    layers, heads, hd = rng.choice([(2, 4, 64), (32, 32, 128), (8, 32, 128), (10, 40, 128), (12, 16, 64)])
    b, prompt = _log(rng, 2, 10), _log(rng, 20, 1130)
    n = rng.randint(1, 16) if kind == "branch" else _log(rng, 16, 200)
    pages = -(-prompt // PAGE) + b * (2 + -(-n // PAGE)) + rng.randint(2, 8)
    return dict(kind=kind, layers=layers, heads=heads, hd=hd, b=b, prompt=prompt, n=n, pages=pages)


# ---- inputs --------------------------------------------------------------------------------------


def _gen(seed, stream=0):
    return torch.Generator(device="cuda").manual_seed(seed * 1000003 + stream)


def _ints(g, lo, hi, n):
    """n whole numbers of [lo, hi] as a list."""
    return (torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * (hi + 1 - lo)).long().add(lo).clamp(lo, hi).tolist()


def _lengths(case):
    """Committed lengths: the prompt and what each sequence has added (given by the case alone)."""
    b, p, n = case["b"], case["prompt"], case["grown"]
    return [p + (n * (7 * s + 3)) % (n + 1) for s in range(b)]


_handles = {}


def _context(layers, heads, hd):
    """The library's context for one decoder shape: a program keeps one for its lifetime."""
    key = (layers, heads, hd)
    if key not in _handles:
        import paper_2403_18647_gb300 as sd
        shape = SimpleNamespace(n_layers=layers, d_model=heads * hd, n_heads=heads, head_dim=hd, ffn_dim=688, vocab=4104,
                                rms_eps=1e-5, rope_theta=1e4, adaptive_id=4096)
        _handles[key] = sd.Context(shape, None, max_position=4096)
    return _handles[key]


def _attention_state(case, seed):
    g = _gen(seed)
    b, q, H, Hk, hd = case["b"], case["q"], case["heads"], case["kv_heads"], case["hd"]
    lens = _lengths(case)
    shared = case["prompt"] // PAGE
    need = [-(-(n + q) // PAGE) for n in lens]
    pages = shared + sum(n - shared for n in need) + 3
    order = torch.randperm(pages, generator=g, device="cuda", dtype=torch.int32)   # pages are handed out in any order
    table = torch.full((b, max(need)), -1, dtype=torch.int32, device="cuda")
    table[:, :shared] = order[:shared]
    at = shared
    for s, n in enumerate(need):
        table[s, shared:n] = order[at:at + n - shared]
        at += n - shared
    t = TYPES[case["type"]]
    x = (torch.randn(b * q, H * hd, generator=g, device="cuda") * 1.5).to(t)
    k = torch.empty(pages, Hk, PAGE, hd, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    v = torch.empty(pages, Hk, PAGE, hd, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    return dict(x=x, k=k, v=v, table=table, shared=torch.full((b,), shared, dtype=torch.int32, device="cuda"),
                lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), out=torch.empty_like(x))


def _cache_state(case, seed):
    """A cache that holds the prompt in its last sequence, on pages anywhere in the pool."""
    g = _gen(seed)
    L, H, hd, b, n, P = case["layers"], case["heads"], case["hd"], case["b"], case["prompt"], case["pages"]
    most = -(-(n + case["n"]) // PAGE) * PAGE
    s = {}
    if own:
        s["kv"] = kv = _context(L, H, hd).kv_paged(b + 1, most, P)
        for name in ("table", "refs", "lens", "k", "v"):
            s[name] = getattr(kv, name)
    else:
        s["table"] = torch.full((b + 1, most // PAGE), -1, dtype=torch.int32, device="cuda")
        s["refs"] = torch.zeros(P, dtype=torch.int32, device="cuda")
        s["lens"] = torch.zeros(b + 1, dtype=torch.int32, device="cuda")
        s["k"] = torch.empty(L, P, H, PAGE, hd, dtype=torch.bfloat16, device="cuda")
        s["v"] = torch.empty_like(s["k"])
    s["k"].normal_(generator=g)
    s["v"].normal_(generator=g)
    held = -(-n // PAGE)
    s["table"][b, :held] = torch.randperm(P, generator=g, device="cuda", dtype=torch.int32)[:held]
    s["refs"][s["table"][b, :held].long()] = 1
    s["lens"][b] = n
    s["from"] = torch.full((b,), b, dtype=torch.int32, device="cuda")
    winner = _ints(g, 0, b - 1, 1)[0]
    s["keep"] = torch.tensor([i if i == winner else -1 for i in range(b)], dtype=torch.int32, device="cuda")
    s["grown"] = torch.tensor([n + c for c in _ints(g, case["n"] // 2, case["n"], b)], dtype=torch.int32, device="cuda")
    return s


def _logprob_state(case, seed):
    g = _gen(seed)
    R, V, pad = case["rows"], case["vocab"], case["pad"]
    x = torch.empty(R, V + pad, device="cuda").normal_(generator=g).mul_(2.0)
    x[:, V:] = 1e4                                     # what lies past the vocabulary is not a logit
    rows = torch.arange(R, device="cuda")
    for c in range(6):                                 # a few tokens stand out, as a model's do
        at = (torch.rand(R, generator=g, device="cuda") * V).long().clamp_(max=V - 1)
        x[rows, at] += 8.0 - c
    x[::3, V - V // 50:V] = -math.inf                  # every third row may not use the vocabulary's last ids
    x = x.to(TYPES[case["type"]])
    noise = torch.rand(R, generator=g, device="cuda")
    best = x[:, :V].float().argmax(-1)
    other = (torch.rand(R, generator=g, device="cuda") * (V - V // 50)).long()
    tokens = torch.where(noise < 0.7, best, other).int()
    tokens[noise > 0.97] = -1                          # rows past the end of an accepted path
    n = case["top"]
    f = lambda *shape: torch.empty(*shape, device="cuda")  # noqa: E731
    i = lambda *shape: torch.empty(*shape, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(logits=x[:, :V], tokens=tokens, logp=f(R), entropy=f(R), rank=i(R), top_ids=i(R, n), top_logp=f(R, n))


def prepare(case, seed):
    if case["kind"] == "attention":
        s = _attention_state(case, seed)
        if own:
            s["ctx"] = _context(1, 40, 128)
    elif case["kind"] == "logprobs":
        s = _logprob_state(case, seed)
        if own:
            s["ctx"] = _context(1, 40, 128)
    else:
        s = _cache_state(case, seed)
        if own:
            s["ctx"] = s["kv"].ctx
    s["case"] = case
    return s


# ---- the plain forms -------------------------------------------------------------------------------


def _plain_attention(s):
    c = s["case"]
    b, q, H, Hk, hd = c["b"], c["q"], c["heads"], c["kv_heads"], c["hd"]
    G = H // Hk
    table = s["table"].long().clamp(min=0)
    n = table.shape[1] * PAGE
    k = s["k"][table].permute(0, 2, 1, 3, 4).reshape(b, Hk, n, hd).float()
    v = s["v"][table].permute(0, 2, 1, 3, 4).reshape(b, Hk, n, hd).float()
    x = s["x"].float().view(b, q, Hk, G, hd).permute(0, 2, 1, 3, 4).reshape(b, Hk, q * G, hd)
    p = torch.matmul(x, k.transpose(2, 3)).mul_(1 / math.sqrt(hd)).view(b, Hk, q, G, n)
    last = s["lens"].long()[:, None] + torch.arange(q, device="cuda")          # the last slot that a row sees
    hidden = torch.arange(n, device="cuda") > last[:, None, :, None, None]
    p = p.masked_fill_(hidden, -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1).view(b, Hk, q * G, 1)
    o = torch.matmul(p.view(b, Hk, q * G, n), v) / total
    o = o.view(b, Hk, q, G, hd).permute(0, 2, 1, 3, 4).reshape(b * q, H * hd)
    return o.to(s["x"].dtype)


def _plain_fork(s, source):
    """Sequence i takes the pages and the length of sequence source[i] (-1: none)."""
    table, refs, lens = s["table"], s["refs"], s["lens"]
    b = source.numel()
    at = source.long().clamp(min=0)
    none = source < 0
    table[:b], lens[:b] = table[at].masked_fill(none[:, None], -1), lens[at].masked_fill(none, 0)
    held = table.reshape(-1).long()
    refs.copy_(torch.zeros(refs.numel() + 1, dtype=torch.int32, device="cuda").index_add_(
        0, held % (refs.numel() + 1), torch.ones_like(held, dtype=torch.int32))[:-1])


def _copy_rows(s, src, dst, rows):
    """Slots [0, rows) of pages src to pages dst, every layer and head."""
    some = (torch.arange(PAGE, device="cuda") < rows[:, None])[None, :, None, :, None]
    for name in ("k", "v"):
        s[name][:, dst] = torch.where(some, s[name][:, src], s[name][:, dst])


def _plain_reserve(s, b, n):
    """Pages of their own for the slots len .. len + n - 1 of the first b sequences, lowest free ids
    first; a page that others hold too is replaced by a copy of its committed slots (the last holder
    keeps it)."""
    table, refs, lens = s["table"][:b], s["refs"], s["lens"][:b, None].long()
    page = torch.arange(table.shape[1], device="cuda")
    wanted = (page >= lens // PAGE) & (page * PAGE < lens + n)
    old = table.long().clamp(min=0)
    same = (table[:, None] == table[None]) & wanted[None]                      # [i, j]: sequence j holds i's page, and wants it
    before = (same & torch.ones(b, b, dtype=torch.bool, device="cuda").tril(-1)[..., None]).sum(1)
    shared = wanted & (table >= 0) & (refs[old] - before > 1)
    fresh = (wanted & (table < 0)) | shared
    free = torch.argsort((refs > 0).int(), stable=True)
    new = free[(fresh.reshape(-1).cumsum(0) - 1).clamp(min=0, max=refs.numel() - 1)].view_as(old)
    rows = (lens - page * PAGE).clamp(0, PAGE)
    at = shared.nonzero(as_tuple=True)
    _copy_rows(s, old[at], new[at], rows[at])
    refs.index_add_(0, old[at], torch.full_like(old[at], -1, dtype=torch.int32))
    refs[new[fresh]] = 1
    table.copy_(torch.where(fresh, new, table.long()))


def _plain_compact(s):
    """The pages in use move to the front of the pool, those past its end to the holes in ascending order."""
    table, refs, lens = s["table"], s["refs"], s["lens"][:, None].long()
    used = refs > 0
    count = used.sum()
    page = torch.arange(refs.numel(), device="cuda")
    src, dst = (used & (page >= count)).nonzero().view(-1), (~used & (page < count)).nonzero().view(-1)
    to = page.clone()
    to[src] = dst
    slot = torch.arange(table.shape[1], device="cuda") * PAGE
    held, filled = table.reshape(-1).long(), (lens - slot).clamp(0, PAGE).reshape(-1)
    rows = torch.zeros(refs.numel() + 1, dtype=torch.int64, device="cuda").scatter_reduce_(
        0, held % (refs.numel() + 1), filled, "amax")[:-1]
    _copy_rows(s, src, dst, rows[src])
    refs[dst], refs[src] = refs[src], torch.zeros_like(src, dtype=torch.int32)
    table.copy_(torch.where(table >= 0, to[table.long().clamp(min=0)], -1))


def _plain_logprobs(s):
    c = s["case"]
    x, t = s["logits"].float(), s["tokens"].long()
    V, n = x.shape[1], c["top"]
    m = x.amax(-1, keepdim=True)
    d = (x - m) / c["temperature"]
    e = d.exp()
    total = e.sum(-1)
    logz = total.log()
    entropy = logz - (e * d.masked_fill(e == 0, 0.0)).sum(-1) / total
    given = t.clamp(min=0)[:, None]
    mine = x.gather(1, given)
    none = t < 0
    logp = (d.gather(1, given)[:, 0] - logz).masked_fill(none, 0.0)
    ids = torch.arange(V, device="cuda")
    rank = ((x > mine).sum(-1) + ((x == mine) & (ids < given)).sum(-1) + 1).masked_fill(none, 0)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :n]
    return dict(logp=logp, entropy=entropy, rank=rank.int(), top_ids=order.int(), top_logp=d.gather(1, order) - logz[:, None])


# ---- one pass ------------------------------------------------------------------------------------------


def run(s):
    c = s["case"]
    if c["kind"] == "attention":
        if not own:
            return _plain_attention(s)
        s["ctx"].op_prefix_attention(s["x"], s["k"], s["v"], s["table"], s["shared"], s["lens"], c["b"], c["q"], c["heads"],
                                     c["kv_heads"], c["hd"], s["out"])
        return s["out"]
    if c["kind"] == "logprobs":
        if not own:
            return _plain_logprobs(s)
        s["ctx"].op_logprobs(s["logits"], s["tokens"], s["logp"], s["entropy"], s["rank"], s["top_ids"], s["top_logp"],
                             temperature=c["temperature"])
        return {n: s[n] for n in ("logp", "entropy", "rank", "top_ids", "top_logp")}
    b = c["b"]
    if own:
        ctx, kv = s["ctx"], s["kv"]
        ctx.kv_fork(kv, s["from"], b)
        ctx.kv_reserve(kv, b, c["n"])
        if c["kind"] == "round":
            ctx.kv_commit(kv, s["grown"], b)
            ctx.kv_fork(kv, s["keep"], b)
            ctx.kv_compact(kv)
    else:
        _plain_fork(s, s["from"])
        _plain_reserve(s, b, c["n"])
        if c["kind"] == "round":
            s["lens"][:b] = s["grown"]
            _plain_fork(s, s["keep"])
            _plain_compact(s)
    return {n: s[n] for n in ("table", "refs", "lens", "k", "v")}


# ---- what a pass cannot do without ------------------------------------------------------------------


def work(case):
    if case["kind"] == "attention":
        b, q, H, Hk, hd = case["b"], case["q"], case["heads"], case["kv_heads"], case["hd"]
        lens, shared = _lengths(case), case["prompt"] // PAGE * PAGE
        slots = shared + sum(n + q - shared for n in lens)
        size = TYPES[case["type"]].itemsize
        pairs = sum(q * n + q * (q + 1) // 2 for n in lens)
        return dict(bytes=4 * Hk * hd * slots + 2 * size * b * q * H * hd, flops=4 * H * hd * pairs)
    if case["kind"] == "logprobs":
        R, V, n = case["rows"], case["vocab"], case["top"]
        return dict(bytes=TYPES[case["type"]].itemsize * R * V + R * (16 + 8 * n), flops=6 * R * V)
    # the prompt's partly filled page is read once and written for every sequence; the pages that
    # are left after a round move once
    row = 4 * case["layers"] * case["heads"] * case["hd"]
    b, n = case["b"], case["prompt"] % PAGE
    bytes_ = (1 + b) * n * row + 8 * (b + 1) * (-(-case["prompt"] // PAGE) + 1) + 8 * case["pages"]
    if case["kind"] == "round":
        bytes_ += 2 * (n + case["n"] * 3 // 4) * row
    return dict(bytes=bytes_, flops=0)


# ---- 64 bits -------------------------------------------------------------------------------------------


def _exact_attention(case, seed):
    s = _attention_state(case, seed)
    b, q, H, Hk, hd = case["b"], case["q"], case["heads"], case["kv_heads"], case["hd"]
    out = torch.empty(b, q, H, hd, dtype=torch.float64, device="cuda")
    x = s["x"].double().view(b, q, H, hd)
    for i, n in enumerate(_lengths(case)):
        at = s["table"][i, :-(-(n + q) // PAGE)].long()
        seen = torch.ones(q, n + q, dtype=torch.bool, device="cuda").tril(n)
        for h in range(Hk):
            k = s["k"][at, h].reshape(-1, hd)[:n + q].double()
            v = s["v"][at, h].reshape(-1, hd)[:n + q].double()
            for g in range(h * (H // Hk), (h + 1) * (H // Hk)):
                w = (x[i, :, g] @ k.t() / math.sqrt(hd)).masked_fill(~seen, -math.inf).softmax(-1)
                out[i, :, g] = w @ v
    return out.view(b * q, H * hd)


def _exact_cache(case, seed):
    """The cache's rules one sequence and one page at a time, on the host."""
    global own
    was, own = own, False
    s = _cache_state(case, seed)
    own = was
    table, refs, lens = s["table"].tolist(), s["refs"].tolist(), s["lens"].tolist()

    def copy(a, z, rows):
        for name in ("k", "v"):
            s[name][:, z, :, :rows] = s[name][:, a, :, :rows]

    def fork(source):
        was_t, was_l = [list(r) for r in table], list(lens)
        for i, a in enumerate(source):
            for p in was_t[i]:
                if p >= 0:
                    refs[p] -= 1
            table[i], lens[i] = (list(was_t[a]), was_l[a]) if a >= 0 else ([-1] * len(table[i]), 0)
            for p in table[i]:
                if p >= 0:
                    refs[p] += 1

    fork(s["from"].tolist())
    for i in range(case["b"]):
        for j in range(lens[i] // PAGE, -(-(lens[i] + case["n"]) // PAGE)):
            old = table[i][j]
            if old >= 0 and refs[old] == 1:
                continue
            new = refs.index(0)
            refs[new] = 1
            table[i][j] = new
            if old >= 0:
                refs[old] -= 1
                copy(old, new, max(0, min(PAGE, lens[i] - j * PAGE)))
    if case["kind"] == "round":
        lens[:case["b"]] = s["grown"].tolist()
        fork(s["keep"].tolist())
        count = sum(r > 0 for r in refs)
        for a in range(count, len(refs)):
            if refs[a]:
                z = refs.index(0)
                copy(a, z, max(max(0, min(PAGE, lens[i] - j * PAGE)) for i, r in enumerate(table) for j, p in enumerate(r) if p == a))
                refs[z], refs[a] = refs[a], 0
                table[:] = [[z if p == a else p for p in r] for r in table]
    whole = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return dict(table=whole(table), refs=whole(refs), lens=whole(lens), k=s["k"], v=s["v"])


def _exact_logprobs(case, seed):
    s = _logprob_state(case, seed)
    out = dict(logp=[], entropy=[], rank=None, top_ids=None, top_logp=[])
    for x, t in zip(s["logits"].split(256), s["tokens"].long().split(256)):
        y = torch.log_softmax(x.double() / case["temperature"], -1)
        out["logp"].append(torch.where(t < 0, 0.0, y.gather(1, t.clamp(min=0)[:, None])[:, 0]))
        out["entropy"].append(-(y.exp() * y.clamp(min=-1e300)).sum(-1))
        out["top_logp"].append(y.topk(case["top"], -1).values)
    return {n: torch.cat(v) if v is not None else None for n, v in out.items()}


def exact(case, seed):
    if case["kind"] == "attention":
        return _exact_attention(case, seed)
    if case["kind"] == "logprobs":
        return _exact_logprobs(case, seed)
    return _exact_cache(case, seed)
