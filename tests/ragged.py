"""Ragged batches on pages for the tests: sequences of `new` rows after `ctx` committed slots."""
import torch

PAGE = 64


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pages:
    """Page table, pools and starts; pages are handed out in random order."""

    def __init__(self, g, Hk, hd, new, ctx, before=0, spare=3, columns=0):
        self.new, self.ctx = list(new), list(ctx)
        need = [-(-(n + m) // PAGE) for n, m in zip(new, ctx)]
        pages = sum(need) + spare
        order = torch.randperm(pages, generator=g, device="cuda").int()
        self.table = torch.full((len(need), max(need + [1]) + columns), -1, dtype=torch.int32, device="cuda")
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        starts = [before]
        for n in new:
            starts.append(starts[-1] + n)
        self.first, self.rows = starts[:-1], starts[-1]
        self.starts, self.lens = ints(starts), ints(self.ctx)
        self.k = torch.randn(pages, Hk, PAGE, hd, generator=g, device="cuda").bfloat16()
        self.v = torch.randn(pages, Hk, PAGE, hd, generator=g, device="cuda").bfloat16()

    def spoil(self, value):
        """What no row may see: unused pages, and the slots past each sequence's new rows."""
        free = torch.ones(self.k.shape[0], dtype=torch.bool, device="cuda")
        free[self.table[self.table >= 0].long()] = False
        for t in (self.k, self.v):
            t[free] = value
            for s, (n, m) in enumerate(zip(self.new, self.ctx)):
                if (n + m) % PAGE:
                    t[self.table[s, (n + m) // PAGE].long(), :, (n + m) % PAGE:] = value
        return self

    def slots(self, s):
        """(pages, places in them) of sequence s's new rows."""
        at = torch.arange(self.ctx[s], self.ctx[s] + self.new[s], device="cuda")
        return self.table[s, at // PAGE].long(), at % PAGE


def attention(p, q, H, Hk, hd):
    """Causal attention of the new rows in 64 bits, (rows, H, hd), and sum_t p_t |v_t| beside it."""
    out = torch.zeros(q.shape[0], H, hd, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(out)
    x = q.double().view(q.shape[0], H, hd)
    for s, (n, m) in enumerate(zip(p.new, p.ctx)):
        if not n:
            continue
        at = torch.full((-(-(n + m) // PAGE),), -1, dtype=torch.long, device="cuda")
        have = p.table[s, :at.numel()].long()
        at[:have.numel()] = have
        bad = (at < 0) | (at >= p.k.shape[0])
        k = p.k[at.masked_fill(bad, 0)].transpose(0, 1).reshape(Hk, -1, hd)[:, :n + m].double()
        v = p.v[at.masked_fill(bad, 0)].transpose(0, 1).reshape(Hk, -1, hd)[:, :n + m].double()
        hidden = ~torch.ones(n, n + m, dtype=torch.bool, device="cuda").tril(m) | bad.repeat_interleave(PAGE)[:n + m]
        v = v.masked_fill(hidden.all(0)[None, :, None], 0.0)
        r = slice(p.first[s], p.first[s] + n)
        for h in range(H):
            w = (x[r, h] @ k[h // (H // Hk)].t() / hd ** 0.5).masked_fill(hidden, float("-inf")).softmax(-1)
            w = w.masked_fill(hidden.all(1)[:, None], 0.0)
            out[r, h] = w @ v[h // (H // Hk)]
            size[r, h] = w @ v[h // (H // Hk)].abs()
    return out, size
