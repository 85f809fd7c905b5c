"""The best of n sampled answers to one prompt.

The prompt is prefilled once; n samples share its pages and draft, verify and commit in blocks of k + 1
positions, every sample's tokens scored as they are accepted.  The sample of the largest mean log
probability stays: it takes sequence 0, the others' pages are given back and the pool is packed.

    python examples/best_of_n.py [--n 8] [--k 5] [--loops 12] [--prompt 300]

runs it on the small decoder of synth.py (random weights)."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def best_of_n(ctx, shape, prompt, n: int, k: int, loops: int, max_len: int, temperature: float = 0.8,
              top_p: float = 0.95, seed: int = 0):
    """-> (cache whose sequence 0 is the best sample, pages in use, its tokens, every sample's mean log probability).

    `loops` two-step loops: each emits a token of draft step 1 and 1 to k + 1 of draft step 2."""
    q, P = k + 1, prompt.numel()
    kv = ctx.kv_paged(n + 1, max_len, -(-P // 64) + n * (-(-(max_len - P) // 64) + 1))
    if P > 1:
        ctx.kv_reserve(kv, 1, P - 1, seq=n)
        ctx.prefill(kv, n, prompt[:-1])                  # the last prompt token opens the first block
    ctx.kv_fork(kv, torch.full((n,), n, dtype=torch.int32, device="cuda"))

    new = lambda *s, t=torch.int32: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    tokens, out, acc = new(n, q), new(n, q), new(n)
    logits, logp = new(n * q, shape.vocab, t=torch.float32), new(n * q, t=torch.float32)
    row = torch.arange(q, device="cuda", dtype=torch.int32)
    total, count = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    emitted = []                                         # [n][q] a step, -1 behind the accepted ones
    tokens[:, 0], tokens[:, 1:] = prompt[-1], shape.adaptive_id
    for step in range(2 * loops):
        verify = k if step % 2 else 0
        ctx.kv_reserve(kv, n, q)
        ctx.block_forward(kv, tokens, logits, n, q)
        ctx.accept_nucleus(kv, logits, tokens, n, q, verify, top_p, temperature, seed, acc, out)
        kept = torch.where(row < acc[:, None], out, -1)
        ctx.op_logprobs(logits, tokens=kept.view(-1), logp=logp, temperature=temperature)
        total += logp.view(n, q).sum(1)
        count += acc
        emitted.append(kept)
        ctx.build_block(kv, 1 if step % 2 else 2, out, acc, tokens, n, q)

    scores = total / count
    best = scores.argmax().int()
    ctx.kv_fork(kv, torch.cat([best[None], torch.full((n,), -1, dtype=torch.int32, device="cuda")]))
    used = new(1)
    ctx.kv_compact(kv, used)
    answer = torch.cat(emitted, 1)[best.long()]
    return kv, used, answer[answer >= 0], scores


def main():
    import paper_2403_18647_gb300 as sd
    import synth
    a = argparse.ArgumentParser()
    for name, value in (("n", 8), ("k", 5), ("loops", 12), ("prompt", 300)):
        a.add_argument("--" + name, type=int, default=value)
    a = a.parse_args()
    shape = synth.SHAPES["tiny"]
    most = a.prompt + (a.loops + 1) * (a.k + 2)
    ctx = sd.Context(shape, synth.make_model(shape, seed=0, device="cuda", gain_std=0.1), max_position=most)
    prompt = synth.prompt_ids(0, 40, a.prompt, 4096).cuda()
    kv, used, answer, scores = best_of_n(ctx, shape, prompt, a.n, a.k, a.loops, most)
    print("mean log probabilities: " + " ".join("%.4f" % s for s in scores.tolist()))
    print("kept %d tokens on %d pages: %s" % (answer.numel(), used.item(), " ".join(str(t) for t in answer.tolist())))
    if ctx.get_error():
        raise SystemExit("device error bits")


if __name__ == "__main__":
    main()
