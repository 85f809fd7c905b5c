"""examples/best_of_n.py: the kept sample and its score against the same tokens fed to a contiguous cache.

Logits of the two paths differ by up to 3e-2 (bf16 rows of the caches move by one place between sums of
another order), a log probability at temperature T by twice that over T, a mean of them by no more."""
import importlib.util
import os

import pytest
import torch

import synth

pytestmark = pytest.mark.gpu

NEAR, T = 3e-2, 0.8


def load():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "best_of_n.py")
    spec = importlib.util.spec_from_file_location("best_of_n", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("n,k,prompt,loops", [(8, 5, 300, 6), (1, 3, 2, 3), (10, 5, 65, 4), (21, 2, 64, 3)])
def test_the_kept_sample(n, k, prompt, loops):
    import paper_2403_18647_gb300 as sd
    shape = synth.SHAPES["tiny"]
    most = prompt + (loops + 1) * (k + 2)
    ctx = sd.Context(shape, synth.make_model(shape, seed=0, device="cuda", gain_std=0.1), max_position=most)
    ids = synth.prompt_ids(0, 40, prompt, 4096).cuda()
    kv, used, answer, scores = load().best_of_n(ctx, shape, ids, n, k, loops, most, temperature=T)
    m = answer.numel()
    assert 2 * loops <= m <= loops * (k + 2)
    # the cache: the prompt and the answer but its last token, on the pool's first pages, nobody else's
    assert kv.lens.tolist() == [prompt - 1 + m] + [0] * n
    pages = kv.table[0][kv.table[0] >= 0].tolist()
    assert sorted(pages) == list(range(used.item())) and kv.refs.sum().item() == used.item()
    assert (kv.table[1:] == -1).all()
    # the answer, token by token, on a contiguous cache
    flat = ctx.kv(1, most)
    if prompt > 1:
        ctx.prefill(flat, 0, ids[:-1])
    fed = torch.cat([ids[-1:], answer])
    lg, total = torch.empty(1, shape.vocab, device="cuda"), 0.0
    for i in range(m):
        ctx.block_forward(flat, fed[i:i + 1].contiguous(), lg, 1, 1)
        total += (lg[0].double() / T).log_softmax(0)[answer[i].long()].item()
        ctx.kv_commit(flat, torch.tensor([prompt + i], dtype=torch.int32, device="cuda"), 1)
    assert abs(total / m - scores.max().item()) <= 2 * NEAR / T
    # and both caches go on alike
    lz = torch.empty_like(lg)
    ctx.kv_reserve(kv, 1, 1)
    ctx.block_forward(flat, answer[-1:].contiguous(), lg, 1, 1)
    ctx.block_forward(kv, answer[-1:].contiguous(), lz, 1, 1)
    assert (lg - lz).abs().max().item() <= NEAR
    assert ctx.get_error() == 0
