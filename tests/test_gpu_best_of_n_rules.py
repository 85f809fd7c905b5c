"""examples/best_of_n.py with a repetition penalty: no penalty is what it was, a strong one leaves no token twice."""
import pytest
import torch

import synth
from test_gpu_best_of_n import load

pytestmark = pytest.mark.gpu


def run(repetition, n=4, k=4, prompt=70, loops=5):
    import paper_2403_18647_gb300 as sd
    shape = synth.SHAPES["tiny"]
    most = prompt + (loops + 1) * (k + 2)
    ctx = sd.Context(shape, synth.make_model(shape, seed=0, device="cuda", gain_std=0.1), max_position=most)
    ids = synth.prompt_ids(0, 40, prompt, 4096).cuda()
    kv, used, answer, scores = load().best_of_n(ctx, shape, ids, n, k, loops, most, repetition=repetition)
    assert ctx.get_error() == 0
    return ids.tolist(), kv.lens.tolist(), answer.tolist(), scores


def test_a_penalty_of_one_changes_nothing():
    _, lens, answer, scores = run(None)
    _, lens1, answer1, scores1 = run(1.0)
    assert lens == lens1 and answer == answer1 and torch.equal(scores, scores1)


def test_a_strong_penalty_leaves_no_token_twice():
    """Positive logits over 1e6 and negative ones times 1e6: what was used is out of reach of the nucleus, as long as some
    unused logit is positive (of 4104 random ones, always)."""
    prompt, lens, answer, _ = run(1e6)
    assert lens[0] == len(prompt) - 1 + len(answer)
    assert len(set(answer)) == len(answer) and not set(answer) & set(prompt)
