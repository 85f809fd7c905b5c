"""Tensors of another type or size than a call reads or writes are refused before anything is queued."""
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
def ctx(sd):
    return sd.Context(synth.SHAPES["tiny"], None, max_position=1024)


def new(*shape, t=torch.float32):
    return torch.zeros(*shape, dtype=t, device="cuda")


def attention():
    """Arguments of a call that is in order: 2 sequences of 3 rows, 4 heads of 64 on 2 cache heads."""
    i = torch.int32
    return dict(q=new(6, 256), k=new(5, 2, PAGE, 64, t=torch.bfloat16), v=new(5, 2, PAGE, 64, t=torch.bfloat16),
                table=torch.tensor([[0, 1], [0, 2]], dtype=i, device="cuda"), shared=torch.ones(2, dtype=i, device="cuda"),
                lens=torch.tensor([70, 80], dtype=i, device="cuda"), out=torch.full((6, 256), 7.0, device="cuda"),
                anc=torch.ones(6, dtype=i, device="cuda"))


def attend(ctx, a):
    ctx.op_prefix_attention(a["q"], a["k"], a["v"], a["table"], a["shared"], a["lens"], 2, 3, 4, 2, 64, a["out"], anc=a["anc"])


WRONG_ATTENTION = {
    "table": [lambda t: t.long(), lambda t: t[:1], lambda t: t.float()], "shared": [lambda t: t.long(), lambda t: t[:1]],
    "lens": [lambda t: t.long(), lambda t: t[:1], lambda t: t.cpu()], "anc": [lambda t: t.long(), lambda t: t[:5]],
    "k": [lambda t: t.float(), lambda t: t[:, :1].contiguous(), lambda t: t[:, :, :32].contiguous(), lambda t: t[:4], lambda t: t.half()],
    "v": [lambda t: t.float(), lambda t: t[:, :1].contiguous(), lambda t: t[..., :32].contiguous(), lambda t: t[:4], lambda t: t.transpose(0, 1)],
    "q": [lambda t: t[:5], lambda t: t[:, :192], lambda t: t.half(), lambda t: t.bfloat16(), lambda t: t.t()],
    "out": [lambda t: t[:5], lambda t: t[:, :192], lambda t: t.half(), lambda t: t.bfloat16()],
}


@pytest.mark.parametrize("name", WRONG_ATTENTION)
def test_attention(ctx, name):
    whole = attention()
    out = whole["out"]
    for wrong in WRONG_ATTENTION[name]:
        a = dict(whole)
        a[name] = wrong(a[name])
        with pytest.raises(ValueError):
            attend(ctx, a)
    torch.cuda.synchronize()
    assert (out == 7).all() and ctx.get_error() == 0
    attend(ctx, whole)
    assert (out == 0).all() and ctx.get_error() == 0


def scores():
    i = torch.int32
    return dict(tokens=new(4, t=i), logp=new(4), entropy=new(4), rank=new(4, t=i), top_ids=new(4, 3, t=i), top_logp=new(4, 3))


WRONG_SCORES = {
    "tokens": [lambda t: t.long(), lambda t: t[:3], lambda t: t.float()], "logp": [lambda t: t.double(), lambda t: t[:3], lambda t: t.bfloat16()],
    "entropy": [lambda t: t.double(), lambda t: t[:3]], "rank": [lambda t: t.long(), lambda t: t[:3]],
    "top_ids": [lambda t: t.long(), lambda t: t[:3], lambda t: t[:, :2].contiguous()],
    "top_logp": [lambda t: t.double(), lambda t: t[:3], lambda t: t[:, :2].contiguous(), lambda t: t.bfloat16(), lambda t: t.view(3, 4)],
}


@pytest.mark.parametrize("name", WRONG_SCORES)
def test_log_probabilities(ctx, name):
    logits = torch.randn(4, 100, device="cuda")
    for wrong in WRONG_SCORES[name]:
        a = scores()
        was = {k: t.clone() for k, t in a.items()}
        with pytest.raises(ValueError):
            ctx.op_logprobs(logits, **{**a, name: wrong(a[name])})
        torch.cuda.synchronize()
        assert all(torch.equal(a[k], was[k]) for k in a)
    a = scores()
    ctx.op_logprobs(logits, **a)
    assert (a["rank"] > 0).all() and ctx.get_error() == 0


def test_fork_and_compact(ctx):
    kv = ctx.kv_paged(3, 128, 6)
    src = new(3, t=torch.int32)
    for call in (lambda: ctx.kv_fork(kv, src.long()), lambda: ctx.kv_fork(kv, src[:2], 3), lambda: ctx.kv_fork(kv, src.cpu()),
                 lambda: ctx.kv_compact(kv, new(1)), lambda: ctx.kv_compact(kv, new(0, t=torch.int32)),
                 lambda: ctx.kv_compact(kv, new(1, t=torch.int64))):
        with pytest.raises(ValueError):
            call()
    ctx.kv_fork(kv, src[:2])
    ctx.kv_fork(kv, src, 2)
    ctx.kv_compact(kv, src)
    assert ctx.get_error() == 0
