"""Log probabilities at the ends of what a call takes."""
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


def test_the_smallest_temperatures(sd, ctx):
    """Where log2(e) / T is not a finite fp32 value the call is refused; above it a distribution is its maximum, shared among
    equal ones."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(3, 5000, generator=g) * 2
    x[1, [7, 4000]] = 30.0
    x[2, :] = -math.inf
    x = x.cuda()
    t = torch.tensor([3, 4000, 0], dtype=torch.int32, device="cuda")
    new = lambda *s: torch.full(s, math.nan, device="cuda")  # noqa: E731
    logp, entropy, top, ids = new(3), new(3), new(3, 3), torch.zeros(3, 3, dtype=torch.int32, device="cuda")
    for temperature in (1e-45, 1e-39, 2.9e-39, 4.2e-39):
        with pytest.raises(sd.SdsatError) as e:
            ctx.op_logprobs(x, t, logp, entropy, top_ids=ids, top_logp=top, temperature=temperature)
        assert e.value.status == 1
    assert logp.isnan().all() and entropy.isnan().all()
    for temperature in (4.3e-39, 1e-38, 1e-30):
        ctx.op_logprobs(x, t, logp, entropy, top_ids=ids, top_logp=top, temperature=temperature)
        half = math.log(2.0)
        assert abs(entropy[1].item() - half) < 1e-6 and entropy[[0, 2]].tolist() == [0.0, 0.0]
        assert abs(logp[1].item() + half) < 1e-6
        below = ((x[0, 3].double() - x[0].max().double()) / float(torch.tensor(temperature))).float().item()
        assert math.isclose(logp[0].item(), below, rel_tol=1e-6) and logp[2].item() == -math.inf
        assert top[0, 0].item() == 0 and (top[0, 1:] < -1e28).all()
        assert ids[1, :2].tolist() == [7, 4000] and ids[2].tolist() == [0, 1, 2]
    assert ctx.get_error() == 0
