"""How exact the block attention over shared pages is: queries and probabilities in three bf16 parts, and the tensor
cores' sums folded into rounded totals, have to show against 64 bits.

Queries of 1.5 N(0, 1), keys and values of N(0, 1), so scores of standard deviation 1.5; rows see 64 slots or more.
Errors of a result, at the 4.5 deviations that the largest of some 10^5 results are from the middle:

  scores    three parts hold 24 bits; a sum of 128 products is cut off, not rounded, at each of the 8 steps of 16 and
            where the parts' sums meet: 10 x 2^-24 of it, 3.4e-6 of a score of 6.75.  Of a key that holds 0.8 of a
            row's weight 0.16 x 3.4e-6 x 3 = 1.6e-6 reach the result; of many small weights less.
  values    32 steps of 16 slots between two folds, each cutting off half of 2^-23 of O on average: 1.9e-6 of O's part of
            a run.  After n slots the runs' parts are 1 / sqrt(54) of their share: 2.6e-7 in the middle, 1.2e-6 at
            4.5 deviations.  One run of all of them would be some 4.5e-6 at 16500 slots.
  rest      exponentials (2^-22), sums of weights, merge and division: 2^-21 of the result.

Allowed: 3e-6 + 2^-21 |ref|.  Values without folds are beyond it where an SM has a long run of one item (9000 slots of one
sequence and row: 3.4e-6 over the relative part, 0.6e-6 with folds).

Few slots show the parts of a probability: one of the 1 to 15 that a row sees counts with all of its value.  Queries
of 0.3 N(0, 1) give scores up to 1.4, whose 10 cut sums are off by 4.2e-7; 0.25 x 4.2e-7 x 6 = 6e-7 reach the result, and
as much is cut off O.  Allowed: 1.5e-6 + 2^-21 |ref|; two parts leave 2^-17 of a probability, up to 1e-5 of a result.
"""
import pytest

import synth
from test_gpu_prefix_attention import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_2403_18647_gb300 as sd
    return sd.Context(synth.SHAPES["13b"], None, max_position=64)


SIZES = [
    (2, 1, 4, 4, 64, [64, 64], 1), (16, 4, 8, 8, 64, [70 + 13 * i for i in range(16)], 1), (8, 6, 32, 32, 128, [2048 + 31 * i for i in range(8)], 32),
    (64, 1, 32, 8, 128, [900 + 7 * i for i in range(64)], 14), (2, 16, 40, 40, 128, [4095, 4200], 63), (1, 1, 40, 40, 128, [9000], 0), (1, 1, 40, 40, 128, [40000], 0),
    (16, 4, 32, 32, 128, [16500 + 33 * i for i in range(16)], 257), (2, 3, 8, 8, 64, [20011, 20100], 312),
]


@pytest.mark.parametrize("b,q,H,Hk,hd,lens,shared", SIZES)
def test_errors_against_64_bits(ctx, b, q, H, Hk, hd, lens, shared):
    c = Case(21, b, q, H, Hk, hd, lens, shared)
    ref = c.reference()
    off = (c.run(ctx).double() - ref).abs()
    assert (off - 2 ** -21 * ref.abs()).max().item() <= 3e-6, off.max().item()
    assert ctx.get_error() == 0


@pytest.mark.parametrize("H,hd", [(40, 128), (64, 64)])
def test_few_slots(ctx, H, hd):
    c = Case(22, 8, 8, H, H, hd, list(range(8)), 0, scale=0.3)
    ref = c.reference()
    off = (c.run(ctx).double() - ref).abs()
    assert (off - 2 ** -21 * ref.abs()).max().item() <= 1.5e-6, off.max().item()
    assert ctx.get_error() == 0
