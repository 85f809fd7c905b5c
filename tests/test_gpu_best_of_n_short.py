"""examples/best_of_n.py from a prompt of one token, which nothing is prefilled for."""
import pytest

from test_gpu_best_of_n import test_the_kept_sample as kept_sample

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,k,loops", [(4, 5, 3), (1, 1, 2)])
def test_a_prompt_of_one_token(n, k, loops):
    kept_sample(n, k, 1, loops)
