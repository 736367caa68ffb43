"""Log-probabilities of words that lie further below the row's greatest than the largest
binary32 number, at temperatures that bring them back into its range."""
import numpy as np
import pytest

from rows_common import logits
from test_gpu_score import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [9, 5003, 32000, 140001])
@pytest.mark.parametrize("temperature", [4.0, 1e4, 1e6])
def test_differences_beyond_the_range(v, dtype, temperature):
    """(3e38 - -3e38) / 4 = 1.5e38: the tokens', and the alternatives' of rows of few other words."""
    rng = np.random.default_rng(v)
    x = logits(rng, 4, v)
    x[0, 1:] = -3e38
    x[0, 0] = 3e38
    x[1] = -2.5e38
    x[1, v // 2] = 2.5e38
    x[1, 3] = -np.inf
    x[2] = rng.choice([3e38, 2e38, -2e38, -3e38], v)
    x[3, 5] = -3e38
    check(x, np.array([v - 1, 0, int(x[2].argmin()), 5]), 5, dtype, temperature=temperature)
    check(x, np.array([0, 3, int(x[2].argmax()), 4]), 5, dtype, temperature=temperature)
