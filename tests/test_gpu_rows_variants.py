"""Sizes that choose kernel variants by the rules on k and a row's vectors, each
with ordinary rows and with rows of ties and masks."""
import numpy as np
import pytest

from rows_common import INF, logits
from test_gpu_rows_top import check

pytestmark = pytest.mark.gpu


def hard_rows(v):
    rng = np.random.default_rng(v + 9)
    x = logits(rng, 6, v)
    x[1] = np.round(x[1])                        # few values
    x[2] = 0.25                                  # one value
    x[3, v // 3:] = -INF                         # banned words
    x[4] = np.sort(x[4])[::-1]
    x[5, : v // 2] -= 40.0                       # the first ones together
    return x


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v,k", [(2600, 300), (4096, 600), (5000, 700), (8000, 1000), (8300, 1000),
                                 (9700, 1024), (4700, 900)])
def test_k_near_the_number_of_vectors(v, k, dtype):
    """Parts whose maxima bound little or nothing, lists that the merge has no room for."""
    check(hard_rows(v), k, dtype, pad=v % 3, shift=k % 4)
