"""Sizes that choose kernel variants by the rules on k and a row's vectors, each
with ordinary rows and with rows of ties and masks."""
import numpy as np
import pytest

from rows_common import INF, logits
from test_gpu_rows_distill import check as check_step
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


# vectors of a row (16 bytes): up to 1,024, 2,048 and 4,096 in whole rows of 256 threads,
# 8,192 in 512; shares a thread by k: one up to 64, two up to 128, four up to 256
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vectors", [700, 1500, 3100, 6001])
@pytest.mark.parametrize("k", [40, 65, 100, 128, 129, 200, 256])
def test_whole_rows(vectors, k, dtype):
    v = vectors * (4 if dtype == "f32" else 8) + 3
    check(hard_rows(v), k, dtype, pad=k % 3, shift=k % 2)


# lists in parts of four vectors a thread and the larger merge
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vectors", [2500, 4000, 4096])
@pytest.mark.parametrize("k", [257, 890, 1000, 1024])
def test_long_lists_in_small_parts(vectors, k, dtype):
    v = vectors * (4 if dtype == "f32" else 8) + 1
    check(hard_rows(v), k, dtype, pad=1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("k", [129, 300, 1024])
def test_long_lists_in_large_parts(k, dtype):
    check(hard_rows(70001), k, dtype, shift=3)


@pytest.mark.parametrize("dtype,v", [("f32", 40001), ("f32", 65535), ("bf16", 100003)])
def test_steps_of_many_long_rows(dtype, v):
    """Rows of more than 128 KB taken whole, in 1,024 threads."""
    rng = np.random.default_rng(v)
    check_step(rng, 98, v, 20, dtype, ragged=True, weighted=True)
