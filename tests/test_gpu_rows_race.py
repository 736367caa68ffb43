"""The race of a verification: its scores are quotients, and the target's own
probabilities count only where the residual of the whole row is empty."""
import numpy as np
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu
from rows_common import TYPES
from test_gpu_rows_verify import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [300, 32000, 70001])
def test_noise_whose_reciprocal_is_beyond_the_type(v, dtype):
    """Flat rows, so scores are 1 / (v noise): finite for noise above 3e-39 / v,
    though 1 / noise is not."""
    dev = need_gpu()
    announce(f"race with least noise {v} {dtype}")
    target = torch.zeros(3, 2, v, dtype=TYPES[dtype], device=dev)
    drafts = torch.zeros(3, 1, v, dtype=TYPES[dtype], device=dev)
    drafts[2] = 0.0
    drafts[2, 0, :3] = 40.0          # rejected: the residual of all words from the fourth on
    noise = torch.full((3, v), 2.0, device=dev)
    noise[:, 7], noise[:, v - 5] = 2e-39, 1e-39
    noise[1, 7], noise[1, v - 5] = 1e-39, 2e-39
    tokens = torch.zeros(3, 1, dtype=torch.int32, device=dev)
    uniform = torch.full((3, 1), 0.5, device=dev)
    got = tk.verify_draft(target, drafts, tokens, uniform, noise)
    assert got[0].tolist() == [1, 1, 0]
    assert got[1].tolist() == [[0, v - 5], [0, 7], [v - 5, -1]]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v", [300, 5000, 70001])
def test_residual_in_few_words(v, dtype):
    """Whole waves and chunks without a residual, beside one word that has it; the
    target's own best word lies elsewhere."""
    rng = np.random.default_rng(v + 11)
    b, draft = 5, 2
    target = rng.normal(size=(b, draft + 1, v)) * 0.5
    drafts = target[:, :draft].copy()
    for s, word in enumerate((0, 3, v // 2, v - 2, v - 1)):
        drafts[s, 0, word] -= 8.0
        target[s, 0, word] += 1.0
    noise = rng.uniform(0.5, 2.0, size=(b, v))
    noise[:, v // 3] = 1e-3
    tokens = np.full((b, draft), v // 4)
    uniform = np.full((b, draft), 1.0 - 2.0 ** -24)     # (q > p there: rejected)
    target[:, 0, v // 4] -= 1.0
    drafts[:, 0, v // 4] += 1.0
    check(rng, b, draft, v, dtype, target=target, drafts=drafts, tokens=tokens, uniform=uniform,
          noise=noise)
