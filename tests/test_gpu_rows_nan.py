"""What a verification gives where a row holds a NaN or +inf, as the header says:
a broken drafts row rejects its token and leaves the target's own distribution,
a broken target row samples nothing; both are reported where they matter."""
import math

import numpy as np
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu
from oracle import rows
from rows_common import INF, TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, INF])
@pytest.mark.parametrize("v", [300, 32000, 70001])
def test_broken_rows(v, bad, dtype):
    dev = need_gpu()
    announce(f"verify with {bad} {v} {dtype}")
    gen = torch.Generator(device=dev).manual_seed(v)
    target = torch.randn(4, 3, v, generator=gen, device=dev).to(TYPES[dtype])
    drafts = target[:, :2].clone()
    tokens = torch.randint(0, v, (4, 2), generator=gen, device=dev, dtype=torch.int32)
    noise = torch.empty(4, v, device=dev).exponential_(generator=gen)
    uniform = torch.full((4, 2), 0.5, device=dev)
    drafts[0, 1, v - 2] = bad          # the second place's drafts
    target[1, 0, v // 2] = bad         # the first place's target
    target[2, 2, 5] = bad              # the place after all drafts
    tokens[3, 0] = -1
    drafts[3, 1, 0] = bad              # beyond the first rejection: no matter
    plan = tk.VerifyPlan(4, 2, v, dtype=TYPES[dtype])

    def call(s):
        status = torch.zeros(1, dtype=torch.int32, device=dev)
        one = slice(s, s + 1)
        got = plan.execute(target[one], drafts[one], tokens[one], uniform[one], noise[one],
                           status=status)
        return [g[0].tolist() for g in got], int(status.item())

    def drawn(s, place):
        p = rows.softmax(target[s, place].double().cpu().numpy())
        score = p / noise[s].double().cpu().numpy()
        return int(np.argmax(score)), p

    t = tokens.tolist()
    (acc, out, logp), status = call(0)
    y, p = drawn(0, 1)
    assert (acc, out, status) == (1, [t[0][0], y, -1], tk.STATUS_NAN)
    assert abs(logp[1] - math.log(p[y])) < 1e-4 and logp[2] == 0.0
    (acc, out, logp), status = call(1)
    assert (acc, out, logp, status) == (0, [-1, -1, -1], [0.0] * 3, tk.STATUS_NAN)
    (acc, out, logp), status = call(2)
    assert (acc, out, status) == (2, [t[2][0], t[2][1], -1], tk.STATUS_NAN) and logp[2] == 0.0
    (acc, out, logp), status = call(3)
    assert (acc, out[1:], status) == (0, [-1, -1], tk.STATUS_INDEX_RANGE) and out[0] >= 0
