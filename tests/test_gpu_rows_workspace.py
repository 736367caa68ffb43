"""Workspaces of the row operators' calls on long rows."""
import torch

import pytest

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu

pytestmark = pytest.mark.gpu


def test_the_gradient_takes_no_workspace(monkeypatch):
    dev = need_gpu()
    gen = torch.Generator(device=dev).manual_seed(1)
    rows, vocab, k = 3, 140001, 20
    t = torch.randn(rows, vocab, generator=gen, device=dev) * 3
    z = t + torch.randn(rows, vocab, generator=gen, device=dev)
    announce("gradient of long rows without a workspace")
    idx, val, tail = tk.top_logits(t, k)
    plan = tk.DistillPlan(rows, vocab, k, dtype=torch.float32)
    assert plan.ws_bytes > 0
    _, stats = plan.forward(z, idx, val, tail=tail)
    want = plan.step(z, idx, val, tail=tail)[1]
    monkeypatch.setattr(plan, "_workspace", lambda *a: pytest.fail("no workspace is needed"))
    got = plan.backward(z, idx, val, stats, tail=tail)
    assert torch.allclose(got, want, rtol=2e-5, atol=1e-9)
