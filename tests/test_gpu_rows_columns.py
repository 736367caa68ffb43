"""Gradients that lie in other columns of the buffer that holds the logits: what
lies between two rows of logits is neither read nor written, so it may hold them."""
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu
from rows_common import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab,gap", [(1, 700, 0), (5, 700, 0), (7, 5003, 1), (3, 32000, 8),
                                            (3, 70001, 5)])
@pytest.mark.parametrize("grad_first", [False, True])
def test_gradient_beside_the_logits(rows, vocab, gap, dtype, grad_first):
    dev = need_gpu()
    announce(f"gradient beside {rows}x{vocab} {dtype} gap={gap} first={grad_first}")
    gen = torch.Generator(device=dev).manual_seed(vocab)
    k = 16
    teacher = torch.randn(rows, vocab, generator=gen, device=dev) * 3
    idx, val, tail = tk.top_logits(teacher, k)
    wide = torch.full((rows, 2 * vocab + 2 * gap), 7.0, dtype=TYPES[dtype], device=dev)
    left, right = wide[:, :vocab], wide[:, vocab + gap: 2 * vocab + gap]
    grad, z = (left, right) if grad_first else (right, left)
    z.copy_(teacher + torch.randn(rows, vocab, generator=gen, device=dev))
    apart = z.clone()
    plan = tk.DistillPlan(rows, vocab, k, dtype=TYPES[dtype], check=True)
    weight = torch.ones(rows, device=dev)
    weight[rows // 2] = 0.0
    want_loss, want = plan.step(apart, idx, val, tail=tail, weight=weight)
    loss, got = plan.step(z, idx, val, tail=tail, weight=weight, grad_out=grad)
    # (vectors begin elsewhere, so sums are added in another order)
    tol = dict(rtol=2e-5 if dtype == "f32" else 2.0 ** -7, atol=1e-6)
    assert got.data_ptr() == grad.data_ptr() and torch.equal(z, apart)
    assert torch.allclose(got.float(), want.float(), **tol)
    assert torch.allclose(loss, want_loss, rtol=2e-5, atol=1e-6)
    _, stats = plan.forward(z, idx, val, tail=tail, weight=weight)
    grad.fill_(7.0)
    back = plan.backward(z, idx, val, stats, tail=tail, weight=weight, grad_out=grad)
    assert torch.equal(z, apart) and torch.allclose(back.float(), want.float(), **tol)
    rest = torch.cat([wide[:, vocab: vocab + gap], wide[:, 2 * vocab + gap:]], 1)
    assert bool((rest == 7.0).all())


def test_columns_that_overlap_are_refused():
    dev = need_gpu()
    vocab, k = 100, 8
    plan = tk.DistillPlan(4, vocab, k, dtype=torch.float32)
    idx = torch.arange(k, dtype=torch.int32, device=dev).repeat(4, 1).contiguous()
    val = torch.zeros(4, k, device=dev)
    wide = torch.zeros(5, 2 * vocab, device=dev)
    z = wide[:4, 50: 50 + vocab]
    for grad in (wide[:4, 49: 49 + vocab], wide[:4, 51: 51 + vocab], wide[:4, 100:],
                 wide[1:5, :vocab], wide[1:5, 51: 51 + vocab]):
        with pytest.raises(tk.TkefError):
            plan.step(z, idx, val, grad_out=grad)
    flat = torch.zeros(4 * 300, device=dev)
    with pytest.raises(tk.TkefError):      # between the rows, at another stride
        plan.step(flat[:1000].view(4, 250)[:, :vocab], idx, val,
                  grad_out=flat[100:].view(-1)[:800].view(4, 200)[:, :vocab])
