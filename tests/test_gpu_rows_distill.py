"""DistillPlan (forward, backward, step) against the oracle, and its gradient
against differences of its own loss."""
import math

import numpy as np
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu
from oracle import rows
from rows_common import (EPS, INF, STORE, TYPES, device_rows, finite_max, logits, rounding, vec)

pytestmark = pytest.mark.gpu


def lists(rng, teacher, k, temperature, val):
    """Each row's list in the wire format, and its values as the kernel sees them."""
    n = teacher.shape[0]
    idx, t, tail = np.zeros((n, k), np.int32), np.zeros((n, k)), np.zeros(n)
    for r in range(n):
        idx[r], t[r], tail[r] = rows.top(teacher[r], k, temperature)
    t_dev = vec(t, TYPES[val])
    return vec(idx, torch.int32), t_dev, vec(tail), idx, t_dev.double().cpu().numpy(), \
        tail.astype(np.float32).astype(np.float64)


def check_row(got_loss, got_grad, z, want, val, tail, weight, temperature, dtype, dloss=1.0):
    v = z.size
    rel = rounding(v, (finite_max(z, val) / temperature) + finite_max(tail))
    if got_loss is not None:
        if not math.isfinite(want.loss):
            assert got_loss == want.loss or (math.isnan(want.loss) and math.isnan(got_loss))
        else:
            # each logarithm is off by rel; they are weighted by probabilities
            # that are off by rel themselves
            spread = 2.0
            if want.p_rest > 0 and want.q_rest > 0:
                spread += abs(math.log(want.p_rest / want.q_rest))
            if want.p.size:
                with np.errstate(all="ignore"):
                    part = want.p * np.abs(np.log(want.p))
                spread += float(np.nansum(part[np.isfinite(part)]))
                spread += finite_max(val) / temperature * 0.125
            tol = abs(weight) * temperature ** 2 * rel * spread + abs(want.loss) * (4 * EPS + rel)
            assert abs(got_loss - want.loss) <= tol, (got_loss, want.loss, tol)
    if got_grad is not None:
        g = want.grad * dloss
        if not np.isfinite(g).all():
            assert np.isnan(got_grad).all()
            return
        ratio = want.p_rest / want.q_rest if want.q_rest > 0 else 0.0
        size = want.q * (1.0 + ratio)
        # listed words hold -p as well; p is at least |grad| / scale - q
        scale = abs(weight * temperature * dloss)
        size = size + np.abs(want.grad) / (abs(weight * temperature) or 1.0)
        half, least = STORE[dtype]
        tol = rel * scale * size * 2 + np.abs(g) * half * 1.01 + least
        bad = np.nonzero(np.abs(got_grad - g) > tol)[0]
        assert bad.size == 0, (bad[:5], got_grad[bad[:5]], g[bad[:5]], tol[bad[:5]])


def check(rng, n, v, k, dtype, temperature=1.0, val="f32", use_tail=True, ragged=False,
          weighted=False, pad=0, shift=0, gpad=None, student=None, teacher=None):
    announce(f"distill {n}x{v} k={k} {dtype} T={temperature} val={val} tail={use_tail} "
             f"ragged={ragged} pad={pad} shift={shift}")
    dev = need_gpu()
    teacher = logits(rng, n, v, 3.0 * temperature) if teacher is None else teacher
    student = teacher + rng.normal(size=(n, v)) * 0.7 * temperature if student is None else student
    z, exact = device_rows(student, dtype, pad, shift)
    idx, t, tail, idx_h, t_h, tail_h = lists(rng, teacher, k, temperature, val)
    count = rng.integers(0, k + 1, n) if ragged else np.full(n, k)
    if ragged:
        count[0] = 0
        count[-1] = k
    weight = rng.uniform(0.5, 1.5, n).astype(np.float32) if weighted else np.ones(n, np.float32)
    if weighted and n > 1:
        weight[1] = 0.0
        z[1] = math.nan
    dloss = rng.uniform(-1, 1, n).astype(np.float32)
    kw = dict(tail=tail if use_tail else None, count=vec(count, torch.int32) if ragged else None,
              weight=vec(weight) if weighted else None)
    plan = tk.DistillPlan(n + 2, v, k, dtype=TYPES[dtype], temperature=temperature,
                          val_dtype=TYPES[val], check=True)
    loss, stats = plan.forward(z, idx, t, **kw)
    step_loss, step_grad = plan.step(z, idx, t, **kw)
    if gpad is None:
        grad = plan.backward(z, idx, t, stats, dloss=vec(dloss), **kw)
    else:
        wide = torch.full((n, v + gpad), 7.0, dtype=TYPES[dtype], device=dev)
        grad = plan.backward(z, idx, t, stats, dloss=vec(dloss), grad_out=wide[:, :v], **kw)
        assert bool((wide[:, v:] == 7.0).all())
    place = z.clone()
    if pad == 0 and shift == 0:
        plan.step(place, idx, t, grad_out=place, **kw)
        assert torch.equal(place, step_grad) or bool(torch.isnan(step_grad).any())
    got = [a.double().cpu().numpy() for a in (loss, step_loss, step_grad, grad)]
    for r in range(n):
        c = int(count[r])
        lo = float(tail_h[r]) if use_tail else -INF
        want = rows.distill(exact[r], idx_h[r, :c], t_h[r, :c], lo, float(weight[r]), temperature)
        args = (exact[r], want, t_h[r, :c], lo, float(weight[r]), temperature, dtype)
        check_row(got[0][r], None, *args)
        check_row(got[1][r], got[2][r], *args)
        check_row(None, got[3][r], *args, dloss=float(dloss[r]))


SIZES = [(1, 1), (2, 1), (2, 2), (5, 5), (8, 3), (9, 9), (64, 16), (65, 64), (255, 255),
         (1000, 33), (1025, 1024), (4097, 64), (8191, 128), (16385, 8), (32000, 8), (32000, 64),
         (32769, 65), (50001, 200), (65537, 257), (131071, 128), (131073, 1000), (262147, 64)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v,k", SIZES)
def test_sizes(v, k, dtype):
    rng = np.random.default_rng(v * 5 + k)
    check(rng, 3, v, k, dtype, temperature=[1.0, 0.5, 2.0][v % 3], val=["f32", "f16"][k % 2],
          use_tail=k < v and v % 2 == 0)
    check(rng, 4, v, k, dtype, ragged=True, weighted=True, use_tail=k < v and v % 2 == 1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("pad,shift,gpad", [(1, 0, 0), (0, 1, 3), (3, 5, 1), (64, 7, 8),
                                            (129, 2, None)])
def test_strides_and_alignment(pad, shift, gpad, dtype):
    rng = np.random.default_rng(pad * 13 + shift)
    for v, k in ((33, 5), (5003, 64), (32000, 64)):
        check(rng, 4, v, k, dtype, pad=pad, shift=shift, gpad=gpad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 9, 300, 1030])
def test_many_rows(n, dtype):
    check(np.random.default_rng(n), n, 2503, 24, dtype, temperature=2.0, val="f16",
          weighted=n > 1, ragged=n > 1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v", [300, 32000, 140001])
def test_masks_and_great_leads(v, dtype):
    rng = np.random.default_rng(v)
    n, k = 8, 20
    teacher = logits(rng, n, v)
    student = teacher + rng.normal(size=(n, v)) * 0.7
    student[0, v // 2:] = -INF
    teacher[0, v // 2:] = -INF
    student[1] = -INF                                  # no word at all
    student[2, np.argsort(-teacher[2])[:3]] = -INF     # words the teacher wants: loss +inf
    student[3, np.argsort(-teacher[3])[:k]] += 60.0    # nearly nothing outside the list
    student[4, np.argsort(-teacher[4])[:k]] -= 60.0    # nearly nothing inside it
    student[5, np.argsort(-teacher[5])[k:]] = -INF     # nothing outside
    student[6] = np.finfo(np.float16).min              # flat, at the lowest value
    student[7, :] = rng.normal(size=v) * 1e-3
    check(rng, n, v, k, dtype, student=student, teacher=teacher)
    check(rng, n, v, k, dtype, student=student, teacher=teacher, use_tail=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_and_infinite_logits(dtype):
    dev = need_gpu()
    v, k = 5000, 8
    z = torch.randn(5, v, device=dev).to(TYPES[dtype])
    z[0, 17] = math.nan
    z[1, 4999] = INF
    idx = torch.arange(k, dtype=torch.int32, device=dev).repeat(5, 1).contiguous() * 100
    val = torch.randn(5, k, device=dev)
    val[2] = -INF                                      # a list without mass
    z[3, 300] = math.nan                               # at a listed word
    plan = tk.DistillPlan(5, v, k, dtype=TYPES[dtype], check=True)
    loss, grad = plan.step(z, idx, val)
    assert torch.isnan(loss).tolist() == [True, True, True, True, False]
    assert torch.isnan(grad).all(dim=1).tolist() == [True, True, True, True, False]
    loss2, stats = plan.forward(z, idx, val)
    assert torch.isnan(loss2).tolist() == [True, True, True, True, False]
    grad2 = plan.backward(z, idx, val, stats)
    assert torch.isnan(grad2).all(dim=1).tolist() == [True, True, True, True, False]


def test_entries_out_of_order_or_range_are_left_out():
    dev = need_gpu()
    v = 40000
    z = torch.randn(3, v, device=dev)
    idx = torch.tensor([[5, 9, 7, 30000], [-1, 5, 9, 30000], [5, 9, 30000, v]],
                       dtype=torch.int32, device=dev)
    val = torch.randn(3, 4, device=dev)
    plan = tk.DistillPlan(3, v, 4, dtype=torch.float32)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    announce("distill with bad entries")
    loss, grad = plan.step(z, idx, val, status=status)
    assert int(status.item()) == tk.STATUS_UNSORTED | tk.STATUS_INDEX_RANGE
    keep = [[0, 1, 3], [1, 2, 3], [0, 1, 2]]
    good = torch.stack([idx[r, k] for r, k in enumerate(keep)]).contiguous()
    good_val = torch.stack([val[r, k] for r, k in enumerate(keep)]).contiguous()
    want_loss, want_grad = tk.distill_step(z, good, good_val)
    assert torch.allclose(loss, want_loss, rtol=1e-5, atol=1e-6)
    assert torch.allclose(grad, want_grad, rtol=1e-5, atol=1e-9)
    with pytest.raises(tk.TkefStatusError):
        tk.distill_step(z, idx, val)


def test_unused_entries_are_not_read():
    dev = need_gpu()
    v = 3001
    z = torch.randn(2, v, device=dev)
    idx = torch.tensor([[3, 8, 2 ** 31 - 1, -7], [1, 0, 0, 0]], dtype=torch.int32, device=dev)
    val = torch.tensor([[0.5, 1.5, math.nan, INF], [2.0, math.nan, 0.0, INF]], device=dev)
    count = torch.tensor([2, 1], dtype=torch.int32, device=dev)
    plan = tk.DistillPlan(2, v, 4, dtype=torch.float32, check=True)
    loss, grad = plan.step(z, idx, val, count=count)
    for r, c in ((0, 2), (1, 1)):
        w = rows.distill(z[r].double().cpu().numpy(), idx[r, :c].cpu().numpy(),
                         val[r, :c].double().cpu().numpy())
        assert loss[r].item() == pytest.approx(w.loss, rel=1e-5)
        assert np.abs(grad[r].cpu().numpy() - w.grad).max() < 1e-6


@pytest.mark.parametrize("use_tail", [True, False])
def test_gradient_against_differences_of_the_loss(use_tail):
    """Central differences along a random direction with steps of h: the
    third derivative leaves h^2 / 6 * |u|^3 * (a few), the losses' rounding
    leaves 2 * error / h."""
    dev = need_gpu()
    rng = np.random.default_rng(9)
    n, v, k, temperature = 6, 700, 12, 1.5
    teacher = logits(rng, n, v, 2.0)
    student = teacher + rng.normal(size=(n, v)) * 0.5
    idx, t, tail, *_ = lists(rng, teacher, k, temperature, "f32")
    plan = tk.DistillPlan(n, v, k, dtype=torch.float32, temperature=temperature, check=True)
    kw = dict(tail=tail if use_tail else None)
    z = vec(student)
    _, grad = plan.step(z, idx, t, **kw)
    u = rng.normal(size=(n, v))
    u /= np.linalg.norm(u, axis=1, keepdims=True)
    h = 0.0625
    up, down = z + vec(u) * h, z - vec(u) * h
    num = (plan.forward(up, idx, t, **kw)[0].double() - plan.forward(down, idx, t, **kw)[0].double())
    real = ((up - down).double() * grad.double()).sum(1)
    err = rounding(v, 12.0) * 8 * temperature ** 2
    assert torch.all((num - real).abs() <= 2 * err + 2 * h ** 3)


def test_autograd_matches_the_step():
    dev = need_gpu()
    rng = np.random.default_rng(10)
    n, v, k = 33, 4001, 16
    teacher = logits(rng, n, v)
    idx, t, tail, *_ = lists(rng, teacher, k, 2.0, "f16")
    z = vec(teacher + rng.normal(size=(n, v)), torch.bfloat16).requires_grad_()
    weight = vec(rng.uniform(0, 1, n))
    plan = tk.DistillPlan(n, v, k, dtype=torch.bfloat16, temperature=2.0,
                          val_dtype=torch.float16)
    plan.loss(z, idx, t, tail=tail, weight=weight).sum().backward()
    loss, grad = plan.step(z.detach(), idx, t, tail=tail, weight=weight)
    assert torch.allclose(z.grad.float(), grad.float(), rtol=2 ** -7, atol=1e-7)


def test_same_inputs_same_bits_and_other_stream():
    dev = need_gpu()
    rng = np.random.default_rng(11)
    n, v, k = 40, 32000, 64
    teacher = logits(rng, n, v)
    idx, t, tail, *_ = lists(rng, teacher, k, 1.0, "f32")
    z = vec(teacher + rng.normal(size=(n, v)), torch.bfloat16)
    plan = tk.DistillPlan(n, v, k, dtype=torch.bfloat16)
    loss, grad = plan.step(z, idx, t, tail=tail)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    loss2, grad2 = plan.step(z, idx, t, tail=tail, stream=s)
    s.synchronize()
    assert torch.equal(loss, loss2) and torch.equal(grad, grad2)
    part, part_grad = plan.step(z[5:9], idx[5:9], t[5:9], tail=tail[5:9])
    assert torch.allclose(part, loss[5:9], rtol=1e-5)
    assert plan.step(z[:0], idx[:0], t[:0], tail=tail[:0])[1].shape == (0, v)


def test_refusals():
    dev = need_gpu()
    plan = tk.DistillPlan(4, 100, 8, dtype=torch.float32)
    z = torch.zeros(4, 100, device=dev)
    idx = torch.arange(8, dtype=torch.int32, device=dev).repeat(4, 1).contiguous()
    val = torch.zeros(4, 8, device=dev)
    for kw in (dict(logits=z.half()), dict(idx=idx.long()), dict(val=val.half()),
               dict(tail=torch.zeros(3, device=dev)), dict(count=torch.zeros(4, device=dev)),
               dict(weight=torch.zeros(4)), dict(idx=idx[:, :7]),
               dict(grad_out=torch.zeros(4, 99, device=dev)),
               dict(grad_out=torch.zeros(4, 100, device=dev).half())):
        with pytest.raises(ValueError):
            plan.step(**{**dict(logits=z, idx=idx, val=val), **kw})
    wide = torch.zeros(4 * 100 + 50, device=dev)
    a, b = wide[:400].view(4, 100), wide[50:450].view(4, 100)
    with pytest.raises(tk.TkefError):          # overlapping, not the same
        plan.step(a, idx, val, grad_out=b)
    with pytest.raises(tk.TkefError):
        tk.DistillPlan(4, 100, 101)
    with pytest.raises(ValueError):
        tk.DistillPlan(4, 100, 8, val_dtype=torch.bfloat16)


LOWEST = {"f32": float(np.finfo(np.float32).min), "f16": -65504.0,
          "bf16": float(torch.finfo(torch.bfloat16).min)}


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v", [300, 32000, 70000, 140001])
def test_masks_at_the_lowest_value_of_the_type(v, dtype):
    """A mask of the type's lowest value leaves a word without probability
    beside ordinary ones, and a row of nothing else uniform."""
    rng = np.random.default_rng(v + 1)
    low = LOWEST[dtype]
    n, k = 6, 12
    teacher = logits(rng, n, v)
    student = teacher + rng.normal(size=(n, v)) * 0.5
    best = [np.argsort(-teacher[r])[:k] for r in range(n)]
    student[0] = low                                   # nothing but the mask
    student[1, v // 3:] = low                          # most words masked
    teacher[1, v // 3:] = -60.0
    student[2] = low
    student[2, best[2]] = teacher[2, best[2]]          # only listed words left
    student[3] = -INF
    student[3, ::2] = low                              # the mask, and masked words
    teacher[3, 1::2] = -60.0
    student[4] = low
    student[4, v - 1] = 1.0                            # one word left, at the end
    teacher[4] = -60.0
    teacher[4, v - 1] = 2.0
    for use_tail in (True, False):
        check(rng, n, v, k, dtype, student=student, teacher=teacher, use_tail=use_tail)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [-1e9, -1e10, -1e30, -2e38])
@pytest.mark.parametrize("v", [300, 32000, 70000, 140001])
def test_masks_of_great_size(v, mask, dtype):
    """Whole threads' and whole rows' words at a large value that is not the
    type's lowest, where a product with the exponent's factor is rounded by more
    than an exponent holds."""
    rng = np.random.default_rng(v + 6)
    n, k = 6, 12
    teacher = logits(rng, n, v)
    student = teacher + rng.normal(size=(n, v)) * 0.5
    best = [np.argsort(-teacher[r])[:k] for r in range(n)]
    student[0] = mask                                  # nothing but the mask
    student[1, v // 3:] = mask
    teacher[1, v // 3:] = -60.0
    student[2] = mask
    student[2, best[2]] = teacher[2, best[2]]          # only listed words left
    student[3] = -mask                                 # as far above zero
    student[4] = mask
    student[4, v - 1] = 1.0                            # one word left, at the end
    teacher[4] = -60.0
    teacher[4, v - 1] = 2.0
    student[5] = mask
    student[5, v // 2: v // 2 + 40] = 0.0
    for temperature in (1.0, 0.8, 1.3):
        check(rng, n, v, k, dtype, temperature=temperature, student=student, teacher=teacher)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_few_and_many_long_rows(dtype):
    """Rows that a call of few takes in chunks and one of many whole."""
    rng = np.random.default_rng(17)
    for n in (2, 98):
        check(rng, n, 70003, 20, dtype, ragged=True, weighted=True)
