"""ScorePlan (execute, forward, backward) against the oracle, and its gradient against
differences of the oracle's scores and under autograd."""
import math

import numpy as np
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu
from oracle import score as oracle
from rows_common import EPS, STORE, TYPES, device_rows, finite_max, logits, rounding, vec

pytestmark = pytest.mark.gpu


def tolerance(x, temperature):
    """Of a logarithm of the row's sum: the sum's relative error, and the logarithm's own
    rounding (two units of at most ln V)."""
    return rounding(x.size, finite_max(x) / temperature) + 4 * EPS * (math.log(x.size) + 1)


def close_log(got, want, x, tol):
    """One log-probability. Beyond the largest binary32 number (3.4e38: a mask at the lowest
    value, times 1 / temperature) its nearest binary32 value is -inf."""
    want = -math.inf if want < -float(np.finfo(np.float32).max) else want
    if math.isnan(want) or math.isinf(want):
        assert got == want or (math.isnan(want) and math.isnan(got)), (got, want)
    else:
        tol = tol + 4 * EPS * (abs(want) + math.log(x.size))
        assert abs(got - want) <= tol, (got, want, tol)


def check_scores(got, x, want, temperature):
    """logp = (x_t - m) / T - ln S: the difference, the factor, the product and the last
    difference round once each, units of |x_t - m| / T <= |logp| + ln V. The entropy's two terms
    are ln S and a mean exponent, each off by the sums' relative error of itself."""
    logp, entropy = got
    tol = tolerance(x, temperature)
    close_log(logp, want.logp, x, tol)
    if math.isnan(want.logp):
        assert math.isnan(entropy)
        return
    mean = want.entropy + math.log(x.size)   # (at least sum p (m - x) / T)
    assert abs(entropy - want.entropy) <= tol * (2 + 2 * mean), (entropy, want.entropy, tol)


def check_gradient(got, x, token, dlogp, dentropy, temperature, dtype):
    want = oracle.score_gradient(x, token, dlogp, dentropy, temperature)
    if not np.isfinite(want).all():
        assert np.isnan(got).all()
        return
    r = oracle.score(x, token, 0, temperature)
    p = np.exp(r.log_p)
    there = r.log_p > -math.inf
    each = abs(dlogp) + abs(dentropy) * (np.abs(np.where(there, r.log_p, 0.0)) + r.entropy + 1.0)
    size = p * each
    if token >= 0:
        size[token] += abs(dlogp)
    # (the hardware's exponential gives 0 below the least normal number, 2^-126, and the sum is at
    # least 1: a probability may be off by that much beside its relative error)
    lost = np.where(there, 2.0 ** -126 * each, 0.0) / temperature
    half, least = STORE[dtype]
    tol = tolerance(x, temperature) * 2 * size / temperature + np.abs(want) * half * 1.01 + least + lost
    bad = np.nonzero(np.abs(got - want) > tol)[0]
    assert bad.size == 0, (bad[:5], got[bad[:5]], want[bad[:5]], tol[bad[:5]])


def check(x, tokens, k, dtype, temperature=1.0, pad=0, shift=0, gpad=None, seed=0, bits=0,
          dlogp=None, dentropy=None):
    n, v = x.shape
    announce(f"score {n}x{v} k={k} {dtype} T={temperature} pad={pad} shift={shift}")
    dev = need_gpu()
    rng = np.random.default_rng(seed)
    z, exact = device_rows(x, dtype, pad, shift)
    tok = vec(tokens, torch.int32)
    dlogp = rng.normal(size=n).astype(np.float32) if dlogp is None else dlogp
    dentropy = rng.normal(size=n).astype(np.float32) if dentropy is None else dentropy
    plan = tk.ScorePlan(n + 2, v, k, dtype=TYPES[dtype], temperature=temperature)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    logp, entropy, idx, val = plan.execute(z, tok, status=status)
    assert int(status.item()) == bits
    logp2, entropy2, stats = plan.forward(z, tok)
    # (whole rows take the same way with and without alternatives)
    grads = []
    for dl, dh in ((dlogp, dentropy), (dlogp, None), (None, dentropy)):
        kw = dict(dlogp=None if dl is None else vec(dl), dentropy=None if dh is None else vec(dh))
        if gpad is not None:
            wide = torch.full((n, v + gpad), 7.0, dtype=TYPES[dtype], device=dev)
            kw["grad_out"] = wide[:, :v]
        grads.append(plan.backward(z, tok, stats, **kw))
        if gpad is not None:
            assert bool((wide[:, v:] == 7.0).all())
    place = z.clone()
    plan.backward(place, tok, stats, dlogp=vec(dlogp), dentropy=vec(dentropy), grad_out=place)
    assert torch.equal(place.view(torch.int16 if dtype != "f32" else torch.int32),
                       grads[0].contiguous().view(torch.int16 if dtype != "f32" else torch.int32))
    a = [t.double().cpu().numpy() for t in (logp, entropy, logp2, entropy2, val)]
    words = idx.cpu().numpy()
    grads = [g.double().cpu().numpy() for g in grads]
    for r in range(n):
        t = int(tokens[r]) if 0 <= tokens[r] < v else -1
        want = oracle.score(exact[r], t, k, temperature)
        check_scores((a[0][r], a[1][r]), exact[r], want, temperature)
        check_scores((a[2][r], a[3][r]), exact[r], want, temperature)
        assert (words[r] == want.words).all(), (r, words[r], want.words)
        for got, w in zip(a[4][r], want.word_logp):
            close_log(got, w, exact[r], tolerance(exact[r], temperature))
        for g, dl, dh in ((grads[0], dlogp[r], dentropy[r]), (grads[1], dlogp[r], 0.0),
                          (grads[2], 0.0, dentropy[r])):
            check_gradient(g[r], exact[r], t, float(dl), float(dh), temperature, dtype)


SIZES = [(1, 0), (1, 1), (2, 1), (5, 5), (8, 3), (9, 9), (64, 64), (65, 20), (255, 64), (1000, 33),
         (1025, 0), (4097, 64), (8191, 20), (8200, 5), (16385, 1), (32000, 20), (32000, 0),
         (32769, 64), (50001, 5), (65537, 20), (131071, 64), (131073, 0), (262147, 20),
         (1 << 20, 64)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v,k", SIZES)
def test_sizes(v, k, dtype):
    rng = np.random.default_rng(v * 7 + k)
    n = 3 if v < 200_000 else 2
    tokens = rng.integers(0, v, n)
    tokens[0] = v - 1
    check(logits(rng, n, v), tokens, k, dtype, temperature=[1.0, 0.5, 2.0][v % 3])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("pad,shift,gpad", [(1, 0, 0), (0, 1, 3), (3, 5, 1), (64, 7, 8),
                                            (129, 2, None)])
def test_strides_and_alignment(pad, shift, gpad, dtype):
    rng = np.random.default_rng(pad * 13 + shift)
    for v, k in ((33, 5), (5003, 20), (32000, 20), (70001, 3)):
        check(logits(rng, 4, v), rng.integers(0, v, 4), k, dtype, pad=pad, shift=shift, gpad=gpad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 9, 300, 1030])
def test_many_rows(n, dtype):
    rng = np.random.default_rng(n)
    tokens = rng.integers(0, 2503, n)
    check(logits(rng, n, 2503, 6.0), tokens, 7, dtype, temperature=2.0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v", [40, 5003, 32000, 140001])
def test_rows_without_a_token(v, dtype):
    """-1 and other words outside the vocabulary; such rows hold NaN and are not read. So are rows
    whose two gradients are 0."""
    rng = np.random.default_rng(v)
    x = logits(rng, 6, v)
    tokens = np.array([3, -1, v - 1, -1, 0, 5])
    x[1] = x[3] = math.nan
    check(x, tokens, 20, dtype)
    tokens[3] = v
    check(x, tokens, 20, dtype, bits=tk.STATUS_INDEX_RANGE)
    tokens[3] = -2 ** 31
    x[5] = 1.0
    dead = np.array([1, 1, 0, 1, 1, 0], np.float32)
    check(x, tokens, 20, dtype, bits=tk.STATUS_INDEX_RANGE, dlogp=dead, dentropy=dead)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v", [70, 5003, 32000, 140001])
def test_masks(v, dtype):
    """Masked words (-inf; the type's lowest value; -1e4), masked tokens, rows with fewer
    unmasked words than alternatives, one word only, none but lowest values, ties."""
    rng = np.random.default_rng(v + 1)
    lowest = float(torch.finfo(TYPES[dtype]).min)
    x = logits(rng, 10, v)
    x[0, v // 2:] = -math.inf
    x[1, 10:] = -math.inf                    # ten words left
    x[2, :] = -math.inf
    x[2, v - 3] = -2.5                       # one
    x[3, 5:] = lowest
    x[4, :] = lowest                         # uniform
    x[5, ::2] = -1e4
    x[6, :] = 1.0                            # ties
    x[7, :] = np.round(x[7])
    x[8, :] = np.arange(v)[::-1] / v         # descending
    x[9, :] = np.arange(v) / v
    tokens = np.array([1, v - 1, v - 3, 1, v - 2, 3, v // 2, 7, 0, v - 1])
    check(x, tokens, 20, dtype)
    tokens[:6] = [v - 1, 3, 0, v - 1, 0, 0]
    check(x, tokens, 64, dtype, temperature=0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [5003, 140001])
def test_great_leads_and_far_rows(v, dtype):
    """A word far ahead of all others; rows far off zero, beyond what a product with
    log2(e) / temperature holds."""
    rng = np.random.default_rng(v + 2)
    x = logits(rng, 6, v)
    x[0, 9] = 200.0
    x[1] += 1e5 if dtype == "f32" else 256.0
    x[2] = 3e38
    x[3] = -3e38
    x[3, :5] = -2.9e38
    x[4] = 1e30
    x[4, 7:] = -1e30
    x[5, :] = 2e9
    x[5, 3] = 2.5e9
    check(x, np.array([9, 3, 4, 2, 6, 3]), 5, dtype)
    check(x, np.array([8, 3, 4, 9, 9, 4]), 5, dtype, temperature=0.1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v", [9, 5003, 32000, 140001])
def test_broken_rows(v, dtype):
    """NaN, +inf, no word at all: NaN results for that row alone, with the status bit."""
    rng = np.random.default_rng(v + 3)
    good = logits(rng, 2, v)
    for bad in ("nan", "all nan", "inf", "two inf", "none"):
        x = np.stack([good[0], good[0], good[1]])
        x[1, v // 2] = {"nan": math.nan, "inf": math.inf, "two inf": math.inf}.get(bad, x[1, v // 2])
        if bad == "two inf":
            x[1, 0] = math.inf
        if bad in ("all nan", "none"):
            x[1] = math.nan if bad == "all nan" else -math.inf
        check(x, np.array([1, 2, 3]), 5, dtype, bits=tk.STATUS_NAN)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_alternatives_that_lie_together(dtype):
    """The greatest words in one thread's share, in one vector, in the row's ends, in one
    chunk of a long row; and many of equal value."""
    for v in (5003, 32000, 140001):
        rng = np.random.default_rng(v + 4)
        x = logits(rng, 5, v) * 0.5
        x[0, 100:164] += 30
        x[1, 5:v:2048] += 30                       # (a thread's vectors lie 2,048 words apart)
        x[2, 3:v:1024] += 30
        x[3, -40:] += 30
        x[4, rng.choice(v, 600, replace=False)] = 40.0
        for k in (5, 64):
            check(x, np.array([101, 5, 3, v - 1, 0]), k, dtype)


def test_no_rows_and_empty_alternatives():
    dev = need_gpu()
    plan = tk.ScorePlan(4, 100, 3, dtype=torch.float32)
    z, t = torch.zeros(0, 100, device=dev), torch.zeros(0, dtype=torch.int32, device=dev)
    assert [o.numel() for o in plan.execute(z, t)] == [0, 0, 0, 0]
    logp, entropy, stats = plan.forward(z, t)
    assert plan.backward(z, t, stats, dlogp=logp).shape == (0, 100)
    z, t = torch.zeros(2, 100, device=dev), torch.zeros(2, dtype=torch.int32, device=dev)
    logp, entropy, idx, val = tk.ScorePlan(4, 100, dtype=torch.float32).execute(z, t)
    assert idx.shape == (2, 0) and val.shape == (2, 0)
    # a uniform row: -log p and the entropy are ln 100, whose logarithm rounds twice
    assert abs(entropy.cpu() - math.log(100)).max() <= 4 * EPS * math.log(100)


def test_gradient_against_differences():
    """The gradient's definition itself: central differences of the oracle's scores; then the
    kernel's gradient against the same, at a step whose truncation (h^2 / 6 of a third
    derivative that is at most 6 here) and rounding (1e-16 / h) are below 1e-9."""
    rng = np.random.default_rng(11)
    x, t, a, b, temp = logits(rng, 1, 40)[0].astype(np.float32).astype(np.float64), 7, 0.7, -1.3, 1.5
    g = oracle.score_gradient(x, t, a, b, temp)
    h = 1e-5
    diff = np.zeros_like(x)
    for i in range(x.size):
        lo, hi = x.copy(), x.copy()
        lo[i] -= h
        hi[i] += h
        p, m = oracle.score(hi, t, 0, temp), oracle.score(lo, t, 0, temp)
        diff[i] = (a * (p.logp - m.logp) + b * (p.entropy - m.entropy)) / (2 * h)
    assert np.abs(diff - g).max() < 1e-9
    z = vec(x[None])
    tok = vec([t], torch.int32)
    plan = tk.ScorePlan(1, 40, dtype=torch.float32, temperature=temp)
    _, _, stats = plan.forward(z, tok)
    got = plan.backward(z, tok, stats, dlogp=vec([a]), dentropy=vec([b]))[0].double().cpu().numpy()
    assert np.abs(got - diff).max() < 1e-9 + tolerance(x, temp) * 2 * 6


@pytest.mark.parametrize("which", ["both", "logp", "entropy", "sum"])
def test_autograd(which):
    rng = np.random.default_rng(12)
    x = logits(rng, 6, 501)
    tokens = np.array([1, -1, 500, 3, 0, 7])
    z = vec(x).requires_grad_()
    plan = tk.ScorePlan(6, 501, dtype=torch.float32, temperature=0.8)
    logp, entropy = plan.score(z, vec(tokens, torch.int32))
    w = rng.normal(size=(2, 6)).astype(np.float32)
    if which == "sum":      # (a gradient whose rows share memory)
        w[:] = 1.0
        (logp.sum() + entropy.sum()).backward()
    else:
        w[0] *= which != "entropy"
        w[1] *= which != "logp"
        loss = 0.0
        if which != "entropy":
            loss = loss + (logp * vec(w[0])).sum()
        if which != "logp":
            loss = loss + (entropy * vec(w[1])).sum()
        loss.backward()
    got = z.grad.double().cpu().numpy()
    exact = z.detach().double().cpu().numpy()
    for r in range(6):
        check_gradient(got[r], exact[r], int(tokens[r]), float(w[0, r]), float(w[1, r]), 0.8, "f32")


def test_one_shot_call_raises_on_status():
    dev = need_gpu()
    z = torch.randn(3, 50, device=dev)
    t = torch.tensor([1, 2, 50], dtype=torch.int32, device=dev)
    with pytest.raises(tk.TkefStatusError):
        tk.score_tokens(z, t, 4)
    t[2] = 49
    logp, entropy, idx, val = tk.score_tokens(z, t, 4)
    want = torch.log_softmax(z, 1)
    assert torch.equal(idx.long(), want.topk(4, dim=1).indices)
    assert (logp - want.gather(1, t.long()[:, None])[:, 0]).abs().max() < 1e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v,k", [(5003, 20), (32000, 64), (140001, 20)])
def test_same_bits_as_alternatives_and_on_every_run(v, k, dtype):
    """A token's log-probability is that of the alternative that it is, bit for bit, and calls
    repeat bit for bit."""
    rng = np.random.default_rng(v + 5)
    z, exact = device_rows(logits(rng, 40, v), dtype)
    tokens = vec(exact.argmax(1), torch.int32)
    plan = tk.ScorePlan(40, v, k, dtype=TYPES[dtype])
    first = [t.clone() for t in plan.execute(z, tokens)]
    assert torch.equal(first[0], first[3][:, 0])
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(plan.execute(z, tokens), first))
