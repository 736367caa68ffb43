"""The row operators' oracle against independent statements of the same
mathematics (CPU only): brute-force order, closed forms, central differences,
sampling frequencies."""
import math

import numpy as np
import pytest

from oracle import rows

INF = math.inf


def test_top_against_sorted_pairs():
    rng = np.random.default_rng(1)
    for v in (1, 2, 5, 40):
        for k in {1, (v + 1) // 2, v}:
            x = rng.integers(-3, 4, v).astype(float)
            best = sorted(range(v), key=lambda i: (-x[i], i))[:k]
            idx, val, tail = rows.top(x, k, 2.0)
            assert idx.tolist() == sorted(best)
            assert val.tolist() == [x[i] for i in sorted(best)]
            rest = [x[i] for i in range(v) if i not in best]
            want = math.log(sum(math.exp(r / 2.0) for r in rest)) if rest else -INF
            assert tail == pytest.approx(want)


def test_top_signed_zeros_tie_and_masked_rest():
    idx, _, tail = rows.top([-0.0, 0.0, -INF, 0.0], 2)
    assert idx.tolist() == [0, 1]
    assert tail == 0.0
    assert rows.top([1.0, -INF, -INF], 1)[2] == -INF


@pytest.mark.parametrize("temperature", [1.0, 0.7, 3.0])
def test_distill_zero_where_student_equals_teacher(temperature):
    z = np.random.default_rng(2).normal(size=50) * 4
    idx, val, tail = rows.top(z, 7, temperature)
    r = rows.distill(z, idx, val, tail, 1.0, temperature)
    assert abs(r.loss) < 1e-12
    assert np.abs(r.grad).max() < 1e-12
    assert r.p.sum() + r.p_rest == pytest.approx(1.0)


def test_distill_of_one_entry_is_cross_entropy():
    z = np.array([0.5, -1.0, 2.0, 0.0])
    r = rows.distill(z, [2], [123.0])
    e = np.exp(z)
    assert r.loss == pytest.approx(-math.log(e[2] / e.sum()))
    assert r.grad == pytest.approx(e / e.sum() - np.eye(4)[2])


def test_distill_whole_list_is_kullback_leibler():
    rng = np.random.default_rng(3)
    z, t = rng.normal(size=9), rng.normal(size=9)
    p, q = np.exp(t) / np.exp(t).sum(), np.exp(z) / np.exp(z).sum()
    r = rows.distill(z, np.arange(9), t)
    assert r.loss == pytest.approx(float(np.sum(p * np.log(p / q))))
    assert r.grad == pytest.approx(q - p)


@pytest.mark.parametrize("tail", [None, -INF])
@pytest.mark.parametrize("temperature", [1.0, 0.6, 2.5])
def test_distill_gradient_against_differences(tail, temperature):
    rng = np.random.default_rng(4)
    teacher = rng.normal(size=30) * 3
    z = teacher + rng.normal(size=30)
    idx, val, mass = rows.top(teacher, 6, temperature)
    mass = mass if tail is None else tail
    r = rows.distill(z, idx, val, mass, 1.7, temperature)
    h = 1e-5
    for i in range(z.size):
        up, down = z.copy(), z.copy()
        up[i] += h
        down[i] -= h
        num = (rows.distill(up, idx, val, mass, 1.7, temperature).loss
               - rows.distill(down, idx, val, mass, 1.7, temperature).loss) / (2 * h)
        assert r.grad[i] == pytest.approx(num, abs=1e-8)


def test_distill_dead_and_impossible_rows():
    nan = np.full(4, math.nan)
    assert rows.distill(nan, [1], [0.0], weight=0.0).loss == 0.0
    assert not rows.distill(nan, [], []).grad.any()
    assert rows.distill([0.0, -INF], [1], [0.0]).loss == INF
    assert math.isnan(rows.distill([-INF, -INF], [1], [0.0]).loss)


def test_verify_accepts_equal_models_and_rejects_impossible_tokens():
    rng = np.random.default_rng(5)
    t = rng.normal(size=(4, 11))
    noise = rng.exponential(size=11)
    r = rows.verify(t, t[:3], [1, 2, 3], [0.999, 0.999, 0.0], noise)
    assert r.accepted == 3 and r.tokens[:3] == [1, 2, 3]
    p = rows.softmax(t[3])
    assert r.tokens[3] == int(np.argmax(p / noise))
    masked = t.copy()
    masked[1, 2] = -INF
    r = rows.verify(masked, t[:3], [1, 2, 3], [0.0, 0.0, 0.0], noise)
    assert r.accepted == 1 and r.tokens[2:] == [-1, -1] and r.logp[2:] == [0.0, 0.0]


def test_verify_distribution_is_the_targets():
    """One drafted token: the first output token follows the target's
    distribution (each frequency within 5 standard deviations)."""
    rng = np.random.default_rng(6)
    t, d = rng.normal(size=(2, 6)) * 1.5, rng.normal(size=(1, 6)) * 1.5
    p, q = rows.softmax(t[0]), rows.softmax(d[0])
    n, seen = 20000, np.zeros(6)
    for x, u, noise in zip(rng.choice(6, n, p=q), rng.random(n), rng.exponential(size=(n, 6))):
        seen[rows.verify(t, d, [x], [u], noise).tokens[0]] += 1
    assert np.all(np.abs(seen / n - p) < 5 * np.sqrt(p * (1 - p) / n))


def test_verify_with_nothing_to_sample():
    r = rows.verify(np.full((2, 3), -INF), np.zeros((1, 3)), [1], [0.5], np.ones(3))
    assert r.accepted == 0 and r.tokens == [-1, -1] and r.logp == [0.0, 0.0]
