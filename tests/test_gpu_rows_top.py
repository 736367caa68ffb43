"""TopLogitsPlan against the oracle: indices and values exactly, the rest's
log-mass within the rounding of a 32-bit sum."""
import math

import numpy as np
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu
from oracle import rows
from rows_common import INF, TYPES, device_rows, finite_max, logits, rounding

pytestmark = pytest.mark.gpu


def check(x, k, dtype, temperature=1.0, val="f32", pad=0, shift=0):
    n, v = x.shape
    announce(f"top {n}x{v} k={k} {dtype} val={val} pad={pad} shift={shift}")
    z, exact = device_rows(x, dtype, pad, shift)
    plan = tk.TopLogitsPlan(n + 1, v, k, dtype=TYPES[dtype], temperature=temperature,
                            val_dtype=TYPES[val], check=True)
    idx, value, tail = plan.execute(z)
    assert idx.shape == value.shape == (n, k) and tail.shape == (n,)
    got_idx, got_val = idx.cpu().numpy(), value.cpu()
    got_tail = tail.double().cpu().numpy()
    for r in range(n):
        want, want_val, want_tail = rows.top(exact[r], k, temperature)
        assert np.array_equal(got_idx[r], want), (r, got_idx[r][:8], want[:8])
        stored = z[r].cpu()[torch.from_numpy(want.astype(np.int64))].to(TYPES[val])
        raw = torch.int16 if TYPES[val] == torch.float16 else torch.int32
        assert torch.equal(got_val[r].view(raw), stored.view(raw))
        if math.isinf(want_tail):
            assert got_tail[r] == want_tail
        else:
            tol = rounding(v, finite_max(exact[r]) / temperature)
            tol += abs(want_tail) * 2.0 ** -23
            assert abs(got_tail[r] - want_tail) <= tol, (r, got_tail[r], want_tail, tol)


SIZES = [(1, 1), (2, 1), (2, 2), (7, 3), (8, 8), (9, 4), (63, 5), (64, 64), (65, 1), (255, 16),
         (1000, 33), (1023, 1023), (2049, 1024), (4097, 64), (8191, 256), (32000, 16),
         (32000, 64), (32769, 65), (50001, 200), (65537, 257), (131071, 300), (131073, 1000),
         (262147, 64)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v,k", SIZES)
def test_sizes(v, k, dtype):
    rng = np.random.default_rng(v * 7 + k)
    check(logits(rng, 3, v), k, dtype, temperature=[1.0, 0.5, 2.0][v % 3],
          val=["f32", "f16"][k % 2])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 1), (3, 5), (64, 7), (129, 2)])
def test_strides_and_alignment(pad, shift, dtype):
    rng = np.random.default_rng(pad * 11 + shift)
    for v, k in ((33, 5), (5003, 64), (32000, 64)):
        check(logits(rng, 4, v), k, dtype, pad=pad, shift=shift)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows_", [1, 7, 300, 1025])
def test_many_rows(rows_, dtype):
    rng = np.random.default_rng(rows_)
    check(logits(rng, rows_, 2503), 32, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v", [300, 32000, 131071, 200000])
def test_ties_masks_and_extremes(v, dtype):
    rng = np.random.default_rng(v)
    x = np.empty((14, v))
    x[0] = 1.5                                    # all equal
    x[1] = -INF                                   # every word masked
    x[2] = np.where(np.arange(v) % 997 == 3, 2.0, -INF)   # few words left
    x[3] = rng.integers(-2, 3, v)                 # five values
    x[4] = np.where(rng.random(v) < 0.5, 0.0, -0.0)       # signed zeros
    x[5] = np.arange(v) / v                       # ascending
    x[6] = -np.arange(v) / v                      # descending
    x[7] = 0.0
    x[7, : v // 2] = np.finfo(np.float32).min if dtype != "f16" else -65504.0
    x[8] = rng.normal(size=v)
    x[8, v // 3] = INF
    x[9] = rng.normal(size=v)
    x[9, [1, v // 2, v - 1]] = [1e4, 3e4, 2e4]    # a great lead: the rest must not vanish
    x[10] = rng.normal(size=v)
    x[10, ::3] = -INF
    x[11] = rng.normal(size=v) * 1e-3             # nearly flat
    x[12] = np.where(np.arange(v) < 40, 1e4, -1e4)        # the rest far below the 40 greatest
    x[13] = -INF
    x[13, [0, v - 1]] = [3.0, -3.0]
    for k in (1, 40, min(300, v)):
        check(x, k, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unselected_infinity_and_nan(dtype):
    dev = need_gpu()
    x = torch.randn(4, 9001, device=dev).to(TYPES[dtype])
    x[0, :9] = INF
    x[2, 77] = math.nan
    x[3, 4321] = -math.nan
    plan = tk.TopLogitsPlan(4, 9001, 8, dtype=TYPES[dtype])
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    announce("top with +inf and NaN")
    idx, _, tail = plan.execute(x, status=status)
    assert int(status.item()) == tk.STATUS_NAN
    assert idx[0].tolist() == list(range(8)) and tail[0].item() == INF
    want = rows.top(x[1].double().cpu().numpy(), 8)
    assert np.array_equal(idx[1].cpu().numpy(), want[0])
    for r in (2, 3):
        i = idx[r].cpu().numpy()
        assert i.min() >= 0 and i.max() < 9001 and np.all(np.diff(i) > 0)
        assert math.isnan(tail[r].item())


def test_fewer_rows_outputs_given_and_other_stream():
    dev = need_gpu()
    plan = tk.TopLogitsPlan(50, 4000, 16, dtype=torch.float32, check=True)
    x = torch.randn(20, 4000, device=dev)
    ref = plan.execute(x)
    idx = torch.empty(20, 16, dtype=torch.int32, device=dev)
    val = torch.empty(20, 16, device=dev)
    tail = torch.empty(20, device=dev)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = plan.execute(x, idx_out=idx, val_out=val, tail_out=tail, stream=s)
    s.synchronize()
    assert got[0] is idx and torch.equal(idx, ref[0]) and torch.equal(val, ref[1])
    assert torch.equal(tail, ref[2])
    part = plan.execute(x[:3])
    assert torch.equal(part[0], ref[0][:3]) and torch.equal(part[2], ref[2][:3])
    none = plan.execute(x[:0])
    assert none[0].shape == (0, 16)
    one = tk.top_logits(x, 16)
    assert torch.equal(one[0], ref[0]) and torch.equal(one[1], ref[1])


def test_refusals():
    dev = need_gpu()
    plan = tk.TopLogitsPlan(4, 100, 8, dtype=torch.bfloat16)
    ok = torch.zeros(4, 100, dtype=torch.bfloat16, device=dev)
    for bad in (ok.float(), ok[:, :99], ok.cpu(), torch.zeros(5, 100, dtype=ok.dtype, device=dev),
                torch.zeros(100, 4, dtype=ok.dtype, device=dev).t(), ok[0]):
        with pytest.raises(ValueError):
            plan.execute(bad)
    with pytest.raises(ValueError):
        plan.execute(ok, idx_out=torch.zeros(4, 8, dtype=torch.int64, device=dev))
    with pytest.raises(tk.TkefError):
        plan.execute(ok[:1].expand(4, 100))
    for kw in (dict(rows=0), dict(vocab=0), dict(k=0), dict(k=101), dict(temperature=0.0),
               dict(temperature=math.nan), dict(vocab=(1 << 20) + 1), dict(vocab=4000, k=1025)):
        with pytest.raises(tk.TkefError):
            tk.TopLogitsPlan(**{**dict(rows=4, vocab=100, k=8), **kw})
    with pytest.raises(ValueError):
        tk.TopLogitsPlan(4, 100, 8, dtype=torch.float64)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v", [300, 32000, 131071, 200000])
def test_masks_at_the_lowest_value_of_the_type(v, dtype):
    rng = np.random.default_rng(v + 2)
    low = -65504.0 if dtype == "f16" else float(torch.finfo(TYPES[dtype]).min)
    x = logits(rng, 5, v)
    x[0] = low
    x[1, v // 4:] = low
    x[2] = low
    x[2, ::1000] = 1.0
    x[3, 1::2] = -INF
    x[3, ::2] = low
    x[4] = low
    x[4, v // 2] = 0.0
    for k in (1, 20, 70):
        check(x, k, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [3000, 32000, 40001, 131071])
def test_clustered_and_tied_rows(v, dtype):
    """The k first together in one place, beside ties that reach past what a
    workgroup keeps, and with fewer ordinary words than k."""
    rng = np.random.default_rng(v + 4)
    n = 9
    x = rng.normal(size=(n, v))
    x[0, 1000:] = -INF                                  # the first words only
    x[1, : v - 700] -= 50.0                             # the last words far ahead
    x[2] = np.round(x[2])                               # few values
    x[3] = np.round(x[3] * 2)
    x[4] = 1.0
    x[4, rng.integers(0, v, 30)] = 2.0                  # 30 above a constant
    x[5] = 1.0
    x[5, v // 2: v // 2 + 500] = 3.0                    # a run of ties above a constant
    x[6] = -INF
    x[6, rng.permutation(v)[:55]] = rng.normal(size=55)
    x[7] = np.sort(x[7])[::-1]
    x[8] = np.repeat(rng.normal(size=(v + 63) // 64), 64)[:v]   # blocks of equal words
    for k in (1, 55, 64, 128, 200, 256, 700):
        check(x, k, dtype, pad=k % 3, shift=k % 5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [-1e9, -1e10, -1e30, -2e38])
@pytest.mark.parametrize("v", [300, 32000, 131071])
def test_masks_of_great_size(v, mask, dtype):
    """Threads, and bounds, whose words are all at a large value that is not
    the type's lowest."""
    rng = np.random.default_rng(v + 6)
    x = logits(rng, 5, v)
    x[0] = mask
    x[1, v // 4:] = mask
    x[2] = mask
    x[2, ::1000] = 1.0
    x[3] = -mask
    x[4] = mask
    x[4, v // 2: v // 2 + 40] = 0.0
    for k in (1, 20, 70):
        check(x, k, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v", [300, 32000, 40001, 131071])
def test_nan_among_ties(v, dtype):
    """One NaN in a row of equal words, or of a few values: beyond the infinity of its
    sign, reported, and no tail."""
    announce(f"nan among ties {v} {dtype}")
    rng = np.random.default_rng(v + 8)
    x = np.ones((6, v))
    x[1] = np.round(rng.normal(size=v))
    x[2] = -INF
    x[3] = -3e4
    x[4] = 2.0
    x[4, ::2] = 1.0
    at = [0, v - 1, v // 2, 17, v // 3, 40]
    for r in range(6):
        x[r, at[r]] = math.nan
    z, exact = device_rows(x, dtype)
    for k in (1, 64, 200):
        plan = tk.TopLogitsPlan(6, v, k, dtype=TYPES[dtype])
        status = torch.zeros(1, dtype=torch.int32, device=need_gpu())
        idx, value, tail = plan.execute(z, status=status)
        assert int(status.item()) == tk.STATUS_NAN
        got = idx.cpu().numpy()
        for r in range(6):
            # (a conversion to bfloat16 makes negative NaNs, which come last)
            order = np.nan_to_num(exact[r], nan=np.copysign(INF, exact[r][at[r]]), neginf=-1e300)
            want = np.sort(np.argsort(-order, kind="stable")[:k])
            assert np.array_equal(got[r], want), (r, k)
            assert math.isnan(float(tail[r])) or k == v
