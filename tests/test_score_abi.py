"""Scores of tokens on the CPU: sizes, arguments, devices and workspaces are checked before any
GPU work (no call here reaches the GPU), and the oracle's pins."""
import ctypes
import math
import types

import numpy as np
import pytest
import torch

import paper_2010_10458_amd as tk
from oracle import score as oracle
from test_rows_devices import OnGpu, current_gpu_is_the_first  # noqa: F401 (a fixture)

VP = ctypes.c_void_p
P = 1 << 20  # an address that nothing dereferences
FAR = P + (1 << 24)


def make(rows=8, vocab=1000, k=16, dtype=tk.DTYPE_BF16, t=1.0):
    h = VP()
    return tk.lib().tkef_score_plan_create(rows, vocab, k, dtype, t, ctypes.byref(h)), h


def size(h):
    ws = ctypes.c_size_t()
    assert tk.lib().tkef_score_plan_info(h, ctypes.byref(ws)) == tk.OK
    return ws.value


@pytest.mark.parametrize("change,code", [
    ({}, tk.OK), (dict(rows=1, vocab=1, k=1), tk.OK), (dict(k=0), tk.OK), (dict(rows=1 << 20), tk.OK),
    (dict(vocab=1 << 20, k=64), tk.OK), (dict(t=1e-6), tk.OK), (dict(t=1e6), tk.OK),
    (dict(rows=0), tk.ERANGE), (dict(rows=(1 << 20) + 1), tk.ERANGE), (dict(vocab=0), tk.ERANGE),
    (dict(vocab=(1 << 20) + 1), tk.ERANGE), (dict(k=-1), tk.ERANGE), (dict(k=65), tk.ERANGE),
    (dict(vocab=10, k=11), tk.ERANGE), (dict(t=0.0), tk.ERANGE), (dict(t=math.nan), tk.ERANGE),
    (dict(t=math.inf), tk.ERANGE), (dict(dtype=3), tk.EINVAL), (dict(dtype=-1), tk.EINVAL)])
def test_plans(change, code):
    rc, h = make(**change)
    assert rc == code and bool(h.value) == (code == tk.OK)
    if code == tk.OK:
        assert size(h) % 256 == 0
        assert tk.lib().tkef_score_plan_destroy(h) == tk.OK


def test_null_plans():
    L = tk.lib()
    assert L.tkef_score_plan_destroy(None) == tk.EINVAL
    assert L.tkef_score_plan_info(None, None) == tk.EINVAL
    assert L.tkef_score_plan_create(1, 10, 2, 0, 1.0, None) == tk.EINVAL
    assert L.tkef_score_forward(None, P, 10, 1, P, P, P, P, P, P, None, 0, None, None) == tk.EINVAL
    assert L.tkef_score_backward(None, P, 10, 1, P, P, P, P, FAR, 10, None, None) == tk.EINVAL


def test_forward_arguments():
    L = tk.lib()
    _, h = make(dtype=tk.DTYPE_F32)

    def call(z=P, ld=1000, rows=8, tok=P, logp=P, ent=P, idx=P, val=P, stats=P, ws=None, n=0,
             status=None):
        return L.tkef_score_forward(h, z, ld, rows, tok, logp, ent, idx, val, stats, ws, n, status,
                                    None)

    assert call(rows=0, z=None, tok=None, logp=None) == tk.OK
    assert call(rows=9) == tk.ERANGE and call(rows=-1) == tk.ERANGE
    assert call(ld=1 << 41) == tk.ERANGE
    for bad in (dict(z=None), dict(z=P + 2), dict(ld=999), dict(tok=None), dict(logp=None),
                dict(idx=None), dict(val=None), dict(tok=P + 2), dict(logp=P + 1), dict(ent=P + 2),
                dict(idx=P + 1), dict(val=P + 2), dict(stats=P + 8), dict(status=P + 1)):
        assert call(**bad) == tk.EINVAL, bad
    assert L.tkef_score_plan_destroy(h) == tk.OK
    _, h = make(vocab=200_000, dtype=tk.DTYPE_F32)
    need = size(h)
    assert need > 0
    for ws, n in ((None, need), (P, need - 1), (P + 128, need)):
        assert call(ld=200_000, ws=ws, n=n) == tk.EWORKSPACE
    assert L.tkef_score_plan_destroy(h) == tk.OK


def test_backward_arguments():
    L = tk.lib()
    _, h = make(dtype=tk.DTYPE_BF16)

    def call(z=P, ld=1000, rows=8, tok=P, stats=P, dl=P, dh=P, grad=FAR, gld=1000, status=None):
        return L.tkef_score_backward(h, z, ld, rows, tok, stats, dl, dh, grad, gld, status, None)

    assert call(rows=0) == tk.OK
    assert call(rows=9) == tk.ERANGE and call(gld=1 << 41) == tk.ERANGE
    for bad in (dict(z=None), dict(ld=999), dict(tok=None), dict(stats=None), dict(dl=None, dh=None),
                dict(grad=None), dict(grad=FAR + 1), dict(gld=999), dict(stats=P + 8),
                dict(dl=P + 2), dict(dh=P + 1), dict(tok=P + 3), dict(status=P + 2),
                dict(grad=P + 2000), dict(grad=P, gld=1001)):
        assert call(**bad) == tk.EINVAL, bad
    assert L.tkef_score_plan_destroy(h) == tk.OK


@pytest.mark.parametrize("dtype,vector", [(tk.DTYPE_F32, 4), (tk.DTYPE_F16, 8), (tk.DTYPE_BF16, 8)])
def test_stated_workspace(dtype, vector):
    """None up to 64 KB a row; beyond, 16 bytes for each 32 KB, or 16 + 8 k for each 64 KB."""
    rows = 1000
    for v in (1, 4096 * vector, 4096 * vector + vector, 131071, 262147, 1 << 20):
        for k in (0, 1, 20, 64):
            if k > v:
                continue
            _, h = make(rows=rows, vocab=v, k=k, dtype=dtype)
            vecs = v // vector
            if vecs <= 4096:
                assert size(h) == 0
            else:
                most = max(16 * -(-vecs // 2048), (16 + 8 * k) * -(-vecs // 4096))
                assert 0 < size(h) <= rows * most + 512
            tk.lib().tkef_score_plan_destroy(h)


def call(which, gpu=0, stream=None, **other):
    p = tk.ScorePlan(4, 100, 8, dtype=torch.float32)
    kw = dict(logits=(4, 100), tokens=(4,))
    if which == "execute":
        kw.update(logp_out=(4,), entropy_out=(4,), idx_out=(4, 8), val_out=(4, 8))
    elif which == "forward":
        kw.update(logp_out=(4,), entropy_out=(4,), stats_out=(4, 4))
    else:
        kw.update(stats=(4, 4), dlogp=(4,), dentropy=(4,), grad_out=(4, 100))
    ints = ("tokens", "idx_out")
    return getattr(p, which)(stream=stream, **{
        k: OnGpu(v, torch.int32 if k in ints else torch.float32, other.get(k, gpu))
        for k, v in kw.items()})


@pytest.mark.parametrize("which", ["execute", "forward", "backward"])
def test_devices(which):
    with pytest.raises(ValueError, match="cuda:1.*stream is on cuda:0"):
        call(which, gpu=1)
    with pytest.raises(ValueError, match="cuda:0.*stream is on cuda:1"):
        call(which, stream=types.SimpleNamespace(device_index=1, cuda_stream=0))
    names = dict(execute=("tokens", "logp_out", "entropy_out", "idx_out", "val_out"),
                 forward=("tokens", "logp_out", "entropy_out", "stats_out"),
                 backward=("tokens", "stats", "dlogp", "dentropy", "grad_out"))[which]
    for name in names:
        with pytest.raises(ValueError, match=name):
            call(which, **{name: 1})


def test_tensors_of_other_types_and_shapes():
    p = tk.ScorePlan(4, 100, 8, dtype=torch.float32)
    z, t, s = OnGpu((4, 100)), OnGpu((4,), torch.int32), OnGpu((4, 4))
    for bad in (OnGpu((4,), torch.int64), OnGpu((5,), torch.int32), torch.zeros(4, dtype=torch.int32)):
        with pytest.raises(ValueError, match="tokens"):
            p.execute(z, bad)
    for bad in (OnGpu((5, 100)), OnGpu((4, 99)), OnGpu((4, 100), torch.float16), OnGpu((400,))):
        with pytest.raises(ValueError, match="logits"):
            p.execute(bad, t)
    with pytest.raises(ValueError, match="dlogp or dentropy"):
        p.backward(z, t, s)
    with pytest.raises(ValueError, match="grad_out"):
        p.backward(z, t, s, dlogp=OnGpu((4,)), grad_out=OnGpu((4, 101)))
    with pytest.raises(ValueError, match="idx_out"):
        p.execute(z, t, logp_out=OnGpu((4,)), entropy_out=OnGpu((4,)), idx_out=OnGpu((4, 8)))


def test_captured_calls_share_no_scratch(monkeypatch):
    state = [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state[0])
    plan = tk.ScorePlan(8, 200_000, 20, dtype=torch.float32)
    assert plan.ws_bytes > 0
    eager = plan._workspace(7, "cpu")
    assert plan._workspace(7, "cpu") is eager
    state[0] = True
    first, second = plan._workspace(7, "cpu"), plan._workspace(7, "cpu")
    assert len({w.data_ptr() for w in (eager, first, second)}) == 3


def test_oracle_pins():
    """Two words of probabilities 3/4 and 1/4; a uniform row; a masked one; ties."""
    x = np.log([3.0, 1.0])
    r = oracle.score(x, 1, 2)
    assert abs(r.logp - math.log(0.25)) < 1e-15
    assert abs(r.entropy - (0.75 * math.log(4 / 3) + 0.25 * math.log(4))) < 1e-15
    assert r.words.tolist() == [0, 1]
    g = oracle.score_gradient(x, 1, 2.0, 0.0)
    assert np.allclose(g, [-1.5, 1.5], atol=1e-15)
    # dH/dx_0 = -p_0 (log p_0 + H) = -p_0 p_1 (log p_0 - log p_1)
    g = oracle.score_gradient(x, 1, 0.0, 1.0, temperature=2.0)
    p = np.array([math.sqrt(3), 1]) / (math.sqrt(3) + 1)
    assert np.allclose(g, np.array([-1, 1]) * p[0] * p[1] * math.log(math.sqrt(3)) / 2, atol=1e-15)
    r = oracle.score(np.array([5.0, -math.inf, 5.0, 5.0, 5.0]), 1, 5)
    assert r.logp == -math.inf and abs(r.entropy - math.log(4)) < 1e-15
    assert r.words.tolist() == [0, 2, 3, 4, 1]
    assert math.isnan(oracle.score(np.full(3, -math.inf), 0, 1).logp)
    assert oracle.score(np.full(3, math.nan), -1, 1).logp == 0.0
