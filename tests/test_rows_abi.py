"""C entry points of the row operators on the CPU: sizes and arguments are
checked on the host before any GPU work (no call here reaches the GPU)."""
import ctypes
import math

import pytest

import paper_2010_10458_amd as tk

VP = ctypes.c_void_p


def make(kind, *args):
    h = VP()
    rc = getattr(tk.lib(), f"tkef_{kind}_plan_create")(*args, ctypes.byref(h))
    return rc, h


def info(kind, h):
    ws = ctypes.c_size_t()
    assert getattr(tk.lib(), f"tkef_{kind}_plan_info")(h, ctypes.byref(ws)) == tk.OK
    return ws.value


LIST = dict(rows=8, vocab=1000, k=16, dtype=tk.DTYPE_BF16, val=tk.VAL_F32, t=1.0)


@pytest.mark.parametrize("kind", ["top", "distill"])
@pytest.mark.parametrize("change,code", [
    ({}, tk.OK), (dict(rows=1, vocab=1, k=1), tk.OK), (dict(rows=1 << 20), tk.OK),
    (dict(vocab=1 << 20, k=1024), tk.OK), (dict(t=1e-6), tk.OK), (dict(t=1e6), tk.OK),
    (dict(rows=0), tk.ERANGE), (dict(rows=(1 << 20) + 1), tk.ERANGE), (dict(rows=-1), tk.ERANGE),
    (dict(vocab=0), tk.ERANGE), (dict(vocab=(1 << 20) + 1), tk.ERANGE),
    (dict(k=0), tk.ERANGE), (dict(k=1001), tk.ERANGE), (dict(vocab=5000, k=1025), tk.ERANGE),
    (dict(t=0.0), tk.ERANGE), (dict(t=-1.0), tk.ERANGE), (dict(t=math.nan), tk.ERANGE),
    (dict(t=math.inf), tk.ERANGE), (dict(dtype=3), tk.EINVAL), (dict(val=2), tk.EINVAL)])
def test_list_plans(kind, change, code):
    a = {**LIST, **change}
    rc, h = make(kind, a["rows"], a["vocab"], a["k"], a["dtype"], a["val"], a["t"])
    assert rc == code
    assert bool(h.value) == (code == tk.OK)
    if code == tk.OK:
        info(kind, h)
        assert getattr(tk.lib(), f"tkef_{kind}_plan_destroy")(h) == tk.OK


@pytest.mark.parametrize("args,code", [
    ((4, 3, 100, tk.DTYPE_F32, 1.0), tk.OK), ((32768, 1, 100, tk.DTYPE_F32, 1.0), tk.OK),
    ((1, 63, 1 << 20, tk.DTYPE_F32, 1.0), tk.OK), ((32769, 1, 100, tk.DTYPE_F32, 1.0), tk.ERANGE),
    ((4, 0, 100, tk.DTYPE_F32, 1.0), tk.ERANGE), ((4, 64, 100, tk.DTYPE_F32, 1.0), tk.ERANGE),
    ((32768, 63, 1 << 17, tk.DTYPE_F32, 1.0), tk.ERANGE), ((0, 3, 100, tk.DTYPE_F32, 1.0), tk.ERANGE),
    ((4, 3, 100, 9, 1.0), tk.EINVAL)])
def test_verify_plans(args, code):
    rc, h = make("verify", *args)
    assert rc == code
    if code == tk.OK:
        assert info("verify", h) > 0
        assert tk.lib().tkef_verify_plan_destroy(h) == tk.OK


def test_null_plans_and_outputs():
    L = tk.lib()
    for kind in ("top", "distill", "verify"):
        assert getattr(L, f"tkef_{kind}_plan_destroy")(None) == tk.EINVAL
        assert getattr(L, f"tkef_{kind}_plan_info")(None, None) == tk.EINVAL
    assert L.tkef_top_plan_create(1, 10, 2, 0, 0, 1.0, None) == tk.EINVAL
    assert L.tkef_top_execute(None, 256, 10, 1, 256, 256, 256, None, 0, None, None) == tk.EINVAL


P = 1 << 20  # an address that nothing dereferences


def test_top_arguments():
    L = tk.lib()
    rc, h = make("top", 8, 1000, 16, tk.DTYPE_F32, tk.VAL_F16, 1.0)

    def call(z=P, ld=1000, rows=8, idx=P, val=P, tail=P, ws=None, nws=0):
        return L.tkef_top_execute(h, z, ld, rows, idx, val, tail, ws, nws, None, None)

    assert call(rows=0, z=None, idx=None, val=None) == tk.OK
    assert call(rows=9) == tk.ERANGE and call(rows=-1) == tk.ERANGE
    assert call(z=None) == tk.EINVAL and call(z=P + 2) == tk.EINVAL
    assert call(ld=999) == tk.EINVAL and call(ld=1 << 41) == tk.ERANGE
    assert call(idx=None) == tk.EINVAL and call(val=None) == tk.EINVAL
    assert call(idx=P + 2) == tk.EINVAL and call(val=P + 1) == tk.EINVAL
    assert call(tail=P + 1) == tk.EINVAL
    assert L.tkef_top_plan_destroy(h) == tk.OK
    # rows too long for one workgroup need a workspace
    rc, h = make("top", 8, 200_000, 64, tk.DTYPE_F32, tk.VAL_F32, 1.0)
    need = info("top", h)
    assert need > 0
    for ws, n in ((None, need), (P, need - 1), (P + 128, need)):
        assert L.tkef_top_execute(h, P, 200_000, 8, P, P, P, ws, n, None, None) == tk.EWORKSPACE
    assert L.tkef_top_plan_destroy(h) == tk.OK


def test_distill_arguments():
    L = tk.lib()
    rc, h = make("distill", 8, 1000, 16, tk.DTYPE_BF16, tk.VAL_F32, 1.0)
    far = P + (1 << 24)

    def step(z=P, ld=1000, rows=8, idx=P, val=P, tail=None, count=None, weight=None, loss=P,
             grad=far, gld=1000):
        return L.tkef_distill_step(h, z, ld, rows, idx, val, tail, count, weight, loss, grad, gld,
                                   None, 0, None, None)

    assert step(rows=0) == tk.OK
    for bad in (dict(idx=None), dict(val=None), dict(loss=None), dict(grad=None), dict(z=P + 1),
                dict(grad=far + 1), dict(gld=999), dict(tail=P + 2), dict(count=P + 2),
                dict(weight=P + 1), dict(val=P + 2), dict(loss=P + 2),
                dict(grad=P + 2000),                # overlaps the logits
                dict(grad=P, gld=1001)):            # the same address, other rows
        assert step(**bad) == tk.EINVAL, bad
    assert step(gld=1 << 41) == tk.ERANGE

    def backward(stats=P, dloss=None):
        return L.tkef_distill_backward(h, P, 1000, 8, P, P, None, None, None, stats, dloss, far,
                                       1000, None, 0, None, None)

    assert backward(stats=None) == tk.EINVAL and backward(stats=P + 8) == tk.EINVAL
    assert backward(dloss=P + 1) == tk.EINVAL
    assert L.tkef_distill_forward(h, P, 1000, 8, P, P, None, None, None, P, P + 4, None, 0, None,
                                  None) == tk.EINVAL
    assert L.tkef_distill_plan_destroy(h) == tk.OK


def test_verify_arguments():
    L = tk.lib()
    rc, h = make("verify", 4, 3, 500, tk.DTYPE_F16, 1.0)
    need = info("verify", h)
    ok = dict(t=P, tb=2000, ti=500, d=P, db=1500, di=500, b=4, tok=P, u=P, e=P, eld=500, length=None,
              acc=P, out=P, logp=P, ws=P, n=need)

    def call(**kw):
        a = {**ok, **kw}
        return L.tkef_verify_execute(h, a["t"], a["tb"], a["ti"], a["d"], a["db"], a["di"], a["b"],
                                     a["tok"], a["u"], a["e"], a["eld"], a["length"], a["acc"],
                                     a["out"], a["logp"], a["ws"], a["n"], None, None)

    assert call(b=0) == tk.OK and call(b=5) == tk.ERANGE
    for bad in (dict(t=None), dict(d=None), dict(ti=499), dict(di=499), dict(tb=-1), dict(db=-1),
                dict(eld=499), dict(tok=None), dict(u=None), dict(e=None), dict(acc=None),
                dict(out=None), dict(t=P + 1), dict(e=P + 2), dict(length=P + 2),
                dict(logp=P + 2)):
        assert call(**bad) == tk.EINVAL, bad
    assert call(tb=1 << 41) == tk.ERANGE and call(eld=1 << 41) == tk.ERANGE
    for bad in (dict(ws=None), dict(n=need - 1), dict(ws=P + 64)):
        assert call(**bad) == tk.EWORKSPACE
    assert L.tkef_verify_plan_bind(None, P, need, None) == tk.EINVAL
    assert L.tkef_verify_plan_bind(h, None, need, None) == tk.EWORKSPACE
    assert L.tkef_verify_plan_destroy(h) == tk.OK
