"""Workspaces of the row operators on the CPU: which calls ask for one (no call
here reaches the GPU)."""
import ctypes
import weakref

import pytest
import torch

import paper_2010_10458_amd as tk

P = 1 << 20  # an address that nothing dereferences


def test_the_gradient_asks_for_no_workspace():
    """Of a plan whose losses need one; the call ends at the missing statistics."""
    L = tk.lib()
    h, ws = ctypes.c_void_p(), ctypes.c_size_t()
    assert L.tkef_distill_plan_create(8, 200_000, 64, tk.DTYPE_F32, tk.VAL_F32, 1.0,
                                      ctypes.byref(h)) == tk.OK
    assert L.tkef_distill_plan_info(h, ctypes.byref(ws)) == tk.OK and ws.value > 0
    far = P + (1 << 24)
    lists = (P, P, None, None, None)
    assert L.tkef_distill_forward(h, P, 200_000, 8, *lists, P, None, None, 0, None,
                                  None) == tk.EWORKSPACE
    assert L.tkef_distill_backward(h, P, 200_000, 8, *lists, None, None, far, 200_000, None, 0,
                                   None, None) == tk.EINVAL
    assert L.tkef_distill_plan_destroy(h) == tk.OK


@pytest.mark.parametrize("make", [
    lambda: tk.TopLogitsPlan(8192, 32000, 512, dtype=torch.bfloat16),
    lambda: tk.DistillPlan(1 << 16, 128_000, 64, dtype=torch.bfloat16)])
def test_large_scratch_is_given_back_after_the_call(make):
    """The lists of 8,192 rows of 32,000 words, k = 512, take 0.5 GB: a plan keeps none of
    it, on however many streams it is used."""
    plan = make()
    assert plan.ws_bytes > 1 << 20
    plan.ws_bytes = 4096
    held = [plan._workspace(stream, "cpu") for stream in (None, 7, 9)]
    assert len({t.data_ptr() for t in held}) == 3 and all(t.numel() == 4096 for t in held)
    gone = [weakref.ref(t) for t in held]
    del held
    assert all(g() is None for g in gone)
