"""The caller's status word of the row operators on the CPU: kernels write it
with atomics, so its place and type are checked (no call here reaches the GPU)."""
import ctypes

import pytest
import torch

import paper_2010_10458_amd as tk

P = 1 << 20  # an address that nothing dereferences
FAR = P + (1 << 24)


def plan(kind, *args):
    h, ws = ctypes.c_void_p(), ctypes.c_size_t()
    assert getattr(tk.lib(), f"tkef_{kind}_plan_create")(*args, ctypes.byref(h)) == tk.OK
    assert getattr(tk.lib(), f"tkef_{kind}_plan_info")(h, ctypes.byref(ws)) == tk.OK
    return h, ws.value


@pytest.mark.parametrize("status", [P + 1, P + 2, P + 3])
def test_c_entry_points_refuse_a_misaligned_word(status):
    L = tk.lib()
    h, _ = plan("top", 8, 1000, 16, tk.DTYPE_F32, tk.VAL_F32, 1.0)
    assert L.tkef_top_execute(h, P, 1000, 8, P, P, P, None, 0, status, None) == tk.EINVAL
    L.tkef_top_plan_destroy(h)
    h, _ = plan("distill", 8, 1000, 16, tk.DTYPE_F32, tk.VAL_F32, 1.0)
    lists = (P, P, None, None, None)
    assert L.tkef_distill_forward(h, P, 1000, 8, *lists, P, None, None, 0, status,
                                  None) == tk.EINVAL
    assert L.tkef_distill_backward(h, P, 1000, 8, *lists, P, None, FAR, 1000, None, 0, status,
                                   None) == tk.EINVAL
    assert L.tkef_distill_step(h, P, 1000, 8, *lists, P, FAR, 1000, None, 0, status,
                               None) == tk.EINVAL
    L.tkef_distill_plan_destroy(h)
    h, ws = plan("verify", 4, 3, 500, tk.DTYPE_F16, 1.0)
    assert L.tkef_verify_execute(h, P, 2000, 500, P, 1500, 500, 4, P, P, P, 500, None, P, P, P, P,
                                 ws, status, None) == tk.EINVAL
    L.tkef_verify_plan_destroy(h)


@pytest.mark.parametrize("make", [
    lambda: tk.TopLogitsPlan(8, 1000, 16), lambda: tk.DistillPlan(8, 1000, 16),
    lambda: tk.VerifyPlan(4, 3, 500)])
def test_the_binding_refuses_other_tensors(make):
    p = make()
    assert p._status_of(None, "cpu") == (None, False)
    for bad in (torch.zeros(1, dtype=torch.int32),              # host memory
                torch.zeros(1, dtype=torch.int64), torch.zeros(1), torch.zeros(0)):
        with pytest.raises(ValueError, match="status"):
            p._status_of(bad, "cpu")
