"""Workspaces of the row operators on the CPU: which calls ask for one (no call
here reaches the GPU)."""
import ctypes

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
