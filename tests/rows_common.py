"""Shared by the row operators' GPU tests: inputs of the three types, derived
tolerances, comparisons against oracle/rows.py."""
import math

import numpy as np
import torch

from gpu_common import need_gpu

INF = math.inf
EPS = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# half a unit in the last place of a stored gradient, relative, and its smallest step
STORE = {"f32": (2.0 ** -24, 2.0 ** -149), "f16": (2.0 ** -11, 2.0 ** -25),
         "bf16": (2.0 ** -8, 2.0 ** -134)}


def rounding(v, biggest):
    """Relative error of a sum of v exponentials 2^(x a - c) held in 32 bits:
    each of 256 threads adds v / 256 terms one after the other and 8 levels
    join them; each exponential has its own rounding (4 units) and log2(e) /
    temperature is rounded once, which shifts an exponent by `biggest` = max
    |x| / temperature units. The factor 8 covers products and quotients of
    several such sums."""
    return EPS * (v / 256 + 64 + 8 * biggest)


def device_rows(x, dtype, pad=0, shift=0):
    """x (float64 numpy, n x v) as a CUDA tensor of `dtype` that is a view of
    rows `pad` elements longer, `shift` elements into its buffer (the gaps hold
    NaN), and its values as numpy float64."""
    dev = need_gpu()
    n, v = x.shape
    ld = v + pad
    buf = torch.full((shift + n * ld,), math.nan, dtype=TYPES[dtype], device=dev)
    view = buf[shift:].view(n, ld)[:, :v]
    view.copy_(torch.from_numpy(x).to(TYPES[dtype]))
    return view, view.double().cpu().numpy()


def logits(rng, n, v, spread=3.0):
    return rng.normal(size=(n, v)) * spread


def finite_max(*arrays):
    """Largest magnitude among logits that are not a mask: words at a type's
    lowest value have no probability beside others and differ by nothing among
    themselves, so their magnitude rounds nothing."""
    best = 0.0
    for a in arrays:
        a = np.abs(np.asarray(a, dtype=np.float64))
        a = a[a < 6e4]
        best = max(best, float(a.max()) if a.size else 0.0)
    return best


def vec(a, dtype=torch.float32):
    return torch.as_tensor(np.asarray(a)).to(dtype).to(need_gpu())
