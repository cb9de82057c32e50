"""Oracle of a layer's head norms (test infrastructure).

``head_norm``: the norm of heads as the append defines it: the mean of the
squares and the root of it in 64 bits, rounded to fp32 once, then two products
rounded one by one.
"""

from __future__ import annotations

import numpy as np


def head_norm(x, weight, eps):
    """x [..., d] fp32; weight [d] (fp32 values) or None; fp32 [..., d]."""
    y = np.asarray(x, np.float32)
    z = y.astype(np.float64)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        mean = (z * z).sum(-1, keepdims=True) / z.shape[-1]
        r = (1.0 / np.sqrt(mean + np.float64(np.float32(eps)))).astype(np.float32)
        y = y * r
        return y if weight is None else y * np.asarray(weight, np.float32)
