"""CPU oracle for the batched product with low-rank adapters.

TEST INFRASTRUCTURE ONLY: shares no code with the CUDA library and must not be reached from any
product path.  float64 numpy, one request at a time:
    Y[b] = W X[b] + scales[a] up[a] (down[a] X[b]),  a = which[b], none where a is outside 0 .. count - 1.
"""
from __future__ import annotations

import numpy as np


def adapters(X, down, up, which, ranks=None, scales=None):
    """The adapters' part of Y, and the same sum over absolute values (what an error is measured against)."""
    X, down, up = (np.asarray(a, np.float64) for a in (X, down, up))
    Y = np.zeros((len(X), up.shape[1]))
    scale = np.zeros_like(Y)
    for b, a in enumerate(which):
        if not 0 <= a < len(down):
            continue
        r = down.shape[1] if ranks is None else min(max(int(ranks[a]), 0), down.shape[1])
        s = 1.0 if scales is None else float(scales[a])
        Y[b] = s * (up[a, :, :r] @ (down[a, :r] @ X[b]))
        scale[b] = abs(s) * (np.abs(up[a, :, :r]) @ (np.abs(down[a, :r]) @ np.abs(X[b])))
    return Y, scale
