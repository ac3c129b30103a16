"""fp64 CPU oracle of layer norm over the last axis, forward and backward (TEST INFRASTRUCTURE ONLY, shares nothing with the
CUDA library).

  mean = avg(x); rstd = (avg((x-mean)^2) + eps)^-1/2; xhat = (x-mean)*rstd; y = gamma*xhat + beta
  with g = dL/dy, d = g*gamma:  dx = rstd*(d - avg(d) - xhat*avg(d*xhat)); dgamma = sum g*xhat; dbeta = sum g over the rows
"""
from __future__ import annotations

import numpy as np


def layer_norm_fwd(x, gamma, beta, eps: float):
    """(y, mean, rstd) in fp64; gamma / beta may be None."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(-1)
    d = x - mean[..., None]
    rstd = 1.0 / np.sqrt((d * d).mean(-1) + eps)
    y = d * rstd[..., None]
    if gamma is not None:
        y = y * np.asarray(gamma, dtype=np.float64)
    if beta is not None:
        y = y + np.asarray(beta, dtype=np.float64)
    return y, mean, rstd


def layer_norm_bwd(g, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) in fp64 from the given statistics."""
    g, x = np.asarray(g, dtype=np.float64), np.asarray(x, dtype=np.float64)
    mean, rstd = np.asarray(mean, dtype=np.float64)[..., None], np.asarray(rstd, dtype=np.float64)[..., None]
    xhat = (x - mean) * rstd
    d = g if gamma is None else g * np.asarray(gamma, dtype=np.float64)
    dx = rstd * (d - d.mean(-1, keepdims=True) - xhat * (d * xhat).mean(-1, keepdims=True))
    rows = tuple(range(g.ndim - 1))
    return dx, (g * xhat).sum(rows), g.sum(rows)
