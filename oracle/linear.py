"""fp64 CPU oracle of the MLP products: z = x w^T + bias, out = act(z) + res, and their gradients (TEST INFRASTRUCTURE ONLY,
shares nothing with the CUDA library).  act: "none", "silu" z*sigmoid(z), "gelu" z*Phi(z) with Phi the normal distribution
function."""
from __future__ import annotations

import numpy as np
from scipy.special import expit, ndtr


def act(z, kind: str):
    z = np.asarray(z, dtype=np.float64)
    return z * expit(z) if kind == "silu" else z * ndtr(z) if kind == "gelu" else z


def act_grad(z, kind: str):
    z = np.asarray(z, dtype=np.float64)
    if kind == "silu":
        return expit(z) * (1.0 + z * expit(-z))
    if kind == "gelu":
        return ndtr(z) + z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
    return np.ones_like(z)


def linear_fwd(x, w, bias=None, kind: str = "none", res=None):
    """(z, out)."""
    z = np.asarray(x, dtype=np.float64) @ np.asarray(w, dtype=np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, dtype=np.float64)
    out = act(z, kind)
    return z, out if res is None else out + np.asarray(res, dtype=np.float64)


def linear_bwd_data(dy, w, z_in=None, kind: str = "none", add=None):
    dx = np.asarray(dy, dtype=np.float64) @ np.asarray(w, dtype=np.float64)
    if add is not None:
        dx = dx + np.asarray(add, dtype=np.float64)
    return dx if z_in is None else dx * act_grad(z_in, kind)


def linear_bwd_weight(x, dy):
    """(dw, dbias)."""
    dy = np.asarray(dy, dtype=np.float64)
    return dy.T @ np.asarray(x, dtype=np.float64), dy.sum(0)
