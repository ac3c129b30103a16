"""fp64 CPU oracle of the AdamW step: global-norm clipping over all gradient tensors, Adam moments with bias correction,
decoupled weight decay, and the moments' 8-bit form.

TEST INFRASTRUCTURE ONLY (same rules as the rest of this package; it shares nothing with the CUDA library).

  clip:   total = sqrt(sum of g^2 over everything);  g <- g * min(max_norm / (total + 1e-6), 1)
  update: m <- beta1*m + (1-beta1)*g;  v <- beta2*v + (1-beta2)*g^2
          p <- p - lr*weight_decay*p - lr * (m / (1-beta1^t)) / (sqrt(v / (1-beta2^t)) + eps)

8-bit form of a moment: 128 neighbours share the scale largest/448 and are held as e4m3 numbers (three fraction bits, exponents
-6 .. 8, subnormals down to 2^-9, no infinities, largest 448); the second moment is held as its root, and a root that is
not zero as at least 2^-9 of the scale.
"""
from __future__ import annotations

import numpy as np

from .optimizer import clip_global_norm

BLOCK = 128


def adamw_update(p, g, m, v, t: int, lr: float, beta1: float, beta2: float, eps: float, weight_decay: float):
    """One tensor, fp64; g is the (already clipped) gradient, t counts from 1.  Returns (p, m, v)."""
    p, g = np.asarray(p, dtype=np.float64), np.asarray(g, dtype=np.float64)
    m = beta1 * np.asarray(m, dtype=np.float64) + (1.0 - beta1) * g
    v = beta2 * np.asarray(v, dtype=np.float64) + (1.0 - beta2) * g * g
    mhat, vhat = m / (1.0 - beta1**t), v / (1.0 - beta2**t)
    return p - lr * weight_decay * p - lr * mhat / (np.sqrt(vhat) + eps), m, v


def clip_adamw_step(params, grads, ms, vs, groups, t, lr, weight_decay, beta1, beta2, eps, max_norm):
    """The whole step over a list of tensors (max_norm <= 0 or inf: no clipping).  Returns (params, ms, vs, total norm)."""
    clipped, total = clip_global_norm(grads, max_norm if 0.0 < max_norm < np.inf else np.inf)
    out = [adamw_update(p, g, m, v, t, lr[k], beta1, beta2, eps, weight_decay[k]) for p, g, m, v, k in zip(params, clipped, ms, vs, groups)]
    return [o[0] for o in out], [o[1] for o in out], [o[2] for o in out], total


def _e4m3_table():
    vals = [m * 2.0**-9 for m in range(8)]
    vals += [(8 + m) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8)]
    return np.array(vals[:-1])  # (the last pattern is NaN)


E4M3 = _e4m3_table()


def to_e4m3(u):
    """Nearest e4m3 number, ties to the even pattern, saturating."""
    u = np.asarray(u, dtype=np.float64)
    a = np.minimum(np.abs(u), 448.0)
    hi = np.clip(np.searchsorted(E4M3, a), 1, len(E4M3) - 1)
    lo = hi - 1
    dl, dh = a - E4M3[lo], E4M3[hi] - a
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.copysign(E4M3[pick], u)


def encode(x, root: bool):
    """(values of the codes, scales) of a tensor; `root`: x is a second moment's root."""
    x = np.asarray(x, dtype=np.float64).reshape(-1)
    n = x.size
    b = np.zeros((-(-n // BLOCK), BLOCK))
    b.reshape(-1)[:n] = x
    most = np.abs(b).max(1)
    some = most >= 2.0**-100
    up = np.where(some, 448.0 / np.where(some, most, 1.0), 0.0)
    u = b * up[:, None]
    if root:
        u = np.where((b > 0) & some[:, None], np.maximum(u, 2.0**-9), u)
    return to_e4m3(u).reshape(-1)[:n], np.where(some, most / 448.0, 0.0)


def decode(q, scale, root: bool):
    q = np.asarray(q, dtype=np.float64).reshape(-1)
    x = q * np.repeat(np.asarray(scale, dtype=np.float64), BLOCK)[: q.size]
    return x * x if root else x
