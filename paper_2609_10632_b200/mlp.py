"""Device-buffer holder for one pre-norm MLP block over the rows (pixels, tokens) of a matrix:

    h = LayerNorm(x);  z = h w1^T + b1;  a = act(z);  y = x + a w2^T + b2

allocates torch tensors and calls the C ABI (include/nb_norm.h, nb_linear.h, nb_adamw.h); no arithmetic happens here.  The
counterpart of ``block.CbsBlock`` for the products, the norm and the optimiser of MLP blocks.
"""
from __future__ import annotations

import torch

from . import binding as nb


class MlpBlock:
    """All tensors of one block on one device: fp32 master parameters, working copies in the activations' type, gradients;
    forward(), backward() and the items of an AdamWPlan."""

    PARAMS = ("w1", "w2", "gamma", "beta", "b1", "b2")
    GROUPS = (0, 0, 1, 2, 2, 2)  # weights (decayed), norm gains, biases

    def __init__(self, rows, channels, hidden, dtype=nb.NB_DTYPE_BF16, act=nb.NB_ACT_GELU, eps=1e-5, device=0):
        self.rows, self.c, self.hidden, self.dtype, self.act, self.eps = rows, channels, hidden, dtype, act, eps
        self.dev = torch.device("cuda", device)
        self.t = {nb.NB_DTYPE_F32: torch.float32, nb.NB_DTYPE_BF16: torch.bfloat16, nb.NB_DTYPE_F16: torch.float16}[dtype]
        e = lambda *sz, dtype=torch.float32: torch.empty(*sz, dtype=dtype, device=self.dev)  # noqa: E731
        self.up, self.down = nb.LinearPlan(channels, hidden, dtype, device), nb.LinearPlan(hidden, channels, dtype, device)
        shapes = dict(w1=(hidden, channels), w2=(channels, hidden), gamma=(channels,), beta=(channels,), b1=(hidden,), b2=(channels,))
        self.param = {k: e(*shapes[k]) for k in self.PARAMS}
        self.grad = {k: e(*shapes[k]) for k in self.PARAMS}
        # what the products read: the masters themselves in fp32, else 16-bit copies that the optimiser rewrites
        self.copy = {k: self.param[k] if dtype == nb.NB_DTYPE_F32 else e(*shapes[k], dtype=self.t) for k in ("w1", "w2")}
        a = lambda n: e(rows, n, dtype=self.t)  # noqa: E731
        self.x, self.h, self.y, self.dy, self.dh, self.dx = (a(channels) for _ in range(6))
        self.z, self.a, self.dz = (a(hidden) for _ in range(3))
        self.mean, self.rstd = e(rows), e(rows)
        need = max(self.up.workspace_bytes(rows), self.down.workspace_bytes(rows))
        with torch.cuda.device(self.dev):
            need = max(need, nb.nb_layer_norm_workspace_bytes(rows, channels))
        self.ws = torch.empty(need, dtype=torch.uint8, device=self.dev)

    def load(self, **params):
        """Copies parameters in and makes the working copies."""
        for k, v in params.items():
            self.param[k].copy_(v)
            if k in self.copy and self.copy[k] is not self.param[k]:
                self.copy[k].copy_(self.param[k])

    def forward(self, stream=None):
        with torch.cuda.device(self.dev):  # (the norm's calls have no plan: they run on the current device)
            self._forward(stream)

    def backward(self, stream=None):
        """All gradients and dx from dy; the gradient of the residual joins in the norm's backward pass."""
        with torch.cuda.device(self.dev):
            self._backward(stream)

    def poll(self, stream=None):
        """Waits for the stream and raises where a product gave up a wait; returns a note where fp16 results of one saturated, else ""."""
        notes = [(name, plan.poll(stream)) for name, plan in (("up", self.up), ("down", self.down))]
        return "; ".join(f"{name}: {note}" for name, note in notes if note)

    def _forward(self, stream):
        p = self.param
        nb.nb_layer_norm_fwd(self.dtype, self.rows, self.c, self.x, p["gamma"], p["beta"], self.eps, self.h, self.mean, self.rstd, stream=stream)
        nb.nb_linear_fwd(self.up, self.rows, self.h, self.copy["w1"], p["b1"], self.act, self.a, self.ws, z=self.z, stream=stream)
        nb.nb_linear_fwd(self.down, self.rows, self.a, self.copy["w2"], p["b2"], nb.NB_ACT_NONE, self.y, self.ws, res=self.x, stream=stream)

    def _backward(self, stream):
        g = self.grad
        nb.nb_linear_bwd_weight(self.down, self.rows, self.a, self.dy, g["w2"], g["b2"], self.ws, stream=stream)
        nb.nb_linear_bwd_data(self.down, self.rows, self.dy, self.copy["w2"], self.dz, self.ws, z_in=self.z, act_in=self.act, stream=stream)
        nb.nb_linear_bwd_weight(self.up, self.rows, self.h, self.dz, g["w1"], g["b1"], self.ws, stream=stream)
        nb.nb_linear_bwd_data(self.up, self.rows, self.dz, self.copy["w1"], self.dh, self.ws, stream=stream)
        nb.nb_layer_norm_bwd(self.dtype, self.rows, self.c, self.dh, self.x, self.param["gamma"], self.mean, self.rstd, self.dx, g["gamma"], g["beta"], self.ws, add=self.dy,
                             stream=stream)

    def optimizer_items(self, bits=32):
        """Items of an AdamWPlan over the block's parameters; moments in `bits` (8: the two weight matrices only)."""
        items = []
        for k, group in zip(self.PARAMS, self.GROUPS):
            p, c = self.param[k], self.copy.get(k)
            c = None if c is p else c
            if bits == 8 and group == 0:
                m, v = (torch.zeros(p.numel(), dtype=torch.float8_e4m3fn, device=self.dev) for _ in range(2))
                items.append((self.grad[k], p, m, v, c, group) + tuple(torch.zeros(-(-p.numel() // 128), device=self.dev) for _ in range(2)))
            else:
                items.append((self.grad[k], p, torch.zeros_like(p), torch.zeros_like(p), c, group))
        return items
