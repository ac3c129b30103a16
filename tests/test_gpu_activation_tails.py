"""SiLU and GELU of the 16-bit tensor-core products over z in [-8, 8], and their derivatives: errors relative to the VALUE.

Identity weights hand the activation a z without rounding (one product that is not zero).  u = half a step of the type, t = |z|:
  out  u|out| + a|out|;    GELU a = 2^-15: the fit's 1.3e-5, the exponent -t^2/2 in base 2 (46 at t = 8, three roundings of 2^-24 each: 5.7e-6
                           of the value), ex2 2^-22, 1/x 2^-23 through five powers, ten roundings of the polynomial: below 2.2e-5
                           SiLU a = 2^-18: the exponent (11.5 at t = 8, two roundings: 9.5e-7), ex2, 1/x, the sum: below 1.8e-6
  dx   u|dx| + a (summands' magnitudes) + 2^-22:  Phi(z) and z phi(z) of opposite signs; s and s z (1 - s)
fp16 values below 2^-14 have steps of 2^-24: 2^-25 on top (twice: SiLU's factors)."""
import numpy as np
import pytest
from scipy.special import expit, ndtr

from oracle import linear as ora

pytestmark = pytest.mark.gpu
KIND = {"silu": 1, "gelu": 2}


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n, rows", [(64, 512), (256, 128), (384, 130)])
def test_tails_of_the_activations(n, rows, dtype, kind):
    import torch

    from paper_2609_10632_b200 import binding as nb

    dt, code = (torch.bfloat16, nb.NB_DTYPE_BF16) if dtype == "bf16" else (torch.float16, nb.NB_DTYPE_F16)
    z = torch.linspace(-8, 8, rows * n, device="cuda").to(dt).view(rows, n)
    plan = nb.LinearPlan(n, n, code)
    assert plan.paths(rows)["fwd"] == 1 and plan.paths(rows)["data"] == 1
    ws = torch.empty(plan.workspace_bytes(rows), dtype=torch.uint8, device="cuda")
    eye, out, dx = torch.eye(n, device="cuda").to(dt), torch.empty_like(z), torch.empty_like(z)
    hz = z.double().cpu().numpy()
    t, u, a, tiny = np.abs(hz), torch.finfo(dt).eps / 2, 2.0**-15 if kind == "gelu" else 2.0**-18, 2.0**-24 if dtype == "f16" else 0.0
    nb.nb_linear_fwd(plan, rows, z, eye, None, KIND[kind], out, ws)
    nb.nb_linear_bwd_data(plan, rows, torch.ones_like(z), eye, dx, ws, z_in=z, act_in=KIND[kind])
    plan.poll()
    want, got = ora.act(hz, kind), out.double().cpu().numpy()
    off = np.abs(got - want) / (u * np.abs(want) + a * np.abs(want) + tiny + 1e-30)
    assert off.max() <= 1, (off.max(), hz.reshape(-1)[off.argmax()])
    want, got = ora.act_grad(hz, kind), dx.double().cpu().numpy()
    if kind == "gelu":
        parts = np.where(hz < 0, ndtr(-t) + t * np.exp(-0.5 * t * t) / np.sqrt(2 * np.pi), 2.0)
    else:
        parts = expit(hz) * (1 + t)
    off = np.abs(got - want) / (u * np.abs(want) + a * parts + np.where(hz < 0, 0.0, 2.0**-22 * (1 + t)) + tiny + 1e-30)
    assert off.max() <= 1, (off.max(), hz.reshape(-1)[off.argmax()])


@pytest.mark.parametrize("dtype, n, rows, flags", [("bf16", 64, 128, 0), ("bf16", 64, 4, 0), ("bf16", 64, 128, 1), ("f32", 64, 128, 0), ("f32", 64, 4, 0), ("bf16", 63, 20, 0)])
def test_infinite_arguments_have_the_limits_values(dtype, n, rows, flags):
    """On every path: act(-inf) = 0, act(inf) = inf, act'(-inf) = 0, act'(inf) = 1; NaN stays; and the largest finite numbers likewise."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    dt, code = (torch.bfloat16, nb.NB_DTYPE_BF16) if dtype == "bf16" else (torch.float32, nb.NB_DTYPE_F32)
    inf, nan = float("inf"), float("nan")
    plan = nb.LinearPlan(n, n, code, flags=flags)
    ws = torch.empty(plan.workspace_bytes(rows), dtype=torch.uint8, device="cuda")
    v = torch.tensor([inf, -inf, nan, 3e38, -3e38, -200.0, 200.0, 0.0], device="cuda")
    for act in (nb.NB_ACT_SILU, nb.NB_ACT_GELU):
        x, w, out, dx = (torch.zeros(*s, device="cuda").to(dt) for s in ((rows, n), (n, n), (rows, n), (rows, n)))
        x[:, 0] = 1.0
        bias = torch.zeros(n, device="cuda")
        bias[:8] = v
        nb.nb_linear_fwd(plan, rows, x, w, bias, act, out, ws)
        want = torch.tensor([inf, 0.0, nan, 3e38, 0.0, 0.0, 200.0, 0.0], device="cuda").to(dt).expand(rows, 8)
        assert torch.equal(out[:, :8].nan_to_num(7.0, 8.0, 9.0), want.nan_to_num(7.0, 8.0, 9.0)) and out[:, 2].isnan().all(), act
        z = torch.zeros(rows, n, device="cuda").to(dt)
        z[:, :8] = v.to(dt)
        w.copy_(torch.eye(n, device="cuda"))
        for call in (lambda: nb.nb_linear_bwd_data(plan, rows, torch.ones_like(z), w, dx, ws, z_in=z, act_in=act), lambda: nb.nb_act_bwd(code, z.numel(), act, torch.ones_like(z), z, dx)):
            call()
            want = torch.tensor([1.0, 0.0, nan, 1.0, 0.0, 0.0, 1.0, 0.5], device="cuda").to(dt).expand(rows, 8)
            assert torch.equal(dx[:, :8].nan_to_num(7.0), want.nan_to_num(7.0)) and dx[:, 2].isnan().all(), (act, dx[0, :8])
