"""The operators of an MLP block run together, as a training step calls them: norm, two products, their gradients, AdamW.

fp32 against the fp64 oracles composed the same way: every tensor to a relative L2 of 1e-5 (the bar of the other fp32 tests: a few
hundred roundings of 2^-24 in a row).  16 bits: the oracle is composed from the values that the GPU stored in between (h, a, z, dz,
dh), so that each step stands for itself: results that are rounded to 16 bits to one such rounding's relative L2, fp32 sums
of 16-bit products to 1e-5."""
import numpy as np
import pytest

from oracle import adamw as oadam
from oracle import linear as olin
from oracle import norm as onorm

pytestmark = pytest.mark.gpu
ACT = {1: "silu", 2: "gelu"}


def _rel(got, want):
    got = got.double().cpu().numpy().reshape(want.shape)
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))


def _block(rows, c, hidden, dtype, act, seed):
    import torch

    from paper_2609_10632_b200.mlp import MlpBlock

    b = MlpBlock(rows, c, hidden, dtype, act)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    b.load(w1=r(hidden, c) * c**-0.5, w2=r(c, hidden) * hidden**-0.5, gamma=1 + 0.2 * r(c), beta=0.1 * r(c), b1=0.1 * r(hidden), b2=0.1 * r(c))
    b.x.copy_(r(rows, c))
    b.dy.copy_(0.1 * r(rows, c))
    return b


def _f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("rows, c, hidden, dtype, act", [(50, 24, 96, 0, 2), (333, 96, 384, 1, 2), (1000, 64, 200, 2, 1), (77, 50, 201, 1, 2), (3, 128, 512, 1, 1), (600, 333, 999, 2, 2)])
def test_forward_and_backward_of_a_block(rows, c, hidden, dtype, act):
    import torch

    b = _block(rows, c, hidden, dtype, act, rows)
    b.forward()
    b.backward()
    torch.cuda.synchronize()
    b.up.poll()
    b.down.poll()
    p = {k: _f64(v) for k, v in b.param.items()}
    w1, w2, x, dy = _f64(b.copy["w1"]), _f64(b.copy["w2"]), _f64(b.x), _f64(b.dy)
    stored = lambda name, want: want if dtype == 0 else _f64(getattr(b, name))  # noqa: E731  (what the next step read)
    h, mean, rstd = onorm.layer_norm_fwd(x, p["gamma"], p["beta"], b.eps)
    z, a = olin.linear_fwd(stored("h", h), w1, p["b1"], ACT[act])
    _, y = olin.linear_fwd(stored("a", a), w2, p["b2"], "none", x)
    dw2, db2 = olin.linear_bwd_weight(stored("a", a), dy)
    dz = olin.linear_bwd_data(dy, w2, stored("z", z), ACT[act])
    dw1, db1 = olin.linear_bwd_weight(stored("h", h), stored("dz", dz))
    dh = olin.linear_bwd_data(stored("dz", dz), w1)
    dx, dgamma, dbeta = onorm.layer_norm_bwd(stored("dh", dh), x, p["gamma"], mean, rstd)
    dx = dx + dy
    one = 1e-5 if dtype == 0 else torch.finfo(b.t).eps / 2
    # (the activations of 16-bit types are approximated within 2.8e-4 |z|: see the products' own test)
    for name, want in (("h", h), ("z", z), ("a", a), ("y", y), ("dz", dz), ("dh", dh), ("dx", dx)):
        assert _rel(getattr(b, name), want) <= one + (5e-4 if dtype and name in ("a", "dz") else 0.0) + 1e-6, name
    for name, want in (("w1", dw1), ("w2", dw2), ("b1", db1), ("b2", db2), ("gamma", dgamma), ("beta", dbeta)):
        assert _rel(b.grad[name], want) <= 1e-5, name


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_training_step(bits):
    """Forward, backward and the optimiser's step recorded once and replayed: the parameters follow those of steps called one by one,
    bit for bit, and the first step is the oracle's."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    def make():
        b = _block(256, 64, 256, nb.NB_DTYPE_BF16, nb.NB_ACT_GELU, 5)
        items = b.optimizer_items(bits)
        plan = nb.AdamWPlan(items)
        ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
        plan.upload(ws)
        step = torch.zeros(1, dtype=torch.int64, device="cuda")

        def go():
            b.forward()
            b.backward()
            plan.step(ws, step, [1e-3] * 3, [0.1, 0.0, 0.0], 0.9, 0.999, 1e-8, 1.0)

        return b, go, step, (items, plan, ws)

    a, go_a, step_a, _a = make()
    before = {k: _f64(v) for k, v in a.param.items()}
    go_a()
    torch.cuda.synchronize()
    names = a.PARAMS
    ps, *_ = oadam.clip_adamw_step([before[k].reshape(-1) for k in names], [_f64(a.grad[k]).reshape(-1) for k in names], [np.zeros(before[k].size) for k in names],
                                   [np.zeros(before[k].size) for k in names], a.GROUPS, 1, [1e-3] * 3, [0.1, 0.0, 0.0], 0.9, 0.999, 1e-8, 1.0)
    for k, want in zip(names, ps):
        assert _rel(a.param[k], want) <= 1e-5, k
    for _ in range(3):
        go_a()
    b, go_b, step_b, _b = make()
    go_b()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        go_b()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert int(step_a) == int(step_b) == 4
    for k in names:
        assert torch.equal(a.param[k], b.param[k]), k
        if k in a.copy:
            assert torch.equal(a.copy[k], b.copy[k]) and torch.equal(a.copy[k], a.param[k].to(a.copy[k].dtype))
