"""The operators of a pre-norm MLP block and of its training, as measured cases over the real range of their entry points.

Three operators:
  norm    layer norm over the channels of each row (pixel or token): forward, or forward and backward with the gradients of
          gamma and beta (nb_layer_norm_fwd / nb_layer_norm_bwd),
  linear  matrix product with bias, activation and residual in its epilogue; its data gradient, times the derivative of the
          activation in front of it; its weight and bias gradient (nb_linear_fwd / _bwd_data / _bwd_weight),
  adamw   one AdamW step over a list of tensors with global-norm clipping, moments in 32 bits or in 8 bits with one scale
          for each 128 elements (AdamWPlan).

`run` computes them in plain torch operations in 32 bits, or, where `own` is true, by the library's calls.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODE = {"f32": 0, "bf16": 1, "f16": 2}  # nb_dtype
ACT = {"none": 0, "silu": 1, "gelu": 2}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS_NORM = 1e-5
LR, WD, BETA1, BETA2, EPS, MAX_NORM, STEP = 2e-4, 0.05, 0.9, 0.999, 1e-8, 1.0, 40
BLOCK = 128  # elements that share a scale in the 8-bit form


# ------------------------------------------------------------------------------------------------ cases
def _norm(name, rows, c, dtype, train):
    return {"name": name, "kind": "norm", "rows": rows, "c": c, "dtype": dtype, "train": train}


def _linear(name, rows, c_in, c_out, dtype, way, act="none", res=False, save_z=False):
    """way: "fwd" (act and res are its epilogue's), "bwd" (act is that of the layer in front), "step" (forward, then backward)."""
    return {"name": name, "kind": "linear", "rows": rows, "c_in": c_in, "c_out": c_out, "dtype": dtype, "way": way, "act": act, "res": res, "save_z": save_z}


def _adamw(name, layers, c, hidden, bits, grad, copy):
    return {"name": name, "kind": "adamw", "layers": layers, "c": c, "hidden": hidden, "bits": bits, "grad": grad, "copy": copy}


def listed():
    return [
        # training on the pixels of 16 images at 160 x 160 (benchmark configuration 3's tensor): many short rows
        _norm("norm pixels", 409600, 96, "bf16", True),
        # long rows, as wide blocks have them, in the fp32 mode
        _norm("norm wide f32", 8192, 4096, "f32", True),
        # a channel count that no vector divides, a row count that no tile divides
        _norm("norm ragged f16", 5003, 1001, "f16", True),
        # serving a single token: the weights are what has to be read
        _linear("linear token", 1, 1024, 4096, "bf16", "fwd", "gelu"),
        # serving a small batch of ragged size, with a residual
        _linear("linear batch", 37, 1000, 520, "f16", "fwd", "silu", True),
        # first layer of an MLP over 16 x 40 x 40 pixels (benchmark configuration 4's rows and channels): forward in training
        _linear("linear up", 25600, 384, 1536, "bf16", "fwd", "gelu", False, True),
        # its second layer's backward pass: gradients of weight and bias, data gradient through the activation in front
        _linear("linear down bwd", 25600, 1536, 384, "bf16", "bwd", "gelu"),
        # a wide layer's whole training step: the largest case
        _linear("linear wide step", 16384, 4096, 4096, "bf16", "step", "none", True),
        # the fp32 mode that 16-bit runs are checked against
        _linear("linear f32 step", 1600, 384, 384, "f32", "step", "none", True),
        # the optimiser of one small block: few short tensors, latency counts
        _adamw("adamw one block", 1, 96, 384, 32, "f32", "bf16"),
        # 12 blocks of 384 channels, 14 million parameters, moments in 32 bits, gradients as the backward calls write them
        _adamw("adamw 12 blocks", 12, 384, 1536, 32, "f32", "bf16"),
        # 12 blocks of 1024 channels, 101 million parameters, moments in 8 bits, 16-bit gradients
        _adamw("adamw 8 bit", 12, 1024, 4096, 8, "bf16", "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "linear", "linear", "adamw"])
    if kind == "norm":
        c = _log(rng, 16, 8192)
        c = c if rng.random() < 0.3 else 8 * max(1, c // 8)
        rows = _log(rng, 1, min(400000, 60_000_000 // c))
        r = _norm("", rows, c, rng.choice(["bf16", "f16", "f32"]), rng.random() < 0.7)
    elif kind == "linear":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        most = 2.0e11 if dtype == "f32" else 1.5e12
        while True:
            rows, c_in, c_out = _log(rng, 1, 40000), _log(rng, 24, 5000), _log(rng, 24, 5000)
            if rng.random() < 0.8:
                c_in, c_out = 8 * (c_in // 8), 8 * (c_out // 8)
            if 6.0 * rows * c_in * c_out <= most and rows * (c_in + c_out) <= 1.5e8:
                break
        way = rng.choice(["fwd", "fwd", "bwd", "step"])
        act = "none" if way == "step" else rng.choice(["none", "silu", "gelu"])
        r = _linear("", rows, c_in, c_out, dtype, way, act, way != "bwd" and rng.random() < 0.5, way == "fwd" and rng.random() < 0.5)
    else:
        c = 8 * _log(rng, 4, 120)
        r = _adamw("", _log(rng, 1, 12), c, rng.choice([2, 3, 4]) * c + rng.choice([0, 0, 5]), rng.choice([32, 8]), rng.choice(["f32", "bf16", "f16"]),
                   rng.choice(["none", "bf16", "f16"]))
    del r["name"]
    return r


# ------------------------------------------------------------------------------------------------ inputs
def _sizes(case):
    """Tensors of a list of MLP blocks, (numel, group): weights first, then norm gains, then biases; every tensor takes whole blocks of a flat buffer."""
    c, h, n = case["c"], case["hidden"], case["layers"]
    return [(c * h, 0)] * (2 * n) + [(c, 1)] * n + [(c, 2)] * (2 * n) + [(h, 2)] * n


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n01 = lambda *sz: torch.randn(*sz, generator=gen, device="cuda")  # noqa: E731
    u01 = lambda *sz: torch.rand(*sz, generator=gen, device="cuda")  # noqa: E731
    s = {"case": case}
    if case["kind"] == "norm":
        rows, c, dt = case["rows"], case["c"], DT[case["dtype"]]
        # channels of different scale and offset, as a residual stream has them
        s["x"] = (n01(rows, c) * (0.3 + 1.7 * u01(c)) + 0.5 * n01(c)).to(dt)
        s["gamma"], s["beta"] = 1.0 + 0.2 * n01(c), 0.1 * n01(c)
        s["y"] = torch.empty_like(s["x"])
        if case["train"]:
            s["g"] = (1e-2 * n01(rows, c)).to(dt)
            s["dx"] = torch.empty_like(s["x"])
            s["mean"], s["rstd"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
            s["dgamma"], s["dbeta"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        if own:
            from paper_2609_10632_b200 import binding as nb

            s["nb"] = nb
            if case["train"]:
                s["ws"] = torch.empty(nb.nb_layer_norm_workspace_bytes(rows, c), dtype=torch.uint8, device="cuda")
    elif case["kind"] == "linear":
        rows, ci, co, dt, way = case["rows"], case["c_in"], case["c_out"], DT[case["dtype"]], case["way"]
        bound = 1.0 / math.sqrt(ci)
        s["w"] = ((2.0 * u01(co, ci) - 1.0) * bound).to(dt)
        s["x"] = n01(rows, ci).to(dt)
        if way != "bwd":
            s["bias"] = (2.0 * u01(co) - 1.0) * bound
            s["res"] = n01(rows, co).to(dt) if case["res"] else None
            s["out"] = torch.empty(rows, co, dtype=dt, device="cuda")
            s["z"] = torch.empty(rows, co, dtype=dt, device="cuda") if case["save_z"] else None
        if way != "fwd":
            s["dy"] = (1e-2 * n01(rows, co)).to(dt)
            s["z_in"] = (0.8 * n01(rows, ci)).to(dt) if case["act"] != "none" else None
            s["dx"] = torch.empty(rows, ci, dtype=dt, device="cuda")
            s["dw"], s["db"] = torch.empty(co, ci, device="cuda"), torch.empty(co, device="cuda")
        if own:
            from paper_2609_10632_b200 import binding as nb

            s["nb"] = nb
            s["plan"] = nb.LinearPlan(ci, co, CODE[case["dtype"]])
            s["ws"] = torch.empty(s["plan"].workspace_bytes(rows), dtype=torch.uint8, device="cuda")
    else:
        sizes = _sizes(case)
        starts, at = [], 0
        for numel, _ in sizes:
            starts.append(at)
            at += -(-numel // BLOCK) * BLOCK
        decayed = at if not any(g for _, g in sizes) else starts[[g for _, g in sizes].index(1)]
        gdt = DT[case["grad"]]
        live = torch.zeros(at, device="cuda")
        for (numel, _), b in zip(sizes, starts):
            live[b : b + numel] = 1.0
        # gradients of channels of different scale; moments as they are after some steps of them
        scale = torch.exp(1.5 * n01(at)) * 1e-4 * live
        s["grad"] = (n01(at) * scale).to(gdt)
        s["param"] = 0.02 * n01(at) * live
        m, r = 0.3 * scale * n01(at), scale * (0.2 * (0.5 + u01(at)))
        s["copy"] = torch.zeros(at, dtype=DT[case["copy"]], device="cuda") if case["copy"] != "none" else None
        s["step"] = torch.full((1,), STEP, dtype=torch.int64, device="cuda")
        s["norm"] = torch.zeros(1, device="cuda")
        s["decayed"] = decayed
        if case["bits"] == 8:
            s["m"], s["m_scale"] = _to8(m)
            s["v"], s["v_scale"] = _root_to8(r)
        else:
            s["m"], s["v"] = m, r * r
        if own:
            from paper_2609_10632_b200 import binding as nb

            cut = lambda t, b, n: None if t is None else t[b : b + n]  # noqa: E731
            items = []
            for (numel, group), b in zip(sizes, starts):
                it = tuple(cut(s[k], b, numel) for k in ("grad", "param", "m", "v", "copy")) + (group,)
                if case["bits"] == 8:
                    it += tuple(cut(s[k], b // BLOCK, -(-numel // BLOCK)) for k in ("m_scale", "v_scale"))
                items.append(it)
            s["plan"] = nb.AdamWPlan(items)
            s["ws"] = torch.empty(s["plan"].workspace_bytes, dtype=torch.uint8, device="cuda")
            s["plan"].upload(s["ws"])
    return s


# ------------------------------------------------------------------------------------------------ 8-bit moments
def _to8(m):
    """Codes (e4m3) and one scale a block: the block's largest magnitude becomes 448; below 2^-100 the block is zero."""
    b = m.view(-1, BLOCK)
    most = b.abs().amax(1, keepdim=True)
    some = most >= 2.0**-100
    up = torch.where(some, 448.0 / most.clamp_min(2.0**-100), torch.zeros_like(most))
    return (b * up).to(torch.float8_e4m3fn).view(-1), torch.where(some, most / 448.0, torch.zeros_like(most)).view(-1)


def _root_to8(r):
    """The root of the second moment likewise; a root that is not zero is held as at least the smallest code."""
    b = r.view(-1, BLOCK)
    most = b.amax(1, keepdim=True)
    some = most >= 2.0**-100
    up = torch.where(some, 448.0 / most.clamp_min(2.0**-100), torch.zeros_like(most))
    q = torch.where((b > 0) & some, (b * up).clamp_min(2.0**-9), torch.zeros_like(b))
    return q.to(torch.float8_e4m3fn).view(-1), torch.where(some, most / 448.0, torch.zeros_like(most)).view(-1)


def _from8(q, scale):
    return (q.view(-1, BLOCK).float() * scale.view(-1, 1)).view(-1)


# ------------------------------------------------------------------------------------------------ activations
def _act(z, act):
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    return z


def _act_grad(z, act):
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return {"norm": _run_norm, "linear": _run_linear, "adamw": _run_adamw}[s["case"]["kind"]](s)


def _run_norm(s):
    case = s["case"]
    rows, c, train = case["rows"], case["c"], case["train"]
    if own:
        nb, dt = s["nb"], CODE[case["dtype"]]
        if not train:
            nb.nb_layer_norm_fwd(dt, rows, c, s["x"], s["gamma"], s["beta"], EPS_NORM, s["y"])
            return {"y": s["y"]}
        nb.nb_layer_norm_fwd(dt, rows, c, s["x"], s["gamma"], s["beta"], EPS_NORM, s["y"], s["mean"], s["rstd"])
        nb.nb_layer_norm_bwd(dt, rows, c, s["g"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], s["ws"])
        return {k: s[k] for k in ("y", "mean", "rstd", "dx", "dgamma", "dbeta")}
    x, dt = s["x"].float(), s["x"].dtype
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS_NORM)
    xhat = d * rstd
    y = (xhat * s["gamma"] + s["beta"]).to(dt)
    if not train:
        return {"y": y}
    g = s["g"].float()
    dh = g * s["gamma"]
    dx = rstd * (dh - dh.mean(1, keepdim=True) - xhat * (dh * xhat).mean(1, keepdim=True))
    # (sums over hundreds of thousands of rows: in 64 bits)
    return {"y": y, "mean": mean.view(-1), "rstd": rstd.view(-1), "dx": dx.to(dt), "dgamma": (g * xhat).sum(0, dtype=torch.float64).float(),
            "dbeta": g.sum(0, dtype=torch.float64).float()}


def _run_linear(s):
    case = s["case"]
    rows, way, act, out = case["rows"], case["way"], case["act"], {}
    if own:
        nb, plan = s["nb"], s["plan"]
        if way != "bwd":
            nb.nb_linear_fwd(plan, rows, s["x"], s["w"], s["bias"], ACT[act], s["out"], s["ws"], z=s["z"], res=s["res"])
        if way != "fwd":
            nb.nb_linear_bwd_data(plan, rows, s["dy"], s["w"], s["dx"], s["ws"], z_in=s["z_in"], act_in=ACT[act])
            nb.nb_linear_bwd_weight(plan, rows, s["x"], s["dy"], s["dw"], s["db"], s["ws"])
        return {k: s[k] for k in ("out", "z", "dx", "dw", "db") if s.get(k) is not None}
    x, w, dt = s["x"].float(), s["w"].float(), s["x"].dtype
    if way != "bwd":
        z = x @ w.t() + s["bias"]
        a = _act(z, act)
        out["out"] = (a if s["res"] is None else a + s["res"].float()).to(dt)
        if s["z"] is not None:
            out["z"] = z.to(dt)
    if way != "fwd":
        dy = s["dy"].float()
        dx = dy @ w
        out["dx"] = (dx if s["z_in"] is None else dx * _act_grad(s["z_in"].float(), act)).to(dt)
        out["dw"], out["db"] = dy.t() @ x, dy.sum(0, dtype=torch.float64).float()
    return out


def _run_adamw(s):
    case = s["case"]
    eight = case["bits"] == 8
    keys = ("param", "m", "v", "norm", "step") + (("copy",) if s["copy"] is not None else ()) + (("m_scale", "v_scale") if eight else ())
    if own:
        s["plan"].step(s["ws"], s["step"], [LR] * 3, [WD, 0.0, 0.0], BETA1, BETA2, EPS, MAX_NORM, total_norm=s["norm"])
        return {k: s[k] for k in keys}
    g = s["grad"].float()
    total = torch.sqrt((g * g).sum(dtype=torch.float64))
    g = g * torch.clamp(MAX_NORM / (total + 1e-6), max=1.0).float()
    s["step"] += 1
    t = s["step"].double()
    bc1, bc2 = (1.0 - BETA1**t).float(), torch.sqrt(1.0 - BETA2**t).float()
    m = _from8(s["m"], s["m_scale"]) if eight else s["m"]
    v = _from8(s["v"], s["v_scale"]).square() if eight else s["v"]
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * g * g
    root = torch.sqrt(v)
    p = s["param"]
    p[: s["decayed"]] *= 1.0 - LR * WD
    p -= LR * (m / bc1) / (root / bc2 + EPS)
    if eight:
        q, e = _to8(m)
        s["m"].copy_(q), s["m_scale"].copy_(e)
        q, e = _root_to8(root)
        s["v"].copy_(q), s["v_scale"].copy_(e)
    else:
        s["m"].copy_(m), s["v"].copy_(v)
    if s["copy"] is not None:
        s["copy"].copy_(p)
    s["norm"].copy_(total)
    return {k: s[k] for k in keys}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] == "norm":
        n, e = case["rows"] * case["c"], SIZE[case["dtype"]]
        stats, affine = 4 * case["rows"], 4 * case["c"]
        # forward: x, y; backward: g, dx (and x again, if no cache holds it: not counted)
        return {"bytes": 2 * n * e + 2 * affine + (2 * n * e + 2 * stats + 2 * affine if case["train"] else 0), "flops": n * (20 if case["train"] else 7)}
    if case["kind"] == "linear":
        rows, ci, co, e, way = case["rows"], case["c_in"], case["c_out"], SIZE[case["dtype"]], case["way"]
        x, y, w = rows * ci * e, rows * co * e, ci * co
        b, one = 0, 2 * rows * ci * co
        f = (one if way != "bwd" else 0) + (2 * one if way != "fwd" else 0)
        if way != "bwd":
            b += x + y + w * e + 4 * co + (y if case["res"] else 0) + (y if case["save_z"] else 0)
        if way != "fwd":
            b += y + x + w * 4 + 4 * co + (x if case["act"] != "none" else 0) + (x + w * e if way == "bwd" else 0)
        return {"bytes": b, "flops": f}
    n = sum(k for k, _ in _sizes(case))
    moments = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (SIZE[case["grad"]] + 8 + moments + (2 if case["copy"] != "none" else 0)), "flops": 16 * n}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    D = torch.float64
    if case["kind"] == "norm":
        x = s["x"].to(D)
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS_NORM) ** -0.5
        xhat = (x - mean[:, None]).mul_(rstd[:, None])
        y = torch.addcmul(s["beta"].to(D), xhat, s["gamma"].to(D))
        if not case["train"]:
            return {"y": y}
        g = s["g"].to(D)
        dbeta, dgamma = g.sum(0), torch.einsum("rc,rc->c", g, xhat)
        g.mul_(s["gamma"].to(D))
        a, b = g.sum(1) / case["c"], torch.einsum("rc,rc->r", g, xhat) / case["c"]
        dx = (g - a[:, None] - xhat * b[:, None]) * rstd[:, None]
        return {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if case["kind"] == "linear":
        way, act, out = case["way"], case["act"], {}
        x, w = s["x"].to(D), s["w"].to(D)
        normal = torch.distributions.Normal(torch.zeros((), dtype=D, device="cuda"), torch.ones((), dtype=D, device="cuda"))
        if way != "bwd":
            z = torch.addmm(s["bias"].to(D), x, w.T)
            a = z * torch.sigmoid(z) if act == "silu" else z * torch.special.ndtr(z) if act == "gelu" else z.clone()
            out["out"] = a if s["res"] is None else a.add_(s["res"].to(D))
            if s["z"] is not None:
                out["z"] = z
        if way != "fwd":
            dy = s["dy"].to(D)
            dx = torch.mm(dy, w)
            if s["z_in"] is not None:
                z = s["z_in"].to(D)
                if act == "silu":
                    dx *= torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
                else:
                    dx *= torch.special.ndtr(z) + z * torch.exp(normal.log_prob(z))
            out["dx"], out["dw"], out["db"] = dx, torch.mm(dy.T, x), dy.sum(0)
        return out
    g = s["grad"].to(D)
    total = torch.linalg.vector_norm(g)
    g *= min(1.0, MAX_NORM / (float(total) + 1e-6))
    t = STEP + 1
    eight = case["bits"] == 8
    each = lambda e: e.to(D).repeat_interleave(BLOCK)  # noqa: E731
    m = s["m"].to(D) * (each(s["m_scale"]) if eight else 1.0)
    v = (s["v"].to(D) * each(s["v_scale"])) ** 2 if eight else s["v"].to(D)
    m += (1.0 - BETA1) * (g - m)
    v += (1.0 - BETA2) * (g * g - v)
    p = s["param"].to(D)
    keep = torch.ones_like(p)
    keep[: s["decayed"]] = 1.0 - LR * WD
    p = p * keep - LR / (1.0 - BETA1**t) * m / ((v / (1.0 - BETA2**t)) ** 0.5 + EPS)
    out = {"param": p, "norm": total.view(1), "step": None, "m": m, "v": v}
    if s["copy"] is not None:
        out["copy"] = p
    if eight:
        for k, val in (("m", m), ("v", v**0.5)):
            b = val.view(-1, BLOCK)
            most = b.abs().max(1).values
            up = torch.where(most >= 2.0**-100, 448.0 / most, 0.0)[:, None] * b
            if k == "v":
                up = torch.where(up > 0, up.clamp(min=2.0**-9), up)
            out[k] = _nearest_e4m3(up)
            out[k + "_scale"] = torch.where(most >= 2.0**-100, most / 448.0, 0.0)
    return out


def _nearest_e4m3(u):
    """The nearest number of three fraction bits and exponents from -6 on, ties to even, at most 448 in magnitude."""
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0**-6))) - 3.0)
    return (torch.round(u / step) * step).clamp(-448.0, 448.0).view(-1)


def _inputs(case, seed):
    """prepare()'s inputs without the library's handles."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was
