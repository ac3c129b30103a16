"""The MLP products (include/nb_linear.h) on the GPU against the fp64 oracle on the values that the GPU reads, element by element.

Tolerances.  S = sum of |a||b| of an element's products, K their number, u = half a step of the stored type.  An fp32 sum in any order
is off by at most K * 2^-24 * S; the tensor cores add 16 products at a time (K/16 additions to the accumulator, each of which may
truncate: 2^-23) and the slices in fp64: E = (K/8 + 16) * 2^-24 * S there, (K + 16) * 2^-24 * S on the CUDA cores.
  z   E + u|z|;  out: 1.13 E (the steepest slope of both activations is 1.13) + a|z| + u|out|, a = 2.5e-4 (SiLU: half of the 2^-10.987 of
      the hardware's tanh), 2.8e-4 (GELU in bf16: the same and 2.6e-5 of the fit) or 2e-5 (GELU in fp16)
  dx  |act'| E + |dy w + add| * e + u|dx|, e = 4e-5 (GELU) or 2.5e-4 (1 + |z|) (SiLU), both zero without activation
  dw, dbias  E + 2^-24 |dw|
(a and e are bounds of earlier approximations; test_gpu_activation_tails.py holds the present ones, which are far smaller.)
(fp32: a = e = 2^-20, some roundings of erfcf and expf.)  fp16 values below 2^-14 have steps of 2^-24: 2^-25 on top."""
import numpy as np
import pytest

from oracle import linear as ora

pytestmark = pytest.mark.gpu

KIND = {"none": 0, "silu": 1, "gelu": 2}


def _dt(torch, name):
    return {"f32": (torch.float32, 0), "bf16": (torch.bfloat16, 1), "f16": (torch.float16, 2)}[name]


class Case:
    def __init__(self, rows, ci, co, dtype, seed=0, flags=0, pad=0, off=0, device_ws=None):
        import torch

        from paper_2609_10632_b200 import binding as nb

        self.torch, self.nb, self.rows, self.ci, self.co, self.pad, self.off = torch, nb, rows, ci, co, pad, off
        self.dt, code = _dt(torch, dtype)
        self.f32, self.f16 = dtype == "f32", dtype == "f16"
        self.u = torch.finfo(self.dt).eps / 2
        self.plan = nb.LinearPlan(ci, co, code, flags=flags)
        self.rng = np.random.default_rng(seed)
        self.ws = torch.empty(self.plan.workspace_bytes(rows), dtype=torch.uint8, device="cuda").fill_(255)
        self.w, self.hw = self.tensor((co, ci), 1.0 / np.sqrt(ci))
        self.x, self.hx = self.matrix(rows, ci, 1.0)
        self.dy, self.hdy = self.matrix(rows, co, 0.1)
        self.bias = torch.from_numpy(self.rng.normal(size=co).astype(np.float32)).cuda()

    def tensor(self, shape, scale):
        t = self.torch.from_numpy((scale * self.rng.normal(size=shape)).astype(np.float32)).cuda().to(self.dt)
        return t, t.double().cpu().numpy()

    def matrix(self, rows, cols, scale=None):
        """A view with the case's pitch and offset in a buffer of 7.0."""
        ld = cols + self.pad
        buf = self.torch.full((self.off + rows * ld + 64,), 7.0, dtype=self.dt, device="cuda")
        v = buf[self.off : self.off + rows * ld].view(rows, ld)[:, :cols]
        v.buf, v.ld = buf, ld
        if scale is None:
            return v
        v.copy_(self.torch.from_numpy((scale * self.rng.normal(size=(rows, cols))).astype(np.float32)))
        return v, v.double().cpu().numpy()

    def untouched_outside(self, v, name):
        mask = self.torch.ones_like(v.buf, dtype=self.torch.bool)
        mask[self.off : self.off + v.shape[0] * v.ld].view(v.shape[0], v.ld)[:, : v.shape[1]] = False
        assert (v.buf[mask] == 7.0).all(), f"{name}: written outside the matrix"

    def tc(self, call):
        """Whether the tensor cores do it: misaligned rows of even layers are left to the CUDA cores."""
        return self.plan.paths(self.rows)[call] == 1 and (self.ci % 8 != 0 or self.co % 8 != 0 or (self.pad % 8 == 0 and self.off % 8 == 0))

    def E(self, a, b, K, tc):
        return ((K / 8 if tc else K) + 16) * 2.0**-24 * (np.abs(a) @ np.abs(b))

    def close(self, name, got, want, tol):
        got = got.double().cpu().numpy()
        assert np.isfinite(got).all(), name
        tol = tol + (2.0**-25 if self.f16 else 0) + 1e-30
        bad = np.abs(got - want) > tol
        assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - want) / tol):.2f} of the tolerance"

    def forward(self, kind="none", bias=True, res=False, keep_z=False, in_place=False):
        nb, ld = self.nb, {}
        out = self.matrix(self.rows, self.co)
        r, hr = self.matrix(self.rows, self.co, 1.0) if res else (None, None)
        z = self.torch.full((self.rows, self.co), 7.0, dtype=self.dt, device="cuda") if keep_z else None
        if in_place:
            out = r
        nb.nb_linear_fwd(self.plan, self.rows, self.x, self.w, self.bias if bias else None, KIND[kind], out, self.ws, z=z, res=r, ld_x=self.x.ld, ld_out=out.ld,
                         ld_res=r.ld if res else 0)
        self.plan.poll()
        hb = self.bias.double().cpu().numpy() if bias else None
        wz, wout = ora.linear_fwd(self.hx, self.hw, hb, kind, hr)
        E = self.E(self.hx, self.hw.T, self.ci, self.tc("fwd"))
        E = E + 2.0**-23 * (np.abs(wz) + (0 if hb is None else np.abs(hb)))  # the bias added in fp32
        a = {"none": 0.0, "gelu": 2e-5 if self.f16 else 2.8e-4, "silu": 2.5e-4}[kind] if not self.f32 else 2.0**-20
        self.close("out", out, wout, 1.13 * E + a * np.abs(wz) + self.u * np.abs(wout) + 2.0**-22 * (np.abs(wz) + (0 if hr is None else np.abs(hr))))
        if keep_z:
            self.close("z", z, wz, E + self.u * np.abs(wz))
        self.untouched_outside(out, "out")
        return out

    def data(self, kind="none", add=False, in_place=False):
        dx = self.matrix(self.rows, self.ci)
        z, hz = self.tensor((self.rows, self.ci), 1.5) if kind != "none" else (None, None)
        ad, had = self.matrix(self.rows, self.ci, 0.5) if add else (None, None)
        if in_place:
            dx = ad
        self.nb.nb_linear_bwd_data(self.plan, self.rows, self.dy, self.w, dx, self.ws, z_in=z, act_in=KIND[kind], add=ad, ld_dy=self.dy.ld, ld_dx=dx.ld, ld_add=ad.ld if add else 0)
        self.plan.poll()
        want, raw = ora.linear_bwd_data(self.hdy, self.hw, hz, kind, had), np.abs(ora.linear_bwd_data(self.hdy, self.hw, None, "none", had))
        E = self.E(self.hdy, self.hw, self.co, self.tc("data"))
        E = E + 2.0**-23 * (raw + (0 if had is None else np.abs(had)))
        slope = np.ones(1) if hz is None else np.abs(ora.act_grad(hz, kind))
        e = 0.0 if hz is None else 2.0**-20 if self.f32 else 4e-5 if kind == "gelu" else 2.5e-4 * (1 + np.abs(hz))
        self.close("dx", dx, want, slope * E + (e + 2.0**-22) * (raw + E) + self.u * np.abs(want))
        self.untouched_outside(dx, "dx")
        return dx

    def weight(self, bias=True):
        dw = self.torch.full((self.co * self.ci + 64,), 7.0, device="cuda")
        db = self.torch.full((self.co + 64,), 7.0, device="cuda") if bias else None
        self.nb.nb_linear_bwd_weight(self.plan, self.rows, self.x, self.dy, dw, db, self.ws, ld_x=self.x.ld, ld_dy=self.dy.ld)
        self.plan.poll()
        wdw, wdb = ora.linear_bwd_weight(self.hx, self.hdy)
        tc = self.tc("weight")
        n = self.co * self.ci
        self.close("dw", dw[:n].view(self.co, self.ci), wdw, self.E(self.hdy.T, self.hx, self.rows, tc) + 2.0**-24 * np.abs(wdw))
        assert (dw[n:] == 7.0).all()
        if bias:
            E = ((self.rows / 8 if tc else self.rows) + 16) * 2.0**-24 * np.abs(self.hdy).sum(0)
            self.close("dbias", db[: self.co], wdb, E + 2.0**-24 * np.abs(wdb))
            assert (db[self.co :] == 7.0).all()
        return dw, db

    def all(self, **kw):
        self.forward()
        self.data()
        self.weight()


SHAPES = [(1, 8, 8), (1, 64, 64), (2, 128, 40), (3, 24, 136), (5, 512, 96), (8, 1024, 256), (9, 64, 64), (16, 72, 200), (37, 1000, 520), (64, 64, 64), (127, 200, 72),
          (128, 128, 128), (129, 136, 264), (256, 256, 256), (300, 384, 96), (513, 96, 384), (1000, 520, 328), (2100, 64, 1032)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows, ci, co", SHAPES)
def test_tensor_core_shapes(rows, ci, co, dtype):
    c = Case(rows, ci, co, dtype, seed=rows)
    assert c.plan.paths(rows) == {"fwd": 2 if rows <= 8 else 1, "data": 1, "weight": 1}
    c.all()


@pytest.mark.parametrize("dtype, flags", [("f32", 0), ("bf16", 1), ("f16", 1)])
@pytest.mark.parametrize("rows, ci, co", [(1, 1, 1), (1, 3, 5), (2, 16, 7), (7, 33, 65), (8, 64, 64), (9, 100, 50), (64, 64, 64), (65, 129, 63), (200, 77, 300), (1000, 48, 20), (70, 1500, 24)])
def test_cuda_core_shapes(rows, ci, co, dtype, flags):
    c = Case(rows, ci, co, dtype, seed=rows, flags=flags)
    assert c.plan.paths(rows)["data"] == 0
    c.all()


@pytest.mark.parametrize("dtype, flags", [("f32", 0), ("bf16", 1)])
@pytest.mark.parametrize("rows, ci, co", [(300, 3500, 1001), (7000, 500, 380), (1061, 1003, 3520)])
def test_cuda_core_large_tiles_with_slices(rows, ci, co, dtype, flags):
    """Few tiles of 128 and long sums: the forward product, the weight gradient and the data gradient, each in slices of k."""
    Case(rows, ci, co, dtype, seed=co, flags=flags).all()


@pytest.mark.parametrize("rows, ci, co", [(5, 1001, 77), (100, 20, 36), (33, 77, 129)])
def test_odd_channel_counts_in_16_bits(rows, ci, co):
    Case(rows, ci, co, "bf16", seed=1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows, ci, co, pad, off", [(1100, 333, 401, 0, 0), (700, 1001, 200, 3, 1), (2000, 264, 259, 0, 0), (130, 1003, 1037, 1, 0), (5000, 77, 363, 5, 2)])
def test_odd_channel_counts_on_padded_copies(rows, ci, co, pad, off, dtype):
    """From 2^27 products on, layers of odd channel counts take the tensor cores: everything an epilogue can be given, pitches included."""
    c = Case(rows, ci, co, dtype, seed=rows, pad=pad, off=off)
    assert c.plan.paths(rows) == {"fwd": 1, "data": 1, "weight": 1}
    c.forward()
    c.forward("gelu", res=True, keep_z=True)
    c.forward("silu", bias=False, res=True, in_place=True)
    c.data()
    c.data("gelu", add=True)
    c.data("silu", add=True, in_place=True)
    c.weight()
    c.weight(bias=False)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows", [4, 200])
@pytest.mark.parametrize("kind", ["none", "silu", "gelu"])
@pytest.mark.parametrize("res, keep_z, bias, in_place", [(False, False, True, False), (True, True, True, False), (True, False, False, True), (False, True, False, False)])
def test_epilogues(kind, rows, res, keep_z, bias, in_place, dtype):
    c = Case(rows, 128, 272, dtype, seed=rows)
    c.forward(kind, bias, res, keep_z, in_place)
    c.data(kind, add=res, in_place=in_place)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("pad, off", [(8, 0), (64, 8), (1, 0), (0, 1), (4, 4), (3, 5)])
@pytest.mark.parametrize("rows", [3, 150])
def test_pitches_and_offsets(rows, pad, off, dtype):
    c = Case(rows, 64, 136, dtype, seed=pad, pad=pad, off=off)
    c.forward("gelu", True, True, True)
    c.data("silu", add=True)
    c.weight()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_tiles_of_every_width(dtype):
    """Shapes for which the choice of tiles takes 64, 128, 192 and 256 columns, single CTAs and pairs, one and several rounds."""
    for rows, ci, co in [(20000, 64, 64), (20000, 128, 192), (9472, 64, 384), (4000, 320, 512), (1500, 704, 1536)]:
        c = Case(rows, ci, co, dtype, seed=co)
        c.forward("gelu", keep_z=True)
        c.data("gelu")
        c.weight()


@pytest.mark.parametrize("rows", [300, 2500, 12000])
@pytest.mark.parametrize("n", [64, 96, 128, 192, 256, 320, 384, 576, 768, 1152, 1536])
def test_epilogue_inputs_at_every_tile_width(n, rows):
    """Residuals and z_in come by TMA, pass by pass: one to four passes a warp, few and many tiles a CTA, short products."""
    c = Case(rows, 72, n, "bf16", seed=n)
    c.forward("gelu", res=True)
    c.forward("silu", res=True, keep_z=True)
    c = Case(rows, n, 72, "bf16", seed=n)
    c.data("gelu")
    c.data("silu", add=True)


def test_a_long_sum_over_rows():
    """90000 rows into one small weight gradient."""
    c = Case(90000, 64, 64, "bf16", seed=2)
    c.weight()


def test_activations_over_their_whole_range():
    """Identity weights hand the activation every bf16 value of a range; far tails are exact zeros and identities."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    v = torch.linspace(-12, 12, 128 * 256, device="cuda").to(torch.bfloat16).view(128, 256)
    v[0, :8] = torch.tensor([0.0, -0.0, 1e30, -1e30, 3e38, -3e38, 1e-30, -65504.0])
    plan = nb.LinearPlan(256, 256, nb.NB_DTYPE_BF16)
    ws = torch.empty(plan.workspace_bytes(128), dtype=torch.uint8, device="cuda")
    eye = torch.eye(256, device="cuda").bfloat16()
    out, dx = torch.empty_like(v), torch.empty_like(v)
    hv = v.double().cpu().numpy()
    for kind, a in (("gelu", 2.8e-4), ("silu", 2.5e-4)):
        nb.nb_linear_fwd(plan, 128, v, eye, None, KIND[kind], out, ws)
        want = ora.act(hv, kind)
        got = out.double().cpu().numpy()
        assert (np.abs(got - want) <= a * np.minimum(np.abs(hv), 20.0) + 2.0**-8 * np.abs(want) * (1 + 2.0**-8)).all()
        nb.nb_linear_bwd_data(plan, 128, torch.ones_like(v), eye, dx, ws, z_in=v, act_in=KIND[kind])
        want = ora.act_grad(hv, kind)
        got = dx.double().cpu().numpy()
        tol = 4e-5 if kind == "gelu" else 2.5e-4 * (1 + np.minimum(np.abs(hv), 20.0))
        assert (np.abs(got - want) <= tol + 2.0**-8 * np.abs(want)).all()
        nb.nb_act_bwd(nb.NB_DTYPE_BF16, v.numel(), KIND[kind], torch.ones_like(v), v, dx)
        assert (np.abs(dx.double().cpu().numpy() - want) <= 1e-6 + 2.0**-8 * np.abs(want)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n, off", [(1, 0), (7, 0), (8, 0), (1000, 1), (4099, 0), (300000, 0)])
def test_act_bwd(n, off, dtype):
    import torch

    from paper_2609_10632_b200 import binding as nb

    dt, code = _dt(torch, dtype)
    u = torch.finfo(dt).eps / 2
    for kind in ("silu", "gelu"):
        buf = [torch.randn(n + off + 8, device="cuda").to(dt) for _ in range(2)] + [torch.full((n + off + 8,), 7.0, device="cuda").to(dt)]
        dy, z, dz = (b[off : off + n] for b in buf)
        want = dy.double().cpu().numpy() * ora.act_grad(z.double().cpu().numpy(), kind)
        nb.nb_act_bwd(code, n, KIND[kind], dy, z, dz)
        got = dz.double().cpu().numpy()
        assert (np.abs(got - want) <= (u + 2.0**-20) * np.abs(want) + 2.0**-20 * np.abs(dy.double().cpu().numpy()) + 2.0**-25).all()
        assert (buf[2][off + n :] == 7.0).all() and (buf[2][:off] == 7.0).all()
        nb.nb_act_bwd(code, n, KIND[kind], dy, z, dy)  # in place
        assert torch.equal(dy, dz)


def test_gradients_against_differences():
    """Central differences of the GPU's own fp32 forward pass (step 2^-5: truncation h^2/6 of a third derivative below 1, rounding
    2^-24 * |sum| / h)."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    rows, ci, co, h = 3, 6, 5, 2.0**-5
    gen = torch.Generator(device="cuda").manual_seed(4)
    r = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    z_in, w, b, g = r(rows, ci), 0.5 * r(co, ci), r(co), r(rows, co)
    plan = nb.LinearPlan(ci, co, nb.NB_DTYPE_F32)
    ws = torch.empty(plan.workspace_bytes(rows), dtype=torch.uint8, device="cuda")

    def loss():
        x = torch.nn.functional.gelu(z_in)
        out = torch.empty(rows, co, device="cuda")
        nb.nb_linear_fwd(plan, rows, x, w, b, nb.NB_ACT_NONE, out, ws)
        return float((out.double() * g.double()).sum())

    x = torch.nn.functional.gelu(z_in)
    dz, dw, db = torch.empty_like(z_in), torch.empty_like(w), torch.empty_like(b)
    nb.nb_linear_bwd_data(plan, rows, g, w, dz, ws, z_in=z_in, act_in=nb.NB_ACT_GELU)
    nb.nb_linear_bwd_weight(plan, rows, x, g, dw, db, ws)
    for t, grad in ((z_in, dz), (w, dw), (b, db)):
        flat = t.view(-1)
        for i in range(flat.numel()):
            was = float(flat[i])
            flat[i] = was + h
            up = loss()
            flat[i] = was - h
            down = loss()
            flat[i] = was
            assert (up - down) / (2 * h) == pytest.approx(float(grad.view(-1)[i]), abs=4e-3)


def test_captured_calls_other_streams_and_repeated_bits():
    import torch

    a, b = Case(700, 256, 512, "bf16", seed=6), Case(700, 256, 512, "bf16", seed=6)
    outs = []
    for c in (a, b):
        outs.append([torch.zeros(700, 512, dtype=torch.bfloat16, device="cuda"), torch.zeros(700, 256, dtype=torch.bfloat16, device="cuda"), torch.zeros(512, 256, device="cuda"),
                     torch.zeros(512, device="cuda")])

    def step(c, o, stream=None):
        c.nb.nb_linear_fwd(c.plan, 700, c.x, c.w, c.bias, 2, o[0], c.ws, stream=stream)
        c.nb.nb_linear_bwd_data(c.plan, 700, c.dy, c.w, o[1], c.ws, stream=stream)
        c.nb.nb_linear_bwd_weight(c.plan, 700, c.x, c.dy, o[2], o[3], c.ws, stream=stream)

    step(a, outs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(b, outs[1])
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for x, y in zip(*outs):
        assert torch.equal(x, y)
    # one plan, two streams, a workspace each
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    ws2 = torch.empty_like(a.ws)
    o1, o2 = [torch.zeros_like(t) for t in outs[0]], [torch.zeros_like(t) for t in outs[0]]
    torch.cuda.synchronize()
    for _ in range(5):
        step(a, o1, s1)
        ws, a.ws = a.ws, ws2
        step(a, o2, s2)
        a.ws = ws
    torch.cuda.synchronize()
    for x, y, z in zip(outs[0], o1, o2):
        assert torch.equal(x, y) and torch.equal(x, z)
    a.plan.poll()


def test_rows_behind_the_last_stay_and_nan_rows_stay_by_themselves():
    import torch

    for rows in (5, 130):
        c = Case(rows, 64, 64, "bf16", seed=7)
        first = c.forward().clone()
        c.x[rows - 2] = float("nan")
        out = c.matrix(rows, 64)
        c.nb.nb_linear_fwd(c.plan, rows, c.x, c.w, c.bias, 0, out, c.ws)
        keep = [r for r in range(rows) if r != rows - 2]
        assert torch.equal(out[keep], first[keep]) and out[rows - 2].isnan().all()
        c.untouched_outside(out, "out")


def test_saturation_in_fp16():
    import torch

    c = Case(200, 64, 64, "f16", seed=8)
    c.x.fill_(300.0)
    c.w.fill_(100.0)
    out = c.matrix(200, 64)
    for rows in (4, 200):
        c.nb.nb_linear_fwd(c.plan, rows, c.x, c.w, None, 0, out, c.ws)
        assert (out[:rows] == 65504.0).all()


def test_offsets_past_32_bits():
    """Rows 131072 elements apart: the last one lies 10 GB behind the first."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    rows, ci, co, ld = 40000, 64, 72, 131072
    buf = torch.zeros(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    x, out = buf[:, :ci], buf[:, 128 : 128 + co]
    x.copy_(torch.randn(rows, ci, device="cuda"))
    w = torch.randn(co, ci, device="cuda").bfloat16()
    plan = nb.LinearPlan(ci, co, 1)
    ws = torch.empty(plan.workspace_bytes(rows), dtype=torch.uint8, device="cuda")
    xc, oc = x.contiguous(), torch.empty(rows, co, dtype=torch.bfloat16, device="cuda")
    nb.nb_linear_fwd(plan, rows, x, w, None, 0, out, ws, ld_x=ld, ld_out=ld, res=out, ld_res=ld)
    nb.nb_linear_fwd(plan, rows, xc, w, None, 0, oc, ws)
    assert torch.equal(out, oc)
    dx, dxc = buf[:, 256 : 256 + ci], torch.empty(rows, ci, dtype=torch.bfloat16, device="cuda")
    nb.nb_linear_bwd_data(plan, rows, out, w, dx, ws, ld_dy=ld, ld_dx=ld)
    nb.nb_linear_bwd_data(plan, rows, oc, w, dxc, ws)
    assert torch.equal(dx, dxc)
    dw, dwc = torch.empty(co, ci, device="cuda"), torch.empty(co, ci, device="cuda")
    nb.nb_linear_bwd_weight(plan, rows, x, out, dw, None, ws, ld_x=ld, ld_dy=ld)
    nb.nb_linear_bwd_weight(plan, rows, xc, oc, dwc, None, ws)
    assert torch.equal(dw, dwc)
    plan.poll()


def test_refusals():
    import torch

    c = Case(64, 64, 64, "bf16", seed=9)
    nb, out, f = c.nb, c.matrix(64, 64), torch.zeros(64 * 64 + 4, device="cuda")
    fwd = lambda **k: nb.nb_linear_fwd(**{**dict(plan=c.plan, rows=64, x=c.x, w=c.w, bias=c.bias, act=0, out=out, workspace=c.ws), **k})  # noqa: E731
    data = lambda **k: nb.nb_linear_bwd_data(**{**dict(plan=c.plan, rows=64, dy=c.dy, w=c.w, dx=out, workspace=c.ws), **k})  # noqa: E731
    wt = lambda **k: nb.nb_linear_bwd_weight(**{**dict(plan=c.plan, rows=64, x=c.x, dy=c.dy, dw=f, dbias=None, workspace=c.ws), **k})  # noqa: E731
    A, B, W, L = nb.NB_ERR_INVALID_ARG, nb.NB_ERR_UNSUPPORTED, nb.NB_ERR_WORKSPACE, nb.NB_ERR_ALIGNMENT
    p = c.w.data_ptr()
    for call, status in [
        (lambda: fwd(rows=0), A), (lambda: fwd(rows=-3), A), (lambda: fwd(rows=0x7fff0000), B), (lambda: fwd(x=None), A), (lambda: fwd(w=None), A), (lambda: fwd(out=None), A),
        (lambda: fwd(act=3), A), (lambda: fwd(act=-1), A), (lambda: fwd(ld_x=63), A), (lambda: fwd(ld_out=8), A), (lambda: fwd(res=out, ld_res=-64), A), (lambda: fwd(w=p + 2), L),
        (lambda: fwd(x=p + 1), L), (lambda: fwd(bias=c.bias[1:]), L), (lambda: fwd(z=p + 1), L), (lambda: fwd(workspace=None), W), (lambda: fwd(workspace=c.ws[:128]), W),
        (lambda: data(dy=None), A), (lambda: data(z_in=out), A), (lambda: data(act_in=2), A), (lambda: data(act_in=7, z_in=out), A), (lambda: data(ld_dx=1), A), (lambda: data(dx=p + 1), L),
        (lambda: wt(dw=None), A), (lambda: wt(dw=f[1:]), L), (lambda: wt(dbias=f[2:]), L), (lambda: wt(ld_dy=32), A), (lambda: wt(workspace=None), W),
    ]:
        with pytest.raises(nb.NbError) as e:
            call()
        assert e.value.status == status
    assert (out.buf == 7.0).all()


@pytest.mark.parametrize("dtype, rows, co, ci, kind", [
    ("f16", 24, 72, 1 << 19, "fwd"), ("f16", 300, 136, 1 << 17, "fwd"), ("f16", 100, 64, 1 << 14, "fwd"), ("f16", 100, 64, (1 << 14) + 8, "fwd"), ("f16", 24, 1 << 19, 72, "data"),
    ("f16", 300, 1 << 17, 200, "data"), ("f16", 20000, 264, 16400, "fwd"), ("f16", 12000, 16400, 520, "data"), ("bf16", 24, 72, 1 << 22, "fwd"), ("bf16", 33, 64, 1 << 17, "fwd"), ("bf16", 140, 1 << 20, 24, "data")])
def test_products_of_very_many_terms(dtype, rows, co, ci, kind):
    """Sums of positive terms, which the tensor cores cut off at every addition, stay within the roundings of their result and a quarter of
    one more: (5/4) u|value|, u half a step of the type (the products' own header gives 0.18 for what stays in the tensor cores)."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    dt, code = _dt(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    K = ci if kind == "fwd" else co
    a = (0.5 + torch.rand(rows, K, device="cuda", generator=gen)).to(dt)
    w = ((0.5 + torch.rand(co, ci, device="cuda", generator=gen)) * (1000.0 / K if dtype == "bf16" else 2.0**-6)).to(dt)
    if dtype == "f16":
        a *= 2.0**-6
    plan = nb.LinearPlan(ci, co, code)
    assert plan.paths(rows)[kind] == 1
    ws = torch.empty(plan.workspace_bytes(rows), dtype=torch.uint8, device="cuda")
    out = torch.full((rows + 1, co if kind == "fwd" else ci), 7.0, device="cuda").to(dt)
    res = torch.zeros_like(out[:rows])
    n = out.shape[1]
    if kind == "fwd":
        nb.nb_linear_fwd(plan, rows, a, w, torch.zeros(n, device="cuda"), 0, out, ws, res=res)
    else:
        nb.nb_linear_bwd_data(plan, rows, a, w, out, ws, add=res)
    plan.poll()
    want = torch.zeros(rows, n, dtype=torch.float64, device="cuda")
    for k in range(0, K, 1 << 15):
        s = slice(k, k + (1 << 15))
        want += a[:, s].double() @ (w[:, s].double().T if kind == "fwd" else w[s].double())
    off = ((out[:rows].double() - want).abs() / want).max().item()
    assert off <= 1.25 * torch.finfo(dt).eps / 2, off / (torch.finfo(dt).eps / 2)
    assert (out[rows] == 7.0).all()


@pytest.mark.parametrize("dtype, k", [("f16", 16392), ("f16", 34000), ("bf16", 131080)])
@pytest.mark.parametrize("rows, n", [(20, 8), (300, 200), (130, 400)])
def test_epilogues_behind_very_many_terms(rows, n, dtype, k):
    """One and several tiles of 128 columns, ragged ones, with everything that an epilogue can be given; a last chunk of one k-block."""
    c = Case(rows, k, n, dtype, seed=n)
    c.forward("gelu", res=True, keep_z=True)
    c.forward("silu", res=True)
    c = Case(rows, n, k, dtype, seed=n)
    c.data("gelu", add=True)
    c.data("silu")
    c.data()


@pytest.mark.parametrize("dtype, flags, rows, ci, co", [("f32", 0, 600000, 500, 700), ("bf16", 1, 33000, 2000, 2100), ("f32", 0, 9001, 4900, 3501), ("f16", 1, 900000, 300, 701)])
def test_weight_gradients_whose_slices_come_in_groups(dtype, flags, rows, ci, co):
    """More slices than are kept at once: two groups of many, groups of one.  E as above with 4096 terms a slice, and a rounding for each group."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    dt, code = _dt(torch, dtype)
    plan = nb.LinearPlan(ci, co, code, flags=flags)
    need = plan.workspace_bytes(rows)
    assert need <= 130 << 20
    ws = torch.empty(need, dtype=torch.uint8, device="cuda").fill_(255)
    x, dy = torch.randn(rows, ci, device="cuda").to(dt), torch.randn(rows, co, device="cuda").to(dt)
    dw, db = torch.full((co * ci + 8,), 7.0, device="cuda"), torch.full((co + 8,), 7.0, device="cuda")
    nb.nb_linear_bwd_weight(plan, rows, x, dy, dw, db, ws)
    want, S = (torch.zeros(co, ci, dtype=torch.float64, device="cuda") for _ in range(2))
    for k in range(0, rows, 1 << 16):
        a, b = dy[k : k + (1 << 16)].double(), x[k : k + (1 << 16)].double()
        want += a.T @ b
        S += a.abs().T @ b.abs()
    assert ((dw[: co * ci].view(co, ci).double() - want).abs() <= (4096 + 16) * 2.0**-24 * S + 8 * 2.0**-24 * S).all() and (dw[co * ci :] == 7.0).all()
    assert ((db[:co].double() - dy.double().sum(0)).abs() <= (4096 + 24) * 2.0**-24 * dy.double().abs().sum(0)).all() and (db[co:] == 7.0).all()
    first = dw.clone()
    nb.nb_linear_bwd_weight(plan, rows, x, dy, dw, None, ws)
    assert torch.equal(dw, first)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_workspace_does_not_grow_with_the_rows(dtype):
    import torch

    from paper_2609_10632_b200 import binding as nb

    for ci, co in ((384, 1536), (4096, 4096), (4096, 16384)):
        plan = nb.LinearPlan(ci, co, _dt(torch, dtype)[1])
        assert all(plan.workspace_bytes(rows) <= ci * co * 4 + (160 << 20) for rows in (1, 100, 25600, 409600, 1 << 20, 1 << 24))
