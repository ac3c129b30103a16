"""Layer norm (include/nb_norm.h) on the GPU against the fp64 oracle on the values that the GPU reads.

Tolerances, per element, with u = half a step of the stored type (torch.finfo.eps / 2) and A = (largest |x| of the row) * rstd:
a sum of up to 2^14 fp32 values in trees of at most 64 additions a thread, then 10 across threads, is off by at most 2^-18 of the
sum of magnitudes (74 roundings of 2^-24); so mean is off by 2^-18 * max|x|, xhat by 2^-18 * (2A + |xhat|), and
  y    by u*|y| + 2^-17 * |gamma| * (A + |xhat|) + 2^-24 * |beta|
  dx   by u*|dx| + 2^-17 * rstd * (|d| + avg|d| + (|xhat| + A) * avg|d*xhat| + |xhat| * avg(|d|) * A) + 2^-24 * |add|
  sums over rows by 2^-17 * sum |g| * (1 + A + |xhat|).
The oracle's backward pass is given the GPU's own mean and rstd (fp32), whose errors the forward test bounds."""
import numpy as np
import pytest

from oracle import norm as ora

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _types(torch):
    from paper_2609_10632_b200 import binding as nb

    return {"f32": (torch.float32, nb.NB_DTYPE_F32, 4), "bf16": (torch.bfloat16, nb.NB_DTYPE_BF16, 2), "f16": (torch.float16, nb.NB_DTYPE_F16, 2)}


def _matrix(torch, rows, c, ld, off, dt, fill=None):
    """A rows x c view with pitch ld that starts `off` elements into its buffer, and the buffer (7.0 outside the view)."""
    buf = torch.full((off + rows * ld + 64,), 7.0, dtype=dt, device="cuda")
    view = buf[off : off + rows * ld].view(rows, ld)[:, :c]
    if fill is not None:
        view.copy_(torch.from_numpy(fill.astype(np.float32)))
    return view, buf


def _outside(torch, view, buf, off, ld):
    mask = torch.ones_like(buf, dtype=torch.bool)
    mask[off : off + view.shape[0] * ld].view(view.shape[0], ld)[:, : view.shape[1]] = False
    return torch.equal(buf[mask], torch.full_like(buf, 7.0)[mask])


def _close(name, got, want, tol):
    got = got.double().cpu().numpy() if hasattr(got, "cpu") else got
    assert np.isfinite(got).all(), name
    bad = np.abs(got - want) > tol
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size}, worst {np.max(np.abs(got - want) / tol):.2f} of the tolerance"


def run(rows, c, dtype, pad=0, off=0, affine=True, add=False, sums=True, seed=0, in_place=False):
    import torch

    from paper_2609_10632_b200 import binding as nb

    dt, code, _ = _types(torch)[dtype]
    rng = np.random.default_rng(seed)
    ld = c + pad
    x, xb = _matrix(torch, rows, c, ld, off, dt, rng.normal(size=(rows, c)) * rng.uniform(0.3, 2.0, c) + rng.normal(size=c))
    g, gb = _matrix(torch, rows, c, ld, off, dt, 0.1 * rng.normal(size=(rows, c)))
    y, yb = _matrix(torch, rows, c, ld, off, dt)
    dx, dxb = _matrix(torch, rows, c, ld, off, dt)
    ad = _matrix(torch, rows, c, ld, off, dt, rng.normal(size=(rows, c)))[0] if add else None
    gamma = torch.from_numpy(rng.normal(size=c).astype(np.float32)).cuda() if affine else None
    beta = torch.from_numpy(rng.normal(size=c).astype(np.float32)).cuda() if affine else None
    mean, rstd = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    dgamma, dbeta = (torch.full((c,), 7.0, device="cuda") for _ in range(2)) if sums else (None, None)
    ws = torch.empty(nb.nb_layer_norm_workspace_bytes(rows, c), dtype=torch.uint8, device="cuda").fill_(255) if sums else None
    hx, hg = x.double().cpu().numpy(), g.double().cpu().numpy()
    hadd = ad.double().cpu().numpy() if add else 0.0
    if in_place:
        x0 = x.clone()
        nb.nb_layer_norm_fwd(code, rows, c, x, gamma, beta, EPS, x, mean, rstd, ld_x=ld, ld_y=ld)
        y.copy_(x)
        x.copy_(x0)
        nb.nb_layer_norm_bwd(code, rows, c, g, x, gamma, mean, rstd, g, dgamma, dbeta, ws, add=ad, ld_g=ld, ld_x=ld, ld_add=ld, ld_dx=ld)
        dx.copy_(g)
    else:
        nb.nb_layer_norm_fwd(code, rows, c, x, gamma, beta, EPS, y, mean, rstd, ld_x=ld, ld_y=ld)
        nb.nb_layer_norm_bwd(code, rows, c, g, x, gamma, mean, rstd, dx, dgamma, dbeta, ws, add=ad, ld_g=ld, ld_x=ld, ld_add=ld, ld_dx=ld)
    torch.cuda.synchronize()
    hga = gamma.double().cpu().numpy() if affine else None
    hbe = beta.double().cpu().numpy() if affine else None
    one = np.ones(c) if hga is None else np.abs(hga)
    want, wmean, wrstd = ora.layer_norm_fwd(hx, hga, hbe, EPS)
    u = torch.finfo(dt).eps / 2
    most = np.abs(hx).max(1, keepdims=True)
    A = most * wrstd[:, None]
    xhat = (hx - wmean[:, None]) * wrstd[:, None]
    _close("mean", mean, wmean, 2.0**-18 * most[:, 0] + 1e-30)
    _close("rstd", rstd, wrstd, 2.0**-18 * wrstd * (1 + A[:, 0]))
    _close("y", y, want, u * np.abs(want) + 2.0**-17 * one * (A + np.abs(xhat)) + 2.0**-24 * (0 if hbe is None else np.abs(hbe)) + 1e-30)
    gm, gr = mean.double().cpu().numpy(), rstd.double().cpu().numpy()
    wdx, wdg, wdb = ora.layer_norm_bwd(hg, hx, hga, gm, gr)
    wdx = wdx + hadd
    xhat = (hx - gm[:, None]) * gr[:, None]
    d = np.abs(hg) * one
    avg = lambda v: v.mean(1, keepdims=True)  # noqa: E731
    tol = u * np.abs(wdx) + 2.0**-17 * gr[:, None] * (d + avg(d) + (np.abs(xhat) + A) * avg(d * np.abs(xhat)) + np.abs(xhat) * avg(d) * A) + 2.0**-24 * np.abs(hadd)
    _close("dx", dx, wdx, tol + 1e-7 * (u > 1e-4) * 1.0 + 1e-30)  # (fp16: results below 2^-14 have steps of 2^-24)
    if sums:
        w = np.abs(hg) * (1 + A + np.abs(xhat))
        _close("dgamma", dgamma, wdg, 2.0**-17 * w.sum(0) + 1e-30)
        _close("dbeta", dbeta, wdb, 2.0**-17 * np.abs(hg).sum(0) + 1e-30)
    for name, v, b in (("x", x, xb), ("y", y, yb), ("dx", dx, dxb), ("g", g, gb)):
        assert _outside(torch, v, b, off, ld), f"{name}: written outside the matrix"
    return {"y": y, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}


# one vector to beyond what registers hold, odd counts, and the borders between the kernels' forms
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("c", [1, 2, 3, 8, 31, 32, 33, 64, 96, 136, 256, 257, 384, 520, 768, 1000, 1001, 1024, 1025, 1032, 2048, 4096, 4097, 4104, 8192, 8193, 8200, 16384, 16392])
def test_channel_counts(c, dtype):
    run(5, c, dtype, seed=c)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 2, 7, 8, 31, 64, 65, 127, 1000, 4001])
@pytest.mark.parametrize("c", [24, 96, 200, 1000, 77])
def test_row_counts(rows, c, dtype):
    run(rows, c, dtype, seed=rows)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad, off", [(8, 0), (8, 8), (1, 0), (0, 1), (3, 5), (16, 24)])
@pytest.mark.parametrize("c", [64, 384, 1024, 17])
def test_channel_slices_and_misaligned_rows(c, pad, off, dtype):
    run(37, c, dtype, pad=pad, off=off, add=True, seed=pad + off)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("c", [96, 1001, 4096, 16400])
@pytest.mark.parametrize("affine, add, sums, in_place", [(False, False, True, False), (True, True, False, False), (False, True, False, True), (True, True, True, True)])
def test_options_and_in_place(c, affine, add, sums, in_place, dtype):
    run(19, c, dtype, affine=affine, add=add, sums=sums, in_place=in_place, seed=c)


def test_many_rows():
    run(40000, 96, "bf16", seed=3)


def test_statistics_of_rows_far_from_zero_and_of_constant_rows():
    """Two passes over the row: a mean of 1000 standard deviations costs nothing but the mean's own rounding; a constant row gives beta."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    rng = np.random.default_rng(5)
    h = rng.normal(size=(6, 512)).astype(np.float32)
    h[1] += 1000.0
    h[2] = 3.25
    h[3] *= 1e-20
    h[4] = 0.0
    h[5] *= 1e15
    x = torch.from_numpy(h).cuda()
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    beta = torch.full((512,), 0.5, device="cuda")
    nb.nb_layer_norm_fwd(nb.NB_DTYPE_F32, 6, 512, x, None, beta, EPS, y, mean, rstd)
    want, wmean, wrstd = ora.layer_norm_fwd(h, None, np.full(512, 0.5), EPS)
    most = np.abs(h.astype(np.float64)).max(1)
    _close("mean", mean, wmean, 2.0**-18 * most + 1e-30)
    _close("rstd", rstd, wrstd, 2.0**-18 * wrstd * (1 + most * wrstd))
    _close("y", y, want, 2.0**-17 * (most * wrstd)[:, None] + 2.0**-17)
    assert (y[2] == 0.5).all() and (y[4] == 0.5).all()
    assert float(rstd[2]) == pytest.approx(EPS**-0.5, rel=1e-6)


@pytest.mark.parametrize("c", [96, 999, 4096, 16400])
def test_a_row_with_nan_or_inf_stays_by_itself(c):
    import torch

    from paper_2609_10632_b200 import binding as nb

    x = torch.randn(9, c, device="cuda")
    y, y2, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
    nb.nb_layer_norm_fwd(0, 9, c, x, None, None, EPS, y, mean, rstd)
    x[3, c // 2], x[5, 0] = float("nan"), float("inf")
    nb.nb_layer_norm_fwd(0, 9, c, x, None, None, EPS, y2, mean, rstd)
    keep = [0, 1, 2, 4, 6, 7, 8]
    assert torch.equal(y[keep], y2[keep]) and y2[3].isnan().all() and y2[5].isnan().any()
    dx, dx2, g = torch.empty_like(x), torch.empty_like(x), torch.randn_like(x)
    nb.nb_layer_norm_bwd(0, 9, c, g, y, None, mean.nan_to_num(), rstd.nan_to_num(), dx)
    g[4, 1] = float("nan")
    nb.nb_layer_norm_bwd(0, 9, c, g, y, None, mean.nan_to_num(), rstd.nan_to_num(), dx2)
    assert torch.equal(dx[[0, 1, 2, 3, 5, 6, 7, 8]], dx2[[0, 1, 2, 3, 5, 6, 7, 8]]) and dx2[4].isnan().all()


def test_gradients_against_differences():
    """d(sum y*g) / dx by central differences of the GPU's own forward pass (fp32, step 2^-6: truncation h^2/6 of the third derivative
    against a rounding of 2^-24 * |sum| / h)."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    rows, c, h = 2, 24, 2.0**-6
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, g = torch.randn(rows, c, device="cuda", generator=gen), torch.randn(rows, c, device="cuda", generator=gen)
    ga, be = torch.randn(c, device="cuda", generator=gen), torch.randn(c, device="cuda", generator=gen)

    def loss(x, ga, be):
        y = torch.empty_like(x)
        nb.nb_layer_norm_fwd(0, rows, c, x, ga, be, EPS, y)
        return float((y.double() * g.double()).sum())

    y, mean, rstd, dx = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    dga, dbe = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    ws = torch.empty(nb.nb_layer_norm_workspace_bytes(rows, c), dtype=torch.uint8, device="cuda")
    nb.nb_layer_norm_fwd(0, rows, c, x, ga, be, EPS, y, mean, rstd)
    nb.nb_layer_norm_bwd(0, rows, c, g, x, ga, mean, rstd, dx, dga, dbe, ws)
    for t, grad, args in ((x, dx, 0), (ga, dga, 1), (be, dbe, 2)):
        flat = t.view(-1)
        for i in range(flat.numel()):
            was = float(flat[i])
            flat[i] = was + h
            up = loss(x, ga, be)
            flat[i] = was - h
            down = loss(x, ga, be)
            flat[i] = was
            assert (up - down) / (2 * h) == pytest.approx(float(grad.view(-1)[i]), abs=5e-3), (args, i)


def test_captured_calls_and_repeated_bits():
    import torch

    from paper_2609_10632_b200 import binding as nb

    rows, c = 3000, 384
    x, g = torch.randn(rows, c, device="cuda").bfloat16(), torch.randn(rows, c, device="cuda").bfloat16()
    ga, be = torch.randn(c, device="cuda"), torch.randn(c, device="cuda")
    ws = torch.empty(nb.nb_layer_norm_workspace_bytes(rows, c), dtype=torch.uint8, device="cuda")
    out = [[torch.zeros_like(x), torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros_like(x), torch.zeros(c, device="cuda"), torch.zeros(c, device="cuda")]
           for _ in range(2)]

    def step(o):
        nb.nb_layer_norm_fwd(1, rows, c, x, ga, be, EPS, o[0], o[1], o[2])
        nb.nb_layer_norm_bwd(1, rows, c, g, x, ga, o[1], o[2], o[3], o[4], o[5], ws)

    step(out[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out[1])
    x2 = x.clone()
    x.normal_()
    graph.replay()
    assert not torch.equal(out[0][0], out[1][0])
    x.copy_(x2)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(*out):
        assert torch.equal(a, b)


def test_offsets_past_32_bits():
    """A 64-channel slice of rows 65536 elements apart: the last rows lie 9 GB behind the first."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    rows, c, ld = 70000, 64, 65536
    buf = torch.zeros(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    buf[:, 8 : 8 + c] = torch.randn(rows, c, device="cuda").bfloat16()
    x = buf[:, 8 : 8 + c]
    y, mean, rstd = torch.empty(rows, c, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    nb.nb_layer_norm_fwd(1, rows, c, x, None, None, EPS, y, mean, rstd, ld_x=ld)
    xc = x.contiguous()
    y2, dx, dx2 = torch.empty_like(y), torch.empty_like(y), torch.empty_like(y)
    nb.nb_layer_norm_fwd(1, rows, c, xc, None, None, EPS, y2)
    assert torch.equal(y, y2)
    nb.nb_layer_norm_bwd(1, rows, c, y, x, None, mean, rstd, dx, ld_x=ld)
    nb.nb_layer_norm_bwd(1, rows, c, y, xc, None, mean, rstd, dx2)
    assert torch.equal(dx, dx2)


@pytest.mark.parametrize("c", [1, 31, 96, 97, 1000])
def test_a_mean_that_times_rstd_overflows(c):
    """Constant rows of 2^120 with rstd 2^12: x - mean is 0, so dx is rstd (g - mean of g).  Lanes without a channel form no 0 * inf."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    rows = 9
    x, g, dx = torch.full((rows, c), 2.0**120, device="cuda"), torch.randn(rows, c, device="cuda"), torch.empty(rows, c, device="cuda")
    mean, rstd = torch.full((rows,), 2.0**120, device="cuda"), torch.full((rows,), 2.0**12, device="cuda")
    nb.nb_layer_norm_bwd(0, rows, c, g, x, None, mean, rstd, dx)
    hg = g.double().cpu().numpy()
    want = 4096.0 * (hg - hg.mean(1, keepdims=True))
    _close("dx", dx, want, 2.0**-17 * 4096.0 * (np.abs(hg) + np.abs(hg).mean(1, keepdims=True)))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("c", [24, 100, 1000, 1001, 1304, 5000, 20000, 100001, 1 << 20])
def test_constant_rows_have_their_constant_as_mean(c, dtype):
    """Constants whose sums are numbers of fp32 at every length, so that y is beta; and one whose sums are not: a lane adds up to 32 terms
    one after the other and five levels follow, 37 roundings of 2^-24, which is below the 2^-18 of this file."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    dt, code, _ = _types(torch)[dtype]
    x = torch.tensor([1000.0, -57.25, 3.0, 0.1], device="cuda").to(dt)[:, None].expand(4, c).contiguous()
    y, mean, rstd, beta = torch.empty_like(x), torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.full((c,), 0.25, device="cuda")
    nb.nb_layer_norm_fwd(code, 4, c, x, None, beta, EPS, y, mean, rstd)
    assert torch.equal(mean[:3], x[:3, 0].float()) and (y[:3] == 0.25).all()
    v = float(x[3, 0])
    assert abs(float(mean[3]) - v) <= 2.0**-18 * v and ((y[3].double() - 0.25).abs() <= 2.0**-18 * v / EPS**0.5 + torch.finfo(dt).eps / 8).all()


def test_rows_of_a_million_channels():
    """Sums of a million terms of one sign and of both, forward and backward, to the roundings of fp32 values summed in fp64."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    c = (1 << 20) + 1
    x = torch.rand(2, c, device="cuda") + torch.tensor([[3.0], [-0.5]], device="cuda")
    g, ga = torch.rand(2, c, device="cuda") + 0.5, torch.rand(c, device="cuda") + 0.5
    y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    nb.nb_layer_norm_fwd(0, 2, c, x, ga, None, EPS, y, mean, rstd)
    nb.nb_layer_norm_bwd(0, 2, c, g, x, ga, mean, rstd, dx)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    want, wmean, wrstd = ora.layer_norm_fwd(f(x), f(ga), None, EPS)
    _close("mean", mean, wmean, 2.0**-22 * np.abs(wmean) + 2.0**-22)  # (eight at a time in fp32: 2^-22 of their sum at most)
    _close("rstd", rstd, wrstd, 2.0**-20 * wrstd)
    _close("y", y, want, 2.0**-19 * (np.abs(want) + f(ga) * 4.0 * wrstd[:, None]))
    wdx, _, _ = ora.layer_norm_bwd(f(g), f(x), f(ga), f(mean), f(rstd))
    _close("dx", dx, wdx, 2.0**-19 * wrstd[:, None] * (2.25 + 2.25 + 2.0 * 2.25 * 2.0))


@pytest.mark.parametrize("c", [8, 96, 999, 4096, 20000])
def test_an_infinite_sum_is_an_infinite_mean(c):
    import torch

    from paper_2609_10632_b200 import binding as nb

    x = torch.randn(3, c, device="cuda")
    x[1, 0], x[2, c - 1] = float("inf"), float("-inf")
    y, mean, rstd = torch.empty_like(x), torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    nb.nb_layer_norm_fwd(0, 3, c, x, None, None, EPS, y, mean, rstd)
    assert mean[0].isfinite() and mean[1] == float("inf") and mean[2] == float("-inf")
