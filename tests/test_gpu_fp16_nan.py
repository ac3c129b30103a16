"""A NaN stays a NaN in fp16: what saturates at +-65504 is what is too large, and a loss scaler that looks for NaN behind any of these
calls finds it."""
import pytest

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.mark.parametrize("rows, c, ld", [(9, 96, 96), (9, 31, 31), (9, 300, 300), (9, 999, 999), (9, 999, 1001), (9, 4096, 4096), (5, 4098, 4099), (9, 16400, 16400)])
def test_layer_norm(rows, c, ld):
    """Every form of the kernels: lanes of a warp, a block, single elements, tiles of rows, rows that are read again."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    m = lambda: torch.randn(rows, ld, device="cuda").half()[:, :c]  # noqa: E731
    x, g, y, dx = m(), m(), m(), m()
    mean, rstd = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    keep = [r for r in range(rows) if r != 3]
    x[3, c // 2] = float("nan")
    nb.nb_layer_norm_fwd(nb.NB_DTYPE_F16, rows, c, x, None, None, EPS, y, mean, rstd, ld_x=ld, ld_y=ld)
    assert y[3].isnan().all() and y[keep].isfinite().all() and mean[3].isnan()
    x[3], mean[3], rstd[3] = 1.0, 0.0, 1.0
    g[3, 1] = float("nan")
    nb.nb_layer_norm_bwd(nb.NB_DTYPE_F16, rows, c, g, x, None, mean, rstd, dx, ld_g=ld, ld_x=ld, ld_dx=ld)
    assert dx[3].isnan().all() and dx[keep].isfinite().all()


@pytest.mark.parametrize("rows, n, flags", [(5, 64, 0), (130, 64, 0), (5, 64, 1), (130, 64, 1), (130, 63, 0), (1500, 333, 0)])
def test_linear(rows, n, flags):
    """A few rows, the tensor cores, the CUDA cores, odd counts there and on padded copies."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    plan = nb.LinearPlan(n, n, nb.NB_DTYPE_F16, flags=flags)
    ws = torch.empty(plan.workspace_bytes(rows), dtype=torch.uint8, device="cuda")
    h = lambda r: torch.randn(r, n, device="cuda").half()  # noqa: E731
    x, w, dy, z, out, dx = h(rows), h(n), h(rows), h(rows), h(rows), h(rows)
    keep = [r for r in range(rows) if r != 2]
    x[2, 1] = float("nan")
    for act in (nb.NB_ACT_NONE, nb.NB_ACT_SILU, nb.NB_ACT_GELU):
        nb.nb_linear_fwd(plan, rows, x, w, None, act, out, ws, z=z)
        assert out[2].isnan().all() and z[2].isnan().all() and out[keep].isfinite().all() and z[keep].isfinite().all()
    z.normal_()
    dy[2, 0] = float("nan")
    for act in (nb.NB_ACT_NONE, nb.NB_ACT_SILU, nb.NB_ACT_GELU):
        nb.nb_linear_bwd_data(plan, rows, dy, w, dx, ws, z_in=z if act else None, act_in=act)
        assert dx[2].isnan().all() and dx[keep].isfinite().all()
    dy.normal_()
    z[2, 4] = float("nan")
    for act in (nb.NB_ACT_SILU, nb.NB_ACT_GELU):
        nb.nb_linear_bwd_data(plan, rows, dy, w, dx, ws, z_in=z, act_in=act)
        assert dx[2, 4].isnan() and int(dx.isnan().sum()) == 1


@pytest.mark.parametrize("n", [16, 4099])
def test_act_bwd(n):
    import torch

    from paper_2609_10632_b200 import binding as nb

    for act in (nb.NB_ACT_SILU, nb.NB_ACT_GELU):
        for which in (0, 1):
            dy, z, dz = (torch.randn(n, device="cuda").half() for _ in range(3))
            (dy, z)[which][n - 1] = float("nan")
            nb.nb_act_bwd(nb.NB_DTYPE_F16, n, act, dy, z, dz)
            assert dz[n - 1].isnan() and int(dz.isnan().sum()) == 1


@pytest.mark.parametrize("bits", [32, 8])
def test_copies_of_the_parameters(bits):
    """AdamW and SGD with a learning rate of 0: the copies are the parameters, rounded; only what is too large saturates."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    inf, nan = float("inf"), float("nan")
    p = torch.tensor([nan, inf, -inf, 1e30, -1e30, 65504.0, 65519.9, 65520.0, 1.0, 2.0**-24, 2.0**-25, 3 * 2.0**-25, -nan] * 11, device="cuda")
    want = torch.where(p.isnan(), p, p.clamp(-65504.0, 65504.0)).half()
    n = p.numel()
    z = lambda: torch.zeros(n, device="cuda")  # noqa: E731
    copy = z().half()
    if bits == 32:
        items = [(z(), p.clone(), z(), z(), copy, 0)]
    else:
        q = lambda: z().to(torch.float8_e4m3fn)  # noqa: E731
        items = [(z(), p.clone(), q(), q(), copy, 0, torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda"))]
    plan = nb.AdamWPlan(items)
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    plan.upload(ws)
    plan.step(ws, torch.zeros(1, dtype=torch.int64, device="cuda"), [0.0] * 3, [0.0] * 3, 0.9, 0.999, 1e-8, 0.0)
    assert torch.equal(copy.nan_to_num(7.0, 8.0, 9.0), want.nan_to_num(7.0, 8.0, 9.0)) and torch.equal(copy.isnan(), p.isnan())


def test_glue_calls_share_the_rounding():
    import torch

    from paper_2609_10632_b200 import binding as nb

    a, b, d = (torch.ones(6, 16, device="cuda").half() for _ in range(3))
    a[2, 3], a[3, 4], b[3, 4] = float("nan"), 60000.0, 60000.0
    nb.nb_slice_add(nb.NB_DTYPE_F16, 6, 16, d, 16, a, 16, b, 16)
    torch.cuda.synchronize()
    assert d[2, 3].isnan() and int(d.isnan().sum()) == 1 and d[3, 4] == 65504.0
