"""fp16 results of the MLP products that saturate are counted, as those of the convolutions are: nb_linear_poll_status stays NB_OK and
says how many, once."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows, n, flags", [(3, 64, 0), (200, 64, 0), (2500, 384, 0), (20, 64, 1), (200, 64, 1), (40, 2000, 1), (40, 63, 0), (1500, 333, 0)])
def test_saturated_results_are_counted(rows, n, flags):
    """A few rows, the tensor cores, the CUDA cores with and without slices, odd counts there and on padded copies: z, out and dx."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    plan = nb.LinearPlan(n, n, nb.NB_DTYPE_F16, flags=flags)
    ws = torch.empty(plan.workspace_bytes(rows), dtype=torch.uint8, device="cuda")
    h = lambda *s: torch.randn(*s, device="cuda").half()  # noqa: E731
    x, w, out, z, dx = h(rows, n), h(n, n), h(rows, n), h(rows, n), h(rows, n)

    def calls(act=nb.NB_ACT_GELU):
        nb.nb_linear_fwd(plan, rows, x, w, None, act, out, ws, z=z)
        nb.nb_linear_bwd_data(plan, rows, x, w, dx, ws)

    calls()
    assert plan.poll() == ""
    x[rows - 1] = 60000.0
    w[5] = -1.0  # z of column 5: -3.8 million; its GELU is zero
    w[:, 6] = 1.0  # dx of column 6 likewise
    w[5, 6] = 0.0
    for act, call in ((nb.NB_ACT_GELU, "fwd"), (nb.NB_ACT_NONE, "fwd"), (None, "data")):
        if call == "fwd":
            nb.nb_linear_fwd(plan, rows, x, w, None, act, out, ws, z=z if act else None)
            assert (z if act else out)[rows - 1, 5] == -65504.0
        else:
            nb.nb_linear_bwd_data(plan, rows, x, w, dx, ws)
            assert dx[rows - 1, 6] == 65504.0
        msg = plan.poll()
        assert "saturated" in msg and int(msg.split()[0]) > 0
        assert plan.poll() == ""  # (once)
    plan.close()


def test_other_types_count_nothing():
    import torch

    from paper_2609_10632_b200 import binding as nb

    for code, dt in ((nb.NB_DTYPE_BF16, torch.bfloat16), (nb.NB_DTYPE_F32, torch.float32)):
        plan = nb.LinearPlan(64, 64, code)
        ws = torch.empty(plan.workspace_bytes(100), dtype=torch.uint8, device="cuda")
        x, w, out = torch.full((100, 64), 60000.0, device="cuda").to(dt), torch.ones(64, 64, device="cuda").to(dt), torch.empty(100, 64, dtype=dt, device="cuda")
        nb.nb_linear_fwd(plan, 100, x, w, None, 0, out, ws)
        assert plan.poll() == "" and float(out[0, 0]) > 1e6


def test_a_block_tells():
    import torch

    from paper_2609_10632_b200 import binding as nb
    from paper_2609_10632_b200.mlp import MlpBlock

    b = MlpBlock(200, 64, 256, nb.NB_DTYPE_F16)
    r = lambda *s: torch.randn(*s, device="cuda")  # noqa: E731
    b.load(w1=r(256, 64) / 8, w2=r(64, 256) / 16, gamma=torch.ones(64, device="cuda"), beta=r(64), b1=r(256), b2=r(64))
    b.x.normal_()
    b.dy.normal_()
    b.forward()
    b.backward()
    assert b.poll() == ""
    b.dy.fill_(60000.0)  # a loss scale far too large: dz and dh saturate
    b.backward()
    note = b.poll()
    assert "up: " in note and "down: " in note and "saturated" in note and b.poll() == ""
