"""Layer norm without a GPU: the oracle by hand, against the framework's own float64 routine and against differences; the
refusals of the C ABI, which come before anything touches a device."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import norm as ora
from paper_2609_10632_b200 import binding as nb
from paper_2609_10632_b200 import build as nbbuild


@pytest.fixture(scope="module")
def lib():
    nbbuild.build()
    return nb.load()


def test_oracle_by_hand():
    # mean 2, deviations -1, 1: variance 1, eps 0 -> xhat -1, 1
    y, mean, rstd = ora.layer_norm_fwd([[1.0, 3.0]], [2.0, 0.5], [10.0, 0.0], 0.0)
    assert y.tolist() == [[8.0, 0.5]] and mean[0] == 2.0 and rstd[0] == 1.0
    dx, dgamma, dbeta = ora.layer_norm_bwd([[1.0, 4.0]], [[1.0, 3.0]], [2.0, 0.5], mean, rstd)
    # d = (2, 2): the mean takes all of it, d*xhat = (-2, 2) has mean 0
    assert dx.tolist() == [[0.0, 0.0]] and dgamma.tolist() == [-1.0, 4.0] and dbeta.tolist() == [1.0, 4.0]


def test_oracle_against_the_framework_and_differences():
    rng = np.random.default_rng(1)
    x, g, ga, be = rng.normal(size=(5, 7)) + 3.0, rng.normal(size=(5, 7)), rng.normal(size=7), rng.normal(size=7)
    t = [torch.tensor(v, requires_grad=True) for v in (x, ga, be)]
    want = torch.nn.functional.layer_norm(t[0], (7,), t[1], t[2], 1e-5)
    want.backward(torch.tensor(g))
    y, mean, rstd = ora.layer_norm_fwd(x, ga, be, 1e-5)
    dx, dga, dbe = ora.layer_norm_bwd(g, x, ga, mean, rstd)
    for got, ref in zip((y, dx, dga, dbe), (want, t[0].grad, t[1].grad, t[2].grad)):
        np.testing.assert_allclose(got, ref.detach().numpy(), rtol=1e-9, atol=1e-12)
    h = 1e-5
    for r, c in [(0, 0), (3, 6), (4, 2)]:
        xp, xm = x.copy(), x.copy()
        xp[r, c] += h
        xm[r, c] -= h
        diff = ((ora.layer_norm_fwd(xp, ga, be, 1e-5)[0] - ora.layer_norm_fwd(xm, ga, be, 1e-5)[0]) * g).sum() / (2 * h)
        assert diff == pytest.approx(dx[r, c], rel=1e-5, abs=1e-8)


P = 0x10000


@pytest.mark.parametrize("over, code, word", [
    (dict(dtype=7), nb.NB_ERR_INVALID_ARG, "dtype"), (dict(rows=0), nb.NB_ERR_INVALID_ARG, "rows"), (dict(rows=-1), nb.NB_ERR_INVALID_ARG, "rows"),
    (dict(c=0), nb.NB_ERR_INVALID_ARG, "positive"), (dict(c=(1 << 24) + 1), nb.NB_ERR_INVALID_ARG, "2^24"), (dict(x=None), nb.NB_ERR_INVALID_ARG, "NULL"),
    (dict(y=None), nb.NB_ERR_INVALID_ARG, "NULL"), (dict(mean=P), nb.NB_ERR_INVALID_ARG, "together"), (dict(eps=0.0), nb.NB_ERR_INVALID_ARG, "eps"),
    (dict(eps=float("nan")), nb.NB_ERR_INVALID_ARG, "eps"), (dict(ld_x=15), nb.NB_ERR_INVALID_ARG, "ld_x"), (dict(ld_y=-16), nb.NB_ERR_INVALID_ARG, "ld_y"),
    (dict(x=P + 1), nb.NB_ERR_ALIGNMENT, "x"), (dict(gamma=P + 2), nb.NB_ERR_ALIGNMENT, "gamma"), (dict(mean=P + 1, rstd=P), nb.NB_ERR_ALIGNMENT, "mean"),
])
def test_forward_refusals(lib, over, code, word):
    d = dict(dtype=1, rows=4, c=16, x=P, ld_x=0, gamma=P, beta=P, eps=1e-5, y=P, ld_y=0, mean=None, rstd=None)
    d.update(over)
    assert lib.nb_layer_norm_fwd(*d.values(), None) == code
    assert word in nb.nb_last_error()


@pytest.mark.parametrize("over, code, word", [
    (dict(dtype=-1), nb.NB_ERR_INVALID_ARG, "dtype"), (dict(rows=0), nb.NB_ERR_INVALID_ARG, "rows"), (dict(g=None), nb.NB_ERR_INVALID_ARG, "NULL"),
    (dict(mean=None), nb.NB_ERR_INVALID_ARG, "NULL"), (dict(dx=None), nb.NB_ERR_INVALID_ARG, "NULL"), (dict(dbeta=None), nb.NB_ERR_INVALID_ARG, "together"),
    (dict(ld_g=8), nb.NB_ERR_INVALID_ARG, "ld_g"), (dict(add=P, ld_add=8), nb.NB_ERR_INVALID_ARG, "ld_add"), (dict(add=P + 1), nb.NB_ERR_ALIGNMENT, "add"),
    (dict(dgamma=P + 2), nb.NB_ERR_ALIGNMENT, "dgamma"), (dict(ws=None), nb.NB_ERR_WORKSPACE, "NULL"), (dict(ws=P + 128), nb.NB_ERR_WORKSPACE, "aligned"),
    (dict(ws_bytes=255), nb.NB_ERR_WORKSPACE, "bytes"),
])
def test_backward_refusals(lib, over, code, word):
    d = dict(dtype=1, rows=4, c=16, g=P, ld_g=0, x=P, ld_x=0, gamma=P, mean=P, rstd=P, add=None, ld_add=0, dx=P, ld_dx=0, dgamma=P, dbeta=P, ws=P, ws_bytes=1 << 20)
    d.update(over)
    assert lib.nb_layer_norm_bwd(*d.values(), None) == code
    assert word in nb.nb_last_error()


def test_workspace_bytes(lib):
    assert lib.nb_layer_norm_workspace_bytes(4, 16, None) == nb.NB_ERR_INVALID_ARG
    assert lib.nb_layer_norm_workspace_bytes(0, 16, ctypes.byref(ctypes.c_size_t())) == nb.NB_ERR_INVALID_ARG
    assert nb.nb_layer_norm_workspace_bytes(1, 1) == 256
    assert nb.nb_layer_norm_workspace_bytes(10**9, 8192) >= 2 * 8192 * 4
