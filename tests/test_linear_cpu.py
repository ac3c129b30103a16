"""The MLP products without a GPU: the oracle by hand, against the framework's own float64 routines and against differences; the
refusals of the C ABI, which come before anything touches a device."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import linear as ora
from paper_2609_10632_b200 import binding as nb
from paper_2609_10632_b200 import build as nbbuild


@pytest.fixture(scope="module")
def lib():
    nbbuild.build()
    return nb.load()


def test_oracle_by_hand():
    z, out = ora.linear_fwd([[1.0, 2.0]], [[3.0, 4.0], [-1.0, 0.5]], [0.5, 0.0], "none", [[1.0, 1.0]])
    assert z.tolist() == [[11.5, 0.0]] and out.tolist() == [[12.5, 1.0]]
    assert ora.act(0.0, "gelu") == 0.0 and ora.act_grad(0.0, "gelu") == 0.5 and ora.act_grad(0.0, "silu") == 0.5
    assert ora.linear_bwd_data([[1.0, 2.0]], [[3.0, 4.0], [-1.0, 0.5]]).tolist() == [[1.0, 5.0]]
    dw, db = ora.linear_bwd_weight([[1.0, 2.0], [0.0, 1.0]], [[1.0, 0.0], [2.0, 3.0]])
    assert dw.tolist() == [[1.0, 4.0], [0.0, 3.0]] and db.tolist() == [3.0, 3.0]


@pytest.mark.parametrize("kind", ["none", "silu", "gelu"])
def test_oracle_against_the_framework_and_differences(kind):
    rng = np.random.default_rng(1)
    x, w, b, res, g = rng.normal(size=(4, 5)), rng.normal(size=(6, 5)), rng.normal(size=6), rng.normal(size=(4, 6)), rng.normal(size=(4, 6))
    t = [torch.tensor(v, requires_grad=True) for v in (x, w, b)]
    f = {"none": lambda v: v, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[kind]
    want = f(torch.nn.functional.linear(*t)) + torch.tensor(res)
    want.backward(torch.tensor(g))
    z, out = ora.linear_fwd(x, w, b, kind, res)
    dz = g * ora.act_grad(z, kind)
    dw, db = ora.linear_bwd_weight(x, dz)
    for got, ref in ((out, want), (ora.linear_bwd_data(dz, w), t[0].grad), (dw, t[1].grad), (db, t[2].grad)):
        np.testing.assert_allclose(got, ref.detach().numpy(), rtol=1e-10, atol=1e-12)
    v = np.linspace(-5, 5, 41)
    np.testing.assert_allclose((ora.act(v + 1e-6, kind) - ora.act(v - 1e-6, kind)) / 2e-6, ora.act_grad(v, kind), rtol=1e-7, atol=1e-8)


@pytest.mark.parametrize("over, code, word", [
    (dict(size=8), nb.NB_ERR_INVALID_ARG, "struct_size"), (dict(c_in=0), nb.NB_ERR_INVALID_ARG, "c_in"), (dict(c_out=-8), nb.NB_ERR_INVALID_ARG, "c_out"),
    (dict(c_in=(1 << 24) + 1), nb.NB_ERR_INVALID_ARG, "2^24"), (dict(dtype=9), nb.NB_ERR_INVALID_ARG, "dtype"), (dict(flags=2), nb.NB_ERR_INVALID_ARG, "flags"),
])
def test_bad_descriptors_are_rejected_before_any_cuda_call(lib, over, code, word):
    d = dict(size=ctypes.sizeof(nb.nb_linear_desc), c_in=64, c_out=64, dtype=1, flags=0)
    d.update(over)
    desc, h = nb.nb_linear_desc(d["size"], d["c_in"], d["c_out"], d["dtype"], d["flags"]), ctypes.c_void_p()
    assert lib.nb_linear_plan_create(ctypes.byref(desc), 0, ctypes.byref(h)) == code
    assert word in nb.nb_last_error() and not h.value


def test_null_plans_and_arguments(lib):
    assert lib.nb_linear_plan_create(None, 0, ctypes.byref(ctypes.c_void_p())) == nb.NB_ERR_INVALID_ARG
    assert lib.nb_linear_plan_destroy(None) == nb.NB_OK
    assert lib.nb_linear_workspace_bytes(None, 1, ctypes.byref(ctypes.c_size_t())) == nb.NB_ERR_INVALID_ARG
    assert lib.nb_linear_paths(None, 1, (ctypes.c_int32 * 3)()) == nb.NB_ERR_INVALID_ARG
    assert lib.nb_linear_poll_status(None, None) == nb.NB_ERR_INVALID_ARG
    assert lib.nb_linear_fwd(None, 1, None, 0, None, None, 0, None, 0, None, None, 0, None, 0, None) == nb.NB_ERR_INVALID_ARG
    assert lib.nb_linear_bwd_data(None, 1, None, 0, None, None, 0, None, 0, None, 0, None, 0, None) == nb.NB_ERR_INVALID_ARG
    assert lib.nb_linear_bwd_weight(None, 1, None, 0, None, 0, None, None, None, 0, None) == nb.NB_ERR_INVALID_ARG
    assert ctypes.sizeof(nb.nb_linear_desc) == 20


@pytest.mark.parametrize("over, code, word", [
    (dict(dtype=4), nb.NB_ERR_INVALID_ARG, "dtype"), (dict(n=0), nb.NB_ERR_INVALID_ARG, "n must"), (dict(act=0), nb.NB_ERR_INVALID_ARG, "act"),
    (dict(act=3), nb.NB_ERR_INVALID_ARG, "act"), (dict(dy=None), nb.NB_ERR_INVALID_ARG, "NULL"), (dict(z=0x10001), nb.NB_ERR_ALIGNMENT, "aligned"),
])
def test_act_bwd_refusals(lib, over, code, word):
    d = dict(dtype=1, n=64, act=2, dy=0x10000, z=0x10000, dz=0x10000)
    d.update(over)
    assert lib.nb_act_bwd(*d.values(), None) == code
    assert word in nb.nb_last_error()


def test_plan_create_without_a_device_fails_loudly(lib):
    if torch.cuda.is_available():
        pytest.skip("a CUDA device is present")
    with pytest.raises(nb.NbError) as e:
        nb.LinearPlan(64, 64, nb.NB_DTYPE_BF16)
    assert e.value.status == nb.NB_ERR_CUDA


def test_every_wait_of_the_tensor_core_products_reports_when_it_gives_up():
    """Read from the source, since no call may make a wait run out: each role waits at a site of its own that the list in common.cuh counts,
    through wait_bar / wait_bar_fast or a bounded loop with give_up behind it; a bare loop over mbar_try_wait only follows a wait
    that has given up (for what is still in flight), or waits for the MMAs issued so far before TMEM is released."""
    import os
    import re

    csrc = os.path.join(os.path.dirname(os.path.abspath(nb.__file__)), "csrc")
    lines = open(os.path.join(csrc, "tc_linear.cuh")).read().split("\n")
    sites = [int(m) for line in lines for m in re.findall(r"\b(?:wait_bar|wait_bar_fast|give_up)\([^;]*p\.status, (\d+)\)", line)]
    assert sorted(sites) == [21, 22, 23, 24, 25]
    assert "21-25" in open(os.path.join(csrc, "common.cuh")).read()
    for i, line in enumerate(lines):
        if "mbar_try_wait" in line:
            assert "drain" in line or "give_up(" in lines[i + 2] or any("if (!ok)" in before for before in lines[i - 6 : i]), (i + 1, line)
