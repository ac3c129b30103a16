"""AdamW without a GPU: the oracle against hand-worked numbers and against the framework's own CPU optimiser in float64, the
8-bit form's number system against torch's, and the list checks of nb_adamw_plan_create."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import adamw as ora
from paper_2609_10632_b200 import binding as nb
from paper_2609_10632_b200 import build as nbbuild


@pytest.fixture(scope="module")
def lib():
    nbbuild.build()
    return nb.load()


def test_oracle_by_hand():
    # m = 0.1*2 = 0.2, v = 0.001*4 = 0.004; mhat = 2, vhat = 4: p = 1 - 0.1*0.5*1 - 0.1*2/(2+0) = 0.85
    p, m, v = ora.adamw_update([1.0], [2.0], [0.0], [0.0], 1, 0.1, 0.9, 0.999, 0.0, 0.5)
    assert np.allclose([p[0], m[0], v[0]], [0.85, 0.2, 0.004], rtol=1e-14)


def test_oracle_follows_the_frameworks_own_optimiser():
    rng = np.random.default_rng(1)
    p0 = [rng.normal(size=50), rng.normal(size=7)]
    ref = [torch.tensor(p, dtype=torch.float64, requires_grad=True) for p in p0]
    opt = torch.optim.AdamW([{"params": [ref[0]], "weight_decay": 0.1, "lr": 3e-3}, {"params": [ref[1]], "weight_decay": 0.0, "lr": 1e-2}], betas=(0.9, 0.99), eps=1e-6)
    ps, ms, vs = p0, [np.zeros(50), np.zeros(7)], [np.zeros(50), np.zeros(7)]
    for t in range(1, 6):
        g = [rng.normal(size=50), rng.normal(size=7)]
        for r, x in zip(ref, g):
            r.grad = torch.tensor(x)
        want_total = float(torch.nn.utils.clip_grad_norm_(ref, 3.0))
        opt.step()
        ps, ms, vs, total = ora.clip_adamw_step(ps, g, ms, vs, [0, 1], t, [3e-3, 1e-2], [0.1, 0.0], 0.9, 0.99, 1e-6, 3.0)
        assert total == pytest.approx(want_total, rel=1e-12)
        for a, r in zip(ps, ref):
            np.testing.assert_allclose(a, r.detach().numpy(), rtol=1e-12)


def test_e4m3_numbers_are_those_of_the_type():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, ora.E4M3)
    rng = np.random.default_rng(2)
    x = np.concatenate([rng.normal(size=4000) * 100, rng.normal(size=4000) * 0.01, ora.E4M3, (ora.E4M3[1:] + ora.E4M3[:-1]) / 2, [1e-5, 448.0]]).astype(np.float32)
    x = np.clip(x, -448.0, 448.0)
    assert np.array_equal(ora.to_e4m3(x.astype(np.float64)), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


def test_encode_keeps_roots_off_zero_and_small_blocks_at_zero():
    q, s = ora.encode([1.0, 1e-9, 0.0], True)
    assert q[0] == 448.0 and q[1] == 2.0**-9 and q[2] == 0.0 and s[0] == 1.0 / 448.0
    q, s = ora.encode([2.0**-101, 0.0], True)
    assert not q.any() and s[0] == 0.0
    q, s = ora.encode(np.full(129, -3.0), False)
    assert (q == -448.0).all() and s.shape == (2,)


def _tensor(**over):
    d = dict(grad=0x10000, param=0x20000, exp_avg=0x30000, exp_avg_sq=0x40000, exp_avg_scale=None, exp_avg_sq_scale=None, param_copy=None, numel=16, group=0,
             copy_dtype=0, grad_dtype=0, state_bits=32)
    d.update(over)
    return nb.nb_adamw_tensor(**d)


@pytest.mark.parametrize("over, code, word", [
    (dict(numel=0), nb.NB_ERR_INVALID_ARG, "numel"),
    (dict(numel=-4), nb.NB_ERR_INVALID_ARG, "numel"),
    (dict(numel=1 << 43), nb.NB_ERR_UNSUPPORTED, "elements"),
    (dict(group=3), nb.NB_ERR_INVALID_ARG, "group"),
    (dict(group=-1), nb.NB_ERR_INVALID_ARG, "group"),
    (dict(grad=None), nb.NB_ERR_INVALID_ARG, "NULL"),
    (dict(param=None), nb.NB_ERR_INVALID_ARG, "NULL"),
    (dict(exp_avg_sq=None), nb.NB_ERR_INVALID_ARG, "NULL"),
    (dict(grad_dtype=5), nb.NB_ERR_INVALID_ARG, "grad_dtype"),
    (dict(copy_dtype=7), nb.NB_ERR_INVALID_ARG, "copy_dtype"),
    (dict(state_bits=16), nb.NB_ERR_INVALID_ARG, "state_bits"),
    (dict(state_bits=8), nb.NB_ERR_INVALID_ARG, "scale"),
    (dict(state_bits=8, exp_avg_scale=0x50000), nb.NB_ERR_INVALID_ARG, "scale"),
    (dict(exp_avg_scale=0x50000, exp_avg_sq_scale=0x60000), nb.NB_ERR_INVALID_ARG, "scale"),
    (dict(state_bits=8, exp_avg_scale=0x50002, exp_avg_sq_scale=0x60000), nb.NB_ERR_ALIGNMENT, "scale"),
    (dict(param=0x20004), nb.NB_ERR_ALIGNMENT, "aligned"),
    (dict(param_copy=0x70008), nb.NB_ERR_ALIGNMENT, "aligned"),
    (dict(exp_avg=0x40000), nb.NB_ERR_INVALID_ARG, "overlap"),         # both moments in one buffer
    (dict(grad=0x20000), nb.NB_ERR_INVALID_ARG, "overlap"),            # the gradient lies in the parameter
    (dict(param_copy=0x20020), nb.NB_ERR_INVALID_ARG, "overlap"),
    (dict(exp_avg=0x30000, exp_avg_sq=0x30030), nb.NB_ERR_INVALID_ARG, "overlap"),
])
def test_bad_lists_are_refused_before_any_cuda_call(lib, over, code, word):
    h = ctypes.c_void_p()
    arr = (nb.nb_adamw_tensor * 1)(_tensor(**over))
    assert lib.nb_adamw_plan_create(arr, 1, 0, ctypes.byref(h)) == code
    assert word in nb.nb_last_error() and not h.value


def test_the_same_tensor_twice_and_neighbours(lib):
    h = ctypes.c_void_p()
    arr = (nb.nb_adamw_tensor * 2)(_tensor(), _tensor(grad=0x11000))
    assert lib.nb_adamw_plan_create(arr, 2, 0, ctypes.byref(h)) == nb.NB_ERR_INVALID_ARG and "overlap" in nb.nb_last_error()
    # two tensors that touch, and that share a gradient: no overlap is reported (without a device the next failure is CUDA's)
    arr = (nb.nb_adamw_tensor * 2)(_tensor(), _tensor(param=0x20040, exp_avg=0x30040, exp_avg_sq=0x40040))
    st = lib.nb_adamw_plan_create(arr, 2, 0, ctypes.byref(h))
    assert st == (nb.NB_OK if torch.cuda.is_available() else nb.NB_ERR_CUDA), nb.nb_last_error()
    lib.nb_adamw_plan_destroy(h)


def test_null_arguments_and_structures(lib):
    h = ctypes.c_void_p()
    assert lib.nb_adamw_plan_create(None, 1, 0, ctypes.byref(h)) == nb.NB_ERR_INVALID_ARG
    arr = (nb.nb_adamw_tensor * 1)(_tensor())
    assert lib.nb_adamw_plan_create(arr, 0, 0, ctypes.byref(h)) == nb.NB_ERR_INVALID_ARG
    assert lib.nb_adamw_plan_create(arr, 1, 0, None) == nb.NB_ERR_INVALID_ARG
    assert lib.nb_adamw_plan_destroy(None) == nb.NB_OK
    assert lib.nb_adamw_step(None, None, 0, None, None, None, None) == nb.NB_ERR_INVALID_ARG
    assert lib.nb_adamw_step_scaled(None, None, 0, None, None, None, None, None, None) == nb.NB_ERR_INVALID_ARG
    assert lib.nb_adamw_upload(None, None, 0, None) == nb.NB_ERR_INVALID_ARG
    assert ctypes.sizeof(nb.nb_adamw_tensor) == 80 and ctypes.sizeof(nb.nb_adamw_hyper) == 56


def test_binding_refuses_tensors_that_do_not_fit():
    t = torch.zeros(256)
    with pytest.raises(nb.NbError) as e:
        nb.AdamWPlan([(t, t, t, t, None, 0)])  # host tensors
    assert e.value.status == nb.NB_ERR_INVALID_ARG
    with pytest.raises(nb.NbError):
        nb.AdamWPlan([(t, t, t, t, None)])
