"""The fused AdamW step (include/nb_adamw.h) on the GPU against the fp64 oracle, in 32 and in 8 bits.

Tolerances.  32 bits: parameters and moments at the fp32 bar of the other optimiser test (relative L2 1e-5; a step takes about
ten roundings of 2^-24).  8 bits: from the state that the GPU held before a step, the oracle's m and sqrt(v) over the GPU's new
scale must round to the code that the GPU wrote, where the value may be off by 2^-20 (at most sixteen roundings of 2^-24) of what it
is a sum of: m = b1*m + (1-b1)*g may cancel, and each summand carries its own rounding errors (the clip coefficient, the two
products), so the bound is 2^-20 * (|b1*m| + |(1-b1)*g|); v has summands of one sign, its bound is relative.  Scales are
the oracle's within the same bound of the block's largest sum of summands.  Copies are the GPU's own parameters rounded, exactly."""
import numpy as np
import pytest

from oracle import adamw as ora
from tests import parity

pytestmark = pytest.mark.gpu

LR, WD = [1e-3, 3e-3, 2e-3], [0.1, 0.0, 0.0]
B1, B2, EPS = 0.9, 0.999, 1e-8
NEAR = 2.0**-20


def _dt(torch, name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


class State:
    """A list of tensors, each with 64 guard elements behind it that no step may touch."""

    GUARD = 64

    def __init__(self, spec, seed, moments="nan"):
        import torch

        from paper_2609_10632_b200 import binding as nb

        self.torch, self.nb, self.spec = torch, nb, spec  # spec: (numel, group, bits, grad dtype, copy dtype or None)
        self.rng = np.random.default_rng(seed)
        self.full, self.t = [], []
        for numel, group, bits, gd, cd in spec:
            blocks = -(-numel // 128)
            mdt = torch.float8_e4m3fn if bits == 8 else torch.float32
            full = {"g": self._buf(numel, _dt(torch, gd)), "p": self._buf(numel, torch.float32), "m": self._buf(numel, mdt), "v": self._buf(numel, mdt),
                    "c": self._buf(numel, _dt(torch, cd)) if cd else None, "ms": self._buf(blocks, torch.float32) if bits == 8 else None,
                    "vs": self._buf(blocks, torch.float32) if bits == 8 else None}
            self.full.append(full)
            n = {"ms": blocks, "vs": blocks}
            self.t.append({k: None if f is None else f[: n.get(k, numel)] for k, f in full.items()})
            self.t[-1]["p"].copy_(torch.from_numpy((0.1 * self.rng.normal(size=numel)).astype(np.float32)))
            for k in ("m", "v", "ms", "vs"):  # the first step takes no notice of what they hold
                if self.t[-1][k] is not None:
                    self.t[-1][k].fill_(float("nan"))
        self.plan = nb.AdamWPlan([(t["g"], t["p"], t["m"], t["v"], t["c"], s[1]) + ((t["ms"], t["vs"]) if s[2] == 8 else ()) for t, s in zip(self.t, spec)])
        self.ws = torch.empty(self.plan.workspace_bytes, dtype=torch.uint8, device="cuda")
        self.plan.upload(self.ws)
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.norm = torch.zeros(1, device="cuda")
        self.snap = [self._guards(f) for f in self.full]

    def _buf(self, n, dt):
        torch = self.torch
        f = torch.zeros(-(-n // 64) * 64 + self.GUARD, dtype=torch.float32, device="cuda")
        f[n:] = 7.5
        return f.to(dt)

    def _guards(self, full):
        return {k: f.view(self.torch.uint8).clone() for k, f in full.items() if f is not None}

    def grads(self, scale, k=None):
        out = []
        for t, (numel, *_r) in zip(self.t, self.spec):
            g = scale * self.rng.normal(size=numel) * np.exp(self.rng.normal(size=numel))
            t["g"].copy_(self.torch.from_numpy(g.astype(np.float32)))
            out.append(t["g"].double().cpu().numpy())
        return out

    def moments(self):
        """What the GPU holds, as (m, v) in fp64."""
        ms, vs = [], []
        for t, (numel, _g, bits, *_r) in zip(self.t, self.spec):
            m, v = t["m"].float().double().cpu().numpy(), t["v"].float().double().cpu().numpy()
            if bits == 8:
                m, v = ora.decode(m, t["ms"].double().cpu().numpy(), False), ora.decode(v, t["vs"].double().cpu().numpy(), True)
            ms.append(m)
            vs.append(v)
        return ms, vs

    def check(self, before, grads, t, max_norm, what):
        ps, ms, vs = before
        old, clip = ms, min(1.0, max_norm / (ora.clip_global_norm(grads, np.inf)[1] + 1e-6)) if 0.0 < max_norm < np.inf else 1.0
        ps, ms, vs, total = ora.clip_adamw_step(ps, grads, ms, vs, [s[1] for s in self.spec], t, LR, WD, B1, B2, EPS, max_norm)
        for i, (x, (numel, _g, bits, _gd, cd)) in enumerate(zip(self.t, self.spec)):
            parity.check(f"{what} param[{i}]", x["p"].double().cpu().numpy(), ps[i], "f32")
            if bits == 32:
                parity.check(f"{what} m[{i}]", x["m"].double().cpu().numpy(), ms[i], "f32")
                parity.check(f"{what} v[{i}]", x["v"].double().cpu().numpy(), vs[i], "f32")
            else:
                for q, s, val, root in ((x["m"], x["ms"], ms[i], False), (x["v"], x["vs"], np.sqrt(vs[i]), True)):
                    _, want_s = ora.encode(val, root)
                    got_s = s.double().cpu().numpy()
                    parts = (B1 * np.abs(old[i]) + (1 - B1) * clip * np.abs(grads[i])) if not root else np.zeros(numel)
                    most = np.pad(parts, (0, -numel % 128)).reshape(-1, 128).max(1)
                    assert (np.abs(got_s - want_s) <= NEAR * (want_s + most / 448.0)).all()
                    u = val / np.repeat(np.where(got_s > 0, got_s, 1.0), 128)[:numel] * np.repeat(got_s > 0, 128)[:numel]
                    if root:
                        u = np.where(u > 0, np.maximum(u, 2.0**-9), u)
                    off = NEAR * np.abs(u)
                    if not root:
                        off = off + NEAR * parts / np.repeat(np.where(got_s > 0, got_s, np.inf), 128)[:numel]
                    got = q.float().double().cpu().numpy()
                    assert ((got == ora.to_e4m3(u + off)) | (got == ora.to_e4m3(u - off))).all(), (what, i, root)
            if cd:
                assert self.torch.equal(x["c"], x["p"].to(x["c"].dtype)), (what, i)
        for full, old, (numel, *_r) in zip(self.full, self.snap, self.spec):  # what lies behind the tensors
            for k, f in full.items():
                if f is not None:
                    n = (-(-numel // 128) if k in ("ms", "vs") else numel) * f.element_size()
                    assert self.torch.equal(f.view(self.torch.uint8)[n:], old[k][n:]), (what, k)
        return total

    def run(self, t, grad_scale, max_norm, norm=True):
        before = ([x["p"].double().cpu().numpy() for x in self.t], *([np.zeros(s[0]) for s in self.spec] for _ in range(2))) if t == 1 else (
            [x["p"].double().cpu().numpy() for x in self.t], *self.moments())
        g = self.grads(grad_scale)
        self.plan.step(self.ws, self.step, LR, WD, B1, B2, EPS, max_norm, total_norm=self.norm if norm else None)
        self.torch.cuda.synchronize()
        total = self.check(before, g, t, max_norm, f"step {t}")
        assert int(self.step) == t
        if norm:
            assert float(self.norm) == pytest.approx(total, rel=2e-6)
        return total


RAGGED = [1, 2, 3, 4, 5, 127, 128, 129, 255, 4095, 4096, 4097, 12289, 640]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gd, cd", [("f32", "bf16"), ("bf16", "f16"), ("f16", None)])
def test_ragged_sizes_three_steps(bits, gd, cd):
    st = State([(n, i % 3, bits, gd, cd) for i, n in enumerate(RAGGED)], seed=bits + len(gd))
    totals = [st.run(1, 0.5, 10.0), st.run(2, 1e-3, 10.0), st.run(3, 0.2, 10.0)]
    assert totals[0] > 10.0 > totals[1]  # the first step clips, the second does not


def test_both_forms_and_all_gradient_types_in_one_list():
    spec = [(5000, 0, 8, "bf16", "bf16"), (640, 1, 32, "f32", None), (70000, 0, 32, "f16", "f16"), (129, 2, 8, "f32", "bf16")]
    st = State(spec, seed=5)
    for t in (1, 2):
        st.run(t, 0.1, 1.0)


@pytest.mark.parametrize("max_norm", [0.0, float("inf"), -1.0])
def test_without_clipping_and_without_a_norm(max_norm):
    st = State([(5000, 0, 32, "f32", None), (300, 1, 8, "bf16", "f16")], seed=6)
    st.run(1, 3.0, max_norm, norm=False)
    st.run(2, 3.0, max_norm, norm=True)
    st.run(3, 3.0, max_norm, norm=False)


def test_small_and_empty_blocks_of_the_8_bit_form():
    """Blocks of zeros, of tiny and of very uneven gradients: nothing divides by a zero root, small blocks stay at zero."""
    import torch

    st = State([(128 * 6, 0, 8, "f32", None)], seed=7)
    x = st.t[0]
    x["p"].fill_(1.0)
    g = torch.zeros(6, 128, device="cuda")
    g[1] = 1e-38  # m and sqrt(v) below 2^-100
    g[2, 5] = 1.0  # one element
    g[3] = 1e-6
    g[3, 0] = 1e3  # 1e9 apart: every other root takes the smallest code
    g[4] = torch.linspace(-1, 1, 128, device="cuda")
    g[5] = 65504.0
    x["g"].copy_(g.view(-1))
    grads = [x["g"].double().cpu().numpy()]
    before = ([x["p"].double().cpu().numpy()], [np.zeros(768)], [np.zeros(768)])
    st.plan.step(st.ws, st.step, LR, WD, B1, B2, EPS, 0.0)
    torch.cuda.synchronize()
    st.check(before, grads, 1, 0.0, "blocks")
    ms, vs = x["ms"].cpu(), x["vs"].cpu()
    assert ms[0] == 0 and vs[0] == 0 and ms[1] == 0 and vs[1] == 0
    q = x["v"].float().cpu().view(6, 128)
    assert (q[3, 1:] == 2.0**-9).all() and (q[2, 6:] == 0).all() and torch.isfinite(x["p"]).all()


def test_loss_scaled_steps_skip_on_overflow():
    import struct

    import torch

    spec = [(5000, 0, 32, "f32", "bf16"), (700, 1, 8, "bf16", "bf16")]
    st = State(spec, seed=8)
    state = torch.zeros(4, dtype=torch.int32, device="cuda")
    state[0] = struct.unpack("i", struct.pack("f", 1024.0))[0]
    read = lambda: (struct.unpack("f", struct.pack("i", int(state[0])))[0], int(state[1]), int(state[2]))  # noqa: E731
    expect = {0: (1024.0, 1, 0), 1: (512.0, 0, 1), 2: (512.0, 1, 0), 3: (1024.0, 0, 0), 4: (512.0, 0, 1)}
    t = 0
    for k in range(5):
        before = [x["p"].double().cpu().numpy() for x in st.t], *(st.moments() if t else ([np.zeros(s[0]) for s in spec], [np.zeros(s[0]) for s in spec]))
        scale = read()[0]
        st.grads(0.3 * scale)
        if k == 1:
            st.t[0]["g"][123] = float("inf")
        if k == 4:
            st.t[1]["g"][699] = float("nan")
        grads = [x["g"].double().cpu().numpy() / scale for x in st.t]
        raw = [{n: b.view(torch.uint8).clone() for n, b in x.items() if b is not None} for x in st.t]
        st.plan.step_scaled(st.ws, state, st.step, LR, WD, B1, B2, EPS, 1.0, growth_interval=2, floor_scale=300.0, total_norm=st.norm)
        torch.cuda.synchronize()
        assert read() == expect[k], k
        if k in (1, 4):
            for x, old in zip(st.t, raw):
                for n, b in x.items():
                    assert b is None or torch.equal(b.view(torch.uint8), old[n]), (k, n)
            assert not np.isfinite(float(st.norm))
        else:
            t += 1
            total = st.check(before, grads, t, 1.0, f"scaled {k}")
            assert float(st.norm) == pytest.approx(total, rel=2e-6)
        assert int(st.step) == t


def test_captured_step_goes_on_counting_and_bits_repeat():
    import torch

    spec = [(20000, 0, 8, "bf16", "bf16"), (20000, 0, 32, "f32", None), (64, 2, 32, "f32", None)]
    a, b = State(spec, seed=9), State(spec, seed=9)
    ga, gb = a.grads(0.1), b.grads(0.1)
    assert all(np.array_equal(x, y) for x, y in zip(ga, gb))
    for _ in range(4):
        a.plan.step(a.ws, a.step, LR, WD, B1, B2, EPS, 1.0, total_norm=a.norm)
    b.plan.step(b.ws, b.step, LR, WD, B1, B2, EPS, 1.0, total_norm=b.norm)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.plan.step(b.ws, b.step, LR, WD, B1, B2, EPS, 1.0, total_norm=b.norm)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert int(a.step) == int(b.step) == 4
    for x, y in zip(a.t, b.t):
        for k in x:
            assert x[k] is None or torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)), k


def test_many_chunks_per_block_and_offsets_past_32_bits():
    """1.1e9 elements in one tensor (4.4 GB of parameters): the last elements against the oracle, the first as well."""
    import torch

    from paper_2609_10632_b200 import binding as nb

    n = 1_100_000_003
    g = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    p = torch.ones(n, device="cuda")
    m, v = (torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    ms, vs = (torch.empty(-(-n // 128), device="cuda") for _ in range(2))
    g[-5:] = torch.tensor([1.0, -2.0, 0.25, 4.0, -8.0], dtype=torch.bfloat16, device="cuda")
    plan = nb.AdamWPlan([(g, p, m, v, None, 0, ms, vs)])
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    plan.upload(ws)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    plan.step(ws, step, LR, WD, B1, B2, EPS, 0.0)
    torch.cuda.synchronize()
    for sl in (slice(0, 64), slice(n - 64, n)):
        want, wm, _ = ora.adamw_update(np.ones(64), g[sl].double().cpu().numpy(), np.zeros(64), np.zeros(64), 1, LR[0], B1, B2, EPS, WD[0])
        parity.check("param", p[sl].double().cpu().numpy(), want, "f32")
    tail = n - n // 128 * 128
    got = m[-tail:].view(torch.float8_e4m3fn).double().cpu().numpy() * float(ms[-1])
    want = 0.1 * g[-tail:].double().cpu().numpy()
    assert (np.abs(got - want) <= np.abs(want) * 2.0**-4 * (1 + NEAR)).all()


def test_another_stream_than_the_current_one():
    import torch

    st = State([(300000, 0, 8, "bf16", "bf16")], seed=10)
    g = st.grads(0.1)
    before = ([st.t[0]["p"].double().cpu().numpy()], [np.zeros(300000)], [np.zeros(300000)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    st.plan.step(st.ws, st.step, LR, WD, B1, B2, EPS, 1.0, total_norm=st.norm, stream=side)
    side.synchronize()
    st.check(before, g, 1, 1.0, "side stream")


def test_refusals():
    import torch

    from paper_2609_10632_b200 import binding as nb

    st = State([(1000, 0, 32, "f32", None)], seed=11)
    args = (LR, WD, B1, B2, EPS, 1.0)
    for call, status in [
        (lambda: st.plan.step(st.ws[:256], st.step, *args), nb.NB_ERR_WORKSPACE),
        (lambda: st.plan.step(None, st.step, *args), nb.NB_ERR_WORKSPACE),
        (lambda: st.plan.step(st.ws, None, *args), nb.NB_ERR_INVALID_ARG),
        (lambda: st.plan.step(st.ws, st.step.data_ptr() + 4, *args), nb.NB_ERR_ALIGNMENT),
        (lambda: st.plan.step(st.ws, st.step, LR, WD, 1.0, B2, EPS, 1.0), nb.NB_ERR_INVALID_ARG),
        (lambda: st.plan.step(st.ws, st.step, LR, WD, B1, -0.1, EPS, 1.0), nb.NB_ERR_INVALID_ARG),
        (lambda: st.plan.step(st.ws, st.step, LR, WD, B1, B2, -1e-8, 1.0), nb.NB_ERR_INVALID_ARG),
        (lambda: st.plan.step_scaled(st.ws, None, st.step, *args), nb.NB_ERR_INVALID_ARG),
    ]:
        with pytest.raises(nb.NbError) as e:
            call()
        assert e.value.status == status
    t = torch.zeros(512, device="cuda")
    for items in [(t, t[:256], t[256:], t[256:], None, 0), (t[:256], t[1:257], t[256:], t[:256], None, 0), (t.double(), t, t, t, None, 0)]:
        with pytest.raises(nb.NbError):
            nb.AdamWPlan([items])
    assert int(st.step) == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_second_moments_beyond_the_range_of_normal_numbers(bits):
    """Without clipping a finite gradient of 1e21 has an infinite v: m / inf is nothing, the parameter only decays.  A v below 2^-126 has
    its root all the same, which is what the update divides by where eps is 0 or tiny: against the moments that the step left
    (32 bits), in fp64, to 1e-5 of the update as elsewhere in this file; v = 0 under an m that is not zero divides by eps alone."""
    import torch

    g = [1e21, -1e30, 3e38, 1e-18, -3e-19, 1e-19, 2e-20, -1e-20, 0.0, 1e-3, 2e-22, -5e-22] + [0.0] * 116 + [1e-19] * 128
    for eps in (0.0, 1e-40, 1e-30, 1e-8):
        st = State([(len(g), 0, bits, "f32", None)], seed=12)
        x = st.t[0]
        x["g"].copy_(torch.tensor(g))
        p0 = x["p"].double().cpu().numpy()
        st.plan.step(st.ws, st.step, LR, WD, B1, B2, eps, 0.0)
        torch.cuda.synchronize()
        p, keep = x["p"].double().cpu().numpy(), 1 - LR[0] * WD[0]
        assert (np.abs(p[:3] - keep * p0[:3]) <= 2.0**-23 * np.abs(p0[:3])).all(), (eps, p[:3], p0[:3])
        hg = np.array(g, dtype=np.float32)
        with np.errstate(over="ignore"):
            m, v = np.float32(0.1) * hg, (np.float32(0.001) * hg) * hg  # (m and v of a first step, each product rounded once)
        if bits == 32:
            m, v = x["m"].cpu().numpy(), x["v"].cpu().numpy()
        m, v = m.astype(np.float64), v.astype(np.float64)
        some = (v > 0) & np.isfinite(v) if eps == 0 else np.isfinite(v)
        some &= ~((v == 0) & (m != 0) & (LR[0] * np.abs(m) * 10 > 1e30 * eps))
        with np.errstate(all="ignore"):
            update = LR[0] * (m / (1 - B1)) / (np.sqrt(v / (1 - B2)) + np.float64(np.float32(eps)))
        assert some.sum() > 130 and np.isfinite(update[some]).all()
        p, p0, update, nan = p[some], p0[some], update[some], np.isnan(p[8]) and not np.isfinite(p[10:12]).any()
        assert (np.abs(p - (keep * p0 - update)) <= 1e-5 * np.abs(update) + 2.0**-22 * (np.abs(p0) + np.abs(update))).all(), eps
        if eps == 0:  # 0 / 0 and m / 0 are what the formula says
            assert nan


@pytest.mark.parametrize("bits", [32, 8])
def test_a_nan_gradient_makes_the_clipped_step_nan(bits):
    """The norm is NaN, so min(max_norm / (norm + 1e-6), 1) is: no tensor takes an unclipped step.  An infinite gradient clips all others to nothing."""
    import torch

    for bad in (float("nan"), float("inf")):
        st = State([(300, 0, bits, "f32", None), (5000, 1, bits, "bf16", None)], seed=13)
        st.grads(5.0)
        st.t[0]["g"][7] = bad
        before = st.t[1]["p"].clone()
        st.plan.step(st.ws, st.step, LR, WD, B1, B2, EPS, 1.0, total_norm=st.norm)
        torch.cuda.synchronize()
        assert st.t[0]["p"][7].isnan() and not np.isfinite(float(st.norm))
        if bad != bad:
            assert st.t[0]["p"].isnan().all() and st.t[1]["p"].isnan().all()
        else:
            assert torch.equal(st.t[1]["p"], before)  # (group 1 has no decay)


def test_a_plan_keeps_its_tensors():
    """A plan holds addresses; moments that nothing else refers to stay allocated as long as it lives."""
    import gc
    import weakref

    import torch

    from paper_2609_10632_b200 import binding as nb

    p, g = torch.zeros(1000, device="cuda"), torch.ones(1000, device="cuda")

    def make():
        m, v = torch.zeros(1000, device="cuda"), torch.zeros(1000, device="cuda")
        return nb.AdamWPlan([(g, p, m, v, None, 0)]), weakref.ref(m), weakref.ref(v)

    plan, m, v = make()
    gc.collect()
    assert m() is not None and v() is not None
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    plan.upload(ws)
    plan.step(ws, torch.zeros(1, dtype=torch.int64, device="cuda"), LR, WD, B1, B2, EPS, 0.0)
    torch.cuda.synchronize()
    assert torch.allclose(m(), torch.full_like(m(), 0.1))
    plan.close()
    gc.collect()
    assert m() is None and v() is None


@pytest.mark.parametrize("bits", [32, 8])
def test_the_detectors_own_parameter_list(bits):
    """The 243 tensors / 25.9 M parameters that the SGD step trains: filters with 16-bit copies (and 8-bit moments), two steps against the oracle."""
    from paper_2609_10632_b200 import workloads as wl

    tensors = wl.detector_parameter_tensors()
    assert len(tensors) == 243
    st = State([(n, group, bits if group == 0 else 32, "f32", "bf16" if group == 0 else None) for _, n, group in tensors], seed=14)
    assert st.run(1, 0.01, 10.0) > 10.0  # clipped
    assert st.run(2, 1e-4, 10.0) < 10.0  # not clipped
