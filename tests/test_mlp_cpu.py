"""MlpBlock without a GPU: which device its calls are made on."""
import contextlib
from collections import defaultdict

import torch

from paper_2609_10632_b200 import mlp


def test_calls_are_made_with_the_blocks_device_current(monkeypatch):
    """The norm's calls have no plan and run on the current device: with another one current, forward() and backward() switch."""
    current, seen = [0], []

    @contextlib.contextmanager
    def device(d):
        before = current[0]
        current[0] = torch.device(d).index
        try:
            yield
        finally:
            current[0] = before

    monkeypatch.setattr(torch.cuda, "device", device)
    for name in ("nb_layer_norm_fwd", "nb_layer_norm_bwd", "nb_linear_fwd", "nb_linear_bwd_data", "nb_linear_bwd_weight"):
        monkeypatch.setattr(mlp.nb, name, lambda *a, _n=name, **k: seen.append((_n, current[0])))
    b = mlp.MlpBlock.__new__(mlp.MlpBlock)
    for name in ("rows", "c", "dtype", "act", "eps", "x", "h", "y", "dy", "dh", "dx", "z", "a", "dz", "mean", "rstd", "up", "down", "ws"):
        setattr(b, name, None)
    b.param, b.grad, b.copy, b.dev = defaultdict(int), defaultdict(int), defaultdict(int), torch.device("cuda", 1)
    b.forward()
    b.backward()
    assert len(seen) == 8 and {d for _, d in seen} == {1}
    assert current[0] == 0
