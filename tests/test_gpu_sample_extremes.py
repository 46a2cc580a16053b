"""Token sampling where logits or temperatures come to the ends of fp32's range, against the
definition in 64 bits, with the bounds of test_gpu_sample."""

import numpy as np
import pytest
import torch

from tests.test_gpu_sample import DEV, _check

pytestmark = pytest.mark.gpu
CUTS = ((0, 0.9, 0.0), (0, 0.3, 0.0), (0, 1.0, 0.0), (0, 1.0, 0.05), (600, 1.0, 0.0), (600, 0.6, 0.02), (100, 0.9, 0.0),
        (3000, 0.97, 0.0))


def _rows(x, temperatures):
    return [(t, k, p, m) for t in temperatures for k, p, m in CUTS], x(len(temperatures) * len(CUTS))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [2, 700, 5001, 140001])
def test_differences_past_the_range(gpu_kvx, V, dtype):
    """Logits of both signs whose differences pass fp32's largest number, at temperatures at which
    the lowest of them still have a weight."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = np.random.default_rng(V)
    # spread evenly: no two weights next to a border by chance
    settings, x = _rows(lambda n: g.uniform(-3.3e38, 3.3e38, (n, V)), (1e31, 2e37, 1e38, 3e38))
    _check(gpu_kvx, torch.tensor(x).to(dt).to(DEV), settings, g.random(len(settings)))
    # two numbers, masked logits between: at an infinite temperature all weights are one
    settings, x = _rows(lambda n: np.where(g.random((n, V)) < 0.4, 2e38, -2e38), (float("inf"),))
    x[1::2, 1::3] = -np.inf
    _check(gpu_kvx, torch.tensor(x).to(dt).to(DEV), settings, g.random(len(settings)), exact=lambda b: True)


@pytest.mark.parametrize("V", [2, 700, 5001, 140001])
def test_temperatures_near_zero(gpu_kvx, V):
    """Logits that differ by as little as the temperature, down to the subnormal numbers."""
    g = np.random.default_rng(V + 1)
    for t in (1e-31, 1e-38, 1e-40):
        settings, x = _rows(lambda n: g.standard_normal((n, V)) * 2 * t, (t,))
        x[::3] -= np.abs(x).max()
        x[1::4, ::5] = -1e30
        x[2::4, 1::7] = -np.inf
        _check(gpu_kvx, torch.tensor(x).to(torch.float32).to(DEV), settings, g.random(len(settings)))
    # next to these, logits of ordinary size: one of them has all the weight, however many follow
    settings, x = _rows(lambda n: g.standard_normal((n, V)), (1e-31, 1e-38, 1e-40, 1e-45))
    x[::2] -= 50.0
    _check(gpu_kvx, torch.tensor(x).to(torch.float32).to(DEV), settings, g.random(len(settings)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sums_of_the_largest_vocabulary(gpu_kvx, dtype):
    """2^20 tokens, the weights' sums next to 2^63.  All equal: borders are met exactly."""
    V, dt = 1 << 20, torch.bfloat16 if dtype == "bf16" else torch.float32
    settings = [(t, k, p, 0.0) for t in (1.0, float("inf")) for k, p in ((0, 0.5), (0, 1.0), (V // 2, 0.75), (V // 2, 1.0))
                for _ in range(3)]
    u = [0.0, 0.5, 1.0 - 2.0 ** -24] * 8
    _check(gpu_kvx, torch.full((len(u), V), -1.5, dtype=dt, device=DEV), settings, u, exact=lambda b: True)
    g = np.random.default_rng(20)
    settings = [(1.0, 0, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.0, 100, 1.0, 0.0), (1.0, 300000, 0.5, 0.0), (2.0, 0, 0.8, 0.1)]
    _check(gpu_kvx, torch.tensor(g.standard_normal((5, V)) * 0.5).to(dt).to(DEV), settings, g.random(5))
