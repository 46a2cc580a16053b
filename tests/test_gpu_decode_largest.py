"""The decoding step's operators at the most requests, prefixes, rows and heads that they take."""

import numpy as np
import pytest
import torch

from tests.test_gpu_norm_rope import ROPES, _case as _rows, _check as _check_rows
from tests.test_gpu_prefix8 import _case, _check
from tests.test_gpu_sample import DEV, SETTINGS, _check as _check_draws, _logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_4096_prefixes_and_requests(gpu_kvx, d, dtype):
    rng = np.random.default_rng(d)
    n = 4096
    lens = [int(x) for x in rng.integers(0, 9, n)]
    c = _case(rng, [int(x) for x in rng.integers(0, 30, n)], [1] * n, lens, [int(x) for x in rng.integers(0, 2, n)], 1, 2, d, 16,
              dtype)
    _check(gpu_kvx, c, f"{dtype} d={d} 4096 prefixes")
    # in large workgroups, whose LDS holds the sums of 4096 prefixes beside their tiles
    c = _case(rng, [int(x) for x in rng.integers(0, 30, n)], [1] * n, lens, [1] * n, 1, 1, d, 16, dtype, Mp=80)
    _check(gpu_kvx, c, f"{dtype} d={d} 4096 prefixes, wide tables")
    c = _case(rng, [1100, 20], [2100, 1996], lens, [1] * n, 1, 1, d, 16, dtype)
    _check(gpu_kvx, c, f"{dtype} d={d} 4096 requests")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_65535_rows_of_logits(gpu_kvx, dtype):
    B = 65535
    g = np.random.default_rng(1)
    _check_draws(gpu_kvx, _logits(B, 21, dtype, 2), [SETTINGS[b % len(SETTINGS)] for b in range(B)], g.random(B))
    with pytest.raises(gpu_kvx.KvxError, match="65535"):
        gpu_kvx.sample_tokens(torch.zeros((B + 1, 1), device=DEV), torch.zeros(B + 1, device=DEV))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_65535_heads(gpu_kvx, dtype):
    q, k, qw, kw, pos = _rows(3, 65000, 535, 64, dtype, 4)
    qo, ko = gpu_kvx.norm_rope(q, k, qw, kw, ROPES[0], pos)
    _check_rows(qo, q, qw, 1e-6, pos, ROPES[0], dtype)
    _check_rows(ko, k, kw, 1e-6, pos, ROPES[0], dtype)
