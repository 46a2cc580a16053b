"""Norm weights far from one over rows far from one, with the bounds of test_gpu_norm_rope: the
normed channels and the outputs are in fp32's range, so every step to them has to be."""

import pytest
import torch

from tests.test_gpu_norm_rope import ROPES, _case, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,weights", [(-40, 100), (-40, 120), (50, -100), (50, -115), (-44, 84), (54, -75), (0, 122),
                                          (-60, 100), (60, -100)])
def test_weights_far_from_one(gpu_kvx, rows, weights, dtype, d):
    q, k, qw, kw, pos = _case(9, 5, 2, d, dtype, d)
    q[:, 0, 3:7] = 0.0
    q, k, qw, kw = q * 2.0 ** rows, k * 2.0 ** rows, qw * 2.0 ** weights, kw * 2.0 ** weights
    assert torch.isfinite(qw).all() and (qw > 0).all()
    for rope in ROPES[:2]:
        qo, ko = gpu_kvx.norm_rope(q, k, qw, kw, rope, pos, eps=0.0)
        _check(qo, q, qw, 0.0, pos, rope, dtype)
        _check(ko, k, kw, 0.0, pos, rope, dtype)
