"""Scales that are NaN or infinite, on pages that only a request's later rows see: those rows
are NaN, the others what they are without (the cache's own NaN codes: test_gpu_attend8_kernels).
Finite outputs: the bounds of test_gpu_attend8, with the 2^-8 of a bf16 output and 2^-16 for
its probabilities' terms."""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from tests._parity import log
from tests.test_gpu_attend8 import _case, _gpu
from tests.test_gpu_attend8_kernels import _wide

pytestmark = pytest.mark.gpu

SHAPES = {   # tokens in the pool, new ones, entries of a table's row; 4 query heads a KV head
    "split": ([290, 34, 3], [4, 3, 1], None),
    "large": ([290, 34, 3], [4, 3, 1], 2 ** 14),
    "two tiles": ([290, 34], [8, 10], 2 ** 14),
    "by rows": ([290, 146], [130, 140], 2 ** 17),
}


@pytest.mark.parametrize("what", ["value NaN", "value inf", "value -inf", "key NaN"])
@pytest.mark.parametrize("kernel", SHAPES)
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_scales_that_are_not_finite(gpu_kvx, kernel, what, dtype, d):
    lens, news, M = SHAPES[kernel]
    rng = np.random.default_rng(600 + d)
    c = _case(rng, lens, news, 2, 4, d, 16, dtype)
    kv, bad = what.split()
    for b, pos in ((0, lens[0] - 1), (1, lens[1] - news[1] // 2)):
        c["scales"][int(kv == "value"), b, c["tables"][b, pos // 16]] = float(bad)
    c = c if M is None else _wide(c, M)
    out, lse = gpu_kvx.attend_cache8(*_gpu(c), with_lse=True)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        want, wl, A, smax = S.attend_cache8(c["q"].double().numpy(), c["codes"], c["scales"], c["tables"],
                                            c["lens"], c["cu"], d ** -0.5)
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    fine = np.isfinite(want)
    log(f"[case] {kernel} {dtype} d={d} {what}: {(~fine).sum()} of {fine.size} outputs not finite")
    assert 0 < (~fine).sum() < fine.size
    assert np.array_equal(np.isnan(got), ~fine), "outputs"
    assert np.array_equal(np.isnan(gl), np.isnan(wl)), "lse"
    with np.errstate(invalid="ignore"):
        E = ((2 * (d + 8) * smax + 2 * max(lens) + 64) * 2.0 ** -24)[..., None]
        bound = E * A if dtype == "f32" else (E + 2.0 ** -15) * A + 2.0 ** -8 * 1.01 * np.abs(want)
        bound = bound + max(lens) * 2.0 ** -126 * 448
    assert np.all(np.abs(got - want)[fine] <= bound[fine])
