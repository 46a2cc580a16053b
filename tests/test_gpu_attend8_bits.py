"""How many bits the attention over the 8-bit pool keeps with bf16 queries, against its
definition in 64 bits.

Bound, element by element, with A, S, n, u and E as in test_gpu_attend8: the probabilities
enter their product as two bf16 terms, 16 bits, so that what is rounded to the output's type
is off by at most
    pre = (E + 1.01 2^-16) A + n 2^-126 (448 + max |V|)
(the last: terms and probabilities under fp32's and bf16's least normal number, 2^-126, may be
lost), and the output by pre + 2^-8 (|out| + pre): bf16 has 8 bits.
"""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from tests._parity import log
from tests.test_gpu_attend8 import _case, _gpu
from tests.test_gpu_attend8_kernels import _wide

pytestmark = pytest.mark.gpu

SHAPES = {   # tokens in the pool, new ones, query heads a KV head, entries of a table's row
    "split": ([300, 40, 17, 5], [1, 2, 1, 1], 4, None),
    "large": ([300, 40, 17, 5], [1, 2, 1, 1], 4, 2 ** 14),
    "two tiles": ([300, 140, 30], [7, 12, 5], 4, 2 ** 14),
    "by rows": ([300, 140, 129], [130, 140, 129], 4, 2 ** 17),
}


def _rounded_once(c, out, scale, label):
    q = c["q"]
    want, _, A, smax = S.attend_cache8(q.double().numpy(), c["codes"], c["scales"], c["tables"], c["lens"],
                                       c["cu"], scale)
    d, n, u = q.shape[2], max(c["lens"]), 2.0 ** -24
    E = ((2 * (d + 8) * smax + 2 * n + 64) * u)[..., None]
    V = np.nanmax(np.abs(S.E4M3[c["codes"][1]])) * np.nanmax(c["scales"][1])
    pre = (E + 1.01 * 2.0 ** -16) * A + n * 2.0 ** -126 * (448 + V)
    bound = pre + 2.0 ** -8 * (np.abs(want) + pre)
    off = np.abs(out.double().cpu().numpy() - want)
    log(f"[parity] {label}: error at {np.max(off / bound):.3f} of its bound")
    assert np.all(off <= bound), label


@pytest.mark.parametrize("kernel", SHAPES)
@pytest.mark.parametrize("d", [64, 128])
def test_outputs_are_rounded_once(gpu_kvx, kernel, d):
    lens, news, G, M = SHAPES[kernel]
    rng = np.random.default_rng(400 + d)
    c = _case(rng, lens, news, 2, G, d, 16, "bf16")
    c = c if M is None else _wide(c, M)
    out = gpu_kvx.attend_cache8(*_gpu(c))
    torch.cuda.synchronize()
    _rounded_once(c, out, d ** -0.5, f"rounded once, {kernel} d={d}")


@pytest.mark.parametrize("kernel", SHAPES)
@pytest.mark.parametrize("d", [64, 128])
def test_own_scales_are_not_rounded(gpu_kvx, kernel, d):
    """A caller's scales that are no powers of two, with equal probabilities, so that nothing
    else is rounded before the output is."""
    lens, news, G, M = SHAPES[kernel]
    rng = np.random.default_rng(500 + d)
    c = _case(rng, lens, news, 2, G, d, 16, "bf16", q_scale=0.0)
    own = rng.integers(0, 2, c["scales"].shape)      # beside powers of two
    c["scales"] = (c["scales"] * (1 + own * rng.uniform(0, 1, own.shape))).astype(np.float32).astype(np.float64)
    c = c if M is None else _wide(c, M)
    out = gpu_kvx.attend_cache8(*_gpu(c))
    torch.cuda.synchronize()
    _rounded_once(c, out, d ** -0.5, f"own scales, {kernel} d={d}")
