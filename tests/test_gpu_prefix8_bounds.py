"""Attention over shared prefixes with its bounds stated (longest, longest_prefix): the kernels'
choice and the grids go by them, the result does not.  Bounds of errors as in test_gpu_prefix8."""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from tests.test_gpu_prefix8 import WIDE, _case, _check

pytestmark = pytest.mark.gpu
CASES = [   # prefixes, requests of each, own tokens, new tokens, H, G, d, P
    ([700, 40], [3, 1], [300, 3, 90, 1], [1, 2, 1, 1], 2, 4, 128, 16),
    ([1], [1], [1], [1], 1, 1, 64, 128),
    ([2500], [40], [1 + 37 * i % 900 for i in range(40)], [1] * 40, 8, 8, 128, 16),
    ([900, 0, 77], [2, 1, 3], [150, 64, 129, 80, 64, 200], [64, 64, 120, 64, 64, 64], 2, 8, 128, 32),
    ([300, 310], [33, 31], [1 + 13 * i % 70 for i in range(64)], [1, 3] * 32, 4, 4, 64, 64),
]


def _names(kvx, c, longest, longest_prefix):
    T, heads, d = c["q"].shape
    H, (n, Mp), (B, M) = c["codes"].shape[1], c["ptables"].shape, c["tables"].shape
    return kvx.prefix_kernel_names(kvx.AttendDims(B, H, heads // H, T, d, longest), kvx.PrefixDims(n, Mp, longest_prefix),
                                   kvx.Pool(c["scales"].shape[2], c["codes"].shape[2] // c["scales"].shape[2], M),
                                   "bf16" if c["q"].dtype == torch.bfloat16 else "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_stated_bounds(gpu_kvx, monkeypatch, case, dtype):
    """Tables as wide as the lengths or much wider; the bounds as they are, for one part only, past
    the tables, and too small (they decide nothing but the choice)."""
    pre, count, lens, news, H, G, d, P = CASES[case]
    seen, definition = set(), S.attend_prefix8
    for Mp, M in ((None, None), (WIDE, WIDE)):
        c = _case(np.random.default_rng(case), pre, count, lens, news, H, G, d, P, dtype, Mp=Mp, M=M)
        once = []
        monkeypatch.setattr(S, "attend_prefix8", lambda *a: once[0] if once else once.append(definition(*a)) or once[0])  # noqa: B023
        own, common = max(lens), max(pre)
        for longest, longest_prefix in ((0, 0), (own, common), (own, 0), (0, common), (2 ** 31 - 1, 2 ** 31 - 1), (1, 1),
                                        (own, 1), (1, common)):
            seen.add(_names(gpu_kvx, c, longest, longest_prefix))
            _check(gpu_kvx, c, f"{dtype} case {case} longest={longest} longest_prefix={longest_prefix}", longest=longest,
                   longest_prefix=longest_prefix)
    if case in (0, 2):
        assert len(seen) > 1      # they decide


def test_one_workspace_for_calls_of_fewer_rows(gpu_kvx):
    """Kept from the longest step of a program, over kernels of every kind."""
    rng = np.random.default_rng(3)
    cases = [_case(rng, [500], [B], [n + 20 * (b % 3) for b in range(B)], [n] * B, 2, 8, 128, 16, "bf16")
             for B, n in ((4, 300), (4, 100), (4, 10), (4, 1))]
    space = None
    for c in cases:
        T, heads, d = c["q"].shape
        need = gpu_kvx.prefix_workspace_bytes(gpu_kvx.AttendDims(4, 2, 8, T, d, 0), gpu_kvx.PrefixDims(1, c["ptables"].shape[1], 0))
        if space is None:
            space = torch.empty(need, dtype=torch.uint8, device="cuda:0")
            space[:gpu_kvx.ATTEND_COUNTER_BYTES].zero_()
        _check(gpu_kvx, c, f"{T} rows in one workspace", workspace=space)
