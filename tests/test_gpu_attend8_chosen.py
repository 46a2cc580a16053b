"""Every attention kernel over the 8-bit pool, by the name that the library gives, on what it
can go wrong at: NaN codes, missing pages, lengths past the table, scales of every kind, units
over several workgroups and several units a workgroup.

Bounds, element by element, with A, S, u as in test_gpu_attend8 and n the most keys that a
request has (at most what its table holds: the others add exact zeros):
    E = (2 (d + 8) S + 2 n + 64) u,   pre = (E + t) A + n 2^-126 (448 + max |V|)
with t = 1.01 2^-16 for bf16 queries (two bf16 terms a probability) and 0 for fp32 (three), and
the output's rounding: pre + 2^-8 (|out| + pre) for bf16.  lse: E + 4 u |lse|.
"""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from tests._parity import log
from tests.test_gpu_attend8 import _case, _gpu

pytestmark = pytest.mark.gpu
P = 16

# Requests, KV heads, query heads each, new tokens of the requests in turn, pages of a table.
FEW, SOME = [1, 2, 1, 4, 1, 1, 3, 1], [5, 9, 6, 4, 7, 5, 8, 6]
SIZES = {"split": (3, 2, 4, [1, 2, 1], 6), "large": (8, 8, 4, FEW, 64), "32 rows": (40, 8, 4, SOME, 26),
         "32 rows, large": (8, 16, 4, SOME, 64), "by rows": (96, 2, 8, [12, 20, 5, 33, 1, 12, 12, 2], 6)}
KERNELS = {   # its sizes, type, head dimension
    "attend8_split_kernel<0, 64, 4, 1>": ("split", "bf16", 64),
    "attend8_split_kernel<0, 128, 4, 1>": ("split", "bf16", 128),
    "attend8_split_kernel<1, 64, 4, 1>": ("split", "f32", 64),
    "attend8_split_kernel<1, 128, 4, 1>": ("split", "f32", 128),
    "attend8_split_kernel<0, 64, 12, 1>": ("large", "bf16", 64),
    "attend8_split_kernel<0, 128, 12, 1>": ("large", "bf16", 128),
    "attend8_split_kernel<1, 64, 12, 1>": ("large", "f32", 64),
    "attend8_split_kernel<1, 128, 8, 1>": ("large", "f32", 128),
    "attend8_split_kernel<0, 64, 4, 2>": ("32 rows", "bf16", 64),
    "attend8_split_kernel<0, 128, 4, 2>": ("32 rows", "bf16", 128),
    "attend8_split_kernel<0, 64, 12, 2>": ("32 rows, large", "bf16", 64),
    "attend8_split_kernel<0, 128, 8, 2>": ("32 rows, large", "bf16", 128),
    "attend8_rows_kernel<64, 2>": ("by rows", "bf16", 64),
    "attend8_rows_kernel<128, 2>": ("by rows", "bf16", 128),
}


def _name(kvx, c):
    T, heads, d = c["q"].shape
    H, (B, M) = c["codes"].shape[1], c["tables"].shape
    return kvx.attend_kernel_name(kvx.AttendDims(B, H, heads // H, T, d, 0),
                                  kvx.Pool(c["scales"].shape[2], c["codes"].shape[2] // c["scales"].shape[2], M),
                                  "bf16" if c["q"].dtype == torch.bfloat16 else "f32")


def _sized(rng, kernel, lens=None, **kw):
    size, dtype, d = KERNELS[kernel]
    B, H, G, news, M = SIZES[size]
    if lens is None:
        lens = rng.integers(0, M * P + 1, B)
        lens[-1] = M * P
    return _case(rng, [int(n) for n in lens], [news[b % len(news)] for b in range(B)], H, G, d, P, dtype, M=M, **kw)


def _slot(c, b, pos):
    return c["tables"][b, pos // P] * P + pos % P


def _check(kvx, kernel, c, label):
    """The call takes the kernel; outputs, their NaN and the rows without keys are the
    definition's; the same again the second time."""
    assert _name(kvx, c) == kernel
    out, lse = kvx.attend_cache8(*_gpu(c), with_lse=True)
    again = kvx.attend_cache8(*_gpu(c), with_lse=True)
    torch.cuda.synchronize()
    as_bits = lambda t: t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)  # noqa: E731
    assert torch.equal(as_bits(out), as_bits(again[0])) and torch.equal(as_bits(lse), as_bits(again[1]))
    d, u = c["q"].shape[2], 2.0 ** -24
    with np.errstate(invalid="ignore", over="ignore"):
        want, wl, A, smax = S.attend_cache8(c["q"].double().numpy(), c["codes"], c["scales"], c["tables"],
                                            c["lens"], c["cu"], d ** -0.5)
        got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
        n = min(max(int(np.max(c["lens"])), 1), c["tables"].shape[1] * P)
        E = (2 * (d + 8) * smax + 2 * n + 64) * u
        V = np.nanmax(np.abs(S.E4M3[c["codes"][1]])) * np.nanmax(c["scales"][1])
        bf16 = c["q"].dtype == torch.bfloat16
        pre = (E[..., None] + (1.01 * 2.0 ** -16 if bf16 else 0)) * A + n * 2.0 ** -126 * (448 + V)
        bound = pre + 2.0 ** -8 * (np.abs(want) + pre) if bf16 else pre
        empty, fine = wl == -np.inf, np.isfinite(want)
        log(f"[parity] {kernel} {label}: {want.shape[0] * want.shape[1]} rows, {empty.sum()} empty, "
            f"{np.isnan(want).sum()} outputs NaN, error at {np.max((np.abs(got - want) / bound)[fine & (bound > 0)]):.3f} of its bound")
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isnan(gl), np.isnan(wl))
        assert np.all(np.abs(got - want)[fine] <= bound[fine])
        some = np.isfinite(wl)
        assert np.all((np.abs(gl - wl) <= E + 4 * u * np.abs(wl))[some])
    assert np.all(gl[empty] == -np.inf) and np.all(got[empty] == 0)
    return want, empty


@pytest.mark.parametrize("kernel", KERNELS)
def test_ragged_requests(gpu_kvx, kernel):
    rng = np.random.default_rng(900)
    _, empty = _check(gpu_kvx, kernel, _sized(rng, kernel), "ragged")
    c = _sized(rng, kernel)
    c["lens"][::3] = 0                       # and requests without keys
    want, empty = _check(gpu_kvx, kernel, c, "without keys")
    assert empty.any() and not empty.all()


@pytest.mark.parametrize("kernel", KERNELS)
def test_lengths_past_the_table(gpu_kvx, kernel):
    """Cut to what the table holds, all of it live pages; negative ones are none."""
    rng = np.random.default_rng(901)
    size, _, _ = KERNELS[kernel]
    B, M = SIZES[size][0], SIZES[size][4]
    c = _sized(rng, kernel, lens=[M * P] * B)
    c["lens"] = np.array([[M * P + 1, 2 ** 31 - 1, -7, M * P, -2 ** 31, 2 ** 31 - P, 5][b % 7] for b in range(B)])
    c["cu"][-1] = 2 ** 31 - 1                # rows past the last one
    _check(gpu_kvx, kernel, c, "past the table")


@pytest.mark.parametrize("kernel", KERNELS)
def test_missing_pages(gpu_kvx, kernel):
    rng = np.random.default_rng(902)
    size, _, _ = KERNELS[kernel]
    B, M = SIZES[size][0], SIZES[size][4]
    c = _sized(rng, kernel, lens=[M * P - 5] * B)
    N = c["scales"].shape[2]
    for b in range(B):
        hole = rng.random(M) < 0.4
        c["tables"][b, hole] = rng.choice([-1, N, -2 ** 31, 2 ** 31 - 1], hole.sum())
    c["tables"][B // 2] = -1
    _check(gpu_kvx, kernel, c, "missing pages")


@pytest.mark.parametrize("kernel", KERNELS)
def test_nan_codes(gpu_kvx, kernel):
    rng = np.random.default_rng(903)
    size, _, d = KERNELS[kernel]
    B, H, _, news, M = SIZES[size]
    lens = [M * P - 5 - b % 20 for b in range(B)]
    c = _sized(rng, kernel, lens=lens)
    for b in range(0, B, 2):                 # among the newest tokens, and one that all rows see
        c["codes"][1, b % H, _slot(c, b, lens[b] - 1), [0, d - 1]] = 0xFF
        c["codes"][1, (b + 1) % H, _slot(c, b, lens[b] - 2), 5] = 0x7F
        c["codes"][1, 0, _slot(c, b, 3), 7] = 0x7F
        c["codes"][0, H - 1, _slot(c, b, lens[b] - 1), 9] = 0x7F
    want, _ = _check(gpu_kvx, kernel, c, "NaN codes")
    assert 0 < np.isnan(want).sum() < want.size


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("what", ["far", "own", "zero", "large scores"])
def test_scales(gpu_kvx, kernel, what):
    rng = np.random.default_rng(904)
    c = _sized(rng, kernel, q_scale=60.0 if what == "large scores" else 1.0)
    shape = c["scales"][1].shape
    if what == "far":
        c["scales"][1] = 2.0 ** rng.integers(-100, 90, shape).astype(float)
    elif what == "own":
        c["scales"] = (c["scales"] * rng.uniform(1, 2, c["scales"].shape)).astype(np.float32).astype(np.float64)
    elif what == "zero":                     # and negative ones
        c["scales"][1] = np.where(rng.random(shape) < 0.3, 0.0, -c["scales"][1])
        c["scales"][0] = np.where(rng.random(shape) < 0.3, 0.0, -c["scales"][0])
    _check(gpu_kvx, kernel, c, f"scales {what}")


@pytest.mark.parametrize("kernel,lens,news,H,G,pages", [
    # one long request over many workgroups (joins in two levels), beside a short one
    ("attend8_split_kernel<0, 128, 12, 1>", [20011, 300], [1, 2], 1, 8, 2100),
    ("attend8_split_kernel<0, 64, 12, 1>", [40011, 7], [1, 3], 1, 8, 2600),
    ("attend8_split_kernel<0, 128, 12, 1>", [16000], [2], 1, 8, 4200),      # 16 rows of 63 parts
    ("attend8_split_kernel<1, 128, 8, 1>", [20011], [2], 1, 4, 4200),
    ("attend8_split_kernel<1, 64, 12, 1>", [20011], [1], 1, 7, 4200),
    ("attend8_split_kernel<0, 128, 8, 2>", [20011, 30], [6, 4], 2, 4, 2100),
    ("attend8_split_kernel<0, 64, 12, 2>", [40011], [3], 1, 8, 8200),
    ("attend8_rows_kernel<128, 2>", [9001, 40], [120, 90], 1, 2, 4200 * 8),
    ("attend8_rows_kernel<64, 2>", [20011], [50], 1, 2, 4200 * 40),
    # several units a workgroup
    ("attend8_split_kernel<0, 128, 12, 1>", [200, 17, 256, 90] * 25, [1, 1, 2, 1] * 25, 4, 8, 16),
    ("attend8_split_kernel<0, 64, 12, 1>", [200, 17, 256, 90] * 25, [1, 1, 2, 1] * 25, 4, 8, 16),
    ("attend8_split_kernel<1, 64, 12, 1>", [200, 17, 256, 90] * 25, [1, 1, 2, 4] * 25, 4, 8, 16),
    ("attend8_split_kernel<1, 128, 8, 1>", [200, 17, 256, 90] * 25, [1, 1, 2, 4] * 25, 4, 8, 16),
    ("attend8_split_kernel<0, 128, 12, 1>", [1200, 17, 256, 90] * 25, [1, 1, 2, 1] * 25, 6, 4, 76),
    ("attend8_split_kernel<0, 128, 8, 2>", [200, 17, 256, 1030] * 25, [7, 6, 3, 11] * 25, 4, 4, 65),
    ("attend8_split_kernel<0, 64, 4, 2>", [200, 17, 256, 90] * 100, [7, 6, 3, 11] * 100, 2, 3, 17),
    ("attend8_rows_kernel<128, 2>", [200, 17, 256, 90] * 18, [40, 17, 60, 33] * 18, 4, 3, 16),
    ("attend8_rows_kernel<64, 2>", [200, 17, 256, 90] * 18, [40, 17, 60, 33] * 18, 4, 3, 16),
])
def test_shares(gpu_kvx, kernel, lens, news, H, G, pages):
    _, dtype, d = KERNELS[kernel]
    rng = np.random.default_rng(905)
    c = _case(rng, lens, news, H, G, d, P, dtype)
    had = c["tables"].shape[1]
    if pages > had:                          # entries that no request reaches
        c["tables"] = np.concatenate([c["tables"], np.full((len(lens), pages - had), 2 ** 30)], 1)
    _check(gpu_kvx, kernel, c, f"shares of {len(lens)} requests")
