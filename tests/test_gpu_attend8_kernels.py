"""The attention kernels that large batches take, on small ones: the choice goes by the
length that the block tables could hold, so wide tables (their other entries are never
looked at) bring the kernel by rows and the large workgroups to cases that the definition
computes quickly.  Bounds as in test_gpu_attend8."""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from tests._parity import log
from tests.test_gpu_attend8 import DEV, _case, _check, _compare, _gpu

pytestmark = pytest.mark.gpu


def _by_rows(c):
    """Widens the tables until the call's pairs reach the kernel by rows (bf16, 64 rows a
    request and more)."""
    T, heads, d = c["q"].shape
    B, M = c["tables"].shape
    P = c["codes"].shape[2] // c["scales"].shape[2]
    assert c["q"].dtype == torch.bfloat16     # requests of 96 rows and more; others go in blocks of 32
    return _wide(c, -(-2 ** 34 // (T * heads * d * P)))


def _large(c):
    """Widens the tables until a request's 4 to 32 rows take one large workgroup a CU (other
    numbers of rows take the small ones)."""
    B, M = c["tables"].shape
    T, heads, _ = c["q"].shape
    assert c["q"].dtype != torch.bfloat16 or T * heads // c["codes"].shape[1] < 64 * B
    P = c["codes"].shape[2] // c["scales"].shape[2]
    return _wide(c, -(-2 ** 20 // (B * c["codes"].shape[1] * P)))


def _two_tiles(c):
    """Widens the tables until requests of 17 to 95 rows take blocks of 32, in large
    workgroups where those are few."""
    B, M = c["tables"].shape
    T, heads, _ = c["q"].shape
    H = c["codes"].shape[1]
    assert c["q"].dtype == torch.bfloat16 and 16 * B < T * heads // H < 96 * B
    P = c["codes"].shape[2] // c["scales"].shape[2]
    return _wide(c, -(-2 ** 17 // (B * H * P)))


def _wide(c, M):
    B, had = c["tables"].shape
    if M > had:
        c["tables"] = np.concatenate([c["tables"], np.full((B, M - had), 2 ** 30)], 1)
    return c


CHUNKS = [   # tokens in the pool, new ones, KV heads, query heads each
    ([64], [64], 1, 1),
    ([70, 200, 33], [33, 64, 33], 2, 8),
    ([513], [257], 2, 2),
    ([5, 0, 300, 1], [70, 0, 290, 1], 1, 3),     # more rows than tokens: empty rows
    ([1000, 3, 129], [128, 128, 1], 2, 5),
    ([127, 128, 129], [127, 128, 129], 1, 7),
    ([300, 40], [20, 17], 3, 16),
    ([90, 33], [30, 33], 2, 17),
    ([200], [10], 1, 40),
    ([64], [64], 1, 2),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_by_rows(gpu_kvx, d, P):
    rng = np.random.default_rng(300 + P + d)
    for lens, news, H, G in CHUNKS:
        c = _by_rows(_case(rng, lens, news, H, G, d, P, "bf16"))
        _check(gpu_kvx, c, f"by rows d={d} P={P} lens={lens} news={news} H={H} G={G}")


@pytest.mark.parametrize("lens,news,H,G,d,P", [
    ([3000, 5], [130, 1], 1, 4, 128, 32),          # a unit over many workgroups: two-level joins
    ([20011], [64], 1, 1, 64, 128),
    ([20011], [64], 1, 2, 64, 128),
    ([9001], [65], 1, 5, 128, 16),
    ([700] * 40, [33] * 40, 1, 4, 64, 16),         # several units a workgroup
    (list(range(64, 364, 3)), [64] * 100, 1, 1, 64, 16),
    (list(range(64, 364, 3)), [64] * 100, 1, 2, 64, 16),
])
def test_by_rows_shares(gpu_kvx, lens, news, H, G, d, P):
    rng = np.random.default_rng(len(lens) + d)
    c = _by_rows(_case(rng, lens, news, H, G, d, P, "bf16"))
    first = _check(gpu_kvx, c, f"by rows, {len(lens)} requests")
    again = gpu_kvx.attend_cache8(*_gpu(c), with_lse=True)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,news,H,G,d,P", [
    ([1], [1], 1, 1, 128, 16),
    ([383, 385], [1, 1], 2, 8, 128, 16),           # the large workgroup's 384 (256) keys
    ([5, 0, 300], [1, 1, 1], 3, 4, 64, 32),
    ([20011], [1], 1, 8, 128, 64),
    ([40011, 7], [3, 1], 1, 4, 64, 128),
    ([2, 40, 7, 90], [5, 3, 7, 4], 2, 3, 128, 16),
    ([1], [1], 1, 4, 128, 16),
    ([30] * 33 + [500], [1] * 34, 2, 1, 64, 16),   # single rows, units enough
    ([300] * 60, [4] * 60, 3, 8, 128, 32),         # several units a workgroup
])
def test_large_workgroups(gpu_kvx, dtype, lens, news, H, G, d, P):
    rng = np.random.default_rng(lens[0])
    c = _large(_case(rng, lens, news, H, G, d, P, dtype))
    first = _check(gpu_kvx, c, f"large {dtype} lens={lens} H={H} G={G} d={d}")
    again = gpu_kvx.attend_cache8(*_gpu(c), with_lse=True)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,news,H,G,P", [
    ([17], [17], 1, 1, 16),
    ([60, 5, 300], [3, 5, 40], 2, 3, 32),            # rows past a block's end, blocks of one tile
    ([0, 33, 9], [7, 33, 12], 2, 2, 16),             # a request without keys, more rows than tokens
    ([20011], [3], 1, 8, 64),                        # a unit over many workgroups
    ([40011, 7], [5, 1], 1, 8, 128),
    ([255, 256, 257, 383, 384, 385], [5] * 6, 1, 8, 16),
    ([31] * 40 + [700], [20] * 41, 2, 1, 16),        # several units a workgroup
    ([300] * 130, [3] * 130, 4, 8, 32),              # many units: small workgroups
    ([90] * 700, [6] * 700, 1, 3, 16),
])
def test_blocks_of_32_rows(gpu_kvx, lens, news, H, G, P, d):
    rng = np.random.default_rng(lens[0] + len(lens))
    c = _two_tiles(_case(rng, lens, news, H, G, d, P, "bf16"))
    first = _check(gpu_kvx, c, f"blocks of 32 lens={lens[:6]} H={H} G={G} d={d}")
    again = gpu_kvx.attend_cache8(*_gpu(c), with_lse=True)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_most_requests_in_large_workgroups(gpu_kvx):
    """4096 requests' prefix sums beside the largest arrays of a workgroup."""
    rng = np.random.default_rng(36)
    lens = rng.integers(0, 40, 4096).tolist()
    for G, d in ((1, 128), (2, 64)):
        c = _case(rng, lens, [int(n > 0) for n in lens], 1, G, d, 16, "bf16")
        _check(gpu_kvx, _wide(c, 65), f"4096 requests, G={G} d={d}")


KERNELS = {"split": lambda c: c, "large": _large, "two tiles": _two_tiles, "by rows": _by_rows}


def _news(kernel, few, many):
    """New tokens: few for the large workgroups, more for blocks of 32 rows, many else."""
    return few if kernel == "large" else [4 * n for n in few] if kernel == "two tiles" else many


@pytest.mark.parametrize("kernel", KERNELS)
def test_extreme_scales_and_scores(gpu_kvx, kernel):
    rng = np.random.default_rng(31)
    for what in ("values", "scores", "factor"):
        c = _case(rng, [300, 140], _news(kernel, [2, 9], [2, 140]), 2, 4, 64, 16, "bf16",
                  q_scale=60.0 if what == "scores" else 1.0)
        if what == "values":
            c["scales"][1] = 2.0 ** rng.integers(-100, 90, c["scales"][1].shape).astype(float)
        _check(gpu_kvx, KERNELS[kernel](c), f"{kernel} {what}", scale=-0.2 if what == "factor" else None)


@pytest.mark.parametrize("kernel", KERNELS)
def test_missing_pages_and_lengths_out_of_range(gpu_kvx, kernel):
    rng = np.random.default_rng(32)
    for d, P in ((128, 16), (64, 64)):
        c = _case(rng, [300, 140, 130, 64], _news(kernel, [3, 14, 2, 1], [3, 140, 2, 64]), 2, 4, d, P, "bf16")
        c["tables"][0, 1], c["tables"][0, -(-300 // P) - 1] = -1, c["scales"].shape[2]
        c["tables"][1, 0] = -2 ** 31
        c["tables"][3, :] = 2 ** 31 - 1
        _check(gpu_kvx, KERNELS[kernel](c), f"{kernel} missing pages d={d}")
        # a table of live pages only, so that the cut length has them all
        news = _news(kernel, [3, 5, 7], [3, 150, 70])
        c = _case(rng, [5 * P, 40, 6 * P], news, 2, 2, d, P, "bf16", M=6)
        c["lens"], c["cu"] = np.array([5 * P, -7, 6 * P]), np.array([0, 3, 3 + news[1], 2 ** 31 - 1])
        _check(gpu_kvx, KERNELS[kernel](c), f"{kernel} clamped d={d}")


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_in_the_cache_reaches_the_rows_that_see_it(gpu_kvx, kernel, dtype):
    """NaN keys and values among the newest tokens: rows before them are as without."""
    if kernel in ("by rows", "two tiles") and dtype == "f32":
        pytest.skip("fp32 queries go by keys, in blocks of 16 rows")
    rng = np.random.default_rng(33)
    for d, P in ((128, 32), (64, 16)):
        for lens, news, G in ((([90, 300], [6, 7], 8), ([33, 70], [33, 3], 1),
                               ([90, 300], [3, 4], 8)) if kernel == "large" else
                              (([33, 70], [33, 3], 1), ([90, 300], [3, 4], 8)) if kernel == "two tiles" else
                              (([90, 300], [80, 70], 1), ([33, 70], [33, 3], 8))):
            c = _case(rng, lens, news, 2, G, d, P, dtype)
            slot = lambda b, p: c["tables"][b, p // P] * P + p % P  # noqa: E731, B023
            c["codes"][1, 0, slot(0, lens[0] - 2), 5] = 0x7F         # a value of the last but one token
            c["codes"][1, 1, slot(1, lens[1] - 1), [0, d - 1]] = 0xFF
            c["codes"][1, 1, slot(0, 0), 3] = 0x7F                   # seen by all rows of request 0
            c["codes"][0, 0, slot(1, lens[1] - 3), 7] = 0x7F         # a key
            c = KERNELS[kernel](c)
            out, lse = gpu_kvx.attend_cache8(*_gpu(c), with_lse=True)
            torch.cuda.synchronize()
            want, wl, _, _ = S.attend_cache8(c["q"].double().numpy(), c["codes"], c["scales"], c["tables"],
                                             c["lens"], c["cu"], d ** -0.5)
            got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
            log(f"[case] NaN {kernel} {dtype} d={d} G={G}: {np.isnan(want).sum()} of {want.size} outputs NaN")
            assert 0 < np.isnan(want).sum() < want.size
            assert np.array_equal(np.isnan(got), np.isnan(want)), "outputs"
            assert np.array_equal(np.isnan(gl), np.isnan(wl)), "lse"
            tol = 0.02 if dtype == "bf16" else 1e-4          # they are right elsewhere too
            assert np.nanmax(np.abs(got - want)) <= tol * np.nanmax(np.abs(want))


@pytest.mark.parametrize("kernel", KERNELS)
def test_scales_that_are_no_powers_of_two(gpu_kvx, kernel):
    """A caller's own scales.  The kernel by rows rounds such values to bf16 (2^-8 of each
    on top of the bound); the others multiply the probabilities."""
    rng = np.random.default_rng(34)
    c = _case(rng, [300, 140], _news(kernel, [2, 9], [2, 140]), 2, 4, 64, 16, "bf16")
    c["scales"] = (c["scales"] * rng.uniform(1, 2, c["scales"].shape)).astype(np.float32).astype(np.float64)
    c = KERNELS[kernel](c)
    if kernel != "by rows":
        _check(gpu_kvx, c, f"{kernel} own scales")
        return
    out, lse = gpu_kvx.attend_cache8(*_gpu(c), with_lse=True)
    torch.cuda.synchronize()
    want, wl, A, smax = S.attend_cache8(c["q"].double().numpy(), c["codes"], c["scales"], c["tables"], c["lens"],
                                        c["cu"], 0.125)
    E = ((2 * 72 * smax + 2 * 300 + 64) * 2.0 ** -24)[..., None]
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= (E + 2.0 ** -8 * 2.02) * A + 2.0 ** -8 * np.abs(want))
    assert np.all(np.abs(lse.double().cpu().numpy() - wl) <= E[..., 0] + 2.0 ** -22 * np.abs(wl))


@pytest.mark.parametrize("kernel", ["large", "two tiles", "by rows"])
def test_far_pages_strides_streams_and_graphs(gpu_kvx, kernel):
    rng = np.random.default_rng(35)
    c = KERNELS[kernel](_case(rng, [500, 230], _news(kernel, [1, 5], [1, 230]), 2, 4, 128, 16, "bf16"))
    a = list(_gpu(c))
    fused = torch.full((a[0].shape[0], 14, 136), float("nan"), dtype=torch.bfloat16, device=DEV)
    fused[:, 3:11, :128] = a[0]
    a[0] = fused[:, 3:11, :128]
    side = torch.cuda.Stream(device=DEV)
    torch.cuda.synchronize()
    out, lse = gpu_kvx.attend_cache8(*a, with_lse=True, stream=side)
    side.synchronize()
    _compare(c, out, lse, 128 ** -0.5, f"{kernel} fused, side stream")
    ws = gpu_kvx.attend_workspace(a[0], a[1], a[3])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = gpu_kvx.attend_cache8(*a, with_lse=True, workspace=ws)
    for n in range(3):
        a[0].copy_(torch.randn(a[0].shape, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        _compare({**c, "q": a[0].cpu()}, out, lse, 128 ** -0.5, f"{kernel} replay {n}")
        eager = gpu_kvx.attend_cache8(*a, with_lse=True)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
    # pages more than 2^32 bytes into a plane
    N, P = 262144 + 8, 128
    c = KERNELS[kernel](_case(rng, [500, 130], _news(kernel, [1, 3], [1, 130]), 1, 4, 128, P, "bf16", spare=2))
    n = c["scales"].shape[2]
    pool = torch.empty((2, 1, N * P, 128), dtype=torch.uint8, device=DEV)
    scales = torch.full((2, 1, N), float("nan"), device=DEV)
    a = list(_gpu(c))
    pool[:, :, (N - n) * P:] = a[1].view(torch.uint8)
    scales[:, :, N - n:] = a[2]
    mine = torch.arange(a[3].shape[1], device=DEV) < -(-a[4][:, None] // P)
    a[1], a[2], a[3] = pool.view(torch.float8_e4m3fn), scales, torch.where(mine, a[3] + (N - n), -1)
    out, lse = gpu_kvx.attend_cache8(*a, with_lse=True)
    torch.cuda.synchronize()
    _compare(c, out, lse, 128 ** -0.5, f"{kernel} far pages")


@pytest.mark.parametrize("lens,news,H,G", [([300, 40, 7], [1, 1, 1], 8, 4), ([300, 140], [2, 9], 2, 4),
                                           ([300, 140], [130, 140], 2, 4), ([3, 0, 2000], [3, 1, 700], 4, 8)])
def test_a_stated_bound_changes_the_kernel_only(gpu_kvx, lens, news, H, G):
    """Whatever bound is stated, one that a request passes too."""
    rng = np.random.default_rng(37)
    c = _wide(_case(rng, lens, news, H, G, 64, 16, "bf16"), 2 ** 16)
    for longest in (max(lens), 1, 2 ** 31 - 1, 0):
        out, lse = gpu_kvx.attend_cache8(*_gpu(c), with_lse=True, longest=longest)
        torch.cuda.synchronize()
        _compare(c, out, lse, 0.125, f"longest={longest} lens={lens}")
    with pytest.raises(gpu_kvx.KvxError):
        gpu_kvx.attend_cache8(*_gpu(c), longest=-1)


def test_a_workspace_serves_all_kernels(gpu_kvx):
    rng = np.random.default_rng(36)
    cases = [KERNELS[k](_case(rng, [900, 230], _news(k, [1, 2], [1, 130]), 2, 4, 128, 16, "bf16")) for k in KERNELS]
    cases.append(_case(rng, [900, 230], [1, 3], 2, 4, 64, 16, "f32"))
    args = [_gpu(c) for c in cases]
    ws = torch.zeros(max(gpu_kvx.attend_workspace(a[0], a[1], a[3]).numel() for a in args), dtype=torch.uint8, device=DEV)
    for _ in range(3):
        for c, a in zip(cases, args):
            out, lse = gpu_kvx.attend_cache8(*a, with_lse=True, workspace=ws)
            torch.cuda.synchronize()
            _compare(c, out, lse, c["q"].shape[2] ** -0.5, "shared workspace")
