"""The 8-bit store on the GPU against its definition: codes and scales are equal, since
the only rounding is e4m3's."""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from tests._parity import log

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _slots(rng, turns, P, N):
    """Slots of packed turns (tokens held, new tokens) over random pages of a pool."""
    perm, at, out = rng.permutation(N), 0, []
    for held, new in turns:
        n = -(-(held + new) // P)
        pages = perm[at:at + n]
        at += n
        p = np.arange(held, held + new)
        out.append(pages[p // P] * P + p % P)
    assert at <= N
    return np.concatenate(out) if out else np.zeros(0, int)


def _pool(rng, L, H, N, P, d):
    """A pool of valid rows with power-of-two scales, as earlier stores leave it."""
    codes = rng.integers(0, 256, (L, 2, H, N * P, d), dtype=np.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x30
    return codes, 2.0 ** rng.integers(-12, -6, (L, 2, H, N))


def _same(codes, want):
    """Equal codes; NaN is NaN whatever its sign."""
    nan = (want & 0x7F) == 0x7F
    return np.array_equal((codes & 0x7F) == 0x7F, nan) and np.array_equal(codes[~nan], want[~nan])


def _run(kvx, k, v, slots, codes, scales, **kw):
    """Runs the store and its definition on copies; returns both pools."""
    pool = torch.from_numpy(codes.copy()).to(DEV).view(torch.float8_e4m3fn)
    sc = torch.from_numpy(scales.astype(np.float32)).to(DEV)
    kvx.store_cache8(k, v, torch.from_numpy(slots.astype(np.int32)).to(DEV), pool, sc, **kw)
    torch.cuda.synchronize()
    codes, scales = codes.copy(), scales.astype(np.float64)
    S.store_cache8(k.double().cpu().numpy(), v.double().cpu().numpy(), slots, codes, scales)
    return pool.view(torch.uint8).cpu().numpy(), sc.double().cpu().numpy(), codes, scales


def _check(kvx, k, v, slots, codes, scales, **kw):
    gc, gs, wc, ws = _run(kvx, k, v, slots, codes, scales, **kw)
    assert np.array_equal(gs, ws, equal_nan=True), "scales"
    assert _same(gc, wc), "codes"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_store_matches_the_definition(gpu_kvx, dtype, d, P):
    rng = np.random.default_rng(P + d)
    g = torch.Generator().manual_seed(P)
    for L, H, turns in ((1, 1, [(0, 1)]), (2, 3, [(P - 1, 1), (0, P), (P, 1), (5, 2 * P + 3), (2 * P - 1, 2)]),
                        (3, 2, [(0, 17), (3, 200), (31, 1), (1, 4 * P)])):
        log(f"[case] store {dtype} d={d} P={P} L={L} H={H} {turns}")
        N = sum(-(-(a + b) // P) for a, b in turns) + 3
        slots = _slots(rng, turns, P, N)
        T = len(slots)
        # rows of very different sizes, so that some pages' scales grow and some hold
        size = torch.exp2(torch.randint(-14, 6, (L, H, T, 1), generator=g).float())
        k, v = ((torch.randn((L, H, T, d), generator=g) * size).to(DT[dtype]).to(DEV) for _ in range(2))
        _check(gpu_kvx, k, v, slots, *_pool(rng, L, H, N, P, d))


def test_store_long_turns(gpu_kvx):
    rng = np.random.default_rng(9)
    turns = [(100, 1000), (0, 777), (4095, 2)]
    for P in (16, 128):
        N = 400
        slots = _slots(rng, turns, P, N)
        k, v = (torch.randn((2, 2, len(slots), 128), device=DEV).to(torch.bfloat16) for _ in range(2))
        _check(gpu_kvx, k, v, slots, *_pool(rng, 2, 2, N, P, 128))


def test_store_takes_rows_as_they_lie(gpu_kvx):
    """A projection's [T, H, d], a slice of a fused one, a mapped cache's halves, one row
    broadcast over heads."""
    rng = np.random.default_rng(10)
    N, P, H, d = 30, 16, 4, 64
    slots = _slots(rng, [(3, 50), (0, 31)], P, N)
    T = len(slots)
    for dtype in (torch.bfloat16, torch.float32):
        codes, scales = _pool(rng, 1, H, N, P, d)
        k, v = (torch.randn((T, H, d), device=DEV).to(dtype).transpose(0, 1)[None] for _ in range(2))
        _check(gpu_kvx, k, v, slots, codes, scales)
        fused = torch.randn((T, 9 * H, d), device=DEV).to(dtype)
        k, v = (fused[:, a:a + H].transpose(0, 1)[None] for a in (2 * H, 7 * H))
        _check(gpu_kvx, k, v, slots, codes, scales)
        one = torch.randn((1, 1, T, d), device=DEV).to(dtype).expand(1, H, T, d)
        _check(gpu_kvx, one, k, slots, codes, scales)
        kv = torch.randn((3, 2, H, T, d), device=DEV).to(dtype)
        _check(gpu_kvx, kv[:, 0], kv[:, 1], slots, *_pool(rng, 3, H, N, P, d))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_special_values(gpu_kvx, dtype):
    """Zeros, least and largest numbers, infinities and NaN."""
    rng = np.random.default_rng(11)
    N, P, d = 12, 16, 64
    slots = _slots(rng, [(0, 16)] * 8, P, N)
    x = torch.randn((1, 1, 128, d))
    x[0, 0, 0:16] = 0
    x[0, 0, 16:32] = torch.randn((16, d)) * 1e-39        # below the least normal number
    x[0, 0, 32:48] *= 1e38
    x[0, 0, 33, 5] = torch.finfo(DT[dtype]).max
    x[0, 0, 48:64, 3] = torch.inf
    x[0, 0, 50, 4] = -torch.inf
    x[0, 0, 64:80] = torch.nan
    x[0, 0, 80:96, 7] = torch.nan
    x[0, 0, 96:112] = -0.0
    x[0, 0, 112:128] *= 2.0 ** -110
    k = x.to(DT[dtype]).to(DEV)
    _check(gpu_kvx, k, -k, slots, *_pool(rng, 1, 1, N, P, d))


def test_store_skips_rows_without_a_slot(gpu_kvx):
    """Rows of refused requests and padding; the rest of the pool keeps its bytes."""
    rng = np.random.default_rng(12)
    N, P, H, d = 9, 16, 2, 128
    slots = _slots(rng, [(4, 30), (0, 40)], P, N)
    slots[[0, 7, 8, 45, 69]] = [-1, N * P, -2 ** 31, 2 ** 31 - 1, -1]
    k, v = (torch.randn((2, H, len(slots), d), device=DEV).to(torch.bfloat16) for _ in range(2))
    codes, scales = _pool(rng, 2, H, N, P, d)
    codes[:] = 0x7F                                       # a pool that held garbage
    scales[:] = np.nan
    slots[slots // P == slots[1] // P] = -1               # keep whole pages only: no row is held
    _check(gpu_kvx, k, v, slots, codes, scales)
    _check(gpu_kvx, k, v, np.full(len(slots), -1), codes, scales)


def test_store_again_changes_nothing(gpu_kvx):
    rng = np.random.default_rng(13)
    N, P = 20, 32
    slots = _slots(rng, [(9, 100), (30, 7)], P, N)
    k, v = (4 * torch.randn((1, 2, len(slots), 64), device=DEV) for _ in range(2))
    codes, scales = _pool(rng, 1, 2, N, P, 64)
    gc, gs, _, _ = _run(gpu_kvx, k, v, slots, codes, scales)
    gc2, gs2, _, _ = _run(gpu_kvx, k, v, slots, gc, gs)
    assert np.array_equal(gc, gc2) and np.array_equal(gs, gs2)


def test_store_scales_that_are_no_powers_of_two(gpu_kvx):
    """Scales of the caller's own: kept where they suffice, and rows divided by them to
    within e4m3's rounding of a quotient that is off by two units in the last place."""
    rng = np.random.default_rng(14)
    N, P, d = 4, 16, 64
    slots = np.arange(5, 12)
    codes, _ = _pool(rng, 1, 1, N, P, d)
    scales = np.full((1, 2, 1, N), np.float32(0.0137))
    k, v = (torch.randn((1, 1, 7, d), device=DEV) for _ in range(2))
    gc, gs, wc, ws = _run(gpu_kvx, k, v, slots, codes, scales)
    assert np.array_equal(gs, ws)
    far = np.abs(gc.astype(int) - wc.astype(int))
    assert far.max() <= 1 and (far > 0).mean() < 1e-3


def test_store_slots_beyond_32_bits(gpu_kvx):
    """A plane of more than 2^32 bytes, written at its end."""
    N, P, d = 262144 + 8, 128, 128
    pool = torch.empty((1, 2, 1, N * P, d), dtype=torch.uint8, device=DEV)
    scales = torch.ones((1, 2, 1, N), dtype=torch.float32, device=DEV)
    assert N * P * d > 2 ** 32
    slots = torch.arange((N - 2) * P + 100, N * P, dtype=torch.int32, device=DEV)
    pool[:, :, :, (N - 2) * P:] = 0x30
    k, v = (torch.randn((1, 1, len(slots), d), device=DEV).to(torch.bfloat16) for _ in range(2))
    codes = pool[:, :, :, (N - 2) * P:].cpu().numpy()
    gpu_kvx.store_cache8(k, v, slots, pool.view(torch.float8_e4m3fn), scales)
    torch.cuda.synchronize()
    ws = np.ones((1, 2, 1, 2))
    S.store_cache8(k.double().cpu().numpy(), v.double().cpu().numpy(), slots.cpu().numpy() - (N - 2) * P, codes, ws)
    assert np.array_equal(pool[:, :, :, (N - 2) * P:].cpu().numpy(), codes)
    assert np.array_equal(scales[:, :, :, N - 2:].cpu().numpy(), ws)


def test_store_on_another_stream_and_in_a_graph(gpu_kvx):
    rng = np.random.default_rng(15)
    N, P, H, d = 40, 16, 2, 128
    slots = _slots(rng, [(9, 100), (0, 7)], P, N)
    k, v = (torch.randn((2, H, len(slots), d), device=DEV).to(torch.bfloat16) for _ in range(2))
    codes, scales = _pool(rng, 2, H, N, P, d)
    side = torch.cuda.Stream(device=DEV)
    torch.cuda.synchronize()
    _check(gpu_kvx, k, v, slots, codes, scales, stream=side)
    pool = torch.from_numpy(codes).to(DEV)
    first = pool.clone()
    sc = torch.from_numpy(scales.astype(np.float32)).to(DEV)
    sc0 = sc.clone()
    st = torch.from_numpy(slots.astype(np.int32)).to(DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gpu_kvx.store_cache8(k, v, st, pool.view(torch.float8_e4m3fn), sc)
    for n in range(3):
        pool.copy_(first)
        sc.copy_(sc0)
        k.copy_(torch.randn(k.shape, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        wc, ws = codes.copy(), scales.astype(np.float64)
        S.store_cache8(k.double().cpu().numpy(), v.double().cpu().numpy(), slots, wc, ws)
        assert np.array_equal(pool.cpu().numpy(), wc) and np.array_equal(sc.double().cpu().numpy(), ws), n


@pytest.mark.parametrize("d,P,T", [(64, 16, 2500), (64, 16, 4096 + 37), (128, 128, 700)])
def test_a_large_call_equals_its_layers_one_by_one(gpu_kvx, d, P, T):
    """Waves that take several small pages, or a long one whole, against calls of one layer."""
    rng = np.random.default_rng(T)
    L, H, turns = 64, 8, [(9, T // 2), (0, 5), (P, T - T // 2 - 5 - 61), (3, 61)]
    N = sum(-(-(a + b) // P) for a, b in turns) + 2
    slots = torch.from_numpy(_slots(rng, turns, P, N).astype(np.int32)).to(DEV)
    slots[T // 2:T // 2 + 5] = -1               # a refused request's
    k, v = (torch.randn((L, H, T, d), device=DEV).to(torch.bfloat16) for _ in range(2))
    k[:, :, T // 2:] *= 40
    pool = torch.randint(0, 0x60, (L, 2, H, N * P, d), dtype=torch.uint8, device=DEV)
    scales = torch.full((L, 2, H, N), 2.0 ** -8, device=DEV)
    one, one_scales = pool.clone(), scales.clone()
    gpu_kvx.store_cache8(k, v, slots, pool.view(torch.float8_e4m3fn), scales)
    for l in range(L):
        gpu_kvx.store_cache8(k[l:l + 1], v[l:l + 1], slots, one[l:l + 1].view(torch.float8_e4m3fn), one_scales[l:l + 1])
    assert torch.equal(pool, one) and torch.equal(scales, one_scales)
    codes, ws = _pool(rng, 1, H, N, P, d)       # and one layer against the definition
    _check(gpu_kvx, k[:1, :, :300], v[:1, :, :300], slots[:300].cpu().numpy().astype(int), codes, ws)
