"""Attention over the 8-bit pool on the GPU against its definition in 64 bits.

Bounds, element by element, with A = sum_j p_j |V_j| and S = max_j sum_c |q_c K_jc| * scale
of a row, n keys, u = 2^-24: scores are off by at most (d + 8) u S (products and sums in
fp32, the factor, the running maximum's subtraction), so a probability by a share of
2 (d + 8) u S + 16 u (its exponential and the rescaling), and sums of n terms by n u:
    E = (2 (d + 8) S + 2 n + 64) u.
fp32: |out - exact| <= E A.  bf16: the probabilities' and the output's rounding, 2^-8
each, on top: <= (E + 2^-8 * 1.01) A + 2^-8 |out|.  lse: <= E + 4 u |lse|.  A probability
under 2^-126, fp32's least normal number, may be lost whole (exp(-500) is no fp32 number):
n 2^-126 max |V| on top of out's.
"""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from tests._parity import log

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(rng, lens, news, H, G, d, P, dtype, M=None, spare=3, q_scale=1.0):
    """Ragged requests over random pages; codes past each request's end and on pages of
    nobody are NaN, and so are the scales of those pages."""
    B = len(lens)
    pages = [-(-n // P) for n in lens]
    N = sum(pages) + spare
    M = max(pages + [1]) + 1 if M is None else M
    perm, at = rng.permutation(N), 0
    tables = rng.integers(-3, N + 3, (B, M))
    codes = rng.integers(0, 256, (2, H, N, P, d), dtype=np.uint8)
    codes[(codes & 0x7F) >= 0x70] &= 0x9F       # largest values of about 16: realistic spread
    scales = 2.0 ** rng.integers(-7, -3, (2, H, N))
    used = np.zeros(N, bool)
    for b in range(B):
        mine = perm[at:at + pages[b]]
        at += pages[b]
        tables[b, :pages[b]] = mine
        used[mine] = True
        if lens[b] % P:
            codes[:, :, mine[-1], lens[b] % P:] = rng.choice([0x7F, 0xFF])
    codes[:, :, ~used] = 0x7F
    scales[:, :, ~used] = np.nan
    cu = np.concatenate([[0], np.cumsum(news)])
    q = torch.from_numpy(rng.standard_normal((cu[-1], H * G, d)) * q_scale).to(DT[dtype])
    return dict(q=q, codes=codes.reshape(2, H, N * P, d), scales=scales, tables=tables,
                lens=np.array(lens), cu=cu)


def _gpu(c):
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)  # noqa: E731
    return (c["q"].to(DEV), torch.from_numpy(c["codes"]).to(DEV).view(torch.float8_e4m3fn),
            torch.from_numpy(c["scales"].astype(np.float32)).to(DEV), i32(c["tables"]),
            i32(c["lens"]), i32(c["cu"]))


def _compare(c, out, lse, scale, label):
    q = c["q"]
    want, wl, A, smax = S.attend_cache8(q.double().cpu().numpy(), c["codes"], c["scales"], c["tables"],
                                        c["lens"], c["cu"], scale)
    d = q.shape[2]
    n = max(int(np.max(c["lens"], initial=1)), 1)
    u = 2.0 ** -24
    E = (2 * (d + 8) * smax + 2 * n + 64) * u
    bound = E[..., None] * A + n * 2.0 ** -126 * np.nanmax(np.abs(S.E4M3[c["codes"][1]])) * np.nanmax(c["scales"][1])
    if q.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (1.01 * A + np.abs(want))
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    rows = ~np.isnan(wl)
    live = rows & np.isfinite(wl)
    with np.errstate(invalid="ignore", divide="ignore"):
        worst = np.nanmax(np.where(bound > 0, np.abs(got - want) / bound, 0.0)[rows], initial=0.0)
    log(f"[parity] {label}: {rows.sum()} rows, error at {worst:.3f} of its bound")
    assert np.all(np.abs(got - want)[rows] <= bound[rows]), label
    assert np.all(np.abs(gl - wl)[live] <= (E + 4 * u * np.abs(wl))[live]), label
    empty = rows & ~live
    assert np.all(gl[empty] == -np.inf) and np.all(got[empty] == 0), label
    return rows


def _check(kvx, c, label, scale=None, **kw):
    d = c["q"].shape[2]
    out, lse = kvx.attend_cache8(*_gpu(c), scale=scale, with_lse=True, **kw)
    torch.cuda.synchronize()
    _compare(c, out, lse, d ** -0.5 if scale is None else scale, label)
    return out, lse


STEPS = [   # lens (with the new tokens), new tokens
    ([1], [1]),
    ([16], [1]),
    ([17, 1, 33], [1, 1, 1]),
    ([5, 0, 64, 63, 65, 300], [1, 1, 1, 1, 1, 1]),       # one that has nothing
    ([1000, 3, 129, 128, 127, 31], [1, 0, 1, 1, 0, 1]),  # two that ask nothing
    ([2, 40, 7, 90], [5, 3, 7, 4]),                      # more rows than tokens: empty rows
    ([70, 200, 33], [33, 64, 33]),                       # chunks
    ([513], [257]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_attention_matches_the_definition(gpu_kvx, dtype, d, P):
    rng = np.random.default_rng(100 + P + d)
    for (lens, news), (H, G) in zip(STEPS, [(1, 1), (2, 8), (2, 3), (3, 4), (1, 16), (2, 5), (1, 8), (2, 2)]):
        c = _case(rng, lens, news, H, G, d, P, dtype)
        _check(gpu_kvx, c, f"{dtype} d={d} P={P} lens={lens} news={news} H={H} G={G}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G", [(1, 1), (8, 1), (1, 7), (3, 6), (2, 16), (1, 17), (1, 40), (5, 2)])
def test_attention_head_counts(gpu_kvx, dtype, H, G):
    rng = np.random.default_rng(H * 100 + G)
    _check(gpu_kvx, _case(rng, [40, 7, 130], [2, 1, 3], H, G, 128, 16, dtype), f"{dtype} H={H} G={G}")
    _check(gpu_kvx, _case(rng, [40, 257], [40, 70], H, G, 64, 32, dtype), f"{dtype} chunks H={H} G={G}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,new,d,P", [(4097, 1, 128, 16), (20011, 1, 64, 128), (9000, 3, 128, 64), (3000, 130, 128, 32)])
def test_attention_long_caches(gpu_kvx, dtype, n, new, d, P):
    rng = np.random.default_rng(n)
    _check(gpu_kvx, _case(rng, [n, 5], [new, 1], 1, 4, d, P, dtype), f"{dtype} {n} keys")


def test_attention_many_requests(gpu_kvx):
    rng = np.random.default_rng(20)
    lens = list(rng.integers(0, 90, 700))
    news = list(rng.integers(0, 3, 700))
    _check(gpu_kvx, _case(rng, lens, news, 1, 4, 64, 16, "bf16"), "700 requests")
    _check(gpu_kvx, _case(rng, [3] * 4096, [1] * 4096, 1, 1, 64, 16, "bf16"), "4096 requests")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_extreme_scales_and_scores(gpu_kvx, dtype):
    """Value scales far from one, scores of some hundreds, a factor of zero and a negative one."""
    rng = np.random.default_rng(21)
    c = _case(rng, [300, 40], [2, 40], 2, 4, 64, 16, dtype)
    c["scales"][1] = 2.0 ** rng.integers(-100, 90, c["scales"][1].shape).astype(float)
    _check(gpu_kvx, c, "value scales")
    c = _case(rng, [300, 40], [2, 40], 2, 4, 64, 16, dtype, q_scale=60.0)
    _check(gpu_kvx, c, "large scores")
    for f in (0.0, -0.2):
        _check(gpu_kvx, _case(rng, [300, 40], [2, 40], 2, 4, 64, 16, dtype), f"factor {f}", scale=f)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_skips_pages_that_are_none(gpu_kvx, dtype):
    """Table entries outside the pool hide their keys, whole requests of them too."""
    rng = np.random.default_rng(22)
    for d, P in ((128, 16), (64, 64)):
        c = _case(rng, [300, 40, 130, 64], [3, 30, 2, 1], 2, 4, d, P, dtype)
        N = c["scales"].shape[2]
        c["tables"][0, 1], c["tables"][0, -2] = -1, N
        c["tables"][1, 0] = -2 ** 31
        c["tables"][3, :] = 2 ** 31 - 1
        _check(gpu_kvx, c, f"missing pages d={d} P={P}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_lengths_out_of_range(gpu_kvx, dtype):
    """Lengths past the table, negative lengths, rows past T: clamped; rows of nobody keep
    what they held."""
    rng = np.random.default_rng(23)
    c = _case(rng, [64, 40, 96], [3, 2, 4], 2, 2, 64, 16, dtype, M=6)
    c["lens"] = np.array([64, -7, 2 ** 31 - 1])
    c["cu"] = np.array([0, 3, 5, 2 ** 31 - 1])
    _check(gpu_kvx, c, "clamped")
    c["lens"], c["cu"] = np.array([64, 40, 96]), np.array([0, 3, 3, 6])
    a = _gpu(c)
    out = torch.full_like(a[0], 7.0)
    got, lse = gpu_kvx.attend_cache8(*a, out=out, with_lse=True)
    torch.cuda.synchronize()
    rows = _compare(c, got, lse, 0.125, "rows of nobody")
    assert rows[:6].all() and not rows[6:].any() and torch.all(out[6:] == 7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_nan_stays_in_its_row(gpu_kvx, dtype):
    rng = np.random.default_rng(24)
    c = _case(rng, [90, 70], [3, 40], 2, 4, 128, 16, dtype)
    clean, _ = gpu_kvx.attend_cache8(*_gpu(c), with_lse=True)
    c["q"][1, 5, 17] = float("nan")
    c["q"][20, 2] = float("nan")
    out, lse = gpu_kvx.attend_cache8(*_gpu(c), with_lse=True)
    torch.cuda.synchronize()
    bad = torch.zeros(out.shape[:2], dtype=torch.bool, device=DEV)
    bad[1, 5] = bad[20, 2] = True
    assert out[bad].isnan().all() and lse[bad].isnan().all()
    assert torch.equal(out[~bad], clean[~bad])


def test_attention_takes_queries_as_they_lie(gpu_kvx):
    """Queries inside a fused projection [T, H*G + 2*H, d], and with padded rows."""
    rng = np.random.default_rng(25)
    for dtype in ("bf16", "f32"):
        for lens, news in (([100, 60], [1, 1]), ([100, 60], [40, 33])):
            c = _case(rng, lens, news, 2, 3, 64, 16, dtype)
            a = list(_gpu(c))
            T = a[0].shape[0]
            fused = torch.full((T, 10, 72), float("nan"), dtype=a[0].dtype, device=DEV)
            fused[:, 2:8, :64] = a[0]
            a[0] = fused[:, 2:8, :64]
            out, lse = gpu_kvx.attend_cache8(*a, with_lse=True)
            torch.cuda.synchronize()
            _compare(c, out, lse, 0.125, f"fused {dtype}")


@pytest.mark.parametrize("news", [1, 70])
def test_attention_beyond_32_bits(gpu_kvx, news):
    """Pages more than 2^32 bytes into a plane."""
    rng = np.random.default_rng(26)
    N, P, d = 262144 + 8, 128, 128
    c = _case(rng, [500, 130], [news, 1], 1, 4, d, P, "bf16", spare=2)
    n = c["scales"].shape[2]
    pool = torch.empty((2, 1, N * P, d), dtype=torch.uint8, device=DEV)
    scales = torch.full((2, 1, N), float("nan"), device=DEV)
    a = list(_gpu(c))
    pool[:, :, (N - n) * P:] = a[1].view(torch.uint8)
    scales[:, :, N - n:] = a[2]
    mine = torch.arange(a[3].shape[1], device=DEV) < -(-a[4][:, None] // P)
    a[1], a[2], a[3] = pool.view(torch.float8_e4m3fn), scales, torch.where(mine, a[3] + (N - n), -1)
    out, lse = gpu_kvx.attend_cache8(*a, with_lse=True)
    torch.cuda.synchronize()
    _compare(c, out, lse, d ** -0.5, "far pages")


def test_attention_is_the_same_every_time(gpu_kvx):
    """Split rows are joined in a fixed order: repeated calls give the same bits, in a
    workspace that calls of other shapes have used."""
    rng = np.random.default_rng(27)
    c = _case(rng, [9000, 700, 33], [1, 1, 2], 2, 4, 128, 16, "bf16")
    o = _case(rng, [300, 40], [70, 40], 2, 4, 128, 32, "bf16")
    a, b = _gpu(c), _gpu(o)
    need = max(gpu_kvx.attend_workspace(x[0], x[1], x[3]).numel() for x in (a, b))
    ws = torch.zeros(need, dtype=torch.uint8, device=DEV)
    first = gpu_kvx.attend_cache8(*a, with_lse=True, workspace=ws)
    other = gpu_kvx.attend_cache8(*b, with_lse=True, workspace=ws)
    for _ in range(5):
        out = gpu_kvx.attend_cache8(*a, with_lse=True, workspace=ws)
        assert torch.equal(out[0], first[0]) and torch.equal(out[1], first[1])
        out = gpu_kvx.attend_cache8(*b, with_lse=True, workspace=ws)
        assert torch.equal(out[0], other[0]) and torch.equal(out[1], other[1])
    _compare(c, *first, 128 ** -0.5, "repeated")


def test_attention_on_another_stream_and_in_a_graph(gpu_kvx):
    rng = np.random.default_rng(28)
    c = _case(rng, [3000, 700, 33], [1, 1, 1], 2, 4, 128, 16, "bf16")
    a = _gpu(c)
    side = torch.cuda.Stream(device=DEV)
    big = torch.randn((4096, 4096), device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):
            big = big @ big
            big = big / big.norm()
    out, lse = gpu_kvx.attend_cache8(*a, with_lse=True, stream=side)
    junk = [torch.full((1 << 22,), float("nan"), device=DEV) for _ in range(8)]
    torch.cuda.synchronize()
    del junk
    _compare(c, out, lse, 128 ** -0.5, "side stream")
    ws = gpu_kvx.attend_workspace(a[0], a[1], a[3])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = gpu_kvx.attend_cache8(*a, with_lse=True, workspace=ws)
    for n in range(3):
        a[0].copy_(torch.randn(a[0].shape, device=DEV))
        lens = [int(rng.integers(1, m + 1)) for m in (3000, 700, 33)]
        a[4].copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        # keys past the shorter lengths are finite here, so the definition may skip them
        _compare({**c, "q": a[0].cpu(), "lens": np.array(lens)}, out, lse, 128 ** -0.5, f"replay {n}")
        eager = gpu_kvx.attend_cache8(*a, with_lse=True)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
