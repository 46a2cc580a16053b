"""Attention over shared prefixes on the GPU against its definition in 64 bits, every kernel of
either part by the name that its rule gives.

Bounds, element by element, as in test_gpu_attend8_chosen, with n the most keys that a row has,
its prefix's included, and for the join of the two parts: two powers of two of differences of
scores, off by 2 u S and 2 u, two products, a sum and a quotient more:
    E = (2 (d + 9) S + 2 n + 80) u,   pre = (E + t) A + n 2^-126 (448 + max |V|)
with t = 1.01 2^-16 for bf16 queries and 0 for fp32, and the output's rounding:
pre + 2^-8 (|out| + pre) for bf16.  lse: E + 4 u |lse|.
"""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from tests._parity import log
from tests.test_gpu_attend8 import DT, _gpu
from tests.test_gpu_attend8_chosen import KERNELS, SIZES

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _case(rng, pre, count, lens, news, H, G, d, P, dtype, first=0, Mp=None, M=None, spare=3):
    """Prefixes of `pre` tokens, each shared by `count` requests in turn from request `first` on;
    requests of `lens` own tokens, `news` of them new.  Codes past each end and on pages of
    nobody are NaN, and so are the scales of those pages."""
    pages = [-(-n // P) for n in list(pre) + list(lens)]
    N, B = sum(pages) + spare, len(lens)
    Mp = max(pages[:len(pre)] + [1]) + 1 if Mp is None else Mp
    M = max(pages[len(pre):] + [1]) + 1 if M is None else M
    codes = rng.integers(0, 256, (2, H, N, P, d), dtype=np.uint8)
    codes[(codes & 0x7F) >= 0x70] &= 0x9F
    scales = 2.0 ** rng.integers(-7, -3, (2, H, N))
    perm, at, used = rng.permutation(N), 0, np.zeros(N, bool)
    ptables, tables = rng.integers(-3, N + 3, (len(pre), Mp)), rng.integers(-3, N + 3, (B, M))
    for i, n in enumerate(list(pre) + list(lens)):
        mine = perm[at:at + pages[i]]
        at += pages[i]
        (ptables[i] if i < len(pre) else tables[i - len(pre)])[:pages[i]] = mine
        used[mine] = True
        if n % P:
            codes[:, :, mine[-1], n % P:] = rng.choice([0x7F, 0xFF])
    codes[:, :, ~used] = 0x7F
    scales[:, :, ~used] = np.nan
    cu = np.concatenate([[0], np.cumsum(news)])
    q = torch.from_numpy(rng.standard_normal((cu[-1], H * G, d))).to(DT[dtype])
    return dict(q=q, codes=codes.reshape(2, H, N * P, d), scales=scales, tables=tables, lens=np.array(lens), cu=cu,
                ptables=ptables, plens=np.array(pre), pcu=first + np.concatenate([[0], np.cumsum(count)]))


def _operands(c):
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)  # noqa: E731
    q, codes, scales, tables, lens, cu = _gpu(c)
    return q, codes, scales, i32(c["ptables"]), i32(c["plens"]), i32(c["pcu"]), tables, lens, cu


def _compare(c, out, lse, scale, label):
    q = c["q"]
    want, wl, A, smax = S.attend_prefix8(q.double().numpy(), c["codes"], c["scales"], c["ptables"], c["plens"], c["pcu"],
                                         c["tables"], c["lens"], c["cu"], scale)
    P = c["codes"].shape[2] // c["scales"].shape[2]
    n = min(int(c["lens"].max(initial=0)), c["tables"].shape[1] * P)
    n = max(n + min(int(c["plens"].max(initial=0)), c["ptables"].shape[1] * P), 1)
    u = 2.0 ** -24
    E = (2 * (q.shape[2] + 9) * smax + 2 * n + 80) * u
    big = 448 + np.nanmax(np.abs(S.E4M3[c["codes"][1]])) * np.nanmax(c["scales"][1])
    bf16 = q.dtype == torch.bfloat16
    bound = (E + (1.01 * 2.0 ** -16 if bf16 else 0))[..., None] * A + n * 2.0 ** -126 * big
    if bf16:
        bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    rows = ~np.isnan(wl)
    live = rows & np.isfinite(wl)
    log(f"[parity] {label}: {rows.sum()} rows, error at "
        f"{np.nanmax((np.abs(got - want) / bound)[rows], initial=0.0):.3f} of its bound")
    assert np.all(np.abs(got - want)[rows] <= bound[rows]), label
    assert np.all(np.abs(gl[live] - wl[live]) <= (E + 4 * u * np.abs(wl))[live]), label
    empty = rows & ~live
    assert np.all(gl[empty] == -np.inf) and np.all(got[empty] == 0), label


def _check(kvx, c, label, scale=None, **kw):
    out, lse = kvx.attend_prefix8(*_operands(c), scale=scale, with_lse=True, **kw)
    torch.cuda.synchronize()
    _compare(c, out, lse, c["q"].shape[2] ** -0.5 if scale is None else scale, label)
    return out, lse


STEPS = [   # prefixes, requests of each, own tokens (the new ones included), new tokens
    ([1], [1], [1], [1]),
    ([0], [2], [3, 1], [1, 1]),                                       # a prefix of nothing
    ([16], [3], [1, 17, 64], [1, 1, 1]),
    ([33, 100], [2, 1], [5, 1, 40], [1, 1, 1]),
    ([300, 5, 64], [1, 0, 4], [1, 20, 3, 1, 9], [1, 2, 0, 1, 5]),     # one that nobody shares
    ([63, 65], [2, 2], [2, 0, 1, 30], [5, 3, 1, 4]),                  # rows without own keys
    ([129], [2], [70, 33], [33, 33]),                                 # chunks
    ([500], [1], [257], [257]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_prefixes_match_the_definition(gpu_kvx, dtype, d, P):
    rng = np.random.default_rng(3 * P + d)
    for step, (H, G) in zip(STEPS, [(1, 1), (2, 8), (2, 3), (3, 4), (1, 16), (2, 5), (1, 8), (2, 2)]):
        c = _case(rng, *step, H, G, d, P, dtype)
        _check(gpu_kvx, c, f"{dtype} d={d} P={P} {step} H={H} G={G}")


def _names(kvx, c):
    T, heads, d = c["q"].shape
    H, (S_, Mp), (B, M) = c["codes"].shape[1], c["ptables"].shape, c["tables"].shape
    return kvx.prefix_kernel_names(kvx.AttendDims(B, H, heads // H, T, d, 0), kvx.PrefixDims(S_, Mp, 0),
                                   kvx.Pool(c["scales"].shape[2], c["codes"].shape[2] // c["scales"].shape[2], M),
                                   "bf16" if c["q"].dtype == torch.bfloat16 else "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_both_parts_in_one_launch(gpu_kvx, dtype, d):
    """Units over several workgroups in both parts, more than 64 of either, rows of nobody's prefix."""
    rng = np.random.default_rng(d + len(dtype))
    name = f"prefix8_split_kernel<{0 if dtype == 'bf16' else 1}, {d}, 4, 1>"
    for c in (_case(rng, [1500, 40], [3, 1], [700, 3, 90, 1], [1, 2, 1, 1], 2, 4, d, 16, dtype),
              _case(rng, [1], [1], [1], [1], 1, 1, d, 128, dtype),
              _case(rng, [0, 700], [1, 1], [1100, 5, 7, 0, 64], [1, 1, 3, 2, 1], 2, 7, d, 32, dtype, first=1),
              _case(rng, [10] * 70, [1] * 70, [3] * 72, [1, 0] * 36, 1, 1, d, 16, dtype, first=1)):
        assert _names(gpu_kvx, c) == (name, name)
        _check(gpu_kvx, c, name)


WIDE = 9000        # entries of a table that keep the parts from one launch


@pytest.mark.parametrize("part", ["common", "own"])
@pytest.mark.parametrize("kernel", KERNELS)
def test_every_kernel(gpu_kvx, kernel, part):
    size, dtype, d = KERNELS[kernel]
    B, H, G, news, M = SIZES[size]
    rng = np.random.default_rng(d + len(kernel))
    news = [news[b % len(news)] for b in range(B)]
    if part == "own":       # as many requests over three prefixes, one of them nobody's
        lens = [int(x) for x in rng.integers(0, M * 16 + 1, B)]
        lens[-1] = M * 16
        count = [B // 2, 0, B - B // 2 - 1]
        c = _case(rng, [37, 16, 200], count, lens, news, H, G, d, 16, dtype, Mp=WIDE, M=M, first=1)
    else:                   # as many prefixes, the rows of each spread over one to three requests
        pages = 200 * M if size == "by rows" else M       # the work that it takes
        pre = [int(x) for x in rng.integers(0, M * 16 + 1, B)]
        pre[-1] = M * 16
        count, mine = [], []
        for n in news:
            cuts = sorted(rng.integers(0, n + 1, int(rng.integers(0, 3))).tolist())
            parts = np.diff([0] + cuts + [n]).tolist()
            count.append(len(parts))
            mine += parts
        c = _case(rng, pre, count, [n + int(rng.integers(0, 9)) for n in mine], mine, H, G, d, 16, dtype, Mp=pages, M=WIDE)
    name = kernel.replace("attend8", f"prefix8_{part}")
    if part == "common":
        name = name.replace("12, 2>", "8, 2>")      # large workgroups of 32 rows have 8 waves there
    assert _names(gpu_kvx, c)[part == "own"] == name
    _check(gpu_kvx, c, f"{part} {kernel}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_plain_call_over_whole_tables_agrees(gpu_kvx, dtype):
    """A prefix of whole pages, listed in every request's own table instead: attend_cache8 gives
    the same to rounding, and exactly the same without prefixes."""
    rng = np.random.default_rng(5)
    c = _case(rng, [160], [7], [int(x) for x in rng.integers(1, 90, 7)], [1, 2, 1, 1, 3, 1, 1], 2, 4, 128, 16, dtype)
    q, codes, scales, ptables, plens, pcu, tables, lens, cu = _operands(c)
    out, lse = _check(gpu_kvx, c, "prefix")
    whole = torch.cat([ptables[:, :10].expand(7, 10), tables], 1).contiguous()
    a, b = gpu_kvx.attend_cache8(q, codes, scales, whole, lens + 160, cu, with_lse=True)
    tol = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -17
    assert (a.float() - out.float()).abs().max() <= tol * a.float().abs().max() and (b - lse).abs().max() <= 2.0 ** -16 * b.abs().max()
    none = torch.zeros((0, 3), dtype=torch.int32, device=DEV), plens[:0], pcu[:1]
    a, b = gpu_kvx.attend_cache8(q, codes, scales, tables, lens, cu, with_lse=True)
    x, y = gpu_kvx.attend_prefix8(q, codes, scales, *none, tables, lens, cu, with_lse=True)
    assert torch.equal(a, x) and torch.equal(b, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_requests_without_a_prefix_and_rows_of_nobody(gpu_kvx, dtype):
    """Requests before and behind the shared ones; rows behind the last request stay as they were;
    one page shared by prefixes of different length; missing pages inside a prefix."""
    rng = np.random.default_rng(6)
    c = _case(rng, [50, 20], [2, 2], [9, 30, 1, 40, 17, 5], [1, 2, 1, 3, 1, 1], 2, 3, 64, 16, dtype, first=1)
    c["ptables"][1, :2] = c["ptables"][0, :2]
    c["ptables"][0, 2] = -1
    o = _operands(c)
    q = torch.cat([o[0], o[0][:4]])
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    got, lse = gpu_kvx.attend_prefix8(q, *o[1:], out=out, with_lse=True)
    assert got is out and (out[len(o[0]):] == 7).all()
    _compare(c, out[:len(o[0])], lse[:len(o[0])], 8.0 ** -1, "outside")


def test_bad_numbers(gpu_kvx):
    """NaN codes and scales of a prefix reach all its rows and no others; lengths, tables and shares
    out of range are clamped."""
    rng = np.random.default_rng(8)
    c = _case(rng, [40, 40], [3, 3], [5, 9, 2, 4, 1, 8], [1, 1, 2, 1, 1, 3], 2, 4, 128, 16, "bf16")
    good, _ = _check(gpu_kvx, c, "good")
    page = int(c["ptables"][0, 1])
    for kv in (0, 1):
        bad = dict(c, codes=c["codes"].copy())
        bad["codes"][kv, 1, page * 16 + 3, 77] = 0x7F
        out = gpu_kvx.attend_prefix8(*_operands(bad))
        hit = torch.zeros(out.shape, dtype=torch.bool, device=DEV)
        hit[:4, 4:8, 77 if kv else slice(None)] = True
        assert torch.isnan(out[hit]).all() and torch.equal(out[~hit], good[~hit])
    bad = dict(c, scales=c["scales"].copy())
    bad["scales"][1, 0, page] = np.inf
    out = gpu_kvx.attend_prefix8(*_operands(bad))
    assert torch.isnan(out[:4, :4]).all() and torch.equal(out[:, 4:], good[:, 4:]) and torch.equal(out[4:], good[4:])
    long = dict(c, plens=np.array([10 ** 9, -5]), lens=np.array([5, 9, 2, 4, 1, 10 ** 9]))
    long["ptables"] = np.concatenate([c["ptables"][:, :3], np.full((2, 2), -1)], 1)
    long["tables"] = np.where(np.arange(c["tables"].shape[1]) < -(-c["lens"][:, None] // 16), c["tables"], -1)
    full = c["codes"].copy()
    full[(full & 0x7F) == 0x7F] = 1      # the pages' ends are seen now
    long["codes"] = full
    _check(gpu_kvx, long, "lengths past the tables")


def test_workspace_streams_and_graphs(gpu_kvx):
    """One workspace for calls of different sizes and kinds in turn, on another stream, and in a
    replayed graph with other work between."""
    rng = np.random.default_rng(9)
    cases = [_case(rng, [700, 30], [20, 12], [int(x) for x in rng.integers(1, 60, 32)], [1] * 32, 2, 8, 128, 16, "bf16"),
             _case(rng, [90], [3], [40, 50, 60], [33, 40, 30], 2, 8, 128, 32, "bf16"),
             _case(rng, [5000], [4], [7, 1, 3, 2], [2, 1, 1, 1], 2, 4, 64, 16, "bf16")]
    ops = [_operands(c) for c in cases]
    spaces = [gpu_kvx.prefix_workspace(o[0], o[1], o[3], o[6]) for o in ops]
    ws = max(spaces, key=lambda w: w.numel())
    want = [gpu_kvx.attend_prefix8(*o, with_lse=True) for o in ops]
    for _ in range(3):
        for o, w in zip(ops, want):
            got = gpu_kvx.attend_prefix8(*o, with_lse=True, workspace=ws)
            assert torch.equal(got[0], w[0]) and torch.equal(got[1], w[1])
    torch.cuda.synchronize()
    assert (ws[:gpu_kvx.ATTEND_COUNTER_BYTES] == 0).all()
    s = torch.cuda.Stream()
    got = gpu_kvx.attend_prefix8(*ops[0], with_lse=True, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0][0])
    q = ops[0][0].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = gpu_kvx.attend_prefix8(q, *ops[0][1:], workspace=ws)
    for n in range(3):
        q.copy_(ops[0][0] * (n + 1))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, gpu_kvx.attend_prefix8(q, *ops[0][1:]))


def test_what_the_binding_refuses(gpu_kvx):
    c = _case(np.random.default_rng(10), [40, 40], [1, 2], [5, 9, 2], [1, 1, 2], 2, 4, 64, 16, "bf16")
    o = list(_operands(c))
    gpu_kvx.attend_prefix8(*o)

    def call(**kw):
        x = list(o)
        for i, v in kw.items():
            x[int(i[1:])] = v
        return gpu_kvx.attend_prefix8(*x)
    for kw in (dict(a3=o[3][0]), dict(a3=o[3].long()), dict(a4=o[4][:1]), dict(a5=o[5][:2]), dict(a4=o[4].cpu()),
               dict(a6=o[6][0]), dict(a7=o[7][:2]), dict(a8=o[8][:3]), dict(a0=o[0][:, :3]), dict(a0=o[0].cpu()),
               dict(a3=o[3].t())):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(longest=-1), dict(longest_prefix=-1), dict(workspace=torch.zeros(64, dtype=torch.uint8, device=DEV)),
               dict(scale=float("nan"))):
        with pytest.raises(gpu_kvx.KvxError):
            gpu_kvx.attend_prefix8(*o, **kw)
    with pytest.raises(gpu_kvx.KvxError, match="overlaps"):
        gpu_kvx.attend_prefix8(*o, out=o[0])


def test_many_prefixes(gpu_kvx):
    rng = np.random.default_rng(12)
    count = [int(x) for x in rng.integers(0, 4, 300)]
    B = sum(count)
    c = _case(rng, [int(x) for x in rng.integers(0, 60, 300)], count, [int(x) for x in rng.integers(0, 40, B)],
              [int(x) for x in rng.integers(0, 3, B)], 1, 4, 64, 16, "bf16")
    _check(gpu_kvx, c, "300 prefixes")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_prefixes(gpu_kvx, dtype):
    rng = np.random.default_rng(13)
    for P, d in ((16, 128), (128, 64)):
        _check(gpu_kvx, _case(rng, [20011, 3], [3, 1], [1, 5, 40, 2], [1, 2, 1, 1], 1, 4, d, P, dtype), f"{dtype} 20011 keys")
