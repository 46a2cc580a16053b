"""Token sampling on the GPU against the definition in 64 bits.

Tokens have to be equal.  Weights are whole numbers of 2^-43 of the best one's, so sums over V of
them are off by at most V 2^-44 of the best weight, which is no more than that of the total; a sum
of V positive doubles, one after another, is off by less than V 2^-52 of the total, the terms'
rounding included.  A draw within that of a border could go to the neighbour, and the test skips
such rows, of which there may be hardly any.  logprob: ln of the
total to V 2^-44 + 2^-40, then fp32's rounding."""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from tests._parity import np32

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
SETTINGS = [(0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.0), (0.7, 50, 1.0, 0.0), (0.7, 50, 0.9, 0.0), (1.0, 0, 0.9, 0.0),
            (1.3, 0, 0.999, 0.0), (1.0, 0, 1.0, 0.1), (0.8, 0, 0.95, 0.02), (2.0, 1000, 1.0, 0.0),
            (2.5, 700, 0.8, 0.001), (1.0, 1, 1.0, 0.0), (1.0, 0, 0.0, 0.0), (1.0, 0, 1.0, 1.0), (0.05, 3, 0.5, 0.0),
            (50.0, 0, 0.5, 0.0), (float("inf"), 0, 1.0, 0.0), (float("inf"), 7, 0.4, 0.0), (-1.0, 5, 0.5, 0.5),
            (1.5, 6000, 0.97, 0.0), (1e-30, 0, 0.9, 0.0), (3.0, 30000, 1.0, 0.0), (1.0, 2 ** 31 - 1, 2.0, -1.0)]


def _check(kvx, logits, settings, u, workspace=None, exact=None):
    B, V = logits.shape
    t, k, p, m = (list(x) for x in zip(*settings))
    f = lambda x: torch.tensor(x, dtype=torch.float32, device=DEV)  # noqa: E731
    tokens, logprob = kvx.sample_tokens(logits, f(u), f(t), torch.tensor(k, dtype=torch.int32, device=DEV), f(p), f(m),
                                        with_logprob=True, workspace=workspace)
    x, tokens, logprob = np32(logits).astype(np.float64), tokens.cpu().numpy(), logprob.cpu().numpy()
    r = np.float32
    skipped = 0
    for b in range(B):
        token, lp, near = S.sample_token(x[b], r(u[b]), float(r(t[b])), k[b], float(r(p[b])), float(r(m[b])))
        if near <= V * (2.0 ** -44 + 2.0 ** -52) and not (exact and exact(b)):
            skipped += 1
            continue
        assert tokens[b] == token, (b, settings[b], u[b], tokens[b], token, near)
        if np.isinf(lp):
            assert logprob[b] == lp
        else:
            assert abs(logprob[b] - lp) <= V * 2.0 ** -44 + 2.0 ** -40 + 2.0 ** -24 * abs(lp) * 1.01, (b, settings[b])
    assert skipped <= 1 + B // 20
    return tokens


def _logits(B, V, dtype, seed, spread=2.0):
    g = np.random.default_rng(seed)
    x = g.standard_normal((B, V)) * spread
    n = min(V, 40)
    for b in range(B):
        x[b, g.integers(0, V, n)] += g.random(n) ** 2 * g.uniform(0, 15)
    return torch.tensor(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 63, 64, 65, 257, 1000, 4096, 4099, 32000, 50001, 131072])
def test_settings(gpu_kvx, V, dtype):
    g = np.random.default_rng(V)
    settings = SETTINGS * 2
    u = g.random(len(settings))
    u[0], u[1], u[3], u[23], u[4] = 0.0, 0.0, 0.0, 1.0 - 2.0 ** -24, 1.0 - 2.0 ** -24
    _check(gpu_kvx, _logits(len(settings), V, dtype, V + 1), settings, u)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [1, 3, 40, 300])
def test_batches(gpu_kvx, B, dtype):
    """Few rows are split over many workgroups, many over few; flat and peaked rows."""
    g = np.random.default_rng(B)
    settings = [SETTINGS[i % len(SETTINGS)] for i in range(4, 4 + B)]
    for spread in (0.3, 3.0):
        _check(gpu_kvx, _logits(B, 20011, dtype, B, spread), settings, g.random(B))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,V", [(300, 60011), (600, 20013), (1100, 8200)])
def test_long_rows_of_large_batches(gpu_kvx, B, V, dtype):
    """Workgroups with many logits a lane, three of them a row or one."""
    g = np.random.default_rng(B)
    few = [(1.0, 50, 0.9, 0.0), (0.7, 128, 1.0, 0.0), (1.5, 1, 1.0, 0.0), (1.0, 20, 1.0, 0.1), (0.0, 5, 1.0, 0.0),
           (1.0, 0, 0.95, 0.0), (1.0, 0, 1.0, 0.0), (1.2, 129, 0.9, 0.0)]
    x = _logits(B, V, dtype, B)
    x[5::9] = -float("inf")
    x[5::9, V // 3:V // 3 + 40] = 1.0
    _check(gpu_kvx, x, [few[b % len(few)] for b in range(B)], g.random(B))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks(gpu_kvx, dtype):
    """Masked logits: -inf and NaN, rows that have one token or none, the least finite number,
    +inf."""
    V, n = 9001, len(SETTINGS)
    g = np.random.default_rng(7)
    for kind in range(7):
        x = _logits(n, V, dtype, 50 + kind)
        if kind == 0:
            x[torch.rand(x.shape, generator=torch.Generator().manual_seed(1)).to(DEV) < 0.9] = -float("inf")
        elif kind == 1:
            x[torch.rand(x.shape, generator=torch.Generator().manual_seed(2)).to(DEV) < 0.5] = float("nan")
        elif kind == 2:
            x[:] = -float("inf")
            x[::2] = float("nan")
        elif kind == 3:
            x[:, :] = -float("inf")
            x[:, 777] = -3.0
        elif kind == 4:
            x[:, 100:] = torch.finfo(x.dtype).min
        elif kind == 5:
            x[:, 5::100] = float("inf")
        else:
            x[:, 1:] = -float("inf")
            x[1::2, 0] = -float("inf")
            x[1::2, V - 1] = torch.finfo(x.dtype).min
        tokens = _check(gpu_kvx, x, SETTINGS, g.random(n), exact=lambda b: kind in (2, 3))
        if kind == 2:
            assert (tokens == -1).all()
        elif kind == 3:
            assert (tokens == 777).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [16, 5000, 70001])
def test_ties(gpu_kvx, V, dtype):
    """Equal logits (both zeros among them): cut by index.  All equal: the weights are one, so that
    every sum is a whole number and borders are met exactly."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    settings, u = [], []
    for k, p in ((0, 0.5), (0, 0.25), (V // 2, 1.0), (V // 4, 0.5), (0, 1.0), (3, 1.0), (5000, 0.75)):
        for r in (0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24):
            settings.append((1.0, k, p, 0.0))
            u.append(r)
    for value in (0.0, 3.0, -1e30):
        x = torch.full((len(u), V), value, dtype=dt, device=DEV)
        if value == 0.0:
            x[:, ::3] = -0.0
        _check(gpu_kvx, x, settings, u, exact=lambda b: True)
    few = torch.tensor([1.5, 0.25, -2.0, 0.0, -0.0], dtype=dt)[torch.arange(V) * 7 % 5].expand(len(u), V).contiguous().to(DEV)
    g = np.random.default_rng(V)
    best = int((few[0] == 1.5).sum())      # top-k among these: whole numbers again
    _check(gpu_kvx, few, settings, g.random(len(u)), exact=lambda b: 0 < settings[b][1] <= best)
    _check(gpu_kvx, few, [SETTINGS[i % len(SETTINGS)] for i in range(len(u))], g.random(len(u)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [3000, 40009, 140001])
def test_spreads(gpu_kvx, V, dtype):
    """High temperatures, logits that differ by much less than a temperature or by next to nothing,
    a few far below all others, most masked: wherever the cut lies in how many tokens."""
    temperatures, cuts = (5.0, 30.0, 1e3, 1e30, float("inf")), ((0, 0.9), (0, 0.3), (V // 2, 1.0), (V // 3, 0.6), (200, 1.0))
    settings = [(t, k, p, 0.0) for t in temperatures for k, p in cuts]
    g = np.random.default_rng(V)
    for kind in range(5):
        x = torch.tensor(g.standard_normal((len(settings), V)) * (2.5, 1e-3, 1e-36, 2.5, 2.5)[kind])
        if kind == 1:
            x += 1.0
        elif kind == 3:
            x[:, ::1000] = -3e4
        elif kind == 4:
            x[torch.rand(x.shape, generator=torch.Generator().manual_seed(V)) < 0.8] = -float("inf")
            x[1::4, 17] = torch.finfo(torch.bfloat16).min
        x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)
        _check(gpu_kvx, x, settings, g.random(len(settings)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [64, 128, 300])
def test_likely_tokens_side_by_side(gpu_kvx, width, dtype):
    """The top-k lie in one run of the vocabulary, anywhere in it, so that one workgroup has them
    all; or every so many tokens."""
    V, settings = 50021, [(1.0, k, p, m) for k in (2, 20, 50, 64, 120, 128) for p, m in ((1.0, 0.0), (0.9, 0.0))]
    g = np.random.default_rng(width)
    for B in (1, 4, len(settings)):
        x = torch.tensor(g.standard_normal((B, V)) * 0.5)
        for b in range(B):
            at = (0, V - width, g.integers(0, V - width))[b % 3]
            some = (np.arange(at, at + width) if b % 4 < 3 else np.arange(width) * 128 % V)
            x[b, some] += torch.tensor(6.0 + g.random(width))
        x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)
        for i in range(0, len(settings), B):
            _check(gpu_kvx, x, (settings * 2)[i:i + B], g.random(B))


def test_rows_apart(gpu_kvx):
    """Views: a stride that is not the row's length, rows that begin anywhere, shared rows."""
    for dtype in ("bf16", "f32"):
        x = _logits(30, 6011, dtype, 9)
        g = np.random.default_rng(9)
        settings = [SETTINGS[i % len(SETTINGS)] for i in range(30)]
        for lo, hi in ((0, 6011), (1, 6010), (3, 400), (5, 13), (7, 8), (2, 4098)):
            _check(gpu_kvx, x[:, lo:hi], settings, g.random(30))
        one = x[4:5].expand(30, 6011)
        _check(gpu_kvx, one, settings, g.random(30))


def test_defaults_and_outputs(gpu_kvx):
    x = _logits(5, 3001, "f32", 11)
    u = torch.rand(5, device=DEV)
    a = gpu_kvx.sample_tokens(x, u)
    out = torch.empty(5, dtype=torch.int32, device=DEV)
    assert gpu_kvx.sample_tokens(x, u, out=out) is out
    want = [S.sample_token(r, v)[0] for r, v in zip(np32(x).astype(np.float64), u.cpu().numpy())]
    assert a.tolist() == want and out.tolist() == want
    assert gpu_kvx.sample_tokens(x[:0], u[:0]).shape == (0,)
    # random numbers outside [0, 1) and NaN
    u = torch.tensor([-1.0, 1.0, 2.0, float("nan"), float("inf")], device=DEV)
    got = gpu_kvx.sample_tokens(x, u).tolist()
    want = [S.sample_token(r, v)[0] for r, v in zip(np32(x).astype(np.float64), [0, 1, 1, 0, 1])]
    assert got[0] == want[0] and got[3] == want[3] and all(0 <= t < 3001 for t in got)
    nan = torch.full((5,), float("nan"), device=DEV)
    assert gpu_kvx.sample_tokens(x, u, nan).tolist() == x.argmax(1).tolist()
    assert gpu_kvx.sample_tokens(x, u, None, None, nan, nan).tolist() == got


def test_repeats_streams_and_graphs(gpu_kvx):
    """The same answer every time, on another stream, and from a replayed graph, with the workspace
    kept and in whatever state."""
    B, V = 24, 60013
    settings = [SETTINGS[i % len(SETTINGS)] for i in range(B)]
    t, k, p, m = (list(v) for v in zip(*settings))
    f = lambda v: torch.tensor(v, dtype=torch.float32, device=DEV)  # noqa: E731
    t, p, m, k = f(t), f(p), f(m), torch.tensor(k, dtype=torch.int32, device=DEV)
    x, u = _logits(B, V, "bf16", 13), torch.rand(B, device=DEV)
    ws = gpu_kvx.sample_workspace(x)
    ws.view(B, -1)[:, gpu_kvx.SAMPLE_COUNTER_BYTES:].fill_(255)
    want = gpu_kvx.sample_tokens(x, u, t, k, p, m, with_logprob=True, workspace=ws)
    for _ in range(5):
        got = gpu_kvx.sample_tokens(x, u, t, k, p, m, with_logprob=True, workspace=ws)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    torch.cuda.synchronize()
    assert (ws.view(B, -1)[:, :gpu_kvx.SAMPLE_COUNTER_BYTES] == 0).all()
    few = gpu_kvx.sample_tokens(x[:3, :500], u[:3], t[:3], k[:3], p[:3], m[:3], workspace=ws)      # other sizes in it
    assert torch.equal(few, gpu_kvx.sample_tokens(x[:3, :500].contiguous(), u[:3], t[:3], k[:3], p[:3], m[:3]))
    s = torch.cuda.Stream()
    got = gpu_kvx.sample_tokens(x, u, t, k, p, m, with_logprob=True, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = gpu_kvx.sample_tokens(x, u, t, k, p, m, with_logprob=True, workspace=ws)
    for n in range(4):
        x.copy_(_logits(B, V, "bf16", 20 + n))
        u.copy_(torch.rand(B, device=DEV))
        g.replay()
        torch.cuda.synchronize()
        want = gpu_kvx.sample_tokens(x, u, t, k, p, m, with_logprob=True)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_the_largest_vocabulary(gpu_kvx):
    V = 1 << 20
    x = _logits(6, V, "bf16", 31, spread=0.5)
    settings = [(1.0, 0, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.0, 100, 1.0, 0.0), (1.0, 300000, 0.5, 0.0), (0.0, 0, 1.0, 0.0),
                (float("inf"), 0, 0.5, 0.0)]
    t, k, p, m = (list(v) for v in zip(*settings))
    f = lambda v: torch.tensor(v, dtype=torch.float32, device=DEV)  # noqa: E731
    u = [0.1, 0.9, 0.5, 0.7, 0.3, 0.37]
    got = gpu_kvx.sample_tokens(x, f(u), f(t), torch.tensor(k, dtype=torch.int32, device=DEV), f(p), f(m)).tolist()
    rows = np32(x).astype(np.float64)
    for b in range(6):
        token, _, near = S.sample_token(rows[b], np.float32(u[b]), t[b], k[b], float(np.float32(p[b])), m[b])
        assert got[b] == token or near <= 2.0 ** -24
    with pytest.raises(gpu_kvx.KvxError, match="1048576"):
        gpu_kvx.sample_tokens(torch.zeros((1, V + 1), device=DEV), f([0.5]))


def test_what_the_binding_refuses(gpu_kvx):
    x, u = torch.zeros((4, 100), device=DEV), torch.zeros(4, device=DEV)
    i = torch.zeros(4, dtype=torch.int32, device=DEV)
    f = gpu_kvx.sample_tokens
    for a in ((x[0], u), (x, u[:3]), (x, u.double()), (x, u.cpu()), (x.cpu(), u), (x[:, ::2], u), (x, u, u[:2]),
              (x, u, u, i.long()), (x, u, u, i[:2]), (x, u, u, i, i), (x, u, u, i, u, i)):
        with pytest.raises(ValueError):
            f(*a)
    with pytest.raises(TypeError):
        f(x, None)
    with pytest.raises(TypeError):
        f(x.half(), u)
    with pytest.raises(ValueError):
        f(x, u, out=i.long())
    with pytest.raises(gpu_kvx.KvxError, match="overlaps"):
        f(x, u, None, i, out=i)
    ws = gpu_kvx.sample_workspace(x)
    for bad in (ws[:-1], ws[:0], ws[128:]):
        with pytest.raises(gpu_kvx.KvxError, match="workspace"):
            f(x, u, workspace=bad)
