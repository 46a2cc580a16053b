"""Norm and rotation of queries and keys on the GPU against the definition in 64 bits.

Tolerance.  u = 2^-24.  The sum of d squares has d + log2 terms of rounding at most (d + 8) u of
itself, half of that after the root; the root, its Newton step and the two products add 6 u; the
rotation three roundings and its coefficients (sine and cosine to u each, and the angle: p w / 2 pi
formed in fp64 is off by at most 4 * 2^-53 |p w| radians) 4 u + 2^-51 |p w| of the plane's size.
The output's rounding adds half a step: 2^-8 (bf16) or u (fp32) of the value."""

import numpy as np
import pytest
import torch

from oracle import kvx_oracle as O
from oracle import serve_oracle as S
from paper_2608_03893_amd import synth
from tests._parity import np32

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
U = 2.0 ** -24
ROPES = [synth.rope_dict(1e6), synth.rope_dict(1e4, style=1),
         synth.rope_dict(5e5, factor=8.0, low_freq_factor=1.0, high_freq_factor=4.0)]


def _check(got, x, w, eps, pos, rope, dtype):
    d = x.shape[2]
    pos = pos.cpu().numpy()
    want, size = S.norm_rope(np32(x).astype(np.float64), None if w is None else np32(w), float(np.float32(eps)), pos, rope)
    got = np32(got).astype(np.float64)
    angle = np.abs(pos).max(initial=0) * O.rope_inv_freq(rope, d).max()
    bound = ((d + 8) / 2 + 10) * U * size + 2.0 ** -51 * angle * size
    bound = bound + (U if dtype == "f32" else 2.0 ** -8) * (np.abs(want) + bound) + 2.0 ** -126
    assert got.shape == want.shape
    assert (np.abs(got - want) <= bound).all(), np.max(np.abs(got - want) / bound)


def _case(T, Hq, Hk, d, dtype, seed, packed=False):
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = (torch.randn((T, Hq + 2 * Hk, d), generator=g) * 3).to(dt).to(DEV)
    q, k = x[:, :Hq], x[:, Hq:Hq + Hk]
    if not packed:
        q, k = q.contiguous(), k.contiguous()
    w = [torch.exp(torch.randn(d, generator=g) * 0.3).to(dt).to(DEV) for _ in range(2)]
    pos = torch.randint(0, 131072, (T,), generator=g).to(torch.int32).to(DEV)
    return q, k, w[0], w[1], pos


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rope", ROPES, ids=["half", "interleaved", "scaled"])
@pytest.mark.parametrize("T,Hq,Hk", [(1, 1, 1), (1, 40, 8), (7, 5, 3), (64, 64, 8), (333, 7, 1), (1500, 9, 2)])
def test_norm_rope(gpu_kvx, T, Hq, Hk, d, dtype, rope):
    q, k, qw, kw, pos = _case(T, Hq, Hk, d, dtype, T * 7 + Hq)
    qo, ko = gpu_kvx.norm_rope(q, k, qw, kw, rope, pos, eps=1e-6)
    _check(qo, q, qw, 1e-6, pos, rope, dtype)
    _check(ko, k, kw, 1e-6, pos, rope, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_of_a_projection_and_missing_operands(gpu_kvx, dtype):
    rope = ROPES[0]
    q, k, qw, kw, pos = _case(37, 12, 4, 128, dtype, 5, packed=True)
    whole = gpu_kvx.norm_rope(q, k, qw, kw, rope, pos)
    dense = gpu_kvx.norm_rope(q.contiguous(), k.contiguous(), qw, kw, rope, pos)
    for a, b in zip(whole, dense):
        assert torch.equal(a, b)
    qo, none = gpu_kvx.norm_rope(q, None, qw, None, rope, pos)
    assert none is None and torch.equal(qo, whole[0])
    for qw_, kw_ in ((None, kw), (qw, None), (None, None)):       # rotated only
        a, b = gpu_kvx.norm_rope(q, k, qw_, kw_, rope, pos)
        _check(a, q, qw_, 1e-6, pos, rope, dtype)
        _check(b, k, kw_, 1e-6, pos, rope, dtype)
    # heads first, as a mapped cache has them; rows that share their memory
    t = q.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(gpu_kvx.norm_rope(t, k, qw, kw, rope, pos)[0], whole[0])
    one = q[:1].expand(37, 12, 128)
    _check(gpu_kvx.norm_rope(one, k, qw, kw, rope, pos)[0], one, qw, 1e-6, pos, rope, dtype)


def test_in_place_and_given_outputs(gpu_kvx):
    for T in (3, 900):
        q, k, qw, kw, pos = _case(T, 10, 2, 64, "bf16", 6)
        want = gpu_kvx.norm_rope(q, k, qw, kw, ROPES[1], pos)
        out = torch.empty_like(q), torch.empty_like(k)
        assert gpu_kvx.norm_rope(q, k, qw, kw, ROPES[1], pos, out=out) is out
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
        gpu_kvx.norm_rope(q, k, qw, kw, ROPES[1], pos, out=(q, k))
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_values(gpu_kvx, dtype):
    """Squares past fp32, tiny rows, zero rows, eps of 0 and large; NaN and infinity stay in
    their head; positions from -2^31 to 2^31 - 1."""
    rope = ROPES[0]
    q, k, qw, kw, pos = _case(6, 4, 1, 128, dtype, 8)
    q[0] *= 1e30
    q[1] *= 1e-30
    q[2, 1] = 0
    q[3, 0] *= 1e19
    for eps in (0.0, 1e-6, 1e4):
        got, _ = gpu_kvx.norm_rope(q, k, qw, kw, rope, pos, eps=eps)
        x = q.clone()
        if eps == 0.0:
            assert torch.isnan(got[2, 1]).all()        # 0 / 0
            got, x = got[:, [0, 2, 3]], x[:, [0, 2, 3]]
        _check(got, x, qw, eps, pos, rope, dtype)
    bad = q.clone()
    bad[4, 2, 5], bad[5, 3, 100] = float("nan"), float("inf")
    got, want = (gpu_kvx.norm_rope(x, k, qw, kw, rope, pos)[0] for x in (bad, q))
    assert torch.isnan(got[4, 2]).all() and torch.isnan(got[5, 3]).any()
    hit = torch.zeros((6, 4), dtype=torch.bool, device=DEV)
    hit[4, 2] = hit[5, 3] = True
    assert torch.equal(got[~hit], want[~hit])
    far = torch.tensor([-2 ** 31, 2 ** 31 - 1, -1, 0, 1, 10 ** 9], dtype=torch.int32, device=DEV)
    q, k, qw, kw, _ = _case(6, 4, 1, 128, dtype, 9)
    _check(gpu_kvx.norm_rope(q, k, qw, kw, rope, far)[0], q, qw, 1e-6, far, rope, dtype)


def test_more_rows_than_a_launch_takes(gpu_kvx):
    """2^25 waves a launch; elements whose offset passes 2^31."""
    T, d = 2 ** 25 + 77, 64
    x = torch.empty((T, 1, d), dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    parts = [slice(0, 500), slice(2 ** 25 - 300, T)]
    for part in parts:
        x[part] = torch.randn(x[part].shape, generator=g, device=DEV).to(x.dtype)
    w = torch.rand(d, generator=g, device=DEV).to(x.dtype)
    pos = torch.arange(T, dtype=torch.int32, device=DEV) % 131072
    out = torch.zeros_like(x)
    gpu_kvx.norm_rope(x, None, w, None, ROPES[0], pos, out=(out, None))
    for part in parts:
        _check(out[part], x[part], w, 1e-6, pos[part], ROPES[0], "bf16")


def test_empty_streams_and_graphs(gpu_kvx):
    q, k, qw, kw, pos = _case(0, 4, 2, 128, "bf16", 1)
    a, b = gpu_kvx.norm_rope(q, k, qw, kw, ROPES[0], pos)
    assert a.shape == q.shape and b.shape == k.shape
    q, k, qw, kw, pos = _case(50, 16, 2, 128, "bf16", 10)
    want = gpu_kvx.norm_rope(q, k, qw, kw, ROPES[0], pos)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = gpu_kvx.norm_rope(q, k, qw, kw, ROPES[0], pos, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = gpu_kvx.norm_rope(q, k, qw, kw, ROPES[0], pos)
    for n in range(3):
        q.copy_(torch.randn(q.shape, device=DEV))
        pos.add_(n)
        g.replay()
        torch.cuda.synchronize()
        want = gpu_kvx.norm_rope(q, k, qw, kw, ROPES[0], pos)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_what_the_binding_refuses(gpu_kvx):
    q, k, qw, kw, pos = _case(4, 4, 2, 64, "bf16", 2)
    f, rope = gpu_kvx.norm_rope, ROPES[0]
    for a in ((q[0], k, qw, kw, rope, pos), (q, k[:3], qw, kw, rope, pos), (q, k.float(), qw, kw, rope, pos),
              (q, k, qw[:32], kw, rope, pos), (q, k, qw.float(), kw, rope, pos), (q, k, qw, kw, rope, pos[:3]),
              (q, k, qw, kw, rope, pos.long()), (q, None, qw, kw, rope, pos), (q.cpu(), k, qw, kw, rope, pos),
              (q, k.cpu(), qw, kw, rope, pos), (q[..., ::2], k[..., ::2], None, None, rope, pos), (q, k[:, :0], qw, kw, rope, pos)):
        with pytest.raises((ValueError, gpu_kvx.KvxError)):
            f(*a)
    with pytest.raises(TypeError):
        f(q.half(), k.half(), None, None, rope, pos)
    with pytest.raises(TypeError):
        f(q, k, qw, kw, rope, pos, out=q)
    with pytest.raises(ValueError):
        f(q, k, qw, kw, rope, pos, out=(q, q))
    for out in ((q, q[:, :2].contiguous()), (k.repeat(1, 2, 1), k)):
        f(q, k, qw, kw, rope, pos, out=out)
    big = torch.zeros((9, 4, 64), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(gpu_kvx.KvxError, match="overlaps"):
        f(big[:4], k, qw, kw, rope, pos, out=(big[1:5], torch.empty_like(k)))
