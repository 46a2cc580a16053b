"""Plain definitions of the serving operators: page plan, 8-bit store and attention
over the 8-bit pool.  NumPy, float64, one request, page or row at a time."""

from __future__ import annotations

import numpy as np

E4M3_MAX = 448.0


def _decode(code: int) -> float:
    """Value of an OCP e4m3 code: sign, 4 exponent bits (bias 7), 3 mantissa bits; no
    infinity, NaN where all but the sign are ones."""
    sign = -1.0 if code & 0x80 else 1.0
    e, m = code >> 3 & 15, code & 7
    if e == 15 and m == 7:
        return float("nan")
    return sign * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))


E4M3 = np.array([_decode(c) for c in range(256)])


def encode_e4m3(x):
    """Nearest e4m3 codes of x (|x| <= 448 where finite), ties to the even code;
    infinities and NaN become NaN."""
    x = np.asarray(x, np.float64)
    grid = E4M3[:127]                                  # 0 .. 448, rising
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert a.max(initial=0.0) <= E4M3_MAX
    hi = np.searchsorted(grid, a)                      # grid[hi - 1] < a <= grid[hi]
    lo = np.maximum(hi - 1, 0)
    down, up = a - grid[lo], grid[hi] - a
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isfinite(x), code, 127)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def page_scale(x):
    """The smallest power of two s >= 2^-118 with |x| <= 448 s over the finite values."""
    x = np.abs(x[np.isfinite(x)]) if x.size else x
    amax = float(x.max(initial=0.0))
    s = 2.0 ** -118
    while amax > E4M3_MAX * s:
        s *= 2.0
    return s


def plan_pages(lens, add, tables, ring, free, T, page_size):
    """Returns lens, cu, positions, slots, free (head, count, refused, rows) and updates
    tables and ring (NumPy int arrays) in place."""
    B, N, M, P = len(lens), len(ring), tables.shape[1], page_size
    head, count = int(free[0]) % N, int(free[1])
    before = [max(int(n), 0) for n in lens]
    after, cu, refused = [int(n) for n in lens], [0], 0
    positions, slots = np.zeros(T, np.int64), np.full(T, -1, np.int64)
    row, taken, asked, back = 0, 0, 0, []
    for b in range(B):
        n = max(int(add[b]), 0)
        have, need = -(-before[b] // P), -(-(before[b] + n) // P)
        start, row = row, row + n
        cu.append(min(row, T))
        if add[b] < 0:
            back += [int(p) for p in tables[b, :min(have, M)]]
            after[b] = 0
            continue
        fits = n == 0 or (need <= M and row <= T)
        ask = need - have if fits and n > 0 else 0
        asked += ask
        granted = fits and (ask == 0 or asked <= count)
        if granted:
            for i in range(ask):
                tables[b, have + i] = ring[(head + taken) % N]
                taken += 1
            after[b] = before[b] + n if n else before[b]
        else:
            refused += 1
        for i in range(n):
            if start + i >= T:
                break
            p = before[b] + i
            positions[start + i] = p
            if granted and 0 <= tables[b, p // P] < N:
                slots[start + i] = tables[b, p // P] * P + p % P
    back = back[:N - count]
    for i, p in enumerate(back):
        ring[(head + count + i) % N] = p
    return (np.array(after), np.array(cu), positions, slots,
            np.array([(head + taken) % N, count - taken + len(back), refused, min(row, T)]))


def store_cache8(k, v, slots, codes, scales):
    """k, v [L, H, T, d] float64; codes [L, 2, H, S, d] uint8 and scales
    [L, 2, H, N] float64 are updated in place."""
    L, H, T, d = k.shape
    S, N = codes.shape[3], scales.shape[3]
    P = S // N
    t = 0
    while t < T:
        if not 0 <= slots[t] < S:
            t += 1
            continue
        page, e = slots[t] // P, t + 1
        while e < T and 0 <= slots[e] < S and slots[e] // P == page:
            e += 1
        held = int(slots[t] % P)
        for l in range(L):
            for h in range(H):
                for kv, x in enumerate((k, v)):
                    rows = x[l, h, t:e]
                    s = page_scale(rows)
                    if held:
                        old = scales[l, kv, h, page]
                        s = max(s, old)
                        was = codes[l, kv, h, page * P:page * P + held]
                        if s > old:
                            codes[l, kv, h, page * P:page * P + held] = encode_e4m3(E4M3[was] * (old / s))
                    scales[l, kv, h, page] = s
                    codes[l, kv, h, slots[t:e]] = encode_e4m3(rows / s)
        t = e


def attend_cache8(q, codes, scales, tables, lens, cu, scale):
    """q [T, H*G, d] float64; codes [2, H, S, d]; scales [2, H, N].  Returns out, lse,
    and for error bounds the size of a row's weighted values sum_j p_j |V_j| and of its
    scores max_j sum_c |q_c K_jc| * |scale|.  Rows outside every request are NaN."""
    T, heads, d = q.shape
    H, S, N = codes.shape[1], codes.shape[2], scales.shape[2]
    G, P, B, M = heads // H, S // N, tables.shape[0], tables.shape[1]
    out = np.full(q.shape, np.nan)
    lse = np.full((T, heads), np.nan)
    size_v, size_s = np.zeros(q.shape), np.zeros((T, heads))
    for b in range(B):
        a, e = min(max(int(cu[b]), 0), T), min(int(cu[b + 1]), T)
        n = min(max(int(lens[b]), 0), M * P)
        page = np.repeat(tables[b, :-(-n // P)].astype(np.int64), P)[:n]
        real = (page >= 0) & (page < N)
        slot = np.where(real, page, 0) * P + np.arange(n) % P
        for h in range(H):
            K = E4M3[codes[0, h, slot]] * scales[0, h, slot // P, None]
            V = E4M3[codes[1, h, slot]] * scales[1, h, slot // P, None]
            for t in range(a, e):
                see = np.flatnonzero(real[:max(n - (e - t) + 1, 0)])
                for x in range(h * G, (h + 1) * G):
                    if len(see) == 0:
                        out[t, x], lse[t, x] = 0.0, -np.inf
                        continue
                    s = scale * (K[see] @ q[t, x])
                    top = s.max()
                    p = np.exp(s - top)
                    lse[t, x] = top + np.log(p.sum())
                    p /= p.sum()
                    out[t, x] = p @ V[see]
                    size_v[t, x] = p @ np.abs(V[see])
                    size_s[t, x] = abs(scale) * (np.abs(K[see]) @ np.abs(q[t, x])).max()
    return out, lse, size_v, size_s
