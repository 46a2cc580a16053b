"""Pins of the serving oracle (CPU): e4m3 against torch's type, the scale rule, pages and
slots against what a plan has to keep, attention against a dense softmax."""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S


def test_e4m3_values_and_rounding_match_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(S.E4M3, want, equal_nan=True)
    x = torch.cat([torch.randn(20000) * 10.0 ** torch.randint(-4, 3, (20000,)),
                   torch.tensor([0.0, -0.0, 448.0, -448.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11])])
    x = x.clamp(-448, 448)
    mid = torch.from_numpy((S.E4M3[:126] + S.E4M3[1:127]) / 2).float()   # ties
    x = torch.cat([x, mid, -mid])
    got = S.encode_e4m3(x.numpy())
    assert np.array_equal(got, x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert set(S.encode_e4m3([np.inf, np.nan, -np.inf]) & 0x7F) == {0x7F}


@pytest.mark.parametrize("amax,want", [(448.0, 1.0), (448.001, 2.0), (224.0, 0.5), (3.5, 2.0 ** -7),
                                       (3.52, 2.0 ** -6), (0.0, 2.0 ** -118), (2.0 ** -130, 2.0 ** -118)])
def test_page_scale(amax, want):
    assert S.page_scale(np.array([[amax / 3, -amax], [np.nan, np.inf]])) == want


def test_plan_keeps_every_page_once():
    rng = np.random.default_rng(0)
    B, N, P, M = 12, 80, 16, 9
    lens, tables = np.zeros(B, int), np.full((B, M), -1)
    ring, free = rng.permutation(N), np.array([17, N])
    for step in range(60):
        add = rng.integers(-1, 30, B) * (rng.random(B) < 0.6)
        before = lens.copy()
        lens, cu, pos, slots, free = S.plan_pages(lens, add, tables, ring, free, 160, P)
        held = [list(tables[b, :-(-lens[b] // P)]) for b in range(B)]
        have = sum(held, []) + [ring[(free[0] + i) % N] for i in range(free[1])]
        assert sorted(have) == list(range(N))
        used = slots[slots >= 0]
        assert len(set(used)) == len(used)
        for b in range(B):
            if add[b] > 0 and lens[b] != before[b]:
                assert lens[b] == before[b] + add[b]
                p = np.arange(before[b], lens[b])
                assert np.array_equal(pos[cu[b]:cu[b + 1]], p)
                assert np.array_equal(slots[cu[b]:cu[b + 1]], tables[b, p // P] * P + p % P)


def test_store_at_once_equals_store_in_turns_where_the_scale_holds():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 1, 2, 23, 64))
    x[:, :, :, 0, 0] = 9.0           # the first row already has the page's scale
    x[:, :, :, 16, 0] = 9.0
    slots = np.concatenate([np.arange(48, 64), np.arange(0, 7)])
    whole = np.zeros((1, 2, 2, 64, 64), np.uint8), np.ones((1, 2, 2, 4))
    turns = np.zeros((1, 2, 2, 64, 64), np.uint8), np.ones((1, 2, 2, 4))
    S.store_cache8(x[0], x[1], slots, *whole)
    for a, e in ((0, 1), (1, 5), (5, 17), (17, 23)):
        S.store_cache8(x[0][:, :, a:e], x[1][:, :, a:e], slots[a:e], *turns)
    assert np.array_equal(whole[0], turns[0]) and np.array_equal(whole[1], turns[1])
    kept = S.E4M3[whole[0][0, 0, :, slots[:16]]] * whole[1][0, 0, :, 3, None]
    assert np.abs(kept - x[0][0][:, :16].transpose(1, 0, 2)).max() <= 9.0 / 16


def test_attention_against_a_dense_softmax():
    rng = np.random.default_rng(2)
    H, G, d, P, N = 2, 3, 64, 16, 7
    codes = rng.integers(0, 120, (2, H, N * P, d), dtype=np.uint8)
    scales = 2.0 ** rng.integers(-9, -5, (2, H, N))
    tables = np.array([[3, 1, 6], [0, 5, -1]])
    lens, cu = np.array([40, 17]), np.array([0, 5, 7])
    q = rng.standard_normal((7, H * G, d)) * 0.1
    out, lse, _, _ = S.attend_cache8(q, codes, scales, tables, lens, cu, 0.125)
    val = S.E4M3[codes].reshape(2, H, N, P, d) * scales[..., None, None]
    for b in range(2):
        kv = torch.from_numpy(val[:, :, tables[b]].reshape(2, H, -1, d)[:, :, :lens[b]])
        n = cu[b + 1] - cu[b]
        x = torch.from_numpy(q[cu[b]:cu[b + 1]]).view(n, H, G, d)
        s = torch.einsum("nhgd,hjd->hgnj", x, kv[0]) * 0.125
        mask = torch.ones(n, lens[b], dtype=torch.bool).tril(lens[b] - n)
        s = s.masked_fill(~mask, -torch.inf)
        want = torch.einsum("hgnj,hjd->nhgd", s.softmax(-1), kv[1]).reshape(n, H * G, d)
        assert np.allclose(out[cu[b]:cu[b + 1]], want.numpy(), rtol=1e-12, atol=1e-12)
        assert np.allclose(lse[cu[b]:cu[b + 1]], s.logsumexp(-1).permute(2, 0, 1).reshape(n, -1).numpy())
