"""The page plan on the GPU against its plain definition: whole numbers, so equal."""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from tests._parity import log

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _t(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def _state(rng, B, N, P, M, longest):
    """Tables that hold the pages of random lengths, the others in the ring."""
    lens = rng.integers(0, longest + 1, B)
    perm, at = rng.permutation(N), 0
    tables = np.full((B, M), -1)
    for b in range(B):
        n = -(-lens[b] // P)
        if n > M or at + n > N:
            lens[b] = n = 0
        tables[b, :n] = perm[at:at + n]
        at += n
    head = int(rng.integers(0, N))
    ring = np.full(N, -7)
    ring[(head + np.arange(N - at)) % N] = perm[at:]
    return lens, tables, ring, np.array([head, N - at])


def _check(kvx, lens, add, tables, ring, free, T, P, out=None):
    g_tables, g_ring = _t(tables), _t(ring)
    got = kvx.plan_pages(_t(lens), _t(add), g_tables, g_ring, _t(free), T, P, out=out)
    want = S.plan_pages(lens, add, tables, ring, free, T, P)     # updates tables and ring
    for name, g, w in zip(got._fields, got, want):
        assert np.array_equal(g.cpu().numpy(), w), name
    assert np.array_equal(g_tables.cpu().numpy(), tables), "block_tables"
    assert np.array_equal(g_ring.cpu().numpy(), ring), "free_ring"
    return got


@pytest.mark.parametrize("B,N,P,M,longest,most,T", [
    (1, 1, 16, 1, 16, 1, 1),              # one page, full
    (1, 400, 16, 400, 5000, 900, 1024),
    (7, 64, 16, 12, 190, 40, 131),        # rows, tables and pages all run out
    (16, 3000, 128, 40, 5000, 1, 16),     # a decoding step
    (255, 9000, 32, 40, 1200, 70, 20000),
    (257, 4000, 16, 30, 400, 90, 9001),
    (1000, 40000, 16, 64, 1000, 50, 30000),
    (4096, 70000, 16, 16, 250, 3, 7000),
])
def test_plan_matches_the_definition(gpu_kvx, B, N, P, M, longest, most, T):
    rng = np.random.default_rng(B + N)
    for n in range(3):
        log(f"[case] plan B={B} N={N} P={P} M={M} T={T} draw {n}")
        lens, tables, ring, free = _state(rng, B, N, P, M, longest)
        add = np.where(rng.random(B) < 0.8, rng.integers(0, most + 1, B), -rng.integers(1, 9, B))
        _check(gpu_kvx, lens, add, tables, ring, free, T, P)


def test_plan_step_by_step(gpu_kvx):
    """Lengths, tables and ring carried from plan to plan, ends and refusals among them."""
    rng = np.random.default_rng(3)
    B, N, P, M = 33, 300, 16, 20
    lens, tables, ring, free = np.zeros(B, int), np.full((B, M), -1), rng.permutation(N), np.array([7, N])
    for step in range(20):
        add = np.where(rng.random(B) < 0.1, -1, rng.integers(0, 40, B) * (rng.random(B) < 0.7))
        log(f"[case] plan step {step}")
        got = _check(gpu_kvx, lens, add, tables, ring, free, 700, P)
        lens, free = got.lens.cpu().numpy(), got.free.cpu().numpy()


def test_plan_of_nothing(gpu_kvx):
    rng = np.random.default_rng(4)
    ring = rng.permutation(5)
    z = np.zeros(0, int)
    _check(gpu_kvx, z, z, np.zeros((0, 3), int), ring, np.array([2, 5]), 6, 16)          # no request
    lens, tables, ring, free = _state(rng, 5, 60, 16, 9, 140)
    _check(gpu_kvx, lens, np.array([0, -1, 0, -1, 0]), tables, ring, free, 0, 16)         # no row
    lens, tables, ring, free = _state(rng, 3, 60, 16, 9, 140)
    lens[1] = -5                                                                          # holds nothing
    tables[1] = -1
    _check(gpu_kvx, lens, np.array([3, 4, 5]), tables, ring, free, 12, 16)


def test_plan_refuses_lengths_that_overflow(gpu_kvx):
    """Lengths and additions near 2^31: refused, and nothing is read or written for them."""
    big = 2 ** 31 - 1
    lens, add = np.array([3, big, 5, 7]), np.array([2, big, big, 1])
    tables, ring = np.array([[0, -1], [-1, -1], [1, -1], [2, -1]]), np.array([3, 4, 5, -1, -1, -1])
    g_tables, g_ring = _t(tables), _t(ring)
    got = gpu_kvx.plan_pages(_t(lens), _t(add), g_tables, g_ring, _t([0, 3]), 8, 16)
    assert got.lens.tolist() == [5, big, 5, 7]
    assert got.cu.tolist() == [0, 2, 8, 8, 8]
    assert got.slots.tolist() == [3, 4] + [-1] * 6
    assert got.free.tolist() == [0, 3, 3, 8]
    assert np.array_equal(g_tables.cpu().numpy(), tables) and np.array_equal(g_ring.cpu().numpy(), ring)


def test_plan_page_ids_outside_the_pool_give_no_slot(gpu_kvx):
    got = gpu_kvx.plan_pages(_t([17]), _t([20]), _t([[0, -1, -1, -1]]), _t([9, 2, 1, 0]), _t([0, 2]), 20, 16)
    want = [-1] * 15 + [-1] * 5            # table entry 1 is -1, the ring's first page 9 of 4
    assert got.slots.tolist() == want and got.lens.tolist() == [37]


def test_plan_on_another_stream_and_in_a_graph(gpu_kvx):
    rng = np.random.default_rng(5)
    lens, tables, ring, free = _state(rng, 40, 900, 16, 30, 300)
    add = rng.integers(0, 30, 40)
    side = torch.cuda.Stream(device=DEV)
    a = [_t(x) for x in (lens, add, tables, ring, free)]
    torch.cuda.synchronize()
    out = gpu_kvx.plan_pages(*a, 700, 16, stream=side)
    want = S.plan_pages(lens, add, tables, ring, free, 700, 16)
    side.synchronize()
    for g, w in zip(out, want):
        assert np.array_equal(g.cpu().numpy(), w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = gpu_kvx.plan_pages(*a, 700, 16, out=out)
    for n in range(3):
        new = rng.integers(0, 30, 40)
        a[1].copy_(_t(new))
        graph.replay()
        torch.cuda.synchronize()
        want = S.plan_pages(lens, new, tables.copy(), ring.copy(), free, 700, 16)
        for g, w in zip(out, want):
            assert np.array_equal(g.cpu().numpy(), w), n
