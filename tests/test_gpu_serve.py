"""The serving example's turns and steps on the GPU against the definitions in 64 bits:
handed-over turns, steps of ragged rows, a conversation that ends and one that begins in
its place, and a captured step replayed.

The pool is compared code for code and scale for scale with the store's definition on the
rows that went in (the mapped rows themselves against the map's definition, by the map's own
tolerance), the plan entry for entry.  Attention: the element bounds that
test_gpu_attend8 derives.
"""

import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import kvx_oracle as O
from oracle import serve_oracle as S
from paper_2608_03893_amd import synth
from tests._parity import TOL, np32

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_mapped.py")
_SPEC = importlib.util.spec_from_file_location("serve_mapped", _PATH)
example = importlib.util.module_from_spec(_SPEC)
_SPEC.loader.exec_module(example)

B, G, P, N, M = 3, 2, 16, 14, 8


class Mirror:
    """The same state by the definitions."""

    def __init__(self, cfg):
        self.cfg = cfg
        self.codes = np.zeros((cfg.L_t, 2, cfg.H, N * P, cfg.d), np.uint8)
        self.scales = np.ones((cfg.L_t, 2, cfg.H, N))
        self.tables, self.ring = np.zeros((B, M), np.int64), np.arange(N)
        self.lens, self.free = np.zeros(B, np.int64), np.array([0, N, 0, 0])

    def plan(self, add, T, p):
        want = S.plan_pages(self.lens, add, self.tables, self.ring, self.free, T, P)
        for name, w in zip(p._fields, want):
            assert np.array_equal(getattr(p, name).cpu().numpy(), w), name
        self.lens, self.cu, _, self.slots, self.free = want

    def pool(self, server):
        assert np.array_equal(server.pool.view(torch.uint8).cpu().numpy(), self.codes)
        assert np.array_equal(server.scales.cpu().numpy(), self.scales)
        assert np.array_equal(server.tables.cpu().numpy(), self.tables)
        assert np.array_equal(server.ring.cpu().numpy(), self.ring)

    def step(self, server, p, add, q, k, v, out):
        cfg = self.cfg
        self.plan(add, q.shape[1], p)
        S.store_cache8(np32(k).transpose(0, 2, 1, 3).astype(np.float64),
                       np32(v).transpose(0, 2, 1, 3).astype(np.float64), self.slots, self.codes, self.scales)
        self.pool(server)
        u, n = 2.0 ** -24, max(int(self.lens.max()), 1)
        for l in range(cfg.L_t):
            want, _, A, size = S.attend_cache8(np32(q[l]).astype(np.float64), self.codes[l], self.scales[l],
                                               self.tables, self.lens, self.cu, cfg.d ** -0.5)
            got, seen = np32(out[l]).astype(np.float64), ~np.isnan(want)
            E = ((2 * (cfg.d + 8) * size + 2 * n + 64) * u)[..., None]
            tiny = n * 2.0 ** -126 * 448 * self.scales.max()
            bound = E * A + tiny if cfg.dtype == "f32" else \
                (E + 2.0 ** -8 * 1.01) * A + 2.0 ** -8 * np.abs(want) + tiny
            assert (np.abs(got - want) <= bound)[seen].all(), l


@pytest.mark.parametrize("name", ["tiny", "qwen3_14b_32b"])
def test_conversations(gpu_kvx, name):
    cfg = synth.CONFIGS[name]
    cfg = cfg.replace(L_s=4, L_t=3 if cfg.d == 128 else 6, k=2, H=2, T=71)
    inp = synth.make_inputs(cfg, DEV)
    server, mirror = example.Server(inp, B, G, N, M, P), Mirror(cfg)
    gen = torch.Generator(DEV).manual_seed(7)

    def hand_over(src, add):
        p, rows = server.hand_over(src, torch.tensor(add, dtype=torch.int32, device=DEV))
        mirror.plan(add, src.shape[3], p)
        want = O.map_cache(np32(src), inp["idx"], np32(inp["W_K"]), np32(inp["W_V"]), np32(inp["b_K"]),
                           np32(inp["b_V"]), inp["rope_src"], inp["rope_tgt"], p.positions.cpu().numpy())
        got = np32(rows).astype(np.float64)
        for l, kv, h in np.ndindex(*want.shape[:3]):
            w = want[l, kv, h]
            assert np.linalg.norm(got[l, kv, h] - w) <= TOL[cfg.dtype] * np.linalg.norm(w)
        S.store_cache8(got[:, 0], got[:, 1], mirror.slots, mirror.codes, mirror.scales)
        mirror.pool(server)

    def decode(add):
        T = sum(max(a, 0) for a in add)
        q, k, v = example.tokens(cfg, T, G, DEV, gen)
        p, out = server.decode(torch.tensor(add, dtype=torch.int32, device=DEV), q, k, v)
        mirror.step(server, p, add, q, k, v, out)

    hand_over(inp["src"], [50, 0, 21])        # two conversations' first turns
    decode([1, 1, 1])                         # the third starts with a token of its own
    decode([5, 1, 17])                        # drafted tokens, a page's end inside them
    hand_over(inp["src"][:, :, :, :33].contiguous(), [3, -1, 30])     # the second one ends
    decode([1, 40, 1])                        # and another begins in its place
    # a captured step, replayed with the program's own work between
    q, k, v = example.tokens(cfg, B, G, DEV, gen)
    one = torch.ones(B, dtype=torch.int32, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p, out = server.decode(one, q, k, v)
    for _ in range(3):
        for t, x in zip((q, k, v), example.tokens(cfg, B, G, DEV, gen)):
            t.copy_(x)
        g.replay()
        torch.cuda.synchronize()
        mirror.step(server, p, [1, 1, 1], q, k, v, out)
    assert mirror.free[2] == 0
    decode([1, 100, 1])                       # too many pages: refused, the others go on
    assert mirror.free[2] == 1
