"""The shared-context example's steps on the GPU against the definitions in 64 bits, every operator
on what went into it: plan entry for entry, normed and rotated rows, pool code for code, attention
over the common and the own keys, the tokens drawn; eager, captured and replayed."""

import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from paper_2608_03893_amd import synth
from tests._parity import np32
from tests.test_gpu_norm_rope import _check as check_rows

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "continue_shared.py")
_SPEC = importlib.util.spec_from_file_location("continue_shared", _PATH)
example = importlib.util.module_from_spec(_SPEC)
_SPEC.loader.exec_module(example)

B, G, P, N, M, V = 5, 2, 16, 40, 12, 1003


class Mirror:
    """The same state by the definitions."""

    def __init__(self, cfg):
        self.cfg = cfg
        self.codes = np.zeros((cfg.L_t, 2, cfg.H, N * P, cfg.d), np.uint8)
        self.scales = np.ones((cfg.L_t, 2, cfg.H, N))
        self.ctables, self.tables, self.ring = np.zeros((1, M), np.int64), np.zeros((B, M), np.int64), np.arange(N)
        self.clens, self.lens, self.free = np.zeros(1, np.int64), np.zeros(B, np.int64), np.array([0, N, 0, 0])

    def plan(self, p, lens, add, tables, T):
        want = S.plan_pages(lens, add, tables, self.ring, self.free, T, P)
        for name, w in zip(p._fields, want):
            assert np.array_equal(getattr(p, name).cpu().numpy(), w), name
        self.free = want[4]
        return want

    def pool(self, c):
        assert np.array_equal(c.pool.view(torch.uint8).cpu().numpy(), self.codes)
        assert np.array_equal(c.scales.cpu().numpy(), self.scales)
        assert np.array_equal(c.context["tables"].cpu().numpy(), self.ctables)
        assert np.array_equal(c.tables.cpu().numpy(), self.tables)

    def hand_over(self, c, p, rows):
        T = rows.shape[3]
        self.clens, _, _, slots, _ = self.plan(p, self.clens, [T], self.ctables, T)
        x = np32(rows).astype(np.float64)
        S.store_cache8(x[:, 0], x[:, 1], slots, self.codes, self.scales)
        self.pool(c)

    def step(self, c, done, u):
        cfg, heads = self.cfg, self.cfg.H * G
        self.lens, cu, pos, slots, _ = self.plan(done.plan, self.lens, [1] * B, self.tables, B)
        assert np.array_equal(done.positions.cpu().numpy(), pos + self.clens[0])
        eps, n = 2.0 ** -24, int(self.clens[0] + self.lens.max())
        for l in range(cfg.L_t):
            rows = done.rows[l]
            check_rows(done.q[l], rows[:, :heads], c.norms[l][0], 1e-6, done.positions, c.inp["rope_tgt"], cfg.dtype)
            check_rows(done.k[l], rows[:, heads:heads + cfg.H], c.norms[l][1], 1e-6, done.positions, c.inp["rope_tgt"], cfg.dtype)
            k, v = (np32(x).astype(np.float64).transpose(1, 0, 2)[None] for x in (done.k[l], rows[:, heads + cfg.H:]))
            S.store_cache8(k, v, slots, self.codes[l:l + 1], self.scales[l:l + 1])
            want, _, A, size = S.attend_prefix8(np32(done.q[l]).astype(np.float64), self.codes[l], self.scales[l], self.ctables,
                                                self.clens, [0, B], self.tables, self.lens, cu, cfg.d ** -0.5)
            got = np32(done.out[l]).astype(np.float64)
            E = ((2 * (cfg.d + 9) * size + 2 * n + 80) * eps)[..., None]        # test_gpu_prefix8 derives it
            tiny = n * 2.0 ** -126 * 448 * self.scales.max()
            bound = E * A + tiny
            if cfg.dtype == "bf16":
                bound = bound + 1.01 * 2.0 ** -16 * A
                bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
            assert (np.abs(got - want) <= bound).all(), l
        self.pool(c)
        logits, r = np32(done.logits).astype(np.float64), np.float32
        for b in range(B):
            token, lp, near = S.sample_token(logits[b], r(u[b]), *(float(c.settings[x][b]) if x != "top_k" else int(c.settings[x][b])
                                                                   for x in ("temperature", "top_k", "top_p", "min_p")))
            if near > V * (2.0 ** -44 + 2.0 ** -52):
                assert int(done.tokens[b]) == token
                assert abs(float(done.logprob[b]) - lp) <= V * 2.0 ** -44 + 2.0 ** -40 + 2.0 ** -24 * abs(lp) * 1.01
        assert torch.equal(c.tokens, done.tokens)


@pytest.mark.parametrize("name", ["tiny", "qwen3_14b_32b"])
def test_continuations(gpu_kvx, name):
    cfg = synth.CONFIGS[name]
    cfg = cfg.replace(L_s=4, L_t=2 if cfg.d == 128 else 3, k=2, H=2, T=83)
    inp = synth.make_inputs(cfg, DEV)
    c, m = example.Continuations(inp, B, G, V, N, M, P), Mirror(cfg)
    for x, values in (("temperature", [0.0, 0.7, 1.0, 1.3, 2.0]), ("top_p", [0.9, 0.9, 0.95, 1.0, 0.99]),
                      ("min_p", [0.0, 0.0, 0.0, 0.05, 0.0])):
        c.settings[x].copy_(torch.tensor(values))
    c.settings["top_k"].copy_(torch.tensor([5, 50, 0, 0, 300]))
    m.hand_over(c, *c.hand_over(inp["src"]))
    for _ in range(3):
        u = c.u.tolist()
        m.step(c, c.step(), u)
        c.u.copy_(torch.rand(B, device=DEV, generator=c.gen))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        done = c.step()
    for _ in range(18):                       # past a page's end
        c.u.copy_(torch.rand(B, device=DEV, generator=c.gen))
        u = c.u.tolist()
        g.replay()
        torch.cuda.synchronize()
        m.step(c, done, u)
    assert m.free[2] == 0
