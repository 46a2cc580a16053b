#!/usr/bin/env python3
"""Many continuations of one context that another model has read.

The source model's cache of the context is mapped into the target model's cache and kept in 8
bits, once; B continuations of it are then sampled from the target model, whose layers read the
common pages together:

  hand_over   plan_pages -> map_cache -> store_cache8
  step        plan_pages -> for every layer: norm_rope of the new tokens' queries and keys,
              store_cache8, attend_prefix8 -> sample_tokens

The target model is a stack of attention layers with random weights of the workload's sizes, since
none are at hand.  A step is captured in a graph; lengths, free pages and the tokens drawn are
carried from step to step on the GPU.

    python examples/continue_shared.py [--workload NAME] [--continuations B] [--context T] [--steps K]
"""

from __future__ import annotations

import argparse
import os
import sys
from typing import NamedTuple

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_03893_amd import kvx, synth  # noqa: E402


class Step(NamedTuple):
    """What a step computed, layer by layer."""
    plan: kvx.PagePlan
    positions: torch.Tensor
    rows: list          # a layer's projection [B, H*G + 2*H, d]
    q: list             # normed and rotated
    k: list
    out: list
    logits: torch.Tensor
    tokens: torch.Tensor
    logprob: torch.Tensor


class Continuations:
    """B continuations of one context, with settings of their own."""

    def __init__(self, inp, B, G, vocabulary, num_pages, max_pages, page_size=16, temperature=0.8, top_k=50, top_p=0.95,
                 min_p=0.0, seed=0):
        cfg, dev = inp["cfg"], inp["src"].device
        self.inp, self.cfg, self.B, self.G, self.page_size = inp, cfg, B, G, page_size
        g = torch.Generator(dev).manual_seed(seed)
        dt, d, heads = cfg.torch_dtype, cfg.d, cfg.H * G
        rand = lambda *s: torch.randn(s, device=dev, generator=g)  # noqa: E731
        self.embed = rand(vocabulary, heads * d).to(dt)
        self.W_in = [(rand(heads * d, (heads + 2 * cfg.H) * d) * (heads * d) ** -0.5).to(dt) for _ in range(cfg.L_t)]
        self.W_out = [(rand(heads * d, heads * d) * (heads * d) ** -0.5).to(dt) for _ in range(cfg.L_t)]
        self.norms = [tuple(torch.exp(0.1 * rand(d)).to(dt) for _ in "qk") for _ in range(cfg.L_t)]
        self.pool = torch.zeros((cfg.L_t, 2, cfg.H, num_pages * page_size, d), dtype=torch.uint8,
                                device=dev).view(torch.float8_e4m3fn)
        self.scales = torch.ones((cfg.L_t, 2, cfg.H, num_pages), device=dev)
        i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
        self.ring, self.free = torch.arange(num_pages, dtype=torch.int32, device=dev), i32(0, num_pages, 0, 0)
        # the context's pages and length, which all continuations share, and their own
        self.context = dict(tables=torch.zeros((1, max_pages), dtype=torch.int32, device=dev), lens=i32(0), cu=i32(0, B))
        self.tables = torch.zeros((B, max_pages), dtype=torch.int32, device=dev)
        self.lens, self.one = i32(*[0] * B), i32(*[1] * B)
        self.tokens = torch.randint(0, vocabulary, (B,), device=dev, generator=g).to(torch.int32)
        f32 = lambda x: torch.full((B,), float(x), device=dev)  # noqa: E731
        self.settings = dict(temperature=f32(temperature), top_k=i32(*[top_k] * B), top_p=f32(top_p), min_p=f32(min_p))
        self.rope = kvx.make_rope(inp["rope_tgt"])
        self.u = torch.rand(B, device=dev, generator=g)       # the step's random numbers
        self.gen = g
        self.attention = kvx.prefix_workspace(torch.empty((B, heads, d), dtype=dt, device=dev), self.pool[0],
                                              self.context["tables"], self.tables)
        self.sampling = kvx.sample_workspace(torch.empty((B, vocabulary), dtype=dt, device=dev))

    def plan(self, lens, add, tables, T):
        p = kvx.plan_pages(lens, add, tables, self.ring, self.free, T, self.page_size)
        lens.copy_(p.lens)
        self.free.copy_(p.free)
        return p

    def hand_over(self, src):
        """Map the source model's rows src [L_s, 2, H, T, d] of the context and keep them."""
        i, T = self.inp, src.shape[3]
        add = torch.tensor([T], dtype=torch.int32, device=src.device)
        p = self.plan(self.context["lens"], add, self.context["tables"], T)
        rows = torch.empty((self.cfg.L_t, 2, self.cfg.H, T, self.cfg.d), dtype=src.dtype, device=src.device)
        kvx.map_cache(src, i["idx"], i["W_K"], i["W_V"], i["b_K"], i["b_V"], i["rope_src"], i["rope_tgt"], p.positions, rows)
        kvx.store_cache8(rows[:, 0], rows[:, 1], p.slots, self.pool, self.scales)
        return p, rows

    def step(self):
        """A token more for every continuation; the tokens drawn are the next step's."""
        cfg, B, heads = self.cfg, self.B, self.cfg.H * self.G
        p = self.plan(self.lens, self.one, self.tables, B)
        positions = p.positions + self.context["lens"]
        x = self.embed[self.tokens.long()]
        done = Step(p, positions, [], [], [], [], None, None, None)
        for l in range(cfg.L_t):
            rows = torch.matmul(x, self.W_in[l]).view(B, heads + 2 * cfg.H, cfg.d)
            q, k = kvx.norm_rope(rows[:, :heads], rows[:, heads:heads + cfg.H], *self.norms[l], self.rope, positions)
            v = rows[:, heads + cfg.H:]
            kvx.store_cache8(k[None].transpose(1, 2), v[None].transpose(1, 2), p.slots, self.pool[l:l + 1],
                             self.scales[l:l + 1])
            out = kvx.attend_prefix8(q, self.pool[l], self.scales[l], self.context["tables"], self.context["lens"],
                                     self.context["cu"], self.tables, p.lens, p.cu, workspace=self.attention)
            x = x + torch.matmul(out.view(B, heads * cfg.d), self.W_out[l])
            for to, what in zip((done.rows, done.q, done.k, done.out), (rows, q, k, out)):
                to.append(what)
        logits = torch.matmul(x, self.embed.t()) * x.shape[1] ** -0.5
        tokens, logprob = kvx.sample_tokens(logits, self.u, **self.settings, with_logprob=True, workspace=self.sampling)
        self.tokens.copy_(tokens)
        return done._replace(logits=logits, tokens=tokens, logprob=logprob)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="qwen3_0.6b_4b", choices=[n for n, c in synth.CONFIGS.items() if not c.sessions])
    ap.add_argument("--continuations", type=int, default=64)
    ap.add_argument("--context", type=int, default=4096)
    ap.add_argument("--group", type=int, default=4, help="query heads for each KV head")
    ap.add_argument("--vocabulary", type=int, default=131072)
    ap.add_argument("--steps", type=int, default=64)
    a = ap.parse_args()
    dev, B = torch.device("cuda:0"), a.continuations
    cfg = synth.CONFIGS[a.workload].replace(T=a.context)
    inp = synth.make_inputs(cfg, dev)
    own = -(-(2 * a.steps + 8) // 16)
    max_pages = max(-(-a.context // 16), own)
    c = Continuations(inp, B, a.group, a.vocabulary, -(-a.context // 16) + B * own, max_pages)
    c.hand_over(inp["src"])
    c.step()                                  # first calls: code and workspaces are loaded
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        done = c.step()
    sequences = []
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(a.steps):
        c.u.copy_(torch.rand(B, device=dev, generator=c.gen))
        g.replay()
        sequences.append(done.tokens.clone())
    end.record()
    end.synchronize()
    ms = begin.elapsed_time(end) / a.steps
    different = len({tuple(s) for s in torch.stack(sequences, 1).tolist()})
    print(f"{B} continuations of {a.context} common tokens, {cfg.L_t} layers: {ms:.3f} ms a step "
          f"({B / ms * 1e3:.0f} tokens/s); {different} different ones, lengths {min(c.lens.tolist())} .. "
          f"{max(c.lens.tolist())}, {c.free.tolist()[1]} of {len(c.ring)} pages free", flush=True)


if __name__ == "__main__":
    main()
