#!/usr/bin/env python3
"""Conversations handed from one model to another and continued there.

The source model's cache of each conversation's new turn is mapped into the target
model's cache (Sec. 3.3, the multi-turn handoff of Sec. 4.6), kept in 8 bits in pages of
a common pool, and read by the target model's queries:

  hand_over   plan_pages -> map_cache -> store_cache8
  decode      plan_pages -> for every layer: store_cache8 of the new tokens' keys and
              values, attend_cache8 of their queries

Queries, keys and values of the new tokens are random here, where a target model's layers
would compute them.  A decoding step of one token each is captured in a graph; the plan's
lengths and free pages are carried from step to step on the GPU, so that the host learns
nothing and waits for nothing in between.

    python examples/serve_mapped.py [--workload NAME] [--conversations B] [--turn T] [--steps K]
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_03893_amd import kvx, synth  # noqa: E402


class Server:
    """The target model's 8-bit cache of B conversations; steps of up to ``rows`` tokens."""

    def __init__(self, inp, B, G, num_pages, max_pages, page_size=16, rows=256):
        cfg, dev = inp["cfg"], inp["src"].device
        self.inp, self.cfg, self.G, self.page_size = inp, cfg, G, page_size
        self.pool = torch.zeros((cfg.L_t, 2, cfg.H, num_pages * page_size, cfg.d), dtype=torch.uint8,
                                device=dev).view(torch.float8_e4m3fn)
        self.scales = torch.ones((cfg.L_t, 2, cfg.H, num_pages), device=dev)
        self.tables = torch.zeros((B, max_pages), dtype=torch.int32, device=dev)
        self.ring = torch.arange(num_pages, dtype=torch.int32, device=dev)
        self.lens = torch.zeros(B, dtype=torch.int32, device=dev)
        self.free = torch.tensor([0, num_pages, 0, 0], dtype=torch.int32, device=dev)
        # one workspace for every attention call: the one of most rows suffices for fewer
        dims = kvx.AttendDims(B, cfg.H, G, rows, cfg.d)
        self.workspace = torch.zeros(kvx.attend_workspace_bytes(dims, cfg.dtype), dtype=torch.uint8, device=dev)

    def plan(self, add, T):
        """Pages and slots of T new tokens, add[b] of them conversation b's (-1: it ended).
        The lengths and the ring are copied in place, so that a captured step reads what
        the step before it left."""
        p = kvx.plan_pages(self.lens, add, self.tables, self.ring, self.free, T, self.page_size)
        self.lens.copy_(p.lens)
        self.free.copy_(p.free)
        return p

    def hand_over(self, src, add):
        """Map the source model's rows src [L_s, 2, H, T, d] of the conversations' new turns
        (packed in order) and keep them; returns the plan and the mapped rows."""
        i, T = self.inp, src.shape[3]
        p = self.plan(add, T)
        rows = torch.empty((self.cfg.L_t, 2, self.cfg.H, T, self.cfg.d), dtype=src.dtype, device=src.device)
        kvx.map_cache(src, i["idx"], i["W_K"], i["W_V"], i["b_K"], i["b_V"], i["rope_src"],
                      i["rope_tgt"], p.positions, rows)
        kvx.store_cache8(rows[:, 0], rows[:, 1], p.slots, self.pool, self.scales)
        return p, rows

    def decode(self, add, q, k, v):
        """New tokens of the target model itself: q [L_t, T, H * G, d], k, v [L_t, T, H, d]
        as its layers' projections leave them; returns the plan and out like q."""
        p = self.plan(add, q.shape[1])
        out = torch.empty_like(q)
        for l in range(self.cfg.L_t):
            kvx.store_cache8(k[l:l + 1].transpose(1, 2), v[l:l + 1].transpose(1, 2), p.slots,
                             self.pool[l:l + 1], self.scales[l:l + 1])
            kvx.attend_cache8(q[l], self.pool[l], self.scales[l], self.tables, p.lens, p.cu,
                              out=out[l], workspace=self.workspace)
        return p, out


def tokens(cfg, T, G, device, gen):
    """Random queries, keys and values of T new tokens."""
    dt = cfg.torch_dtype
    q = torch.randn((cfg.L_t, T, cfg.H * G, cfg.d), device=device, generator=gen).to(dt)
    k, v = (torch.randn((cfg.L_t, T, cfg.H, cfg.d), device=device, generator=gen).to(dt) for _ in "kv")
    return q, k, v


def timed(fn, n):
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(n):
        fn()
    b.record()
    b.synchronize()
    return a.elapsed_time(b) / n


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="qwen3_14b_32b",
                    choices=[n for n, c in synth.CONFIGS.items() if not c.sessions])
    ap.add_argument("--conversations", type=int, default=16)
    ap.add_argument("--turn", type=int, default=1024, help="tokens of each conversation's turn")
    ap.add_argument("--group", type=int, default=8, help="query heads for each KV head")
    ap.add_argument("--steps", type=int, default=64)
    a = ap.parse_args()
    dev, B = torch.device("cuda:0"), a.conversations
    cfg = synth.CONFIGS[a.workload].replace(T=B * a.turn)
    inp = synth.make_inputs(cfg, dev)
    max_pages = -(-(2 * a.turn + 4 * a.steps + 64) // 16)
    s = Server(inp, B, a.group, B * max_pages, max_pages)
    full = torch.full((B,), a.turn, dtype=torch.int32, device=dev)
    one = torch.ones(B, dtype=torch.int32, device=dev)
    gen = torch.Generator(dev).manual_seed(cfg.seed)
    q, k, v = tokens(cfg, B, a.group, dev, gen)

    s.hand_over(inp["src"], full)      # first calls: code and workspaces are loaded
    s.decode(one, q, k, v)
    ms = timed(lambda: s.hand_over(inp["src"], full), 1)
    print(f"{B} turns of {a.turn} tokens mapped and kept in 8 bits: {ms:.2f} ms, "
          f"{B * a.turn / ms * 1e3:.0f} tokens/s", flush=True)
    eager = timed(lambda: s.decode(one, q, k, v), a.steps)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.decode(one, q, k, v)
    g.replay()
    graph = timed(g.replay, a.steps)
    lens, left = s.lens.tolist(), s.free.tolist()
    print(f"decoding step of {B} tokens, {cfg.L_t} layers: {eager:.3f} ms, captured {graph:.3f} ms "
          f"({B / graph * 1e3:.0f} tokens/s); lengths {min(lens)} .. {max(lens)}, "
          f"{left[1]} of {len(s.ring)} pages free, {left[2]} refused", flush=True)


if __name__ == "__main__":
    main()
