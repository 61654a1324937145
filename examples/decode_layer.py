"""Decode steps of one decoder layer's attention block on one shard.

    python examples/decode_layer.py --model 8b --batch 64 --context 2048 --steps 50 [--budget 1024] [--fp8 | --int8]
        [--window 1024 --sinks 4] [--norm]

A prompt's tokens go through the same in chunks: the qkv projection, the entry
into the cache, the attention of all of them (KVCache.attend_prompt) and the o
projection.

A step is what a serving engine runs for each new token of a batch in which
every request names its own adapter: the qkv projection (Pool.forward_shard),
the rotary embedding and entry into the cache (KVCache.append), attention over
the cache (KVCache.attend) and the o projection, whose output is the shard's
partial of the tensor-parallel sum.  With a budget the steps keep account of
the attention that every entry gets and evict what got least (a prompt's
entries begin with none: its own attention adds no weights).  With a window they
attend to the last entries and the first few (sinks).  The step is
captured once into a HIP graph and replayed.  Weights, adapters and
activations are random, the shapes those of the Llama models.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2510_23346_amd as bd  # noqa: E402
from workloads import MODELS, model_projs  # noqa: E402

NAMES = {"1b": "llama-3.2-1b", "8b": "llama-3.1-8b", "70b": "llama-3.1-70b"}


class AttentionBlock:
    """The attention block of one layer on one shard, with its cache.

    ``projs``: the qkv projection (slices q, k, v) and the o projection;
    ``room``: the most entries a sequence may hold (before an eviction)."""

    def __init__(self, projs, head_dim, batch, room, *, page_size=64, slots=4, rank=16, budget=0, recent=0, fp8=False,
                 int8=False, window=0, sinks=0, norm=False, theta=500000.0, positions=16384, seed=0):
        self.qkv, self.o = projs
        self.batch, self.budget, self.recent = batch, budget, recent
        self.window, self.sinks = window, sinks
        hq, hkv = self.qkv.slices[0] // head_dim, self.qkv.slices[1] // head_dim
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda shape, std: (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)  # noqa: E731
        # the projections: base weights packed once, adapters in the pool
        self.w = [rand((p.d_out, p.d_in), p.d_in ** -0.5) for p in projs]
        self.packed = [bd.pack_weight(w) for w in self.w]
        self.pool = bd.Pool(projs, slots, rank, max(batch, 1024))
        self.adapters = []
        for s in range(slots):
            A = [[rand((p.d_in, rank), p.d_in ** -0.5) for _ in p.slices] for p in projs]
            B = [[rand((rank, n), rank ** -0.5) for n in p.slices] for p in projs]
            bits = lambda t: t.view(torch.int16).cpu().numpy().view(np.uint16)  # noqa: E731
            self.pool.load_adapter(s, rank, 2.0, [[bits(x) for x in a] for a in A], [[bits(x) for x in b] for b in B])
            self.adapters.append((A, B))
        self.ids = torch.arange(batch, dtype=torch.int32, device="cuda") % slots
        # the cache and the sequences' pages (in any order; here shuffled)
        width = -(-room // page_size)
        scale = {"k_scale": 0.02, "v_scale": 0.02} if fp8 else {}
        self.cache = bd.KVCache(hq, hkv, head_dim, batch * width, page_size, batch, weights=budget > 0,
                                fmt=bd.KV_INT8 if int8 else bd.KV_FP8_E4M3 if fp8 else bd.KV_BF16, **scale)
        # weights of the heads' norms, where the model has them
        self.norms = {}
        if norm:
            self.norms = {k: (1 + rand((head_dim,), 0.1).float()).to(torch.bfloat16) for k in ("q_norm", "k_norm")}
        self.table = torch.randperm(batch * width, generator=g, device="cuda").to(torch.int32).view(batch, width)
        f = theta ** (-torch.arange(0, head_dim, 2, device="cuda", dtype=torch.float64) / head_dim)
        angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * f
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        # state of the batch, on the device: a captured step reads and updates it
        i32 = lambda: torch.zeros(batch, dtype=torch.int32, device="cuda")  # noqa: E731
        self.lens, self.index, self.positions, self.starts = i32(), i32(), i32(), i32()
        self.seqs = torch.arange(batch, dtype=torch.int32, device="cuda")
        self.x = rand((batch, self.qkv.d_in), 1.0)
        self.qkv_out = rand((batch, self.qkv.d_out), 0.0)
        self.q = self.qkv_out[:, :self.qkv.slices[0]]          # rotated in place
        self.attn = rand((batch, self.o.d_in), 0.0)
        self.out = rand((batch, self.o.d_out), 0.0)

    def prompt(self, seq, x, slot, start=0):
        """A prompt's tokens ``start`` on (``x``: their activations [n, d_in]):
        their entry into the cache, their attention to it and the o projection's
        partial [n, d_out], which is returned."""
        n = x.shape[0]
        rows = lambda p: torch.empty((n, p.d_out), dtype=torch.bfloat16, device="cuda")  # noqa: E731
        qkv, out = rows(self.qkv), rows(self.o)
        q = qkv[:, :self.qkv.slices[0]]
        at = torch.arange(start, start + n, dtype=torch.int32, device="cuda")
        segs = bd.Segments([0], [n], [slot])
        self.pool.forward_shard(0, x, self.packed[0], None, qkv, segs=segs)
        self.cache.append(qkv, self.cos, self.sin, torch.full_like(at, seq), at, at, self.table, self.lens, q, **self.norms)
        attn = torch.empty((n, self.o.d_in), dtype=torch.bfloat16, device="cuda")
        self.cache.attend_prompt(q, torch.tensor([0, n], dtype=torch.int32, device="cuda"), self.table[seq:seq + 1],
                                 self.lens[seq:seq + 1], attn, window=self.window, sinks=self.sinks)
        self.pool.forward_shard(1, attn, self.packed[1], None, out, segs=segs)
        return out

    def begin(self):
        """After the prompts: where the next token of each sequence goes."""
        self.index.copy_(self.lens)
        self.positions.copy_(self.lens)

    def step(self):
        self.pool.forward_shard(0, self.x, self.packed[0], self.ids, self.qkv_out)
        self.cache.append(self.qkv_out, self.cos, self.sin, self.seqs, self.index, self.positions, self.table, self.lens,
                          self.q, **self.norms)
        if self.window:
            torch.sub(self.lens, self.window, out=self.starts)          # (below zero: from the first on)
        self.cache.attend(self.q, self.table, self.lens, self.attn, starts=self.starts if self.window else None,
                          sinks=self.sinks, accumulate=self.budget > 0)
        self.pool.forward_shard(1, self.attn, self.packed[1], self.ids, self.out)
        if self.budget:
            self.cache.evict(self.table, self.lens, self.budget, self.recent)
        self.index.copy_(self.lens)
        self.positions.add_(1)

    def close(self):
        self.cache.close()
        self.pool.close()


def shard_projs(model, tp):
    """(qkv and o projections, head size) of a model's shard."""
    m = MODELS[NAMES[model]]
    by = {p.name: p for p in model_projs(NAMES[model], tp)}
    return [by["qkv"], by["o"]], m.head_dim


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--model", choices=sorted(NAMES), default="8b")
    ap.add_argument("--tp", type=int, default=8)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--context", type=int, default=2048, help="prompt tokens of every sequence")
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--page-size", type=int, default=64)
    ap.add_argument("--budget", type=int, default=0, help="entries to keep per sequence and kv head (0: all)")
    ap.add_argument("--recent", type=int, default=64)
    ap.add_argument("--fp8", action="store_true", help="8-bit cache (e4m3, one scale)")
    ap.add_argument("--int8", action="store_true", help="8-bit cache (a scale for each 16 entries of a head; no budget)")
    ap.add_argument("--window", type=int, default=0, help="entries that are attended to (0: all)")
    ap.add_argument("--sinks", type=int, default=0, help="first entries that stay visible beside the window")
    ap.add_argument("--norm", action="store_true", help="norms of the query and key heads")
    a = ap.parse_args()
    projs, d = shard_projs(a.model, a.tp)
    block = AttentionBlock(projs, d, a.batch, a.context + a.steps + 8, page_size=a.page_size, budget=a.budget,
                           recent=min(a.recent, a.budget), fp8=a.fp8, int8=a.int8, window=a.window,
                           sinks=a.sinks, norm=a.norm, positions=a.context + a.steps + 8)
    g = torch.Generator(device="cuda").manual_seed(1)
    for s in range(a.batch):
        for at in range(0, a.context, 1024):        # the pool takes 1024 tokens a call: longer prompts in chunks
            n = min(1024, a.context - at)
            block.prompt(s, torch.randn((n, projs[0].d_in), generator=g, device="cuda").to(torch.bfloat16), s % 4, at)
    block.begin()
    block.step()                            # warm up, then capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.step()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        graph.replay()
    torch.cuda.synchronize()
    us = (time.perf_counter() - t) / a.steps * 1e6
    if block.cache.device_error() or block.pool.device_error():
        raise SystemExit("a device error was raised")
    print(f"{a.model} attention block, 1/{a.tp} shard: {a.batch} sequences at {a.context}+ entries: {us:.1f} us a step; "
          f"entries now {int(block.lens.min())}..{int(block.lens.max())}")
    block.close()


if __name__ == "__main__":
    main()
