"""Timing of the arbitrator's attention for one round (Sec. 3.3).

The arbitrator LM reads q = [c, SEP, draft block, SEP, target block, SEP]
with a hybrid mask: the context is causal (and, decoding round after round,
already cached), the 2K+3 region tokens see the whole context and each other.
So each of its layers, per round, is one ``cospec_verify_attn`` call with the
region as a full-mask block (COSPEC_ATTN_BLOCK_FULL) over the paged context.
This module times those L calls, replayed from a CUDA graph, on synthetic
inputs shaped like the paper's draft/arbitrator backbones.

  python -m paper_2605_24793_gb300.arbitrator --k 25 --batch 1 --context 4096

The arbitrator is the draft's backbone with low-rank adapters (rank 16, scale 32), so its projections are the
backbone's with a second product beside them: ``RegionLayer`` runs a layer's attention block of that kind for rows of
several sequences, each with its own adapter or none (a drafting row), over an 8-bit cache, and
``--adapters`` times it.

  python -m paper_2605_24793_gb300.arbitrator --adapters 4 --batch 16 --k 25
"""
from __future__ import annotations

import argparse
import json

import numpy as np
import torch

from . import cospec as C
from . import workload as W

# Qwen3-4B-like backbone (the paper's draft for Qwen3-32B): 36 layers, 32 query /
# 8 KV heads, head_dim 128; the vocabulary plays no part here.
BACKBONE = dict(layers=36, hidden=2560, q_heads=32, kv_heads=8, head_dim=128)


def region_config(k: int, batch: int, context: int, layers: int) -> W.RoundConfig:
    """A workload whose block is the arbitrator's region: 2K+3 rows."""
    bb = dict(BACKBONE)
    bb["layers"] = layers
    return W.RoundConfig(f"arbitrator_k{k}_b{batch}_c{context}", 5, batch=batch, ctx_lo=context,
                         ctx_hi=context, k=2 * k + 2, vocab=1024, mlp_hidden=64, mismatch_rate=0.3,
                         mismatch_topk=8, shuffled_pages=batch > 1, **bb)


def time_region_attention(cfg: W.RoundConfig, steps: int = 50, warmup: int = 5) -> dict:
    inp = W.make_round_inputs(cfg, device="cuda")
    q, kb, vb = inp["q"], inp["k_blk"], inp["v_blk"]
    kp, vp = inp["k_pages"], inp["v_pages"]
    out = torch.empty_like(q[0])
    max_ctx = int(np.max(inp["ctx_len_np"]))

    def layers():
        for l in range(cfg.layers):
            pl = 0 if kp.shape[0] == 1 else l
            C.verify_attn(q[l], kb[l], vb[l], kp[pl], vp[pl], inp["page_table"], inp["ctx_len"], out,
                          max_ctx, kv_stable=l > 0, block_full=True)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        layers()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        layers()
    for _ in range(warmup):
        g.replay()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    e0.record(s)
    with torch.cuda.stream(s):
        for _ in range(steps):
            g.replay()
    e1.record(s)
    e1.synchronize()
    us = e0.elapsed_time(e1) * 1e3 / (steps * cfg.layers)
    ctx = inp["ctx_len_np"].astype(np.int64)
    kv_bytes = float(ctx.sum()) * 2 * cfg.kv_heads * cfg.head_dim * 2
    blk_bytes = 2.0 * cfg.batch * cfg.rows * (cfg.kv_heads + cfg.q_heads) * cfg.head_dim * 2
    kernel, splits = C.verify_attn_plan(q[0], kp[0], inp["page_table"], max_ctx)
    return {"workload": cfg.name, "region_rows": cfg.rows, "batch": cfg.batch,
            "context": int(ctx.max()), "layers": cfg.layers, "us_per_layer": us,
            "gbs": (kv_bytes + blk_bytes) / (us * 1e-6) / 1e9,
            "kernel": C.ATTN_KERNEL_NAMES[kernel], "splits": splits,
            "device_error": C.get_device_error()}


class RegionLayer:
    """The attention block of one arbitrator layer for a region's rows [B, R, hidden]: query / key / value projection with adapters
    into one buffer, rotation to the positions behind the cached context, attention of the region (bidirectional
    inside) over the 8-bit cache, output projection with adapters.  Weights and adapters are drawn from ``seed``."""

    def __init__(self, pool: C.Kv8Pool, rope: C.Rope, page_table, ctx_len, rows: int, hidden: int, q_heads: int, adapters: int,
                 rank: int = 16, scale: float = 32.0, max_ctx: int = None, layer: int = 0, seed: int = 0, device="cuda"):
        B, D, hkv = ctx_len.shape[0], pool.head_dim, pool.kv_heads
        self.pool, self.rope, self.page_table, self.ctx_len, self.layer = pool, rope, page_table, ctx_len, layer
        self.max_ctx = int(ctx_len.max()) if max_ctx is None else int(max_ctx)
        self.shape, self.heads = (B, rows), (q_heads, hkv, D)
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        new = lambda *s, std: torch.empty(s, dtype=torch.bfloat16, device=device).normal_(0.0, std, generator=g)  # noqa: E731
        wide = (q_heads + 2 * hkv) * D
        self.w_qkv, self.w_out = new(wide, hidden, std=hidden ** -0.5), new(hidden, q_heads * D, std=(q_heads * D) ** -0.5)
        self.a_qkv, self.b_qkv = new(adapters, rank, hidden, std=hidden ** -0.5), new(adapters, wide, rank, std=0.02)
        self.a_out, self.b_out = new(adapters, rank, q_heads * D, std=(q_heads * D) ** -0.5), new(adapters, hidden, rank, std=0.02)
        self.scaling = torch.full((adapters,), scale / rank, device=device)
        empty = lambda *s, dt=torch.bfloat16: torch.empty(s, dtype=dt, device=device)  # noqa: E731
        self.qkv = empty(B, rows, q_heads + 2 * hkv, D)
        self.q, self.k, self.v = self.qkv[:, :, :q_heads], self.qkv[:, :, q_heads:q_heads + hkv], self.qkv[:, :, q_heads + hkv:]
        self.q_rot, self.k_rot, self.attn = empty(B, rows, q_heads, D), empty(B, rows, hkv, D), empty(B, rows, q_heads, D)
        self.u_qkv, self.u_out = (empty(B * rows, rank, dt=torch.float32) for _ in range(2))
        self.out = empty(B, rows, hidden)

    def run(self, x: torch.Tensor, adapter: torch.Tensor) -> torch.Tensor:
        """x bf16 [B, R, hidden], adapter int32 [B * R] (-1: none).  Returns [B, R, hidden]; nothing synchronises with the host."""
        n = self.shape[0] * self.shape[1]
        C.lora_forward(x.view(n, -1), self.w_qkv, self.a_qkv, self.b_qkv, self.scaling, adapter, self.qkv.view(n, -1), self.u_qkv)
        C.kv8_rotate(self.q, self.k, self.rope, self.ctx_len, self.q_rot, self.k_rot)
        C.kv8_attn(self.q_rot, self.k_rot, self.v, self.pool, self.layer, self.page_table, self.ctx_len, self.attn, self.max_ctx, block_full=True)
        C.lora_forward(self.attn.view(n, -1), self.w_out, self.a_out, self.b_out, self.scaling, adapter, self.out.view(n, -1), self.u_out)
        return self.out


def time_region_layer(k: int, batch: int, context: int, adapters: int, steps: int = 50, layers: int = 8) -> dict:
    """Microseconds a layer of ``layers`` captured layers, each with weights and a cache of its own."""
    from .kv8round import quantise_cache, rope_tables
    cfg = region_config(k, batch, context, 1)
    inp = W.make_round_inputs(cfg, device="cuda")
    pool = quantise_cache(inp["k_pages"], inp["v_pages"], inp["page_table"], inp["ctx_len"])
    rope = rope_tables(inp["page_table"].shape[1] * 16, cfg.head_dim)
    blocks = [RegionLayer(pool, rope, inp["page_table"], inp["ctx_len"], cfg.rows, cfg.hidden, cfg.q_heads, adapters, seed=l) for l in range(layers)]
    x = torch.randn((batch, cfg.rows, cfg.hidden), device="cuda").to(torch.bfloat16)
    adapter = (torch.arange(batch, device="cuda", dtype=torch.int32) % adapters).repeat_interleave(cfg.rows)

    def run():
        for b in blocks:
            b.run(x, adapter)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        run()
    for _ in range(3):
        g.replay()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(steps):
        g.replay()
    e1.record()
    e1.synchronize()
    return {"workload": cfg.name, "rows": batch * cfg.rows, "adapters": adapters, "us_per_layer": e0.elapsed_time(e1) * 1e3 / (steps * layers),
            "what": "projection, rotation, region attention over the 8-bit cache, projection", "device_error": C.get_device_error()}


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--k", type=int, nargs="+", default=[7, 25])
    ap.add_argument("--batch", type=int, nargs="+", default=[1, 16])
    ap.add_argument("--context", type=int, default=4096)
    ap.add_argument("--layers", type=int, default=BACKBONE["layers"])
    ap.add_argument("--adapters", type=int, default=0, help="time a layer with its projections, this many adapters in the batch")
    args = ap.parse_args()
    from . import build as B
    C.load_library(B.build())
    for k in args.k:
        for b in args.batch:
            if args.adapters > 0:
                print(json.dumps(time_region_layer(k, b, args.context, args.adapters)), flush=True)
                torch.cuda.empty_cache()
                continue
            res = time_region_attention(region_config(k, b, args.context, args.layers))
            print(json.dumps(res), flush=True)
            torch.cuda.empty_cache()


if __name__ == "__main__":
    main()
