"""A verify/arbitrate round over an 8-bit KV cache (App. F, Inference Procedure, with the cache
held as e4m3 codes): rotate the block's queries and keys to their positions, attend every
layer over the cache (or over the pages that a cheap score selects for each block row), LM
head, arbitration, accepted length, and the accepted rows of every layer appended to the cache,
rotated and quantised on the way.

The cache takes about half the bytes of the bf16 one.  A round is made from a bf16 cache, which it reads
once and keeps no reference to: the memory is free when the caller lets go of it.  Nothing in a round synchronises with the host; a round can be captured and replayed as ``VerifyRound``.

  python -m paper_2605_24793_gb300.kv8round --config qwen3_8b_b1
  python -m paper_2605_24793_gb300.kv8round --config qwen3_8b_b16 --layers 4 --pages 64
"""
from __future__ import annotations

import argparse
import json
from typing import Dict, Optional

import numpy as np
import torch

from . import cospec as C
from . import workload as W
from .round import VerifyRound

PAGE = 16


def rope_tables(positions: int, head_dim: int, base: float = 1e6, device="cuda") -> C.Rope:
    """The usual rotation tables: angle p * base^(-2 i / head_dim), pairs (i, i + head_dim / 2)."""
    ang = np.arange(positions)[:, None] * base ** (-np.arange(0, head_dim, 2) / head_dim)
    return C.Rope(*(torch.from_numpy(f(ang).astype(np.float32)).to(device) for f in (np.cos, np.sin)))


def quantise_cache(k_pages, v_pages, page_table, ctx_len) -> C.Kv8Pool:
    """An 8-bit cache with the contents of a bf16 one (pools [L, pages, Hkv, 16, D], the same page
    table): every sequence's ctx_len[b] cached tokens, a few thousand at a time."""
    L, N, H, P, D = k_pages.shape
    B, width = page_table.shape
    pool = C.new_kv8_pool(L, N, H, D, device=k_pages.device)
    ids = page_table.long().clamp(min=0)
    step = max(1, 4096 // B)                       # pages of every sequence at a time
    for p0 in range(0, width, step):
        at = ids[:, p0:p0 + step]
        n = at.shape[1] * P
        start = torch.full_like(ctx_len, p0 * P)
        rows = (ctx_len - start).clamp(0, n)
        for l in range(L):
            k, v = (t[l][at].transpose(2, 3).reshape(B, n, H, D) for t in (k_pages, v_pages))
            C.kv8_append(pool, k, v, page_table, start, rows, layer=l)
    return pool


class Kv8Round(VerifyRound):
    """``inputs`` as VerifyRound's, their q and k_blk before the rotation and their cache (already
    rotated) quantised into ``self.pool``; ``rope`` None builds the usual tables.  ``pages``: with a number,
    each block row attends to that many cached pages (the first ``sink``, the last ``recent`` and
    those of the largest scores) instead of all.  ``max_ctx`` (the longest context that rounds will reach),
    ``temperature``, ``seed`` and ``sps_q`` are VerifyRound's."""

    def __init__(self, inputs: Dict[str, object], draft: np.ndarray, lam: float = 0.6, mode: int = C.POLICY_MLP, keep_attn: bool = False,
                 rope: Optional[C.Rope] = None, pages: Optional[int] = None, sink: int = 1, recent: int = 4, max_ctx: Optional[int] = None,
                 temperature: Optional[float] = None, seed: int = 0, sps_q: Optional[torch.Tensor] = None):
        self.pages = None if pages is None else int(pages)
        super().__init__(inputs, draft, lam, mode, keep_attn, max_ctx, temperature, seed, sps_q)
        cfg, dev = self.cfg, self.q.device
        if self.k_pages.shape[0] != cfg.layers:
            raise ValueError("the cache must hold every layer")
        self.pool = quantise_cache(self.k_pages, self.v_pages, self.page_table, self.ctx_len)
        self.k_pages = self.v_pages = None
        self.inp = {n: t for n, t in self.inp.items() if n not in ("k_pages", "v_pages")}
        self.rope = rope if rope is not None else rope_tables(self.page_table.shape[1] * PAGE, cfg.head_dim, device=dev)
        self.q_rot, self.k_rot = torch.empty_like(self.q), torch.empty_like(self.k_blk)
        self.start = self.ctx_len.clone()
        self.sink, self.recent = int(sink), int(recent)
        if self.pages is not None:
            self.sel = torch.empty((cfg.batch, cfg.rows, cfg.kv_heads, self.pages), dtype=torch.int32, device=dev)
        # the accepted lengths and tokens come from the commit call with no layers: its pools are never touched
        self.no_blk = torch.empty((0, cfg.batch, cfg.rows, cfg.kv_heads, cfg.head_dim), dtype=torch.bfloat16, device=dev)
        self.no_pool = torch.empty((1, 1, cfg.kv_heads, PAGE, cfg.head_dim), dtype=torch.bfloat16, device=dev)

    def _count_launches(self) -> int:
        cfg = self.cfg
        per_layer = 1 if self.pages is None else 2
        decide = 2 if self.sps else (1 if cfg.k > 0 else 0)
        # rotation, layers, LM head (main and merge per launch), arbitration or acceptance, accepted length, append
        return 1 + cfg.layers * per_layer + 2 * ((cfg.m_rows + 1023) // 1024) + decide + 1 + 1

    def rotate(self) -> None:
        C.kv8_rotate(self.q, self.k_blk, self.rope, self.ctx_len, self.q_rot, self.k_rot)

    def attention(self, l: int, kv_stable: Optional[bool] = None) -> torch.Tensor:
        out = self.attn_out[l if self.attn_out.shape[0] > 1 else 0]
        stable = l > 0 if kv_stable is None else kv_stable
        sel = None
        if self.pages is not None:
            sel = C.kv8_select(self.q_rot[l], self.pool, l, self.page_table, self.ctx_len, self.sel, self.sink, self.recent)
        return C.kv8_attn(self.q_rot[l], self.k_rot[l], self.v_blk[l], self.pool, l, self.page_table, self.ctx_len, out, self.max_ctx,
                          sel=sel, kv_stable=stable)

    def commit(self):
        """Accepted lengths and tokens, then the accepted rows of every layer into the cache from
        where the context ended before."""
        self.start.copy_(self.ctx_len)
        C.accept_commit(self.draft, self.target if self.sps else self.argmax, self.accept, self.no_blk, self.no_blk, self.no_pool, self.no_pool, self.page_table,
                        self.ctx_len, self.accept_len, self.emitted)
        C.kv8_append(self.pool, self.k_blk, self.v_blk, self.page_table, self.start, self.accept_len, self.rope)
        return self.accept_len, self.emitted

    def run(self, restore: bool = True) -> None:
        if restore:
            self.restore_context()
        self.rotate()
        for l in range(self.cfg.layers):
            self.attention(l)
        self.lmhead()
        if self.cfg.k > 0 or self.sps:
            self.arbitrate()
        self.commit()


def timed(rnd: VerifyRound, reps: int) -> float:
    """Milliseconds of a captured round."""
    rnd.capture()
    for _ in range(3):
        rnd.replay()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(reps):
        rnd.replay()
    b.record()
    b.synchronize()
    return a.elapsed_time(b) / reps


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--config", default="qwen3_8b_b1", choices=sorted(W.CONFIGS))
    ap.add_argument("--layers", type=int, default=None)
    ap.add_argument("--k", type=int, default=None)
    ap.add_argument("--pages", type=int, default=None, help="cached pages that a block row reads (default: all)")
    ap.add_argument("--reps", type=int, default=20)
    args = ap.parse_args()
    from . import build as B
    C.load_library(B.build())
    cfg = W.CONFIGS[args.config]
    cfg = cfg.replace(layers=args.layers if args.layers is not None else cfg.layers, k=args.k if args.k is not None else cfg.k)
    inp = W.make_round_inputs(cfg, device="cuda")
    draft = np.random.default_rng(cfg.index).integers(0, cfg.vocab, (cfg.batch, cfg.k)).astype(np.int32)
    rnd, plain = Kv8Round(inp, draft, cfg.lam, pages=args.pages), VerifyRound(inp, draft, cfg.lam)
    ms8, ms16 = timed(rnd, args.reps), timed(plain, args.reps)       # (each starts from the context it was made with)
    pool = rnd.pool
    nbytes = sum(t.numel() * t.element_size() for t in (pool.k, pool.v, pool.scale, pool.summary, pool.summary_scale))
    print(json.dumps({"workload": cfg.name, "layers": cfg.layers, "k": cfg.k, "pages": args.pages, "ms_per_round": ms8,
                      "ms_per_round_bf16_cache": ms16, "cache_bytes": nbytes, "bf16_cache_bytes": 2 * pool.k.numel() * 2,
                      "launches": rnd.launches_per_round, "device_error": C.get_device_error()}))


if __name__ == "__main__":
    main()
