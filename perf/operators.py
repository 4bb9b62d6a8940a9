"""The 8-bit paged KV cache's operators as cases that can be timed.

A verify round keeps its keys and values in pages of 16 tokens, held in 8 bits (e4m3)
with a power-of-two scale for each page and KV head.  The kinds of case:

  append   rotate the new rows' keys (and queries) and append them to the cache
  attn     attention of a block of rows over the cache and the block's own bf16 rows
  sparse   the same over the pages that a score of page summaries selects for each row
  layer    the three steps of one layer of a round: rotate, attend, append the accepted rows

Sizes are those of the workloads in ``workload.CONFIGS`` and of the tests: the
Qwen3-8B, Qwen3-32B and Llama-3-8B shapes at their batch sizes, the tiny round and
the paper's default draft length K = 25.  The plain form (``own`` false) needs torch alone.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
PAGE = 16
F8 = torch.float8_e4m3fn


def listed():
    qwen8 = dict(q_heads=32, kv_heads=8, head_dim=128)
    tiny = dict(q_heads=8, kv_heads=2, head_dim=64)
    return [
        # A token of one user enters the cache of one small layer: all latency.
        dict(name="append_tiny", kind="append", layers=1, batch=1, rows=1, ctx_lo=256, ctx_hi=256, queries=True, fused=False, rot=64, inter=False, **tiny),
        # The commit after a round: up to K + 1 = 8 accepted rows of 16 sequences in all 36 layers.
        dict(name="append_b16_k7", kind="append", layers=36, batch=16, rows=8, ctx_lo=64, ctx_hi=512, queries=False, fused=False, rot=128, inter=False, **qwen8),
        # A new request's 4096 tokens, queries rotated too, cut out of the fused projection's output.
        dict(name="append_4096", kind="append", layers=2, batch=1, rows=4096, ctx_lo=0, ctx_hi=0, queries=True, fused=True, rot=128, inter=False, **qwen8),
        # One user decoding a token at a time: one layer at 4096 tokens.
        dict(name="attn_b1_decode", kind="attn", batch=1, rows=1, ctx_lo=4096, ctx_hi=4096, fused=False, full=False, **qwen8),
        # A serving batch of ragged contexts, K = 7.
        dict(name="attn_b16_k7", kind="attn", batch=16, rows=8, ctx_lo=2048, ctx_hi=8192, fused=False, full=False, **qwen8),
        # The same batch at the paper's default draft length.
        dict(name="attn_b16_k25", kind="attn", batch=16, rows=26, ctx_lo=2048, ctx_hi=8192, fused=False, full=False, **qwen8),
        # Long reasoning: one layer of the Llama-3-8B-shaped batch-64 workload, the largest.
        dict(name="attn_llama_b64_k7", kind="attn", batch=64, rows=8, ctx_lo=8192, ctx_hi=32768, fused=False, full=False, **qwen8),
        # Contexts from nothing to a few pages, rows and lengths odd, projections in one buffer.
        dict(name="attn_short_odd", kind="attn", batch=7, rows=5, ctx_lo=0, ctx_hi=77, fused=True, full=False, **tiny),
        # One user at 32768 tokens who reads 64 pages (1024 tokens) of them.
        dict(name="sparse_b1_decode", kind="sparse", batch=1, rows=1, ctx_lo=32768, ctx_hi=32768, pages=64, sink=1, recent=4, fused=False, **qwen8),
        # The long-reasoning batch, decoding, 128 pages a row.
        dict(name="sparse_b64_decode", kind="sparse", batch=64, rows=1, ctx_lo=8192, ctx_hi=32768, pages=128, sink=1, recent=4, fused=False, **qwen8),
        # A serving batch verifying K = 7: every row of the block chooses its own pages.
        dict(name="sparse_b16_k7", kind="sparse", batch=16, rows=8, ctx_lo=8192, ctx_hi=16384, pages=128, sink=1, recent=4, fused=False, **qwen8),
        # One layer of a round at batch 4: rotate, attend, append.
        dict(name="layer_b4_k5", kind="layer", batch=4, rows=6, ctx_lo=1000, ctx_hi=4096, fused=True, rot=128, inter=False, **qwen8),
    ]


def _log_int(rng, lo, hi):
    """An integer in [lo, hi], uniform in the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HEADS = [(32, 8, 128), (32, 8, 128), (64, 8, 128), (8, 2, 64), (16, 8, 64), (12, 4, 128), (6, 6, 64)]


def draw(rng):
    kind = rng.choice(["append", "attn", "attn", "sparse", "sparse", "layer"])
    hq, hkv, d = rng.choice(_HEADS)
    case = dict(kind=kind, q_heads=hq, kv_heads=hkv, head_dim=d, fused=rng.random() < 0.5)
    if kind == "append":
        batch = _log_int(rng, 1, 64)
        rows = _log_int(rng, 1, 4096 // batch)
        layers = _log_int(rng, 1, max(1, min(36, 8192 // (batch * rows))))
        lo = rng.randint(0, 200)
        return dict(case, layers=layers, batch=batch, rows=rows, ctx_lo=lo, ctx_hi=lo + rng.randint(0, 300),
                    queries=rng.random() < 0.5 and layers * batch * rows * hq <= 8192 * 32, rot=rng.choice([d, d, d // 2]), inter=rng.random() < 0.3)
    if kind == "attn":
        batch, rows = _log_int(rng, 1, 64), _log_int(rng, 1, 26)
        hi = _log_int(rng, 16, min(32768, 64 * 32768 * 8 * 32 // (batch * rows * hq)))
        return dict(case, batch=batch, rows=rows, ctx_lo=rng.choice([0, hi // 4, hi]), ctx_hi=hi, full=rng.random() < 0.2)
    if kind == "sparse":
        hi = _log_int(rng, 200, 32768)
        sink, recent = rng.randint(0, 2), rng.randint(1, 5)
        batch = _log_int(rng, 1, 64)
        return dict(case, batch=batch, rows=_log_int(rng, 1, max(1, min(16, 128 // batch))), ctx_lo=rng.choice([0, hi // 4, hi]), ctx_hi=hi,
                    pages=sink + recent + _log_int(rng, 4, 160), sink=sink, recent=recent)
    hi = _log_int(rng, 100, 8192)
    return dict(case, batch=_log_int(rng, 1, 32), rows=_log_int(rng, 1, 16), ctx_lo=rng.randint(0, hi), ctx_hi=hi, rot=rng.choice([d, d, d // 2]),
                inter=rng.random() < 0.3)


# ---------------------------------------------------------------- inputs (plain torch, from the seed alone)
def _contexts(case, seed):
    """Ragged context lengths spread evenly over [ctx_lo, ctx_hi], in an order of the seed."""
    B, lo, hi = case["batch"], case["ctx_lo"], case["ctx_hi"]
    rng = np.random.default_rng(int(seed))
    ctx = lo + np.floor((hi - lo + 1) * (np.arange(B) + rng.random(B)) / B).astype(np.int64)
    return np.minimum(rng.permutation(ctx), hi).astype(np.int32)


def _pages(case, ctx, seed):
    """A shuffled page table with room for the context and the rows, -1 elsewhere, over a pool
    whose size is the same for every seed."""
    B, R, lo, hi = case["batch"], case["rows"], case["ctx_lo"], case["ctx_hi"]
    width = (hi + R + PAGE - 1) // PAGE
    need = (ctx.astype(np.int64) + R + PAGE - 1) // PAGE
    most = np.minimum(lo + (hi - lo + 1) * np.arange(1, B + 1) // B, hi)
    total = int(((most + R + PAGE - 1) // PAGE).sum())
    order = np.random.default_rng(int(seed) + 1).permutation(total).astype(np.int32)
    table = np.full((B, width), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += int(n)
    return table, total


def _projections(g, case, lead, fused):
    """q, k, v of the rows as a model's projections leave them: each by itself, or parts of one buffer."""
    R, Hq, Hkv, D = case["rows"], case["q_heads"], case["kv_heads"], case["head_dim"]
    buf = torch.empty((*lead, R, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    # a few channels of the keys are larger than the rest, as trained models have them
    gain = torch.exp(0.5 * torch.empty((Hkv, D), device=DEV).normal_(generator=g)).to(torch.bfloat16)
    buf[..., Hq:Hq + Hkv, :] *= gain
    q, k, v = buf[..., :Hq, :], buf[..., Hq:Hq + Hkv, :], buf[..., Hq + Hkv:, :]
    return (q, k, v) if fused else (q.contiguous(), k.contiguous(), v.contiguous())


def _pow2(a, top, e):
    """The smallest power of two s with a <= c s, c = top * 2^e (1/2 <= top < 1), exponent in [-100, 120]; 2^-100 for 0."""
    m, x = torch.frexp(a)
    k = torch.where(a > 0, x - e + (m > top).to(torch.int32), torch.full_like(x, -100)).clamp(-100, 120)
    return ((k.to(torch.int32) + 127) << 23).view(torch.float32)


def _pow2_448(a):
    return _pow2(a, 0.875, 9)


def _pow2_127(a):
    return _pow2(a, 0.9921875, 7)


def _cache(g, case, layers, num):
    """Full pages of codes with their scales and summaries.  Keys of a page have something in common, as neighbouring tokens' have."""
    Hkv, D = case["kv_heads"], case["head_dim"]
    gain = torch.exp(0.5 * torch.empty((Hkv, 1, D), device=DEV).normal_(generator=g))
    s = dict(k=torch.empty((layers, num, Hkv, PAGE, D), dtype=F8, device=DEV), v=torch.empty((layers, num, Hkv, D, PAGE), dtype=F8, device=DEV),
             scale=torch.empty((layers, num, Hkv, 2), device=DEV), summary=torch.empty((layers, num, Hkv, D), dtype=torch.int8, device=DEV),
             summary_scale=torch.empty((layers, num, Hkv), device=DEV))
    step = max(1, (1 << 28) // (Hkv * PAGE * D))
    for layer in range(layers):
        for n0 in range(0, num, step):
            n = min(step, num - n0)
            x = torch.empty((n, Hkv, PAGE, D), device=DEV).normal_(generator=g)
            x += torch.empty((n, Hkv, 1, D), device=DEV).normal_(0.0, 0.7, generator=g)
            x *= gain
            sk = _pow2_448(x.abs().amax((2, 3)))
            codes = (x / sk[..., None, None]).to(F8)
            s["k"][layer, n0:n0 + n] = codes
            t = codes.float().sum(2)
            u = _pow2_127(t.abs().amax(2))
            s["summary"][layer, n0:n0 + n] = torch.round(t / u[..., None]).to(torch.int8)
            s["summary_scale"][layer, n0:n0 + n] = u * sk
            x.normal_(generator=g)
            sv = _pow2_448(x.abs().amax((2, 3)))
            s["v"][layer, n0:n0 + n] = (x / sv[..., None, None]).to(F8).transpose(2, 3)
            s["scale"][layer, n0:n0 + n, :, 0] = sk
            s["scale"][layer, n0:n0 + n, :, 1] = sv
    return s


def prepare(case, seed):
    kind = case["kind"]
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 13)
    ctx = _contexts(case, seed)
    table, num = _pages(case, ctx, seed)
    B, R, Hq, Hkv, D = case["batch"], case["rows"], case["q_heads"], case["kv_heads"], case["head_dim"]
    layers = case.get("layers", 1)
    s = _cache(g, case, layers, num)
    s.update(case=dict(case), table=torch.from_numpy(table).to(DEV), ctx=torch.from_numpy(ctx).to(DEV), max_ctx=int(ctx.max()))
    lead = (layers, B) if kind == "append" else (B,)
    s["q"], s["kn"], s["vn"] = _projections(g, case, lead, case["fused"])
    if kind in ("append", "layer"):
        # rows that a round keeps: one at least, all of them for a prompt
        rows = np.random.default_rng(int(seed) + 2).integers(1, R + 1, B) if R <= 32 else np.full(B, R)
        s["rows"] = torch.from_numpy(rows.astype(np.int32)).to(DEV)
        pos = torch.arange(case["ctx_hi"] + R, dtype=torch.float64, device=DEV)[:, None]
        inv = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=DEV) / case["rot"])
        s["cos"], s["sin"] = torch.cos(pos * inv).float(), torch.sin(pos * inv).float()
        s["k_rot"] = torch.empty((*lead, R, Hkv, D), dtype=torch.bfloat16, device=DEV)
    s["q_rot"] = torch.empty((*lead, R, Hq, D), dtype=torch.bfloat16, device=DEV)
    s["out"] = torch.empty((B, R, Hq, D), dtype=torch.bfloat16, device=DEV)
    if kind == "sparse":
        s["sel"] = torch.empty((B, R, Hkv, case["pages"]), dtype=torch.int32, device=DEV)
    return s


# ---------------------------------------------------------------- the plain form
def _rotate(s, x):
    """x [..., B, R, H, D] rotated to its positions, in 32 bits."""
    case = s["case"]
    pos = s["ctx"].long()[:, None] + torch.arange(case["rows"], device=DEV)
    c, n = s["cos"][pos][:, :, None, :], s["sin"][pos][:, :, None, :]
    h = case["rot"] // 2
    x = x.float()
    a, b = (x[..., 0:2 * h:2], x[..., 1:2 * h:2]) if case["inter"] else (x[..., :h], x[..., h:2 * h])
    ra, rb = a * c - b * n, b * c + a * n
    turned = torch.stack((ra, rb), dim=-1).flatten(-2) if case["inter"] else torch.cat((ra, rb), dim=-1)
    return torch.cat((turned, x[..., 2 * h:]), dim=-1)


def _append(s, k, v):
    """k, v [L, B, R, Hkv, D] in 32 bits appended at positions ctx.. of the pages, the pool rewritten in place."""
    case = s["case"]
    R, P = case["rows"], s["table"].shape[1]
    T = (R + PAGE - 2) // PAGE + 1                                     # pages that R rows can touch
    ctx, rows = s["ctx"].long(), s["rows"].long()
    t = torch.arange(T, device=DEV)
    page = ctx[:, None] // PAGE + t                                    # [B, T]
    j = page[:, :, None] * PAGE + torch.arange(PAGE, device=DEV) - ctx[:, None, None]
    new = (j >= 0) & (j < rows[:, None, None])                         # [B, T, 16]
    old = (j < 0) & (t[:, None] == 0)
    kept = new.any(2) | (t == 0)
    # a page without new rows stands for the sequence's first one again, with the same contents
    first = lambda x: torch.where(kept.view(kept.shape + (1,) * (x.dim() - 3)), x, x[:, :, :1])  # noqa: E731
    phys = torch.gather(s["table"].long(), 1, page.clamp(max=P - 1))
    phys = torch.where(kept, phys, phys[:, :1])
    B = phys.shape[0]
    at = torch.arange(B, device=DEV)[:, None, None]
    has_old = old.any(2)[None, :, :, None]

    def codes_of(x, pool, which):                                      # x [L, B, R, H, D] -> codes [L, B, T, H, 16, D], scale [L, B, T, H]
        xp = x[:, at, j.clamp(0, R - 1)].transpose(3, 4)               # [L, B, T, H, 16, D]
        mn, mo = new[None, :, :, None, :, None], old[None, :, :, None, :, None]
        before = pool.view(torch.uint8)[:, phys].view(F8)
        before = before.transpose(4, 5) if which else before
        was = s["scale"][:, phys][..., which]
        sc = _pow2_448(torch.where(mn, xp.abs(), 0).amax((4, 5)))
        sc = torch.where(has_old, torch.maximum(sc, was), sc)
        sc = torch.where(new.any(2)[None, :, :, None], sc, was)
        moved = (before.float() * (was / sc)[..., None, None]).to(F8)
        got = torch.where(mn, (xp / sc[..., None, None]).to(F8).view(torch.uint8), torch.where(mo, moved.view(torch.uint8), before.contiguous().view(torch.uint8)))
        return got, sc

    kc, ks = codes_of(k, s["k"], 0)
    vc, vs = codes_of(v, s["v"], 1)
    total = torch.where((new | old)[None, :, :, None, :, None], kc.view(F8).float(), 0).sum(4)
    u = _pow2_127(total.abs().amax(-1))
    some = new.any(2)[None, :, :, None]
    sums = torch.where(some[..., None], torch.round(total / u[..., None]).to(torch.int8), s["summary"][:, phys])
    sums_s = torch.where(some, u * ks, s["summary_scale"][:, phys])
    s["k"].view(torch.uint8)[:, phys] = first(kc)
    s["v"].view(torch.uint8)[:, phys] = first(vc).transpose(4, 5)
    s["scale"][:, phys] = first(torch.stack((ks, vs), dim=-1))
    s["summary"][:, phys] = first(sums)
    s["summary_scale"][:, phys] = first(sums_s)


def _softmax(x):
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _attend(s, q, kb, vb):
    """Attention of the block's rows over the whole cache and the block, [B, R, Hq, D]."""
    case = s["case"]
    B, R, Hq, D = q.shape
    Hkv = kb.shape[2]
    G, P = Hq // Hkv, s["table"].shape[1]
    ids = s["table"].long().clamp(min=0)
    seen = torch.arange(P * PAGE, device=DEV) < s["ctx"][:, None]                            # [B, N]
    sc = s["scale"][0][ids]                                                                  # [B, P, H, 2]
    k = (s["k"][0].view(torch.uint8)[ids].view(F8).float() * sc[..., 0, None, None]).permute(0, 2, 1, 3, 4).reshape(B, Hkv, P * PAGE, D)
    v = (s["v"][0].view(torch.uint8)[ids].view(F8).float() * sc[..., 1, None, None]).permute(0, 2, 1, 4, 3).reshape(B, Hkv, P * PAGE, D)
    v = torch.where(seen[:, None, :, None], v, 0)
    rows = q.float().view(B, R, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, R * G, D) * (1.0 / math.sqrt(D))
    x = torch.where(seen[:, None, None, :], rows @ k.transpose(2, 3), -math.inf)
    y = (rows @ kb.float().permute(0, 2, 3, 1)).view(B, Hkv, R, G, R)
    if not case.get("full"):
        y = torch.where(torch.ones(R, R, dtype=torch.bool, device=DEV).tril()[:, None, :], y, -math.inf)
    p = _softmax(torch.cat((x, y.view(B, Hkv, R * G, R)), dim=-1))
    o = p[..., :P * PAGE] @ v + p[..., P * PAGE:] @ vb.float().transpose(1, 2)
    return o.view(B, Hkv, R, G, D).permute(0, 2, 1, 3, 4).reshape(B, R, Hq, D).to(torch.bfloat16)


def _select(s, q):
    """The pages that each row and KV head reads, [B, R, Hkv, n], ascending, -1 after the last."""
    case = s["case"]
    B, R, Hq, D = q.shape
    Hkv, P, n = case["kv_heads"], s["table"].shape[1], case["pages"]
    ids = s["table"].long().clamp(min=0)
    num = (s["ctx"].long() + PAGE - 1) // PAGE
    x = q.float().view(B, R, Hkv, Hq // Hkv, D).transpose(1, 2)                              # [B, H, R, G, D]
    x = torch.round(x / _pow2_127(x.abs().amax((3, 4)))[..., None, None])
    score = (x.flatten(2, 3) @ s["summary"][0][ids].float().permute(0, 2, 3, 1)).view(B, Hkv, R, Hq // Hkv, P).amax(3)
    score = score * s["summary_scale"][0][ids].transpose(1, 2)[:, :, None, :]                # [B, H, R, P]
    p = torch.arange(P, device=DEV)
    num = num[:, None, None, None]
    score = torch.where((p < case["sink"]) | (p >= num - case["recent"]), math.inf, score)
    score = torch.where(p < num, score, -math.inf)
    pick = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :n]
    pick = torch.sort(torch.where(pick < num, pick, P))[0]
    pick = torch.where(pick < P, pick, -1)
    return torch.nn.functional.pad(pick, (0, n - pick.shape[-1]), value=-1).transpose(1, 2).to(torch.int32).contiguous()


def _attend_pages(s, q, kb, vb, sel):
    """Attention of each row over its own pages and the block's rows up to it."""
    B, R, Hq, D = q.shape
    Hkv, n = sel.shape[2], sel.shape[3]
    G = Hq // Hkv
    pg = sel.long()
    ids = torch.gather(s["table"].long()[:, None, None, :].expand(B, R, Hkv, -1), 3, pg.clamp(min=0)).clamp(min=0)
    h = torch.arange(Hkv, device=DEV)[:, None]
    pos = pg[..., None] * PAGE + torch.arange(PAGE, device=DEV)                              # [B, R, H, n, 16]
    seen = ((pg[..., None] >= 0) & (pos < s["ctx"][:, None, None, None, None])).flatten(3)
    sc = s["scale"][0][ids, h]                                                               # [B, R, H, n, 2]
    k = (s["k"][0].view(torch.uint8)[ids, h].view(F8).float() * sc[..., 0, None, None]).flatten(3, 4)
    v = (s["v"][0].view(torch.uint8)[ids, h].view(F8).float() * sc[..., 1, None, None]).transpose(4, 5).flatten(3, 4)
    v = torch.where(seen[..., None], v, 0)
    rows = q.float().view(B, R, Hkv, G, D) * (1.0 / math.sqrt(D))
    x = torch.where(seen[..., None, :], rows @ k.transpose(3, 4), -math.inf)
    y = rows @ kb.float().permute(0, 2, 3, 1)[:, None]                                       # [B, R, H, G, R]
    y = torch.where(torch.ones(R, R, dtype=torch.bool, device=DEV).tril()[:, None, None, :], y, -math.inf)
    p = _softmax(torch.cat((x, y), dim=-1))
    o = p[..., :n * PAGE] @ v + p[..., n * PAGE:] @ vb.float().transpose(1, 2)[:, None]
    return o.reshape(B, R, Hq, D).to(torch.bfloat16)


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "append":
        k = _rotate(s, s["kn"])
        _append(s, k, s["vn"].float())
        out = dict(k_rot=k.to(torch.bfloat16))
        if s["case"]["queries"]:
            out["q_rot"] = _rotate(s, s["q"]).to(torch.bfloat16)
        return dict(out, **_pool_of(s))
    if kind == "attn":
        return _attend(s, s["q"], s["kn"], s["vn"])
    if kind == "sparse":
        sel = _select(s, s["q"])
        return dict(sel=sel, out=_attend_pages(s, s["q"], s["kn"], s["vn"], sel))
    k = _rotate(s, s["kn"])
    out = _attend(s, _rotate(s, s["q"]).to(torch.bfloat16), k.to(torch.bfloat16), s["vn"])
    _append(s, k[None], s["vn"].float()[None])
    return dict(out=out, **_pool_of(s))


def _pool_of(s):
    return {n: s[n] for n in ("k", "v", "scale", "summary", "summary_scale")}


# ---------------------------------------------------------------- a pass
def run(state):
    s = state
    if not own:
        return _plain(s)
    from paper_2605_24793_gb300 import cospec as C
    case = s["case"]
    kind = case["kind"]
    if "pool" not in s:                      # the handles that a program keeps beside its tensors
        s["pool"] = C.Kv8Pool(s["k"], s["v"], s["scale"], s["summary"], s["summary_scale"])
        s["rope"] = C.Rope(s["cos"], s["sin"], case["inter"]) if "cos" in s else None
    if kind == "append":
        q_rot = s["q_rot"] if case["queries"] else None
        C.kv8_append(s["pool"], s["kn"], s["vn"], s["table"], s["ctx"], s["rows"], s["rope"], k_out=s["k_rot"],
                     q=s["q"] if case["queries"] else None, q_out=q_rot)
        out = dict(k_rot=s["k_rot"], **_pool_of(s))
        return dict(out, q_rot=q_rot) if case["queries"] else out
    if kind == "attn":
        return C.kv8_attn(s["q"], s["kn"], s["vn"], s["pool"], 0, s["table"], s["ctx"], s["out"], s["max_ctx"], block_full=case["full"])
    if kind == "sparse":
        C.kv8_select(s["q"], s["pool"], 0, s["table"], s["ctx"], s["sel"], case["sink"], case["recent"])
        C.kv8_attn(s["q"], s["kn"], s["vn"], s["pool"], 0, s["table"], s["ctx"], s["out"], s["max_ctx"], sel=s["sel"])
        return dict(sel=s["sel"], out=s["out"])
    C.kv8_rotate(s["q"], s["kn"], s["rope"], s["ctx"], s["q_rot"], s["k_rot"])
    C.kv8_attn(s["q_rot"], s["k_rot"], s["vn"], s["pool"], 0, s["table"], s["ctx"], s["out"], s["max_ctx"])
    C.kv8_append(s["pool"], s["kn"], s["vn"], s["table"], s["ctx"], s["rows"], s["rope"], layer=0)
    return dict(out=s["out"], **_pool_of(s))


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind = case["kind"]
    B, R, Hq, Hkv, D = case["batch"], case["rows"], case["q_heads"], case["kv_heads"], case["head_dim"]
    keys = B * (case["ctx_lo"] + case["ctx_hi"]) / 2
    kept = B * ((R + 1) / 2 if R <= 32 else R)                       # rows that enter the cache
    # codes of K and V, scales and summaries by the page
    store = kept * Hkv * (2 * D + (8 + D + 4) / PAGE)
    if kind == "append":
        L = case["layers"]
        nbytes = L * (2.0 * (B * R + kept) * Hkv * D + 2.0 * B * R * Hkv * D + store + (4.0 * B * R * Hq * D if case["queries"] else 0))
        return dict(bytes=nbytes, flops=3.0 * L * B * R * case["rot"] * (Hkv + (Hq if case["queries"] else 0)))
    rows_io = 4.0 * B * R * (Hq + Hkv) * D                           # q and out, block keys and values
    own_keys = R if case.get("full") else (R + 1) / 2
    if kind == "sparse":
        # each row's pages, if all rows of a block chose the same ones
        most = min(case["pages"], math.ceil((case["ctx_lo"] + case["ctx_hi"]) / 2 / PAGE))
        nbytes = rows_io + 4.0 * B * R * Hkv * case["pages"] + keys / PAGE * Hkv * (D + 4) + B * Hkv * most * (2 * PAGE * D + 8)
        return dict(bytes=nbytes, flops=2.0 * B * R * Hq * D * (keys / B / PAGE + 2 * (most * PAGE + own_keys)))
    nbytes = rows_io + keys * Hkv * (2 * D + 8 / PAGE)
    flops = 4.0 * Hq * D * R * (keys + B * own_keys)
    if kind == "layer":
        nbytes += store
    return dict(bytes=nbytes, flops=flops)


# ---------------------------------------------------------------- the definition in 64 bits
def _x_turn(x, pos, cos, sin, rot, inter):
    """Each pair (x[a], x[b]) times e^(i angle): x [R, H, D] in 64 bits."""
    a = np.arange(0, rot, 2) if inter else np.arange(rot // 2)
    b = a + 1 if inter else a + rot // 2
    a, b = torch.from_numpy(a).to(DEV), torch.from_numpy(b).to(DEV)
    z = torch.complex(x[..., a], x[..., b]) * torch.complex(cos[pos].double(), sin[pos].double())[:, None, :]
    y = x.clone()
    y[..., a], y[..., b] = z.real, z.imag
    return y


def _x_scale(m, c):
    """Power of two by the logarithm, mended by a comparison."""
    if m == 0:
        return 2.0 ** -100
    e = math.ceil(math.log2(m / c))
    while m > c * 2.0 ** e:
        e += 1
    while m <= c * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** min(120, max(-100, e))


def _x_append(s, case, kt, vt):
    """Codes as the numbers they round, scales: page by page."""
    L, Hkv = kt.shape[0], case["kv_heads"]
    got = dict(k=s["k"].double(), v=s["v"].double(), scale=s["scale"].double())
    ctx, rows, table = s["ctx"].tolist(), s["rows"].tolist(), s["table"].tolist()
    for b in range(case["batch"]):
        for p in range(ctx[b] // PAGE, (ctx[b] + rows[b] - 1) // PAGE + 1):
            lo, hi, n = max(ctx[b], p * PAGE), min(ctx[b] + rows[b], (p + 1) * PAGE), table[b][p]
            for which, x in ((0, kt), (1, vt)):
                part = x[:, b, lo - ctx[b]:hi - ctx[b]].transpose(1, 2)                     # [L, H, rows, D]
                top = part.abs().amax((2, 3)).tolist()
                sc = torch.tensor([[_x_scale(top[a][h], 448.0) for h in range(Hkv)] for a in range(L)], dtype=torch.float64, device=DEV)
                page = got["v"][:, n].transpose(2, 3) if which else got["k"][:, n]
                if lo > p * PAGE:
                    was = got["scale"][:, n, :, which]
                    sc = torch.maximum(sc, was)
                    page[:, :, :lo - p * PAGE] *= (was / sc)[..., None, None]
                page[:, :, lo - p * PAGE:hi - p * PAGE] = part / sc[..., None, None]
                got["scale"][:, n, :, which] = sc
    return got


def _x_attn(s, b, q, kb, vb, pages, h, full):
    """One sequence and KV head: rows q [R, G, D] in 64 bits over the pages (a list, or one per row) and the block."""
    R, G, D = q.shape
    C, table = int(s["ctx"][b]), s["table"][b].long()
    out = torch.empty((R, G, D), dtype=torch.float64, device=DEV)
    every = [pages] * R if not isinstance(pages, list) else pages
    shared = None
    for j in range(R):
        if shared is None or isinstance(pages, list):
            at = every[j]
            ph = table[at]
            k = s["k"][0][:, h].view(torch.uint8)[ph].view(F8).double() * s["scale"][0, ph, h, 0].double()[:, None, None]
            v = (s["v"][0][:, h].view(torch.uint8)[ph].view(F8).double() * s["scale"][0, ph, h, 1].double()[:, None, None]).transpose(1, 2)
            ok = (at[:, None] * PAGE + torch.arange(PAGE, device=DEV) < C).flatten()
            shared = (k.flatten(0, 1)[ok], v.flatten(0, 1)[ok])
        m = R if full else j + 1
        kk, vv = torch.cat((shared[0], kb[:m])), torch.cat((shared[1], vb[:m]))
        x = q[j] @ kk.T / math.sqrt(D)
        out[j] = torch.softmax(x, dim=-1) @ vv
    return out


def exact(case, seed):
    kind = case["kind"]
    B, R, Hq, Hkv, D = case["batch"], case["rows"], case["q_heads"], case["kv_heads"], case["head_dim"]
    G = Hq // Hkv
    if kind in ("append", "layer") and B * (R / PAGE + 2) > 3000:
        return None
    s = prepare(case, seed)
    ctx = s["ctx"].tolist()
    if kind in ("append", "layer"):
        lead = s["kn"] if kind == "append" else s["kn"][None]
        turn = lambda x, b: torch.stack([_x_turn(y[b].double(), ctx[b] + torch.arange(R, device=DEV), s["cos"], s["sin"], case["rot"], case["inter"]) for y in x])  # noqa: E731
        kt = torch.stack([turn(lead, b) for b in range(B)], dim=1)
        pool = _x_append(s, case, kt, (s["vn"] if kind == "append" else s["vn"][None]).double())
        pool.update(summary=None, summary_scale=None)
        if kind == "append":
            pool["k_rot"] = kt
            if case["queries"]:
                pool["q_rot"] = torch.stack([turn(s["q"], b) for b in range(B)], dim=1)
            return pool
    out = torch.empty((B, R, Hkv, G, D), dtype=torch.float64, device=DEV)
    sel = torch.full((B, R, Hkv, case.get("pages", 1)), -1, dtype=torch.int32, device=DEV)
    for b in range(B):
        num = -(-ctx[b] // PAGE)
        pages = torch.arange(num, device=DEV)
        qb = s["q"][b].double() if kind != "layer" else turn(s["q"][None], b)[0]
        kb = s["kn"][b].double() if kind != "layer" else kt[0, b]
        qb = qb.view(R, Hkv, G, D)
        for h in range(Hkv):
            if kind == "sparse":
                su = s["summary"][0, s["table"][b, :num].long(), h].double()
                ss = s["summary_scale"][0, s["table"][b, :num].long(), h].double()
                top = qb[:, h].abs().amax((1, 2)).tolist()
                lists = []
                for j in range(R):
                    qi = torch.round(qb[j, h] / _x_scale(top[j], 127.0))
                    sc = (su @ qi.T).amax(1) * ss
                    sc[:case["sink"]] = math.inf
                    sc[max(0, num - case["recent"]):] = math.inf
                    order = torch.argsort(sc, descending=True, stable=True)[:case["pages"]]
                    lists.append(torch.sort(order)[0])
                    sel[b, j, h, :len(order)] = lists[-1].int()
                out[b, :, h] = _x_attn(s, b, qb[:, h], kb[:, h], s["vn"][b, :, h].double(), lists, h, False)
            else:
                out[b, :, h] = _x_attn(s, b, qb[:, h], kb[:, h], s["vn"][b, :, h].double(), pages, h, case.get("full", False))
    out = out.view(B, R, Hq, D)
    if kind == "attn":
        return out
    if kind == "sparse":
        return dict(sel=sel, out=out)
    return dict(out=out, **pool)
