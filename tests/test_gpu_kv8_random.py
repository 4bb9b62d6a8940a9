"""The 8-bit cache's attention on random shapes, plans, masks and magnitudes against the float64 oracle: contexts of many
pages a CTA, scales drawn by the page, the token or the channel, lists, strided inputs.  Tolerance as in the other tests: within
2^-8 (|o| + sum p |v|)."""
import math

import numpy as np
import pytest
import torch

from oracle import cospec_kv8 as K
from paper_2605_24793_gb300 import build as BLD
from paper_2605_24793_gb300 import cospec as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    C.load_library(BLD.build())
    torch.cuda.set_device(0)
    C.get_device_error()


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _magnitudes(rng, kind, n):
    """Powers of two for n pages: alike, a little apart, a few far away, anywhere."""
    if kind == "alike":
        return np.zeros(n)
    if kind == "near":
        return rng.integers(-5, 6, n).astype(float)
    e = np.zeros(n)
    if kind == "few":
        for p in rng.integers(0, n, 3):
            e[p] = rng.integers(-70, 110)
        return e
    return rng.integers(-60, 60, n).astype(float)


@pytest.mark.parametrize("seed", range(48))
def test_random_attention(seed):
    rng = np.random.default_rng(seed)
    H = int(rng.choice([1, 2, 3]))
    D = int(rng.choice([64, 128]))
    G = int(rng.choice([1, 2, 4, 5, 8, 16]))
    R = int(rng.integers(1, min(64, 512 // G, 400 // (G * H) + 1) + 1))
    B = int(rng.integers(1, 4))
    long = rng.random() < 0.4
    ctx = [int(x) for x in rng.integers(0, 9500 if long else 900, B)]
    if rng.random() < 0.3:
        ctx[0] = ctx[0] // 128 * 128
    T = max(max(ctx), 1)
    pages = -(-T // 16)
    k, v = rng.standard_normal((2, B, T, H, D))
    q, kb, vb = rng.standard_normal((B, R, H * G, D)), rng.standard_normal((B, R, H, D)), rng.standard_normal((B, R, H, D))
    kind = str(rng.choice(["alike", "near", "few", "any"]))
    q[..., 0] = 8.0
    k[..., 0] = kb[..., 0] = 0.0
    for b in range(B):
        e = _magnitudes(rng, kind, pages)
        v[b] *= np.repeat(2.0 ** e, 16)[:T, None, None]
        # weights that make up for the magnitude, or nearly nothing, or neither
        bits = np.where(rng.random(pages) < 0.5, np.maximum(e, 0), rng.choice([0, 0, 100], pages))
        if kind != "alike":
            k[b, ..., 0] = np.repeat(-bits * math.log(2.0) * math.sqrt(D) / 8.0, 16)[:T, None]
    if rng.random() < 0.5:
        for _ in range(4):                     # tokens and channels
            b, t = int(rng.integers(B)), int(rng.integers(T))
            v[b, t] *= 2.0 ** int(rng.integers(-30, 40))
            v[b, int(rng.integers(T)), :, int(rng.integers(D))] *= 2.0 ** int(rng.integers(-30, 40))
    if rng.random() < 0.5:
        j = int(rng.integers(R))
        vb[:, j] *= 2.0 ** int(rng.integers(-60, 60))
        kb[:, j, :, 1:] *= 2.0 ** int(rng.integers(-20, 3))
    full = rng.random() < 0.3
    table = rng.permutation(B * pages).reshape(B, pages).astype(np.int32)
    pool, ref = C.new_kv8_pool(1, B * pages, H, D), K.new_pool(1, B * pages, H, D)
    kt, vt = _dev(k[None]), _dev(v[None])
    fused = _dev(np.concatenate([q, kb, vb], axis=2))
    qd, kbd, vbd = fused[:, :, :H * G], fused[:, :, H * G:H * G + H], fused[:, :, H * G + H:]
    C.kv8_append(pool, kt, vt, _ints(table), _ints([0] * B), _ints(ctx))
    K.append(ref, _np(kt), _np(vt), table, [0] * B, ctx)
    sel = None
    if rng.random() < 0.35:
        n = int(rng.integers(1, 40))
        sel = np.full((B, R, H, n), -1, np.int32)
        for b in range(B):
            num = -(-ctx[b] // 16)
            for j in range(R):
                for h in range(H):
                    c = np.sort(rng.choice(num, min(num, int(rng.integers(0, n + 1))), replace=False)) if num else np.zeros(0, int)
                    sel[b, j, h, :len(c)] = c
    o, mag = K.attention(_np(qd), _np(kbd), _np(vbd), ref, 0, table, ctx, sel=sel, full=full)
    bound = 2.0 ** -8 * (np.abs(o) + mag)
    out = torch.empty((B, R, H * G, D), dtype=torch.bfloat16, device="cuda")
    for max_ctx in {max(ctx), 0, pages * 16}:
        for stable in (False, True):
            out.fill_(math.nan)
            torch.cuda.synchronize()
            C.kv8_attn(qd, kbd, vbd, pool, 0, _ints(table), _ints(ctx), out, max_ctx, sel=None if sel is None else _ints(sel), block_full=full,
                       kv_stable=stable)
            assert C.get_device_error() == 0
            err = np.abs(_np(out) - o)
            bad = ~(err <= bound)
            assert not bad.any(), (f"B {B} R {R} G {G} H {H} D {D} ctx {ctx} {kind} full {full} max_ctx {max_ctx} stable {stable} sel {sel is not None}: "
                                   f"{bad.sum()} of {bad.size}, worst {np.nanmax(err / bound):.3g}, {np.isnan(err).sum()} NaN")
