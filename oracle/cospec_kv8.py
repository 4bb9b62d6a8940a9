"""Float64 oracle of the 8-bit paged KV cache: codes and scales, appending with the position
rotation, the page selection and the attention that reads the cache.  Test infrastructure
only: NumPy, written from the definitions, sharing nothing with the CUDA path."""
from __future__ import annotations

import math

import numpy as np

PAGE = 16


def _code_values() -> np.ndarray:
    """The number that each e4m3 code stands for: sign, 4 exponent bits of bias 7, 3 of fraction,
    subnormal at exponent 0, NaN at the last code of either sign, no infinities."""
    out = np.empty(256)
    for c in range(256):
        s, e, f = c >> 7, (c >> 3) & 15, c & 7
        x = f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        out[c] = math.nan if (e, f) == (15, 7) else (-x if s else x)
    return out


CODES = _code_values()
_POS = CODES[:127]


def encode(x: np.ndarray) -> np.ndarray:
    """Nearest code, ties to the even one; not finite: NaN (0x7f)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dh, dl = _POS[hi] - a, a - _POS[lo]
    c = np.where(dl < dh, lo, np.where(dl > dh, hi, np.where(lo % 2 == 0, lo, hi)))
    c = np.where(a >= 448.0, 126, c) | np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), c, 0x7F).astype(np.uint8)


def same_codes(a: np.ndarray, b: np.ndarray) -> bool:
    """Equal as numbers (a NaN has two codes, and so has zero)."""
    return bool(np.array_equal(CODES[a], CODES[b], equal_nan=True))


def pow2(a: float, c: float) -> float:
    """Smallest power of two s with a <= c s, its exponent in [-100, 120]."""
    if not a > 0:
        return 2.0 ** -100
    k = math.frexp(a / c)[1]
    while a > c * 2.0 ** k:
        k += 1
    while a <= c * 2.0 ** (k - 1):
        k -= 1
    return 2.0 ** min(120, max(-100, k))


def new_pool(layers, pages, heads, dim):
    return dict(k=np.zeros((layers, pages, heads, PAGE, dim), np.uint8), v=np.zeros((layers, pages, heads, dim, PAGE), np.uint8),
                scale=np.zeros((layers, pages, heads, 2)), summary=np.zeros((layers, pages, heads, dim), np.int8),
                summary_scale=np.zeros((layers, pages, heads)))


def rotate(x, pos, cos, sin, interleaved):
    """x [..., D] turned by the angles of position pos."""
    half = cos.shape[1]
    y = np.array(x, dtype=np.float64)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = float(cos[pos, i]), float(sin[pos, i])
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def append(pool, k, v, table, start, rows):
    """k, v [L, B, R, H, D] (already rotated): rows 0..rows[b]-1 into positions start[b]..; in place."""
    L, B, R, H, D = k.shape
    for b in range(B):
        n, st = int(rows[b]), int(start[b])
        for page in range(st // PAGE, (st + n - 1) // PAGE + 1 if n else 0):
            lo, hi, ph = max(st, page * PAGE), min(st + n, (page + 1) * PAGE), int(table[b][page])
            f, t = lo - page * PAGE, hi - page * PAGE
            for l in range(L):
                for h in range(H):
                    for which, x in ((0, k), (1, v)):
                        new = x[l, b, lo - st:hi - st, h].astype(np.float64)
                        fin = new[np.isfinite(new)]
                        s = pow2(float(np.max(np.abs(fin))) if fin.size else 0.0, 448.0)
                        cells = pool["v"][l, ph, h].T if which else pool["k"][l, ph, h]     # [16, D], a view
                        if f > 0:
                            was = pool["scale"][l, ph, h, which]
                            s = max(s, was)
                            if s != was:
                                cells[:f] = encode(CODES[cells[:f]] * (was / s))
                        cells[f:t] = encode(new / s)
                        pool["scale"][l, ph, h, which] = s
                    tot = np.nansum(CODES[pool["k"][l, ph, h, :t]], axis=0)
                    u = pow2(float(np.max(np.abs(tot))), 127.0)
                    pool["summary"][l, ph, h] = np.rint(tot / u).astype(np.int8)
                    # held in fp32, where a page of zeros (2^-100 times 2^-100) has the scale 0
                    pool["summary_scale"][l, ph, h] = np.float32(u * pool["scale"][l, ph, h, 0])


def select(q, pool, layer, table, ctx, pages, sink, recent):
    """q [B, R, Hq, D] -> chosen pages [B, R, H, pages], ascending, -1 after the last."""
    B, R, Hq, D = q.shape
    H = pool["k"].shape[2]
    G = Hq // H
    sel = np.full((B, R, H, pages), -1, np.int32)
    for b in range(B):
        num = -(-int(ctx[b]) // PAGE)
        for j in range(R):
            for h in range(H):
                if num <= pages:
                    sel[b, j, h, :num] = np.arange(num)
                    continue
                x = q[b, j, h * G:(h + 1) * G].astype(np.float64)
                fin = np.isfinite(x)
                a = pow2(float(np.max(np.abs(np.where(fin, x, 0)))), 127.0)
                qi = np.rint(np.where(fin, x, 0) / a).astype(np.int64)
                score = np.empty(num)
                for p in range(num):
                    ph = table[b][p]
                    score[p] = np.max(qi @ pool["summary"][layer, ph, h].astype(np.int64)) * pool["summary_scale"][layer, ph, h]
                forced = set(range(sink)) | set(range(num - recent, num))
                rest = sorted((p for p in range(num) if p not in forced), key=lambda p: (-score[p], p))
                chosen = sorted(forced | set(rest[:pages - len(forced)]))
                sel[b, j, h, :len(chosen)] = chosen
    return sel


def attention(q, kb, vb, pool, layer, table, ctx, sel=None, full=False, scale=None):
    """q [B, R, Hq, D], block kb / vb [B, R, H, D] -> (out [B, R, Hq, D], the sum of p |v| in the same
    places, which bounds what rounding the weights p can do)."""
    B, R, Hq, D = q.shape
    H = kb.shape[2]
    G = Hq // H
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        C = int(ctx[b])
        num = -(-C // PAGE)
        for h in range(H):
            def cached(pages):
                ks, vs = [], []
                for p in pages:
                    ph, n = int(table[b][p]), min(PAGE, C - p * PAGE)
                    ks.append(CODES[pool["k"][layer, ph, h, :n]] * pool["scale"][layer, ph, h, 0])
                    vs.append(CODES[pool["v"][layer, ph, h, :, :n]].T * pool["scale"][layer, ph, h, 1])
                return (np.concatenate(ks), np.concatenate(vs)) if ks else (np.zeros((0, D)), np.zeros((0, D)))

            shared = cached(range(num)) if sel is None else None
            for j in range(R):
                kc, vc = shared if sel is None else cached([p for p in sel[b, j, h] if p >= 0])
                m = R if full else j + 1
                kk = np.concatenate([kc, kb[b, :m, h].astype(np.float64)])
                vv = np.concatenate([vc, vb[b, :m, h].astype(np.float64)])
                s = q[b, j, h * G:(h + 1) * G].astype(np.float64) @ kk.T * scale
                e = np.exp(s - s.max(axis=1, keepdims=True))
                p = e / e.sum(axis=1, keepdims=True)
                out[b, j, h * G:(h + 1) * G] = p @ vv
                mag[b, j, h * G:(h + 1) * G] = p @ np.abs(vv)
    return out, mag
