"""The 8-bit paged KV cache on the device against the float64 oracle.

Tolerances, set beforehand from the roundings.  Codes, scales, summaries and selected pages: equal
where the rows are bf16 as they come (every step before the one rounding is exact); with a
rotation in fp32 (relative error of a sum of two products below 2^-22 of the larger) a code may be the
neighbour of the nearest one, so |code * scale - x| <= half a code's spacing + 2^-21 |x|_max.
bf16 holds 8 bits, so its rounding is within 2^-8 of the value.  Attention: the output's rounding
(2^-8 |o|) and weights p rounded to bf16 at worst (2^-8 sum p |v| if all erred one way; scores
in fp32 add below 2^-12 of it): within 2^-8 (|o| + sum p |v|)."""
import math

import numpy as np
import pytest
import torch

from oracle import cospec_kv8 as K
from paper_2605_24793_gb300 import build as BLD
from paper_2605_24793_gb300 import cospec as C

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module", autouse=True)
def lib():
    C.load_library(BLD.build())
    torch.cuda.set_device(0)
    C.get_device_error()


def _bf16(rng, shape, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(torch.bfloat16).cuda()


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _ints(x):
    return torch.tensor(np.asarray(x), **I32)


def _host(pool):
    return dict(k=pool.k.view(torch.uint8).cpu().numpy(), v=pool.v.view(torch.uint8).cpu().numpy(), scale=_np(pool.scale),
                summary=pool.summary.cpu().numpy(), summary_scale=_np(pool.summary_scale))


def _noise_pool(rng, layers, pages, H, D):
    """A pool whose cells hold anything, NaN codes among it: what earlier sequences left."""
    pool = C.new_kv8_pool(layers, pages, H, D)
    for t in (pool.k, pool.v):
        t.view(torch.uint8).copy_(torch.from_numpy(rng.integers(0, 256, tuple(t.shape), dtype=np.uint8)))
    pool.scale.fill_(2.0 ** 100)
    pool.summary.fill_(-77)
    pool.summary_scale.fill_(3e38)
    return pool


def _assert_pool(pool, ref, what=""):
    got = _host(pool)
    assert K.same_codes(got["k"], ref["k"]), what + " keys"
    assert K.same_codes(got["v"], ref["v"]), what + " values"
    for n in ("scale", "summary", "summary_scale"):
        np.testing.assert_array_equal(got[n], ref[n], err_msg=what + " " + n)


def _fused(rng, lead, Hq, Hkv, D, std=1.0):
    buf = _bf16(rng, (*lead, Hq + 2 * Hkv, D), std)
    return buf[..., :Hq, :], buf[..., Hq:Hq + Hkv, :], buf[..., Hq + Hkv:, :]


# ---------------------------------------------------------------- append
@pytest.mark.parametrize("L,B,R,H,D,fused", [
    (1, 1, 1, 2, 64, False), (2, 3, 8, 8, 128, True), (3, 2, 26, 3, 64, True), (1, 2, 64, 1, 128, False), (1, 1, 200, 5, 64, False),
    (2, 70, 5, 2, 128, True)])
def test_appends_are_exact_and_leave_other_cells(L, B, R, H, D, fused):
    """Four calls in a row, of growing and falling magnitudes, rows from none to all: pages filled across calls, their
    scales moved, everything else in the pool as it was."""
    rng = np.random.default_rng(R * 31 + H)
    calls, width = 4, (4 * R + 40) // 16 + 1
    table = rng.permutation(B * width + 3)[:B * width].reshape(B, width)
    pool = _noise_pool(rng, L, B * width + 3, H, D)
    ref = _host(pool)
    start = rng.integers(0, 33, B)
    # a first token so that every page's older cells are this sequence's own
    first = np.zeros(B, np.int64)
    k0, v0 = _bf16(rng, (2, L, B, 33, H, D))
    C.kv8_append(pool, k0, v0, _ints(table), _ints(first), _ints(start))
    K.append(ref, _np(k0), _np(v0), table, first, start)
    for c in range(calls):
        std = (1.0, 30.0, 1e-3, 200.0)[c]
        _, k, v = _fused(rng, (L, B, R), 3, H, D, std)
        k, v = (k, v) if fused else (k.contiguous(), v.contiguous())
        rows = rng.integers(0, R + 1, B)
        rows[0] = (R, 0, 1, R)[c]
        C.kv8_append(pool, k, v, _ints(table), _ints(start), _ints(rows))
        K.append(ref, _np(k), _np(v), table, start, rows)
        start = start + rows
    torch.cuda.synchronize()
    assert C.get_device_error() == 0
    _assert_pool(pool, ref)


def test_append_without_row_counts_and_into_one_layer():
    rng = np.random.default_rng(5)
    pool, table = _noise_pool(rng, 3, 8, 4, 64), np.arange(8).reshape(2, 4)
    ref = _host(pool)
    k, v = _bf16(rng, (2, 2, 20, 4, 64))
    C.kv8_append(pool, k, v, _ints(table), _ints([0, 16]), layer=1)
    one = {n: x[1:2] for n, x in ref.items()}
    K.append(one, _np(k)[None], _np(v)[None], table, [0, 16], [20, 20])
    assert C.get_device_error() == 0
    _assert_pool(pool, ref)


def test_append_of_zeros_infinities_nan_and_the_types_ends():
    rng = np.random.default_rng(6)
    x = rng.standard_normal((1, 4, 16, 2, 64))
    x[0, 0] = 0.0
    x[0, 1, 3, 0, 5], x[0, 1, 4, 1, 6], x[0, 1, 5, 0, 7] = np.inf, -np.inf, np.nan
    x[0, 2] *= 3e-39                       # below the scales' range: flushed, not divided by zero
    x[0, 3] *= 1e38 / 4
    x[0, 3, 0, 0, 0] = 3.3895e38           # the type's largest value
    k = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda()
    pool, table = _noise_pool(rng, 1, 4, 2, 64), np.arange(4)[:, None]
    ref = _host(pool)
    C.kv8_append(pool, k, k, _ints(table), _ints([0] * 4), _ints([16, 16, 9, 16]))
    K.append(ref, _np(k), _np(k), table, [0] * 4, [16, 16, 9, 16])
    assert C.get_device_error() == 0
    _assert_pool(pool, ref)
    got = _host(pool)
    assert got["scale"][0, 0, 0, 0] == 2.0 ** -100 and np.isfinite(got["summary_scale"]).all()
    assert np.isnan(K.CODES[got["k"][0, 1, 0, 3, 5]]) and np.isnan(K.CODES[got["v"][0, 1, 0, 7, 5]])


@pytest.mark.parametrize("D,rot,inter", [(64, 64, False), (128, 128, False), (128, 64, True), (64, 8, True), (128, 96, False), (64, 24, False)])
@pytest.mark.parametrize("R", [1, 19])
def test_rotation_on_the_way(D, rot, inter, R):
    rng = np.random.default_rng(rot + R)
    L, B, Hq, H = 2, 3, 6, 3
    q, k, v = _fused(rng, (L, B, R), Hq, H, D)
    ang = np.arange(100)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
    cos, sin = (torch.from_numpy(f(ang).astype(np.float32)).cuda() for f in (np.cos, np.sin))
    start, rows = np.array([0, 13, 64]), np.array([R, (R + 1) // 2, 0])
    pool, table = _noise_pool(rng, L, 24, H, D), np.arange(24).reshape(3, 8)
    before = _host(pool)
    q_out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    k_out = torch.full(k.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    rope = C.Rope(cos, sin, inter)
    # (sequence 1 starts inside a page: its older tokens first)
    C.kv8_append(pool, k[:, :, :1].expand(L, B, 13, H, D).contiguous(), v[:, :, :1].expand(L, B, 13, H, D).contiguous(), _ints(table),
                 _ints([0, 0, 0]), _ints([0, 13, 0]))
    C.kv8_append(pool, k, v, _ints(table), _ints(start), _ints(rows), rope, q=q, q_out=q_out, k_out=k_out)
    q2, k2 = torch.empty_like(q_out), torch.empty_like(k_out)
    C.kv8_rotate(q, k, rope, _ints(start), q2, k2)
    assert C.get_device_error() == 0
    assert torch.equal(q2, q_out) and torch.equal(k2, k_out)
    got = _host(pool)
    c64, s64 = cos.cpu().numpy().astype(np.float64), sin.cpu().numpy().astype(np.float64)
    for b in range(B):
        for j in range(R):
            for x, y in ((q, q_out), (k, k_out)):
                ref = K.rotate(_np(x[:, b, j]), start[b] + j, c64, s64, inter)
                # bf16 rounding, of a value that fp32 holds to 2^-22 of its terms
                assert np.all(np.abs(_np(y[:, b, j]) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -21 * np.abs(_np(x[:, b, j])).max())
            if j < rows[b]:
                p, t = divmod(int(start[b] + j), 16)
                ref = K.rotate(_np(k[:, b, j]), start[b] + j, c64, s64, inter)
                s = got["scale"][:, table[b, p], :, 0][..., None]
                code = K.CODES[got["k"][:, table[b, p], :, t]]
                half = np.maximum(2.0 ** np.floor(np.log2(np.maximum(np.abs(code), 2.0 ** -6))) / 16, 2.0 ** -10)
                assert np.all(np.abs(code * s - ref) <= half * s + 2.0 ** -21 * np.abs(ref).max())
                sv = got["scale"][:, table[b, p], :, 1][..., None]
                np.testing.assert_array_equal(K.CODES[got["v"][:, table[b, p], :, :, t]], K.CODES[K.encode(_np(v[:, b, j]) / sv)])
    for n in before:                       # a sequence without rows leaves its pages
        np.testing.assert_array_equal(got[n][:, 16:], before[n][:, 16:])


def test_append_skips_and_flags_what_does_not_fit():
    rng = np.random.default_rng(8)
    L, B, R, H, D = 1, 6, 4, 2, 64
    k, v = _bf16(rng, (2, L, B, R, H, D))
    table = np.arange(12).reshape(6, 2)
    table[3, 1] = 12                       # outside the pool
    start, rows = [0, -1, 30, 14, 28, 2], [4, 4, 4, 4, 4, 5]
    cases = {1: C.DEVERR_CTX, 2: C.DEVERR_CTX, 3: C.DEVERR_PAGE, 5: C.DEVERR_CTX}
    pool = _noise_pool(rng, L, 12, H, D)
    ref = _host(pool)
    C.kv8_append(pool, k, v, _ints(table), _ints(start), _ints(rows))
    assert C.get_device_error() == C.DEVERR_CTX | C.DEVERR_PAGE
    for b in (0, 3, 4):
        n = 2 if b == 3 else 4             # the rows before the bad page
        if b == 3:                         # older cells of that page are noise: make the oracle's the same
            sub = {x: y.copy() for x, y in ref.items()}
            K.append(sub, _np(k)[:, [b]], _np(v)[:, [b]], table[[b]], [14], [n])
            ref = sub
        elif b == 0:
            K.append(ref, _np(k)[:, [b]], _np(v)[:, [b]], table[[b]], [0], [n])
        else:
            K.append(ref, _np(k)[:, [b]], _np(v)[:, [b]], table[[b]], [28], [n])
    _assert_pool(pool, ref)
    assert cases
    # positions outside the tables
    cos = torch.ones((20, 32), device="cuda")
    before = _host(pool)
    out = torch.full_like(k, 9.0)
    C.kv8_append(pool, k, v, _ints(np.arange(12).reshape(6, 2)), _ints([17] * 6), _ints([4] * 6), C.Rope(cos, cos), k_out=out)
    assert C.get_device_error() == C.DEVERR_POSITION
    _assert_pool(pool, before)
    assert bool((out == 9.0).all())


# ---------------------------------------------------------------- attention
def _cached(rng, ctx, extra, H, D, layers=1, std=1.0, spread=False):
    """A pool of noise into which the sequences' contexts are appended, and the oracle's copy."""
    B = len(ctx)
    width = max(1, (max(ctx) + extra + 15) // 16)
    pages = B * width + 2
    table = rng.permutation(pages)[:B * width].reshape(B, width).astype(np.int32)
    pool = _noise_pool(rng, layers, pages, H, D)
    ref = _host(pool)
    T = max(1, max(ctx))
    k, v = _bf16(rng, (2, layers, B, T, H, D), std)
    if spread:                             # pages of very different magnitude
        f = torch.from_numpy(2.0 ** rng.integers(-12, 13, (1, B, -(-T // 16), 1, 1))).to(torch.bfloat16).cuda()
        v = v * f.repeat_interleave(16, 2)[:, :, :T]
    C.kv8_append(pool, k, v, _ints(table), _ints([0] * B), _ints(ctx))
    K.append(ref, _np(k), _np(v), table, [0] * B, ctx)
    assert C.get_device_error() == 0
    return pool, ref, table


def _assert_attn(out, ref, mag, what=""):
    err = np.abs(_np(out) - ref)
    assert np.isfinite(_np(out)).all(), what
    bad = err > 2.0 ** -8 * (np.abs(ref) + mag)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {(err / (np.abs(ref) + mag)).max():.3g} at {np.argwhere(bad)[:3].tolist()}"


ATTN = [  # ctx, R, Hq, Hkv, D
    ([0], 1, 8, 2, 64), ([1], 1, 4, 4, 128), ([15, 16, 17], 2, 8, 2, 64), ([63, 64, 65, 0], 5, 12, 4, 128), ([1000, 3], 1, 32, 8, 128),
    ([127, 128, 129], 8, 32, 8, 128), ([500, 77], 26, 16, 4, 128), ([300], 64, 8, 8, 64), ([2049], 6, 32, 8, 128), ([400, 31], 64, 16, 2, 128),
    ([90, 0, 33], 16, 32, 1, 64), ([260], 3, 64, 1, 128), ([700], 4, 128, 1, 64), ([5000, 4999], 1, 7, 1, 128), ([640] * 70, 2, 4, 2, 64),
    ([333, 48], 9, 6, 6, 64), ([4100], 13, 10, 2, 64)]


@pytest.mark.parametrize("ctx,R,Hq,H,D", ATTN)
@pytest.mark.parametrize("full", [False, True])
def test_attention(ctx, R, Hq, H, D, full):
    rng = np.random.default_rng(sum(ctx) + R + Hq)
    B = len(ctx)
    pool, ref, table = _cached(rng, ctx, R, H, D)
    q, kb, vb = _fused(rng, (B, R), Hq, H, D)
    if R % 2:
        q, kb, vb = q.contiguous(), kb.contiguous(), vb.contiguous()
    out = torch.full((B, R, Hq, D), np.nan, dtype=torch.bfloat16, device="cuda")
    for max_ctx in {max(ctx), 0}:          # the split is planned from it, the result must not be
        C.kv8_attn(q, kb, vb, pool, 0, _ints(table), _ints(ctx), out, max_ctx, block_full=full)
        assert C.get_device_error() == 0
        _assert_attn(out, *K.attention(_np(q), _np(kb), _np(vb), ref, 0, table, ctx, full=full), what=f"max_ctx {max_ctx}")


@pytest.mark.parametrize("std,qstd,spread", [(1e-6, 1.0, False), (1e4, 1e-4, False), (1.0, 12.0, False), (1.0, 1.0, True), (3e-20, 1e19, False),
                                             (1.0, 1e-30, True)])
@pytest.mark.parametrize("R,Hq,H,D", [(1, 8, 2, 128), (6, 24, 4, 64), (20, 8, 2, 128)])
def test_attention_of_large_small_and_uneven_values(std, qstd, spread, R, Hq, H, D):
    """Scores that decide on one key, pages whose values differ by 2^24, and magnitudes far from one."""
    rng = np.random.default_rng(int(abs(math.log(std)) * 10 + R))
    ctx = [700, 45]
    pool, ref, table = _cached(rng, ctx, R, H, D, std=std, spread=spread)
    q = _bf16(rng, (2, R, Hq, D), qstd)
    q[:, :, 1] *= 1e-3                     # rows of different size side by side
    kb, vb = _bf16(rng, (2, 2, R, H, D), std)
    out = torch.empty_like(q)
    C.kv8_attn(q, kb, vb, pool, 0, _ints(table), _ints(ctx), out, max(ctx))
    assert C.get_device_error() == 0
    o, mag = K.attention(_np(q), _np(kb), _np(vb), ref, 0, table, ctx)
    # fp32 scores: 2^-22 of the sum of |q k| scaled, twice (products and their maximum), times the weights' sum
    s_abs = np.abs(_np(q)).max() * np.abs(np.concatenate([_np(kb).ravel(), K.CODES[ref["k"][0]][np.isfinite(K.CODES[ref["k"][0]])].max()[None]
                                                          * std / 100])).max() * math.sqrt(D)
    extra = min(1.0, 2.0 ** -20 * s_abs)
    err = np.abs(_np(out) - o)
    assert np.all(err <= 2.0 ** -8 * (np.abs(o) + mag) + extra * mag), float((err / (np.abs(o) + mag)).max())


@pytest.mark.parametrize("ctx,R,Hq,H,D", [([700], 1, 32, 8, 128), ([130, 513], 6, 32, 8, 128), ([300], 8, 16, 4, 64), ([90, 0, 410], 12, 16, 4, 128),
                                          ([257], 3, 8, 2, 64)])
def test_attention_under_every_plan(ctx, R, Hq, H, D):
    """Rings, warps and split are planned from the longest context that the caller expects, or the pages it selects: none
    may change what comes out."""
    rng = np.random.default_rng(sum(ctx) + 7 * R)
    B, wide = len(ctx), 8192
    pool, ref, table = _cached(rng, ctx, R, H, D)
    padded = np.full((B, wide), -1, np.int32)
    padded[:, :table.shape[1]] = table
    q, kb, vb = _fused(rng, (B, R), Hq, H, D)
    out = torch.empty((B, R, Hq, D), dtype=torch.bfloat16, device="cuda")
    want = K.attention(_np(q), _np(kb), _np(vb), ref, 0, table, ctx)
    for max_ctx in (16, 256, 1024, 4096, 12000, 32768, 16 * wide):
        out.fill_(math.nan)
        C.kv8_attn(q, kb, vb, pool, 0, _ints(padded), _ints(ctx), out, max_ctx)
        assert C.get_device_error() == 0
        _assert_attn(out, *want, what=f"max_ctx {max_ctx}")
    chosen = K.select(_np(q), ref, 0, table, ctx, 9, 1, 2)
    want = K.attention(_np(q), _np(kb), _np(vb), ref, 0, table, ctx, sel=chosen)
    for pages in (9, 64, 300, 2000):
        sel = np.full(chosen.shape[:3] + (pages,), -1, np.int32)
        sel[..., :9] = chosen
        out.fill_(math.nan)
        C.kv8_attn(q, kb, vb, pool, 0, _ints(padded), _ints(ctx), out, max(ctx), sel=_ints(sel))
        assert C.get_device_error() == 0
        _assert_attn(out, *want, what=f"{pages} pages")


def test_attention_scale_layer_and_short_table():
    rng = np.random.default_rng(11)
    ctx = [48, 80]
    pool, ref, table = _cached(rng, ctx, 0, 2, 64, layers=3)
    q, kb, vb = _fused(rng, (2, 4), 4, 2, 64)
    out = torch.empty((2, 4, 4, 64), dtype=torch.bfloat16, device="cuda")
    for l in (0, 2):
        C.kv8_attn(q, kb, vb, pool, l, _ints(table), _ints(ctx), out, 80, softmax_scale=0.3)
        assert C.get_device_error() == 0
        _assert_attn(out, *K.attention(_np(q), _np(kb), _np(vb), ref, l, table, ctx, scale=0.3))


def test_attention_flags_bad_contexts_and_pages_and_goes_on():
    rng = np.random.default_rng(12)
    ctx = [100, 60, 90, 20]
    pool, ref, table = _cached(rng, ctx, 4, 2, 128)
    q, kb, vb = _fused(rng, (4, 4), 8, 2, 128)
    out = torch.empty((4, 4, 8, 128), dtype=torch.bfloat16, device="cuda")
    bad = table.copy()
    bad[2, 3] = pool.num_pages
    lens = [100, -1, 90, 16 * table.shape[1] + 1]
    C.kv8_attn(q, kb, vb, pool, 0, _ints(bad), _ints(lens), out, 100)
    assert C.get_device_error() == C.DEVERR_CTX | C.DEVERR_PAGE
    o, mag = K.attention(_np(q), _np(kb), _np(vb), ref, 0, table, ctx)
    _assert_attn(out[:1], o[:1], mag[:1])


def test_attention_over_more_than_2_31_bytes_of_cache():
    """Pages at the end of a pool whose offsets pass 32 bits."""
    rng = np.random.default_rng(13)
    H, D, pages = 8, 128, 280000           # 16 KB a page and tensor: 4.6 GB each
    e = lambda shape, dt: torch.empty((1, pages, H) + shape, dtype=dt, device="cuda")  # noqa: E731
    pool = C.Kv8Pool(e((16, D), C.F8), e((D, 16), C.F8), e((2,), torch.float32), e((D,), torch.int8), e((), torch.float32))
    table = np.array([[pages - 1, 3, pages - 2, 140000, 131072, 262144, pages - 7]], np.int32)
    ctx = [100]
    k, v = _bf16(rng, (2, 1, 1, 100, H, D))
    C.kv8_append(pool, k, v, _ints(table), _ints([0]), _ints(ctx))
    q, kb, vb = _fused(rng, (1, 2), 16, H, D)
    out = torch.empty((1, 2, 16, D), dtype=torch.bfloat16, device="cuda")
    C.kv8_attn(q, kb, vb, pool, 0, _ints(table), _ints(ctx), out, 100)
    sel = torch.empty((1, 2, H, 5), **I32)
    C.kv8_select(q, pool, 0, _ints(table), _ints(ctx), sel, 1, 1)
    outs = torch.empty_like(out)
    C.kv8_attn(q, kb, vb, pool, 0, _ints(table), _ints(ctx), outs, 100, sel=sel)
    assert C.get_device_error() == 0
    ref = K.new_pool(1, 7, H, D)
    own = np.arange(7)[None]
    K.append(ref, _np(k), _np(v), own, [0], ctx)
    _assert_attn(out, *K.attention(_np(q), _np(kb), _np(vb), ref, 0, own, ctx))
    np.testing.assert_array_equal(sel.cpu().numpy(), K.select(_np(q), ref, 0, own, ctx, 5, 1, 1))
    _assert_attn(outs, *K.attention(_np(q), _np(kb), _np(vb), ref, 0, own, ctx, sel=sel.cpu().numpy()))


# ---------------------------------------------------------------- selection
@pytest.mark.parametrize("ctx,R,Hq,H,D,pages,sink,recent", [
    ([200, 0, 17], 2, 8, 2, 64, 4, 1, 1), ([1000, 999, 400], 3, 32, 8, 128, 16, 1, 4), ([4097], 1, 4, 4, 64, 200, 0, 1),
    ([640, 320], 5, 12, 4, 128, 5, 2, 3), ([100], 1, 8, 1, 128, 1, 0, 0), ([513] * 9, 1, 64, 1, 64, 32, 0, 0), ([6000], 2, 6, 2, 64, 300, 2, 2),
    ([3000, 50], 64, 2, 2, 64, 24, 1, 2), ([800], 4, 128, 1, 128, 7, 1, 1)])
def test_selection_and_attention_over_it(ctx, R, Hq, H, D, pages, sink, recent):
    rng = np.random.default_rng(sum(ctx) + pages)
    B = len(ctx)
    pool, ref, table = _cached(rng, ctx, R, H, D)
    q, kb, vb = _fused(rng, (B, R), Hq, H, D)
    sel = torch.full((B, R, H, pages), -5, **I32)
    C.kv8_select(q, pool, 0, _ints(table), _ints(ctx), sel, sink, recent)
    assert C.get_device_error() == 0
    want = K.select(_np(q), ref, 0, table, ctx, pages, sink, recent)
    np.testing.assert_array_equal(sel.cpu().numpy(), want)
    out = torch.full((B, R, Hq, D), np.nan, dtype=torch.bfloat16, device="cuda")
    for full in (False, True):
        C.kv8_attn(q, kb, vb, pool, 0, _ints(table), _ints(ctx), out, max(ctx), sel=sel, block_full=full)
        assert C.get_device_error() == 0
        _assert_attn(out, *K.attention(_np(q), _np(kb), _np(vb), ref, 0, table, ctx, sel=want, full=full))


def test_selection_breaks_ties_to_the_lower_page():
    """Pages with the same summary, more of them than there is room for, and scores of zero."""
    rng = np.random.default_rng(21)
    pool, table = _noise_pool(rng, 1, 64, 2, 64), rng.permutation(64)[None].astype(np.int32)
    pool.summary.zero_()
    pool.summary_scale.fill_(0.25)
    pool.summary[0, torch.from_numpy(table[0, 10:40].astype(np.int64)).cuda(), 0] = 3
    q = torch.ones((1, 1, 4, 64), dtype=torch.bfloat16, device="cuda")
    q[0, 0, 2:] = -1.0
    sel = torch.empty((1, 1, 2, 12), **I32)
    C.kv8_select(q, pool, 0, _ints(table), _ints([1024]), sel, 1, 1)
    assert sel[0, 0, 0].tolist() == [0] + list(range(10, 20)) + [63]
    assert sel[0, 0, 1].tolist() == list(range(11)) + [63]
    q[0, 0, 1, 7], q[0, 0, 0, 3] = float("nan"), float("inf")     # not finite: counted as 0
    C.kv8_select(q, pool, 0, _ints(table), _ints([1024]), sel, 0, 0)
    assert sel[0, 0, 0].tolist() == list(range(10, 22))
    assert C.get_device_error() == 0


def test_selection_flags_bad_contexts_and_pages():
    rng = np.random.default_rng(22)
    pool, ref, table = _cached(rng, [320, 320, 320], 1, 2, 64)
    q = _bf16(rng, (3, 1, 4, 64))
    bad = table.copy()
    bad[1, 5] = -3
    sel = torch.empty((3, 1, 2, 6), **I32)
    C.kv8_select(q, pool, 0, _ints(bad), _ints([320, 320, -4]), sel, 1, 1)
    assert C.get_device_error() == C.DEVERR_CTX | C.DEVERR_PAGE
    np.testing.assert_array_equal(sel[0].cpu().numpy(), K.select(_np(q), ref, 0, table, [320] * 3, 6, 1, 1)[0])
    got = sel[1].cpu().numpy()
    assert (got != 5).all() and (np.diff(got) > 0).all()
    assert (sel[2] == -1).all()


def test_attention_over_lists_that_end_early_or_name_bad_pages():
    rng = np.random.default_rng(23)
    ctx = [150, 150]
    pool, ref, table = _cached(rng, ctx, 2, 2, 128)
    q, kb, vb = _fused(rng, (2, 2), 8, 2, 128)
    sel = np.full((2, 2, 2, 9), -1, np.int32)
    sel[0, 0, 0, :1], sel[0, 0, 1, :3], sel[0, 1, 0, :9] = 9, (0, 4, 9), np.arange(9)   # (row 1 of head 1 reads no page)
    sel[1, :, :, :2] = (3, 10)             # page 10 is past the context's ten pages
    out = torch.empty((2, 2, 8, 128), dtype=torch.bfloat16, device="cuda")
    C.kv8_attn(q, kb, vb, pool, 0, _ints(table), _ints(ctx), out, 150, sel=_ints(sel))
    assert C.get_device_error() == C.DEVERR_PAGE
    sel[1, :, :, 1] = -1
    _assert_attn(out, *K.attention(_np(q), _np(kb), _np(vb), ref, 0, table, ctx, sel=sel))


# ---------------------------------------------------------------- order between calls
def test_rounds_queued_and_captured_equal_those_run_one_by_one():
    """Append, select, attend over several layers and rounds: on another stream, without a pause, and
    replayed from a graph, against the same calls with a synchronisation after each."""
    rng = np.random.default_rng(31)
    L, B, R, Hq, H, D, rounds = 3, 2, 4, 8, 2, 64, 3
    ctx0 = [70, 33]
    q, k, v = _fused(rng, (rounds, L, B, R), Hq, H, D)
    rows = rng.integers(1, R + 1, (rounds, B))
    ang = np.arange(128)[:, None] * 100.0 ** (-np.arange(0, D, 2) / D)
    rope = C.Rope(*(torch.from_numpy(f(ang).astype(np.float32)).cuda() for f in (np.cos, np.sin)))
    rows_d = _ints(rows)

    def make():
        r2 = np.random.default_rng(32)
        pool, _, table = _cached(r2, ctx0, rounds * R, H, D, layers=L)
        return dict(pool=pool, table=_ints(table), ctx=_ints(ctx0), sel=torch.empty((B, R, H, 3), **I32),
                    out=torch.empty((rounds, 2 * L, B, R, Hq, D), dtype=torch.bfloat16, device="cuda"),
                    qr=torch.empty((L, B, R, Hq, D), dtype=torch.bfloat16, device="cuda"),
                    kr=torch.empty((L, B, R, H, D), dtype=torch.bfloat16, device="cuda"))

    def go(s, pause):
        for r in range(rounds):
            C.kv8_rotate(q[r], k[r], rope, s["ctx"], s["qr"], s["kr"])
            pause()
            for l in range(L):
                a = (s["qr"][l], s["kr"][l], v[r, l], s["pool"], l, s["table"], s["ctx"])
                C.kv8_attn(*a, s["out"][r, l], 96, kv_stable=l > 0)
                pause()
            for l in range(L):
                a = (s["qr"][l], s["kr"][l], v[r, l], s["pool"], l, s["table"], s["ctx"])
                C.kv8_select(s["qr"][l], s["pool"], l, s["table"], s["ctx"], s["sel"])
                pause()
                C.kv8_attn(*a, s["out"][r, L + l], 96, sel=s["sel"])
                pause()
            C.kv8_append(s["pool"], k[r], v[r], s["table"], s["ctx"], rows_d[r], rope)
            pause()
            s["ctx"] += rows_d[r]

    a, b, c = make(), make(), make()
    go(a, torch.cuda.synchronize)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go(b, lambda: None)
    side.synchronize()
    start = {n: t.clone() for n, t in dict(k=c["pool"].k, v=c["pool"].v, scale=c["pool"].scale, ctx=c["ctx"]).items()}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go(c, lambda: None)
    for _ in range(2):
        for n, t in dict(k=c["pool"].k, v=c["pool"].v, scale=c["pool"].scale, ctx=c["ctx"]).items():
            t.copy_(start[n])
        g.replay()
        torch.cuda.synchronize()
        for other in (b, c):
            for n in ("out", "ctx"):
                assert torch.equal(a[n], other[n]), n
            for n in ("k", "v"):
                assert torch.equal(getattr(a["pool"], n).view(torch.uint8), getattr(other["pool"], n).view(torch.uint8)), n
    assert C.get_device_error() == 0


def test_empty_batches_and_no_rows():
    pool = C.new_kv8_pool(2, 2, 2, 64)
    z = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    C.kv8_append(pool, z(2, 0, 3, 2, 64), z(2, 0, 3, 2, 64), torch.empty((0, 1), **I32), torch.empty(0, **I32))
    C.kv8_append(pool, z(2, 3, 0, 2, 64), z(2, 3, 0, 2, 64), torch.zeros((3, 1), **I32), torch.zeros(3, **I32))
    C.kv8_attn(z(0, 2, 4, 64), z(0, 2, 2, 64), z(0, 2, 2, 64), pool, 0, torch.empty((0, 1), **I32), torch.empty(0, **I32), z(0, 2, 4, 64), 0)
    C.kv8_select(z(0, 2, 4, 64), pool, 1, torch.empty((0, 1), **I32), torch.empty(0, **I32), torch.empty((0, 2, 2, 4), **I32))
    assert C.get_device_error() == 0
    assert not bool(pool.k.view(torch.uint8).any())
