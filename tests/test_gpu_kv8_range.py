"""Attention over the 8-bit cache where values of one head differ by far more than f16's range, against the float64 oracle.

A page (or a token, a channel, a block row) of huge values that the softmax passes over, or whose small weight makes it
count as much as the rest, must leave everything else as precise as ever.  Tolerance as in the attention's other tests, from
the roundings: weights to bf16 at worst (2^-8 of each product), the output to bf16 (2^-8), scores in fp32 below 2^-12 of
it: within 2^-8 (|o| + sum p |v|), channel by channel."""
import math

import numpy as np
import pytest
import torch

from oracle import cospec_kv8 as K
from paper_2605_24793_gb300 import build as BLD
from paper_2605_24793_gb300 import cospec as C

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")
PULL = 8.0                             # channel 0 of every query


@pytest.fixture(scope="module", autouse=True)
def lib():
    C.load_library(BLD.build())
    torch.cuda.set_device(0)
    C.get_device_error()


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _key(bits, D):
    """Channel 0 of a key whose weight is 2^-bits beside the others' ordinary ones."""
    return -bits * math.log(2.0) * math.sqrt(D) / PULL


def _inputs(rng, ctx, R, Hq, H, D):
    B, T = len(ctx), max(ctx)
    k, v = rng.standard_normal((2, B, T, H, D))
    q, kb, vb = rng.standard_normal((B, R, Hq, D)), rng.standard_normal((B, R, H, D)), rng.standard_normal((B, R, H, D))
    q[..., 0] = PULL
    k[..., 0] = kb[..., 0] = 0
    return k, v, q, kb, vb


def _check(k, v, q, kb, vb, ctx, what, sel=None, full=False):
    B, T, H, D = k.shape
    rng = np.random.default_rng(1)
    width = -(-T // 16)
    table = rng.permutation(B * width).reshape(B, width).astype(np.int32)
    pool, ref = C.new_kv8_pool(1, B * width, H, D), K.new_pool(1, B * width, H, D)
    kt, vt, q, kb, vb = (_dev(x) for x in (k[None], v[None], q, kb, vb))
    ints = lambda x: torch.tensor(np.asarray(x), **I32)  # noqa: E731
    C.kv8_append(pool, kt, vt, ints(table), ints([0] * B), ints(ctx))
    K.append(ref, _np(kt), _np(vt), table, [0] * B, ctx)
    out = torch.full(q.shape, math.nan, dtype=torch.bfloat16, device="cuda")
    C.kv8_attn(q, kb, vb, pool, 0, ints(table), ints(ctx), out, max(ctx), sel=None if sel is None else ints(sel), block_full=full)
    assert C.get_device_error() == 0
    o, mag = K.attention(_np(q), _np(kb), _np(vb), ref, 0, table, ctx, sel=sel, full=full)
    err = np.abs(_np(out) - o)
    bound = 2.0 ** -8 * (np.abs(o) + mag)
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.nanmax(err / bound):.3g} of the bound, {np.isnan(err).sum()} NaN"


# rows per KV head of every form on mma.sync: 1, 8 (columns), 12 (rows), 24 (columns), 32 (two plans by context)
SHAPES = [(1, 2, 2, 128), (2, 8, 2, 64), (3, 8, 2, 128), (6, 8, 2, 128), (8, 8, 2, 128), (8, 4, 1, 64)]
UNEVEN = [(12, 100), (20, 100), (24, 100), (32, 100), (60, 100), (30, 60), (40, 40), (60, 60), (100, 100), (120, 200), (-30, 0), (-60, 0)]


@pytest.mark.parametrize("R,Hq,H,D", SHAPES)
@pytest.mark.parametrize("n,bits", UNEVEN)
def test_a_page_far_from_the_others(R, Hq, H, D, n, bits):
    """One page's values 2^n times the others', its weight 2^-bits: first, in the middle, last, and two of them side by side."""
    rng = np.random.default_rng(1000 * R + Hq + n + bits)
    ctx = [700, 45]
    for pages in ((0,), (1,), (20,), (42,), (43,), (2, 3, 30)):
        k, v, q, kb, vb = _inputs(rng, ctx, R, Hq, H, D)
        for p in pages:
            k[0, p * 16:p * 16 + 16, :, 0] = _key(bits, D)
            v[0, p * 16:p * 16 + 16] *= 2.0 ** n
        _check(k, v, q, kb, vb, ctx, f"pages {pages}")


@pytest.mark.parametrize("R,Hq,H,D", SHAPES)
@pytest.mark.parametrize("n", [16, 30, 60])
def test_a_token_and_a_channel_far_from_the_others(R, Hq, H, D, n):
    """A token that the softmax passes over, beside whose values its page's others are held as 0 and keep their weights; and
    one with an ordinary weight, huge in a single channel."""
    rng = np.random.default_rng(2000 * R + Hq + n)
    ctx = [300, 45]
    k, v, q, kb, vb = _inputs(rng, ctx, R, Hq, H, D)
    k[0, 83, :, 0] = _key(120, D)
    v[0, 83] *= 2.0 ** n
    _check(k, v, q, kb, vb, ctx, "token")
    k, v, q, kb, vb = _inputs(rng, ctx, R, Hq, H, D)
    v[0, 83, :, 5] *= 2.0 ** n
    v[1, 3, :, 7] *= 2.0 ** n
    _check(k, v, q, kb, vb, ctx, "channel")


@pytest.mark.parametrize("R,Hq,H,D", SHAPES)
@pytest.mark.parametrize("n", [30, 60])
def test_every_page_but_one_far_above(R, Hq, H, D, n):
    """The one page of ordinary values has the weight: the smallest scale decides what has to be kept."""
    rng = np.random.default_rng(3000 * R + Hq + n)
    ctx = [500, 45]
    for page in (0, 7, 31):
        k, v, q, kb, vb = _inputs(rng, ctx, R, Hq, H, D)
        v *= 2.0 ** n
        k[..., 0] = _key(100, D)
        k[0, page * 16:page * 16 + 16, :, 0] = 0
        v[0, page * 16:page * 16 + 16] *= 2.0 ** -n
        kb[..., 0] = _key(100, D)
        _check(k, v, q, kb, vb, ctx, f"page {page}")


@pytest.mark.parametrize("R,Hq,H,D", SHAPES)
def test_pages_of_every_magnitude_and_of_zeros(R, Hq, H, D):
    """Scales that climb by 2^6 a page while the weights fall alike, that lie anywhere, and pages of zeros between."""
    rng = np.random.default_rng(4000 * R + Hq)
    ctx = [640, 45]
    for kind in ("climb", "fall", "any", "zeros"):
        k, v, q, kb, vb = _inputs(rng, ctx, R, Hq, H, D)
        for p in range(40):
            at = slice(p * 16, p * 16 + 16)
            e = {"climb": 2.5 * p, "fall": 100 - 2.5 * p, "any": float(rng.integers(-60, 60)), "zeros": 0.0}[kind]
            v[0, at] *= 2.0 ** round(e)
            k[0, at, :, 0] = _key(round(e) if kind != "any" else int(rng.integers(0, 80)), D)
            if kind == "zeros" and p % 5 in (0, 1):
                v[0, at] = 0
        _check(k, v, q, kb, vb, ctx, kind)


@pytest.mark.parametrize("R,Hq,H,D", [s for s in SHAPES if s[0] > 1])
@pytest.mark.parametrize("n", [12, 40, 100])
def test_block_rows_far_from_the_cache(R, Hq, H, D, n):
    """A block row of huge values: hidden from the rows before it, seen with next to no weight, or seen by all of a full block; and
    a block of small ones."""
    rng = np.random.default_rng(5000 * R + Hq + n)
    ctx = [200, 0, 45]
    for full in (False, True):
        k, v, q, kb, vb = _inputs(rng, ctx, R, Hq, H, D)
        vb[:, R - 1] *= 2.0 ** n
        kb[0, R - 1, :, 0] = _key(100, D)
        _check(k, v, q, kb, vb, ctx, f"full {full}", full=full)
    k, v, q, kb, vb = _inputs(rng, ctx, R, Hq, H, D)
    vb *= 2.0 ** -n
    _check(k, v, q, kb, vb, ctx, "small")


@pytest.mark.parametrize("R,Hq,H,D", [(1, 2, 2, 128), (3, 24, 2, 128), (2, 40, 2, 64), (2, 64, 2, 128), (2, 72, 1, 64)])
@pytest.mark.parametrize("n,bits", [(24, 100), (40, 40), (-30, 0)])
def test_selected_pages_far_from_the_others(R, Hq, H, D, n, bits):
    rng = np.random.default_rng(6000 * R + Hq + n)
    ctx = [700, 45]
    sel = np.full((2, R, H, 12), -1, np.int32)
    sel[0] = np.sort(np.concatenate([[0, 20, 43], rng.choice(np.arange(1, 20), 9, replace=False)]))
    sel[1, ..., :3] = (0, 1, 2)
    for pages in ((0,), (20,), (43,), (0, 20)):
        k, v, q, kb, vb = _inputs(rng, ctx, R, Hq, H, D)
        for p in pages:
            k[0, p * 16:p * 16 + 16, :, 0] = _key(bits, D)
            v[0, p * 16:p * 16 + 16] *= 2.0 ** n
        _check(k, v, q, kb, vb, ctx, f"pages {pages}", sel=sel)


# ---------------------------------------------------------------- above 32 rows per KV head: tcgen05
TC_SHAPES = [(10, 16, 4, 64), (26, 8, 2, 128), (64, 4, 2, 64), (64, 8, 2, 128)]


@pytest.mark.parametrize("R,Hq,H,D", TC_SHAPES)
@pytest.mark.parametrize("n,bits", UNEVEN)
def test_a_page_far_from_the_others_above_32_rows(R, Hq, H, D, n, bits):
    test_a_page_far_from_the_others(R, Hq, H, D, n, bits)


@pytest.mark.parametrize("R,Hq,H,D", TC_SHAPES)
@pytest.mark.parametrize("n", [16, 30, 60])
def test_a_token_and_a_channel_far_from_the_others_above_32_rows(R, Hq, H, D, n):
    test_a_token_and_a_channel_far_from_the_others(R, Hq, H, D, n)


@pytest.mark.parametrize("R,Hq,H,D", TC_SHAPES)
def test_pages_of_every_magnitude_above_32_rows(R, Hq, H, D):
    for n in (30, 60):
        test_every_page_but_one_far_above(R, Hq, H, D, n)
    test_pages_of_every_magnitude_and_of_zeros(R, Hq, H, D)


@pytest.mark.parametrize("R,Hq,H,D", TC_SHAPES)
@pytest.mark.parametrize("n", [12, 40, 100])
def test_block_rows_far_from_the_cache_above_32_rows(R, Hq, H, D, n):
    test_block_rows_far_from_the_cache(R, Hq, H, D, n)


@pytest.mark.parametrize("R,Hq,H,D", [(3, 8, 2, 128), (8, 8, 2, 64)] + TC_SHAPES)
@pytest.mark.parametrize("n", [12, 40, 70])
def test_a_block_key_far_from_the_others(R, Hq, H, D, n):
    """A key of the block 2^n times the rest, hidden from the rows before it: their scores stay as precise as ever."""
    rng = np.random.default_rng(7000 * R + Hq + n)
    ctx = [100, 0, 45]
    k, v, q, kb, vb = _inputs(rng, ctx, R, Hq, H, D)
    kb[:, R - 1] *= 2.0 ** n
    kb[:, R - 1, :, 0] = _key(200, D) * 2.0 ** n           # (and its own row passes it over)
    _check(k, v, q, kb, vb, ctx, "hidden")


@pytest.mark.parametrize("R,Hq,H,D", SHAPES + TC_SHAPES + [(1, 8, 1, 64), (26, 16, 4, 64)])
@pytest.mark.parametrize("n", [120, 124, -90, -104])
def test_values_near_the_types_ends(R, Hq, H, D, n):
    """All values 2^n times ordinary ones: their sums before the division leave fp32, the result does not."""
    rng = np.random.default_rng(8000 * R + Hq + n + 200)
    for ctx in ([700, 45], [2000, 0]):
        k, v, q, kb, vb = _inputs(rng, ctx, R, Hq, H, D)
        _check(k, v * 2.0 ** n, q, kb, vb * 2.0 ** n, ctx, f"contexts {ctx}")


@pytest.mark.parametrize("R,Hq,H,D", [(3, 24, 2, 128), (1, 2, 2, 64)])
def test_selected_values_near_the_types_end(R, Hq, H, D):
    rng = np.random.default_rng(9000 * R)
    ctx = [700, 45]
    sel = np.full((2, R, H, 40), -1, np.int32)
    sel[0] = np.arange(4, 44)
    sel[1, ..., :3] = (0, 1, 2)
    k, v, q, kb, vb = _inputs(rng, ctx, R, Hq, H, D)
    _check(k, v * 2.0 ** 124, q, kb, vb * 2.0 ** 124, ctx, "sel", sel=sel)
