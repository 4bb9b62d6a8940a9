"""The page selection of the 8-bit cache against the float64 oracle, on summaries written directly: scores at the ends of
fp32, contexts of up to 32768 pages, tables wider than the contexts.  Lists are exact, so they have to be equal."""
import numpy as np
import pytest
import torch

from oracle import cospec_kv8 as K
from paper_2605_24793_gb300 import build as BLD
from paper_2605_24793_gb300 import cospec as C

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")
GUARD = -12345


@pytest.fixture(scope="module", autouse=True)
def lib():
    C.load_library(BLD.build())
    torch.cuda.set_device(0)
    C.get_device_error()


def _pool(rng, pages, H, D):
    """A pool whose summaries alone matter: int8 noise, scales that are powers of two."""
    pool = C.new_kv8_pool(1, pages, H, D)
    pool.summary.copy_(torch.from_numpy(rng.integers(-127, 128, (1, pages, H, D)).astype(np.int8)))
    pool.summary_scale.copy_(torch.from_numpy(2.0 ** rng.integers(-9, -3, (1, pages, H)).astype(np.float32)))
    return pool


def _select(q, pool, table, ctx, pages, sink, recent):
    """The lists, and that nothing was written behind them."""
    B, R, _, _ = q.shape
    n = B * R * pool.kv_heads * pages
    buf = torch.full((n + 4096,), GUARD, **I32)
    sel = buf[:n].view(B, R, pool.kv_heads, pages)
    C.kv8_select(q, pool, 0, torch.tensor(np.asarray(table), **I32), torch.tensor(np.asarray(ctx), **I32), sel, sink, recent)
    assert C.get_device_error() == 0
    assert bool((buf[n:] == GUARD).all())
    return sel.cpu().numpy()


def _want(q, pool, table, ctx, pages, sink, recent):
    ref = dict(k=np.empty((1, 1, pool.kv_heads, 0, 0)), summary=pool.summary.cpu().numpy(),
               summary_scale=pool.summary_scale.cpu().numpy().astype(np.float64))
    return K.select(q.float().cpu().numpy().astype(np.float64), ref, 0, table, ctx, pages, sink, recent)


@pytest.mark.parametrize("R,Hq,D", [(1, 2, 64), (1, 4, 128), (5, 2, 128), (2, 20, 64)])
def test_scores_at_the_ends_of_fp32(R, Hq, D):
    """Pages whose keys come near the type's end (from 2^104 on a score passes fp32): with a product of zero and with others,
    beside ordinary pages and the smallest that a summary has."""
    rng = np.random.default_rng(R * 100 + Hq)
    pages, n = 90, 20
    pool = _pool(rng, pages, 1, D)
    table = rng.permutation(pages)[None].astype(np.int32)
    scale = pool.summary_scale[0, :, 0]
    scale[torch.from_numpy(table[0, 40:60].astype(np.int64)).cuda()] = 2.0 ** -115
    for p, e in ((7, 104), (9, 110), (11, 126), (30, 126), (31, 120), (33, 125), (70, 104), (89, 126)):
        at = int(table[0, p])
        if p in (7, 9, 11, 70):               # nothing but a channel in which every query is zero
            pool.summary[0, at, 0] = 0
            pool.summary[0, at, 0, 3] = 127
        scale[at] = 2.0 ** e
    q = torch.from_numpy(rng.standard_normal((1, R, Hq, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    q[..., 3] = 0
    for sink, recent in ((0, 0), (1, 4)):
        np.testing.assert_array_equal(_select(q, pool, table, [pages * 16], n, sink, recent), _want(q, pool, table, [pages * 16], n, sink, recent))


def test_a_page_of_keys_near_the_types_end():
    """Through the append: a page of keys of 2^120 in one channel, queries that are zero there."""
    rng = np.random.default_rng(4)
    H, D, pages, n = 2, 64, 40, 12
    k = rng.standard_normal((1, 1, pages * 16, H, D)).astype(np.float32)
    k[0, 0, 5 * 16:6 * 16] = 0
    k[0, 0, 5 * 16:6 * 16, :, 9] = 2.0 ** 120
    kt = torch.from_numpy(k).to(torch.bfloat16).cuda()
    pool = C.new_kv8_pool(1, pages, H, D)
    table = rng.permutation(pages)[None].astype(np.int32)
    C.kv8_append(pool, kt, kt, torch.tensor(table, **I32), torch.zeros(1, **I32))
    q = torch.from_numpy(rng.standard_normal((1, 3, 4, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    q[..., 9] = 0
    np.testing.assert_array_equal(_select(q, pool, table, [pages * 16], n, 1, 1), _want(q, pool, table, [pages * 16], n, 1, 1))


def test_a_scale_that_is_not_finite_is_no_page():
    rng = np.random.default_rng(5)
    pages, n = 64, 10
    pool = _pool(rng, pages, 1, 64)
    table = rng.permutation(pages)[None].astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((1, 1, 2, 64)).astype(np.float32)).to(torch.bfloat16).cuda()
    want = _want(q, pool, table, [pages * 16], n + 2, 0, 0)[0, 0, 0]
    dropped = [int(want[0]), int(want[-1])]    # two of those chosen lose their scale: the others stay
    for p, x in zip(dropped, (float("inf"), float("nan"))):
        pool.summary_scale[0, int(table[0, p]), 0] = x
    got = _select(q, pool, table, [pages * 16], n, 0, 0)[0, 0, 0]
    assert got.tolist() == [p for p in want.tolist() if p not in dropped]


# ---------------------------------------------------------------- long contexts
def _long(rng, ctx, H, D, width=None):
    """Pools and shuffled tables of contexts of many pages: B tables in one pool, -1 behind each context."""
    need = [-(-c // 16) for c in ctx]
    width = max(need) if width is None else width
    order, at = rng.permutation(sum(need)).astype(np.int32), 0
    table = np.full((len(ctx), width), -1, np.int32)
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return _pool(rng, sum(need), H, D), table


def _rows(rng, B, R, Hq, D):
    return torch.from_numpy(rng.standard_normal((B, R, Hq, D)).astype(np.float32)).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("pages", [1025, 2049, 4097, 8193, 32768])
@pytest.mark.parametrize("R,Hq,H,D,n", [(1, 4, 1, 128, 64), (1, 8, 2, 64, 300), (3, 8, 2, 128, 40), (8, 2, 1, 64, 128), (2, 12, 1, 128, 17)])
def test_one_long_context(pages, R, Hq, H, D, n):
    """Several steps of 32 pages a warp and, in the list, runs of more than 128 pages a warp; the last page partly filled."""
    rng = np.random.default_rng(pages + R)
    ctx = [pages * 16 - 5]
    pool, table = _long(rng, ctx, H, D)
    q = _rows(rng, 1, R, Hq, D)
    np.testing.assert_array_equal(_select(q, pool, table, ctx, n, 1, 4), _want(q, pool, table, ctx, n, 1, 4))


@pytest.mark.parametrize("R,Hq,D,n", [(1, 4, 128, 100), (1, 32, 64, 24), (2, 4, 64, 60)])
def test_many_ragged_contexts(R, Hq, D, n):
    rng = np.random.default_rng(R * 7 + Hq)
    ctx = [int(x) for x in rng.integers(0, 1400 * 16, 64)]
    ctx[5], ctx[9], ctx[40] = 0, 3, 1400 * 16
    pool, table = _long(rng, ctx, 1, D)
    q = _rows(rng, 64, R, Hq, D)
    np.testing.assert_array_equal(_select(q, pool, table, ctx, n, 1, 2), _want(q, pool, table, ctx, n, 1, 2))


@pytest.mark.parametrize("width", [600, 2048, 9000, 32768])
@pytest.mark.parametrize("R,Hq,H,D", [(1, 8, 2, 128), (7, 8, 2, 128), (1, 40, 2, 64), (16, 4, 1, 64)])
def test_tables_wider_than_the_contexts(width, R, Hq, H, D):
    """Clusters and shared memory go by the table's width: up to the largest of both, and every smaller one."""
    rng = np.random.default_rng(width + R)
    ctx = [590 * 16, 100, 333 * 16 + 7]
    pool, table = _long(rng, ctx, H, D, width)
    q = _rows(rng, 3, R, Hq, D)
    np.testing.assert_array_equal(_select(q, pool, table, ctx, 33, 2, 3), _want(q, pool, table, ctx, 33, 2, 3))


@pytest.mark.parametrize("pages", [1500, 5000])
def test_ties_across_a_long_context(pages):
    """Equal scores over many runs of the list: the lower pages, whole and in order."""
    rng = np.random.default_rng(pages)
    pool, table = _long(rng, [pages * 16], 1, 64)
    pool.summary.zero_()
    pool.summary[0, torch.from_numpy(table[0, ::3].astype(np.int64)).cuda(), 0, 0] = 5
    pool.summary_scale.fill_(0.5)
    q = torch.ones((1, 1, 2, 64), dtype=torch.bfloat16, device="cuda")
    for n in (7, 300, pages // 3 + 50, pages - 1):
        np.testing.assert_array_equal(_select(q, pool, table, [pages * 16], n, 0, 1), _want(q, pool, table, [pages * 16], n, 0, 1))
