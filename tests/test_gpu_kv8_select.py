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
