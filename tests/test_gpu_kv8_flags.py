"""What the 8-bit cache's calls skip and flag, one bad sequence at a time: its flag and no other, its output as described, the
other sequences as ever.  Attention on mma.sync and, above 32 rows per KV head, on tcgen05."""
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


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _ints(x):
    return torch.tensor(np.asarray(x), **I32)


def _host(pool):
    return dict(k=pool.k.view(torch.uint8).cpu().numpy(), v=pool.v.view(torch.uint8).cpu().numpy(), scale=_np(pool.scale),
                summary=pool.summary.cpu().numpy(), summary_scale=_np(pool.summary_scale))


@pytest.mark.parametrize("start,rows,page,flag", [
    (-1, 4, None, C.DEVERR_CTX), (30, 4, None, C.DEVERR_CTX), (2, 5, None, C.DEVERR_CTX), (2, -1, None, C.DEVERR_CTX), (1 << 30, 1, None, C.DEVERR_CTX),
    (0, 4, 12, C.DEVERR_PAGE), (0, 4, -1, C.DEVERR_PAGE), (20, 3, 1 << 30, C.DEVERR_PAGE)])
def test_append_flags_one_sequence(start, rows, page, flag):
    """Sequence 1 of three does not fit, or its page is outside the pool: its rows are skipped, the others' are appended."""
    rng = np.random.default_rng(abs(start) % 97 + rows + 5)
    L, B, R, H, D = 2, 3, 4, 3, 64
    k, v = (_dev(x) for x in rng.standard_normal((2, L, B, R, H, D)))
    table = np.arange(6).reshape(3, 2)
    starts, num = [0, start, 16], [4, rows, 2]
    bad = table.copy()
    if page is not None:
        bad[1, start // 16] = page
    pool = C.new_kv8_pool(L, 6, H, D)
    ref = _host(pool)
    C.kv8_append(pool, k, v, _ints(bad), _ints(starts), _ints(num))
    assert C.get_device_error() == flag
    for b in (0, 2):
        K.append(ref, _np(k)[:, [b]], _np(v)[:, [b]], table[[b]], [starts[b]], [num[b]])
    got = _host(pool)
    for n in got:
        np.testing.assert_array_equal(got[n], ref[n], err_msg=n)


@pytest.mark.parametrize("start", [-1, 17])
def test_rotation_flags_one_sequence(start):
    rng = np.random.default_rng(3)
    q, k = _dev(rng.standard_normal((3, 4, 4, 64))), _dev(rng.standard_normal((3, 4, 2, 64)))
    cos = torch.ones((20, 32), device="cuda")
    qo, ko = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
    C.kv8_rotate(q, k, C.Rope(cos, torch.zeros_like(cos)), _ints([0, start, 16]), qo, ko)
    assert C.get_device_error() == C.DEVERR_POSITION       # (without a cache only the tables can be missed)
    for x, y in ((q, qo), (k, ko)):
        assert bool((y[1] == 9.0).all()) and torch.equal(y[[0, 2]], x[[0, 2]])


ATTN = [(1, 8, 2, 128), (4, 8, 2, 128), (6, 16, 4, 64), (8, 8, 2, 128), (10, 16, 4, 64), (26, 8, 2, 128), (64, 8, 2, 64)]


def _cached(rng, ctx, H, D):
    B, width = len(ctx), -(-max(ctx) // 16) + 1
    table = rng.permutation(B * width).reshape(B, width).astype(np.int32)
    pool, ref = C.new_kv8_pool(1, B * width, H, D), K.new_pool(1, B * width, H, D)
    k, v = (_dev(x) for x in rng.standard_normal((2, 1, B, max(ctx), H, D)))
    C.kv8_append(pool, k, v, _ints(table), _ints([0] * B), _ints(ctx))
    K.append(ref, _np(k), _np(v), table, [0] * B, ctx)
    return pool, ref, table


@pytest.mark.parametrize("R,Hq,H,D", ATTN)
@pytest.mark.parametrize("length", [-1, None])
def test_attention_skips_a_sequence_whose_context_does_not_fit(R, Hq, H, D, length):
    rng = np.random.default_rng(R + Hq)
    ctx = [300, 60, 90]
    pool, ref, table = _cached(rng, ctx, H, D)
    q, kb, vb = (_dev(rng.standard_normal((3, R, n, D))) for n in (Hq, H, H))
    lens = [300, 16 * table.shape[1] + 1 if length is None else length, 90]
    out = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device="cuda")
    C.kv8_attn(q, kb, vb, pool, 0, _ints(table), _ints(lens), out, 300)
    assert C.get_device_error() == C.DEVERR_CTX
    assert bool((out[1] == 0).all())
    o, mag = K.attention(_np(q), _np(kb), _np(vb), ref, 0, table, ctx)
    err = np.abs(_np(out) - o)
    assert np.all((err <= 2.0 ** -8 * (np.abs(o) + mag))[[0, 2]])


@pytest.mark.parametrize("R,Hq,H,D", ATTN)
@pytest.mark.parametrize("gone", [(0,), (3,), (4,), (7, 8), (2, 5, 18), (18,), tuple(range(19))])
def test_attention_goes_on_without_pages_outside_the_pool(R, Hq, H, D, gone):
    """Pages of both halves of a tile, of its first and last, of the context's end, and all of them."""
    rng = np.random.default_rng(R + Hq + len(gone))
    ctx = [300, 60]
    pool, ref, table = _cached(rng, ctx, H, D)
    q, kb, vb = (_dev(rng.standard_normal((2, R, n, D))) for n in (Hq, H, H))
    bad = table.copy()
    bad[0, list(gone)] = [(-1, pool.num_pages, 1 << 30)[i % 3] for i in range(len(gone))]
    out = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device="cuda")
    C.kv8_attn(q, kb, vb, pool, 0, _ints(bad), _ints(ctx), out, 300)
    assert C.get_device_error() == C.DEVERR_PAGE
    left = np.full((2, R, H, 19), -1)
    rest = [p for p in range(19) if p not in gone]
    left[0, ..., :len(rest)], left[1, ..., :4] = rest, range(4)
    o, mag = K.attention(_np(q), _np(kb), _np(vb), ref, 0, table, ctx, sel=left)
    err = np.abs(_np(out) - o)
    assert np.all(err <= 2.0 ** -8 * (np.abs(o) + mag)), float((err / (np.abs(o) + mag)).max())


@pytest.mark.parametrize("length", [-3, 16 * 24 + 1])
def test_selection_flags_one_sequence(length):
    rng = np.random.default_rng(9)
    ctx = [320, 200, 320]
    pool, ref, table = _cached(rng, ctx, 2, 64)
    table = np.concatenate([table, np.zeros((3, 24 - table.shape[1]), np.int32)], axis=1)
    q = _dev(rng.standard_normal((3, 2, 4, 64)))
    sel = torch.full((3, 2, 2, 6), -9, **I32)
    C.kv8_select(q, pool, 0, _ints(table), _ints([320, length, 320]), sel, 1, 1)
    assert C.get_device_error() == C.DEVERR_CTX
    assert bool((sel[1] == -1).all())
    want = K.select(_np(q), ref, 0, table, ctx, 6, 1, 1)
    np.testing.assert_array_equal(sel.cpu().numpy()[[0, 2]], want[[0, 2]])
