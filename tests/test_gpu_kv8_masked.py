"""What the mask hides from a row of the block stays hidden: infinities and NaN in later rows' keys and values, and in cells behind
a context's end.  Rows that see them get what the formula says (float64 oracle)."""
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


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _ints(x):
    return torch.tensor(np.asarray(x), **I32)


def _check(rng, ctx, q, kb, vb, H, full, sel=None):
    B, R, Hq, D = q.shape
    T = max(max(ctx), 1)
    k, v = rng.standard_normal((2, 1, B, T, H, D))
    width = -(-T // 16) + 1
    table = rng.permutation(B * width).reshape(B, width).astype(np.int32)
    pool, ref = C.new_kv8_pool(1, B * width, H, D), K.new_pool(1, B * width, H, D)
    for t in (pool.k, pool.v):
        t.view(torch.uint8).fill_(0x7f)                     # NaN wherever nothing is appended
    kt, vt, q, kb, vb = (_dev(x) for x in (k, v, q, kb, vb))
    C.kv8_append(pool, kt, vt, _ints(table), _ints([0] * B), _ints(ctx))
    K.append(ref, _np(kt), _np(vt), table, [0] * B, ctx)
    out = torch.full(q.shape, 123.0, dtype=torch.bfloat16, device="cuda")
    C.kv8_attn(q, kb, vb, pool, 0, _ints(table), _ints(ctx), out, max(ctx), sel=None if sel is None else _ints(sel), block_full=full)
    assert C.get_device_error() == 0
    with np.errstate(all="ignore"):
        o, mag = K.attention(_np(q), _np(kb), _np(vb), ref, 0, table, ctx, sel=sel, full=full)
    got, fin = _np(out), np.isfinite(o)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(o))
    np.testing.assert_array_equal(got[np.isinf(o)], o[np.isinf(o)])
    err = np.abs(got - o)[fin]
    bound = (2.0 ** -8 * (np.abs(o) + mag))[fin]
    assert np.all(err <= bound), float((err / bound).max())
    return o


SHAPES = [(2, 8, 2, 64), (8, 4, 4, 128), (3, 8, 2, 128), (6, 8, 2, 128), (8, 8, 2, 128), (20, 4, 2, 64), (26, 8, 2, 128), (64, 8, 2, 64)]


@pytest.mark.parametrize("R,Hq,H,D", SHAPES)
@pytest.mark.parametrize("full", [False, True])
def test_values_that_are_not_finite(R, Hq, H, D, full):
    rng = np.random.default_rng(R * 10 + Hq)
    for ctx in ([130, 0, 45], [1500, 16, 3]):
        q, kb, vb = rng.standard_normal((3, R, Hq, D)), rng.standard_normal((3, R, H, D)), rng.standard_normal((3, R, H, D))
        vb[0, R - 1, 0, 3], vb[0, R - 1, H - 1, 5], vb[0, R - 1, 0, D - 1] = math.nan, math.inf, -math.inf
        vb[0, R // 2, 0, 3], vb[0, R // 2, 0, 9], vb[0, R // 2, 0, D - 1] = -math.inf, math.inf, math.inf
        vb[1, R - 1] = math.nan
        o = _check(rng, ctx, q, kb, vb, H, full)
        assert np.isfinite(o[:, 0]).all() != full           # (a causal first row sees none of them)


@pytest.mark.parametrize("R,Hq,H,D", SHAPES)
def test_keys_that_are_not_finite(R, Hq, H, D):
    rng = np.random.default_rng(R * 11 + Hq)
    for x in (math.nan, math.inf, -math.inf):
        q, kb, vb = rng.standard_normal((3, R, Hq, D)), rng.standard_normal((3, R, H, D)), rng.standard_normal((3, R, H, D))
        q[..., 3] = np.abs(q[..., 3]) + 0.1
        kb[0, R - 1, 0, 3] = kb[1, R - 1, H - 1, 3] = x
        o = _check(rng, [130, 0, 45], q, kb, vb, H, False)
        assert np.isfinite(o[:, :R - 1]).all()


@pytest.mark.parametrize("R,Hq,H,D", [(4, 8, 2, 128), (3, 48, 2, 64)])
def test_values_that_are_not_finite_beside_selected_pages(R, Hq, H, D):
    rng = np.random.default_rng(R)
    q, kb, vb = rng.standard_normal((2, R, Hq, D)), rng.standard_normal((2, R, H, D)), rng.standard_normal((2, R, H, D))
    vb[0, R - 1, 0, 3], vb[0, 1, 1, 5] = math.nan, math.inf
    sel = np.full((2, R, H, 6), -1, np.int32)
    sel[0, ..., :4] = (0, 2, 5, 9)
    sel[1, ..., :1] = 1
    _check(rng, [155, 20], q, kb, vb, H, False, sel=sel)
