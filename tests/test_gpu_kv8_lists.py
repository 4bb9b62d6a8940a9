"""Lists of selected pages that end before their arrays do: the first -1 ends them, whatever stands behind it."""
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


@pytest.mark.parametrize("R,Hq,H,D", [(1, 8, 2, 128), (3, 24, 2, 64), (2, 40, 2, 128), (2, 64, 2, 128), (4, 4, 4, 64)])
@pytest.mark.parametrize("width", [9, 70, 1000])
def test_what_stands_behind_the_first_end_is_not_read(R, Hq, H, D, width):
    """A reused list: page numbers, pages twice and pages that do not exist behind a single -1, at every length."""
    rng = np.random.default_rng(R * 100 + width)
    ctx = [150, 150, 31]
    B, T = 3, 150
    k, v = rng.standard_normal((2, 1, B, T, H, D))
    q, kb, vb = rng.standard_normal((B, R, Hq, D)), rng.standard_normal((B, R, H, D)), rng.standard_normal((B, R, H, D))
    table = rng.permutation(B * 10).reshape(B, 10).astype(np.int32)
    pool, ref = C.new_kv8_pool(1, B * 10, H, D), K.new_pool(1, B * 10, H, D)
    kt, vt, q, kb, vb = (_dev(x) for x in (k, v, q, kb, vb))
    ints = lambda x: torch.tensor(np.asarray(x), **I32)  # noqa: E731
    C.kv8_append(pool, kt, vt, ints(table), ints([0] * B), ints(ctx))
    K.append(ref, _np(kt), _np(vt), table, [0] * B, ctx)
    for stale in ("pages", "none"):
        sel, want = np.empty((B, R, H, width), np.int32), np.full((B, R, H, width), -1, np.int32)
        sel[:] = rng.integers(0, 2, sel.shape) if stale == "pages" else rng.integers(50, 100, sel.shape)
        for b in range(B):
            for j in range(R):
                for h in range(H):
                    pages = np.sort(rng.choice(10 if b < 2 else 2, int(rng.integers(0, 9 if b < 2 else 3)), replace=False))
                    sel[b, j, h, :len(pages)] = want[b, j, h, :len(pages)] = pages
                    if len(pages) < width:
                        sel[b, j, h, len(pages)] = -1
        out = torch.full(q.shape, math.nan, dtype=torch.bfloat16, device="cuda")
        C.kv8_attn(q, kb, vb, pool, 0, ints(table), ints(ctx), out, max(ctx), sel=ints(sel))
        assert C.get_device_error() == 0
        o, mag = K.attention(_np(q), _np(kb), _np(vb), ref, 0, table, ctx, sel=want)
        assert np.all(np.abs(_np(out) - o) <= 2.0 ** -8 * (np.abs(o) + mag))
