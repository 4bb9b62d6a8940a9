"""The block's own rows, where weight concentrates, lose no more than the cache's: with an empty or short cache the outputs are
within their rounding to bf16 (2^-8 |o|) and f16's of the weights (2^-11 of the sum of p |v|, at most 2^-12 more of it from
scores in fp32) of the float64 oracle, on every form of the attention."""
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


@pytest.mark.parametrize("ctx", [[0, 0], [0, 16], [40, 3]])
@pytest.mark.parametrize("R,Hq,H,D", [(2, 8, 2, 64), (8, 2, 2, 128), (3, 8, 2, 128), (6, 8, 2, 128), (8, 8, 2, 128), (64, 2, 1, 64), (16, 2, 2, 128),
                                      (26, 8, 2, 128), (64, 8, 2, 64)])
def test_short_contexts_are_as_precise_as_long_ones(ctx, R, Hq, H, D):
    rng = np.random.default_rng(R * 3 + Hq + sum(ctx))
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()  # noqa: E731
    np_ = lambda t: t.float().cpu().numpy().astype(np.float64)  # noqa: E731
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    k, v = (dev(x) for x in rng.standard_normal((2, 1, 2, 48, H, D)))
    # one sign: the errors of the weights' rounding do not cancel against outputs near zero
    q, kb, vb = dev(rng.standard_normal((2, R, Hq, D))), dev(rng.standard_normal((2, R, H, D))), dev(np.abs(rng.standard_normal((2, R, H, D))))
    table = np.arange(6).reshape(2, 3)
    pool, ref = C.new_kv8_pool(1, 6, H, D), K.new_pool(1, 6, H, D)
    C.kv8_append(pool, k, v, ints(table), ints([0, 0]), ints(ctx))
    K.append(ref, np_(k), np_(v), table, [0, 0], ctx)
    out = torch.empty_like(q)
    sel = np.broadcast_to(np.arange(3), (2, R, H, 3)).copy()
    sel[..., :] = np.where(sel < (np.array(ctx)[:, None, None, None] + 15) // 16, sel, -1)
    for s in (None, sel):
        C.kv8_attn(q, kb, vb, pool, 0, ints(table), ints(ctx), out, 48, sel=None if s is None else ints(s))
        assert C.get_device_error() == 0
        o, mag = K.attention(np_(q), np_(kb), np_(vb), ref, 0, table, ctx, sel=s)
        # the weights' part shows beside the output's rounding: taken out by rounding the oracle's bounds
        lo, hi = (torch.from_numpy(o + x * (2.0 ** -11 + 2.0 ** -12) * mag).to(torch.float32).to(torch.bfloat16).double().numpy() for x in (-1, 1))
        got = np_(out)
        bad = (got < lo) | (got > hi)
        assert not bad.any(), f"{bad.sum()} of {bad.size}"
