"""What the 8-bit cache's calls refuse, on the host (CPU): the C entry points' statuses and the
binding's exceptions, before anything is launched."""
import ctypes as ct

import pytest
import torch

from paper_2605_24793_gb300 import build as B
from paper_2605_24793_gb300 import cospec as C

OK, INVALID, UNSUPPORTED = 0, -1, -2
P = ct.c_void_p(1 << 20)              # an aligned address that is never read
ODD = ct.c_void_p((1 << 20) + 2)


@pytest.fixture(scope="module")
def lib():
    return C.load_library(B.build())


def _pool(**kw):
    d = dict(layers=2, num_pages=8, num_kv_heads=2, head_dim=64, k=P.value, v=P.value, scale=P.value, summary=P.value, summary_scale=P.value)
    d.update(kw)
    return C.Kv8PoolC(*(d[n] for n, _ in C.Kv8PoolC._fields_))


def _dims(**kw):
    d = dict(batch=2, rows=4, num_q_heads=4, num_kv_heads=2, head_dim=64, page_size=16, max_pages_per_seq=4, num_pages=8, softmax_scale=0.0, flags=0)
    d.update(kw)
    return C.AttnDims(*(d[n] for n, _ in C.AttnDims._fields_))


S = C.Strides(8, 8, 8)
BAD = C.Strides(8, 8, 4)


def _append(lib, pool=None, first=0, layers=2, batch=2, rows=4, hq=4, rope=None, q=None, qs=S, k=P, ks=S, v=P, vs=S, table=P, width=4, start=P,
            num=None, qo=None, ko=None):
    r = lambda x: None if x is None else ct.byref(x)  # noqa: E731
    return lib.cospec_kv8_append(r(_pool() if pool is None else pool), first, layers, batch, rows, hq, r(rope), q, r(qs), k, r(ks), v, r(vs), table,
                                 width, start, num, qo, ko, None)


@pytest.mark.parametrize("kw,want", [
    (dict(batch=0), OK), (dict(rows=0), OK), (dict(layers=0), OK), (dict(batch=-1), INVALID), (dict(rows=-1), INVALID), (dict(layers=-1), INVALID),
    (dict(first=1, layers=2), INVALID), (dict(first=2, layers=0), INVALID), (dict(first=-1, layers=1), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(ks=None), INVALID), (dict(vs=BAD), INVALID), (dict(k=ODD), INVALID), (dict(table=None), INVALID),
    (dict(width=0), INVALID), (dict(width=1 << 28), UNSUPPORTED), (dict(start=None), INVALID), (dict(qo=P), INVALID), (dict(qo=P, q=P, hq=0), INVALID),
    (dict(qo=ODD, q=P), INVALID), (dict(ko=ODD), INVALID), (dict(q=P, qs=BAD, qo=P), INVALID),
    (dict(rope=C.RopeC(None, P.value, 8, 64, 0)), INVALID), (dict(rope=C.RopeC(P.value, P.value, 0, 64, 0)), INVALID),
    (dict(rope=C.RopeC(P.value, P.value, 8, 60, 0)), INVALID), (dict(rope=C.RopeC(P.value, P.value, 8, 72, 0)), INVALID),
    (dict(rope=C.RopeC(P.value, ODD.value, 8, 64, 0)), INVALID)])
def test_append(lib, kw, want):
    assert _append(lib, **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(layers=0), INVALID), (dict(num_pages=0), INVALID), (dict(num_kv_heads=0), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(v=None), INVALID),
    (dict(scale=None), INVALID), (dict(summary=None), INVALID), (dict(scale=ODD.value), INVALID), (dict(k=ODD.value), INVALID)])
def test_pools(lib, kw, want):
    assert _append(lib, pool=_pool(**kw)) == want


def test_null_pool(lib):
    assert lib.cospec_kv8_append(None, *[0] * 5, None, None, None, P, None, P, None, P, 1, P, None, None, None, None) == INVALID


def _select(lib, dims=None, pool=None, layer=0, q=P, qs=S, table=P, ctx=P, pages=4, sink=1, recent=1, sel=P):
    r = lambda x: None if x is None else ct.byref(x)  # noqa: E731
    return lib.cospec_kv8_select(r(_dims() if dims is None else dims), r(_pool() if pool is None else pool), layer, q, r(qs), table, ctx, pages, sink,
                                 recent, sel, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dims=_dims(batch=0)), OK), (dict(dims=_dims(num_pages=7)), INVALID), (dict(dims=_dims(num_kv_heads=1)), INVALID),
    (dict(dims=_dims(head_dim=128)), INVALID), (dict(dims=_dims(rows=65)), UNSUPPORTED), (dict(dims=_dims(max_pages_per_seq=32769)), UNSUPPORTED),
    (dict(pool=_pool(summary=None, summary_scale=None)), INVALID), (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(q=None), INVALID),
    (dict(qs=BAD), INVALID), (dict(table=None), INVALID), (dict(ctx=None), INVALID), (dict(sel=None), INVALID), (dict(pages=0), INVALID),
    (dict(sink=-1), INVALID), (dict(recent=-1), INVALID), (dict(sink=3, recent=2), INVALID), (dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1), INVALID)])
def test_select(lib, kw, want):
    assert _select(lib, **kw) == want


def _attn(lib, dims=None, max_ctx=10, pool=None, layer=0, q=P, qs=S, k=P, ks=S, v=P, vs=S, table=P, ctx=P, sel=None, pages=0, out=P):
    r = lambda x: None if x is None else ct.byref(x)  # noqa: E731
    return lib.cospec_kv8_attn(r(_dims() if dims is None else dims), max_ctx, r(_pool() if pool is None else pool), layer, q, r(qs), k, r(ks), v,
                               r(vs), table, ctx, sel, pages, out, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dims=_dims(batch=0)), OK), (dict(dims=_dims(num_pages=9)), INVALID), (dict(dims=_dims(page_size=32)), UNSUPPORTED),
    (dict(dims=_dims(head_dim=96)), UNSUPPORTED), (dict(dims=_dims(rows=0)), INVALID), (dict(dims=_dims(num_q_heads=3)), INVALID),
    (dict(dims=_dims(num_q_heads=514, rows=2)), UNSUPPORTED), (dict(dims=_dims(flags=8)), INVALID), (dict(max_ctx=-1), INVALID),
    (dict(max_ctx=65), INVALID), (dict(dims=_dims(softmax_scale=float("nan"))), INVALID), (dict(layer=5), INVALID), (dict(q=None), INVALID),
    (dict(k=ODD), INVALID), (dict(vs=BAD), INVALID), (dict(ks=None), INVALID), (dict(table=None), INVALID), (dict(ctx=None), INVALID),
    (dict(out=None), INVALID), (dict(out=ODD), INVALID), (dict(sel=P, pages=0), INVALID), (dict(pool=_pool(scale=None)), INVALID)])
def test_attn(lib, kw, want):
    assert _attn(lib, **kw) == want


def test_the_binding_refuses_host_tensors_and_types():
    f8 = torch.zeros((1, 2, 2, 16, 64), dtype=torch.uint8).view(C.F8)
    with pytest.raises(ValueError, match="CUDA"):
        C.Kv8Pool(f8, f8, torch.zeros((1, 2, 2, 2)))
    with pytest.raises(TypeError):
        C.Kv8Pool(f8.view(torch.uint8), f8, torch.zeros((1, 2, 2, 2)))
    with pytest.raises(ValueError, match="CUDA"):
        C.Rope(torch.zeros((4, 32)), torch.zeros((4, 32)))
    x = torch.zeros((2, 3, 4, 64))
    with pytest.raises(TypeError):
        C._rows_ref(x, "q", x.shape)
    with pytest.raises(ValueError, match="dense"):
        C._rows_ref(x.to(torch.bfloat16).transpose(1, 2), "q", (2, 4, 3, 64))
    with pytest.raises(ValueError, match="CUDA"):
        C._on_device(0, None, x)
    # the layers', batch's and rows' strides, of fused projections too; one element has none
    y = torch.zeros((2, 3, 10, 64), dtype=torch.bfloat16)
    st = C._rows_ref(y[:, :, 2:6], "k", (2, 3, 4, 64))._obj
    assert (st.layer, st.batch, st.row) == (0, 1920, 640)
    st = C._rows_ref(y[None, :1, :, :1], "k", (1, 1, 3, 1, 64))._obj
    assert (st.layer, st.batch, st.row) == (0, 0, 640)
