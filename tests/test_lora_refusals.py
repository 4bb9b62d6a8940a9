"""What the adapters' and the policy loss's calls refuse, on the host (CPU): the C entry points' statuses and the binding's
exceptions, before anything is launched."""
import ctypes as ct

import pytest
import torch

from paper_2605_24793_gb300 import build as B
from paper_2605_24793_gb300 import cospec as C

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
P = ct.c_void_p(1 << 20)              # an aligned address that is never read
ODD = ct.c_void_p((1 << 20) + 8)


@pytest.fixture(scope="module")
def lib():
    return C.load_library(B.build())


def _dims(**kw):
    d = dict(rows=4, in_features=64, out_features=128, rank=16, num_adapters=2, dropout=0.0, site=0, x_stride=0, y_stride=0, dx_stride=0)
    d.update(kw)
    return C.LoraDims(*(d[n] for n, _ in C.LoraDims._fields_))


def _forward(lib, dims=None, **kw):
    a = dict(x=P, w=P, a=P, b=P, scaling=P, adapter=P, seed=None, u=P, y=P)
    a.update(kw)
    return lib.cospec_lora_forward(ct.byref(_dims() if dims is None else dims), *a.values(), None)


def _backward(lib, dims=None, flags=0, **kw):
    a = dict(dy=P, x=P, w=P, a=P, b=P, scaling=P, adapter=P, seed=None, u=P, t=P, dx=P, da=P, db=P)
    a.update(kw)
    return lib.cospec_lora_backward(ct.byref(_dims() if dims is None else dims), *a.values(), flags, None)


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), INVALID), (dict(in_features=0), INVALID), (dict(out_features=0), INVALID), (dict(rank=0), INVALID), (dict(num_adapters=0), INVALID),
    (dict(in_features=68), UNSUPPORTED), (dict(out_features=132), UNSUPPORTED), (dict(rank=12), UNSUPPORTED), (dict(rank=136), UNSUPPORTED),
    (dict(num_adapters=65536), UNSUPPORTED), (dict(rows=(8 << 20) + 1), UNSUPPORTED), (dict(dropout=-0.1), INVALID), (dict(dropout=1.0), INVALID),
    (dict(dropout=float("nan")), INVALID), (dict(dropout=0.999999), UNSUPPORTED), (dict(dropout=0.1), INVALID), (dict(x_stride=56), INVALID),
    (dict(x_stride=68), INVALID), (dict(y_stride=120), INVALID), (dict(dx_stride=56), INVALID), (dict(x_stride=-8), INVALID),
    (dict(y_stride=(1 << 30) + 8), UNSUPPORTED)])
def test_dims(lib, kw, want):
    assert _forward(lib, _dims(**kw)) == want
    assert _backward(lib, _dims(**kw)) == want


@pytest.mark.parametrize("name", ["x", "w", "a", "b", "scaling", "adapter", "u", "y"])
def test_forward_pointers(lib, name):
    assert _forward(lib, **{name: None}) == INVALID
    if name not in ("scaling", "adapter"):
        assert _forward(lib, **{name: ODD}) == INVALID


def test_forward_without_rows_or_dims(lib):
    assert _forward(lib, _dims(rows=0), x=None, w=None, u=None, y=None) == OK
    assert lib.cospec_lora_forward(None, *[P] * 9, None) == INVALID
    assert _forward(lib, _dims(dropout=0.1), seed=ct.c_void_p((1 << 20) + 4)) == INVALID


@pytest.mark.parametrize("name", ["dy", "x", "w", "a", "b", "scaling", "adapter", "u", "t"])
def test_backward_pointers(lib, name):
    assert _backward(lib, **{name: None}) == INVALID
    if name not in ("scaling", "adapter"):
        assert _backward(lib, **{name: ODD}) == INVALID


def test_backward_outputs_and_flags(lib):
    for n in ("dx", "da", "db"):
        assert _backward(lib, **{n: ODD}) == INVALID
    assert _backward(lib, flags=2) == INVALID
    # what a missing output would have needed is not asked for
    for kw in (dict(dx=None, w=None, a=None), dict(da=None, x=None), dict(db=None, u=None)):
        assert _backward(lib, **{**kw, "dy": None}) == INVALID
    if not torch.cuda.is_available():
        # accepted arguments get as far as the (missing) device
        for kw in (dict(dx=None, w=None, a=None), dict(da=None, x=None), dict(db=None, u=None)):
            assert _backward(lib, **kw) == -4


def _loss(lib, R=4, K=5, H=16, ws_bytes=1 << 30, params=None, scale=1.0, **kw):
    a = dict(draft=P, argmax=P, stats=P, w1=P, b1=P, w2=P, b2=P, accept=P, eff=P, adv=P, p_old=P, p_ref=P, loss=P, p_new=P, dz=P, dw1=P, db1=P, dw2=P, db2=P,
             ws=P)
    a.update(kw)
    v = list(a.values())
    prm = C.RLParams() if params is None else params
    return lib.cospec_arbitrate_loss(R, K, *v[:3], H, *v[3:12], ct.byref(prm), scale, *v[12:], ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(R=-1), INVALID), (dict(K=0), INVALID), (dict(H=0), INVALID), (dict(K=65), UNSUPPORTED), (dict(H=1025), UNSUPPORTED),
    (dict(R=1 << 27, K=16), UNSUPPORTED), (dict(scale=float("inf")), INVALID), (dict(params=C.RLParams(clip_eps=-0.1)), INVALID),
    (dict(params=C.RLParams(clip_eps=float("nan"))), INVALID), (dict(params=C.RLParams(beta_kl=float("inf"))), INVALID),
    (dict(ws_bytes=64), WORKSPACE), (dict(ws=None), WORKSPACE), (dict(ws=ODD), WORKSPACE), (dict(w1=ODD), INVALID)] + [
    ({n: None}, INVALID) for n in ("draft", "argmax", "stats", "w1", "b1", "w2", "b2", "accept", "eff", "adv", "p_old", "p_ref", "loss", "p_new", "dz",
                                   "dw1", "db1", "dw2", "db2")])
def test_loss(lib, kw, want):
    assert _loss(lib, **kw) == want


def test_loss_workspace(lib):
    f = lib.cospec_arbitrate_loss_workspace
    assert f(0) == 0 and f(1025) == 0 and 0 < f(1) == f(64) < f(65) < f(1024)


class _Cuda:
    """A CPU tensor that says it is on the GPU: the binding's checks of shapes run, and no call is made."""

    def __init__(self, t):
        self.t = t

    is_cuda = True

    def get_device(self):
        return 0

    def __getattr__(self, n):
        return getattr(self.t, n)


def _t(*shape, dtype=torch.bfloat16):
    return _Cuda(torch.zeros(shape, dtype=dtype))


def _lora(**kw):
    f32, i32 = torch.float32, torch.int32
    a = dict(x=_t(4, 64), w=_t(128, 64), a=_t(2, 16, 64), b=_t(2, 128, 16), scaling=_t(2, dtype=f32), adapter=_t(4, dtype=i32), y=_t(4, 128),
             u=_t(4, 16, dtype=f32))
    a.update(kw)
    return a


@pytest.mark.parametrize("kw", [
    dict(x=_t(4, 72)), dict(x=_t(3, 64)), dict(x=_t(4, 64, dtype=torch.float16)), dict(w=_t(128, 72)), dict(a=_t(2, 16, 72)), dict(b=_t(2, 120, 16)),
    dict(b=_t(3, 128, 16)), dict(b=_t(2, 128, 8)), dict(scaling=_t(3, dtype=torch.float32)), dict(scaling=_t(2)), dict(adapter=_t(4, dtype=torch.int64)),
    dict(y=_t(4, 120)), dict(u=_t(4, 8, dtype=torch.float32)), dict(u=_t(4, 16)), dict(x=_Cuda(torch.zeros(64, 4, dtype=torch.bfloat16).T)),
    dict(x=_Cuda(torch.zeros(4, 68, dtype=torch.bfloat16)[:, :64])), dict(x=_Cuda(torch.zeros(1, 64, dtype=torch.bfloat16).expand(4, 64))), dict(site=-1),
    dict(site=1 << 32), dict(seed=_t(2, dtype=torch.int64)), dict(seed=_t(1, dtype=torch.int32)), dict(x=torch.zeros(4, 64, dtype=torch.bfloat16))])
def test_binding_shapes(kw):
    with pytest.raises((ValueError, TypeError)):
        C.lora_forward(**_lora(**kw))


@pytest.mark.parametrize("kw", [dict(dy=_t(4, 120)), dict(dx=_t(4, 72)), dict(da=_t(2, 16, 72, dtype=torch.float32)), dict(da=_t(2, 16, 64)),
                                dict(db=_t(2, 16, 128, dtype=torch.float32)), dict(t=_t(4, 8, dtype=torch.float32)), dict(u=_t(3, 16, dtype=torch.float32))])
def test_binding_shapes_backward(kw):
    f32 = torch.float32
    a = _lora()
    del a["y"]
    a.update(dy=_t(4, 128), dx=_t(4, 64), da=_t(2, 16, 64, dtype=f32), db=_t(2, 128, 16, dtype=f32), t=_t(4, 16, dtype=f32))
    a.update(kw)
    with pytest.raises((ValueError, TypeError)):
        C.lora_backward(**a)


def _loss_args(**kw):
    f, i, b = torch.float32, torch.int32, torch.uint8
    a = dict(draft=_t(4, 5, dtype=i), argmax=_t(4, 6, dtype=i), stats=_t(4, 6, 5, dtype=f), w1=_t(7, 8, dtype=f), b1=_t(7, dtype=f), w2=_t(7, dtype=f),
             b2=_t(1, dtype=f), accept=_t(4, 5, dtype=b), eff=_t(4, 5, dtype=b), adv=_t(4, 5, dtype=f), p_old=_t(4, 5, dtype=f), p_ref=_t(4, 5, dtype=f))
    a.update(kw)
    return a


@pytest.mark.parametrize("kw", [
    dict(draft=_t(4, 5, dtype=torch.int64)), dict(argmax=_t(4, 5, dtype=torch.int32)), dict(stats=_t(4, 5, 5, dtype=torch.float32)),
    dict(w1=_t(7, 9, dtype=torch.float32)), dict(b1=_t(8, dtype=torch.float32)), dict(w2=_t(6, dtype=torch.float32)), dict(b2=_t(2, dtype=torch.float32)),
    dict(accept=_t(4, 6, dtype=torch.uint8)), dict(eff=_t(4, 5, dtype=torch.float32)), dict(adv=_t(5, 4, dtype=torch.float32)),
    dict(p_old=_t(4, 5)), dict(p_ref=_t(3, 5, dtype=torch.float32))])
def test_binding_shapes_loss(kw):
    with pytest.raises((ValueError, TypeError)):
        C.arbitrate_loss(**_loss_args(**kw))
