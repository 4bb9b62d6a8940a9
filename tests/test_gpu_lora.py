"""The adapters' passes against the float64 reference, with error bounds from the arithmetic:

An mma of 16 products adds them to the running sum with at most 17 truncations at 2^-24 of the largest term and one of
the sum at 2^-23, so a contraction of length C over terms whose absolute sum is S is off by less than (2^-19 + C 2^-27) S
(C / 16 steps of 2^-23).  u and t are such sums, times a factor rounded to 2^-22.  y and dx add the adapters' part from
two bf16 parts (2^-17 of each term) and are rounded to bf16 once (2^-8 of the value, half a step).  dA and dB take fp32
t and u, whose own error, for t, comes on top."""
import numpy as np
import pytest
import torch

from oracle import cospec_lora as L
from paper_2605_24793_gb300 import build as BLD
from paper_2605_24793_gb300 import cospec as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    C.load_library(BLD.build())
    torch.cuda.set_device(0)
    C.get_device_error()


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _long(c):
    return 2.0 ** -19 + c * 2.0 ** -27


def _rows(rng, M, W, wide, scale=1.0):
    x = torch.from_numpy((rng.standard_normal((M, W + (64 if wide else 0))) * scale).astype(np.float32)).to(torch.bfloat16).cuda()
    return x[:, 32:32 + W] if wide else x


def _make(seed, M, K, N, r, n, wide=False, none=0.2, runs=True):
    rng = np.random.default_rng(seed)
    bf = lambda *s, k=1.0: torch.from_numpy((rng.standard_normal(s) * k).astype(np.float32)).to(torch.bfloat16).cuda()  # noqa: E731
    ids = np.sort(rng.integers(0, n, M)) if runs else rng.integers(0, n, M)
    ids[rng.random(M) < none] = -1
    c = dict(x=_rows(rng, M, K, wide), w=bf(N, K, k=0.05), a=bf(n, r, K, k=0.1), b=bf(n, N, r, k=0.1),
             scaling=torch.from_numpy(rng.uniform(0.5, 2, n).astype(np.float32)).cuda(),
             adapter=torch.from_numpy(ids.astype(np.int32)).cuda())
    return c, _rows(rng, M, N, wide)


def _host(c):
    h = {k: _np(v) for k, v in c.items() if k != "adapter"}
    h["adapter"] = c["adapter"].cpu().numpy()
    return h


SEED = (0x1234567 << 32) | 0x89ABCDEF


def _seed():
    return torch.tensor([SEED], dtype=torch.int64, device="cuda")


def _forward(c, dropout=0.0, site=3, wide=False, **kw):
    M, N, r = c["x"].shape[0], c["w"].shape[0], c["a"].shape[1]
    buf = torch.full((M + 2, N + (64 if wide else 0)), 77.0, dtype=torch.bfloat16, device="cuda")
    y = buf[1:M + 1, 32:32 + N] if wide else buf[1:M + 1]
    u = torch.full((M + 1, r), 5.0, device="cuda")
    C.lora_forward(**c, y=y, u=u[:M], dropout=dropout, seed=_seed() if dropout else None, site=site, **kw)
    assert C.get_device_error() == 0
    # nothing around the rows is touched
    assert (buf[0] == 77).all() and (buf[M + 1] == 77).all() and (u[M] == 5).all()
    if wide:
        assert (buf[:, :32] == 77).all() and (buf[:, 32 + N:] == 77).all()
    return y, u[:M]


def _check_forward(c, y, u, dropout=0.0, site=3):
    M, K = c["x"].shape
    mask, kept = L.keep_mask(M, K, dropout, SEED, site)
    o = L.forward(**_host(c), mask=mask, kept=kept)
    tol_u = _long(K) * o["abs_u"] + 2.0 ** -22 * np.abs(o["u"])
    assert (np.abs(_np(u) - o["u"]) <= tol_u).all()
    # u's error, its two parts and the sums, then half a bf16 step
    exact = _long(K + 512) * (o["abs_y"] + o["abs_low"]) + 2.0 ** -17 * o["abs_low"]
    host = _host(c)
    for m, i in enumerate(host["adapter"]):
        if i >= 0:
            exact[m] += np.abs(host["b"][i]) @ tol_u[m]
    assert (np.abs(_np(y) - o["y"]) <= 2.0 ** -8 * (np.abs(o["y"]) + exact) + exact).all()
    return o


SHAPES = [  # rows, in, out, rank, adapters, wide, rows side by side
    (1, 64, 64, 16, 1, False, True), (1, 2560, 4096, 16, 2, False, True), (3, 8, 8, 8, 1, False, True), (17, 72, 136, 8, 3, True, False),
    (64, 512, 640, 16, 20, False, False), (53, 200, 264, 24, 3, True, True), (129, 320, 384, 40, 5, False, False),
    (130, 1000, 1048, 64, 4, True, True), (256, 256, 128, 128, 2, False, True), (257, 264, 520, 16, 70, False, False),
    (301, 136, 1000, 72, 3, True, False), (848, 320, 256, 16, 4, False, True), (1100, 128, 264, 32, 2, False, True)]


@pytest.mark.parametrize("M,K,N,r,n,wide,runs", SHAPES)
def test_forward(M, K, N, r, n, wide, runs):
    c, _ = _make(M + K, M, K, N, r, n, wide, runs=runs)
    y, u = _forward(c, wide=wide)
    _check_forward(c, y, u)


# contractions longer than the ring of stages on every SM, with and without more adapter steps than stages
LONG = [(64, 1536, 20000, 16, 20), (257, 1024, 20000, 64, 9), (700, 4096, 1304, 128, 3), (256, 1024, 20000, 16, 100), (1300, 264, 2048, 24, 5),
        (2000, 512, 4096, 16, 40)]


@pytest.mark.parametrize("M,K,N,r,n", LONG)
def test_long_contractions(M, K, N, r, n):
    c, _ = _make(M + r, M, K, N, r, n, runs=False)
    y, u = _forward(c)
    _check_forward(c, y, u)
    c, dy = _make(M + r + 1, M, N, K, r, n, runs=False)
    for dropout in (0.0, 0.1) if M in (64, 1300) else (0.0,):
        _, u = _forward(c, dropout)
        _check_backward(c, dy, u, _backward(c, dy, u, dropout), dropout)


# rows of many adapters in turn, more than one window of ordered rows, a window that ends inside a tile; more ranks than a CTA takes
MANY = [(2500, 520, 136, 16, 40), (4200, 200, 264, 64, 13), (600, 1160, 264, 32, 64), (900, 136, 1344, 128, 6), (4100, 264, 136, 24, 4), (2300, 328, 136, 16, 700),
        (2100, 264, 136, 8, 255), (2100, 264, 136, 8, 256)]


@pytest.mark.parametrize("M,K,N,r,n", MANY)
@pytest.mark.parametrize("dropout", [0.0, 0.2])
def test_rows_of_many_adapters_in_turn(M, K, N, r, n, dropout):
    c, dy = _make(M + n, M, K, N, r, n, wide=dropout > 0, runs=False)
    y, u = _forward(c, dropout)
    _check_forward(c, y, u, dropout)
    _check_backward(c, dy, u, _backward(c, dy, u, dropout), dropout)


@pytest.mark.parametrize("M,K,N,r,n", [(1, 5576, 136, 64, 1), (2, 2752, 80, 128, 15), (5, 120, 2000, 72, 3), (130, 264, 136, 40, 7)])
def test_a_row_by_several_ctas(M, K, N, r, n):
    c, dy = _make(M + n, M, K, N, r, n, none=0.1)
    y, u = _forward(c, 0.2)
    _check_forward(c, y, u, 0.2)
    _check_backward(c, dy, u, _backward(c, dy, u, 0.2), 0.2)


@pytest.mark.parametrize("M,K,N,n", [(40, 192, 256, 3), (90, 136, 264, 40), (300, 192, 520, 3), (3000, 520, 136, 9)])
@pytest.mark.parametrize("dropout", [0.0, 0.3])
def test_an_adapter_that_is_not_finite_spoils_its_own_rows_only(M, K, N, n, dropout):
    c, dy = _make(M + 9, M, K, N, 16, n, none=0.2, runs=False)
    y0, u0 = _forward(c, dropout)
    g0 = _backward(c, dy, u0, dropout)
    bad = {k: v.clone() for k, v in c.items()}
    bad["a"][1, 3, ::7], bad["b"][1, 5::11, 2], bad["b"][1, 4] = float("inf"), float("nan"), float("-inf")
    others = c["adapter"] != 1
    assert others.any() and not others.all()
    y1, u1 = _forward(bad, dropout)
    assert torch.equal(u0[others], u1[others]) and not torch.isfinite(y1[~others]).all()
    dx, da, db, t = _backward(bad, dy, u0, dropout)
    assert not torch.isfinite(dx[~others]).all()
    # rows of other adapters as before, but for what is summed in another order: half a step and the sums' terms
    for a, b, size in ((y0, y1, _np(c["x"]).__abs__() @ _np(c["w"]).__abs__().T), (g0[0], dx, _np(dy).__abs__() @ _np(c["w"]).__abs__())):
        a, b = _np(a)[others.cpu()], _np(b)[others.cpu()]
        assert np.isfinite(b).all()
        low = 2.0 ** -10 * np.abs(size[others.cpu()])       # u's and t's terms: 2^-17 of them, and they are below 100 x the others
        assert (np.abs(a - b) <= 2.0 ** -7 * np.abs(a) + low).all()
    keep = [i for i in range(n) if i != 1]
    assert torch.equal(da[keep], g0[1][keep]) and torch.equal(db[keep], g0[2][keep])


@pytest.mark.parametrize("M,K,N,r,n,wide,runs", [SHAPES[i] for i in (0, 3, 4, 7, 9)])
@pytest.mark.parametrize("dropout", [0.05, 0.5])
def test_forward_dropout(M, K, N, r, n, wide, runs, dropout):
    c, _ = _make(M + K + 1, M, K, N, r, n, wide, runs=runs)
    y, u = _forward(c, dropout, 2 ** 32 - 1, wide)
    _check_forward(c, y, u, dropout, 2 ** 32 - 1)


def _backward(c, dy, u, dropout=0.0, site=3, accumulate=None, wide=False, want=(True, True, True)):
    M, K = c["x"].shape
    n, r = c["a"].shape[:2]
    buf = torch.full((M + 2, K + (64 if wide else 0)), 77.0, dtype=torch.bfloat16, device="cuda")
    dx = buf[1:M + 1, 32:32 + K] if wide else buf[1:M + 1]
    da = torch.full((n, r, K), 3.0 if accumulate else float("nan"), device="cuda")
    db = torch.full((n, c["w"].shape[0], r), -2.0 if accumulate else float("nan"), device="cuda")
    t = torch.empty((M, r), device="cuda")
    C.lora_backward(dy, **c, u=u, dx=dx if want[0] else None, da=da if want[1] else None, db=db if want[2] else None, t=t, dropout=dropout,
                    seed=_seed() if dropout else None, site=site, accumulate=bool(accumulate))
    assert C.get_device_error() == 0
    assert (buf[0] == 77).all() and (buf[M + 1] == 77).all()
    return dx, da, db, t


def _check_backward(c, dy, u, got, dropout=0.0, site=3, off=(0.0, 0.0)):
    dx, da, db, _ = got
    M, K = c["x"].shape
    N = c["w"].shape[0]
    mask, kept = L.keep_mask(M, K, dropout, SEED, site)
    h = _host(c)
    o = L.backward(_np(dy), **h, u=_np(u), mask=mask, kept=kept)
    tol_t = _long(N) * o["abs_t"] + 2.0 ** -22 * np.abs(o["t"])
    exact = _long(N + 512) * (o["abs_dx"] + o["abs_low"]) + 2.0 ** -17 * o["abs_low"]
    tol_a = np.zeros(o["da"].shape)
    for m, i in enumerate(h["adapter"]):
        if i >= 0:
            exact[m] += tol_t[m] @ np.abs(h["a"][i])
            tol_a[i] += np.outer(tol_t[m], np.abs(h["x"][m]))
    assert (np.abs(_np(dx) - o["dx"]) <= 2.0 ** -8 * (np.abs(o["dx"]) + exact) + exact).all()
    # three parts a term: three times the products; the sum that is added to is rounded once more
    for x, ref, tol, base in ((da, o["da"], tol_a + _long(3 * M) * o["abs_da"], off[0]), (db, o["db"], _long(3 * M) * o["abs_db"], off[1])):
        ref = ref + base
        assert (np.abs(x.cpu().numpy().astype(np.float64) - ref) <= tol + 2.0 ** -23 * (np.abs(ref) + abs(base))).all()
    return o


@pytest.mark.parametrize("M,K,N,r,n,wide,runs", SHAPES)
def test_backward(M, K, N, r, n, wide, runs):
    c, dy = _make(M + K + 2, M, K, N, r, n, wide, runs=runs)
    _, u = _forward(c)
    _check_backward(c, dy, u, _backward(c, dy, u, wide=wide))


@pytest.mark.parametrize("M,K,N,r,n,wide,runs", [SHAPES[i] for i in (0, 3, 4, 7, 9, 11)])
@pytest.mark.parametrize("dropout", [0.05, 0.5])
def test_backward_dropout(M, K, N, r, n, wide, runs, dropout):
    c, dy = _make(M + K + 3, M, K, N, r, n, wide, runs=runs)
    _, u = _forward(c, dropout)
    _check_backward(c, dy, u, _backward(c, dy, u, dropout, wide=wide), dropout)


def test_accumulate_and_parts():
    c, dy = _make(5, 90, 136, 264, 16, 4)
    _, u = _forward(c)
    _check_backward(c, dy, u, _backward(c, dy, u, accumulate=True), off=(3.0, -2.0))
    whole = _backward(c, dy, u)
    for want in ((True, False, False), (False, True, False), (False, False, True)):
        part = _backward(c, dy, u, want=want)
        for w, p, q in zip(want, part, whole):
            if w:
                assert torch.equal(p, q)


def test_rows_without_an_adapter_and_adapters_without_rows():
    c, dy = _make(6, 40, 128, 192, 16, 5, none=0.0)
    c["adapter"].fill_(-1)
    y, u = _forward(c)
    _check_forward(c, y, u)
    assert (u == 0).all()
    got = _backward(c, dy, u)
    _check_backward(c, dy, u, got)
    assert (got[1] == 0).all() and (got[2] == 0).all()
    c["adapter"][7] = 3
    y, u = _forward(c)
    _check_forward(c, y, u)
    got = _backward(c, dy, u)
    assert (got[1][[0, 1, 2, 4]] == 0).all() and (got[2][[0, 1, 2, 4]] == 0).all() and (got[1][3] != 0).any()


@pytest.mark.parametrize("M", [5, 40, 300])
def test_what_others_hold_stays_with_them(M):
    """Infinities and NaN in another adapter's factors, in another row and in dropped places reach no row."""
    K, N = 192, 256
    c, dy = _make(7, M, K, N, 16, 3, none=0.0, runs=False)
    c["adapter"][:] = torch.arange(M, device="cuda") % 2
    dropout = 0.3
    mask, kept = L.keep_mask(M, K, dropout, SEED, 3)
    y0, u0 = _forward(c, dropout)
    g0 = _backward(c, dy, u0, dropout)
    bad = {k: v.clone() for k, v in c.items()}
    bad["a"][2] = float("nan")
    bad["b"][2] = float("inf")
    bad["scaling"][2] = float("nan")
    y1, u1 = _forward(bad, dropout)
    assert torch.equal(y0, y1) and torch.equal(u0, u1)
    g1 = _backward(bad, dy, u0, dropout)
    assert all(torch.equal(p, q) for p, q in zip(g0[:3], g1[:3]))
    # a row with NaN, of adapter 1: rows and gradients of adapter 0 stay
    bad = {k: v.clone() for k, v in c.items()}
    bad["x"][3] = float("nan")
    dyb = dy.clone()
    dyb[3] = float("inf")
    y1, u1 = _forward(bad, dropout)
    keep = torch.arange(M, device="cuda") != 3
    assert torch.equal(y0[keep], y1[keep]) and torch.equal(u0[keep], u1[keep]) and torch.isnan(y1[3]).all()
    g1 = _backward(bad, dyb, u0, dropout)
    assert torch.equal(g0[0][keep], g1[0][keep]) and torch.equal(g0[1][0], g1[1][0]) and torch.equal(g0[2][0], g1[2][0])
    # NaN in x at dropped places only: u and dA as before
    bad = {k: v.clone() for k, v in c.items()}
    bad["x"][torch.from_numpy(mask == 0).cuda()] = float("nan")
    _, u1 = _forward(bad, dropout)
    assert torch.equal(u0, u1)
    assert torch.equal(_backward(bad, dy, u0, dropout)[1], g0[1])


def test_bad_adapter_ids_are_flagged_and_count_as_none():
    c, dy = _make(8, 33, 64, 128, 8, 2)
    good = c["adapter"].clone()
    good[4], good[20] = -1, -1
    c["adapter"][4], c["adapter"][20] = 2, -7
    y = torch.empty((33, 128), dtype=torch.bfloat16, device="cuda")
    u = torch.empty((33, 8), device="cuda")
    C.lora_forward(**c, y=y, u=u)
    with pytest.raises(C.CospecError):
        C._check(C.load_library().cospec_get_device_error(__import__("ctypes").byref(__import__("ctypes").c_int()), None))
    y1, u1 = _forward(dict(c, adapter=good))
    assert torch.equal(y, y1) and torch.equal(u, u1)


def test_bad_ids_among_rows_in_turn():
    """More rows than one window, a fifth of the ids outside the adapters: flagged, and as rows without one."""
    M, n = 2300, 12
    c, _ = _make(11, M, 1160, 136, 16, n, runs=False)
    good = c["adapter"].clone()
    rng = np.random.default_rng(3)
    bad = torch.from_numpy(rng.random(M) < 0.2).cuda()
    c["adapter"][bad] = torch.from_numpy(rng.choice(np.array([-2, n, 65535, 2 ** 31 - 1, -2 ** 31], dtype=np.int64), int(bad.sum())).astype(np.int32)).cuda()
    y = torch.empty((M, 136), dtype=torch.bfloat16, device="cuda")
    u = torch.empty((M, 16), device="cuda")
    C.lora_forward(**c, y=y, u=u)
    assert C.get_device_error() == C.DEVERR_ADAPTER
    good[bad] = -1
    c["adapter"] = good
    _check_forward(c, y, u)


def test_repeated_and_captured():
    """Repeated calls agree bit for bit; a captured forward and backward takes the seed and the inputs of its replay."""
    c, dy = _make(9, 200, 256, 384, 16, 3)
    seed = _seed()
    M, K, N, r = 200, 256, 384, 16
    y, u = torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), torch.empty((M, r), device="cuda")
    dx, t = torch.empty((M, K), dtype=torch.bfloat16, device="cuda"), torch.empty((M, r), device="cuda")
    da, db = torch.empty((3, r, K), device="cuda"), torch.empty((3, N, r), device="cuda")

    def step():
        C.lora_forward(**c, y=y, u=u, dropout=0.2, seed=seed, site=9)
        C.lora_backward(dy, **c, u=u, dx=dx, da=da, db=db, t=t, dropout=0.2, seed=seed, site=9)

    def result():
        torch.cuda.synchronize()
        return [v.clone() for v in (y, u, dx, da, db)]

    step()
    first = result()
    step()
    assert all(torch.equal(p, q) for p, q in zip(first, result()))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        step()
        step()
    seed += 1
    c["x"].mul_(0.5)
    g.replay()
    replayed = result()
    assert not torch.equal(replayed[1], first[1])
    step()
    assert all(torch.equal(p, q) for p, q in zip(replayed, result()))
    assert C.get_device_error() == 0


def test_gradients_are_differences():
    """<dy, y(A + h D) - y(A - h D)> / 2h = <dA, D>, and the same for B and x, through the kernels' own forward pass.  The
    bound is y's rounding (2^-8 of each value, as independent errors: four of their root mean square) over 2 h."""
    c, dy = _make(10, 96, 128, 192, 8, 2, none=0.1)
    dy = (dy.float() / 8).to(torch.bfloat16)
    y, u = _forward(c, 0.25)
    g = _backward(c, dy, u, 0.25)
    rng = np.random.default_rng(1)
    for k, grad in (("a", g[1]), ("b", g[2]), ("x", g[0].float())):
        # whole steps of powers of two on values rounded to multiples of 2^-6 keep the moved inputs exact
        D = torch.from_numpy(rng.integers(-1, 2, c[k].shape).astype(np.float32)).cuda()
        base = (torch.round(c[k].float() * 64) / 64)
        h = 2.0 ** -3
        moved = dict(c, **{k: base.to(torch.bfloat16)})
        y0, u0 = _forward(moved, 0.25)
        grad = dict(zip("xab", (lambda q: (q[0].float(), q[1], q[2]))(_backward(moved, dy, u0, 0.25))))[k]
        ends = [_forward(dict(moved, **{k: (base + s * h * D).to(torch.bfloat16)}), 0.25)[0].double() for s in (1, -1)]
        for s, e in ((1, 0), (-1, 1)):
            assert torch.equal((base + s * h * D).to(torch.bfloat16).float(), base + s * h * D)
        slope = float((dy.double() * (ends[0] - ends[1])).sum()) / (2 * h)
        want = float((grad.double() * D.double()).sum())
        noise = float(((dy.double() * ends[0]) ** 2).sum().sqrt()) * 2.0 ** -8 / h
        noise += float(((grad.double() * D.double()) ** 2).sum().sqrt()) * 2.0 ** -8
        assert abs(slope - want) <= 4 * noise
        assert noise * 4 < 0.5 * abs(want) or abs(want) < 8 * noise


def test_another_stream_and_threads():
    import threading
    c, dy = _make(11, 150, 192, 256, 16, 4)
    y0, u0 = _forward(c, 0.1)
    out, streams = {}, [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()

    def work(i):
        torch.cuda.set_device(0)
        y = torch.empty((150, 256), dtype=torch.bfloat16, device="cuda")
        u = torch.empty((150, 16), device="cuda")
        seed = _seed()
        torch.cuda.synchronize()
        for _ in range(20):
            C.lora_forward(**c, y=y, u=u, dropout=0.1, seed=seed, site=3, stream=streams[i])
        streams[i].synchronize()
        out[i] = (y, u)

    th = [threading.Thread(target=work, args=(i,)) for i in range(3)]
    [t.start() for t in th]
    [t.join() for t in th]
    assert all(torch.equal(out[i][0], y0) and torch.equal(out[i][1], u0) for i in range(3))
    assert C.get_device_error() == 0


def test_no_rows():
    c, dy = _make(12, 4, 64, 64, 8, 2)
    c["x"], c["adapter"] = c["x"][:0], c["adapter"][:0]
    e = lambda *s, dt=torch.float32: torch.full(s, 9.0, dtype=dt, device="cuda")  # noqa: E731
    C.lora_forward(**c, y=e(0, 64, dt=torch.bfloat16), u=e(0, 8))
    da, db = e(2, 8, 64), e(2, 64, 8)
    C.lora_backward(dy[:0], **c, u=e(0, 8), dx=e(0, 64, dt=torch.bfloat16), da=da, db=db, t=e(0, 8))
    assert (da == 0).all() and (db == 0).all()
    da.fill_(4)
    C.lora_backward(dy[:0], **c, u=e(0, 8), dx=None, da=da, db=None, t=e(0, 8), accumulate=True)
    assert (da == 4).all() and C.get_device_error() == 0
