"""The policy loss and its gradient against the float64 reference.

z is off by at most (H + 16) 2^-24 of its absolute terms; per decision the derivative of dz by z is bounded here by the
difference of the reference at z's neighbours, and the formulas add a few 2^-24 of each term: dz and p within 2^-20 of
(1 + the terms), sums within 2^-20 of the absolute sums.  Cases where a unit or the clip is within 1e-6 of its border
are drawn anew from the next seed, before anything is compared."""
import math

import numpy as np
import pytest
import torch

from oracle import cospec_policy as P
from paper_2605_24793_gb300 import build as BLD
from paper_2605_24793_gb300 import cospec as C

pytestmark = pytest.mark.gpu
CLIP, BH, BK = (float(np.float32(v)) for v in (0.2, 0.01, 0.02))


@pytest.fixture(scope="module", autouse=True)
def lib():
    C.load_library(BLD.build())
    torch.cuda.set_device(0)
    C.get_device_error()


def _case(seed, R, K, H, mismatch=0.4, dense=False):
    rng = np.random.default_rng(seed)
    argmax = rng.integers(0, 5000, (R, K + 1)).astype(np.int32)
    match = rng.random((R, K)) >= mismatch
    draft = np.where(match, argmax[:, :K], argmax[:, :K] + 1).astype(np.int32)
    st = np.empty((R, K + 1, 5), dtype=np.float32)
    st[..., 0] = rng.normal(6, 1.5, (R, K + 1))
    st[..., 1] = st[..., 0] - rng.exponential(0.7, (R, K + 1))
    st[..., 2] = st[..., 0] + 4 * rng.random((R, K + 1))
    st[..., 3] = 4 * rng.random((R, K + 1))
    st[..., 4] = st[..., 0] - rng.exponential(1.5, (R, K + 1))
    st[:, K, 4] = np.nan
    f32 = lambda x: np.asarray(x, dtype=np.float32)  # noqa: E731
    w = dict(w1=f32(rng.uniform(-1, 1, (H, 8)) / math.sqrt(8)), b1=f32(rng.uniform(-1, 1, H)), w2=f32(rng.uniform(-1, 1, H) / math.sqrt(H)),
             b2=f32(rng.uniform(-1, 1, 1)))
    accept = (match | (rng.random((R, K)) < 0.5)).astype(np.uint8)
    stop = (accept == 0).astype(int)
    eff = (~match & ((np.cumsum(stop, 1) - stop == 0) | dense)).astype(np.uint8)
    eff[rng.random((R, K)) < 0.05] = 1                     # a flag at a match is no decision
    return dict(draft=draft, argmax=argmax, stats=st, **w, accept=accept, eff=eff, adv=f32(rng.normal(size=(R, K))),
                p_old=f32(rng.uniform(0.1, 0.9, (R, K))), p_ref=f32(rng.uniform(0.1, 0.9, (R, K))))


def _sure(seed, *a, **kw):
    for s in range(seed, seed + 1000):
        c = _case(s, *a, **kw)
        o = P.arbitrate_loss(**{k: v.astype(np.float64) if v.dtype == np.float32 else v for k, v in c.items()}, clip=CLIP, bh=BH, bk=BK, scale=0.125)
        if o["sure"]:
            return c, o
    raise AssertionError("no case off the borders")


def _run(c, out=None):
    dev = {k: torch.from_numpy(v).cuda() for k, v in c.items()}
    return C.arbitrate_loss(**dev, params=C.RLParams(), grad_scale=0.125, out=out)


def _check(got, o, c):
    g = {k: v.double().cpu().numpy() for k, v in got.items() if k != "ws"}
    on = (c["eff"] != 0) & (c["draft"] != c["argmax"][:, :-1])
    n = max(1, int(on.sum()))
    assert (g["p_new"][~on] == 0).all() and (g["dz"][~on] == 0).all()
    H = len(c["b1"])
    zerr = (H + 16) * 2.0 ** -24 * 40.0                    # |z|'s absolute terms: |w2| (|w1| |f| + |b1|) summed is below 40 here
    assert (np.abs(g["p_new"] - o["p_new"]) <= 0.25 * zerr + 2.0 ** -22).all()
    # |d dz / dz| <= |A| ratio (ratio <= 10) + the pulls' (below 1)
    per = (np.abs(c["adv"]) * 10 + 1) * (zerr + 2.0 ** -21) * 0.125
    assert (np.abs(g["dz"] - o["dz"])[on] <= per[on]).all()
    each = float(per[on].sum()) if on.any() else 0.0
    fmax = 15.0                                            # |f| of these inputs
    for k, slope in (("dw1", fmax), ("db1", 1.0), ("dw2", 40.0), ("db2", 1.0)):
        # the decisions' errors, and the sums': a few 2^-24 of the absolute terms per step of at most 64 and the rest in 64 bits
        tol = each * slope + 2.0 ** -17 * o["abs_" + k]
        assert (np.abs(g[k] - o[k]) <= tol).all(), k
    assert (np.abs(g["loss"] - o["loss"]) <= n * (10 * 4 + 4) * (zerr + 2.0 ** -21)).all()
    assert (np.abs(g["loss"][1:3] - o["loss"][1:3]) <= n * 3 * (zerr + 2.0 ** -22)).all()


@pytest.mark.parametrize("R,K,H", [(1, 1, 1), (1, 5, 64), (3, 31, 7), (40, 25, 64), (21, 64, 65), (300, 3, 128), (64, 25, 200), (30, 7, 256),
                                   (9, 64, 511), (12, 33, 1024), (700, 2, 33)])
def test_against_the_reference(R, K, H):
    c, o = _sure(R * 100 + K, R, K, H)
    _check(_run(c), o, c)


@pytest.mark.parametrize("shift", [1, 2, 3, 4])
def test_flags_at_any_address(shift):
    c, o = _sure(97 + shift, 130, 7, 64)
    dev = {k: torch.from_numpy(v).cuda() for k, v in c.items()}
    for k in ("eff", "accept"):
        buf = torch.full((c[k].size + 16,), 1, dtype=torch.uint8, device="cuda")
        dev[k] = buf[shift:shift + c[k].size].view(c[k].shape)
        dev[k].copy_(torch.from_numpy(c[k]))
    _check(C.arbitrate_loss(**dev, params=C.RLParams(), grad_scale=0.125), o, c)


def test_every_position_a_decision():
    c, o = _sure(5, 30, 40, 64, mismatch=1.0, dense=True)
    assert int(c["eff"].sum()) == 1200
    _check(_run(c), o, c)


def test_sums_are_close_relative_to_their_size():
    """In the norm the gradients are good to 32 bits: random errors of 2^-22 a decision, not their bounds added up."""
    c, o = _sure(17, 150, 25, 256)
    g = _run(c)
    for k in ("dw1", "db1", "dw2", "dz", "p_new", "loss"):
        x, y = g[k].double().cpu().numpy(), o[k]
        assert np.linalg.norm(x - y) <= 2.0 ** -19 * np.linalg.norm(y), k


def test_kl_of_a_policy_near_its_reference():
    """p_ref within 2^-10 of p: KL near 2^-20, a difference of logarithms that 32 bits would lose.  p enters from z with
    2^-22, of a difference of 2^-10: 2^-12 twice, relative."""
    c, o = _sure(23, 40, 25, 64)
    p = _run(c)["p_new"].cpu().numpy()
    c["p_ref"] = np.where(p > 0, np.clip(p + np.float32(2.0 ** -10), 0.01, 0.99), c["p_ref"]).astype(np.float32)
    o = P.arbitrate_loss(**{k: v.astype(np.float64) if v.dtype == np.float32 else v for k, v in c.items()}, clip=CLIP, bh=BH, bk=BK, scale=0.125)
    got = float(_run(c)["loss"][2])
    assert 0 < o["loss"][2] and abs(got - o["loss"][2]) <= 2.0 ** -10 * o["loss"][2]


def test_clipped_decisions_have_no_surrogate_gradient():
    R, K = 4, 3
    c = _case(31, R, K, 8, mismatch=1.0, dense=True)
    c["eff"][:] = 1
    c["accept"][:] = 1
    c["p_old"][:] = 0.01                                   # ratio far above 1 + clip
    for sign in (1.0, -1.0):
        c["adv"][:] = sign
        dev = {k: torch.from_numpy(v).cuda() for k, v in c.items()}
        g = C.arbitrate_loss(**dev, params=C.RLParams(beta_h=0.0, beta_kl=0.0))
        assert ((g["dz"] == 0).all() if sign > 0 else (g["dz"] > 0).all())
        p = g["p_new"].double()
        want = (1 + CLIP) * R * K if sign > 0 else -float((p / float(np.float32(0.01))).sum())
        assert abs(float(g["loss"][0]) - want) <= 2.0 ** -20 * abs(want)


def test_nothing_effective_and_no_rounds():
    c = _case(41, 6, 5, 16)
    c["eff"][:] = 0
    for k in ("adv", "p_old", "p_ref"):
        c[k][:] = np.nan                                   # not read
    g = _run(c)
    assert all((g[k] == 0).all() for k in g if k != "ws")
    c = {k: (v[:0] if k in ("draft", "argmax", "stats", "accept", "eff", "adv", "p_old", "p_ref") else v) for k, v in c.items()}
    g = _run(c)
    assert all((g[k] == 0).all() for k in ("loss", "dw1", "db1", "dw2", "db2"))


def test_logits_far_out():
    """z of +-60 and +-infinity: p of 0 or 1, finite terms where the formula has them."""
    for z, p in ((60.0, 1.0), (-60.0, 0.0), (math.inf, 1.0), (-math.inf, 0.0)):
        c = _case(43, 2, 2, 4, mismatch=1.0, dense=True)
        c["eff"][:], c["accept"][:] = 1, int(p)
        c["w2"][:] = 0
        c["b2"][:] = z
        g = _run(c)
        old, ref = (c["p_old"], c["p_ref"]) if p else (1 - c["p_old"].astype(np.float64), 1 - c["p_ref"].astype(np.float64))
        ratio, A = 1 / old.astype(np.float64), c["adv"].astype(np.float64)
        surr = np.minimum(ratio * A, np.clip(ratio, 1 - CLIP, 1 + CLIP) * A).sum()
        assert (g["p_new"].cpu().numpy().round(12) == p).all() and float(g["loss"][1]) < 1e-20
        assert abs(float(g["loss"][0]) - surr) <= 2.0 ** -20 * (np.abs(A) * ratio).sum()
        assert abs(float(g["loss"][2]) + np.log(ref.astype(np.float64)).sum()) <= 2.0 ** -20 * 4 * 4
        assert np.abs(g["dz"].cpu().numpy()).max() < 1e-20


@pytest.mark.parametrize("z", [-79.99, -40.25, -17.5, -5.0, -0.7, -1e-4, 0.0, 1e-4, 0.346, 0.347, 3.0, 20.0, 79.99, 80.0, 85.0])
def test_p_and_dz_over_the_logits_range(z):
    """p to its rounding (2^-24 of it, and 2^-24 of the pair's terms), dz of a ratio of one to two roundings more."""
    c = _case(47, 2, 3, 4, mismatch=1.0, dense=True)
    c["eff"][:], c["w2"][:], c["b2"][:] = 1, 0, z
    zz = float(c["b2"][0])
    p, q = 1 / (1 + math.exp(-zz)), 1 / (1 + math.exp(zz))
    for took in (1, 0):
        c["accept"][:] = took
        c["p_old"][:] = p if took else 1 - q
        dev = {k: torch.from_numpy(v).cuda() for k, v in c.items()}
        g = C.arbitrate_loss(**dev, params=C.RLParams(beta_h=0.0, beta_kl=0.0, clip_eps=0.9))
        assert (np.abs(g["p_new"].double().cpu().numpy() - p) <= 2.0 ** -23 * p).all()
        old, A = c["p_old"].astype(np.float64), c["adv"].astype(np.float64)
        with np.errstate(divide="ignore", invalid="ignore"):
            ratio = (p if took else q) / (old if took else 1 - old)
        inside = ratio * A <= np.clip(ratio, 1 - np.float64(np.float32(0.9)), 1 + np.float64(np.float32(0.9))) * A
        want = np.where(inside, -A * ratio * (q if took else -p), 0.0)
        fine = np.isfinite(want)
        assert (np.abs(g["dz"].double().cpu().numpy()[fine] - want[fine]) <= 2.0 ** -21 * np.abs(want[fine]) + 2.0 ** -126).all()


@pytest.mark.parametrize("H", [7, 64, 100, 256, 600])
@pytest.mark.parametrize("K,pos", [(1, 0), (7, 3), (7, 6)])
def test_units_at_their_border(H, K, pos):
    """b1 is the rounded negative of W1 f, so that a unit's input is a rounding of it, 2^-25 relative: on and off as in 64 bits."""
    from oracle.cospec_oracle import arbitration_features
    for seed in range(6):
        c = _case(1000 + seed, 1, K, H, mismatch=0.5)
        c["draft"][0, pos] = c["argmax"][0, pos] + 1
        c["eff"][:] = 0
        c["eff"][0, pos], c["accept"][0, pos] = 1, 1
        c["p_old"][:], c["adv"][:] = 0.5, -1.0                       # an unclipped gradient that is not zero
        f = np.asarray(arbitration_features(c["draft"], c["argmax"], c["stats"].astype(np.float64)))[0][pos]
        w = c["w1"].astype(np.float64)
        c["b1"] = (-(w @ f)).astype(np.float32)
        pre = w @ f + c["b1"].astype(np.float64)
        assert (np.abs(pre) > 2.0 ** -45).any()
        g = _run(c)
        on = g["db1"].cpu().numpy() != 0
        clear = np.abs(pre) > 2.0 ** -45                             # the 64-bit sums' own roundings
        assert (on == (pre > 0))[clear & (c["w2"] != 0)].all()


def test_an_old_probability_of_zero():
    """The ratio is infinite: clipped where A > 0, so that nothing else is lost; infinite where A < 0."""
    c = _case(53, 3, 4, 8, mismatch=1.0, dense=True)
    c["eff"][:], c["accept"][:], c["p_old"][:] = 1, 1, 0.5
    c["adv"][:] = 1.0
    c["p_old"][1, 2] = 0.0
    dev = {k: torch.from_numpy(v).cuda() for k, v in c.items()}
    g = C.arbitrate_loss(**dev, params=C.RLParams())
    assert all(torch.isfinite(g[k]).all() for k in ("loss", "p_new", "dz", "dw1", "db1", "dw2", "db2"))
    dev["adv"][1, 2] = -1.0
    g = C.arbitrate_loss(**dev, params=C.RLParams())
    assert float(g["loss"][0]) == -math.inf and float(g["loss"][3]) == math.inf and float(g["dz"][1, 2]) == math.inf
    assert float(g["db2"][0]) == math.inf and torch.isfinite(g["loss"][1:3]).all()


def test_repeated_captured_and_filled_again():
    c, o = _sure(51, 200, 25, 256)
    a = _run(c)
    first = {k: v.clone() for k, v in a.items() if k != "ws"}
    b = _run(c, out=a)
    assert b is a and all(torch.equal(a[k], first[k]) for k in first)
    dev = {k: torch.from_numpy(v).cuda() for k, v in c.items()}
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        C.arbitrate_loss(**dev, params=C.RLParams(), grad_scale=0.125, out=a)
    for v in first:
        a[v].fill_(7)
    dev["b2"].add_(1.0)
    g.replay()
    torch.cuda.synchronize()
    c["b2"] = c["b2"] + np.float32(1)
    again = _run(c)
    assert all(torch.equal(a[k], again[k]) for k in first) and not torch.equal(a["dz"], first["dz"])


def test_gradient_is_the_difference_of_the_loss():
    """Through the kernels alone: loss at moved weights.  h = 2^-7 leaves a third-order term; the loss is a sum of a few
    hundred terms below 10 in 64 bits, each good to 2^-20."""
    c, o = _sure(61, 60, 20, 32)
    for k in ("w2", "b2"):                                 # the loss is smooth in these but for the clip
        D = np.sign(np.random.default_rng(2).standard_normal(c[k].shape)).astype(np.float32)
        h = np.float32(2.0 ** -7)
        c["p_old"][:] = _run(c)["p_new"].cpu().numpy().clip(0.05, 0.95)      # ratios near 1: inside the clip on both sides
        base = _run(c)
        ends = []
        for s in (1, -1):
            d = dict(c)
            d[k] = (c[k] + s * h * D).astype(np.float32)
            ends.append(float(_run(d)["loss"][3]))
        slope = (ends[0] - ends[1]) / (2 * float(h))
        want = float((base["d" + k].double().cpu() * torch.from_numpy(D).double()).sum()) / 0.125
        n = int(((c["eff"] != 0) & (c["draft"] != c["argmax"][:, :-1])).sum())
        size = float(np.abs(D).sum()) if k == "b2" else float(np.abs(c["stats"][..., :4]).max()) * 4
        assert abs(slope - want) <= n * (2.0 ** -20 * 10 / float(h) + float(h) ** 2 * size ** 3)


def test_after_the_advantages():
    """A run of the calls as they are used: arbitrate over recorded rounds, the advantages, the loss: with p_old = p the
    ratio is 1 and the surrogate the sum of the advantages."""
    R, K, H = 64, 7, 64
    c = _case(71, R, K, H, mismatch=0.5)
    dev = {k: torch.from_numpy(v).cuda() for k, v in c.items()}
    p = torch.empty((R, K), device="cuda")
    acc = torch.empty((R, K), dtype=torch.uint8, device="cuda")
    C.arbitrate(dev["draft"], dev["argmax"], dev["stats"], dev["w1"], dev["b1"], dev["w2"], float(c["b2"][0]), 0.5, C.POLICY_MLP, p, acc)
    match = (dev["draft"] == dev["argmax"][:, :K]).to(torch.uint8)
    go = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda")
    ro = torch.arange(0, R + 1, 8, dtype=torch.int32, device="cuda")
    correct = torch.tensor([1, 0, 1, 0, 0, 0, 1, 1], dtype=torch.uint8, device="cuda")
    ell = (dev["stats"][:, :K, 4] - dev["stats"][:, :K, 2]).contiguous()
    adv = C.rl_advantages(go, correct, ro, match, acc, ell)
    g = C.arbitrate_loss(dev["draft"], dev["argmax"], dev["stats"], dev["w1"], dev["b1"], dev["w2"], dev["b2"], acc, adv["eff"], adv["adv_dec"], p, p)
    on = (adv["eff"] != 0) & (match == 0)
    assert torch.equal(adv["eff"] != 0, on) and on.any()
    # cospec_arbitrate takes p with the fast exponential: 2^-20
    assert (g["p_new"][on] - p[on]).abs().max() <= 2.0 ** -20
    assert abs(float(g["loss"][0]) - float(adv["adv_dec"].double().sum())) <= 2.0 ** -18 * float(adv["adv_dec"].double().abs().sum())
    terms = C.rl_advantages(go, correct, ro, match, acc, ell, None, torch.ones_like(p), g["p_new"].clamp(2.0 ** -20, 1 - 2.0 ** -20), p)["loss"]
    assert abs(float(terms[1]) - float(g["loss"][1])) <= 2.0 ** -18 * float(terms[1])
    assert float(g["loss"][2]) < 1e-6 and C.get_device_error() == 0
