"""The float64 references of the adapters and of the policy loss, held against torch's products and derivatives, against
differences, and by hand (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import cospec_lora as L
from oracle import cospec_policy as P
from oracle.philox import philox4x32_10


def _case(seed, M=7, K=24, N=16, r=8, n=3):
    rng = np.random.default_rng(seed)
    return dict(x=rng.standard_normal((M, K)), w=rng.standard_normal((N, K)), a=rng.standard_normal((n, r, K)), b=rng.standard_normal((n, N, r)),
                scaling=rng.uniform(0.5, 2, n), adapter=rng.integers(-1, n, M))


@pytest.mark.parametrize("dropout", [0.0, 0.4])
def test_adapters_against_autograd(dropout):
    c = _case(1)
    mask, kept = L.keep_mask(7, 24, dropout, 99, 5)
    t = {k: torch.tensor(c[k], requires_grad=k in ("x", "a", "b")) for k in ("x", "w", "a", "b", "scaling")}
    y = t["x"] @ t["w"].T
    rows = []
    for m, i in enumerate(c["adapter"]):
        low = t["b"][i] @ (t["a"][i] @ (t["x"][m] * torch.tensor(mask[m]))) * t["scaling"][i] / kept if i >= 0 else 0 * y[m]
        rows.append(y[m] + low)
    y = torch.stack(rows)
    f = L.forward(**c, mask=mask, kept=kept)
    assert np.allclose(f["y"], y.detach().numpy(), rtol=1e-13, atol=1e-13)
    dy = np.random.default_rng(2).standard_normal(f["y"].shape)
    y.backward(torch.tensor(dy))
    g = L.backward(dy, **c, u=f["u"], mask=mask, kept=kept)
    for k, name in (("x", "dx"), ("a", "da"), ("b", "db")):
        assert np.allclose(g[name], t[k].grad.numpy(), rtol=1e-12, atol=1e-12)


def test_mask_by_hand():
    seed, site = (7 << 32) | 3, 11
    mask, kept = L.keep_mask(3, 20, 0.25, seed, site)
    assert kept == 0.75
    words = [int(w[0]) for w in philox4x32_10(np.array([1]), np.array([2]), np.array([site]), np.array([2]), 3, 7)]
    want = [(words[0] & 0xFFFF) >= 16384, (words[0] >> 16) >= 16384, (words[1] & 0xFFFF) >= 16384, (words[1] >> 16) >= 16384]
    assert mask[2, 8:12].tolist() == [float(v) for v in want]
    assert abs(L.keep_mask(64, 256, 0.25, seed, site)[0].mean() - 0.75) < 4 * math.sqrt(0.25 * 0.75 / (64 * 256))
    assert (L.keep_mask(2, 8, 0.0, seed, site)[0] == 1).all()


def test_decision_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(3)
    for _ in range(200):
        z, adv, old, ref, took = rng.normal(0, 2), rng.normal(), rng.uniform(0.05, 0.95), rng.uniform(0.05, 0.95), rng.random() < 0.5
        loss = lambda v: (lambda d: -d[1] - 0.3 * d[2] + 0.7 * d[3])(P.decision(v, took, adv, old, ref, 0.2, 0.3, 0.7))  # noqa: E731
        h = 1e-5
        p = P.decision(z, took, adv, old, ref, 0.2, 0.3, 0.7)
        ratio = p[0] / old if took else (1 - p[0]) / (1 - old)
        if min(abs(ratio - 0.8), abs(ratio - 1.2)) < 1e-3:
            continue
        # truncation h^2 |loss'''| / 6 and rounding 2^-52 / h
        assert abs((loss(z + h) - loss(z - h)) / (2 * h) - p[4]) < 1e-8


def test_decision_by_hand():
    # p = 1/2, pi_old = 1/4: ratio 2, clipped to 1.2 for A > 0 (no gradient), plain for A < 0
    p, surr, ent, kl, dz = P.decision(0.0, True, 1.0, 0.25, 0.5, 0.2, 0.0, 0.0)
    assert (p, surr, dz) == (0.5, 1.2, 0.0) and math.isclose(ent, math.log(2)) and abs(kl) < 1e-15
    assert P.decision(0.0, True, -1.0, 0.25, 0.5, 0.2, 0.0, 0.0)[4] == 1.0          # -A ratio (1 - p)
    assert math.isclose(P.decision(0.0, False, 1.0, 0.5, 0.25, 0.2, 0.0, 1.0)[4], 0.5 + 0.25 * math.log(3))


def test_policy_weights_against_autograd():
    rng = np.random.default_rng(4)
    R, K, H = 5, 4, 6
    argmax = rng.integers(0, 9, (R, K + 1))
    draft = np.where(rng.random((R, K)) < 0.4, argmax[:, :K], 10)
    stats = rng.normal(0, 2, (R, K + 1, 5))
    w1, b1, w2, b2 = rng.normal(size=(H, 8)), rng.normal(size=H), rng.normal(size=H), rng.normal(size=1)
    acc, eff = rng.integers(0, 2, (R, K)), rng.integers(0, 2, (R, K))
    adv, old, ref = rng.normal(size=(R, K)), rng.uniform(0.2, 0.8, (R, K)), rng.uniform(0.2, 0.8, (R, K))
    o = P.arbitrate_loss(draft, argmax, stats, w1, b1, w2, b2, acc, eff, adv, old, ref, 0.2, 0.1, 0.3, 0.5)
    from oracle.cospec_oracle import arbitration_features
    f = torch.tensor(np.asarray(arbitration_features(draft, argmax, stats)))
    par = [torch.tensor(v, requires_grad=True) for v in (w1, b1, w2, b2)]
    on = torch.tensor((eff != 0) & (draft != argmax[:, :K]))
    z = (torch.relu(f @ par[0].T + par[1]) @ par[2] + par[3])[on]
    took, A = torch.tensor(acc)[on] != 0, torch.tensor(adv)[on]
    q, qo, qr = torch.sigmoid(z), torch.tensor(old)[on], torch.tensor(ref)[on]
    ratio = torch.where(took, q / qo, (1 - q) / (1 - qo))
    loss = -torch.minimum(ratio * A, ratio.clamp(0.8, 1.2) * A).sum() + 0.1 * (q * q.log() + (1 - q) * (1 - q).log()).sum()
    loss = loss + 0.3 * (q * (q / qr).log() + (1 - q) * ((1 - q) / (1 - qr)).log()).sum()
    assert math.isclose(float(loss), o["loss"][3], rel_tol=1e-12)
    (0.5 * loss).backward()
    for v, name in zip(par, ("dw1", "db1", "dw2", "db2")):
        assert np.allclose(v.grad.numpy(), o[name], rtol=1e-11, atol=1e-12)
