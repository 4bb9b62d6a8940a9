"""The RL stage's objective through the decision MLP in float64 -- TEST INFRASTRUCTURE ONLY, written from the paper's
Sec. 3.4: per effective decision the clipped surrogate, the Bernoulli entropy and the KL divergence, and their
gradients by the chain rule, one decision at a time."""
from __future__ import annotations

import math

import numpy as np

from oracle.cospec_oracle import arbitration_features


def _softplus(x: float) -> float:
    return max(x, 0.0) + math.log1p(math.exp(-abs(x)))


def decision(z, took, adv, old, ref, clip, bh, bk):
    """(p, surrogate, entropy, kl, d loss / d z) of one decision."""
    p, q = 1 / (1 + math.exp(-z)) if z > -700 else 0.0, 1 / (1 + math.exp(z)) if z < 700 else 0.0
    pi, pi_old = (p, old) if took else (q, 1 - old)
    ratio = pi / pi_old
    plain, cut = ratio * adv, min(max(ratio, 1 - clip), 1 + clip) * adv
    ent = p * _softplus(-z) + q * _softplus(z)
    kl = p * (-_softplus(-z) - math.log(ref)) + q * (-_softplus(z) - math.log1p(-ref))
    dz = -plain * (q if took else -p) if plain <= cut else 0.0
    # d entropy / dz = -z p q;  d kl / dz = p q (z - logit ref)
    dz += p * q * (bh * z + bk * (z - (math.log(ref) - math.log1p(-ref))))
    return p, min(plain, cut), ent, kl, dz


def arbitrate_loss(draft, argmax, stats, w1, b1, w2, b2, accept, eff, adv, p_old, p_ref, clip, bh, bk, scale=1.0):
    """All outputs of the call, and `sure`: False where a unit or the clip is within 1e-6 of its border."""
    R, K = draft.shape
    H = len(b1)
    out = dict(loss=np.zeros(4), p_new=np.zeros((R, K)), dz=np.zeros((R, K)), dw1=np.zeros((H, 8)), db1=np.zeros(H), dw2=np.zeros(H), db2=np.zeros(1),
               abs_dw1=np.zeros((H, 8)), abs_db1=np.zeros(H), abs_dw2=np.zeros(H), abs_db2=np.zeros(1), sure=True)
    for r in range(R):
        f_all = np.asarray(arbitration_features(draft[r:r + 1], argmax[r:r + 1], stats[r:r + 1].astype(np.float64)))[0]
        for i in range(K):
            if not eff[r, i] or draft[r, i] == argmax[r, i]:
                continue
            f = f_all[i]
            pre = w1 @ f + b1
            h = np.maximum(pre, 0.0)
            z = float(w2 @ h + b2[0])
            p, surr, ent, kl, dz = decision(z, accept[r, i] != 0, float(adv[r, i]), float(p_old[r, i]), float(p_ref[r, i]), clip, bh, bk)
            out["loss"][:3] += (surr, ent, kl)
            out["p_new"][r, i], g = p, scale * dz
            out["dz"][r, i] = g
            on = (pre > 0) * g * w2
            out["dw1"] += np.outer(on, f)
            out["db1"] += on
            out["dw2"] += g * h
            out["db2"] += g
            out["abs_dw1"] += np.outer(np.abs(on), np.abs(f))
            out["abs_db1"] += np.abs(on)
            out["abs_dw2"] += abs(g) * (pre > 0) * (np.abs(w1) @ np.abs(f) + np.abs(b1))
            out["abs_db2"] += abs(g)
            ratio = (p / p_old[r, i]) if accept[r, i] else (1 - p) / (1 - p_old[r, i])
            if np.min(np.abs(pre)) < 1e-6 or min(abs(ratio - 1 - clip), abs(ratio - 1 + clip)) < 1e-6:
                out["sure"] = False
    s = out["loss"]
    s[3] = -s[0] - bh * s[1] + bk * s[2]
    return out
