"""The arbitrator's training and its adapters as cases that can be timed.

The arbitrator shares the draft's backbone and differs by low-rank adapters (rank 16, scale 32,
dropout 0.05); its decisions are trained with a clipped policy loss.  The kinds of case:

  forward   y = x W^T + s_a drop(x) A_a^T B_a^T, every row with its own adapter a (-1: none)
  backward  its gradients for x and for every adapter's A and B, W staying as it is
  loss      the clipped objective with entropy and KL over recorded rounds, through the decision
            MLP: its terms, its gradient for the logits and for the MLP's weights

Widths are those of the backbones in ``workload.CONFIGS`` and ``arbitrator.BACKBONE`` (a fused
query / key / value projection, a query or an output projection) or generic.  The plain form
(``own`` false) needs torch alone.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
CLIP, BETA_H, BETA_KL = 0.2, 0.01, 0.02


def listed():
    return [
        # One user's token under the arbitrator's adapter: the query projection of the 2560-wide backbone, all latency.
        dict(name="fwd_b1", kind="forward", rows=1, d_in=2560, d_out=4096, rank=16, adapters=1, layout="runs", base=0.0, drop=0.0, fused=False),
        # A serving batch of 64 tokens, a request a row, 32 adapters and some requests without one: fused query / key / value projection.
        dict(name="fwd_b64_mixed", kind="forward", rows=64, d_in=4096, d_out=6144, rank=16, adapters=32, layout="rows", base=0.2, drop=0.0, fused=False),
        # One round of 16 sequences at the paper's default K = 25: regions of 53 rows, each with one of four adapters.
        dict(name="fwd_b16_k25", kind="forward", rows=848, d_in=2560, d_out=6144, rank=16, adapters=4, layout="runs", base=0.1, drop=0.0, fused=False),
        # Odd sizes: widths that end inside a tile, a rank of 24, rows cut out of a wider buffer.
        dict(name="fwd_odd", kind="forward", rows=301, d_in=1000, d_out=1048, rank=24, adapters=3, layout="rows", base=0.3, drop=0.0, fused=True),
        # A training step's 4096 tokens with dropout.
        dict(name="fwd_train_4096", kind="forward", rows=4096, d_in=2560, d_out=6144, rank=16, adapters=1, layout="runs", base=0.0, drop=0.05, fused=False),
        # The widest projection, 8192 tokens: the largest.
        dict(name="fwd_train_8192", kind="forward", rows=8192, d_in=5120, d_out=8192, rank=64, adapters=2, layout="runs", base=0.0, drop=0.05, fused=False),
        # The gradients of one region.
        dict(name="bwd_k25", kind="backward", rows=53, d_in=2560, d_out=4096, rank=16, adapters=1, layout="runs", base=0.0, drop=0.05, fused=False),
        # Odd sizes again.
        dict(name="bwd_odd", kind="backward", rows=301, d_in=1000, d_out=1048, rank=24, adapters=3, layout="rows", base=0.3, drop=0.1, fused=True),
        # A training step's 4096 tokens.
        dict(name="bwd_train_4096", kind="backward", rows=4096, d_in=2560, d_out=6144, rank=16, adapters=1, layout="runs", base=0.0, drop=0.05, fused=False),
        # Several adapters trained at once, a higher rank, no dropout.
        dict(name="bwd_multi", kind="backward", rows=2048, d_in=4096, d_out=4096, rank=64, adapters=8, layout="runs", base=0.1, drop=0.0, fused=False),
        # The rounds of one prompt's rollouts at K = 5.
        dict(name="loss_64", kind="loss", rounds=64, k=5, hidden=64, mismatch=0.3),
        # A batch of 256 prompts with 8 rollouts of up to 64 rounds at K = 25, the wider MLP.
        dict(name="loss_66k_k25", kind="loss", rounds=66560, k=25, hidden=256, mismatch=0.3),
    ]


def _log_int(rng, lo, hi):
    """An integer in [lo, hi], uniform in the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["forward", "forward", "backward", "backward", "loss"])
    if kind == "loss":
        k = rng.randint(1, 31)
        return dict(kind=kind, rounds=_log_int(rng, 1, 1600000 // k), k=k, hidden=rng.choice([_log_int(rng, 1, 256), 64, 256]),
                    mismatch=rng.choice([0.1, 0.3, 0.6]))
    d_in, d_out = 8 * _log_int(rng, 8, 1024), 8 * _log_int(rng, 8, 1024)
    rows = _log_int(rng, 1, min(8192, 8192 * 5120 * 8192 // (d_in * d_out) // (1 if kind == "forward" else 2)))
    rank = rng.choice([8, 16, 16, 16, 24, 32, 64, 128])
    return dict(kind=kind, rows=rows, d_in=d_in, d_out=d_out, rank=rank, adapters=_log_int(rng, 1, min(64, 2048 // rank)),
                layout=rng.choice(["runs", "runs", "rows"]), base=rng.choice([0.0, 0.1, 0.5]), drop=rng.choice([0.0, 0.05, 0.3]),
                fused=rng.random() < 0.3)


# ---------------------------------------------------------------- inputs (plain torch, from the seed alone)
def _normal(g, shape, std, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def _rows(g, case, width, std):
    """Rows of `width` values: a tensor by itself, or a part of a wider buffer."""
    if case["fused"]:
        return _normal(g, (case["rows"], width + 256), std)[:, 128:128 + width]
    return _normal(g, (case["rows"], width), std)


def _adapter_of_rows(case, seed):
    """Each row's adapter: requests of a few rows side by side, or every row its own."""
    rng = np.random.default_rng(int(seed) + 5)
    M, n = case["rows"], case["adapters"]
    if case["layout"] == "rows":
        ids = rng.integers(0, n, M)
        ids[rng.random(M) < case["base"]] = -1
    else:
        cuts = np.sort(rng.integers(0, M + 1, min(M, 2 * n) - 1)) if M > 1 else np.zeros(0, dtype=np.int64)
        run = np.searchsorted(cuts, np.arange(M), side="right")
        of_run = rng.permutation(np.arange(2 * n) % n)
        of_run[rng.random(2 * n) < case["base"]] = -1
        ids = of_run[run]
    return torch.from_numpy(ids.astype(np.int32)).to(DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    s = dict(case=dict(case))
    if case["kind"] == "loss":
        return _prepare_loss(s, case, g)
    M, K, N, r, n = case["rows"], case["d_in"], case["d_out"], case["rank"], case["adapters"]
    s["x"] = _rows(g, case, K, 1.0)
    s["w"] = _normal(g, (N, K), 0.02)
    s["a"] = torch.empty((n, r, K), dtype=torch.bfloat16, device=DEV).uniform_(-1 / math.sqrt(K), 1 / math.sqrt(K), generator=g)
    s["b"] = _normal(g, (n, N, r), 0.02)
    s["scaling"] = 32.0 / r * torch.empty(n, device=DEV).uniform_(0.5, 1.5, generator=g)
    s["adapter"] = _adapter_of_rows(case, seed)
    s["seed"] = torch.tensor([(int(seed) * 0x9E3779B97F4A7C15 + 12345) % (1 << 63)], dtype=torch.int64, device=DEV)
    s["site"] = 7
    if case["kind"] == "forward":
        s["y"] = torch.empty((M, N), dtype=torch.bfloat16, device=DEV)
        s["u"] = torch.empty((M, r), device=DEV)
        return s
    s["dy"] = _rows(g, case, N, 1.0 / math.sqrt(M))
    s["u"] = _low(s, _dropped(s, s["x"].float()), s["a"].float().flatten(0, 1).T).sum(1)      # as the forward pass leaves it
    s["dx"] = torch.empty((M, K), dtype=torch.bfloat16, device=DEV)
    s["da"] = torch.empty((n, r, K), device=DEV)
    s["db"] = torch.empty((n, N, r), device=DEV)
    s["t"] = torch.empty((M, r), device=DEV)
    return s


def _prepare_loss(s, case, g):
    n, K, H = case["rounds"], case["k"], case["hidden"]
    rand = lambda *shape: torch.empty(shape, device=DEV).uniform_(generator=g)  # noqa: E731
    norm = lambda *shape: torch.empty(shape, device=DEV).normal_(generator=g)  # noqa: E731
    s["argmax"] = torch.randint(0, 150000, (n, K + 1), dtype=torch.int32, device=DEV, generator=g)
    match = rand(n, K) >= case["mismatch"]
    s["draft"] = torch.where(match, s["argmax"][:, :K], s["argmax"][:, :K] + 1).contiguous()
    top = 6.0 + 1.5 * norm(n, K + 1)
    st = torch.empty((n, K + 1, 5), device=DEV)
    st[..., 0] = top
    st[..., 1] = top + torch.log(rand(n, K + 1).clamp(min=1e-6)) * 0.7
    st[..., 2] = top + 4.0 * rand(n, K + 1)
    st[..., 3] = 4.0 * rand(n, K + 1)
    st[:, :K, 4] = torch.where(match, top[:, :K], top[:, :K] + 1.5 * torch.log(rand(n, K).clamp(min=1e-6)))
    st[:, K, 4] = math.nan                                       # the bonus row scores no draft
    s["stats"] = st
    s["w1"] = (rand(H, 8) * 2 - 1) / math.sqrt(8.0)
    s["b1"] = (rand(H) * 2 - 1) / math.sqrt(8.0)
    s["w2"] = (rand(H) * 2 - 1) / math.sqrt(H)
    s["b2"] = (rand(1) * 2 - 1) / math.sqrt(H)
    # the behaviour and the reference policy: near the present one, as after a few updates
    z = _logits(_features(s["draft"], s["argmax"], st), s)
    s["p_old"] = torch.sigmoid(z + 0.25 * norm(n, K))
    s["p_ref"] = torch.sigmoid(z + 0.5 * norm(n, K))
    keep = rand(n, K) < s["p_old"]
    s["accept"] = (match | keep).to(torch.uint8)
    stop = (~match & ~keep).to(torch.int32)
    s["eff"] = (~match & (torch.cumsum(stop, 1) - stop == 0)).to(torch.uint8)
    s["adv"] = norm(n, K) * s["eff"]
    s["out"] = None
    return s


# ---------------------------------------------------------------- the plain form
def _mulhilo(m, c):
    """High and low 32 bits of the product of two 32-bit numbers, in 64-bit integers (which wrap)."""
    p = m * c
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _kept(s):
    """The truth values of the dropout mask, [M, K]: 16 bits of Philox4x32-10 at counter (k / 8, m, site, 2) against the threshold."""
    M, K = s["case"]["rows"], s["case"]["d_in"]
    seed = s["seed"]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    n = (K + 7) // 8
    c0 = torch.arange(n, device=DEV).expand(M, n)
    c1 = torch.arange(M, device=DEV)[:, None].expand(M, n)
    c2, c3 = torch.full_like(c0, s["site"]), torch.full_like(c0, 2)
    for _ in range(10):
        h0, l0 = _mulhilo(0xD2511F53, c0)
        h1, l1 = _mulhilo(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack((c0, c1, c2, c3), dim=-1)
    halves = torch.stack((words & 0xFFFF, words >> 16), dim=-1)
    return halves.view(M, 8 * n)[:, :K] >= _threshold(s["case"])


def _threshold(case):
    return int(math.floor(case["drop"] * 65536 + 0.5))


def _dropped(s, x):
    """x with the dropped places zero, without the 1 / (1 - p) of the places kept."""
    return torch.where(_kept(s), x, 0.0) if s["case"]["drop"] > 0 else x


def _low(s, x, every):
    """[M, adapters, r]: the rows of x against every adapter, zero but for the row's own, scaled."""
    n = s["case"]["adapters"]
    mine = s["adapter"][:, None] == torch.arange(n, device=DEV)
    c = s["scaling"] * (65536.0 / (65536 - _threshold(s["case"])))
    return torch.where(mine[..., None], (x @ every).view(-1, n, s["case"]["rank"]) * c[:, None], 0.0)


def _forward(s):
    x = s["x"].float()
    u = _low(s, _dropped(s, x), s["a"].float().flatten(0, 1).T)
    y = x @ s["w"].float().T + u.flatten(1) @ s["b"].float().transpose(1, 2).flatten(0, 1)
    return dict(y=y.to(torch.bfloat16), u=u.sum(1))


def _backward(s):
    case = s["case"]
    n, r = case["adapters"], case["rank"]
    x, dy, a = s["x"].float(), s["dy"].float(), s["a"].float().flatten(0, 1)
    t = _low(s, dy, s["b"].float().permute(1, 0, 2).flatten(1))
    dx = dy @ s["w"].float() + _dropped(s, t.flatten(1) @ a)
    da = t.flatten(1).T @ _dropped(s, x)
    mine = s["adapter"][:, None] == torch.arange(n, device=DEV)
    u = torch.where(mine[..., None], s["u"][:, None, :], 0.0)
    db = (dy.T @ u.flatten(1)).view(-1, n, r).transpose(0, 1)
    return dict(dx=dx.to(torch.bfloat16), da=da.view(n, r, -1), db=db.contiguous())


def _features(draft, argmax, st):
    """The eight features of every draft position, [n, K, 8]."""
    K = draft.shape[1]
    match = (draft == argmax[:, :K]).float()
    here, after = st[:, :K], st[:, 1:]
    nxt = torch.cat((after[:, :K - 1, 4] - after[:, :K - 1, 2], torch.zeros_like(after[:, :1, 4])), dim=1)
    at = torch.arange(1, K + 1, device=DEV).float().expand_as(match)
    return torch.stack((here[..., 4] - here[..., 2], here[..., 0] - here[..., 2], here[..., 0] - here[..., 1], here[..., 3],
                        after[..., 0] - after[..., 2], nxt, at / K, (torch.cumsum(match, 1) - match) / K), dim=-1)


def _logits(f, s):
    return torch.clamp(f @ s["w1"].T + s["b1"], min=0.0) @ s["w2"] + s["b2"]


def _loss(s):
    n, K = s["draft"].shape
    of = ((s["eff"] != 0) & (s["draft"] != s["argmax"][:, :K])).flatten().nonzero()[:, 0]
    f = _features(s["draft"], s["argmax"], s["stats"]).flatten(0, 1)[of]
    pre = f @ s["w1"].T + s["b1"]
    hid = torch.clamp(pre, min=0.0)
    # the probabilities and the terms in 64 bits: KL is a small difference, the clip a border, the sums are long
    z = (hid.double() @ s["w2"].double() + s["b2"].double())
    took = s["accept"].flatten()[of] != 0
    adv, old, ref = (s[k].flatten()[of].double() for k in ("adv", "p_old", "p_ref"))
    p, q = 1 / (1 + torch.exp(-z)), 1 / (1 + torch.exp(z))
    ratio = torch.where(took, p / old, q / (1 - old))
    low, high = 1 - float(np.float32(CLIP)), 1 + float(np.float32(CLIP))
    plain, cut = ratio * adv, torch.clamp(ratio, low, high) * adv
    ent = -(p * torch.log(p) + q * torch.log(q))
    kl = p * torch.log(p / ref) + q * torch.log(q / (1 - ref))
    inside = plain <= cut
    bh, bk = float(np.float32(BETA_H)), float(np.float32(BETA_KL))
    dz = torch.where(inside, -plain * torch.where(took, q, -p), 0.0) + p * q * (bh * z + bk * (z - torch.log(ref / (1 - ref))))
    sums = torch.stack((torch.minimum(plain, cut).sum(), ent.sum(), kl.sum()))
    loss = torch.cat((sums, (-sums[0] - bh * sums[1] + bk * sums[2])[None]))
    c = 1.0 / n
    g = (dz * c).float()
    gh = torch.where(pre > 0, g[:, None] * s["w2"], 0.0)
    spread = lambda v: torch.zeros(n * K, device=DEV).index_put((of,), v).view(n, K)  # noqa: E731
    return dict(loss=loss.float(), p_new=spread(p.float()), dz=spread(g), dw1=gh.T @ f, db1=gh.sum(0, dtype=torch.float64).float(),
                dw2=hid.T @ g, db2=g.sum(0, keepdim=True, dtype=torch.float64).float())


# ---------------------------------------------------------------- a pass
def run(state):
    s = state
    kind = s["case"]["kind"]
    if not own:
        return _forward(s) if kind == "forward" else _backward(s) if kind == "backward" else _loss(s)
    from paper_2605_24793_gb300 import cospec as C
    if kind == "forward":
        C.lora_forward(s["x"], s["w"], s["a"], s["b"], s["scaling"], s["adapter"], s["y"], s["u"], dropout=s["case"]["drop"], seed=s["seed"],
                       site=s["site"])
        return dict(y=s["y"], u=s["u"])
    if kind == "backward":
        C.lora_backward(s["dy"], s["x"], s["w"], s["a"], s["b"], s["scaling"], s["adapter"], s["u"], s["dx"], s["da"], s["db"], s["t"],
                        dropout=s["case"]["drop"], seed=s["seed"], site=s["site"])
        return dict(dx=s["dx"], da=s["da"], db=s["db"])
    s["out"] = C.arbitrate_loss(s["draft"], s["argmax"], s["stats"], s["w1"], s["b1"], s["w2"], s["b2"], s["accept"], s["eff"], s["adv"], s["p_old"],
                                s["p_ref"], C.RLParams(clip_eps=CLIP, beta_h=BETA_H, beta_kl=BETA_KL), grad_scale=1.0 / s["case"]["rounds"],
                                out=s["out"])
    return {k: s["out"][k] for k in ("loss", "p_new", "dz", "dw1", "db1", "dw2", "db2")}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["kind"] == "loss":
        n, K, H, m = case["rounds"], case["k"], case["hidden"], case["mismatch"]
        # mismatches up to the first that is rejected (about half of them are)
        eff = n * m * (1 - (1 - m / 2) ** K) / (m / 2)
        nbytes = n * (4.0 * K + 4 * (K + 1) + 20 * (K + 1) + 2 * K + 12 * K + 8 * K) + 8.0 * (10 * H + 1)
        # per decision and unit: 8 + 1 multiply-adds forward, 1 for w2, 1 for the unit's gradient, 8 for w1
        return dict(bytes=nbytes, flops=eff * H * 2.0 * 19)
    M, K, N, r, n = case["rows"], case["d_in"], case["d_out"], case["rank"], case["adapters"]
    mine = M * (1 - case["base"])
    used = min(n, mine)
    if case["kind"] == "forward":
        return dict(bytes=2.0 * (M * (K + N) + N * K + used * r * (K + N)) + 4.0 * M * (r + 1), flops=2.0 * M * N * K + 2.0 * mine * r * (K + N))
    return dict(bytes=2.0 * (M * (2 * K + N) + N * K + used * r * (K + N)) + 4.0 * n * r * (K + N) + 4.0 * M * (r + 1),
                flops=2.0 * M * N * K + 4.0 * mine * r * (K + N))


# ---------------------------------------------------------------- the definition in 64 bits
def _x_mask(case, seed64, site):
    """The kept places by NumPy's unsigned 64-bit products, row counters along the first axis."""
    M, K = case["rows"], case["d_in"]
    n = -(-K // 8)
    u = np.uint64
    low = u(0xFFFFFFFF)
    c = [np.broadcast_to(np.arange(n, dtype=u)[None, :], (M, n)), np.broadcast_to(np.arange(M, dtype=u)[:, None], (M, n)), u(site), u(2)]
    key = [seed64 & 0xFFFFFFFF, seed64 >> 32]
    for i in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        k = [u((key[0] + i * 0x9E3779B9) & 0xFFFFFFFF), u((key[1] + i * 0xBB67AE85) & 0xFFFFFFFF)]
        c = [(b >> u(32)) ^ c[1] ^ k[0], b & low, (a >> u(32)) ^ c[3] ^ k[1], a & low]
    bits = np.empty((M, n, 8), dtype=np.uint16)
    for w in range(4):
        bits[:, :, 2 * w], bits[:, :, 2 * w + 1] = c[w] & u(0xFFFF), c[w] >> u(16)
    return torch.from_numpy(bits.reshape(M, 8 * n)[:, :K].astype(np.int32)).to(DEV) >= round(case["drop"] * 65536)


def _x_lora(case, seed):
    s = prepare(case, seed)
    x, w = s["x"].double(), s["w"].double()
    keep = _x_mask(case, int(s["seed"]), s["site"]).double() if case["drop"] > 0 else torch.ones_like(x)
    xd = x * keep
    factor = s["scaling"].double() / (1 - round(case["drop"] * 65536) / 65536.0)
    groups = [(i, (s["adapter"] == i).nonzero()[:, 0]) for i in range(case["adapters"])]
    if case["kind"] == "forward":
        y, u = x @ w.T, torch.zeros_like(s["u"], dtype=torch.float64)
        for i, at in groups:
            u[at] = factor[i] * (xd[at] @ s["a"][i].double().T)
            y[at] += u[at] @ s["b"][i].double().T
        return dict(y=y, u=u)
    dy = s["dy"].double()
    dx, da, db = dy @ w, torch.zeros_like(s["da"], dtype=torch.float64), torch.zeros_like(s["db"], dtype=torch.float64)
    for i, at in groups:
        t = factor[i] * (dy[at] @ s["b"][i].double())
        dx[at] += keep[at] * (t @ s["a"][i].double())
        da[i] = t.T @ xd[at]
        db[i] = dy[at].T @ s["u"][at].double()
    return dict(dx=dx, da=da, db=db)


def _x_loss(case, seed):
    """The objective on the CPU in 64 bits; its gradient for the weights is torch's own."""
    s = {k: v.cpu() if torch.is_tensor(v) else v for k, v in prepare(case, seed).items()}
    n, K, st = case["rounds"], case["k"], s["stats"].double()
    at = ((s["eff"] != 0) & (s["draft"] != s["argmax"][:, :K])).nonzero()
    i, j = at[:, 0], at[:, 1]
    before = torch.cumsum(torch.nn.functional.pad((s["draft"] == s["argmax"][:, :K]).double(), (1, 0)), 1)[i, j]
    a, b = st[i, j], st[i, j + 1]
    f = torch.stack((a[:, 4] - a[:, 2], a[:, 0] - a[:, 2], a[:, 0] - a[:, 1], a[:, 3], b[:, 0] - b[:, 2],
                     torch.where(j + 1 < K, b[:, 4] - b[:, 2], 0.0), (j + 1) / K, before / K), dim=1).double()
    par = [s[k].double().requires_grad_() for k in ("w1", "b1", "w2", "b2")]
    z = torch.relu(f @ par[0].T + par[1]) @ par[2] + par[3]
    z.retain_grad()
    took = s["accept"][i, j] != 0
    adv, old, ref = (s[k][i, j].double() for k in ("adv", "p_old", "p_ref"))
    new = torch.distributions.Bernoulli(logits=z)
    ratio = torch.exp(new.log_prob(took.double()) - torch.log(torch.where(took, old, 1 - old)))
    eps, bh, bk = (float(np.float32(v)) for v in (CLIP, BETA_H, BETA_KL))
    terms = (torch.minimum(ratio * adv, ratio.clamp(1 - eps, 1 + eps) * adv).sum(), new.entropy().sum(),
             torch.distributions.kl_divergence(new, torch.distributions.Bernoulli(probs=ref)).sum())
    total = -terms[0] - bh * terms[1] + bk * terms[2]
    (total / n).backward()
    full = lambda v: torch.zeros((n, K), dtype=torch.float64).index_put((i, j), v)  # noqa: E731
    out = dict(loss=torch.stack((*terms, total)).detach(), p_new=full(torch.sigmoid(z).detach()), dz=full(z.grad), dw1=par[0].grad, db1=par[1].grad,
               dw2=par[2].grad, db2=par[3].grad)
    return {k: v.to(DEV) for k, v in out.items()}


def exact(case, seed):
    return _x_loss(case, seed) if case["kind"] == "loss" else _x_lora(case, seed)
