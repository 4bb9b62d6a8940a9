"""The adapters and the policy loss in the runs they are made for: a layer of the arbitrator over the 8-bit cache, a training
step over two projections, an update of the decision MLP."""
import math

import numpy as np
import pytest
import torch

from paper_2605_24793_gb300 import arbitrator as A
from paper_2605_24793_gb300 import build as BLD
from paper_2605_24793_gb300 import cospec as C
from paper_2605_24793_gb300 import rlstage
from paper_2605_24793_gb300 import workload as W
from paper_2605_24793_gb300.kv8round import quantise_cache, rope_tables

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def lib():
    C.load_library(BLD.build())
    torch.cuda.set_device(0)
    C.get_device_error()


def _layer(B=3, ctx=70, rows=9, hidden=320, adapters=2):
    cfg = W.CONFIGS["tiny"].replace(batch=B, ctx_lo=ctx, ctx_hi=ctx, k=rows - 1, hidden=hidden, shuffled_pages=True, qkv_std=1.0)
    inp = W.make_round_inputs(cfg, device="cuda")
    pool = quantise_cache(inp["k_pages"], inp["v_pages"], inp["page_table"], inp["ctx_len"])
    rope = rope_tables(inp["page_table"].shape[1] * 16, cfg.head_dim)
    return A.RegionLayer(pool, rope, inp["page_table"], inp["ctx_len"], rows, hidden, cfg.q_heads, adapters, seed=3)


def _projection(x, w, a, b, scaling, adapter):
    y = x @ w.float().T
    for i in range(a.shape[0]):
        mine = (adapter == i).float()[:, None]
        y = y + mine * scaling[i] * ((x @ a[i].float().T) @ b[i].float().T)
    return y.to(torch.bfloat16).float()


def _reference(L, x, adapter):
    """The layer in 32-bit torch, rounded to bf16 where the calls hand on bf16."""
    B, R = L.shape
    hq, hkv, D = L.heads
    qkv = _projection(x.float().view(B * R, -1), L.w_qkv, L.a_qkv, L.b_qkv, L.scaling, adapter).view(B, R, hq + 2 * hkv, D)
    pos = L.ctx_len.long()[:, None] + torch.arange(R, device="cuda")
    c, s = L.rope.cos[pos][:, :, None], L.rope.sin[pos][:, :, None]

    def turn(z):
        p, q = z[..., :D // 2], z[..., D // 2:]
        return torch.cat((p * c - q * s, q * c + p * s), -1).to(torch.bfloat16).float()

    q, k, v = turn(qkv[:, :, :hq]), turn(qkv[:, :, hq:hq + hkv]), qkv[:, :, hq + hkv:]
    out = torch.empty((B, R, hq, D), device="cuda")
    for b in range(B):
        n = int(L.ctx_len[b])
        ids = L.page_table[b, :-(-n // 16)].long()
        for h in range(hkv):
            sc = L.pool.scale[0, ids, h]
            kc = (L.pool.k[0][ids, h].float() * sc[:, 0, None, None]).flatten(0, 1)[:n]
            vc = (L.pool.v[0][ids, h].float() * sc[:, 1, None, None]).transpose(1, 2).flatten(0, 1)[:n]
            kk, vv = torch.cat((kc, k[b, :, h])), torch.cat((vc, v[b, :, h]))
            g = hq // hkv
            p = torch.softmax(q[b, :, h * g:(h + 1) * g] @ kk.T / math.sqrt(D), -1)
            out[b, :, h * g:(h + 1) * g] = p @ vv
    out = out.to(torch.bfloat16).float().view(B * R, hq * D)
    return _projection(out, L.w_out, L.a_out, L.b_out, L.scaling, adapter).view(B, R, -1)


@pytest.mark.parametrize("B,ctx,rows,hidden,adapters", [(3, 70, 9, 320, 2), (1, 16, 1, 64, 1), (2, 33, 53, 512, 5)])
def test_region_layer(B, ctx, rows, hidden, adapters):
    L = _layer(B, ctx, rows, hidden, adapters)
    x = torch.randn((B, rows, hidden), device="cuda").to(torch.bfloat16)
    adapter = torch.randint(-1, adapters, (B * rows,), dtype=torch.int32, device="cuda")
    y = L.run(x, adapter).float()
    assert C.get_device_error() == 0
    ref = _reference(L, x, adapter)
    # the attention's tolerance on its output, through a projection of unit gain: 2e-2 + 1e-2 |ref|
    assert ((y - ref).abs() <= 2e-2 + 1e-2 * ref.abs()).all()


def test_region_layer_captured():
    L = _layer()
    x = torch.randn((3, 9, 320), device="cuda").to(torch.bfloat16)
    adapter = torch.zeros(27, dtype=torch.int32, device="cuda")
    L.run(x, adapter)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        L.run(x, adapter)
    x.normal_()
    adapter[5:] = 1
    g.replay()
    torch.cuda.synchronize()
    a = L.out.clone()
    assert torch.equal(a, L.run(x, adapter)) and C.get_device_error() == 0


def test_training_step_of_two_projections():
    """y = P2(P1(x)), both with adapters and dropout, against autograd in 32 bits with the same masks (read off the first pass's
    linearity: an identity factor's u is the dropped row).  The hidden rows and their gradient are rounded to bf16 (half a step 2^-8 at most,
    2^-9.8 in the mean) and enter once more by a product each: in the norm the gradients agree to 2^-7."""
    M, K, H, N, r, n = 200, 128, 192, 256, 16, 3
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    bf = lambda *s, std: torch.empty(s, device="cuda").normal_(0.0, std, generator=g).to(torch.bfloat16)  # noqa: E731
    x, dy = bf(M, K, std=1.0), bf(M, N, std=1.0)
    p1 = (bf(H, K, std=K ** -0.5), bf(n, r, K, std=K ** -0.5), bf(n, H, r, std=0.1))
    p2 = (bf(N, H, std=H ** -0.5), bf(n, r, H, std=H ** -0.5), bf(n, N, r, std=0.1))
    sc = torch.tensor([1.0, 2.0, 0.5], device="cuda")
    ids = (torch.arange(M, device="cuda") % (n + 1) - 1).to(torch.int32)
    seed = torch.tensor([77], dtype=torch.int64, device="cuda")
    f32 = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    e16 = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    h, y, u1, u2, dh, dx, t = e16(M, H), e16(M, N), f32(M, r), f32(M, r), e16(M, H), e16(M, K), f32(M, r)
    grads = [f32(n, r, K), f32(n, H, r), f32(n, r, H), f32(n, N, r)]
    C.lora_forward(x, *p1, sc, ids, h, u1, dropout=0.2, seed=seed, site=0)
    C.lora_forward(h, *p2, sc, ids, y, u2, dropout=0.2, seed=seed, site=1)
    C.lora_backward(dy, h, *p2, sc, ids, u2, dh, grads[2], grads[3], t, dropout=0.2, seed=seed, site=1)
    C.lora_backward(dh, x, *p1, sc, ids, u1, dx, grads[0], grads[1], t, dropout=0.2, seed=seed, site=0)
    assert C.get_device_error() == 0
    kept = 1 - math.floor(0.2 * 65536 + 0.5) / 65536

    def mask(width, site):
        ones, out = torch.ones((M, width), dtype=torch.bfloat16, device="cuda"), torch.empty((M, width), device="cuda")
        one = torch.ones(1, device="cuda")
        for c in range(0, width, 8):
            a = torch.zeros((1, 8, width), dtype=torch.bfloat16, device="cuda")
            a[0, torch.arange(8), c + torch.arange(8)] = 1
            u = f32(M, 8)
            C.lora_forward(ones, torch.zeros((8, width), dtype=torch.bfloat16, device="cuda"), a, torch.zeros((1, 8, 8), dtype=torch.bfloat16, device="cuda"),
                           one, torch.zeros(M, dtype=torch.int32, device="cuda"), e16(M, 8), u, dropout=0.2, seed=seed, site=site)
            out[:, c:c + 8] = u * kept
        assert ((out - out.round()).abs() < 1e-5).all()
        return out.round()

    m1, m2 = mask(K, 0), mask(H, 1)
    assert abs(float(m1.mean()) - 0.8) < 0.02 and not torch.equal(m1, m2[:, :K])
    X = x.float().requires_grad_()
    P = [q.float().requires_grad_() for q in (p1[1], p1[2], p2[1], p2[2])]
    mine = [(ids == i).float()[:, None] for i in range(n)]
    hid = X @ p1[0].float().T + sum(mine[i] * sc[i] / kept * (((X * m1) @ P[0][i].T) @ P[1][i].T) for i in range(n))
    out = hid @ p2[0].float().T + sum(mine[i] * sc[i] / kept * (((hid * m2) @ P[2][i].T) @ P[3][i].T) for i in range(n))
    out.backward(dy.float())
    near = lambda a, b: float((a.float() - b).norm() / b.norm()) <= 2.0 ** -7  # noqa: E731
    assert near(y, out.detach()) and near(dx, X.grad)
    assert all(near(a, q.grad) for a, q in zip(grads, P))


def test_policy_step():
    """The step's parts by themselves give the same; its tensors are filled again, also from a graph."""
    R, K, H = 300, 7, 64
    draft, argmax, st, w1, b1, w2, b2 = [torch.from_numpy(a).cuda() for a in W.policy_rounds(5, R, K, H)]
    rng = np.random.default_rng(5)
    go = torch.tensor([0, 5, 10], dtype=torch.int32, device="cuda")
    ro = torch.arange(0, R + 1, 30, dtype=torch.int32, device="cuda")
    co = torch.from_numpy((rng.random(10) < 0.5).astype(np.uint8)).cuda()
    p, ref = (torch.from_numpy(rng.uniform(0.1, 0.9, (R, K)).astype(np.float32)).cuda() for _ in range(2))
    act = ((draft == argmax[:, :K]) | torch.from_numpy(rng.random((R, K)) < 0.5).cuda()).to(torch.uint8)
    step = rlstage.PolicyStep(go, co, ro, draft, argmax, st, (w1, b1, w2, b2), p, ref, act)
    out = step.run()
    first = {k: v.clone() for k, v in out.items() if k != "ws"}
    adv = step.advantages()
    again = C.arbitrate_loss(draft, argmax, st, w1, b1, w2, b2, act, adv["eff"], adv["adv_dec"], p, ref, C.RLParams(), grad_scale=1.0 / R)
    assert all(torch.equal(first[k], again[k]) for k in first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step.run()
    for k in first:
        out[k].fill_(9)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(first[k], out[k]) for k in first) and C.get_device_error() == 0
