"""A verify/arbitrate round over an 8-bit cache against the oracles: the context quantised from a bf16
cache, queries and keys rotated on the way, every layer attended (all pages, or selected ones), the
accepted rows appended, round after round."""
import numpy as np
import pytest
import torch

from oracle import cospec_kv8 as K
from oracle import cospec_oracle as O
from paper_2605_24793_gb300 import build as BLD
from paper_2605_24793_gb300 import cospec as C
from paper_2605_24793_gb300 import workload as W
from paper_2605_24793_gb300.kv8round import Kv8Round

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    C.load_library(BLD.build())
    torch.cuda.set_device(0)
    C.get_device_error()


def _rotated32(x, start, cos, sin):
    """Half-style rotation of x [L, B, R, H, D] in fp32, each product and sum rounded by itself: the kernel's own steps."""
    x = x.float().cpu().numpy()
    h = cos.shape[1]
    pos = start[:, None] + np.arange(x.shape[2])
    c, s = cos[pos][None, :, :, None], sin[pos][None, :, :, None]
    a, b = x[..., :h], x[..., h:]
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


def _bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("pages", [None, 3])
@pytest.mark.parametrize("heads,D,k", [((8, 2), 64, 4), ((12, 4), 128, 7), ((16, 2), 128, 5)])
def test_rounds_match_the_oracles(pages, heads, D, k):
    cfg = W.CONFIGS["tiny"].replace(batch=3, ctx_lo=40, ctx_hi=150, layers=2, q_heads=heads[0], kv_heads=heads[1], head_dim=D, k=k,
                                    shuffled_pages=True, qkv_std=1.0)
    inp = W.make_round_inputs(cfg, device="cuda", extra_tokens=2 * cfg.rows)
    host = {n: (v.cpu() if torch.is_tensor(v) else v) for n, v in inp.items()}
    host["mlp"] = inp["mlp"]
    x = O.lmhead_logits(host["hidden"], host["w"])
    draft = W.synth_drafts(cfg, O.topk_ids(x, 8).reshape(cfg.batch, cfg.rows, 8))
    ref = O.cospec_round(host, draft, cfg.lam, with_attention=False, with_commit=False)
    rnd = Kv8Round(inp, draft, cfg.lam, keep_attn=True, pages=pages, sink=1, recent=1)
    cos, sin = rnd.rope.cos.cpu().numpy(), rnd.rope.sin.cpu().numpy()
    table, ctx = inp["page_table_np"], inp["ctx_len_np"].astype(np.int64)
    pool = K.new_pool(cfg.layers, rnd.pool.num_pages, cfg.kv_heads, D)
    T = int(ctx.max())
    cached = []
    for t in (host["k_pages"], host["v_pages"]):
        rows = np.zeros((cfg.layers, cfg.batch, T, cfg.kv_heads, D))
        for b in range(cfg.batch):
            at = np.arange(ctx[b])
            rows[:, b, :ctx[b]] = t.float().numpy()[:, table[b][at // 16], :, at % 16].transpose(1, 0, 2, 3)
        cached.append(rows)
    K.append(pool, cached[0], cached[1], table, [0] * cfg.batch, ctx)
    scale = rnd.pool.scale.cpu().numpy()
    for p, which in ((pool["k"], rnd.pool.k), (pool["v"], rnd.pool.v)):
        got = which.view(torch.uint8).cpu().numpy()
        for b in range(cfg.batch):
            for n in range(-(-int(ctx[b]) // 16)):
                assert K.same_codes(got[:, table[b][n]], p[:, table[b][n]])
                np.testing.assert_array_equal(scale[:, table[b][n]], pool["scale"][:, table[b][n]])
    for _ in range(2):
        rnd.run(restore=False)
        torch.cuda.synchronize()
        assert C.get_device_error() == 0
        kr = _rotated32(inp["k_blk"], ctx, cos, sin)
        qr = _bf16(_rotated32(inp["q"], ctx, cos, sin))
        vb = host["v_blk"].double().numpy()
        for l in range(cfg.layers):
            sel = None if pages is None else K.select(qr[l], pool, l, table, ctx, pages, 1, 1)
            o, mag = K.attention(qr[l], _bf16(kr[l]), vb[l], pool, l, table, ctx, sel=sel)
            err = np.abs(rnd.attn_out[l].double().cpu().numpy() - o)
            assert np.all(err <= 2.0 ** -8 * (np.abs(o) + mag)), float((err / (np.abs(o) + mag)).max())
        np.testing.assert_array_equal(rnd.accept_len.cpu().numpy(), ref["s"])
        np.testing.assert_array_equal(rnd.emitted.cpu().numpy(), ref["emitted"])
        K.append(pool, kr.astype(np.float64), vb, table, ctx, ref["s"])
        ctx = ctx + ref["s"]
        np.testing.assert_array_equal(rnd.ctx_len.cpu().numpy(), ctx)
        for name, t in (("k", rnd.pool.k), ("v", rnd.pool.v)):
            got = t.view(torch.uint8).cpu().numpy()
            for b in range(cfg.batch):
                for n in range(-(-int(ctx[b]) // 16)):
                    used = min(16, int(ctx[b]) - 16 * n)
                    cut = (lambda c: c[:, table[b][n], :, :used]) if name == "k" else (lambda c: c[:, table[b][n], :, :, :used])
                    assert K.same_codes(cut(got), cut(pool[name])), (name, b, n)
        # the next round's block: the same projections at later positions
        rnd.max_ctx = int(ctx.max())


def test_a_captured_round_repeats():
    cfg = W.CONFIGS["tiny"].replace(batch=2, ctx_lo=100, ctx_hi=300, layers=3, shuffled_pages=True, qkv_std=1.0)
    draft = np.zeros((cfg.batch, cfg.k), np.int32)
    for pages in (None, 8):
        inp = W.make_round_inputs(cfg, device="cuda")       # (a round advances its inputs' context lengths)
        rnd = Kv8Round(inp, draft, cfg.lam, keep_attn=True, pages=pages)
        rnd.run(restore=False)
        torch.cuda.synchronize()
        want = [t.clone() for t in (rnd.attn_out, rnd.accept_len, rnd.emitted, rnd.ctx_len)]
        rnd.capture()
        for _ in range(3):
            rnd.replay()
        torch.cuda.synchronize()
        assert C.get_device_error() == 0
        for a, b in zip(want, (rnd.attn_out, rnd.accept_len, rnd.emitted, rnd.ctx_len)):
            assert torch.equal(a, b)


def test_a_round_needs_every_layers_cache():
    cfg = W.CONFIGS["tiny"].replace(layers=2)
    inp = W.make_round_inputs(cfg, device="cuda", alias_layers=True)
    with pytest.raises(ValueError, match="every layer"):
        Kv8Round(inp, np.zeros((cfg.batch, cfg.k), np.int32))
