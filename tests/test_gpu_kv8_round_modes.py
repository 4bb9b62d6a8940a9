"""A round over the 8-bit cache in VerifyRound's other modes: sampled candidates, speculative sampling, a longest context given
beforehand.  The hidden rows are inputs, so decisions and tokens are those of the round over the bf16 cache."""
import numpy as np
import pytest
import torch

from oracle import cospec_oracle as O
from paper_2605_24793_gb300 import build as BLD
from paper_2605_24793_gb300 import cospec as C
from paper_2605_24793_gb300 import workload as W
from paper_2605_24793_gb300.kv8round import Kv8Round
from paper_2605_24793_gb300.round import VerifyRound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    C.load_library(BLD.build())
    torch.cuda.set_device(0)
    C.get_device_error()


def _cfg(**kw):
    return W.CONFIGS["tiny"].replace(batch=4, k=5, ctx_lo=30, ctx_hi=300, layers=2, qkv_std=1.0, shuffled_pages=True, **kw)


def _pair(cfg, draft, **kw):
    inputs = [W.make_round_inputs(cfg, device="cuda", extra_tokens=2 * cfg.rows) for _ in range(2)]
    return Kv8Round(inputs[0], draft, cfg.lam, **kw), VerifyRound(inputs[1], draft, cfg.lam, **kw)


def _same(a, b, rounds=2):
    for r in range(rounds):
        for rnd in (a, b):
            rnd.seed.fill_(r + 11)
            rnd.run(restore=False)
        torch.cuda.synchronize()
        assert C.get_device_error() == 0
        for n in ("argmax", "accept", "accept_len", "emitted", "ctx_len"):
            assert torch.equal(getattr(a, n), getattr(b, n)), (r, n)


@pytest.mark.parametrize("T", [None, 0.7, 1.0])
def test_sampled_rounds(T):
    cfg = _cfg()
    draft = np.random.default_rng(1).integers(0, cfg.vocab, (cfg.batch, cfg.k)).astype(np.int32)
    a, b = _pair(cfg, draft, temperature=T, seed=11, max_ctx=320)
    assert a.max_ctx == 320 and a.temperature == T and int(a.seed) == 11
    _same(a, b)


def test_speculative_sampling_rounds():
    cfg = _cfg()
    inp = W.make_round_inputs(cfg, device="cuda")
    x = O.lmhead_logits(inp["hidden"].cpu(), inp["w"].cpu()).reshape(cfg.batch, cfg.rows, cfg.vocab)
    q = W.draft_distributions(cfg, x, noise=1.0)
    draft = W.sample_from(cfg, q)
    a, b = _pair(cfg, draft, seed=7, sps_q=torch.from_numpy(q).cuda())
    _same(a, b)
    assert torch.equal(a.target, b.target)
    a.capture()
    a.replay()
    torch.cuda.synchronize()
    assert C.get_device_error() == 0


def test_the_bf16_cache_is_let_go():
    """A round made from a bf16 cache holds no reference to it, and runs, packs its inputs and replays without it."""
    import gc
    import weakref
    cfg = _cfg().replace(ctx_lo=2000, ctx_hi=3000)
    draft = np.random.default_rng(2).integers(0, cfg.vocab, (cfg.batch, cfg.k)).astype(np.int32)
    inp = W.make_round_inputs(cfg, device="cuda")
    refs = [weakref.ref(inp[n]) for n in ("k_pages", "v_pages")]
    nbytes = sum(inp[n].numel() * 2 for n in ("k_pages", "v_pages"))
    rnd = Kv8Round(inp, draft, cfg.lam)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    del inp
    gc.collect()
    assert all(r() is None for r in refs)
    assert before - torch.cuda.memory_allocated() >= nbytes
    rnd.run()
    want = [t.clone() for t in (rnd.attn_out, rnd.accept_len, rnd.emitted)]
    rnd.pack_step_io()
    rnd.capture()
    rnd.replay()
    torch.cuda.synchronize()
    assert C.get_device_error() == 0
    for a, b in zip(want, (rnd.attn_out, rnd.accept_len, rnd.emitted)):
        assert torch.equal(a, b)
