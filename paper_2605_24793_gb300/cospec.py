"""Python binding of libcospec.so: the calls of include/cospec.h, same names.

Argument marshalling only -- shapes are read off the tensors and checked
against one another (a mis-shaped tensor would make a kernel read or write
past its end), pointers and the current CUDA stream are passed through
ctypes, and every step runs in the library's CUDA kernels.  There is no CPU or PyTorch fallback: if the
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcospec.so")

POLICY_MLP, POLICY_TARGET, POLICY_DRAFT = 0, 1, 2
DEVERR_PAGE, DEVERR_CTX, DEVERR_TOKEN, DEVERR_TIMEOUT, DEVERR_OFFSETS = 1, 2, 4, 8, 16
DEVERR_POSITION = 32

EXPORTED = ("cospec_status_string", "cospec_last_cuda_error", "cospec_get_device_error", "cospec_num_sms",
            "cospec_verify_attn", "cospec_lmhead_workspace", "cospec_lmhead_argmax_features",
            "cospec_arbitrate", "cospec_accept_commit", "cospec_lmhead_argmax_features_noalloc",
            "cospec_lmhead_sample_features", "cospec_verify_attn_plan", "cospec_rl_workspace",
            "cospec_rl_advantages", "cospec_verify_attn_plan_model",
            "cospec_lmhead_logits_features", "cospec_sps_workspace", "cospec_sps_accept", "cospec_accept_commit_launches",
            "cospec_verify_attn_variant", "cospec_kv8_append", "cospec_kv8_select", "cospec_kv8_attn")


class AttnDims(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int), ("rows", ctypes.c_int), ("num_q_heads", ctypes.c_int),
                ("num_kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("page_size", ctypes.c_int), ("max_pages_per_seq", ctypes.c_int),
                ("num_pages", ctypes.c_int), ("softmax_scale", ctypes.c_float),
                ("flags", ctypes.c_int)]


class RLParams(ctypes.Structure):
    """cospec_rl_params; defaults are the paper's (App. C)."""
    _fields_ = [(n, ctypes.c_float) for n in
                ("alpha", "beta", "eta_fail", "eps", "clip_eps", "beta_h", "beta_kl")]

    def __init__(self, alpha=1.0, beta=0.25, eta_fail=0.5, eps=1e-6, clip_eps=0.2, beta_h=0.01,
                 beta_kl=0.02):
        super().__init__(alpha, beta, eta_fail, eps, clip_eps, beta_h, beta_kl)


ATTN_KV_STABLE = 1
ATTN_BLOCK_FULL = 2


class Kv8PoolC(ctypes.Structure):
    """cospec_kv8_pool."""
    _fields_ = [(n, ctypes.c_int) for n in ("layers", "num_pages", "num_kv_heads", "head_dim")] + [
        (n, ctypes.c_void_p) for n in ("k", "v", "scale", "summary", "summary_scale")]


class RopeC(ctypes.Structure):
    """cospec_rope."""
    _fields_ = [("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p)] + [
        (n, ctypes.c_int) for n in ("positions", "rot_dim", "interleaved")]


class Strides(ctypes.Structure):
    """cospec_kv8_strides."""
    _fields_ = [(n, ctypes.c_longlong) for n in ("layer", "batch", "row")]


class CospecError(RuntimeError):
    pass


_lib: Optional[ctypes.CDLL] = None

_vp, _i, _sz, _f = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_float
_PDIMS = ctypes.POINTER(AttnDims)
_PPOOL, _PROPE, _PSTR = ctypes.POINTER(Kv8PoolC), ctypes.POINTER(RopeC), ctypes.POINTER(Strides)
# cospec_resident_fn: (kernel, rows, block_rows, splits, user) -> resident clusters
RESIDENT_FN = ctypes.CFUNCTYPE(ctypes.c_longlong, _i, _i, _i, _i, _vp)


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libcospec.so (built by ``paper_2605_24793_gb300.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise CospecError(f"{path} is missing; build it with python -m paper_2605_24793_gb300.build")
    lib = ctypes.CDLL(path)
    sig = {
        "cospec_status_string": (ctypes.c_char_p, [_i]),
        "cospec_last_cuda_error": (ctypes.c_char_p, []),
        "cospec_get_device_error": (_i, [ctypes.POINTER(_i), _vp]),
        "cospec_num_sms": (_i, []),
        "cospec_verify_attn": (_i, [_PDIMS, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
        "cospec_verify_attn_plan": (_i, [_PDIMS, _i, ctypes.POINTER(_i), ctypes.POINTER(_i)]),
        "cospec_verify_attn_variant": (_i, [_PDIMS, _i, ctypes.POINTER(_i)]),
        "cospec_verify_attn_plan_model": (_i, [_PDIMS, _i, _i, RESIDENT_FN, _vp,
                                               ctypes.POINTER(_i), ctypes.POINTER(_i)]),
        "cospec_rl_workspace": (_sz, [_i, _i]),
        "cospec_rl_advantages": (_i, [_i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp,
                                      ctypes.POINTER(RLParams), _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                      _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
        "cospec_lmhead_workspace": (_sz, [_i, _i, _i]),
        "cospec_lmhead_argmax_features": (_i, [_i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
        "cospec_lmhead_argmax_features_noalloc": (_i, [_i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp]),
        "cospec_lmhead_sample_features": (_i, [_i, _i, _i, _vp, _vp, _vp, _f, _vp, _vp, _vp, _vp,
                                               _sz, _vp]),
        "cospec_lmhead_logits_features": (_i, [_i, _i, _i, _vp, _vp, _vp, _f, _vp, _vp, _vp, _vp,
                                               _sz, _vp]),
        "cospec_sps_workspace": (_sz, [_i]),
        "cospec_sps_accept": (_i, [_i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz,
                                   _vp]),
        "cospec_arbitrate": (_i, [_i, _i, _vp, _vp, _vp, _i, _vp, _vp, _vp, _f, _f, _i, _vp, _vp, _vp]),
        "cospec_accept_commit": (_i, [_i, _i, _i, _PDIMS, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                      ctypes.c_longlong, _vp, _vp, _vp, _vp, _vp]),
        "cospec_accept_commit_launches": (_i, [_PDIMS, _i]),
        "cospec_kv8_append": (_i, [_PPOOL, _i, _i, _i, _i, _i, _PROPE, _vp, _PSTR, _vp, _PSTR, _vp, _PSTR, _vp,
                                   _i, _vp, _vp, _vp, _vp, _vp]),
        "cospec_kv8_select": (_i, [_PDIMS, _PPOOL, _i, _vp, _PSTR, _vp, _vp, _i, _i, _i, _vp, _vp]),
        "cospec_kv8_attn": (_i, [_PDIMS, _i, _PPOOL, _i, _vp, _PSTR, _vp, _PSTR, _vp, _PSTR, _vp, _vp, _vp, _i,
                                 _vp, _vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(status: int) -> None:
    if status != 0:
        lib = load_library()
        msg = lib.cospec_status_string(status).decode()
        if status == -4:   # COSPEC_ERR_CUDA: name the runtime error behind it
            msg += f": {lib.cospec_last_cuda_error().decode()}"
        raise CospecError(f"cospec call failed: {msg} ({status})")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _req(t: torch.Tensor, dtype, name: str, ndim: Optional[int] = None):
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name}: expected {ndim} dims, got {t.dim()}")


def _need(cond: bool, msg: str) -> None:
    if not cond:
        raise ValueError(msg)


def _same_device(*tensors: Optional[torch.Tensor]) -> None:
    """Every tensor on the current CUDA device (the library launches there)."""
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.device.index != dev:
            raise ValueError(f"tensor on {t.device}, but the current device is cuda:{dev}")


def check_attn_shapes(q, k_blk, v_blk, k_pages, v_pages, page_table, ctx_len, out) -> None:
    """Shapes of one verify-attention call agree: q / out [B,R,Hq,D], block
    K/V [B,R,Hkv,D], pools [num_pages,Hkv,P,D], page_table [B,max_pages],
    ctx_len [B]."""
    _need(q.dim() == 4, "q must be [B, R, Hq, D]")
    B, R, Hq, D = q.shape
    _need(k_pages.dim() == 4, "k_pages must be [num_pages, Hkv, P, D]")
    _need(tuple(v_pages.shape) == tuple(k_pages.shape), "v_pages must have k_pages' shape")
    Hkv = k_pages.shape[1]
    _need(k_pages.shape[3] == D, "k_pages head_dim differs from q's")
    _need(tuple(k_blk.shape) == (B, R, Hkv, D), "k_blk must be [B, R, Hkv, D]")
    _need(tuple(v_blk.shape) == (B, R, Hkv, D), "v_blk must be [B, R, Hkv, D]")
    _need(tuple(out.shape) == tuple(q.shape), "out must have q's shape")
    _need(page_table.dim() == 2 and page_table.shape[0] == B, "page_table must be [B, max_pages]")
    _need(ctx_len.dim() == 1 and ctx_len.shape[0] == B, "ctx_len must be [B]")


def check_arbitrate_shapes(draft, argmax, stats, w1, b1, w2, mode, p_out, accept) -> None:
    """draft [B,K]; argmax B*(K+1) ids; stats B*(K+1)*5; p_out / accept B*K;
    for the MLP policy w1 [H,8], b1 [H], w2 [H]."""
    _need(draft.dim() == 2, "draft must be [B, K]")
    B, K = draft.shape
    _need(argmax.numel() == B * (K + 1) and stats.numel() == B * (K + 1) * 5,
          "argmax / stats must hold K+1 rows per sequence")
    _need(p_out.numel() == B * K and accept.numel() == B * K, "p_out / accept must hold B*K values")
    if mode == POLICY_MLP:
        _need(w1.dim() == 2 and w1.shape[1] == 8, "w1 must be [H, 8]")
        H = w1.shape[0]
        _need(b1.numel() == H and w2.numel() == H, "b1 / w2 must hold H values")


def check_commit_shapes(draft, argmax, accept, k_blk, v_blk, k_pages, v_pages, page_table,
                        ctx_len, accept_len, emitted) -> None:
    """draft [B,K]; argmax B*(K+1); accept B*K; block K/V [L,B,K+1,Hkv,D];
    pools [L or 1,num_pages,Hkv,P,D]; page_table [B,max_pages]; ctx_len,
    accept_len [B]; emitted B*(K+1)."""
    _need(draft.dim() == 2, "draft must be [B, K]")
    B, K = draft.shape
    _need(argmax.numel() == B * (K + 1), "argmax must hold K+1 ids per sequence")
    _need(accept.numel() == B * K, "accept must hold B*K values")
    _need(k_blk.dim() == 5 and tuple(v_blk.shape) == tuple(k_blk.shape),
          "k_blk / v_blk must both be [L, B, K+1, Hkv, D]")
    L = k_blk.shape[0]
    _need(k_pages.dim() == 5 and tuple(v_pages.shape) == tuple(k_pages.shape),
          "k_pages / v_pages must both be [L, num_pages, Hkv, P, D]")
    _need(k_pages.shape[0] in (L, 1), "pools must hold every layer, or one shared by all")
    _need(tuple(k_blk.shape[1:]) == (B, K + 1, k_pages.shape[2], k_pages.shape[4]),
          "k_blk must be [L, B, K+1, Hkv, D] with the pools' Hkv and D")
    _need(page_table.dim() == 2 and page_table.shape[0] == B, "page_table must be [B, max_pages]")
    _need(ctx_len.numel() == B and accept_len.numel() == B, "ctx_len / accept_len must be [B]")
    _need(emitted.numel() == B * (K + 1), "emitted must hold K+1 tokens per sequence")


def attn_dims(q: torch.Tensor, k_pages: torch.Tensor, page_table: torch.Tensor,
              softmax_scale: float = 0.0, flags: int = 0) -> AttnDims:
    """Geometry of one verify-attention call from q [B,R,Hq,D], the layer's
    pool [num_pages,Hkv,P,D] and the page table [B,max_pages]."""
    B, R, Hq, D = q.shape
    num_pages, Hkv, P, D2 = k_pages.shape[-4:]
    assert D2 == D
    return AttnDims(B, R, Hq, Hkv, D, P, page_table.shape[1], num_pages, softmax_scale, flags)


def num_sms() -> int:
    return load_library().cospec_num_sms()


ATTN_MMA_SYNC, ATTN_TCGEN05 = 0, 1
ATTN_KERNEL_NAMES = {ATTN_MMA_SYNC: "mma.sync", ATTN_TCGEN05: "tcgen05"}


def verify_attn_plan(q, k_pages, page_table, max_ctx: int, kv_stable: bool = False):
    """(kernel, splits) cospec_verify_attn would use for these tensors (and
    the stable-cache flag, which the plan of small batches depends on)."""
    dims = attn_dims(q, k_pages, page_table, flags=ATTN_KV_STABLE if kv_stable else 0)
    kernel, splits = ctypes.c_int(), ctypes.c_int()
    _check(load_library().cospec_verify_attn_plan(ctypes.byref(dims), int(max_ctx),
                                                  ctypes.byref(kernel), ctypes.byref(splits)))
    return kernel.value, splits.value


ATTN_ONE_TILE, ATTN_TWO_TILES, ATTN_CTA_PAIR = 1, 2, 3    # tcgen05 variants (0: mma.sync)


def verify_attn_variant(q, k_pages, page_table, max_ctx: int, kv_stable: bool = False) -> int:
    """Which of the attention kernels cospec_verify_attn would use for these tensors."""
    dims = attn_dims(q, k_pages, page_table, flags=ATTN_KV_STABLE if kv_stable else 0)
    variant = ctypes.c_int()
    _check(load_library().cospec_verify_attn_variant(ctypes.byref(dims), int(max_ctx), ctypes.byref(variant)))
    return variant.value


def verify_attn_plan_model(dims: AttnDims, max_ctx: int, num_sms: int, resident):
    """(kernel, splits) of cospec_verify_attn_plan_model: the plan for a
    device of ``num_sms`` SMs whose residency is ``resident(kernel, rows,
    block_rows, splits)`` -> clusters resident at once.  Host only."""
    cb = RESIDENT_FN(lambda k, r, kb, s, _user: int(resident(k, r, kb, s)))
    kernel, splits = ctypes.c_int(), ctypes.c_int()
    _check(load_library().cospec_verify_attn_plan_model(ctypes.byref(dims), int(max_ctx),
                                                        int(num_sms), cb, None,
                                                        ctypes.byref(kernel), ctypes.byref(splits)))
    return kernel.value, splits.value


def verify_attn(q, k_blk, v_blk, k_pages, v_pages, page_table, ctx_len, out, max_ctx,
                softmax_scale: float = 0.0, stream=None, kv_stable: bool = False,
                block_full: bool = False) -> torch.Tensor:
    """Verify attention of one layer (Sec. 3.1, Eq. 2).  See include/cospec.h.
    ``kv_stable``: the kernel queued just before writes neither ctx_len, the
    page table nor the cached pages (COSPEC_ATTN_KV_STABLE);
    those before it are waited for by the last call without the flag.  ``block_full``:
    block rows see the whole block (the arbitrator's draft/target region,
    Sec. 3.3; COSPEC_ATTN_BLOCK_FULL)."""
    for t, n in ((q, "q"), (k_blk, "k_blk"), (v_blk, "v_blk"), (k_pages, "k_pages"),
                 (v_pages, "v_pages"), (out, "out")):
        _req(t, torch.bfloat16, n)
    _req(page_table, torch.int32, "page_table", 2)
    _req(ctx_len, torch.int32, "ctx_len", 1)
    check_attn_shapes(q, k_blk, v_blk, k_pages, v_pages, page_table, ctx_len, out)
    _same_device(q, k_blk, v_blk, k_pages, v_pages, page_table, ctx_len, out)
    dims = attn_dims(q, k_pages, page_table, softmax_scale,
                     (ATTN_KV_STABLE if kv_stable else 0) | (ATTN_BLOCK_FULL if block_full else 0))
    _check(load_library().cospec_verify_attn(
        ctypes.byref(dims), int(max_ctx), _ptr(q), _ptr(k_blk), _ptr(v_blk), _ptr(k_pages),
        _ptr(v_pages), _ptr(page_table), _ptr(ctx_len), _ptr(out), _stream(stream)))
    return out


def lmhead_workspace_bytes(M: int, d: int, V: int) -> int:
    return load_library().cospec_lmhead_workspace(M, d, V)


def new_lmhead_workspace(M: int, d: int, V: int, device="cuda") -> torch.Tensor:
    return torch.empty(lmhead_workspace_bytes(M, d, V), dtype=torch.uint8, device=device)


def lmhead_argmax_features(hidden, w, draft_for_row, argmax, stats, ws, stream=None):
    """LM head + argmax + statistics (Eq. 2, Eq. 23).  stats [M,5] = (max,
    second, lse, entropy, draft logit)."""
    _req(hidden, torch.bfloat16, "hidden", 2)
    _req(w, torch.bfloat16, "w", 2)
    _req(draft_for_row, torch.int32, "draft_for_row", 1)
    _req(argmax, torch.int32, "argmax", 1)
    _req(stats, torch.float32, "stats", 2)
    _req(ws, torch.uint8, "ws", 1)
    M, d = hidden.shape
    V = w.shape[0]
    if w.shape[1] != d or draft_for_row.numel() != M or argmax.numel() != M or tuple(stats.shape) != (M, 5):
        raise ValueError("inconsistent LM-head shapes")
    _same_device(hidden, w, draft_for_row, argmax, stats, ws)
    _check(load_library().cospec_lmhead_argmax_features(
        M, d, V, _ptr(hidden), _ptr(w), _ptr(draft_for_row), _ptr(argmax), _ptr(stats), _ptr(ws),
        ws.numel(), _stream(stream)))
    return argmax, stats


def lmhead_sample_features(hidden, w, draft_for_row, temperature: float, seed, sample, stats, ws,
                           stream=None):
    """Stochastic-decoding LM head (Sec. 3.1, App. C.3): sample [M] is a
    Gumbel-max draw from softmax(x / T) with Philox4x32-10 noise keyed by the
    int64 device scalar ``seed`` (read when the kernel runs); stats as in
    lmhead_argmax_features."""
    _req(hidden, torch.bfloat16, "hidden", 2)
    _req(w, torch.bfloat16, "w", 2)
    _req(draft_for_row, torch.int32, "draft_for_row", 1)
    _req(sample, torch.int32, "sample", 1)
    _req(stats, torch.float32, "stats", 2)
    _req(ws, torch.uint8, "ws", 1)
    _req(seed, torch.int64, "seed")
    if seed.numel() != 1:
        raise ValueError("seed must hold one value")
    M, d = hidden.shape
    V = w.shape[0]
    if w.shape[1] != d or draft_for_row.numel() != M or sample.numel() != M or tuple(stats.shape) != (M, 5):
        raise ValueError("inconsistent LM-head shapes")
    _same_device(hidden, w, draft_for_row, seed, sample, stats, ws)
    _check(load_library().cospec_lmhead_sample_features(
        M, d, V, _ptr(hidden), _ptr(w), _ptr(draft_for_row), float(temperature), _ptr(seed),
        _ptr(sample), _ptr(stats), _ptr(ws), ws.numel(), _stream(stream)))
    return sample, stats


def lmhead_logits_features(hidden, w, draft_for_row, temperature: float, argmax, stats, logits,
                           ws, stream=None):
    """LM head for speculative sampling at temperature T: logits [M, V] fp32
    receives x / T, stats [M, 5] the statistics of x / T, argmax [M] the
    argmax."""
    _req(hidden, torch.bfloat16, "hidden", 2)
    _req(w, torch.bfloat16, "w", 2)
    _req(draft_for_row, torch.int32, "draft_for_row", 1)
    _req(argmax, torch.int32, "argmax", 1)
    _req(stats, torch.float32, "stats", 2)
    _req(logits, torch.float32, "logits", 2)
    _req(ws, torch.uint8, "ws", 1)
    M, d = hidden.shape
    V = w.shape[0]
    if (w.shape[1] != d or draft_for_row.numel() != M or argmax.numel() != M
            or tuple(stats.shape) != (M, 5) or tuple(logits.shape) != (M, V)):
        raise ValueError("inconsistent LM-head shapes")
    _same_device(hidden, w, draft_for_row, argmax, stats, logits, ws)
    _check(load_library().cospec_lmhead_logits_features(
        M, d, V, _ptr(hidden), _ptr(w), _ptr(draft_for_row), float(temperature), _ptr(argmax),
        _ptr(stats), _ptr(logits), _ptr(ws), ws.numel(), _stream(stream)))
    return argmax, stats, logits


def new_sps_workspace(B: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(1, int(load_library().cospec_sps_workspace(B))), dtype=torch.uint8,
                       device=device)


def sps_accept(draft, stats, logits, q, seed, target, accept, ratio, ws, stream=None):
    """Speculative-sampling acceptance (the exact-match baseline at a
    temperature): draft [B, K], stats [B*(K+1), 5] and logits [B*(K+1), V]
    of x / T, q [B, K, V] the draft's distributions, seed an int64 device
    scalar; fills target [B, K+1], accept [B, K], ratio [B, K]."""
    _req(draft, torch.int32, "draft", 2)
    _req(stats, torch.float32, "stats", 2)
    _req(logits, torch.float32, "logits", 2)
    _req(q, torch.float32, "q", 3)
    _req(seed, torch.int64, "seed")
    _req(target, torch.int32, "target")
    _req(accept, torch.uint8, "accept")
    _req(ratio, torch.float32, "ratio")
    _req(ws, torch.uint8, "ws", 1)
    B, K = draft.shape
    R = K + 1
    V = logits.shape[1]
    if (seed.numel() != 1 or tuple(stats.shape) != (B * R, 5) or logits.shape[0] != B * R
            or tuple(q.shape) != (B, K, V) or target.numel() != B * R or accept.numel() != B * K
            or ratio.numel() != B * K):
        raise ValueError("inconsistent speculative-sampling shapes")
    _same_device(draft, stats, logits, q, seed, target, accept, ratio, ws)
    _check(load_library().cospec_sps_accept(
        B, K, V, _ptr(draft), _ptr(stats), _ptr(logits), _ptr(q), _ptr(seed), _ptr(target),
        _ptr(accept), _ptr(ratio), _ptr(ws), ws.numel(), _stream(stream)))
    return target, accept, ratio


def lmhead_argmax_features_noalloc(hidden, w, draft_for_row, argmax, stats, stream=None):
    """The LM-head call without a workspace, for callers that cannot allocate
    device memory: partials go to a fixed scratch array inside the library
    (at most 512 rows per call; calls must not overlap on the GPU)."""
    _req(hidden, torch.bfloat16, "hidden", 2)
    _req(w, torch.bfloat16, "w", 2)
    _req(draft_for_row, torch.int32, "draft_for_row", 1)
    _req(argmax, torch.int32, "argmax", 1)
    _req(stats, torch.float32, "stats", 2)
    M, d = hidden.shape
    V = w.shape[0]
    if w.shape[1] != d or draft_for_row.numel() != M or argmax.numel() != M or tuple(stats.shape) != (M, 5):
        raise ValueError("inconsistent LM-head shapes")
    _same_device(hidden, w, draft_for_row, argmax, stats)
    _check(load_library().cospec_lmhead_argmax_features_noalloc(
        M, d, V, _ptr(hidden), _ptr(w), _ptr(draft_for_row), _ptr(argmax), _ptr(stats),
        _stream(stream)))
    return argmax, stats


def rl_advantages(group_off, correct, round_off, match, accept, ell, params: RLParams = None,
                  ratio=None, p_new=None, p_ref=None, stream=None) -> dict:
    """RL-stage rewards and advantages (Sec. 3.4).  Inputs are CUDA tensors:
    group_off int32 [G+1], correct uint8 [M], round_off int32 [M+1],
    match / accept uint8 [R, K], ell float32 [R, K]; optional ratio / p_new /
    p_ref float32 [R, K] for the objective.  Returns the output tensors."""
    params = params if params is not None else RLParams()
    _req(group_off, torch.int32, "group_off", 1)
    _req(round_off, torch.int32, "round_off", 1)
    _req(correct, torch.uint8, "correct", 1)
    _req(match, torch.uint8, "match", 2)
    _req(accept, torch.uint8, "accept", 2)
    _req(ell, torch.float32, "ell", 2)
    G, M = group_off.numel() - 1, correct.numel()
    R, K = match.shape
    if round_off.numel() != M + 1 or tuple(accept.shape) != (R, K) or tuple(ell.shape) != (R, K):
        raise ValueError("inconsistent RL shapes")
    obj = [t for t in (ratio, p_new, p_ref) if t is not None]
    for t, n in zip(obj, ("ratio", "p_new", "p_ref")):
        _req(t, torch.float32, n, 2)
        if tuple(t.shape) != (R, K):
            raise ValueError(f"{n} must be [R, K]")
    _same_device(group_off, correct, round_off, match, accept, ell, *obj)
    dev = match.device
    out = dict(g=torch.empty((R, K), dtype=torch.float32, device=dev),
               eff=torch.empty((R, K), dtype=torch.uint8, device=dev),
               rho=torch.empty(R, dtype=torch.float32, device=dev),
               J=torch.empty(M, dtype=torch.float32, device=dev),
               Jbar=torch.empty(M, dtype=torch.float32, device=dev),
               adv=torch.empty(M, dtype=torch.float32, device=dev),
               adv_dec=torch.empty((R, K), dtype=torch.float32, device=dev))
    loss = torch.empty(4, dtype=torch.float32, device=dev) if obj else None
    lib = load_library()
    ws = torch.empty(lib.cospec_rl_workspace(G, M), dtype=torch.uint8, device=dev)
    _check(lib.cospec_rl_advantages(
        G, M, R, K, _ptr(group_off), _ptr(correct), _ptr(round_off), _ptr(match), _ptr(accept),
        _ptr(ell), ctypes.byref(params), _ptr(ratio), _ptr(p_new), _ptr(p_ref), _ptr(out["g"]),
        _ptr(out["eff"]), _ptr(out["rho"]), _ptr(out["J"]), _ptr(out["Jbar"]), _ptr(out["adv"]),
        _ptr(out["adv_dec"]), _ptr(loss), _ptr(ws), ws.numel(), _stream(stream)))
    if loss is not None:
        out["loss"] = loss
    return out


def arbitrate(draft, argmax, stats, w1, b1, w2, b2: float, lam: float, mode: int, p_out, accept,
              stream=None):
    """Mismatch arbitration (Eq. 3, Eq. 13-14, Eq. 17).  draft [B,K],
    argmax [B,K+1], stats [B,K+1,5]; p_out [B,K] float32, accept [B,K] uint8."""
    _req(draft, torch.int32, "draft", 2)
    _req(argmax, torch.int32, "argmax")
    _req(stats, torch.float32, "stats")
    _req(p_out, torch.float32, "p_out")
    _req(accept, torch.uint8, "accept")
    B, K = draft.shape
    H = 0
    if mode == POLICY_MLP:
        for t, n in ((w1, "w1"), (b1, "b1"), (w2, "w2")):
            _req(t, torch.float32, n)
        H = w1.shape[0]
    check_arbitrate_shapes(draft, argmax, stats, w1, b1, w2, mode, p_out, accept)
    _same_device(draft, argmax, stats, p_out, accept,
                 *((w1, b1, w2) if mode == POLICY_MLP else ()))
    _check(load_library().cospec_arbitrate(
        B, K, _ptr(draft), _ptr(argmax), _ptr(stats), H, _ptr(w1) if mode == 0 else None,
        _ptr(b1) if mode == 0 else None, _ptr(w2) if mode == 0 else None, float(b2), float(lam),
        int(mode), _ptr(p_out), _ptr(accept), _stream(stream)))
    return p_out, accept


def accept_commit_launches(dims: AttnDims, num_layers: int) -> int:
    """Kernels accept_commit launches for a block of these dimensions."""
    n = load_library().cospec_accept_commit_launches(ctypes.byref(dims), int(num_layers))
    if n < 0:
        _check(n)
    return n


def accept_commit(draft, argmax, accept, k_blk, v_blk, k_pages, v_pages, page_table, ctx_len,
                  accept_len, emitted, stream=None):
    """Accepted length / emitted tokens (Eq. 15) and KV commit.
    k_blk, v_blk [L,B,R,Hkv,D]; pools [L,num_pages,Hkv,P,D] (any layer stride)."""
    _req(draft, torch.int32, "draft", 2)
    _req(argmax, torch.int32, "argmax")
    _req(accept, torch.uint8, "accept")
    for t, n in ((k_blk, "k_blk"), (v_blk, "v_blk")):
        _req(t, torch.bfloat16, n, 5)
    for t, n in ((k_pages, "k_pages"), (v_pages, "v_pages")):
        if t.dtype != torch.bfloat16 or not t.is_cuda or t.dim() != 5 or not t[0].is_contiguous():
            raise ValueError(f"{n}: expected bf16 CUDA [L,num_pages,Hkv,P,D] with contiguous layers")
    _req(page_table, torch.int32, "page_table", 2)
    _req(ctx_len, torch.int32, "ctx_len", 1)
    _req(accept_len, torch.int32, "accept_len", 1)
    _req(emitted, torch.int32, "emitted")
    check_commit_shapes(draft, argmax, accept, k_blk, v_blk, k_pages, v_pages, page_table,
                        ctx_len, accept_len, emitted)
    _same_device(draft, argmax, accept, k_blk, v_blk, k_pages, v_pages, page_table, ctx_len,
                 accept_len, emitted)
    B, K = draft.shape
    L = k_blk.shape[0]
    if k_pages.stride(0) != v_pages.stride(0):
        raise ValueError("k_pages / v_pages must hold their layers with the same stride")
    # A single pool standing for every layer receives layer 0's rows only (the
    # library rejects several layers committed into one pool: their writes
    # would race for the same cells).
    if k_pages.shape[0] == 1 and L > 1:
        L = 1
        k_blk, v_blk = k_blk[:1], v_blk[:1]
    layer_stride = int(k_pages.stride(0))
    dims = AttnDims(B, K + 1, 0, k_pages.shape[2], k_pages.shape[4], k_pages.shape[3],
                    page_table.shape[1], k_pages.shape[1], 0.0, 0)
    dims.num_q_heads = dims.num_kv_heads
    _check(load_library().cospec_accept_commit(
        B, K, L, ctypes.byref(dims), _ptr(draft), _ptr(argmax), _ptr(accept), _ptr(k_blk),
        _ptr(v_blk), _ptr(k_pages), _ptr(v_pages), layer_stride, _ptr(page_table),
        _ptr(ctx_len), _ptr(accept_len), _ptr(emitted), _stream(stream)))
    return accept_len, emitted


# ---------------------------------------------------------------- 8-bit KV cache
F8 = torch.float8_e4m3fn


class Kv8Pool:
    """The arrays of an 8-bit paged cache (cospec_kv8_pool), checked once: k e4m3
    [L, pages, Hkv, 16, D], v e4m3 [L, pages, Hkv, D, 16], scale float32
    [L, pages, Hkv, 2] and, for the page selection, summary int8 [L, pages, Hkv, D] with
    summary_scale float32 [L, pages, Hkv]."""

    def __init__(self, k, v, scale, summary=None, summary_scale=None):
        _req(k, F8, "k", 5)
        _req(v, F8, "v", 5)
        _req(scale, torch.float32, "scale", 4)
        L, N, H, P, D = k.shape
        _need(P == 16 and tuple(v.shape) == (L, N, H, D, P), "k must be [L, pages, Hkv, 16, D] and v [L, pages, Hkv, D, 16]")
        _need(tuple(scale.shape) == (L, N, H, 2), "scale must be [L, pages, Hkv, 2]")
        _need((summary is None) == (summary_scale is None), "summary and summary_scale go together")
        if summary is not None:
            _req(summary, torch.int8, "summary", 4)
            _req(summary_scale, torch.float32, "summary_scale", 3)
            _need(tuple(summary.shape) == (L, N, H, D), "summary must be [L, pages, Hkv, D]")
            _need(tuple(summary_scale.shape) == (L, N, H), "summary_scale must be [L, pages, Hkv]")
        self.k, self.v, self.scale, self.summary, self.summary_scale = k, v, scale, summary, summary_scale
        self.layers, self.num_pages, self.kv_heads, self.head_dim = L, N, H, D
        self.device, self.index = k.device, k.get_device()
        for t in (v, scale, summary, summary_scale):
            _need(t is None or t.device == k.device, "a pool's arrays must be on one device")
        self.c = Kv8PoolC(L, N, H, D, *(0 if t is None else t.data_ptr() for t in (k, v, scale, summary, summary_scale)))
        self.ref = ctypes.byref(self.c)


def new_kv8_pool(layers: int, num_pages: int, kv_heads: int, head_dim: int, summaries: bool = True,
                 device="cuda") -> Kv8Pool:
    """An empty 8-bit cache."""
    z = lambda shape, dt: torch.zeros((layers, num_pages, kv_heads) + shape, dtype=dt, device=device)  # noqa: E731
    return Kv8Pool(z((16, head_dim), torch.uint8).view(F8), z((head_dim, 16), torch.uint8).view(F8),
                   z((2,), torch.float32), *((z((head_dim,), torch.int8), z((), torch.float32)) if summaries else ()))


class Rope:
    """Tables of the position rotation (cospec_rope): cos, sin float32 [positions, rot_dim / 2]."""

    def __init__(self, cos, sin, interleaved: bool = False):
        _req(cos, torch.float32, "cos", 2)
        _req(sin, torch.float32, "sin", 2)
        _need(tuple(sin.shape) == tuple(cos.shape) and cos.shape[1] % 4 == 0 and cos.numel() > 0,
              "cos / sin must both be [positions, rot_dim / 2], rot_dim a multiple of 8")
        _need(sin.device == cos.device, "cos / sin must be on one device")
        self.cos, self.sin, self.device = cos, sin, cos.device
        self.c = RopeC(cos.data_ptr(), sin.data_ptr(), cos.shape[0], 2 * cos.shape[1], int(bool(interleaved)))
        self.ref = ctypes.byref(self.c)


# A call's Python side is most of a small call's time: geometry structures are kept by their
# values, and each check is one comparison on the good path.
_BF16, _F32, _I32, _I8 = torch.bfloat16, torch.float32, torch.int32, torch.int8
_KEPT = 4096                      # structures kept of a kind
_strides_kept: dict = {}
_dims_kept: dict = {}


def _keep(kept: dict, key, make):
    if len(kept) >= _KEPT:
        kept.clear()
    ref = kept[key] = ctypes.byref(make())
    return ref


def _rows_ref(t: torch.Tensor, name: str, shape):
    """Checks bf16 rows [(layers,) batch, rows, heads, head_dim] whose heads and dimensions are
    dense, and returns a reference to their strides (cospec_kv8_strides)."""
    if t.dtype is not _BF16:
        raise TypeError(f"{name}: expected {_BF16}, got {t.dtype}")
    n = t.shape
    if n != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(n)}")
    key = (n, t.stride())
    ref = _strides_kept.get(key)
    return ref if ref is not None else _new_strides(t, name, key)


def _new_strides(t, name, key):
    n, st = key
    if t.numel() and ((st[-1] != 1 and n[-1] > 1) or (st[-2] != n[-1] and n[-2] > 1)):
        raise ValueError(f"{name}: heads and dimensions must be dense")
    lead = [0 if size == 1 else s for size, s in zip(n[:-2], st[:-2])]     # (one element has no stride)
    return _keep(_strides_kept, key, lambda: Strides(*([0] * (3 - len(lead)) + lead)))


def _dense(t: torch.Tensor, name: str, dtype, shape) -> None:
    if t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")


def _on_device(dev: int, *tensors) -> None:
    """Names the tensor that is not on the current device (the calls compare the indices themselves)."""
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"a tensor is on {t.device}, but the current device is cuda:{dev}" if t.is_cuda
                             else "every tensor must be a CUDA tensor")


_current = torch._C._cuda_getDevice


def _stream_ptr(stream, dev: int) -> int:
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _at(t):
    return None if t is None else t.data_ptr()


def kv8_append(pool: Kv8Pool, k, v, page_table, start, rows=None, rope: Optional[Rope] = None, layer: Optional[int] = None,
               q=None, q_out=None, k_out=None, stream=None) -> None:
    """Append rows of keys (rotated by ``rope``) and values to an 8-bit cache: k, v bf16
    [L, B, R, Hkv, D] for every layer of the pool or, with ``layer``, [B, R, Hkv, D] for that one; they may
    be parts of a fused projection's output (any strides of the leading dimensions).  Row j of sequence
    b enters position start[b] + j for j < rows[b] (all rows without ``rows``).  k_out / q_out receive
    all rows of k / q rotated, in bf16.  See include/cospec.h."""
    shape = k.shape
    _need(len(shape) == (5 if layer is None else 4), "k must be [L, B, R, Hkv, D], or [B, R, Hkv, D] with layer")
    first, L = (0, shape[0]) if layer is None else (int(layer), 1)
    _need(0 <= first < pool.layers and (layer is not None or L == pool.layers), "layer outside the pool")
    _need(shape[-2] == pool.kv_heads and shape[-1] == pool.head_dim, "k must have the pool's heads and head_dim")
    B = shape[-4]
    vs = _rows_ref(v, "v", shape)
    _need(page_table.dim() == 2, "page_table must be [B, max_pages]")
    _dense(page_table, "page_table", _I32, (B, page_table.shape[1]))
    if rows is not None:
        _dense(rows, "rows", _I32, (B,))
    _need(pool.device == k.device, "the pool is on another device")
    _launch_append(pool.ref, first, L, shape, rope, q, k, v, vs, page_table, start, rows, q_out, k_out, stream)


def kv8_rotate(q, k, rope: Rope, start, q_out, k_out, stream=None) -> None:
    """The rotation of kv8_append by itself: q [B, R, Hq, D] and k [B, R, Hkv, D] (or with a leading
    layer dimension) turned to positions start[b] + j, in bf16, nothing appended."""
    shape = k.shape
    _need(len(shape) in (4, 5), "k must be [B, R, Hkv, D] or [L, B, R, Hkv, D]")
    pool = _dims_kept.get(shape[-2:]) or _keep(_dims_kept, shape[-2:], lambda: Kv8PoolC(1, 1, shape[-2], shape[-1], 0, 0, 0, 0, 0))
    _launch_append(pool, 0, shape[0] if len(shape) == 5 else 1, shape, rope, q, k, None, None, None, start, None, q_out, k_out, stream)


def _launch_append(pool_ref, first, L, shape, rope, q, k, v, vs, page_table, start, rows, q_out, k_out, stream):
    ks = _rows_ref(k, "k", shape)
    B, R = shape[-4], shape[-3]
    _dense(start, "start", _I32, (B,))
    _need((q is None) == (q_out is None), "q and q_out go together")
    Hq, qs = 0, None
    if q is not None:
        _need(q.shape[:-2] == shape[:-2] and q.shape[-1] == shape[-1], "q must have k's batch, rows and head_dim")
        Hq = q.shape[-2]
        qs = _rows_ref(q, "q", q.shape)
        _dense(q_out, "q_out", _BF16, q.shape)
    if k_out is not None:
        _dense(k_out, "k_out", _BF16, shape)
    dev = _current()
    for t in (k, v, q, q_out, k_out, page_table, start, rows, None if rope is None else rope.cos):
        if t is not None and t.get_device() != dev:
            _on_device(dev, t)
    _check((_lib or load_library()).cospec_kv8_append(
        pool_ref, first, L, B, R, Hq, None if rope is None else rope.ref, _at(q), qs, k.data_ptr(), ks, _at(v), vs, _at(page_table),
        0 if page_table is None else page_table.shape[1], start.data_ptr(), _at(rows), _at(q_out), _at(k_out), _stream_ptr(stream, dev)))


def _kv8_dims(q, pool: Kv8Pool, layer: int, page_table, ctx_len, softmax_scale=0.0, flags=0):
    """The call's checked geometry: q's shape and a reference to cospec_attn_dims."""
    shape, table = q.shape, page_table.shape
    if len(shape) != 4 or shape[3] != pool.head_dim:
        raise ValueError("q must be [B, R, Hq, D] with the pool's D")
    if not 0 <= layer < pool.layers:
        raise ValueError("layer outside the pool")
    if len(table) != 2:
        raise ValueError("page_table must be [B, max_pages]")
    B = shape[0]
    _dense(page_table, "page_table", _I32, (B, table[1]))
    _dense(ctx_len, "ctx_len", _I32, (B,))
    key = (shape, table[1], pool.kv_heads, pool.num_pages, softmax_scale, flags)
    return shape, _dims_kept.get(key) or _keep(_dims_kept, key, lambda: AttnDims(
        B, shape[1], shape[2], pool.kv_heads, shape[3], 16, table[1], pool.num_pages, softmax_scale, flags))


def kv8_select(q, pool: Kv8Pool, layer: int, page_table, ctx_len, sel, sink: int = 1, recent: int = 2, stream=None) -> torch.Tensor:
    """The pages each block row reads: sel int32 [B, R, Hkv, pages] receives for row q[b, j] and each
    KV head the first ``sink`` and last ``recent`` pages of its context and those of the largest
    scores by the pages' summaries, ascending, -1 after the last."""
    shape, dims = _kv8_dims(q, pool, layer, page_table, ctx_len)
    qs = _rows_ref(q, "q", shape)
    _need(pool.summary is not None, "the pool has no summaries")
    pages = sel.shape[-1]
    _dense(sel, "sel", _I32, (shape[0], shape[1], pool.kv_heads, pages))
    dev = _current()
    if not dev == q.get_device() == page_table.get_device() == ctx_len.get_device() == sel.get_device() == pool.index:
        _on_device(dev, q, page_table, ctx_len, sel, pool.k)
    _check((_lib or load_library()).cospec_kv8_select(dims, pool.ref, layer, q.data_ptr(), qs, page_table.data_ptr(), ctx_len.data_ptr(),
                                                      pages, int(sink), int(recent), sel.data_ptr(), _stream_ptr(stream, dev)))
    return sel


def kv8_attn(q, k_blk, v_blk, pool: Kv8Pool, layer: int, page_table, ctx_len, out, max_ctx: int, softmax_scale: float = 0.0,
             sel=None, kv_stable: bool = False, block_full: bool = False, stream=None) -> torch.Tensor:
    """Verify attention over layer ``layer`` of an 8-bit cache and the block's own bf16 rows; with
    ``sel`` (kv8_select) over each row's chosen pages only.  q, k_blk and v_blk [B, R, H, D] may be parts of a
    fused projection's output.  Flags as verify_attn; see include/cospec.h."""
    shape, dims = _kv8_dims(q, pool, layer, page_table, ctx_len, softmax_scale,
                            (ATTN_KV_STABLE if kv_stable else 0) | (ATTN_BLOCK_FULL if block_full else 0))
    block = (shape[0], shape[1], pool.kv_heads, pool.head_dim)
    qs, ks, vs = _rows_ref(q, "q", shape), _rows_ref(k_blk, "k_blk", block), _rows_ref(v_blk, "v_blk", block)
    _dense(out, "out", _BF16, shape)
    pages = 0
    if sel is not None:
        pages = sel.shape[-1]
        _dense(sel, "sel", _I32, (shape[0], shape[1], pool.kv_heads, pages))
    dev = _current()
    if not (dev == q.get_device() == k_blk.get_device() == v_blk.get_device() == page_table.get_device() == ctx_len.get_device()
            == out.get_device() == pool.index) or (sel is not None and sel.get_device() != dev):
        _on_device(dev, q, k_blk, v_blk, page_table, ctx_len, sel, out, pool.k)
    _check((_lib or load_library()).cospec_kv8_attn(
        dims, int(max_ctx), pool.ref, layer, q.data_ptr(), qs, k_blk.data_ptr(), ks, v_blk.data_ptr(), vs, page_table.data_ptr(),
        ctx_len.data_ptr(), _at(sel), pages, out.data_ptr(), _stream_ptr(stream, dev)))
    return out


def get_device_error(stream=None) -> int:
    """Read and clear the device error word (synchronises the stream)."""
    flags = ctypes.c_int(0)
    st = load_library().cospec_get_device_error(ctypes.byref(flags), _stream(stream))
    if st not in (0, -5):
        _check(st)
    return flags.value
