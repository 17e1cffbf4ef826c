"""Python binding of libsdverify.so (the C ABI in include/sd_verify.h).

Argument marshalling only: every step of the verify pass runs in the HIP
kernels of the library.  torch tensors are accepted where the C ABI takes a
device pointer; torch supplies device memory and streams, nothing else.  If
the library has not been built, loading raises -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsdverify.so")

SD_OK, SD_EINVAL, SD_ENOMEM, SD_EHIP, SD_ESTATE, SD_EDEVICE, SD_ENOTIMPL, SD_ENODEV, SD_ELIMIT = (
    0, -1, -2, -3, -4, -5, -6, -7, -8)
SD_NOALLOC_MAX_USERS, SD_NOALLOC_MAX_SLOTS, SD_NOALLOC_MAX_VOCAB = 64, 1024, 1 << 20
SD_F32, SD_BF16 = 0, 1
SD_GREEDY, SD_STOCHASTIC, SD_FORCE = 0, 1, 2
SD_LOGITS_AS_NEEDED, SD_LOGITS_ALL, SD_LOGITS_UNFUSED = 0, 1, 2
MODES = {"greedy": SD_GREEDY, "stochastic": SD_STOCHASTIC, "force": SD_FORCE}

EXPORTS = ("sd_verify_query_sizes", "sd_verify_init", "sd_verify_destroy", "sd_user_reset",
           "sd_user_release", "sd_user_state", "sd_kv_write", "sd_kv_read", "sd_verify_batch",
           "sd_verify_batch_graph", "sd_verify_batch_sparse", "sd_draft_batch", "sd_accept", "sd_sample_logits",
           "sd_sample_logits_noalloc", "sd_debug_logits", "sd_debug_wait_limit", "sd_profile_begin", "sd_profile_end",
           "sd_filter_query_size", "sd_sample_filtered", "sd_filter_logits", "sd_lora_query_size",
           "sd_lora_apply", "sd_tree_query_size", "sd_tree_attention", "sd_kv_copy_pages", "sd_kv_compact",
           "sd_adjust_logits", "sd_verify_batch_tree", "sd_accept_tree", "sd_user_fork", "sd_user_pages",
           "sd_batch_rules", "sd_user_sampling", "sd_adapters_set", "sd_user_adapter", "sd_calib_hbm", "sd_calib_mfma", "sd_status_str")
SD_FILTER_MAX_ROWS, SD_FILTER_MAX_VOCAB = 65535, 1 << 20
SD_LORA_MAX_RANK, SD_LORA_MAX_SEGS = 128, 4
SD_TREE_MAX_SLOTS, SD_TREE_MAX_USERS, SD_KV_COMPACT_MAX = 256, 16384, 256
SD_K_QKV, SD_K_ATTN, SD_K_O, SD_K_GATEUP, SD_K_DOWN, SD_K_LMHEAD, SD_K_SAMPLER, SD_K_SMALL = range(1, 9)


class sd_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab", "qk_norm",
        "dtype", "page_tokens", "n_pages", "max_users", "max_draft", "max_batch_users",
        "max_batch_tokens", "max_ctx", "max_pending")] + [("rope_base", ctypes.c_float),
                                                          ("rms_eps", ctypes.c_float),
                                                          ("logits_out", ctypes.c_int32)]


class sd_layer_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "wq", "wk", "wv", "wo", "wg", "wu", "wd", "norm1", "norm2", "qnorm", "knorm")]


class sd_weights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("lm_head", ctypes.c_void_p),
                ("norm_f", ctypes.c_void_p), ("layers", ctypes.POINTER(sd_layer_weights))]


class sd_filter(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("temperature", "top_k", "top_p", "min_p")]


class sd_lora(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_adapters", "rank", "d_in", "d_out", "n_seg")] + [
        ("seg_off", ctypes.c_int32 * (SD_LORA_MAX_SEGS + 1)), ("dtype", ctypes.c_int32),
        ("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("scale", ctypes.c_void_p)]


class sd_layer_adapters(ctypes.Structure):
    _fields_ = [(n, sd_lora) for n in ("qkv", "o", "down")]


class sd_kv_pool(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "n_pages", "n_kv_heads", "head_dim", "dtype")] + [
        ("base", ctypes.c_void_p)]


class sd_tree(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_users", "n_slots", "max_slots", "max_pages")] + [
        (n, ctypes.c_void_p) for n in ("slot_off", "prefix", "page_table", "parent")]


class sd_logit_rules(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_void_p), ("n_tokens", ctypes.c_int64)] + [(n, ctypes.c_void_p) for n in (
        "hist", "row_token", "row_parent", "repetition", "presence", "frequency", "bias_token", "bias_value")] + [
        ("n_bias", ctypes.c_int64), ("bias", ctypes.c_void_p), ("mask", ctypes.c_void_p), ("n_masks", ctypes.c_int32),
        ("mask_row", ctypes.c_void_p)]


class SdError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn}: {status_str(status)} ({status})")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64
        P = ctypes.POINTER
        L.sd_status_str.restype = ctypes.c_char_p
        L.sd_status_str.argtypes = [i32]
        L.sd_verify_query_sizes.argtypes = [P(sd_config), P(u64), P(u64), P(u64)]
        L.sd_verify_init.argtypes = [P(sd_config), P(sd_weights), vp, vp, vp, P(vp)]
        L.sd_verify_destroy.argtypes = [vp]
        L.sd_user_reset.argtypes = [vp, i32, i32, i32]
        L.sd_user_release.argtypes = [vp, i32]
        L.sd_user_state.argtypes = [vp, i32, P(i32), P(i32)]
        L.sd_kv_write.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp]
        L.sd_kv_read.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp]
        L.sd_verify_batch.argtypes = [vp, i32, i32, vp, vp, vp, vp, i32, u64, u64, vp, vp]
        L.sd_verify_batch_graph.argtypes = [vp, i32, i32, vp, vp, vp, vp, i32, u64, u64, vp, vp]
        L.sd_draft_batch.argtypes = [vp, i32, i32, vp, i32, u64, u64, vp, vp, vp]
        L.sd_verify_batch_sparse.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, i32, i32, u64, u64,
                                             vp, vp]
        L.sd_accept.argtypes = [vp, i32, vp, vp, i32]
        L.sd_sample_logits.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, i32, u64, u64, vp, vp]
        L.sd_sample_logits_noalloc.argtypes = [i32, vp, vp, i32, vp, vp, vp, i32, u64, u64, vp, vp, vp]
        L.sd_debug_logits.argtypes = [vp, i32, vp, vp]
        L.sd_debug_wait_limit.argtypes = [vp, i32]
        L.sd_profile_begin.argtypes = [vp, i32, i32]
        L.sd_profile_end.argtypes = [vp, P(ctypes.c_double), P(i32)]
        i64 = ctypes.c_int64
        L.sd_filter_query_size.argtypes = [i32, i32, P(u64)]
        L.sd_sample_filtered.argtypes = [i32, i32, vp, i32, i64, P(sd_filter), vp, vp, vp, vp, vp, u64, vp]
        L.sd_filter_logits.argtypes = [i32, i32, vp, i32, i64, P(sd_filter), vp, i64, vp, vp, u64, vp]
        L.sd_lora_query_size.argtypes = [P(sd_lora), i32, P(u64)]
        L.sd_lora_apply.argtypes = [P(sd_lora), i32, vp, vp, vp, i64, vp, i64, vp, i64, i32, vp, u64, vp]
        f32 = ctypes.c_float
        L.sd_tree_query_size.argtypes = [P(sd_kv_pool), P(sd_tree), i32, P(u64)]
        L.sd_tree_attention.argtypes = [P(sd_kv_pool), i32, P(sd_tree), i32, vp, vp, i64, vp, vp, i64, f32, vp, u64, vp]
        L.sd_kv_copy_pages.argtypes = [P(sd_kv_pool), i32, vp, vp, vp]
        L.sd_kv_compact.argtypes = [P(sd_kv_pool), i32, vp, vp, i32, vp, i32, vp, vp]
        L.sd_adjust_logits.argtypes = [i32, i32, vp, i32, i64, P(sd_logit_rules), vp, i64, vp]
        L.sd_verify_batch_tree.argtypes = [vp, i32, i32, vp, vp, vp, vp, i32, u64, u64, vp]
        L.sd_accept_tree.argtypes = [vp, i32, vp, vp, vp, i32]
        L.sd_user_fork.argtypes = [vp, i32, i32, i32, i32, vp]
        L.sd_user_pages.argtypes = [vp, i32, vp, i32, P(i32)]
        L.sd_batch_rules.argtypes = [vp, i32, i32, P(sd_logit_rules)]
        L.sd_user_sampling.argtypes = [vp, i32, f32, i32, f32, f32]
        L.sd_adapters_set.argtypes = [vp, i32, P(sd_layer_adapters)]
        L.sd_user_adapter.argtypes = [vp, i32, i32]
        L.sd_calib_hbm.argtypes = [vp, ctypes.c_size_t, i32, i32, P(ctypes.c_double), vp]
        L.sd_calib_mfma.argtypes = [vp, i32, P(ctypes.c_double), vp]
        for name in EXPORTS:
            if name != "sd_status_str":
                getattr(L, name).restype = i32
        _lib = L
    return _lib


def status_str(s: int) -> str:
    return lib().sd_status_str(int(s)).decode()


def _check(fn: str, s: int) -> int:
    if s != SD_OK:
        raise SdError(fn, s)
    return s


def _dev(t) -> Optional[int]:
    """Device pointer of a torch tensor (or an int / None)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_cuda and t.is_contiguous(), "device arguments must be contiguous GPU tensors"
    return t.data_ptr()


def _host_i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _stream(s) -> Optional[int]:
    if s is None:
        return None
    if isinstance(s, int):
        return s
    return s.cuda_stream


# ---------------------------------------------------------------------------
# thin wrappers with the C names (raise SdError on a nonzero status)
# ---------------------------------------------------------------------------

def sd_verify_query_sizes(cfg: sd_config):
    """Returns (kv_pool_bytes, workspace_bytes, weight_pack_bytes)."""
    kv, ws, wp = ctypes.c_uint64(), ctypes.c_uint64(), ctypes.c_uint64()
    _check("sd_verify_query_sizes", lib().sd_verify_query_sizes(
        ctypes.byref(cfg), ctypes.byref(kv), ctypes.byref(ws), ctypes.byref(wp)))
    return kv.value, ws.value, wp.value


class _Context:
    """What sd_adapters_set and others need to know of a context, and the adapters
    and batches' rules that the library reads in place."""

    def __init__(self, n_layers: int, device: int, vocab: int = 0, max_draft: int = 0):
        self.n_layers, self.device, self.adapters = n_layers, device, None
        self.vocab, self.max_draft, self.rules = vocab, max_draft, {}


_contexts: Dict[int, _Context] = {}


def sd_verify_init(cfg: sd_config, weights: sd_weights, kv_pool, workspace, weight_pack=None) -> int:
    import torch
    out = ctypes.c_void_p()
    _check("sd_verify_init", lib().sd_verify_init(ctypes.byref(cfg), ctypes.byref(weights),
                                                  _dev(kv_pool), _dev(workspace), _dev(weight_pack),
                                                  ctypes.byref(out)))
    _contexts[out.value] = _Context(cfg.n_layers, torch.cuda.current_device(), cfg.vocab, cfg.max_draft)
    return out.value


def sd_verify_destroy(ctx: int) -> None:
    _check("sd_verify_destroy", lib().sd_verify_destroy(ctx))
    _contexts.pop(ctx, None)


def sd_user_reset(ctx: int, user: int, prefix_len: int, root_token: int) -> None:
    _check("sd_user_reset", lib().sd_user_reset(ctx, user, prefix_len, root_token))


def sd_user_release(ctx: int, user: int) -> None:
    _check("sd_user_release", lib().sd_user_release(ctx, user))


def sd_user_state(ctx: int, user: int):
    p, r = ctypes.c_int32(), ctypes.c_int32()
    _check("sd_user_state", lib().sd_user_state(ctx, user, ctypes.byref(p), ctypes.byref(r)))
    return p.value, r.value


def sd_kv_write(ctx: int, user: int, layer: int, pos0: int, n: int, k, v, stream=None) -> None:
    _check("sd_kv_write", lib().sd_kv_write(ctx, user, layer, pos0, n, _dev(k), _dev(v), _stream(stream)))


def sd_kv_read(ctx: int, user: int, layer: int, pos0: int, n: int, k, v, stream=None) -> None:
    _check("sd_kv_read", lib().sd_kv_read(ctx, user, layer, pos0, n, _dev(k), _dev(v), _stream(stream)))


def sd_verify_batch(ctx: int, batch: int, assign: Sequence[int], draft_len: Sequence[int],
                    draft_tokens, q, mode, seed: int = 0, round_: int = 0, accept_u=None,
                    stream=None) -> None:
    a, L = _host_i32(assign), _host_i32(draft_len)
    mode = MODES[mode] if isinstance(mode, str) else int(mode)
    _check("sd_verify_batch", lib().sd_verify_batch(
        ctx, batch, a.size, a.ctypes.data, L.ctypes.data, _dev(draft_tokens), _dev(q), mode,
        int(seed), int(round_), _dev(accept_u), _stream(stream)))


def sd_verify_batch_graph(ctx: int, batch: int, assign: Sequence[int], draft_len: Sequence[int],
                          draft_tokens, q, mode, seed: int = 0, round_: int = 0, accept_u=None,
                          stream=None) -> None:
    a, L = _host_i32(assign), _host_i32(draft_len)
    mode = MODES[mode] if isinstance(mode, str) else int(mode)
    _check("sd_verify_batch_graph", lib().sd_verify_batch_graph(
        ctx, batch, a.size, a.ctypes.data, L.ctypes.data, _dev(draft_tokens), _dev(q), mode,
        int(seed), int(round_), _dev(accept_u), _stream(stream)))


def sd_verify_batch_sparse(ctx: int, batch: int, assign: Sequence[int], draft_len: Sequence[int],
                           draft_tokens, q_idx, q_val, q_rest, mode, seed: int = 0, round_: int = 0,
                           accept_u=None, stream=None) -> None:
    """q_idx int32 [nd][K], q_val fp32 [nd][K], q_rest fp32 [nd] (device)."""
    a, L = _host_i32(assign), _host_i32(draft_len)
    mode = MODES[mode] if isinstance(mode, str) else int(mode)
    k = int(q_idx.shape[1]) if hasattr(q_idx, "shape") else 0
    _check("sd_verify_batch_sparse", lib().sd_verify_batch_sparse(
        ctx, batch, a.size, a.ctypes.data, L.ctypes.data, _dev(draft_tokens), _dev(q_idx), _dev(q_val),
        _dev(q_rest), k, mode, int(seed), int(round_), _dev(accept_u), _stream(stream)))


def sd_draft_batch(ctx: int, batch: int, assign: Sequence[int], mode, seed: int = 0,
                   round_: int = 0, probs=None, probs_row=None, stream=None) -> None:
    a = _host_i32(assign)
    pr = None if probs_row is None else _host_i32(probs_row)
    mode = MODES[mode] if isinstance(mode, str) else int(mode)
    _check("sd_draft_batch", lib().sd_draft_batch(
        ctx, batch, a.size, a.ctypes.data, mode, int(seed), int(round_), _dev(probs),
        None if pr is None else pr.ctypes.data, _stream(stream)))


def sd_sample_logits(ctx: int, batch: int, assign, draft_len, draft_tokens, q, logits, mode,
                     seed: int = 0, round_: int = 0, accept_u=None, stream=None) -> None:
    a, L = _host_i32(assign), _host_i32(draft_len)
    mode = MODES[mode] if isinstance(mode, str) else int(mode)
    _check("sd_sample_logits", lib().sd_sample_logits(
        ctx, batch, a.size, a.ctypes.data, L.ctypes.data, _dev(draft_tokens), _dev(q), _dev(logits),
        mode, int(seed), int(round_), _dev(accept_u), _stream(stream)))


def sd_sample_logits_noalloc(user_ids, draft_len, vocab: int, draft_tokens, q, logits, mode,
                             result, seed: int = 0, round_: int = 0, accept_u=None,
                             stream=None) -> None:
    """Context-free accept/resample on caller logits; result: device int32
    [2*B + 1] (n_acc, token, flag word), written asynchronously."""
    u, L = _host_i32(user_ids), _host_i32(draft_len)
    if u.size != L.size:
        raise ValueError("user_ids and draft_len differ in length")
    mode = MODES[mode] if isinstance(mode, str) else int(mode)
    _check("sd_sample_logits_noalloc", lib().sd_sample_logits_noalloc(
        u.size, u.ctypes.data, L.ctypes.data, int(vocab), _dev(draft_tokens), _dev(q), _dev(logits),
        mode, int(seed), int(round_), _dev(accept_u), _dev(result), _stream(stream)))


def _dtype(t, what: str) -> int:
    name = str(t.dtype)
    if name not in _DTYPES:
        raise ValueError(f"{what}: float32 or bfloat16, not {name}")
    return _DTYPES[name]


_DTYPES = {"torch.float32": SD_F32, "torch.bfloat16": SD_BF16}


def _vec(t, n: int, dtype: str, what: str, at) -> Optional[int]:
    """Device pointer of a contiguous [n] tensor of one type on device `at`, or None."""
    if t is None:
        return None
    if str(t.dtype) != dtype or tuple(t.shape) != (n,) or not t.is_contiguous() or t.device != at:
        raise ValueError(f"{what}: a contiguous {dtype} tensor of {n} on {at}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _matrix(t, cols: Optional[int], what: str, at):
    """(device pointer, row stride) of a [rows][cols] tensor whose rows are contiguous and apart."""
    if t.dim() != 2 or t.device != at or (cols is not None and t.shape[1] != cols):
        raise ValueError(f"{what}: a matrix{'' if cols is None else f' of {cols} columns'} on {at}, not "
                         f"{tuple(t.shape)} on {t.device}")
    n, c = t.shape
    if (c > 1 and t.stride(1) != 1) or (n > 1 and t.stride(0) < c):
        raise ValueError(f"{what}: rows must be contiguous and apart, strides are {t.stride()}")
    return t.data_ptr(), (t.stride(0) if n > 1 else c)


def _on_current_device(t, what: str):
    import torch
    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        raise ValueError(f"{what}: on {t.device}, not on the current GPU")
    return t.device


def _workspace(t, at):
    if t.device != at or not t.is_contiguous():
        raise ValueError(f"workspace: a contiguous tensor on {at}")
    return t.data_ptr(), t.numel() * t.element_size()


def _filter(n: int, at, temperature, top_k, top_p, min_p) -> sd_filter:
    return sd_filter(_vec(temperature, n, "torch.float32", "temperature", at), _vec(top_k, n, "torch.int32", "top_k", at),
                     _vec(top_p, n, "torch.float32", "top_p", at), _vec(min_p, n, "torch.float32", "min_p", at))


def sd_filter_query_size(n_rows: int, vocab: int) -> int:
    """Bytes of workspace of sd_sample_filtered and sd_filter_logits."""
    b = ctypes.c_uint64()
    _check("sd_filter_query_size", lib().sd_filter_query_size(int(n_rows), int(vocab), ctypes.byref(b)))
    return b.value


def sd_sample_filtered(logits, u, token, workspace, temperature=None, top_k=None, top_p=None, min_p=None,
                       prob=None, kept=None, stream=None) -> None:
    """One token a row of logits (float32 or bfloat16 [n][vocab], rows any
    distance apart) from uniforms u [n] under per-row options (device
    tensors [n]; None: off).  Writes token int32 [n] and, where given, prob
    float32 [n] and kept int32 [n]."""
    at = _on_current_device(logits, "logits")
    ptr, stride = _matrix(logits, None, "logits", at)
    n, vocab = logits.shape
    f = _filter(n, at, temperature, top_k, top_p, min_p)
    ws, size = _workspace(workspace, at)
    _check("sd_sample_filtered", lib().sd_sample_filtered(
        n, vocab, ptr, _dtype(logits, "logits"), stride, ctypes.byref(f), _vec(u, n, "torch.float32", "u", at),
        _vec(token, n, "torch.int32", "token", at), _vec(prob, n, "torch.float32", "prob", at),
        _vec(kept, n, "torch.int32", "kept", at), ws, size, _stream(stream)))


def sd_filter_logits(logits, out, workspace, temperature=None, top_k=None, top_p=None, min_p=None, kept=None,
                     stream=None) -> None:
    """The filtered rows: out float32 [n][vocab] = (logit - largest) / T
    where a token is kept, -inf elsewhere.  out may be logits."""
    at = _on_current_device(logits, "logits")
    ptr, stride = _matrix(logits, None, "logits", at)
    n, vocab = logits.shape
    optr, ostride = _matrix(out, vocab, "out", at)
    if out.shape[0] != n or _dtype(out, "out") != SD_F32:
        raise ValueError(f"out: float32 of {n} rows, not {out.dtype} of {out.shape[0]}")
    f = _filter(n, at, temperature, top_k, top_p, min_p)
    ws, size = _workspace(workspace, at)
    _check("sd_filter_logits", lib().sd_filter_logits(
        n, vocab, ptr, _dtype(logits, "logits"), stride, ctypes.byref(f), optr, ostride,
        _vec(kept, n, "torch.int32", "kept", at), ws, size, _stream(stream)))


class Lora:
    """The adapters of one projection (sd_lora) with the tensors they live in."""

    def __init__(self, desc: sd_lora, a, b, scale):
        self.desc, self.a, self.b, self.scale = desc, a, b, scale
        self.ref = ctypes.byref(desc)


def make_lora(a, b, scale=None, segs: Optional[Sequence[int]] = None) -> Lora:
    """Adapters from a [n][n_seg * rank][d_in] and b [n][d_out][rank] (float32
    or bfloat16, contiguous) and scale float32 [n] (None: 1).  segs: widths
    of the projection's column segments, each with rows of `a` of its own
    (None: one)."""
    at = _on_current_device(a, "a")
    if a.dim() != 3 or b.dim() != 3 or a.shape[0] != b.shape[0] or a.dtype != b.dtype or b.device != at:
        raise ValueError("a [n][n_seg * rank][d_in] and b [n][d_out][rank] of one type on one GPU")
    if not a.is_contiguous() or not b.is_contiguous():
        raise ValueError("a and b must be contiguous")
    n, d_out, rank = b.shape
    segs = [d_out] if segs is None else [int(x) for x in segs]
    if not 1 <= len(segs) <= SD_LORA_MAX_SEGS or min(segs) < 1 or sum(segs) != d_out or a.shape[1] != len(segs) * rank:
        raise ValueError(f"segments {segs} do not fit a {tuple(a.shape)} and b {tuple(b.shape)}")
    off = (ctypes.c_int32 * (SD_LORA_MAX_SEGS + 1))()
    for i, w in enumerate(segs):
        off[i + 1] = off[i] + w
    d = sd_lora(n, rank, a.shape[2], d_out, len(segs), off, _dtype(a, "a"), a.data_ptr(), b.data_ptr(),
                _vec(scale, n, "torch.float32", "scale", at))
    return Lora(d, a, b, scale)


def sd_lora_query_size(w: Lora, n_rows: int) -> int:
    """Bytes of workspace of sd_lora_apply for up to n_rows rows."""
    b = ctypes.c_uint64()
    _check("sd_lora_query_size", lib().sd_lora_query_size(w.ref, int(n_rows), ctypes.byref(b)))
    return b.value


def sd_lora_apply(w: Lora, adapter, x, y_in, y_out, workspace, x_lo=None, stream=None) -> None:
    """y_out[t] = y_in[t] + scale[a] B_a (A_a x[t]) with a = adapter[t] (int32
    [n]; outside the adapters: y_in[t]).  y_out may be y_in."""
    at = _on_current_device(x, "x")
    n = x.shape[0]
    if w.a.device != at:
        raise ValueError(f"adapters on {w.a.device}, x on {at}")
    xp, xs = _matrix(x, w.desc.d_in, "x", at)
    yi, ys = _matrix(y_in, w.desc.d_out, "y_in", at)
    yo, yos = _matrix(y_out, w.desc.d_out, "y_out", at)
    lo = None
    if x_lo is not None:
        lo, los = _matrix(x_lo, w.desc.d_in, "x_lo", at)
        if x_lo.shape != x.shape or los != xs or x_lo.dtype != x.dtype:
            raise ValueError("x_lo: a plane like x")
    if y_in.shape[0] != n or y_out.shape[0] != n or y_in.dtype != y_out.dtype or x.dtype != w.a.dtype:
        raise ValueError("x, y_in and y_out: as many rows each, x of the adapters' type, y_out of y_in's")
    ws, size = _workspace(workspace, at)
    _check("sd_lora_apply", lib().sd_lora_apply(
        w.ref, n, _vec(adapter, n, "torch.int32", "adapter", at), xp, lo, xs, yi, ys, yo, yos, _dtype(y_in, "y_in"),
        ws, size, _stream(stream)))


class KVPool:
    """A paged cache (sd_kv_pool) with the tensor it lives in."""

    def __init__(self, desc: sd_kv_pool, base):
        self.desc, self.base, self.device = desc, base, base.device
        self.ref = ctypes.byref(desc)


def make_kv_pool(base, n_layers: int, n_pages: int, n_kv_heads: int, head_dim: int, dtype: Optional[int] = None) -> KVPool:
    """A paged cache in a contiguous tensor of n_layers * n_pages * 2 *
    n_kv_heads * 16 * head_dim elements (float32 or bfloat16, or bytes
    with dtype SD_F32 or SD_BF16, as Verifier.kv_pool is)."""
    at = _on_current_device(base, "base")
    dtype = _dtype(base, "base") if dtype is None else int(dtype)
    es = 2 if dtype == SD_BF16 else 4
    want = n_layers * n_pages * 2 * n_kv_heads * 16 * head_dim * es
    if not base.is_contiguous() or base.numel() * base.element_size() != want:
        raise ValueError(f"base: a contiguous tensor of {want} bytes on {at}, not {base.numel() * base.element_size()}")
    return KVPool(sd_kv_pool(n_layers, n_pages, n_kv_heads, head_dim, dtype, base.data_ptr()), base)


def _table(t, rows: Optional[int], what: str, at):
    """(device pointer, columns) of a contiguous int32 matrix."""
    if str(t.dtype) != "torch.int32" or t.dim() != 2 or not t.is_contiguous() or t.device != at or (
            rows is not None and t.shape[0] != rows):
        raise ValueError(f"{what}: a contiguous int32 matrix{'' if rows is None else f' of {rows} rows'} on {at}, not "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr(), t.shape[1]


class Tree:
    """Users' trees of drafts (sd_tree) with the tensors they live in."""

    def __init__(self, desc: sd_tree, tensors, device):
        self.desc, self.tensors, self.device = desc, tensors, device
        self.ref = ctypes.byref(desc)


def make_tree(slot_off, prefix, page_table, parent=None, *, max_slots: int, n_slots: Optional[int] = None) -> Tree:
    """Trees from device int32 slot_off [n + 1], prefix [n], page_table
    [n][max_pages] and parent [n_slots] (None: chains; n_slots is then
    needed).  max_slots: the most slots of a user."""
    at = _on_current_device(slot_off, "slot_off")
    n = slot_off.numel() - 1
    table, max_pages = _table(page_table, n, "page_table", at)
    if parent is not None:
        if n_slots is not None and n_slots != parent.numel():
            raise ValueError(f"parent of {parent.numel()} slots, not {n_slots}")
        n_slots = parent.numel()
    elif n_slots is None:
        raise ValueError("n_slots is needed without parent")
    d = sd_tree(n, int(n_slots), int(max_slots), max_pages, _vec(slot_off, n + 1, "torch.int32", "slot_off", at),
                _vec(prefix, n, "torch.int32", "prefix", at), table, _vec(parent, n_slots, "torch.int32", "parent", at))
    return Tree(d, (slot_off, prefix, page_table, parent), at)


def sd_tree_query_size(pool: KVPool, tree: Tree, n_q_heads: int) -> int:
    """Bytes of workspace of sd_tree_attention."""
    b = ctypes.c_uint64()
    _check("sd_tree_query_size", lib().sd_tree_query_size(pool.ref, tree.ref, int(n_q_heads), ctypes.byref(b)))
    return b.value


def _heads(t, like, what: str, at):
    """(device pointer, row stride) of [n_slots][heads][head_dim] rows, each contiguous."""
    if t.dim() != 3 or t.device != at or (like is not None and (t.shape != like.shape or t.dtype != like.dtype)):
        raise ValueError(f"{what}: [slots][heads][head_dim] on {at}{'' if like is None else ' like q'}, not {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    n, h, d = t.shape
    if (d > 1 and t.stride(2) != 1) or (h > 1 and t.stride(1) != d) or (n > 1 and t.stride(0) < h * d):
        raise ValueError(f"{what}: a slot's heads must be contiguous and slots apart, strides are {t.stride()}")
    return t.data_ptr(), (t.stride(0) if n > 1 else h * d)


def sd_tree_attention(pool: KVPool, layer: int, tree: Tree, q, out, workspace, q_lo=None, out_lo=None,
                      scale: Optional[float] = None, stream=None) -> None:
    """out[t][h] = attention of slot t's query head h over what it sees of its
    user's cache: q, out [n_slots][heads][head_dim] of the pool's type (q_lo,
    out_lo: second bf16 planes), scale 1 / sqrt(head_dim) by default."""
    at = _on_current_device(q, "q")
    if pool.device != at or tree.device != at:
        raise ValueError(f"pool on {pool.device}, trees on {tree.device}, q on {at}")
    qp, qs = _heads(q, None, "q", at)
    op, os_ = _heads(out, q, "out", at)
    if q.shape[0] != tree.desc.n_slots or q.shape[2] != pool.desc.head_dim or _dtype(q, "q") != pool.desc.dtype:
        raise ValueError(f"q: {tree.desc.n_slots} slots of heads of {pool.desc.head_dim} in the pool's type, not {q.dtype} "
                         f"{tuple(q.shape)}")
    ql = ol = None
    if q_lo is not None:
        ql, s = _heads(q_lo, q, "q_lo", at)
        if s != qs:
            raise ValueError("q_lo: strides like q's")
    if out_lo is not None:
        ol, s = _heads(out_lo, q, "out_lo", at)
        if s != os_:
            raise ValueError("out_lo: strides like out's")
    ws, size = _workspace(workspace, at)
    _check("sd_tree_attention", lib().sd_tree_attention(
        pool.ref, int(layer), tree.ref, q.shape[1], qp, ql, qs, op, ol, os_,
        q.shape[2] ** -0.5 if scale is None else float(scale), ws, size, _stream(stream)))


def sd_kv_copy_pages(pool: KVPool, src, dst, stream=None) -> None:
    """Pages dst[i] := pages src[i] (device int32) in every layer."""
    at = _on_current_device(src, "src")
    if pool.device != at:
        raise ValueError(f"pool on {pool.device}, src on {at}")
    n = src.numel()
    _check("sd_kv_copy_pages", lib().sd_kv_copy_pages(
        pool.ref, n, _vec(src, n, "torch.int32", "src", at), _vec(dst, n, "torch.int32", "dst", at), _stream(stream)))


def sd_kv_compact(pool: KVPool, prefix, page_table, keep, n_keep, stream=None) -> None:
    """Position prefix[b] + i := position prefix[b] + keep[b][i], i < n_keep[b], in
    every layer and head (device int32 [n], [n][max_pages], [n][max_keep], [n])."""
    at = _on_current_device(prefix, "prefix")
    if pool.device != at:
        raise ValueError(f"pool on {pool.device}, prefix on {at}")
    n = prefix.numel()
    table, max_pages = _table(page_table, n, "page_table", at)
    kp, max_keep = _table(keep, n, "keep", at)
    _check("sd_kv_compact", lib().sd_kv_compact(
        pool.ref, n, _vec(prefix, n, "torch.int32", "prefix", at), table, max_pages, kp, max_keep,
        _vec(n_keep, n, "torch.int32", "n_keep", at), _stream(stream)))


class LogitRules:
    """Rules on rows of logits (sd_logit_rules) with the tensors they live in."""

    def __init__(self, desc: sd_logit_rules, n_rows: int, vocab: int, tensors, device):
        self.desc, self.n_rows, self.vocab, self.tensors, self.device = desc, n_rows, vocab, tensors, device
        self.ref = ctypes.byref(desc)


def make_logit_rules(n_rows: int, vocab: int, *, tokens=None, hist=None, repetition=None, presence=None, frequency=None,
                     row_token=None, row_parent=None, bias_token=None, bias_value=None, bias=None, mask=None,
                     mask_row=None) -> LogitRules:
    """Rules for n_rows rows of `vocab` logits (device tensors, None: off):
    tokens int32 [n] and hist int32 [n_rows][3]; repetition, presence, frequency
    float32 [n_rows]; row_token, row_parent int32 [n_rows]; bias_token int32
    [m], bias_value float32 [m] and bias int32 [n_rows][2]; mask int32 [k][ceil(vocab
    / 32)] (bits of allowed tokens) and mask_row int32 [n_rows]."""
    tensors = (tokens, hist, repetition, presence, frequency, row_token, row_parent, bias_token, bias_value, bias, mask,
               mask_row)
    given = [t for t in tensors if t is not None]
    if not given:
        raise ValueError("no rules")
    at = _on_current_device(given[0], "rules")
    for a, b, names in ((tokens, hist, "tokens and hist"), (row_token, row_parent, "row_token and row_parent"),
                        (bias_token, bias, "bias_token and bias"), (bias_token, bias_value, "bias_token and bias_value"),
                        (mask, mask_row, "mask and mask_row")):
        if (a is None) != (b is None):
            raise ValueError(f"{names} belong together")

    def table(t, cols, what):
        if t is None:
            return None
        p, c = _table(t, None if what == "mask" else n_rows, what, at)
        if c != cols:
            raise ValueError(f"{what}: {cols} columns, not {c}")
        return p

    i32, f32 = "torch.int32", "torch.float32"
    size = lambda t: 0 if t is None else t.numel()  # noqa: E731
    d = sd_logit_rules(
        _vec(tokens, size(tokens), i32, "tokens", at), size(tokens), table(hist, 3, "hist"),
        _vec(row_token, n_rows, i32, "row_token", at), _vec(row_parent, n_rows, i32, "row_parent", at),
        _vec(repetition, n_rows, f32, "repetition", at), _vec(presence, n_rows, f32, "presence", at),
        _vec(frequency, n_rows, f32, "frequency", at), _vec(bias_token, size(bias_token), i32, "bias_token", at),
        _vec(bias_value, size(bias_token), f32, "bias_value", at), size(bias_token), table(bias, 2, "bias"),
        table(mask, (vocab + 31) // 32, "mask"), 0 if mask is None else mask.shape[0],
        _vec(mask_row, n_rows, i32, "mask_row", at))
    return LogitRules(d, n_rows, vocab, tensors, at)


def sd_adjust_logits(logits, rules: LogitRules, out, stream=None) -> None:
    """out float32 [n][vocab] = the rows of logits (float32 or bfloat16) under the
    rules.  out may be logits."""
    at = _on_current_device(logits, "logits")
    ptr, stride = _matrix(logits, rules.vocab, "logits", at)
    optr, ostride = _matrix(out, rules.vocab, "out", at)
    n = logits.shape[0]
    if n != rules.n_rows or out.shape[0] != n or _dtype(out, "out") != SD_F32 or rules.device != at:
        raise ValueError(f"logits and out: {rules.n_rows} rows, out float32, on the rules' {rules.device}, not {n} and "
                         f"{out.dtype} of {out.shape[0]} on {at}")
    _check("sd_adjust_logits", lib().sd_adjust_logits(
        n, rules.vocab, ptr, _dtype(logits, "logits"), stride, rules.ref, optr, ostride, _stream(stream)))


def sd_user_sampling(ctx: int, user: int, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0,
                     min_p: float = 0.0) -> None:
    top_k = max(-1, min(int(top_k), 2**31 - 1))  # (more than any vocab is off as well)
    _check("sd_user_sampling", lib().sd_user_sampling(ctx, user, float(temperature), top_k, float(top_p), float(min_p)))


def sd_adapters_set(ctx: int, layers) -> None:
    """layers: per layer of the context's model a dict of Lora under "qkv", "o",
    "down" (any of them left out) on the context's GPU, or None to take all
    adapters away.  Their tensors are kept alive until the next call that
    succeeds or sd_verify_destroy; changing the list or its dicts
    afterwards changes nothing."""
    known = _contexts.get(ctx)
    if known is None:
        raise ValueError("not a context of sd_verify_init")
    if layers is None:
        _check("sd_adapters_set", lib().sd_adapters_set(ctx, 0, None))
        known.adapters = None
        return
    if len(layers) != known.n_layers:
        raise ValueError(f"adapters of {len(layers)} layers, the model has {known.n_layers}")
    arr = (sd_layer_adapters * len(layers))()
    keep, n = [], 0
    for dst, src in zip(arr, layers):
        for name, w in src.items():
            if name not in ("qkv", "o", "down"):
                raise ValueError(f"no adapters beside {name}")
            if w.a.device.index != known.device:
                raise ValueError(f"adapters beside {name} on {w.a.device}, the context on GPU {known.device}")
            setattr(dst, name, w.desc)
            keep.append((w.a, w.b, w.scale))
            n = w.desc.n_adapters
    _check("sd_adapters_set", lib().sd_adapters_set(ctx, n, arr))
    known.adapters = keep


def sd_user_adapter(ctx: int, user: int, adapter: int) -> None:
    _check("sd_user_adapter", lib().sd_user_adapter(ctx, user, int(adapter)))


def sd_accept(ctx: int, batch: int, n_users: int, commit: bool = False):
    """Returns (n_accepted[M], out_token[M]); entries of users outside the
    batch are -1."""
    n_acc = np.full(n_users, -1, np.int32)
    tok = np.full(n_users, -1, np.int32)
    _done(ctx, batch, "sd_accept", lib().sd_accept(ctx, batch, n_acc.ctypes.data, tok.ctypes.data, int(commit)))
    return n_acc, tok


def sd_verify_batch_tree(ctx: int, batch: int, assign: Sequence[int], draft_len: Sequence[int], draft_tokens,
                         parent: Sequence[int], mode, seed: int = 0, round_: int = 0, stream=None) -> None:
    """parent (host) [sum l_m]: the parent of each draft, 0 the root, else the
    number (1 ..) of an earlier draft of its user."""
    a, L, par = _host_i32(assign), _host_i32(draft_len), _host_i32(parent)
    if a.size != L.size:
        raise ValueError("assign and draft_len differ in length")
    if par.size != int(L[a == batch].sum()):
        raise ValueError(f"parent: {int(L[a == batch].sum())} drafts, not {par.size}")
    mode = MODES[mode] if isinstance(mode, str) else int(mode)
    _check("sd_verify_batch_tree", lib().sd_verify_batch_tree(
        ctx, batch, a.size, a.ctypes.data, L.ctypes.data, _dev(draft_tokens), par.ctypes.data, mode,
        int(seed), int(round_), _stream(stream)))


def sd_accept_tree(ctx: int, batch: int, n_users: int, commit: bool = False):
    """Returns (n_accepted[M], out_token[M], path[M][max_draft]); entries of users
    outside the batch are -1."""
    known = _contexts.get(ctx)
    if known is None:
        raise ValueError("not a context of sd_verify_init")
    n_acc, tok = np.full(n_users, -1, np.int32), np.full(n_users, -1, np.int32)
    path = np.full((n_users, known.max_draft), -1, np.int32)
    _done(ctx, batch, "sd_accept_tree", lib().sd_accept_tree(ctx, batch, n_acc.ctypes.data, tok.ctypes.data,
                                                             path.ctypes.data, int(commit)))
    return n_acc, tok, path


def sd_user_fork(ctx: int, user: int, from_: int, prefix_len: int, root_token: int, stream=None) -> None:
    _check("sd_user_fork", lib().sd_user_fork(ctx, user, from_, prefix_len, root_token, _stream(stream)))


def sd_user_pages(ctx: int, user: int) -> np.ndarray:
    """The pages that a user holds, in order."""
    n = ctypes.c_int32()
    _check("sd_user_pages", lib().sd_user_pages(ctx, user, None, 0, ctypes.byref(n)))
    pages = np.zeros(n.value, np.int32)
    _check("sd_user_pages", lib().sd_user_pages(ctx, user, pages.ctypes.data, pages.size, ctypes.byref(n)))
    return pages


def sd_batch_rules(ctx: int, batch: int, rules: Optional[LogitRules]) -> None:
    """Rules of the logits of the next pass of `batch` (None: none), one row a query
    slot, without row_token and row_parent.  Their tensors are kept alive
    until the pass is accepted."""
    known = _contexts.get(ctx)
    if known is None:
        raise ValueError("not a context of sd_verify_init")
    if rules is None:
        _check("sd_batch_rules", lib().sd_batch_rules(ctx, batch, 0, None))
        known.rules.pop(batch, None)
        return
    if rules.vocab != known.vocab or rules.device.index != known.device:
        raise ValueError(f"rules for {rules.vocab} tokens on {rules.device}, the context has {known.vocab} on GPU {known.device}")
    _check("sd_batch_rules", lib().sd_batch_rules(ctx, batch, rules.n_rows, rules.ref))
    known.rules[batch] = rules


def _done(ctx: int, batch: int, fn: str, status: int) -> None:
    """A pass is over, with or without decisions: its rules are no longer read."""
    known = _contexts.get(ctx)
    if known is not None and status in (SD_OK, SD_EDEVICE):
        known.rules.pop(batch, None)
    _check(fn, status)


def sd_debug_logits(ctx: int, batch: int, dst, stream=None) -> None:
    _check("sd_debug_logits", lib().sd_debug_logits(ctx, batch, _dev(dst), _stream(stream)))


def sd_debug_wait_limit(ctx: int, max_polls: int) -> None:
    _check("sd_debug_wait_limit", lib().sd_debug_wait_limit(ctx, max_polls))


def sd_profile_begin(ctx: int, kclass: int, max_launches: int = 4096) -> None:
    _check("sd_profile_begin", lib().sd_profile_begin(ctx, kclass, max_launches))


def sd_profile_end(ctx: int):
    """Returns (total_ms, launches) of the profiled kernel class."""
    ms, n = ctypes.c_double(), ctypes.c_int32()
    _check("sd_profile_end", lib().sd_profile_end(ctx, ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def sd_calib_hbm(buf_ptr: int, nbytes: int, mode: int, reps: int, stream: int = 0) -> float:
    """Achieved GB/s (bytes read + written) of a copy (mode 0) or read-only
    stream (mode 1) over the caller's device buffer."""
    gbs = ctypes.c_double()
    _check("sd_calib_hbm", lib().sd_calib_hbm(buf_ptr, nbytes, mode, reps, ctypes.byref(gbs), stream))
    return gbs.value


def sd_calib_mfma(sink_ptr: int, iters: int, stream: int = 0) -> float:
    """Achieved dense bf16 MFMA TFLOP/s of a register-only MFMA loop."""
    tf = ctypes.c_double()
    _check("sd_calib_mfma", lib().sd_calib_mfma(sink_ptr, iters, ctypes.byref(tf), stream))
    return tf.value


def make_config(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, vocab, qk_norm, dtype,
                n_pages, max_users, max_draft, max_batch_users, max_batch_tokens, max_ctx,
                max_pending=2, rope_base=1e6, rms_eps=1e-6, logits_out=0) -> sd_config:
    return sd_config(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, vocab, int(qk_norm),
                     int(dtype), 16, n_pages, max_users, max_draft, max_batch_users, max_batch_tokens,
                     max_ctx, max_pending, float(rope_base), float(rms_eps), int(logits_out))
