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
           "sd_lora_apply", "sd_user_sampling", "sd_adapters_set", "sd_user_adapter", "sd_calib_hbm", "sd_calib_mfma", "sd_status_str")
SD_FILTER_MAX_ROWS, SD_FILTER_MAX_VOCAB = 65535, 1 << 20
SD_LORA_MAX_RANK, SD_LORA_MAX_SEGS = 128, 4
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
    """What sd_adapters_set needs to know of a context, and the adapters that the
    library reads in place."""

    def __init__(self, n_layers: int, device: int):
        self.n_layers, self.device, self.adapters = n_layers, device, None


_contexts: Dict[int, _Context] = {}


def sd_verify_init(cfg: sd_config, weights: sd_weights, kv_pool, workspace, weight_pack=None) -> int:
    import torch
    out = ctypes.c_void_p()
    _check("sd_verify_init", lib().sd_verify_init(ctypes.byref(cfg), ctypes.byref(weights),
                                                  _dev(kv_pool), _dev(workspace), _dev(weight_pack),
                                                  ctypes.byref(out)))
    _contexts[out.value] = _Context(cfg.n_layers, torch.cuda.current_device())
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
    _check("sd_accept", lib().sd_accept(ctx, batch, n_acc.ctypes.data, tok.ctypes.data, int(commit)))
    return n_acc, tok


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
