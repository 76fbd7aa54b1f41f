"""ctypes binding of libspo.so: one Python function per C entry point, same names.

Argument marshalling only.  Tensors are torch CUDA tensors used as device
buffers (``data_ptr()``), the stream is torch's current stream; every step of
the path runs inside the library's CUDA kernels.  There is no CPU fallback: if
the shared library has not been built, loading it raises.
"""

from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, Structure, c_char_p, c_float, c_int32, c_int64, c_size_t, c_void_p

# SPO_LIBRARY_PATH points at another build of the same library (e.g. one compiled with different tile options).
_LIB_PATH = os.environ.get("SPO_LIBRARY_PATH") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libspo.so")

SPO_OK = 0
ERR_INVALID_ARG, ERR_BAD_SHAPE, ERR_BAD_ALIGNMENT = -1, -2, -3
ERR_UNSUPPORTED_DTYPE, ERR_UNSUPPORTED_ARCH, ERR_WORKSPACE_TOO_SMALL, ERR_CUDA = -4, -5, -6, -7
DEV_ID_OUT_OF_RANGE, DEV_NONFINITE, DEV_UNIFORMS_EXHAUSTED, DEV_TIMEOUT, DEV_ZERO_TOTAL_WEIGHT = 1, 2, 4, 8, 16
DTYPE_F32, DTYPE_BF16 = 0, 1
(WS_SAMPLE, WS_ADVANTAGES, WS_LOSS_FWD, WS_LOSS_BWD, WS_UPDATE_REPEATS, WS_ACTIVE_ROWS, WS_LOSS_BWD_ROWS,
 WS_LOSS_FWD_BWD, WS_LOSS_FWD_BWD_ROWS, WS_LOGPROBS, WS_LOGPROBS_BWD,
 WS_MUON, WS_LAYERNORM_BWD, WS_GRAD_NORM) = range(14)
AGG_TOKEN_MEAN, AGG_SEQ_MEAN = 0, 1
SUR_PPO_CLIP, SUR_CISPO, SUR_GSPO = 0, 1, 2
MUON_SCALE_NONE, MUON_SCALE_SPECTRAL, MUON_SCALE_RMS = 0, 1, 2
NORM_LAYER, NORM_RMS = 0, 1
ADAMW_BLOCK = 256                # elements of an 8-bit state that share a scale

EXPORTS = [
    "spo_default_params", "spo_tracker_init", "spo_sample_prompts", "spo_advantages",
    "spo_advantages_static", "spo_advantages_apply", "spo_advantages_update",
    "spo_tracker_update", "spo_tracker_update_repeats", "spo_loss_fwd", "spo_loss_bwd", "spo_loss_fwd_bwd", "spo_loss_fwd_bwd_slabs", "spo_dw_slab_rows", "spo_loss_fwd_bwd_scatter", "spo_loss_stats", "spo_loss_mask_rows", "spo_loss_fwd_bwd_rows", "spo_loss_active_rows", "spo_loss_bwd_rows",
    "spo_logprobs", "spo_logprobs_bwd", "spo_default_muon_params", "spo_orthogonalize", "spo_muon_update",
    "spo_layernorm_fwd", "spo_layernorm_bwd", "spo_grad_norm", "spo_default_adamw_params", "spo_adamw_update", "spo_adamw_decode",
    "spo_workspace_bytes",
    "spo_status_string", "spo_last_cuda_error", "spo_version", "spo_selftest_bounded_wait",
]


class SpoParams(Structure):
    _fields_ = [
        ("rho_min", c_float), ("rho_max", c_float), ("d_half", c_float), ("eps_explore", c_float),
        ("clip_lo", c_float), ("clip_hi", c_float), ("norm_eps", c_float), ("norm_ddof", c_int32),
        ("agg_mode", c_int32), ("global_tokens", c_int32), ("global_responses", c_int32),
        ("surrogate", c_int32), ("dual_clip", c_float), ("near_zero_tau_lo", c_float),
        ("near_zero_tau_hi", c_float),
    ]


class SpoMuonParams(Structure):
    _fields_ = [
        ("lr", c_float), ("momentum", c_float), ("weight_decay", c_float), ("eps", c_float),
        ("coef_a", c_float), ("coef_b", c_float), ("coef_c", c_float),
        ("steps", c_int32), ("nesterov", c_int32), ("scale_mode", c_int32),
    ]


class SpoAdamwParams(Structure):
    _fields_ = [
        ("lr", c_float), ("beta1", c_float), ("beta2", c_float), ("eps", c_float), ("weight_decay", c_float), ("step", c_int32),
    ]


class SpoGradTensor(Structure):
    _fields_ = [("g", c_void_p), ("n", c_int64), ("dtype", c_int32), ("reserved", c_int32)]


class SpoAdamwTensor(Structure):
    _fields_ = [
        ("w", c_void_p), ("g", c_void_p), ("m", c_void_p), ("v", c_void_p), ("m_scale", c_void_p), ("v_scale", c_void_p),
        ("copy", c_void_p), ("n", c_int64), ("w_dtype", c_int32), ("g_dtype", c_int32), ("state_bits", c_int32),
        ("lr_scale", c_float), ("decay_scale", c_float), ("reserved", c_int32),
    ]


MAX_DW_SHARDS = 16


class SpoDwShards(Structure):
    _fields_ = [("n_shards", c_int32), ("rows_per_shard", c_int64), ("shard", c_void_p * MAX_DW_SHARDS)]


class SpoError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = lib().spo_status_string(status).decode()
        if status == ERR_CUDA:
            msg += " [cudaError %d]" % lib().spo_last_cuda_error()
        super().__init__("%s: %s (%d)" % (where, msg, status))


_lib = None


def lib():
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                "libspo.so is missing (%s): build it with `python -m paper_2509_13232_b200.build`; "
                "there is no fallback path" % _LIB_PATH)
        L = ctypes.CDLL(_LIB_PATH)
        P = POINTER(SpoParams)
        L.spo_default_params.argtypes = [P]
        L.spo_tracker_init.argtypes = [c_void_p, c_void_p, c_int64, P, c_void_p]
        L.spo_sample_prompts.argtypes = [c_void_p, c_int64, c_void_p, c_int32, c_int32, c_void_p, c_void_p,
                                         c_void_p, c_size_t, P, c_void_p, c_void_p]
        L.spo_advantages.argtypes = [c_void_p, c_int64, c_void_p, c_void_p, c_int32, c_void_p, c_void_p,
                                     c_void_p, c_void_p, c_size_t, P, c_void_p, c_void_p]
        L.spo_advantages_static.argtypes = [c_void_p, c_int64, c_void_p, c_void_p, c_int32, c_void_p, c_void_p,
                                            c_void_p, P, c_void_p, c_void_p]
        L.spo_advantages_update.argtypes = [c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_int32, c_int32,
                                            c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, P, c_void_p, c_void_p]
        L.spo_advantages_apply.argtypes = [c_void_p, c_int32, c_float, c_float, c_void_p, P, c_void_p]
        L.spo_tracker_update.argtypes = [c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_int32, c_int32,
                                         P, c_void_p, c_void_p]
        L.spo_tracker_update_repeats.argtypes = [c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_int32, c_int32,
                                                 c_void_p, c_size_t, P, c_void_p, c_void_p]
        L.spo_loss_fwd.argtypes = [c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_int64, c_int32, c_int32, c_int32,
                                   c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_void_p, c_size_t, P, c_void_p, c_void_p]
        L.spo_loss_bwd.argtypes = [c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_float,
                                   c_int64, c_int32, c_int32, c_void_p, c_int32, c_void_p, c_int32,
                                   c_void_p, c_size_t, P, c_void_p, c_void_p]
        L.spo_loss_fwd_bwd.argtypes = [c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_int64, c_int32, c_int32, c_int32, c_float,
                                       c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_void_p, c_int32, c_void_p, c_int32,
                                       c_void_p, c_size_t, P, c_void_p, c_void_p]
        L.spo_loss_fwd_bwd_slabs.argtypes = list(L.spo_loss_fwd_bwd.argtypes) + [c_int32, POINTER(c_void_p)]
        L.spo_loss_fwd_bwd_scatter.argtypes = list(L.spo_loss_fwd_bwd.argtypes) + [POINTER(SpoDwShards)]
        L.spo_dw_slab_rows.argtypes = [c_int32, c_int32, c_int32, POINTER(c_int64)]
        L.spo_loss_stats.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int32, c_void_p, P,
                                     c_void_p]
        L.spo_loss_mask_rows.argtypes = [c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
        L.spo_loss_fwd_bwd_rows.argtypes = [c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                            c_int64, c_int32, c_int32, c_int32, c_void_p, c_int64, c_float,
                                            c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                            c_void_p, c_int32, c_void_p, c_int32,
                                            c_void_p, c_size_t, P, c_void_p, c_void_p]
        L.spo_loss_active_rows.argtypes = [c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
        L.spo_loss_bwd_rows.argtypes = [c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_float,
                                        c_int64, c_int32, c_int32, c_void_p, c_int64, c_void_p, c_int32, c_void_p,
                                        c_int32, c_void_p, c_size_t, P, c_void_p, c_void_p]
        L.spo_logprobs.argtypes = [c_void_p, c_int64, c_void_p, c_int32, c_void_p, c_void_p, c_int64, c_int32, c_int32,
                                   c_float, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_void_p, c_size_t, c_void_p, c_void_p]
        L.spo_logprobs_bwd.argtypes = [c_void_p, c_int64, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_void_p, c_void_p, c_void_p, c_int64, c_int32, c_int32, c_float,
                                       c_void_p, c_int32, c_void_p, c_int32, c_int32,
                                       c_void_p, c_size_t, c_void_p, c_void_p]
        PM = POINTER(SpoMuonParams)
        L.spo_default_muon_params.argtypes = [PM]
        L.spo_orthogonalize.argtypes = [c_void_p, c_int32, c_int32, c_int64, c_int64, c_void_p, c_int32,
                                        c_void_p, c_size_t, PM, c_void_p, c_void_p]
        L.spo_muon_update.argtypes = [c_void_p, c_int32, c_void_p, c_void_p, c_int32, c_int32, c_int64, c_int64,
                                      c_void_p, c_size_t, PM, c_void_p, c_void_p]
        L.spo_layernorm_fwd.argtypes = [c_void_p, c_int64, c_void_p, c_int32, c_void_p, c_void_p, c_int32, c_void_p, c_int64, c_int32,
                                        c_float, c_int32, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
        L.spo_layernorm_bwd.argtypes = [c_void_p, c_int32, c_void_p, c_int64, c_int32, c_void_p, c_int32, c_void_p, c_void_p, c_void_p,
                                        c_void_p, c_int64, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_int32, c_int32,
                                        c_void_p, c_size_t, c_void_p, c_void_p]
        L.spo_grad_norm.argtypes = [c_void_p, c_int32, c_float, c_float, c_void_p, c_void_p, c_size_t, c_void_p, c_void_p]
        PA = POINTER(SpoAdamwParams)
        L.spo_default_adamw_params.argtypes = [PA]
        L.spo_adamw_update.argtypes = [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, PA, c_void_p, c_void_p]
        L.spo_adamw_decode.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p]
        L.spo_selftest_bounded_wait.argtypes = [ctypes.c_uint32, c_void_p, c_void_p, c_void_p]
        L.spo_workspace_bytes.argtypes = [c_int32, c_int64, c_int32, c_int32, c_int64, c_int32, c_int32]
        L.spo_workspace_bytes.restype = c_size_t
        L.spo_status_string.argtypes = [c_int32]
        L.spo_status_string.restype = c_char_p
        for name in EXPORTS:
            if name not in ("spo_workspace_bytes", "spo_status_string"):
                getattr(L, name).restype = c_int32
        _lib = L
    return _lib


def default_params(**overrides) -> SpoParams:
    p = SpoParams()
    rc = lib().spo_default_params(ctypes.byref(p))
    if rc != SPO_OK:
        raise SpoError(rc, "spo_default_params")
    for k, v in overrides.items():
        setattr(p, k, v)
    return p


def _ptr(t):
    return None if t is None else c_void_p(t.data_ptr())


def _stream():
    import torch
    return c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(rc, where):
    if rc != SPO_OK:
        raise SpoError(rc, where)


def _dtype_code(t):
    import torch
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    if t.dtype == torch.float32:
        return DTYPE_F32
    raise TypeError("H/W/dH must be float32 or bfloat16, got %s" % t.dtype)


def spo_workspace_bytes(which, T=0, d=0, V=0, N=0, B=0, M=0) -> int:
    return int(lib().spo_workspace_bytes(which, T, d, V, N, B, M))


def spo_tracker_init(ab, v0, params):
    _check(lib().spo_tracker_init(_ptr(ab), _ptr(v0), v0.numel(), ctypes.byref(params), _stream()),
           "spo_tracker_init")


def spo_sample_prompts(ab, uniforms, B, out_ids, out_w, ws, params, d_status):
    _check(lib().spo_sample_prompts(_ptr(ab), ab.shape[0], _ptr(uniforms), uniforms.numel(), B, _ptr(out_ids),
                                    _ptr(out_w), _ptr(ws), ws.numel() * ws.element_size(), ctypes.byref(params),
                                    _ptr(d_status), _stream()), "spo_sample_prompts")


def spo_advantages(ab, ids, r, a_raw, a_norm, stats, ws, params, d_status):
    _check(lib().spo_advantages(_ptr(ab), ab.shape[0], _ptr(ids), _ptr(r), ids.numel(), _ptr(a_raw), _ptr(a_norm),
                                _ptr(stats), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                ctypes.byref(params), _ptr(d_status), _stream()), "spo_advantages")


def spo_advantages_update(ab, ids, r, kl, kl_is_table, a_raw, a_norm, stats, ws, params, d_status):
    _check(lib().spo_advantages_update(_ptr(ab), ab.shape[0], _ptr(ids), _ptr(r), _ptr(kl), int(kl_is_table),
                                       ids.numel(), _ptr(a_raw), _ptr(a_norm), _ptr(stats), _ptr(ws),
                                       0 if ws is None else ws.numel() * ws.element_size(), ctypes.byref(params),
                                       _ptr(d_status), _stream()), "spo_advantages_update")


def spo_advantages_apply(a_raw, mu, sigma, a_norm, params):
    _check(lib().spo_advantages_apply(_ptr(a_raw), a_raw.numel(), c_float(mu), c_float(sigma), _ptr(a_norm),
                                      ctypes.byref(params), _stream()), "spo_advantages_apply")


ADVANTAGES_STATIC_MAX_B = 4194304


def spo_advantages_static(ab, ids, r, a_raw, a_norm, stats, params, d_status):
    """spo_advantages for callers that cannot supply scratch memory: same inputs and outputs,
    no `ws`; the library's own fixed device array holds the partial sums (B <= ADVANTAGES_STATIC_MAX_B;
    calls must not overlap on the GPU)."""
    _check(lib().spo_advantages_static(_ptr(ab), ab.shape[0], _ptr(ids), _ptr(r), ids.numel(), _ptr(a_raw),
                                       _ptr(a_norm), _ptr(stats), ctypes.byref(params), _ptr(d_status),
                                       _stream()), "spo_advantages_static")


def spo_tracker_update(ab, ids, r, kl, kl_is_table, params, d_status):
    _check(lib().spo_tracker_update(_ptr(ab), ab.shape[0], _ptr(ids), _ptr(r), _ptr(kl), int(kl_is_table),
                                    ids.numel(), ctypes.byref(params), _ptr(d_status), _stream()),
           "spo_tracker_update")


def spo_tracker_update_repeats(ab, ids, r, kl, kl_is_table, ws, params, d_status):
    _check(lib().spo_tracker_update_repeats(_ptr(ab), ab.shape[0], _ptr(ids), _ptr(r), _ptr(kl), int(kl_is_table),
                                            ids.numel(), _ptr(ws), ws.numel() * ws.element_size(),
                                            ctypes.byref(params), _ptr(d_status), _stream()),
           "spo_tracker_update_repeats")


def spo_loss_fwd(H, W, y, logp_old, mask, cu_seqlens, a_norm, loss, logp, lse, coef, seq_sums, ws, params,
                 d_status, entropy=None):
    T, d = H.shape
    V = W.shape[0]
    S = cu_seqlens.numel() - 1
    _check(lib().spo_loss_fwd(_ptr(H), _ptr(W), _dtype_code(W), _ptr(y), _ptr(logp_old), _ptr(mask),
                              _ptr(cu_seqlens), _ptr(a_norm), T, d, V, S, _ptr(loss), _ptr(logp), _ptr(lse),
                              _ptr(coef), _ptr(seq_sums), _ptr(entropy), _ptr(ws), ws.numel() * ws.element_size(),
                              ctypes.byref(params), _ptr(d_status), _stream()), "spo_loss_fwd")


def spo_loss_bwd(H, W, y, lse, coef, grad_loss, dH, dW, dW_accumulate, ws, params, d_status):
    T, d = H.shape
    V = W.shape[0]
    _check(lib().spo_loss_bwd(_ptr(H), _ptr(W), _dtype_code(W), _ptr(y), _ptr(lse), _ptr(coef),
                              c_float(grad_loss), T, d, V, _ptr(dH), _dtype_code(dH), _ptr(dW),
                              int(dW_accumulate), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                              ctypes.byref(params), _ptr(d_status), _stream()), "spo_loss_bwd")


def spo_loss_fwd_bwd(H, W, y, logp_old, mask, cu_seqlens, a_norm, grad_loss, loss, logp, lse, coef, seq_sums, dH, dW,
                     dW_accumulate, ws, params, d_status, entropy=None):
    T, d = H.shape
    V = W.shape[0]
    S = cu_seqlens.numel() - 1
    _check(lib().spo_loss_fwd_bwd(_ptr(H), _ptr(W), _dtype_code(W), _ptr(y), _ptr(logp_old), _ptr(mask),
                                  _ptr(cu_seqlens), _ptr(a_norm), T, d, V, S, c_float(grad_loss), _ptr(loss),
                                  _ptr(logp), _ptr(lse), _ptr(coef), _ptr(seq_sums), _ptr(entropy), _ptr(dH),
                                  _dtype_code(dH), _ptr(dW), int(dW_accumulate), _ptr(ws),
                                  ws.numel() * ws.element_size(), ctypes.byref(params), _ptr(d_status), _stream()),
           "spo_loss_fwd_bwd")


MAX_DW_SLABS = 64


def spo_dw_slab_rows(V, d, n_wanted):
    """Vocabulary-row bounds [0, ..., V] of the slabs a request for n_wanted slabs comes to (host only)."""
    buf = (c_int64 * (n_wanted + 1))()
    n = lib().spo_dw_slab_rows(V, d, n_wanted, buf)
    if n < 0:
        raise SpoError(n, "spo_dw_slab_rows")
    return [int(buf[k]) for k in range(n + 1)]


def spo_loss_fwd_bwd_slabs(H, W, y, logp_old, mask, cu_seqlens, a_norm, grad_loss, loss, logp, lse, coef, seq_sums, dH,
                           dW, dW_accumulate, ws, params, d_status, events, entropy=None):
    """spo_loss_fwd_bwd with the last dW contraction cut into len(events) slabs; `events` are
    torch.cuda.Event objects that already own a CUDA event (recorded once), one is recorded behind each slab."""
    T, d = H.shape
    V = W.shape[0]
    S = cu_seqlens.numel() - 1
    handles = (c_void_p * len(events))(*[c_void_p(ev.cuda_event) for ev in events])
    _check(lib().spo_loss_fwd_bwd_slabs(_ptr(H), _ptr(W), _dtype_code(W), _ptr(y), _ptr(logp_old), _ptr(mask),
                                        _ptr(cu_seqlens), _ptr(a_norm), T, d, V, S, c_float(grad_loss), _ptr(loss),
                                        _ptr(logp), _ptr(lse), _ptr(coef), _ptr(seq_sums), _ptr(entropy), _ptr(dH),
                                        _dtype_code(dH), _ptr(dW), int(dW_accumulate), _ptr(ws),
                                        ws.numel() * ws.element_size(), ctypes.byref(params), _ptr(d_status), _stream(),
                                        len(events), handles), "spo_loss_fwd_bwd_slabs")


def dw_shards(shard_ptrs, rows_per_shard) -> SpoDwShards:
    """Shard table for spo_loss_fwd_bwd_scatter: shard_ptrs[k] is the device address (an int, or a tensor) of the
    fp32 [rows_per_shard][d] buffer that owns vocabulary rows k*rows_per_shard ..; it may be peer memory."""
    sh = SpoDwShards()
    sh.n_shards = len(shard_ptrs)
    sh.rows_per_shard = int(rows_per_shard)
    for k, ptr in enumerate(shard_ptrs):
        sh.shard[k] = ptr if isinstance(ptr, int) else ptr.data_ptr()
    return sh


def spo_loss_fwd_bwd_scatter(H, W, y, logp_old, mask, cu_seqlens, a_norm, grad_loss, loss, logp, lse, coef, seq_sums,
                             dH, dW, dW_accumulate, ws, params, d_status, shards, entropy=None):
    """spo_loss_fwd_bwd whose last dW contraction adds the finished dW into the shards that own its rows."""
    T, d = H.shape
    V = W.shape[0]
    S = cu_seqlens.numel() - 1
    _check(lib().spo_loss_fwd_bwd_scatter(_ptr(H), _ptr(W), _dtype_code(W), _ptr(y), _ptr(logp_old), _ptr(mask),
                                          _ptr(cu_seqlens), _ptr(a_norm), T, d, V, S, c_float(grad_loss), _ptr(loss),
                                          _ptr(logp), _ptr(lse), _ptr(coef), _ptr(seq_sums), _ptr(entropy), _ptr(dH),
                                          _dtype_code(dH), _ptr(dW), int(dW_accumulate), _ptr(ws),
                                          ws.numel() * ws.element_size(), ctypes.byref(params), _ptr(d_status),
                                          _stream(), ctypes.byref(shards)), "spo_loss_fwd_bwd_scatter")


def spo_loss_stats(logp, logp_old, mask, cu_seqlens, a_norm, out, params):
    _check(lib().spo_loss_stats(_ptr(logp), _ptr(logp_old), _ptr(mask), _ptr(cu_seqlens), _ptr(a_norm), logp.numel(),
                                cu_seqlens.numel() - 1, _ptr(out), ctypes.byref(params), _stream()), "spo_loss_stats")


def spo_loss_mask_rows(mask, rows, d_count, ws):
    _check(lib().spo_loss_mask_rows(_ptr(mask), mask.numel(), _ptr(rows), _ptr(d_count), _ptr(ws),
                                    ws.numel() * ws.element_size(), _stream()), "spo_loss_mask_rows")


def spo_loss_fwd_bwd_rows(H, W, y, logp_old, cu_seqlens, a_norm, rows, n_listed, grad_loss, loss, logp, lse, coef,
                          seq_sums, dH, dW, dW_accumulate, ws, params, d_status):
    T, d = H.shape
    V = W.shape[0]
    S = cu_seqlens.numel() - 1
    _check(lib().spo_loss_fwd_bwd_rows(_ptr(H), _ptr(W), _dtype_code(W), _ptr(y), _ptr(logp_old), _ptr(cu_seqlens),
                                       _ptr(a_norm), T, d, V, S, _ptr(rows), int(n_listed), c_float(grad_loss),
                                       _ptr(loss), _ptr(logp), _ptr(lse), _ptr(coef), _ptr(seq_sums), _ptr(dH),
                                       _dtype_code(dH), _ptr(dW), int(dW_accumulate), _ptr(ws),
                                       ws.numel() * ws.element_size(), ctypes.byref(params), _ptr(d_status),
                                       _stream()), "spo_loss_fwd_bwd_rows")


def spo_selftest_bounded_wait(limit_us, reached_end, d_status):
    _check(lib().spo_selftest_bounded_wait(int(limit_us), _ptr(reached_end), _ptr(d_status), _stream()),
           "spo_selftest_bounded_wait")


def spo_loss_active_rows(coef, rows, d_count, ws):
    _check(lib().spo_loss_active_rows(_ptr(coef), coef.numel(), _ptr(rows), _ptr(d_count), _ptr(ws),
                                      ws.numel() * ws.element_size(), _stream()), "spo_loss_active_rows")


def spo_loss_bwd_rows(H, W, y, lse, coef, grad_loss, rows, n_active, dH, dW, dW_accumulate, ws, params, d_status):
    T, d = H.shape
    V = W.shape[0]
    _check(lib().spo_loss_bwd_rows(_ptr(H), _ptr(W), _dtype_code(W), _ptr(y), _ptr(lse), _ptr(coef),
                                   c_float(grad_loss), T, d, V, _ptr(rows), int(n_active), _ptr(dH), _dtype_code(dH),
                                   _ptr(dW), int(dW_accumulate), _ptr(ws), ws.numel() * ws.element_size(),
                                   ctypes.byref(params), _ptr(d_status), _stream()), "spo_loss_bwd_rows")


MAX_TOP_K = 20


class _Args:
    """Checks of one call's tensors: type, shape, layout and device (the current one).  The methods return addresses."""

    __slots__ = ("torch", "device")

    def __init__(self):
        import torch
        self.torch = torch
        self.device = torch.cuda.current_device()

    def here(self, name, t):
        if t.get_device() != self.device:
            raise ValueError("%s must be on the current CUDA device, is on %s" % (name, t.device))

    def need(self, name, t, dtype, shape):
        try:                                    # the call that is right pays one pass over the conditions
            if (dtype is None or t.dtype is dtype) and t.shape == shape and t.is_contiguous() and t.get_device() == self.device:
                return t.data_ptr()
        except AttributeError:
            pass
        if not isinstance(t, self.torch.Tensor):
            raise TypeError("%s must be a tensor, got %s" % (name, type(t).__name__))
        if dtype is not None and t.dtype is not dtype:
            raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
        if t.shape != shape:
            raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
        if not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
        self.here(name, t)
        return t.data_ptr()

    def may(self, name, t, dtype, shape):
        if t is None:
            return None
        return self.need(name, t, dtype, shape)

    def rows(self, H, W):
        """H [T, d] (rows contiguous, any row pitch) against W [V, d]: (T, d, V, row pitch of H)."""
        if not isinstance(H, self.torch.Tensor) or not isinstance(W, self.torch.Tensor) or H.dim() != 2 or W.dim() != 2:
            raise ValueError("H and W must be matrices")
        (T, d), V = H.shape, W.shape[0]
        self.need("W", W, H.dtype, (V, d))
        self.here("H", H)
        if T > 0 and d > 1 and H.stride(1) != 1:
            raise ValueError("the rows of H must be contiguous")
        ld = H.stride(0) if T > 1 else max(d, 1)
        if ld < d:
            raise ValueError("the rows of H overlap")
        return T, d, V, ld

    def scratch(self, ws):
        if not isinstance(ws, self.torch.Tensor) or not ws.is_contiguous():
            raise ValueError("ws must be a contiguous tensor")
        self.here("ws", ws)
        return ws.data_ptr(), ws.numel() * ws.element_size()

    def status(self, d_status):
        if d_status is None:
            return None
        if not isinstance(d_status, self.torch.Tensor) or d_status.dtype is not self.torch.int32 or d_status.numel() < 1:
            raise TypeError("d_status must be an int32 tensor")
        self.here("d_status", d_status)
        return d_status.data_ptr()

    def stream(self):
        raw = getattr(self.torch._C, "_cuda_getCurrentRawStream", None)      # without building a Stream object: 3 us
        return raw(self.device) if raw else self.torch.cuda.current_stream().cuda_stream


def spo_logprobs(H, W, y, mask, logp, lse, entropy, top_ids, top_logp, ws, d_status, inv_temperature=1.0):
    """Log-probabilities of the tokens y under softmax(inv_temperature * H W^T), with log-sum-exp and, where the
    tensors are given, entropy and the top_ids.shape[1] most likely alternatives.  H may be a slice of a wider buffer
    (rows contiguous); y and logp may both be None."""
    c = _Args()
    f32, i32 = c.torch.float32, c.torch.int32
    T, d, V, ld = c.rows(H, W)
    if (top_ids is None) != (top_logp is None):
        raise ValueError("top_ids and top_logp come together")
    K, row = 0, (T,)
    if top_ids is not None:
        if not isinstance(top_ids, c.torch.Tensor) or top_ids.dim() != 2:
            raise TypeError("top_ids must be a tensor [T, K]")
        K = top_ids.shape[1]
    ids, ids_logp = c.may("top_ids", top_ids, i32, (T, K)), c.may("top_logp", top_logp, f32, (T, K))
    w, n = c.scratch(ws)
    rc = lib().spo_logprobs(
        H.data_ptr(), ld, W.data_ptr(), _dtype_code(W), c.may("y", y, i32, row), c.may("mask", mask, c.torch.uint8, row), T, d, V,
        inv_temperature, K, c.may("logp", logp, f32, row), c.need("lse", lse, f32, row), c.may("entropy", entropy, f32, row),
        ids, ids_logp, w, n, c.status(d_status), c.stream())
    _check(rc, "spo_logprobs")


def spo_logprobs_bwd(H, W, y, mask, lse, entropy, g_logp, g_lse, g_entropy, dH, dW, dW_accumulate, ws, d_status,
                     inv_temperature=1.0):
    """Gradients dH, dW of spo_logprobs for upstream gradients of logp, lse and entropy (None = zero)."""
    c = _Args()
    f32 = c.torch.float32
    T, d, V, ld = c.rows(H, W)
    row = (T,)
    w, n = c.scratch(ws)
    rc = lib().spo_logprobs_bwd(
        H.data_ptr(), ld, W.data_ptr(), _dtype_code(W), c.may("y", y, c.torch.int32, row), c.may("mask", mask, c.torch.uint8, row),
        c.need("lse", lse, f32, row), c.may("entropy", entropy, f32, row), c.may("g_logp", g_logp, f32, row),
        c.may("g_lse", g_lse, f32, row), c.may("g_entropy", g_entropy, f32, row), T, d, V, inv_temperature,
        c.need("dH", dH, None, (T, d)), _dtype_code(dH), c.need("dW", dW, None, (V, d)), _dtype_code(dW), int(dW_accumulate), w, n,
        c.status(d_status), c.stream())
    _check(rc, "spo_logprobs_bwd")


def default_muon_params(**overrides) -> SpoMuonParams:
    p = SpoMuonParams()
    _check(lib().spo_default_muon_params(ctypes.byref(p)), "spo_default_muon_params")
    for k, v in overrides.items():
        setattr(p, k, v)
    return p


def _matrices(G):
    """(batch, m, n) of a matrix or a batch of them."""
    import torch
    if not isinstance(G, torch.Tensor) or G.dim() not in (2, 3):
        raise ValueError("expected a matrix [m, n] or a batch of matrices [batch, m, n]")
    return (1, *G.shape) if G.dim() == 2 else tuple(G.shape)


def spo_orthogonalize(G, out, ws, params, d_status):
    """out = the Newton-Schulz orthogonalisation of the matrix (or of each matrix of the batch) G."""
    c = _Args()
    b, m, n = _matrices(G)
    w, nb = c.scratch(ws)
    rc = lib().spo_orthogonalize(c.need("G", G, None, G.shape), _dtype_code(G), b, m, n, c.need("out", out, None, G.shape),
                                 _dtype_code(out), w, nb, ctypes.byref(params), c.status(d_status), c.stream())
    _check(rc, "spo_orthogonalize")


def spo_muon_update(W, momentum, G, ws, params, d_status):
    """One Muon step of W (in place) for the gradient G, with the fp32 momentum buffer (in place)."""
    c = _Args()
    b, m, n = _matrices(G)
    w, nb = c.scratch(ws)
    rc = lib().spo_muon_update(c.need("W", W, None, G.shape), _dtype_code(W), c.need("momentum", momentum, c.torch.float32, G.shape),
                               c.need("G", G, None, G.shape), _dtype_code(G), b, m, n, w, nb, ctypes.byref(params),
                               c.status(d_status), c.stream())
    _check(rc, "spo_muon_update")


def _hidden_rows(c, name, t):
    """(T, d, row pitch) of a matrix [T, d] whose rows are contiguous, at any pitch."""
    if not isinstance(t, c.torch.Tensor) or t.dim() != 2:
        raise ValueError("%s must be a matrix [T, d]" % name)
    c.here(name, t)
    T, d = t.shape
    if T > 0 and d > 1 and t.stride(1) != 1:
        raise ValueError("the rows of %s must be contiguous" % name)
    ld = t.stride(0) if T > 1 else max(d, 1)
    if ld < d:
        raise ValueError("the rows of %s overlap" % name)
    return T, d, ld


def _vectors(c, first, second, names, d, default):
    """(address, address, type code) of two optional vectors [d] of one type."""
    dtype = first.dtype if first is not None else second.dtype if second is not None else None
    code = default if dtype is None else DTYPE_BF16 if dtype is c.torch.bfloat16 else DTYPE_F32 if dtype is c.torch.float32 else None
    if code is None:
        raise TypeError("%s must be float32 or bfloat16, got %s" % (names[0], dtype))
    return c.may(names[0], first, dtype, (d,)), c.may(names[1], second, dtype, (d,)), code


def spo_layernorm_fwd(x, residual, weight, bias, mask, y, h, mean, rstd, d_status, eps=1e-6, kind=NORM_LAYER):
    """y = the layer norm (kind=NORM_RMS: the RMS norm) of the rows of x, or of h = x + residual where both tensors are given.  x may be
    a slice of a wider buffer (rows contiguous, the first one beginning on 16 bytes); weight, bias, mask, mean and rstd may be None."""
    c = _Args()
    f32 = c.torch.float32
    T, d, ld = _hidden_rows(c, "x", x)
    w, b, w_code = _vectors(c, weight, bias, ("weight", "bias"), d, DTYPE_F32)
    full, row = (T, d), (T,)
    rc = lib().spo_layernorm_fwd(
        x.data_ptr(), ld, c.may("residual", residual, x.dtype, full), _dtype_code(x), w, b, w_code,
        c.may("mask", mask, c.torch.uint8, row), T, d, eps, kind, c.need("y", y, None, full), _dtype_code(y),
        c.may("h", h, x.dtype, full), c.may("mean", mean, f32, row), c.may("rstd", rstd, f32, row), c.status(d_status), c.stream())
    _check(rc, "spo_layernorm_fwd")


def spo_layernorm_bwd(dy, x, weight, mask, mean, rstd, dh, dx, dw, db, dw_accumulate, ws, d_status, kind=NORM_LAYER):
    """Gradients dx, dw, db of spo_layernorm_fwd: x are the rows that were normalised (the forward's h where it had a residual), dh
    what reaches them past the norm.  weight, mask, dh, dw and db may be None, and ws where dw and db are."""
    c = _Args()
    f32 = c.torch.float32
    T, d, ld = _hidden_rows(c, "x", x)
    w, _, w_code = _vectors(c, weight, None, ("weight", ""), d, DTYPE_F32)
    pw, pb, dw_code = _vectors(c, dw, db, ("dw", "db"), d, DTYPE_F32)
    full, row = (T, d), (T,)
    scratch, n = (None, 0) if ws is None else c.scratch(ws)
    rc = lib().spo_layernorm_bwd(
        c.need("dy", dy, None, full), _dtype_code(dy), x.data_ptr(), ld, _dtype_code(x), w, w_code,
        c.may("mask", mask, c.torch.uint8, row), c.may("mean", mean, f32, row), c.need("rstd", rstd, f32, row),
        c.may("dh", dh, x.dtype, full), T, d, kind, c.need("dx", dx, x.dtype, full), pw, pb, dw_code, int(dw_accumulate), scratch, n,
        c.status(d_status), c.stream())
    _check(rc, "spo_layernorm_bwd")


class TensorList:
    """The table of one spo_grad_norm or spo_adamw_update: the addresses of tensors that stay alive with it.  Made once, used in every
    step while the tensors keep their memory.  A tensor that is given other memory (p.data = ...) needs another list: this one holds the
    memory that its addresses lie in, and goes on with that."""

    __slots__ = ("table", "address", "count", "device", "tensors", "memory")

    def __init__(self, table, device, tensors, memory):
        self.table, self.address, self.count, self.device, self.tensors = table, ctypes.addressof(table), len(tensors), device, tensors
        self.memory = [t.untyped_storage() for t in memory if t is not None]

    def here(self, c):
        if self.count and self.device != c.device:
            raise ValueError("the tensors of the list must be on the current CUDA device, are on cuda:%d" % self.device)


def _one_device(torch, tensors):
    """Checks every (name, tensor): on one CUDA device and contiguous; its number (-1: no tensors)."""
    device = -1
    for name, t in tensors:
        if not isinstance(t, torch.Tensor):
            raise TypeError("%s must be a tensor, got %s" % (name, type(t).__name__))
        if not t.is_cuda or device not in (-1, t.get_device()):
            raise ValueError("the tensors of a list must be on one CUDA device, %s is on %s" % (name, t.device))
        if not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
        device = t.get_device()
    return device


def grad_list(grads) -> TensorList:
    """The table of the gradients (contiguous fp32 or bf16 tensors of any shape) that spo_grad_norm reads."""
    import torch
    grads = list(grads)
    device = _one_device(torch, [("grads[%d]" % i, g) for i, g in enumerate(grads)])
    table = (SpoGradTensor * max(len(grads), 1))()
    for q, g in zip(table, grads):
        q.g, q.n, q.dtype = g.data_ptr(), g.numel(), _dtype_code(g)
    return TensorList(table, device, grads, grads)


def spo_grad_norm(grads, out, ws, d_status, max_norm=0.0, grad_scale=1.0):
    """out[0] = the norm of all gradients of the list (times |grad_scale|), out[1] = the factor that clips them to max_norm (0: no
    clipping) and scales them, out[2] = 1 where the norm is finite."""
    c = _Args()
    grads.here(c)
    w, n = c.scratch(ws)
    rc = lib().spo_grad_norm(grads.address, grads.count, max_norm, grad_scale, c.need("out", out, c.torch.float32, (4,)), w, n,
                             c.status(d_status), c.stream())
    _check(rc, "spo_grad_norm")


def default_adamw_params(**overrides) -> SpoAdamwParams:
    p = SpoAdamwParams()
    _check(lib().spo_default_adamw_params(ctypes.byref(p)), "spo_default_adamw_params")
    for k, v in overrides.items():
        setattr(p, k, v)
    return p


def adamw_list(weights, grads, m, v, m_scale=None, v_scale=None, copies=None, lr_scale=None, decay_scale=None) -> TensorList:
    """The table of one spo_adamw_update: lists of tensors, one entry for each weight.  States are fp32 (32 bits) or int8 / uint8
    (8 bits, with scales of ceil(n / ADAMW_BLOCK) fp32 elements; None for a 32-bit entry); copies are bf16 or None; lr_scale and
    decay_scale are numbers (default 1)."""
    import torch
    weights = list(weights)
    k = len(weights)
    f32, bf16 = torch.float32, torch.bfloat16

    def column(name, values, fill=None):
        values = [fill] * k if values is None else list(values)
        if len(values) != k:
            raise ValueError("%s has %d entries for %d weights" % (name, len(values), k))
        return values

    columns = [("weights", weights)] + [(name, column(name, x)) for name, x in (
        ("grads", list(grads)), ("m", list(m)), ("v", list(v)), ("m_scale", m_scale), ("v_scale", v_scale), ("copies", copies))]
    rates, decays = column("lr_scale", lr_scale, 1.0), column("decay_scale", decay_scale, 1.0)
    device = _one_device(torch, [("%s[%d]" % (name, i), t) for name, x in columns for i, t in enumerate(x)
                                 if t is not None or name in ("weights", "grads", "m", "v")])
    table = (SpoAdamwTensor * max(k, 1))()
    spans = []                                      # (first byte, byte behind the last, written)

    def cover(t, written):
        if t is not None and t.numel():
            spans.append((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), written))
        return None if t is None else t.data_ptr()

    for i, (w, g, mi, vi, ms, vs, copy) in enumerate(zip(*[x for _, x in columns])):
        n, q = w.numel(), table[i]
        if g.shape != w.shape:
            raise ValueError("grads[%d] must have shape %s, got %s" % (i, tuple(w.shape), tuple(g.shape)))
        for name, t in (("m", mi), ("v", vi), ("copies", copy)):
            if t is not None and t.numel() != n:
                raise ValueError("%s[%d] must have %d elements, has %d" % (name, i, n, t.numel()))
        if (mi.dtype, vi.dtype) == (f32, f32):
            q.state_bits = 32
            if ms is not None or vs is not None:
                raise ValueError("m_scale[%d] and v_scale[%d] belong to 8-bit states" % (i, i))
        elif (mi.dtype, vi.dtype) == (torch.int8, torch.uint8):
            q.state_bits = 8
            for name, t in (("m_scale", ms), ("v_scale", vs)):
                if t is None or t.dtype != f32 or t.numel() != -(-n // ADAMW_BLOCK):
                    raise ValueError("%s[%d] must be a float32 tensor of %d elements" % (name, i, -(-n // ADAMW_BLOCK)))
        else:
            raise TypeError("m[%d] and v[%d] must be float32, or int8 and uint8" % (i, i))
        if copy is not None and copy.dtype != bf16:
            raise TypeError("copies[%d] must be bfloat16" % i)
        q.w, q.g, q.m, q.v = cover(w, True), cover(g, False), cover(mi, True), cover(vi, True)
        q.m_scale, q.v_scale, q.copy = cover(ms, True), cover(vs, True), cover(copy, True)
        q.n, q.w_dtype, q.g_dtype = n, _dtype_code(w), _dtype_code(g)
        q.lr_scale, q.decay_scale = rates[i], decays[i]
    read = written = 0
    for begin, end, out in sorted(spans):
        if begin < written or (out and begin < read):
            raise ValueError("tensors of the list share memory that is written (the same tensor twice?)")
        read, written = max(read, end), max(written, end if out else 0)
    return TensorList(table, device, list(zip(*[x for _, x in columns])), [t for _, x in columns for t in x])


def spo_adamw_update(tensors, d_scale, d_step, d_lr, params, d_status):
    """One AdamW step over the tensors of the list: weights, states and copies in place.  d_scale [1] (spo_grad_norm's out[1:2]) multiplies
    the gradients; d_step [2] int32 counts the steps on the device (None: params.step is the step); d_lr [1] replaces params.lr."""
    c = _Args()
    f32 = c.torch.float32
    tensors.here(c)
    rc = lib().spo_adamw_update(tensors.address, tensors.count, c.may("d_scale", d_scale, f32, (1,)), c.may("d_lr", d_lr, f32, (1,)),
                                c.may("d_step", d_step, c.torch.int32, (2,)), ctypes.byref(params), c.status(d_status), c.stream())
    _check(rc, "spo_adamw_update")


def spo_adamw_decode(m, m_scale, v, v_scale, m_out, v_out):
    """The fp32 values of 8-bit states; m, m_scale and m_out, or v, v_scale and v_out, may be None together."""
    c = _Args()
    t = m if m is not None else v
    if not isinstance(t, c.torch.Tensor):
        raise TypeError("m or v must be a tensor")
    f32, shape, blocks = c.torch.float32, t.shape, (-(-t.numel() // ADAMW_BLOCK),)
    if (m is None) != (m_out is None) or (v is None) != (v_out is None):
        raise ValueError("m and m_out, v and v_out come together")
    rc = lib().spo_adamw_decode(
        c.may("m", m, c.torch.int8, shape), None if m is None else c.need("m_scale", m_scale, f32, blocks),
        c.may("v", v, c.torch.uint8, shape), None if v is None else c.need("v_scale", v_scale, f32, blocks), t.numel(),
        c.may("m_out", m_out, f32, shape), c.may("v_out", v_out, f32, shape), c.stream())
    _check(rc, "spo_adamw_decode")
