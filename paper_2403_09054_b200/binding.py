"""Thin ctypes binding of the C ABI declared in ``include/keyformer.h``.

Argument marshalling only (for the operators that need no context in the compiled ``_kf_torch``): every step of the path runs
in the CUDA kernels of ``libkeyformer_b200.so``.  PyTorch supplies device memory and streams.  There is
no fallback: if the library cannot be loaded, importing this module fails.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os

import numpy as np
import torch

from . import build as _build

KF_OK, KF_EINVAL, KF_ENOSPC, KF_ESTATE, KF_ECUDA, KF_ETIMEOUT, KF_EBOUNDS = 0, -1, -2, -3, -4, -5, -6
KF_NOISE_GUMBEL, KF_NOISE_NONE, KF_NOISE_CONST, KF_NOISE_GAUSS = 0, 1, 2, 3
KF_BIAS_NONE, KF_BIAS_ALIBI = 0, 1
KF_PREFILL_TENSOR, KF_PREFILL_SIMT = 0, 1
KF_POS_ORIGINAL, KF_POS_NEW = 0, 1
KF_DECODE_AUTO, KF_DECODE_CUDA_CORES, KF_DECODE_TENSOR = 0, 1, 2
KF_TYPE_FP16, KF_TYPE_BF16, KF_TYPE_FP32 = 0, 1, 2
KF_NORM_NONE, KF_NORM_RMS = 0, 1
KF_ROTARY_PAIRS, KF_ROTARY_HALVES = 0, 1

EXPORTS = ("kf_workspace_bytes", "kf_create", "kf_prefill_score_prune", "kf_decode_step",
           "kf_decode_step_host", "kf_view_state", "kf_poll_error", "kf_launch_count",
           "kf_destroy", "kf_strerror", "kf_decode_step_static", "kf_state_bytes", "kf_export_state", "kf_import_state",
           "kf_prefill_attend", "kf_prefill_attend_score_prune", "kf_view_place", "kf_compact_layer", "kf_check_canaries", "kf_describe_decode",
           "kf_packed_slot_bytes", "kf_pack_cache", "kf_unpack_cache", "kf_packed_scratch_bytes", "kf_decode_step_packed",
           "kf_qk_norm_rotate", "kf_beam_scratch_bytes", "kf_beam_select", "kf_reorder_rows", "kf_reorder_beams",
           "kf_prefill_attend_ragged", "kf_pages_write", "kf_pages_read", "kf_pages_attend_scratch_bytes", "kf_pages_attend",
           "kf_pages_update_scratch_bytes", "kf_pages_update", "kf_pages_compact")


class kf_config(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32), ("batch", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
        ("budget_k", C.c_int32), ("recent_w", C.c_int32), ("max_prompt_len", C.c_int32), ("gen_len_T", C.c_int32),
        ("tau_init", C.c_float), ("tau_end", C.c_float), ("noise_seed", C.c_uint64),
        ("noise_mode", C.c_int32), ("bias_mode", C.c_int32), ("h_alibi_slopes", C.POINTER(C.c_float)),
        ("logit_scale", C.c_float), ("noise_const", C.c_float),
        ("decode_splits", C.c_int32), ("prefill_impl", C.c_int32),
        ("noise_mu", C.c_float), ("noise_sigma", C.c_float), ("pos_mode", C.c_int32),
        ("n_kv_heads", C.c_int32), ("rotary_dims", C.c_int32), ("rotary_base", C.c_float), ("decode_impl", C.c_int32), ("debug_canaries", C.c_int32), ("debug_fail_first_wait", C.c_int32),
    ]


class kf_static_step(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
        ("budget_k", C.c_int32), ("recent_w", C.c_int32), ("layer", C.c_int32), ("position", C.c_int32),
        ("noise_mode", C.c_int32), ("bias_mode", C.c_int32), ("reserved", C.c_int32),
        ("tau", C.c_double), ("noise_seed", C.c_uint64), ("logit_scale", C.c_float), ("noise_const", C.c_float),
        ("d_alibi_slopes", C.c_void_p),
    ]


KF_STATIC_SCRATCH_BYTES = 16 << 20


class kf_packed_step(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("budget_k", C.c_int32), ("recent_w", C.c_int32), ("layer", C.c_int32), ("position", C.c_int32),
        ("noise_mode", C.c_int32), ("bias_mode", C.c_int32), ("tau", C.c_double), ("noise_seed", C.c_uint64),
        ("logit_scale", C.c_float), ("noise_const", C.c_float), ("noise_mu", C.c_float), ("noise_sigma", C.c_float),
        ("d_alibi_slopes", C.c_void_p), ("debug_fail_first_wait", C.c_int32),
    ]


class kf_qk_norm_args(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("n_tokens", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("input_type", C.c_int32), ("batch_stride", C.c_int64), ("token_stride", C.c_int64),
        ("norm_mode", C.c_int32), ("eps", C.c_float), ("rotary_dims", C.c_int32), ("rotary_style", C.c_int32),
        ("rotary_base", C.c_float), ("position0", C.c_int32),
    ]


class kf_beam_args(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("beams", C.c_int32), ("vocab", C.c_int32), ("take", C.c_int32),
        ("logits_type", C.c_int32), ("pad_token", C.c_int32), ("row_stride", C.c_int64),
    ]


class kf_row_buffer(C.Structure):
    _fields_ = [("d_base", C.c_void_p), ("row_bytes", C.c_int64), ("outer_stride", C.c_int64), ("outer", C.c_int32)]


class kf_ragged_args(C.Structure):
    _fields_ = [
        ("tokens", C.c_int32), ("sequences", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("type", C.c_int32), ("bias_mode", C.c_int32), ("logit_scale", C.c_float), ("d_alibi_slopes", C.c_void_p),
        ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64), ("k_token_stride", C.c_int64), ("k_head_stride", C.c_int64),
        ("v_token_stride", C.c_int64), ("v_head_stride", C.c_int64), ("out_token_stride", C.c_int64), ("out_head_stride", C.c_int64),
        ("debug_fail_first_wait", C.c_int32), ("debug_fail_after", C.c_int32),
    ]


class kf_page_cache(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("page_tokens", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("sequences", C.c_int32),
                ("table_width", C.c_int32)]


class kf_page_rows(C.Structure):
    _fields_ = [("tokens", C.c_int32), ("type", C.c_int32), ("k_token_stride", C.c_int64), ("k_head_stride", C.c_int64), ("v_token_stride", C.c_int64),
                ("v_head_stride", C.c_int64)]


class kf_pages_attend_args(C.Structure):
    _fields_ = [
        ("cache", kf_page_cache), ("n_heads", C.c_int32), ("type", C.c_int32), ("bias_mode", C.c_int32), ("logit_scale", C.c_float),
        ("d_alibi_slopes", C.c_void_p), ("q_sequence_stride", C.c_int64), ("q_head_stride", C.c_int64), ("out_sequence_stride", C.c_int64),
        ("out_head_stride", C.c_int64), ("debug_fail_first_wait", C.c_int32), ("debug_fail_after", C.c_int32),
    ]


class kf_pages_update_args(C.Structure):
    _fields_ = [("cache", kf_page_cache), ("n_layers", C.c_int32), ("grow", C.c_int32)]


def _load() -> C.CDLL:
    path = _build.LIB
    if not os.path.exists(path):
        path = _build.build()
    lib = C.CDLL(path)
    vp, i32 = C.c_void_p, C.c_int32
    cfgp = C.POINTER(kf_config)
    lib.kf_workspace_bytes.restype = C.c_size_t
    lib.kf_workspace_bytes.argtypes = [cfgp]
    lib.kf_create.restype = C.c_int
    lib.kf_create.argtypes = [cfgp, vp, C.c_size_t, vp, C.POINTER(vp)]
    lib.kf_prefill_score_prune.restype = C.c_int
    lib.kf_prefill_score_prune.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp]
    lib.kf_prefill_attend.restype = C.c_int
    lib.kf_prefill_attend.argtypes = [vp, i32, vp, vp, vp, vp, vp]
    lib.kf_prefill_attend_score_prune.restype = C.c_int
    lib.kf_prefill_attend_score_prune.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.kf_decode_step.restype = C.c_int
    lib.kf_decode_step.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.kf_decode_step_host.restype = C.c_int
    lib.kf_decode_step_host.argtypes = [vp, i32, i32, vp, vp, vp, vp, i32, vp]
    lib.kf_decode_step_static.restype = C.c_int
    lib.kf_decode_step_static.argtypes = [C.POINTER(kf_static_step)] + [vp] * 11
    lib.kf_state_bytes.restype = C.c_size_t
    lib.kf_state_bytes.argtypes = [vp]
    lib.kf_export_state.restype = C.c_int
    lib.kf_export_state.argtypes = [vp, i32, vp, C.c_size_t, C.POINTER(i32), C.POINTER(i32), vp]
    lib.kf_import_state.restype = C.c_int
    lib.kf_import_state.argtypes = [vp, i32, vp, C.c_size_t, i32, i32, vp]
    lib.kf_compact_layer.restype = C.c_int
    lib.kf_compact_layer.argtypes = [vp, i32, vp]
    lib.kf_view_place.restype = C.c_int
    lib.kf_view_place.argtypes = [vp, i32, C.POINTER(vp)]
    lib.kf_view_state.restype = C.c_int
    lib.kf_view_state.argtypes = [vp, i32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp)]
    lib.kf_poll_error.restype = C.c_int
    lib.kf_poll_error.argtypes = [vp, vp]
    lib.kf_check_canaries.restype = C.c_int
    lib.kf_check_canaries.argtypes = [vp, vp, C.POINTER(i32)]
    lib.kf_describe_decode.restype = C.c_int
    lib.kf_describe_decode.argtypes = [vp, C.c_char_p, C.c_size_t]
    lib.kf_launch_count.restype = C.c_int64
    lib.kf_launch_count.argtypes = [vp]
    i64, szt = C.c_int64, C.c_size_t
    lib.kf_packed_slot_bytes.restype = i32
    lib.kf_packed_slot_bytes.argtypes = [i32]
    lib.kf_pack_cache.restype = lib.kf_unpack_cache.restype = C.c_int
    lib.kf_pack_cache.argtypes = lib.kf_unpack_cache.argtypes = [i64, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.kf_packed_scratch_bytes.restype = szt
    lib.kf_packed_scratch_bytes.argtypes = [C.POINTER(kf_packed_step)]
    lib.kf_decode_step_packed.restype = C.c_int
    lib.kf_decode_step_packed.argtypes = [C.POINTER(kf_packed_step)] + [vp] * 12 + [szt, vp]
    lib.kf_qk_norm_rotate.restype = C.c_int
    lib.kf_qk_norm_rotate.argtypes = [C.POINTER(kf_qk_norm_args)] + [vp] * 8
    lib.kf_beam_scratch_bytes.restype = szt
    lib.kf_beam_scratch_bytes.argtypes = [C.POINTER(kf_beam_args)]
    lib.kf_beam_select.restype = C.c_int
    lib.kf_beam_select.argtypes = [C.POINTER(kf_beam_args)] + [vp] * 7 + [szt, vp]
    lib.kf_reorder_rows.restype = C.c_int
    lib.kf_reorder_rows.argtypes = [C.POINTER(kf_row_buffer), i32, i32, i32, vp, vp]
    lib.kf_reorder_beams.restype = C.c_int
    lib.kf_reorder_beams.argtypes = [vp, i32, i32, vp, vp]
    cache = C.POINTER(kf_page_cache)
    lib.kf_prefill_attend_ragged.restype = C.c_int
    lib.kf_prefill_attend_ragged.argtypes = [C.POINTER(kf_ragged_args)] + [vp] * 6
    lib.kf_pages_write.restype = lib.kf_pages_read.restype = C.c_int
    lib.kf_pages_write.argtypes = lib.kf_pages_read.argtypes = [cache, C.POINTER(kf_page_rows)] + [vp] * 8
    lib.kf_pages_attend_scratch_bytes.restype = lib.kf_pages_update_scratch_bytes.restype = szt
    lib.kf_pages_attend_scratch_bytes.argtypes = [C.POINTER(kf_pages_attend_args)]
    lib.kf_pages_attend.restype = C.c_int
    lib.kf_pages_attend.argtypes = [C.POINTER(kf_pages_attend_args)] + [vp] * 7 + [szt, vp]
    lib.kf_pages_update_scratch_bytes.argtypes = [C.POINTER(kf_pages_update_args)]
    lib.kf_pages_update.restype = C.c_int
    lib.kf_pages_update.argtypes = [C.POINTER(kf_pages_update_args)] + [vp] * 9 + [szt, vp]
    lib.kf_pages_compact.restype = C.c_int
    lib.kf_pages_compact.argtypes = [cache, i32, i32] + [vp] * 8
    lib.kf_destroy.restype = C.c_int
    lib.kf_destroy.argtypes = [vp]
    lib.kf_strerror.restype = C.c_char_p
    lib.kf_strerror.argtypes = [C.c_int]
    return lib


LIB = _load()
LIB_PATH = _build.LIB


class _TorchSide:
    """Stands for the compiled extension until a call first needs it: the context's calls go through ctypes alone and do not depend on it."""

    def __getattr__(self, name):
        global _kf_torch
        path = _build.torch_lib()
        if not os.path.exists(path):
            _build.build_torch()
        spec = importlib.util.spec_from_file_location("_kf_torch", path)      # links against the library loaded above
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        _kf_torch = module
        return getattr(module, name)


_kf_torch = _TorchSide()


class KeyformerError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {LIB.kf_strerror(code).decode()} ({code})")


def _check(code: int, where: str) -> None:
    if code != KF_OK:
        raise KeyformerError(code, where)


def kf_strerror(code: int) -> str:
    return LIB.kf_strerror(code).decode()


def make_config(*, n_layers, batch, n_heads, head_dim, budget_k, recent_w, max_prompt_len, gen_len_T,
                tau_init=1.0, tau_end=2.0, noise_seed=0, noise_mode=KF_NOISE_GUMBEL, bias_mode=KF_BIAS_NONE,
                alibi_slopes=None, logit_scale=0.0, noise_const=0.5772, decode_splits=0,
                prefill_impl=KF_PREFILL_TENSOR, noise_mu=0.5772, noise_sigma=1.2825, pos_mode=KF_POS_ORIGINAL,
                n_kv_heads=0, rotary_dims=0, rotary_base=10000.0, decode_impl=0, debug_canaries=0, debug_fail_first_wait=0):
    """Fill a kf_config; returns (config, keepalive) where keepalive holds the slopes array."""
    cfg = kf_config()
    cfg.n_layers, cfg.batch, cfg.n_heads, cfg.head_dim = n_layers, batch, n_heads, head_dim
    cfg.budget_k, cfg.recent_w, cfg.max_prompt_len, cfg.gen_len_T = budget_k, recent_w, max_prompt_len, gen_len_T
    cfg.tau_init, cfg.tau_end = tau_init, tau_end
    cfg.noise_seed = noise_seed & 0xFFFFFFFFFFFFFFFF
    cfg.noise_mode, cfg.bias_mode = noise_mode, bias_mode
    keep = None
    if alibi_slopes is not None:
        keep = np.ascontiguousarray(alibi_slopes, dtype=np.float32)
        cfg.h_alibi_slopes = keep.ctypes.data_as(C.POINTER(C.c_float))
    cfg.logit_scale, cfg.noise_const = logit_scale, noise_const
    cfg.decode_splits, cfg.prefill_impl = decode_splits, prefill_impl
    cfg.noise_mu, cfg.noise_sigma = noise_mu, noise_sigma
    cfg.pos_mode = pos_mode
    cfg.n_kv_heads, cfg.decode_impl = n_kv_heads, decode_impl
    cfg.rotary_dims, cfg.rotary_base = rotary_dims, rotary_base
    cfg.debug_canaries, cfg.debug_fail_first_wait = debug_canaries, debug_fail_first_wait
    return cfg, keep


def kf_workspace_bytes(cfg: kf_config) -> int:
    return int(LIB.kf_workspace_bytes(C.byref(cfg)))


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _dev_ptr(t, dtype, numel, name):
    if t is None:
        return None
    if not (t.is_cuda and t.is_contiguous() and t.dtype == dtype and t.numel() == numel):
        raise ValueError(f"{name}: expected a contiguous CUDA {dtype} tensor with {numel} elements, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def kf_decode_step_static(*, batch, n_heads, head_dim, budget_k, recent_w, layer, position, tau,
                          K, V, pos, acc, length, q, knew, vnew, out, score_out=None, noise_seed=0,
                          noise_mode=KF_NOISE_GUMBEL, noise_const=0.5772, bias_mode=KF_BIAS_NONE,
                          alibi_slopes_dev=None, logit_scale=0.0, stream=None) -> int:
    """One generation step on caller-held cache tensors, using the library's built-in scratch block
    (for callers that cannot allocate device memory).  Returns the KF_* status code."""
    a = kf_static_step()
    a.batch, a.n_heads, a.head_dim, a.budget_k, a.recent_w = batch, n_heads, head_dim, budget_k, recent_w
    a.layer, a.position, a.noise_mode, a.bias_mode, a.reserved = layer, position, noise_mode, bias_mode, 0
    a.tau, a.noise_seed, a.logit_scale, a.noise_const = tau, noise_seed & 0xFFFFFFFFFFFFFFFF, logit_scale, noise_const
    a.d_alibi_slopes = None if alibi_slopes_dev is None else alibi_slopes_dev.data_ptr()
    U = batch * n_heads
    return int(LIB.kf_decode_step_static(
        C.byref(a),
        _dev_ptr(K, torch.float16, U * budget_k * head_dim, "K"), _dev_ptr(V, torch.float16, U * budget_k * head_dim, "V"),
        _dev_ptr(pos, torch.int32, U * budget_k, "pos"), _dev_ptr(acc, torch.float32, U * budget_k, "acc"),
        _dev_ptr(length, torch.int32, U, "length"),
        _dev_ptr(q, torch.float16, U * head_dim, "q"), _dev_ptr(knew, torch.float16, U * head_dim, "knew"),
        _dev_ptr(vnew, torch.float16, U * head_dim, "vnew"), _dev_ptr(out, torch.float16, U * head_dim, "out"),
        _dev_ptr(score_out, torch.float32, U * (budget_k + 1), "score_out"), _stream_ptr(stream)))


# ---- operators that need no context.  Tensors of a call live on one CUDA device, which need not be the current one; work goes
# to `stream`, or to that device's current stream.  The calls' tensors are checked in the compiled _kf_torch (ValueError).
def kf_packed_slot_bytes(head_dim) -> int:
    return int(LIB.kf_packed_slot_bytes(head_dim))


def kf_pack_cache(*, K, V, cache, length=None, stream=None):
    """Rows K, V (fp16 [..., n, d]) to slots 0 .. n-1 of the 4-bit cache (uint8 [..., k, 5d/4]); with `length` (int32 [...])
    only the rows below it."""
    _check(_kf_torch.pack_cache(K, V, cache, length, stream), "kf_pack_cache")


def kf_unpack_cache(*, cache, K, V, length=None, stream=None):
    """Slots 0 .. n-1 of a 4-bit cache back to rows K, V (fp16 [..., n, d]): the values that the codes stand for."""
    _check(_kf_torch.unpack_cache(K, V, cache, length, stream), "kf_unpack_cache")


def kf_packed_scratch_bytes(*, batch, n_heads, head_dim, budget_k, n_kv_heads=0) -> int:
    """Bytes of scratch a kf_decode_step_packed of this shape needs; 0 if the shape is not supported."""
    a = kf_packed_step(batch=batch, n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, budget_k=budget_k, noise_mode=KF_NOISE_NONE, tau=1.0)
    return int(LIB.kf_packed_scratch_bytes(C.byref(a)))


def kf_decode_step_packed(*, batch, n_heads, head_dim, budget_k, recent_w, layer, position, tau, cache, pos, acc, length,
                          q, knew, vnew, out, n_kv_heads=0, score_out=None, slot_out=None, row_out=None, noise_seed=0,
                          noise_mode=KF_NOISE_GUMBEL, noise_const=0.5772, noise_mu=0.5772, noise_sigma=1.2825,
                          bias_mode=KF_BIAS_NONE, alibi_slopes_dev=None, logit_scale=0.0, scratch=None, stream=None):
    """One generation step over a cache in 4 bits (kf_pack_cache), all state in the caller's tensors.  `scratch`: a uint8 CUDA tensor of
    kf_packed_scratch_bytes(...) bytes; without one torch's allocator provides it for the call."""
    _check(_kf_torch.decode_step_packed(batch, n_heads, n_kv_heads, head_dim, budget_k, recent_w, layer, position, noise_mode, bias_mode, tau, noise_seed,
                                        logit_scale, noise_const, noise_mu, noise_sigma, alibi_slopes_dev, cache, pos, acc, length, q, knew, vnew, out,
                                        score_out, slot_out, row_out, scratch, stream), "kf_decode_step_packed")


def kf_qk_norm_rotate(*, qkv, n_heads, n_kv_heads, head_dim, q, k, v=None, positions=None, position0=0, norm_mode=KF_NORM_NONE,
                      q_weight=None, k_weight=None, eps=1e-6, rotary_dims=0, rotary_base=10000.0, rotary_style=KF_ROTARY_PAIRS, stream=None):
    """Projection rows (fp16 or bf16 [B, n, (H + 2 Hkv) d], any batch and token stride) to normed and rotated head-major q, k and to v
    (fp16 [B, H, n, d], [B, Hkv, n, d]; for n = 1 also without that dimension)."""
    _check(_kf_torch.qk_norm_rotate(qkv, n_heads, n_kv_heads, head_dim, q, k, v, positions, position0, norm_mode, q_weight, k_weight, eps, rotary_dims,
                                    rotary_base, rotary_style, stream), "kf_qk_norm_rotate")


def kf_beam_select(*, logits, scores, out_scores, out_parent, out_token, finished=None, pad_token=0, scratch=None, stream=None):
    """The best continuations over beams and vocabulary: logits (fp16, bf16 or fp32 [B, beams, V], rows evenly spaced), scores
    (fp32 [B, beams]); out_* [B, take], best first.  `finished`: uint8 or bool [B, beams], beams that go on with pad_token alone."""
    _check(_kf_torch.beam_select(logits, scores, out_scores, out_parent, out_token, finished, pad_token, scratch, stream), "kf_beam_select")


def kf_reorder_rows(*, buffers, parent, n_layers=1, stream=None):
    """In every tensor of `buffers` (contiguous [batch * beams, ...], or [n_layers, batch * beams, ...]) row (b, i) becomes what row
    (b, parent[b, i]) was, in place; parent: int32 [batch, beams]."""
    _check(_kf_torch.reorder_rows(buffers, parent, n_layers, stream), "kf_reorder_rows")


def _fits32(*sizes) -> bool:
    """Whether sizes keep their values in the int32 fields of an argument struct (ctypes would drop the upper bits)."""
    return all(0 <= n < 2 ** 31 for n in sizes)


def kf_prefill_attend_ragged(*, q, k, v, begin, out, bias_mode=KF_BIAS_NONE, alibi_slopes_dev=None, logit_scale=0.0, debug_fail_first_wait=0, debug_fail_after=0,
                             stream=None):
    """Causal attention over prompts that lie one after the other: sequence s has rows begin[s] .. begin[s + 1] - 1 (int32 [S + 1]) of q, out
    [T, H, d] and k, v [T, Hkv, d] (fp16 or bf16, contiguous features, any strides of tokens and heads: views of a projection's rows, or
    ``x[0].transpose(0, 1)`` of kf_qk_norm_rotate's head-major rows).  A prompt sees its own rows only.  T is at least 1."""
    _check(_kf_torch.attend_ragged(q, k, v, begin, out, bias_mode, alibi_slopes_dev, logit_scale, debug_fail_first_wait, debug_fail_after, stream),
           "kf_prefill_attend_ragged")


def kf_pages_write(*, k, v, length, table, cache, scale, begin=None, stream=None):
    """Rows begin[s] .. begin[s + 1] - 1 of k, v [T, Hkv, d] (without `begin` row s) become tokens length[s], ... of sequence s in the 8-bit pages
    of cache (int8 [pages, Hkv, 2, page, d]) and scale (fp32 [pages, Hkv, 2]) that table (int32 [S, width]) names.  `length` is left as it is."""
    _check(_kf_torch.pages_write(k, v, begin, length, table, cache, scale, stream), "kf_pages_write")


def kf_pages_read(*, table, cache, scale, k, v, begin, first=None, stream=None):
    """Tokens first[s] (0), ... of every sequence as the values that their codes stand for: rows begin[s] .. of k, v [T, Hkv, d]."""
    _check(_kf_torch.pages_read(k, v, begin, first, table, cache, scale, stream), "kf_pages_read")


def kf_pages_attend(*, q, table, length, cache, scale, out, bias_mode=KF_BIAS_NONE, alibi_slopes_dev=None, logit_scale=0.0, debug_fail_first_wait=0,
                    debug_fail_after=0, scratch=None, stream=None):
    """One query token per sequence, q and out [S, H, d], over the length[s] tokens of its pages.  `scratch`: a uint8 CUDA tensor of
    kf_pages_attend_scratch_bytes(...) bytes; without one torch's allocator provides it for the call."""
    _check(_kf_torch.pages_attend(q, table, length, cache, scale, out, bias_mode, alibi_slopes_dev, logit_scale, debug_fail_first_wait, debug_fail_after,
                                  scratch, stream), "kf_pages_attend")


def kf_pages_attend_scratch_bytes(*, sequences, table_width, n_pages, page_tokens, n_heads, n_kv_heads, head_dim) -> int:
    """Bytes of scratch a kf_pages_attend of this shape needs; 0 if the shape is not supported."""
    if not _fits32(sequences, table_width, n_pages, page_tokens, n_heads, n_kv_heads, head_dim):
        return 0
    a = kf_pages_attend_args(cache=kf_page_cache(n_pages, page_tokens, n_kv_heads, head_dim, sequences, table_width), n_heads=n_heads)
    a.q_head_stride = a.out_head_stride = head_dim
    a.q_sequence_stride = a.out_sequence_stride = head_dim * n_heads
    return int(LIB.kf_pages_attend_scratch_bytes(C.byref(a)))


def kf_pages_update(*, table, length, refs, cache, scale, missing, parent=None, grow=0, scratch=None, stream=None):
    """Sequences forked (sequence s goes on from parent[s], int32 [S]; -1: it has ended), part-filled pages copied in all layers (cache
    [layers, pages, ...] or [pages, ...]), pages given back, and room made for grow (a number or int32 [S]) more tokens; table, length, refs (int32 [pages]) in
    place, `missing` (int32 [1]): pages there were none for.  `scratch`: a uint8 CUDA tensor of kf_pages_update_scratch_bytes(...) bytes."""
    _check(_kf_torch.pages_update(table, length, refs, cache, scale, parent, grow, missing, scratch, stream), "kf_pages_update")


def kf_pages_update_scratch_bytes(*, sequences, table_width, n_pages, page_tokens, n_kv_heads, head_dim, n_layers=1) -> int:
    """Bytes of scratch a kf_pages_update of this shape needs; 0 if the shape is not supported."""
    if not _fits32(sequences, table_width, n_pages, page_tokens, n_kv_heads, head_dim, n_layers):
        return 0
    a = kf_pages_update_args(cache=kf_page_cache(n_pages, page_tokens, n_kv_heads, head_dim, sequences, table_width), n_layers=n_layers)
    return int(LIB.kf_pages_update_scratch_bytes(C.byref(a)))


def kf_pages_compact(*, cache, scale, table, length, keep, n_keep, new_table, stream=None):
    """Row j < n_keep[s] of (s, head) in the pages of new_table becomes token keep[s, head, j] (int32 [S, Hkv, width]) in those of table.  Places in the new pages are
    not positions in the text: ALiBi then counts kept rows, and what is rotated later keeps its own count of positions."""
    _check(_kf_torch.pages_compact(cache, scale, table, length, keep, n_keep, new_table, stream), "kf_pages_compact")


class Keyformer:
    """A context (kf_create .. kf_destroy) over a torch-allocated workspace."""

    def __init__(self, device="cuda:0", stream=None, **cfg_kwargs):
        if not torch.cuda.is_available():
            raise KeyformerError(KF_ECUDA, "Keyformer(): no CUDA device (the library has no CPU path)")
        self.device = torch.device(device)
        self.cfg, self._keep = make_config(**cfg_kwargs)
        nbytes = kf_workspace_bytes(self.cfg)
        if nbytes == 0:
            raise KeyformerError(KF_EINVAL, "kf_workspace_bytes")
        self.workspace_bytes = nbytes
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            base = self.workspace.data_ptr()
            self._ws_ptr = (base + 255) // 256 * 256
            h = C.c_void_p()
            _check(LIB.kf_create(C.byref(self.cfg), self._ws_ptr, nbytes, _stream_ptr(stream), C.byref(h)), "kf_create")
        self._h = h
        self.kv_heads = self.cfg.n_kv_heads if self.cfg.n_kv_heads > 0 else self.cfg.n_heads
        self.units_q = self.cfg.batch * self.cfg.n_heads       # (batch row, query head) pairs
        self.units = self.cfg.batch * self.kv_heads            # caches per layer: (batch row, key/value head) pairs

    # ---- the C calls, same names ---------------------------------------------------------
    def kf_prefill_score_prune(self, layer, q, k, v, score_out=None, stream=None):
        d = self.cfg.head_dim
        n = q.shape[-2]
        _check(LIB.kf_prefill_score_prune(
            self._h, layer, n,
            _dev_ptr(q, torch.float16, self.units_q * n * d, "q"), _dev_ptr(k, torch.float16, self.units * n * d, "k"),
            _dev_ptr(v, torch.float16, self.units * n * d, "v"),
            _dev_ptr(score_out, torch.float32, self.units * n, "score_out"), _stream_ptr(stream)),
            "kf_prefill_score_prune")

    def kf_prefill_attend(self, q, k, v, out, stream=None):
        d = self.cfg.head_dim
        n = q.shape[-2]
        _check(LIB.kf_prefill_attend(
            self._h, n, _dev_ptr(q, torch.float16, self.units_q * n * d, "q"), _dev_ptr(k, torch.float16, self.units * n * d, "k"),
            _dev_ptr(v, torch.float16, self.units * n * d, "v"), _dev_ptr(out, torch.float16, self.units_q * n * d, "out"),
            _stream_ptr(stream)), "kf_prefill_attend")

    def kf_prefill_attend_score_prune(self, layer, q, k, v, out, score_out=None, stream=None):
        d = self.cfg.head_dim
        n = q.shape[-2]
        _check(LIB.kf_prefill_attend_score_prune(
            self._h, layer, n, _dev_ptr(q, torch.float16, self.units_q * n * d, "q"),
            _dev_ptr(k, torch.float16, self.units * n * d, "k"), _dev_ptr(v, torch.float16, self.units * n * d, "v"),
            _dev_ptr(out, torch.float16, self.units_q * n * d, "out"),
            _dev_ptr(score_out, torch.float32, self.units * n, "score_out"), _stream_ptr(stream)),
            "kf_prefill_attend_score_prune")

    def kf_decode_step(self, layer, step, q, knew, vnew, out, score_out=None, stream=None):
        d = self.cfg.head_dim
        _check(LIB.kf_decode_step(
            self._h, layer, step,
            _dev_ptr(q, torch.float16, self.units_q * d, "q"), _dev_ptr(knew, torch.float16, self.units * d, "knew"),
            _dev_ptr(vnew, torch.float16, self.units * d, "vnew"), _dev_ptr(out, torch.float16, self.units_q * d, "out"),
            _dev_ptr(score_out, torch.float32, self.units * (self.cfg.budget_k + 1), "score_out"),
            _stream_ptr(stream)), "kf_decode_step")

    def kf_decode_step_host(self, layer, step, q, knew, vnew, out, wait=True, stream=None):
        d = self.cfg.head_dim
        for name, t, numel in (("q", q, self.units_q * d), ("knew", knew, self.units * d), ("vnew", vnew, self.units * d),
                               ("out", out, self.units_q * d)):
            if t.is_cuda or not t.is_contiguous() or t.dtype != torch.float16 or t.numel() != numel:
                raise ValueError(f"{name}: expected a contiguous host float16 tensor with {numel} elements")
        _check(LIB.kf_decode_step_host(self._h, layer, step, q.data_ptr(), knew.data_ptr(), vnew.data_ptr(),
                                       out.data_ptr(), 1 if wait else 0, _stream_ptr(stream)), "kf_decode_step_host")

    def kf_view_state(self, layer):
        """Zero-copy torch views (K, V, pos, acc, len) of one layer's cache inside the workspace."""
        ptrs = [C.c_void_p() for _ in range(5)]
        _check(LIB.kf_view_state(self._h, layer, *[C.byref(p) for p in ptrs]), "kf_view_state")
        B, H, k, d = self.cfg.batch, self.kv_heads, self.cfg.budget_k, self.cfg.head_dim   # one cache per key/value head
        base = self.workspace.data_ptr()

        def view(ptr, nbytes, dtype, shape):
            off = ptr.value - base
            return self.workspace[off:off + nbytes].view(dtype).view(shape)
        K = view(ptrs[0], B * H * k * d * 2, torch.float16, (B, H, k, d))
        V = view(ptrs[1], B * H * k * d * 2, torch.float16, (B, H, k, d))
        pos = view(ptrs[2], B * H * k * 4, torch.int32, (B, H, k))
        acc = view(ptrs[3], B * H * k * 4, torch.float32, (B, H, k))
        ln = view(ptrs[4], B * H * 4, torch.int32, (B, H))
        return K, V, pos, acc, ln

    def kf_compact_layer(self, layer, stream=None):
        """Reorder the layer's cache entries into ascending position, in place."""
        _check(LIB.kf_compact_layer(self._h, layer, _stream_ptr(stream)), "kf_compact_layer")

    def kf_reorder_beams(self, layer, parent, stream=None):
        """Batch rows follow their beam's parent (int32 CUDA [requests, beams], requests * beams = batch); layer -1: all layers."""
        if parent.dim() != 2 or parent.numel() != self.cfg.batch:
            raise ValueError(f"parent: expected [requests, beams] with {self.cfg.batch} elements, got {tuple(parent.shape)}")
        _check(LIB.kf_reorder_beams(self._h, layer, parent.shape[1], _dev_ptr(parent, torch.int32, self.cfg.batch, "parent"),
                                    _stream_ptr(stream)), "kf_reorder_beams")

    def kf_view_place(self, layer):
        """Zero-copy torch view of one layer's places (KF_POS_NEW only), int32 [B, H, k]."""
        ptr = C.c_void_p()
        _check(LIB.kf_view_place(self._h, layer, C.byref(ptr)), "kf_view_place")
        B, H, k = self.cfg.batch, self.kv_heads, self.cfg.budget_k
        off = ptr.value - self.workspace.data_ptr()
        return self.workspace[off:off + B * H * k * 4].view(torch.int32).view(B, H, k)

    def kf_state_bytes(self) -> int:
        return int(LIB.kf_state_bytes(self._h))

    def kf_export_state(self, layer, image, stream=None):
        """Copy one layer's cache image into the uint8 CUDA tensor `image`; returns (n_prompt, last_step)."""
        n_prompt, last_step = C.c_int32(), C.c_int32()
        _check(LIB.kf_export_state(self._h, layer, _dev_ptr(image, torch.uint8, image.numel(), "image"), image.numel(),
                                   C.byref(n_prompt), C.byref(last_step), _stream_ptr(stream)), "kf_export_state")
        return n_prompt.value, last_step.value

    def kf_import_state(self, layer, image, n_prompt, last_step, stream=None):
        _check(LIB.kf_import_state(self._h, layer, _dev_ptr(image, torch.uint8, image.numel(), "image"), image.numel(),
                                   n_prompt, last_step, _stream_ptr(stream)), "kf_import_state")

    def kf_poll_error(self, stream=None) -> int:
        return int(LIB.kf_poll_error(self._h, _stream_ptr(stream)))

    def kf_check_canaries(self, stream=None):
        """(status, index of the first sub-buffer whose guard was overwritten or -1); debug layout only."""
        bad = C.c_int32(-1)
        rc = int(LIB.kf_check_canaries(self._h, _stream_ptr(stream), C.byref(bad)))
        return rc, bad.value

    def kf_describe_decode(self) -> str:
        buf = C.create_string_buffer(256)
        _check(min(0, int(LIB.kf_describe_decode(self._h, buf, len(buf)))), "kf_describe_decode")
        return buf.value.decode()

    def kf_launch_count(self) -> int:
        return int(LIB.kf_launch_count(self._h))

    def kf_destroy(self):
        if self._h is not None and self._h.value:
            LIB.kf_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.kf_destroy()
        except Exception:
            pass
