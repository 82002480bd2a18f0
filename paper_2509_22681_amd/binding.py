"""ctypes binding of libflame_gr.so: argument marshalling only.

Function names mirror the C ABI (include/flame_gr.h).  PyTorch tensors are accepted wherever the
ABI takes a device pointer; numpy arrays wherever it takes a host pointer.  Nothing here computes
any part of the forward, and nothing falls back to another implementation: if the library has not
been built, importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional

import numpy as np
# PyTorch provides device memory and streams.  It must be imported before the library is loaded so
# that both resolve libamdhip64.so.7 to the one HIP runtime PyTorch bundles: two HIP runtimes in one
# process do not both see the device.
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libflame_gr.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()' "
        "or python paper_2509_22681_amd/build.py)")

_lib = C.CDLL(LIB_PATH)

FLAME_GR_F32, FLAME_GR_BF16 = 0, 1
FLAME_GR_ATTN_SILU, FLAME_GR_ATTN_SOFTMAX = 0, 1
STATUS = {0: "OK", -1: "INVALID_ARGUMENT", -2: "CAPACITY_EXCEEDED", -3: "HIP_ERROR", -4: "BAD_HANDLE",
          -5: "UNSUPPORTED"}
# what is timed apart; "assemble" holds the bias expansion and the weights' operand copies ("bias" is always 0), and "outproj" the next layer's
# projections where one launch does both
KERNEL_KINDS = ("assemble", "bias", "uvqk", "attn", "ln_gate", "outproj", "score")


class flame_gr_config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("n_buckets", C.c_int32), ("max_rel_dist", C.c_int32), ("dtype", C.c_int32),
                ("ln_eps", C.c_float), ("attn_scale", C.c_float),
                ("max_requests", C.c_int32), ("max_total_tokens", C.c_int32),
                ("max_seq_tokens", C.c_int32), ("n_streams", C.c_int32), ("attn_kind", C.c_int32),
                ("kv_cache", C.c_int32), ("latency_mode", C.c_int32), ("weights_static", C.c_int32)]


class flame_gr_weights(C.Structure):
    _fields_ = [("w1", C.c_void_p), ("b1", C.c_void_p), ("rab", C.c_void_p), ("ln_g", C.c_void_p),
                ("ln_b", C.c_void_p), ("w2", C.c_void_p), ("b2", C.c_void_p), ("w_s", C.c_void_p),
                ("b_s", C.c_float), ("temperature", C.c_void_p)]


_i32p = C.POINTER(C.c_int32)
_lib.flame_gr_create.argtypes = [C.POINTER(flame_gr_config), C.POINTER(C.c_void_p)]
_lib.flame_gr_create.restype = C.c_int
_lib.flame_gr_forward.argtypes = [C.c_void_p, C.POINTER(flame_gr_weights), C.c_void_p, _i32p, C.c_void_p, _i32p,
                                  C.c_int32, C.c_void_p, C.c_void_p]
_lib.flame_gr_forward.restype = C.c_int
_lib.flame_gr_forward_hidden.argtypes = _lib.flame_gr_forward.argtypes
_lib.flame_gr_forward_hidden.restype = C.c_int
_lib.flame_gr_forward_static.argtypes = [C.POINTER(flame_gr_config), C.POINTER(flame_gr_weights), C.c_void_p, _i32p, C.c_void_p, _i32p,
                                         C.c_int32, C.c_void_p, C.c_void_p]
_lib.flame_gr_forward_static.restype = C.c_int
_lib.flame_gr_static_scratch_bytes.argtypes = [C.POINTER(flame_gr_config), C.c_int64, C.POINTER(C.c_int64)]
_lib.flame_gr_static_scratch_bytes.restype = C.c_int
_lib.flame_gr_capture.argtypes = [C.c_void_p, C.c_int32, C.POINTER(flame_gr_weights), C.c_void_p, _i32p, C.c_void_p, _i32p,
                                  C.c_int32, C.c_void_p, C.c_void_p]
_lib.flame_gr_capture.restype = C.c_int
_lib.flame_gr_replay.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
_lib.flame_gr_replay.restype = C.c_int
_lib.flame_gr_prefill.argtypes = [C.c_void_p, C.POINTER(flame_gr_weights), C.c_void_p, _i32p, _i32p, C.c_int32, C.c_void_p]
_lib.flame_gr_prefill.restype = C.c_int
_lib.flame_gr_score.argtypes = [C.c_void_p, C.POINTER(flame_gr_weights), C.c_void_p, _i32p, C.c_int32, C.c_void_p, C.c_void_p]
_lib.flame_gr_score.restype = C.c_int
_lib.flame_gr_destroy.argtypes = [C.c_void_p]
_lib.flame_gr_destroy.restype = C.c_int
_lib.flame_gr_last_error.argtypes = [C.c_void_p]
_lib.flame_gr_last_error.restype = C.c_char_p
_lib.flame_gr_host_bucket_table.argtypes = [C.c_int32, C.c_int32, _i32p]
_lib.flame_gr_host_bucket_table.restype = C.c_int
_lib.flame_gr_host_mask.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
_lib.flame_gr_host_mask.restype = C.c_int
_lib.flame_gr_host_plan.argtypes = [C.POINTER(flame_gr_config), _i32p, _i32p, C.c_int32, _i32p, _i32p, _i32p, C.c_int32]
_lib.flame_gr_host_plan.restype = C.c_int
_lib.flame_gr_host_workspace_rows.argtypes = [C.POINTER(flame_gr_config), C.POINTER(C.c_int64)]
_lib.flame_gr_host_workspace_rows.restype = C.c_int
_lib.flame_gr_host_plan_reserved.argtypes = [C.POINTER(flame_gr_config), _i32p, _i32p, _i32p, C.c_int32, _i32p, _i32p, C.c_int32]
_lib.flame_gr_host_plan_reserved.restype = C.c_int
_lib.flame_gr_debug_capture.argtypes = [C.c_void_p, C.c_int32]
_lib.flame_gr_debug_capture.restype = C.c_int
_lib.flame_gr_debug_stage.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
_lib.flame_gr_debug_stage.restype = C.c_int
_lib.flame_gr_debug_device_mask.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
_lib.flame_gr_debug_device_mask.restype = C.c_int
_lib.flame_gr_debug_profile.argtypes = [C.c_void_p, C.c_int32]
_lib.flame_gr_debug_profile.restype = C.c_int
_lib.flame_gr_debug_profile_read.argtypes = [C.c_void_p, C.POINTER(C.c_float), _i32p]
_lib.flame_gr_debug_profile_read.restype = C.c_int

class flame_dso_config(C.Structure):
    _fields_ = [("hist_len", C.c_int32), ("n_profiles", C.c_int32), ("profiles", _i32p),
                ("n_executors", C.c_int32), ("explicit_shapes", C.c_int32), ("max_batch", C.c_int32)]


_lib.flame_dso_create.argtypes = [C.POINTER(flame_gr_config), C.POINTER(flame_gr_weights), C.POINTER(flame_dso_config),
                                  C.POINTER(C.c_void_p)]
_lib.flame_dso_create.restype = C.c_int
_lib.flame_dso_submit.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.POINTER(C.c_int64)]
_lib.flame_dso_submit.restype = C.c_int
_lib.flame_dso_submit_jagged.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.POINTER(C.c_int64)]
_lib.flame_dso_submit_jagged.restype = C.c_int
_lib.flame_dso_wait.argtypes = [C.c_void_p, C.c_int64]
_lib.flame_dso_wait.restype = C.c_int
_lib.flame_dso_drain.argtypes = [C.c_void_p]
_lib.flame_dso_drain.restype = C.c_int
_lib.flame_dso_flush.argtypes = [C.c_void_p]
_lib.flame_dso_flush.restype = C.c_int
_lib.flame_dso_destroy.argtypes = [C.c_void_p]
_lib.flame_dso_destroy.restype = C.c_int
_lib.flame_dso_last_error.argtypes = [C.c_void_p]
_lib.flame_dso_last_error.restype = C.c_char_p
_lib.flame_dso_route.argtypes = [_i32p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _i32p, C.c_int32, _i32p]
_lib.flame_dso_route.restype = C.c_int
_lib.flame_dso_stats.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
_lib.flame_dso_stats.restype = C.c_int

class flame_climber_head_config(C.Structure):
    _fields_ = [("n_blocks", C.c_int32), ("d_model", C.c_int32), ("n_tasks", C.c_int32), ("expert_width", C.c_int32)]


class flame_climber_head_weights(C.Structure):
    _fields_ = [("wg", C.c_void_p), ("cg", C.c_void_p), ("a_w", C.c_void_p), ("a_b", C.c_void_p), ("v", C.c_void_p),
                ("c", C.c_void_p)]


_lib.flame_climber_head.argtypes = [C.POINTER(flame_climber_head_config), C.POINTER(flame_climber_head_weights),
                                    C.POINTER(C.c_void_p), C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.flame_climber_head.restype = C.c_int
_lib.flame_climber_block_range.argtypes = [C.c_int32, C.c_int32, C.c_int32, _i32p, _i32p]
_lib.flame_climber_block_range.restype = C.c_int
_lib.flame_climber_last_error.argtypes = []
_lib.flame_climber_last_error.restype = C.c_char_p


class flame_kv_config(C.Structure):
    torch_dtype = None          # of the tensors (make_kv_config sets it)
    _fields_ = [("dtype", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("scale", C.c_float)]


class flame_kv_rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class flame_kv_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_stride", C.c_int64), ("slot_stride", C.c_int64), ("head_stride", C.c_int64),
                ("n_pages", C.c_int32), ("page_size", C.c_int32), ("page_table", C.c_void_p), ("table_stride", C.c_int64), ("pages_per_seq", C.c_int32)]


class flame_kv_rotation(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("frequencies", C.POINTER(C.c_double))]


_kv_cfg, _kv_rows_p, _kv_cache_p = C.POINTER(flame_kv_config), C.POINTER(flame_kv_rows), C.POINTER(flame_kv_cache)
_lib.flame_kv_append.argtypes = [_kv_cfg, _kv_cache_p, _kv_rows_p, _kv_rows_p, _kv_rows_p, _kv_rows_p, C.POINTER(flame_kv_rotation), C.c_void_p, C.c_void_p,
                                 C.c_int32, C.c_int64, C.c_void_p, C.c_void_p]
_lib.flame_kv_append.restype = C.c_int
_lib.flame_kv_prompt.argtypes = [_kv_cfg, _kv_rows_p, _kv_rows_p, _kv_rows_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_int64, _kv_rows_p, C.c_void_p, C.c_void_p]
_lib.flame_kv_prompt.restype = C.c_int
_lib.flame_kv_extend.argtypes = [_kv_cfg, _kv_cache_p, _kv_rows_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, _kv_rows_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
_lib.flame_kv_extend.restype = C.c_int
_lib.flame_kv_decode.argtypes = [_kv_cfg, _kv_cache_p, _kv_rows_p, C.c_void_p, C.c_int32, _kv_rows_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
_lib.flame_kv_decode.restype = C.c_int
_lib.flame_kv_workspace_bytes.argtypes = [_kv_cfg, C.c_int32, C.c_int64, C.POINTER(C.c_int64)]
_lib.flame_kv_workspace_bytes.restype = C.c_int
_lib.flame_kv_rotation_frequencies.argtypes = [C.c_int32, C.c_double, C.POINTER(C.c_double)]
_lib.flame_kv_rotation_frequencies.restype = C.c_int
_lib.flame_kv_last_error.argtypes = []
_lib.flame_kv_last_error.restype = C.c_char_p


class flame_kv_groups(C.Structure):
    _fields_ = [("group_offsets", C.c_void_p), ("prefix_lens", C.c_void_p), ("n_groups", C.c_int32)]


class flame_kvq_cache(C.Structure):
    _fields_ = [("form", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p), ("page_stride", C.c_int64), ("slot_stride", C.c_int64),
                ("head_stride", C.c_int64), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("page_table", C.c_void_p), ("table_stride", C.c_int64), ("pages_per_seq", C.c_int32)]


_kvq_cache_p, _kv_groups_p = C.POINTER(flame_kvq_cache), C.POINTER(flame_kv_groups)
for _name, _cache in (("flame_kv_shared", _kv_cache_p), ("flame_kvq_shared", _kvq_cache_p)):
    getattr(_lib, _name).argtypes = [_kv_cfg, _cache, _kv_rows_p, C.c_void_p, C.c_void_p, _kv_groups_p, C.c_int32, C.c_int64, _kv_rows_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
    getattr(_lib, _name).restype = C.c_int
_lib.flame_kv_shared_workspace_bytes.argtypes = [_kv_cfg, C.c_int32, C.c_int32, C.c_int64, C.POINTER(C.c_int64)]
_lib.flame_kv_shared_workspace_bytes.restype = C.c_int
_lib.flame_kvq_append.argtypes = [_kv_cfg, _kvq_cache_p, _kv_rows_p, _kv_rows_p, _kv_rows_p, _kv_rows_p, C.POINTER(flame_kv_rotation), C.c_void_p, C.c_void_p,
                                  C.c_int32, C.c_int64, C.c_void_p, C.c_void_p]
_lib.flame_kvq_append.restype = C.c_int
_lib.flame_kvq_read.argtypes = [_kv_cfg, _kvq_cache_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, _kv_rows_p, _kv_rows_p, C.c_void_p, C.c_void_p]
_lib.flame_kvq_read.restype = C.c_int
_lib.flame_kvq_extend.argtypes = [_kv_cfg, _kvq_cache_p, _kv_rows_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, _kv_rows_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
_lib.flame_kvq_extend.restype = C.c_int
_lib.flame_kvq_decode.argtypes = [_kv_cfg, _kvq_cache_p, _kv_rows_p, C.c_void_p, C.c_int32, _kv_rows_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
_lib.flame_kvq_decode.restype = C.c_int

KV_EXPORTS = ("flame_kv_append", "flame_kv_prompt", "flame_kv_extend", "flame_kv_decode", "flame_kv_shared", "flame_kv_workspace_bytes", "flame_kv_shared_workspace_bytes",
              "flame_kv_rotation_frequencies", "flame_kv_last_error")
KVQ_EXPORTS = ("flame_kvq_append", "flame_kvq_read", "flame_kvq_extend", "flame_kvq_decode", "flame_kvq_shared")

CLIMBER_EXPORTS = ("flame_climber_head", "flame_climber_block_range", "flame_climber_last_error")

DSO_EXPORTS = ("flame_dso_create", "flame_dso_submit", "flame_dso_submit_jagged", "flame_dso_wait", "flame_dso_drain", "flame_dso_flush", "flame_dso_destroy",
               "flame_dso_last_error", "flame_dso_route", "flame_dso_stats")

EXPORTS = ("flame_gr_create", "flame_gr_forward", "flame_gr_forward_hidden", "flame_gr_forward_static", "flame_gr_static_scratch_bytes", "flame_gr_capture", "flame_gr_replay", "flame_gr_prefill", "flame_gr_score", "flame_gr_destroy",
           "flame_gr_last_error",
           "flame_gr_host_bucket_table", "flame_gr_host_mask", "flame_gr_host_plan", "flame_gr_host_plan_reserved", "flame_gr_host_workspace_rows",
           "flame_gr_debug_capture", "flame_gr_debug_stage", "flame_gr_debug_device_mask",
           "flame_gr_debug_profile", "flame_gr_debug_profile_read")


class FlameGRError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


def _check(rc: int, h=None):
    if rc != 0:
        msg = _lib.flame_gr_last_error(h)
        raise FlameGRError(rc, msg.decode() if msg else "")


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.int32)


def _ptr(t) -> Optional[int]:
    """Device (torch tensor) or host (numpy) pointer, or None."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr() if t.numel() else None


def make_config(n_layers, d_model, n_heads, n_buckets, max_rel_dist, dtype, *, ln_eps=1e-6, attn_scale=1.0,
                max_requests=0, max_total_tokens=0, max_seq_tokens=0, n_streams=0, kv_cache=0,
                attn_kind="silu", latency_mode=0, weights_static=0) -> flame_gr_config:
    dt = {"f32": FLAME_GR_F32, "bf16": FLAME_GR_BF16}.get(dtype, dtype)
    ak = {"silu": FLAME_GR_ATTN_SILU, "softmax": FLAME_GR_ATTN_SOFTMAX}.get(attn_kind, attn_kind)
    return flame_gr_config(n_layers, d_model, n_heads, n_buckets, max_rel_dist, dt, ln_eps, attn_scale,
                           max_requests, max_total_tokens, max_seq_tokens, n_streams, ak, int(kv_cache), int(latency_mode),
                           int(weights_static))


# ---------------------------------------------------------------------------------------------
# the three calls of the boundary, plus helpers, under their C names
# ---------------------------------------------------------------------------------------------
def flame_gr_create(cfg: flame_gr_config) -> C.c_void_p:
    h = C.c_void_p()
    _check(_lib.flame_gr_create(C.byref(cfg), C.byref(h)))
    return h


def flame_gr_destroy(h) -> None:
    _check(_lib.flame_gr_destroy(h))


def pack_weights(w: Dict[str, object]) -> flame_gr_weights:
    """dict of device tensors (+ python float b_s) -> struct of device pointers."""
    return flame_gr_weights(_ptr(w["w1"]), _ptr(w["b1"]), _ptr(w["rab"]), _ptr(w["ln_g"]), _ptr(w["ln_b"]),
                            _ptr(w["w2"]), _ptr(w["b2"]), _ptr(w.get("w_s")), float(w.get("b_s", 0.0)),
                            _ptr(w.get("temperature")))


def flame_gr_forward(h, weights, history_emb, history_offsets, cand_emb, cand_offsets, scores, stream=None) -> None:
    """weights: flame_gr_weights or dict; *_emb / scores: device tensors; *_offsets: host int32 arrays.
    stream: torch.cuda.Stream, raw hipStream_t integer, or None for the current torch stream."""
    ws = weights if isinstance(weights, flame_gr_weights) else pack_weights(weights)
    ho, co = _i32(history_offsets), _i32(cand_offsets)
    n = len(ho) - 1
    if len(co) - 1 != n:
        raise ValueError("offset arrays differ in length")
    if stream is None:
        sp = torch.cuda.current_stream().cuda_stream
    else:
        sp = getattr(stream, "cuda_stream", stream)
    rc = _lib.flame_gr_forward(h, C.byref(ws), _ptr(history_emb), ho.ctypes.data_as(_i32p), _ptr(cand_emb),
                               co.ctypes.data_as(_i32p), n, _ptr(scores), C.c_void_p(sp))
    _check(rc, h)


def flame_gr_forward_static(cfg: flame_gr_config, weights, history_emb, history_offsets, cand_emb, cand_offsets, scores,
                            stream=None) -> None:
    """flame_gr_forward without a handle, in the library's static device workspace (no allocation)."""
    ws = weights if isinstance(weights, flame_gr_weights) else pack_weights(weights)
    ho, co = _i32(history_offsets), _i32(cand_offsets)
    n = len(ho) - 1
    if len(co) - 1 != n:
        raise ValueError("offset arrays differ in length")
    sp = torch.cuda.current_stream().cuda_stream if stream is None else getattr(stream, "cuda_stream", stream)
    rc = _lib.flame_gr_forward_static(C.byref(cfg), C.byref(ws), _ptr(history_emb), ho.ctypes.data_as(_i32p), _ptr(cand_emb),
                                      co.ctypes.data_as(_i32p), n, _ptr(scores), C.c_void_p(sp))
    _check(rc)


def flame_gr_static_scratch_bytes(cfg: flame_gr_config, padded_rows: int) -> int:
    out = C.c_int64(0)
    _check(_lib.flame_gr_static_scratch_bytes(C.byref(cfg), padded_rows, C.byref(out)))
    return out.value


def _stream_ptr(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


def flame_gr_capture(h, weights, history_emb, history_offsets, cand_emb, cand_offsets, scores, slot: int = 0,
                     record_stream=None) -> None:
    """Record the forward of this fixed batch (shape, buffers) into graph `slot` of the handle."""
    ws = weights if isinstance(weights, flame_gr_weights) else pack_weights(weights)
    ho, co = _i32(history_offsets), _i32(cand_offsets)
    n = len(ho) - 1
    if len(co) - 1 != n:
        raise ValueError("offset arrays differ in length")
    rc = _lib.flame_gr_capture(h, slot, C.byref(ws), _ptr(history_emb), ho.ctypes.data_as(_i32p), _ptr(cand_emb),
                               co.ctypes.data_as(_i32p), n, _ptr(scores),
                               C.c_void_p(getattr(record_stream, "cuda_stream", record_stream) or 0))
    _check(rc, h)


def flame_gr_replay(h, stream=None, slot: int = 0) -> None:
    _check(_lib.flame_gr_replay(h, slot, C.c_void_p(_stream_ptr(stream))), h)


def flame_gr_prefill(h, weights, history_emb, history_offsets, cand_capacity, stream=None) -> None:
    """History stage of the two-stage path; cand_capacity: host int32 [n_requests]."""
    ws = weights if isinstance(weights, flame_gr_weights) else pack_weights(weights)
    ho, cc = _i32(history_offsets), _i32(cand_capacity)
    n = len(ho) - 1
    if len(cc) != n:
        raise ValueError("cand_capacity must have one entry per request")
    rc = _lib.flame_gr_prefill(h, C.byref(ws), _ptr(history_emb), ho.ctypes.data_as(_i32p), cc.ctypes.data_as(_i32p), n,
                               C.c_void_p(_stream_ptr(stream)))
    _check(rc, h)


def flame_gr_score(h, weights, cand_emb, cand_offsets, scores, stream=None) -> None:
    """Candidate stage of the two-stage path, against the history cached by the last prefill."""
    ws = weights if isinstance(weights, flame_gr_weights) else pack_weights(weights)
    co = _i32(cand_offsets)
    rc = _lib.flame_gr_score(h, C.byref(ws), _ptr(cand_emb), co.ctypes.data_as(_i32p), len(co) - 1, _ptr(scores),
                             C.c_void_p(_stream_ptr(stream)))
    _check(rc, h)


def flame_gr_forward_hidden(h, weights, history_emb, history_offsets, cand_emb, cand_offsets, hidden, stream=None) -> None:
    """As flame_gr_forward, with the candidates' final residual rows (device fp32 [sum M, d]) as the output."""
    ws = weights if isinstance(weights, flame_gr_weights) else pack_weights(weights)
    ho, co = _i32(history_offsets), _i32(cand_offsets)
    n = len(ho) - 1
    if len(co) - 1 != n:
        raise ValueError("offset arrays differ in length")
    rc = _lib.flame_gr_forward_hidden(h, C.byref(ws), _ptr(history_emb), ho.ctypes.data_as(_i32p), _ptr(cand_emb),
                                      co.ctypes.data_as(_i32p), n, _ptr(hidden), C.c_void_p(_stream_ptr(stream)))
    _check(rc, h)


def flame_gr_last_error(h=None) -> str:
    return _lib.flame_gr_last_error(h).decode()


def flame_gr_host_bucket_table(n_buckets: int, max_rel_dist: int) -> np.ndarray:
    out = np.empty(max(max_rel_dist, 0), np.int32)
    _check(_lib.flame_gr_host_bucket_table(n_buckets, max_rel_dist, out.ctypes.data_as(_i32p)))
    return out


def flame_gr_host_mask(L: int, M: int, n_buckets: int, max_rel_dist: int):
    N = L + M
    mask = np.empty((N, N), np.uint8)
    bucket = np.empty((N, N), np.int32)
    _check(_lib.flame_gr_host_mask(L, M, n_buckets, max_rel_dist, mask.ctypes.data, bucket.ctypes.data))
    return mask, bucket


def flame_gr_host_plan(cfg: flame_gr_config, history_offsets, cand_offsets):
    """-> (tok_off [B+1], segments [S,6]: request, L, cand_begin, M, row_start, group)"""
    ho, co = _i32(history_offsets), _i32(cand_offsets)
    n = len(ho) - 1
    tok = np.zeros(n + 1, np.int32)
    nseg = C.c_int32(0)
    _check(_lib.flame_gr_host_plan(C.byref(cfg), ho.ctypes.data_as(_i32p), co.ctypes.data_as(_i32p), n,
                                   tok.ctypes.data_as(_i32p), C.byref(nseg), None, 0))
    seg = np.zeros((max(nseg.value, 1), 6), np.int32)
    _check(_lib.flame_gr_host_plan(C.byref(cfg), ho.ctypes.data_as(_i32p), co.ctypes.data_as(_i32p), n,
                                   tok.ctypes.data_as(_i32p), C.byref(nseg), seg.ctypes.data_as(_i32p), len(seg)))
    return tok, seg[:nseg.value]


def flame_gr_host_workspace_rows(cfg: flame_gr_config) -> int:
    rows = C.c_int64(0)
    _check(_lib.flame_gr_host_workspace_rows(C.byref(cfg), C.byref(rows)))
    return rows.value


def flame_gr_host_plan_reserved(cfg: flame_gr_config, history_offsets, cand_offsets, cand_capacity):
    """-> segments [S,6] of the two-stage layout: request, L, cand_begin, M, row_start, group"""
    ho, co, cc = _i32(history_offsets), _i32(cand_offsets), _i32(cand_capacity)
    n = len(ho) - 1
    if len(co) - 1 != n or len(cc) != n:
        raise ValueError("offset and capacity arrays differ in length")
    seg = np.zeros((max(n, 1), 6), np.int32)
    nseg = C.c_int32(0)
    _check(_lib.flame_gr_host_plan_reserved(C.byref(cfg), ho.ctypes.data_as(_i32p), co.ctypes.data_as(_i32p),
                                            cc.ctypes.data_as(_i32p), n, C.byref(nseg), seg.ctypes.data_as(_i32p), len(seg)))
    return seg[:nseg.value]


def flame_gr_debug_capture(h, layer: int) -> None:
    _check(_lib.flame_gr_debug_capture(h, layer), h)


def flame_gr_debug_stage(h, which: int, n_tokens: int, d: int) -> np.ndarray:
    out = np.empty((n_tokens, d), np.float32)
    _check(_lib.flame_gr_debug_stage(h, which, out.ctypes.data), h)
    return out


def flame_gr_debug_device_mask(h, L: int, M: int):
    N = L + M
    mask = np.empty((N, N), np.uint8)
    bucket = np.empty((N, N), np.int32)
    _check(_lib.flame_gr_debug_device_mask(h, L, M, mask.ctypes.data, bucket.ctypes.data), h)
    return mask, bucket


def flame_gr_debug_profile(h, enable: bool) -> None:
    _check(_lib.flame_gr_debug_profile(h, int(enable)), h)


def flame_gr_debug_profile_read(h):
    """-> {kind: (milliseconds, launches)} for the last forward run with profiling on."""
    ms = (C.c_float * len(KERNEL_KINDS))()
    n = (C.c_int32 * len(KERNEL_KINDS))()
    _check(_lib.flame_gr_debug_profile_read(h, ms, n), h)
    return {k: (float(ms[i]), int(n[i])) for i, k in enumerate(KERNEL_KINDS)}


# ---------------------------------------------------------------------------------------------
# request orchestrator (include/flame_dso.h); embeddings and scores are HOST numpy arrays here
# ---------------------------------------------------------------------------------------------
def _dso_check(rc: int, dso=None):
    if rc != 0:
        msg = _lib.flame_dso_last_error(dso)
        raise FlameGRError(rc, msg.decode() if msg else "")


def flame_dso_create(cfg: flame_gr_config, weights, hist_len: int, profiles, n_executors: int,
                     explicit_shapes=True, max_batch: int = 1) -> C.c_void_p:
    """explicit_shapes: True/1 graph executors, False/0 eager dynamic shapes, 2 jagged micro-batches of max_batch."""
    ws = weights if isinstance(weights, flame_gr_weights) else pack_weights(weights)
    prof = _i32(profiles)
    dc = flame_dso_config(hist_len, len(prof), prof.ctypes.data_as(_i32p), n_executors, int(explicit_shapes), max_batch)
    out = C.c_void_p()
    _dso_check(_lib.flame_dso_create(C.byref(cfg), C.byref(ws), C.byref(dc), C.byref(out)))
    return out


def host_embedding(a, dtype: str) -> np.ndarray:
    """fp32 numpy values -> the raw host layout the orchestrator expects (bf16 as uint16 bit patterns;
    the values are expected to be bf16-representable already, as the workload generators make them)."""
    a = np.ascontiguousarray(a, dtype=np.float32)
    if dtype == "f32":
        return a
    bits = a.view(np.uint32)
    if (bits & 0xFFFF).any():
        raise ValueError("values are not bf16-representable")
    return np.ascontiguousarray((bits >> 16).astype(np.uint16))


def flame_dso_submit(dso, history_emb: np.ndarray, cand_emb: np.ndarray, scores: np.ndarray) -> int:
    """history_emb / cand_emb: contiguous host arrays in the model dtype (see host_embedding);
    scores: contiguous float32 host array [n_cand], filled by the wait that retires the ticket."""
    if not (cand_emb.flags.c_contiguous and scores.flags.c_contiguous and scores.dtype == np.float32):
        raise ValueError("cand_emb and scores must be contiguous, scores float32")
    t = C.c_int64(0)
    hp = history_emb.ctypes.data if history_emb is not None and history_emb.size else None
    _dso_check(_lib.flame_dso_submit(dso, hp, cand_emb.ctypes.data, int(cand_emb.shape[0]), scores.ctypes.data, C.byref(t)), dso)
    return t.value


def flame_dso_submit_jagged(dso, history_emb: np.ndarray, cand_emb: np.ndarray, scores: np.ndarray) -> int:
    """Mode 2: a request whose history length is history_emb.shape[0] (at most the capacity given at create)."""
    if not (cand_emb.flags.c_contiguous and scores.flags.c_contiguous and scores.dtype == np.float32):
        raise ValueError("cand_emb and scores must be contiguous, scores float32")
    L = int(history_emb.shape[0]) if history_emb is not None else 0
    if L and not history_emb.flags.c_contiguous:
        raise ValueError("history_emb must be contiguous")
    t = C.c_int64(0)
    hp = history_emb.ctypes.data if L else None
    _dso_check(_lib.flame_dso_submit_jagged(dso, hp, L, cand_emb.ctypes.data, int(cand_emb.shape[0]), scores.ctypes.data,
                                            C.byref(t)), dso)
    return t.value


def flame_dso_wait(dso, ticket: int) -> None:
    _dso_check(_lib.flame_dso_wait(dso, ticket), dso)


def flame_dso_flush(dso) -> None:
    _dso_check(_lib.flame_dso_flush(dso), dso)


def flame_dso_drain(dso) -> None:
    _dso_check(_lib.flame_dso_drain(dso), dso)


def flame_dso_destroy(dso) -> None:
    _dso_check(_lib.flame_dso_destroy(dso))


def flame_dso_last_error(dso=None) -> str:
    return _lib.flame_dso_last_error(dso).decode()


def flame_dso_stats(dso) -> Dict[str, int]:
    out = (C.c_int64 * 4)()
    _dso_check(_lib.flame_dso_stats(dso, out), dso)
    return dict(zip(("requests", "chunks", "candidate_rows_computed", "waits_for_a_busy_executor"), (int(v) for v in out)))


def flame_dso_route(profiles, hist_len: int, d_model: int, n_cand: int, explicit_shapes: bool = True):
    """-> list of (profile index, candidates taken)"""
    prof = _i32(profiles)
    n = C.c_int32(0)
    rc = _lib.flame_dso_route(prof.ctypes.data_as(_i32p), len(prof), hist_len, d_model, int(explicit_shapes), n_cand, None, 0,
                              C.byref(n))
    if rc not in (0, -2):
        raise FlameGRError(rc, "flame_dso_route")
    buf = np.zeros((max(n.value, 1), 2), np.int32)
    rc = _lib.flame_dso_route(prof.ctypes.data_as(_i32p), len(prof), hist_len, d_model, int(explicit_shapes), n_cand,
                              buf.ctypes.data_as(_i32p), len(buf), C.byref(n))
    if rc != 0:
        raise FlameGRError(rc, "flame_dso_route")
    return [(int(a), int(b)) for a, b in buf[:n.value]]


# ---------------------------------------------------------------------------------------------
# fusion of the sub-sequence blocks and task head (include/flame_climber.h)
# ---------------------------------------------------------------------------------------------
def flame_climber_block_range(L: int, n_blocks: int, b: int):
    lo, hi = C.c_int32(0), C.c_int32(0)
    rc = _lib.flame_climber_block_range(L, n_blocks, b, C.byref(lo), C.byref(hi))
    if rc != 0:
        raise FlameGRError(rc, "flame_climber_block_range")
    return lo.value, hi.value


def flame_climber_head(head: Dict[str, object], hidden, fused, probs, stream=None) -> None:
    """head: dict of device fp32 tensors wg [Nb,d,Nb*d], cg [Nb,d], a_w [T,E,d], a_b [T,E], v [T,E], c [T];
    hidden: list of Nb device fp32 tensors [rows, d]; fused [rows, d] workspace; probs [rows, T] output."""
    nb = len(hidden)
    rows, d = (int(hidden[0].shape[0]), int(hidden[0].shape[1])) if nb else (0, 0)
    T, E = int(head["a_w"].shape[0]), int(head["a_w"].shape[1])
    cfg = flame_climber_head_config(nb, d, T, E)
    ws = flame_climber_head_weights(*[_ptr(head[k]) for k in ("wg", "cg", "a_w", "a_b", "v", "c")])
    ptrs = (C.c_void_p * max(nb, 1))(*[_ptr(h) for h in hidden])
    rc = _lib.flame_climber_head(C.byref(cfg), C.byref(ws), ptrs, rows, _ptr(fused), _ptr(probs), C.c_void_p(_stream_ptr(stream)))
    if rc != 0:
        raise FlameGRError(rc, _lib.flame_climber_last_error().decode())


# ---------------------------------------------------------------------------------------------
# softmax attention on a paged key/value cache (include/flame_kv.h).  Tensors are checked here for what the C side cannot see: shapes,
# element types, and that they lie on the current device.
# ---------------------------------------------------------------------------------------------
FLAME_KV_F32, FLAME_KV_BF16, FLAME_KV_F16 = 0, 1, 2
FLAME_KV_FAULT_PAGE, FLAME_KV_FAULT_LENGTH, FLAME_KV_FAULT_OFFSET = 1, 2, 4
_KV_DTYPES = {"f32": FLAME_KV_F32, "bf16": FLAME_KV_BF16, "f16": FLAME_KV_F16}
_KV_TORCH = (torch.float32, torch.bfloat16, torch.float16)


def _kv_check(rc: int):
    if rc != 0:
        raise FlameGRError(rc, _lib.flame_kv_last_error().decode())


def make_kv_config(dtype, n_q_heads, n_kv_heads, head_dim, scale=0.0) -> flame_kv_config:
    """dtype: "f32", "bf16" or "f16"; scale of the logits, 0 for 1 / sqrt(head_dim)."""
    cfg = flame_kv_config(_KV_DTYPES.get(dtype, dtype), n_q_heads, n_kv_heads, head_dim, scale)
    cfg.torch_dtype = _KV_TORCH[cfg.dtype] if 0 <= cfg.dtype < 3 else None
    return cfg


# A call of a few new tokens takes a few microseconds on the GPU, so these checks count: each attribute of a tensor is asked for once.
def _kv_rows(cfg, t, heads: int, dev: int, what: str, written: bool = False):
    rows, h, dim = t.shape
    sr, sh, sd = t.stride()
    if h != heads or dim != cfg.head_dim or t.dtype is not cfg.torch_dtype:
        raise ValueError(f"{what} must be [rows, {heads}, {cfg.head_dim}] of {cfg.torch_dtype}")
    if t.get_device() != dev:
        raise ValueError(f"{what} is not on the current device")
    if sd != 1:
        raise ValueError(f"{what}: the features of a head must lie side by side")
    # a stride of a dimension of one is never used, whatever torch says it is
    if rows < 2:
        sr = 0
    if h == 1:
        sh = 0
    if written and ((sr == 0 and rows > 1) or (sh == 0 and h > 1)):
        raise ValueError(f"{what} is written and must not be an expanded tensor")
    return C.byref(flame_kv_rows(t.data_ptr(), sr, sh))


def _kv_ints(t, n: int, dev: int, what: str) -> int:
    if t.dtype is not torch.int32 or t.dim() != 1 or t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous int32 tensor of {n} entries")
    if t.get_device() != dev:
        raise ValueError(f"{what} is not on the current device")
    return t.data_ptr()


def _kv_workspace(workspace, dev: int):
    if workspace is None:
        return None, 0
    if not workspace.is_contiguous() or workspace.get_device() != dev:
        raise ValueError("the workspace must be contiguous and on the current device")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _kv_stream(stream, dev: int) -> int:
    # (the number alone: building torch's stream object takes longer than the rest of a call)
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else getattr(stream, "cuda_stream", stream)


def pack_kv_cache(cfg: flame_kv_config, k_pool, v_pool, page_table) -> flame_kv_cache:
    """k_pool, v_pool: device tensors [n_pages, page_size, n_kv_heads, head_dim] (any strides, the same for both, features side by side: a pool
    laid out [n_pages, n_kv_heads, page_size, head_dim] comes transposed); page_table: device int32 [n_seqs, pages_per_seq].  The struct keeps
    the tensors alive; their contents may change."""
    n_pages, page_size, heads, dim = k_pool.shape
    if heads != cfg.n_kv_heads or dim != cfg.head_dim or k_pool.dtype is not cfg.torch_dtype:
        raise ValueError(f"k_pool must be [n_pages, page_size, {cfg.n_kv_heads}, {cfg.head_dim}] of {cfg.torch_dtype}")
    if v_pool.shape != k_pool.shape or v_pool.dtype is not k_pool.dtype or v_pool.device != k_pool.device:
        raise ValueError("v_pool must be like k_pool")
    if page_table.dtype is not torch.int32 or page_table.dim() != 2 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
        raise ValueError("page_table must be int32 [n_seqs, pages_per_seq], the entries of a row side by side")
    if not k_pool.is_cuda or page_table.device != k_pool.device:
        raise ValueError("the pools and the page table must be on one device")
    used = [i for i in range(4) if k_pool.shape[i] > 1]
    if [k_pool.stride(i) for i in used] != [v_pool.stride(i) for i in used] or k_pool.stride(3) != 1:
        raise ValueError("k_pool and v_pool must have the same strides, and the features of a head side by side")
    if any(k_pool.stride(i) == 0 for i in used):
        raise ValueError("the pools must not be expanded tensors")
    stride = [k_pool.stride(i) if k_pool.shape[i] > 1 else 0 for i in range(3)]
    c = flame_kv_cache(k_pool.data_ptr(), v_pool.data_ptr(), *stride, n_pages, page_size, page_table.data_ptr(),
                       page_table.stride(0) if page_table.shape[0] > 1 else 0, page_table.shape[1])
    c.tensors = (k_pool, v_pool, page_table)
    c.n_seqs, c.device, c.shape = page_table.shape[0], k_pool.get_device(), (cfg.dtype, heads, dim)
    return c


def _kv_cache_for(cfg, cache, n_seqs: int, dev: int):
    if cache.shape != (cfg.dtype, cfg.n_kv_heads, cfg.head_dim):
        raise ValueError("the cache was packed for another configuration")
    if cache.n_seqs < n_seqs:
        raise ValueError("the page table has fewer rows than there are sequences")
    if cache.device != dev:
        raise ValueError("the cache is not on the current device")
    return C.byref(cache)


def make_kv_rotation(frequencies, interleaved: bool = False) -> flame_kv_rotation:
    """frequencies: host float64 [rot_dim / 2], radians per position (flame_kv_rotation_frequencies, or those of any other scheme)."""
    f = np.ascontiguousarray(frequencies, dtype=np.float64)
    r = flame_kv_rotation(2 * f.size, int(bool(interleaved)), f.ctypes.data_as(C.POINTER(C.c_double)))
    r.array = f
    return r


def flame_kv_rotation_frequencies(rot_dim: int, base: float = 10000.0) -> np.ndarray:
    out = np.empty(max(rot_dim // 2, 0), np.float64)
    _kv_check(_lib.flame_kv_rotation_frequencies(rot_dim, base, out.ctypes.data_as(C.POINTER(C.c_double))))
    return out


def flame_kv_workspace_bytes(cfg: flame_kv_config, n_seqs: int, n_tokens: Optional[int] = None) -> int:
    """Bytes of a workspace for every flame_kv_extend and flame_kv_decode of up to this many sequences and query rows (n_tokens None: one row each)."""
    out = C.c_int64(0)
    _kv_check(_lib.flame_kv_workspace_bytes(C.byref(cfg), n_seqs, n_seqs if n_tokens is None else n_tokens, C.byref(out)))
    return out.value


def flame_kv_append(cfg, cache, k, v, offsets, kv_lens, q=None, q_out=None, rotation=None, faults=None, stream=None) -> None:
    """k, v: device rows [n_tokens, n_kv_heads, head_dim]; offsets [n_seqs + 1] and kv_lens [n_seqs] (with the new tokens): device int32;
    q, q_out: rows [n_tokens, n_q_heads, head_dim]; rotation: make_kv_rotation or None; faults: device int32 [1] or None."""
    n_seqs, n, dev = len(kv_lens), len(k), torch.cuda.current_device()
    if len(v) != n or (q is None) != (q_out is None) or (q is not None and not len(q) == len(q_out) == n):
        raise ValueError("k, v, q and q_out must have the same rows, and q comes with q_out")
    rc = _lib.flame_kv_append(cfg, _kv_cache_for(cfg, cache, n_seqs, dev), _kv_rows(cfg, k, cfg.n_kv_heads, dev, "k"), _kv_rows(cfg, v, cfg.n_kv_heads, dev, "v"),
                              None if q is None else _kv_rows(cfg, q, cfg.n_q_heads, dev, "q"), None if q is None else _kv_rows(cfg, q_out, cfg.n_q_heads, dev, "q_out", True),
                              rotation, _kv_ints(offsets, n_seqs + 1, dev, "offsets"), _kv_ints(kv_lens, n_seqs, dev, "kv_lens"), n_seqs, n,
                              None if faults is None else _kv_ints(faults, 1, dev, "faults"), _kv_stream(stream, dev))
    if rc:
        _kv_check(rc)


def flame_kv_prompt(cfg, q, k, v, q_offsets, out, k_offsets=None, faults=None, stream=None) -> None:
    """q, out: device rows [n_tokens, n_q_heads, head_dim]; k, v: [n_keys, n_kv_heads, head_dim]; offsets: device int32 [n_seqs + 1]."""
    n_seqs, n, n_keys, dev = len(q_offsets) - 1, len(q), len(k), torch.cuda.current_device()
    if len(out) != n or len(v) != n_keys:
        raise ValueError("out must have the rows of q, and v those of k")
    rc = _lib.flame_kv_prompt(cfg, _kv_rows(cfg, q, cfg.n_q_heads, dev, "q"), _kv_rows(cfg, k, cfg.n_kv_heads, dev, "k"), _kv_rows(cfg, v, cfg.n_kv_heads, dev, "v"),
                              _kv_ints(q_offsets, n_seqs + 1, dev, "q_offsets"), None if k_offsets is None else _kv_ints(k_offsets, n_seqs + 1, dev, "k_offsets"), n_seqs, n, n_keys,
                              _kv_rows(cfg, out, cfg.n_q_heads, dev, "out", True), None if faults is None else _kv_ints(faults, 1, dev, "faults"), _kv_stream(stream, dev))
    if rc:
        _kv_check(rc)


def flame_kv_extend(cfg, cache, q, q_offsets, kv_lens, out, workspace=None, faults=None, stream=None) -> None:
    """q, out: device rows [n_tokens, n_q_heads, head_dim], the newest tokens of every sequence; q_offsets [n_seqs + 1], kv_lens [n_seqs]: device int32;
    workspace: device tensor of flame_kv_workspace_bytes bytes for these sequences and rows or for more."""
    n_seqs, n, dev = len(kv_lens), len(q), torch.cuda.current_device()
    if len(out) != n:
        raise ValueError("out must have the rows of q")
    wp, wb = _kv_workspace(workspace, dev)
    rc = _lib.flame_kv_extend(cfg, _kv_cache_for(cfg, cache, n_seqs, dev), _kv_rows(cfg, q, cfg.n_q_heads, dev, "q"), _kv_ints(q_offsets, n_seqs + 1, dev, "q_offsets"),
                              _kv_ints(kv_lens, n_seqs, dev, "kv_lens"), n_seqs, n, _kv_rows(cfg, out, cfg.n_q_heads, dev, "out", True), wp, wb,
                              None if faults is None else _kv_ints(faults, 1, dev, "faults"), _kv_stream(stream, dev))
    if rc:
        _kv_check(rc)


def flame_kv_decode(cfg, cache, q, kv_lens, out, workspace=None, faults=None, stream=None) -> None:
    """q, out: device rows [n_seqs, n_q_heads, head_dim], one new token of every sequence; kv_lens: device int32 [n_seqs];
    workspace: device tensor of flame_kv_workspace_bytes bytes for these sequences or for more."""
    n_seqs, dev = len(kv_lens), torch.cuda.current_device()
    if len(q) != n_seqs or len(out) != n_seqs:
        raise ValueError("q and out must have one row per sequence")
    wp, wb = _kv_workspace(workspace, dev)
    rc = _lib.flame_kv_decode(cfg, _kv_cache_for(cfg, cache, n_seqs, dev), _kv_rows(cfg, q, cfg.n_q_heads, dev, "q"), _kv_ints(kv_lens, n_seqs, dev, "kv_lens"), n_seqs,
                              _kv_rows(cfg, out, cfg.n_q_heads, dev, "out", True), wp, wb, None if faults is None else _kv_ints(faults, 1, dev, "faults"), _kv_stream(stream, dev))
    if rc:
        _kv_check(rc)


def flame_kv_shared_workspace_bytes(cfg: flame_kv_config, n_groups: int, n_seqs: int, n_tokens: Optional[int] = None) -> int:
    """Bytes of a workspace for every flame_kv_shared and flame_kvq_shared of up to this many groups, sequences and query rows (n_tokens None: one row each)."""
    out = C.c_int64(0)
    _kv_check(_lib.flame_kv_shared_workspace_bytes(C.byref(cfg), n_groups, n_seqs, n_seqs if n_tokens is None else n_tokens, C.byref(out)))
    return out.value


def _kv_shared(call, cfg, cache, q, q_offsets, kv_lens, group_offsets, prefix_lens, out, workspace, faults, stream) -> None:
    n_seqs, n_groups, n, dev = len(kv_lens), len(group_offsets) - 1, len(q), torch.cuda.current_device()
    if len(out) != n or (q_offsets is None and n != n_seqs):
        raise ValueError("out must have the rows of q, and without q_offsets those are one per sequence")
    wp, wb = _kv_workspace(workspace, dev)
    groups = flame_kv_groups(_kv_ints(group_offsets, n_groups + 1, dev, "group_offsets"), _kv_ints(prefix_lens, n_seqs, dev, "prefix_lens"), n_groups)
    rc = call(cfg, cache, _kv_rows(cfg, q, cfg.n_q_heads, dev, "q"), None if q_offsets is None else _kv_ints(q_offsets, n_seqs + 1, dev, "q_offsets"), _kv_ints(kv_lens, n_seqs, dev, "kv_lens"),
              C.byref(groups), n_seqs, n, _kv_rows(cfg, out, cfg.n_q_heads, dev, "out", True), wp, wb, None if faults is None else _kv_ints(faults, 1, dev, "faults"), _kv_stream(stream, dev))
    if rc:
        _kv_check(rc)


def flame_kv_shared(cfg, cache, q, q_offsets, kv_lens, group_offsets, prefix_lens, out, workspace=None, faults=None, stream=None) -> None:
    """flame_kv_extend (q_offsets None: flame_kv_decode) for groups of sequences that begin with the same tokens: sequences group_offsets[g]..group_offsets[g + 1] share their first
    prefix_lens[b] tokens with the first of them.  group_offsets [n_groups + 1], prefix_lens [n_seqs]: device int32; workspace: of flame_kv_shared_workspace_bytes bytes."""
    _kv_shared(_lib.flame_kv_shared, cfg, _kv_cache_for(cfg, cache, len(kv_lens), torch.cuda.current_device()), q, q_offsets, kv_lens, group_offsets, prefix_lens, out, workspace, faults, stream)


# ---------------------------------------------------------------------------------------------
# the cache in 8 or 4 bits (include/flame_kvq.h)
# ---------------------------------------------------------------------------------------------
FLAME_KVQ_F8, FLAME_KVQ_F4 = 1, 2
_KVQ_FORMS = {"f8": FLAME_KVQ_F8, "f4": FLAME_KVQ_F4}


def make_kvq_pool(cfg: flame_kv_config, form, n_pages: int, page_size: int, device="cuda:0"):
    """k_pool, v_pool, k_scales, v_scales of zeros for pack_kvq_cache: uint8 [n_pages, page_size, n_kv_heads, head_dim (f8) or head_dim / 2 (f4)] and [..., head_dim / 32]."""
    row = cfg.head_dim // {FLAME_KVQ_F8: 1, FLAME_KVQ_F4: 2}[_KVQ_FORMS.get(form, form)]
    shapes = [(n_pages, page_size, cfg.n_kv_heads, row)] * 2 + [(n_pages, page_size, cfg.n_kv_heads, cfg.head_dim // 32)] * 2
    return tuple(torch.zeros(s, dtype=torch.uint8, device=device) for s in shapes)


def pack_kvq_cache(cfg: flame_kv_config, form, k_pool, v_pool, k_scales, v_scales, page_table) -> flame_kvq_cache:
    """form: "f8" or "f4"; pools: device uint8 [n_pages, page_size, n_kv_heads, head_dim (f8) or head_dim / 2 (f4)] (any strides, the same for both, a head's bytes side by side and the other
    strides multiples of them); scales: uint8 [n_pages, page_size, n_kv_heads, head_dim / 32], with strides that are the pools' by 32 (f8) or 16 (f4); page_table: device int32
    [n_seqs, pages_per_seq].  The struct keeps the tensors alive; their contents may change."""
    form = _KVQ_FORMS.get(form, form)
    if form not in (FLAME_KVQ_F8, FLAME_KVQ_F4) or cfg.torch_dtype is None:
        raise ValueError('form must be "f8" or "f4", and the configuration one of make_kv_config')
    bits = 8 if form == FLAME_KVQ_F8 else 4
    n_pages, page_size, heads, row = k_pool.shape
    if heads != cfg.n_kv_heads or row * 8 != cfg.head_dim * bits or k_pool.dtype is not torch.uint8:
        raise ValueError(f"k_pool must be [n_pages, page_size, {cfg.n_kv_heads}, {cfg.head_dim * bits // 8}] of torch.uint8")
    if v_pool.shape != k_pool.shape or v_pool.dtype is not torch.uint8 or v_pool.device != k_pool.device:
        raise ValueError("v_pool must be like k_pool")
    for t in (k_scales, v_scales):
        if tuple(t.shape) != (n_pages, page_size, heads, cfg.head_dim // 32) or t.dtype is not torch.uint8 or t.device != k_pool.device:
            raise ValueError(f"scales must be [n_pages, page_size, {heads}, {cfg.head_dim // 32}] of torch.uint8 beside the pools")
    if page_table.dtype is not torch.int32 or page_table.dim() != 2 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
        raise ValueError("page_table must be int32 [n_seqs, pages_per_seq], the entries of a row side by side")
    if not k_pool.is_cuda or page_table.device != k_pool.device:
        raise ValueError("the pools and the page table must be on one device")
    used = [i for i in range(3) if k_pool.shape[i] > 1]
    if [k_pool.stride(i) for i in used] != [v_pool.stride(i) for i in used] or k_pool.stride(3) != 1 or v_pool.stride(3) != 1:
        raise ValueError("k_pool and v_pool must have the same strides, and a head's bytes side by side")
    if any(k_pool.stride(i) == 0 for i in used):
        raise ValueError("the pools must not be expanded tensors")
    for t in (k_scales, v_scales):
        if [t.stride(i) * bits * 4 for i in used] != [k_pool.stride(i) for i in used] or (t.shape[3] > 1 and t.stride(3) != 1):
            raise ValueError("the scales' strides must be the pools' by 32 (f8) or 16 (f4), and a head's scales side by side")
    stride = [k_pool.stride(i) if k_pool.shape[i] > 1 else 0 for i in range(3)]
    c = flame_kvq_cache(form, k_pool.data_ptr(), v_pool.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(), *stride, n_pages, page_size, page_table.data_ptr(),
                        page_table.stride(0) if page_table.shape[0] > 1 else 0, page_table.shape[1])
    c.tensors = (k_pool, v_pool, k_scales, v_scales, page_table)
    c.n_seqs, c.device, c.shape = page_table.shape[0], k_pool.get_device(), (cfg.dtype, heads, cfg.head_dim)
    return c


def flame_kvq_append(cfg, cache, k, v, offsets, kv_lens, q=None, q_out=None, rotation=None, faults=None, stream=None) -> None:
    """flame_kv_append into a cache of pack_kvq_cache: keys and values are quantised as they are written."""
    n_seqs, n, dev = len(kv_lens), len(k), torch.cuda.current_device()
    if len(v) != n or (q is None) != (q_out is None) or (q is not None and not len(q) == len(q_out) == n):
        raise ValueError("k, v, q and q_out must have the same rows, and q comes with q_out")
    rc = _lib.flame_kvq_append(cfg, _kv_cache_for(cfg, cache, n_seqs, dev), _kv_rows(cfg, k, cfg.n_kv_heads, dev, "k"), _kv_rows(cfg, v, cfg.n_kv_heads, dev, "v"),
                               None if q is None else _kv_rows(cfg, q, cfg.n_q_heads, dev, "q"), None if q is None else _kv_rows(cfg, q_out, cfg.n_q_heads, dev, "q_out", True),
                               rotation, _kv_ints(offsets, n_seqs + 1, dev, "offsets"), _kv_ints(kv_lens, n_seqs, dev, "kv_lens"), n_seqs, n,
                               None if faults is None else _kv_ints(faults, 1, dev, "faults"), _kv_stream(stream, dev))
    if rc:
        _kv_check(rc)


def flame_kvq_read(cfg, cache, offsets, kv_lens, k, v, faults=None, stream=None) -> None:
    """k, v: device rows [n_tokens, n_kv_heads, head_dim], written: rows offsets[b]..offsets[b + 1] are the tokens of sequence b up to its kv_lens[b]-th, as the cache holds them."""
    n_seqs, n, dev = len(kv_lens), len(k), torch.cuda.current_device()
    if len(v) != n:
        raise ValueError("k and v must have the same rows")
    rc = _lib.flame_kvq_read(cfg, _kv_cache_for(cfg, cache, n_seqs, dev), _kv_ints(offsets, n_seqs + 1, dev, "offsets"), _kv_ints(kv_lens, n_seqs, dev, "kv_lens"), n_seqs, n,
                             _kv_rows(cfg, k, cfg.n_kv_heads, dev, "k", True), _kv_rows(cfg, v, cfg.n_kv_heads, dev, "v", True),
                             None if faults is None else _kv_ints(faults, 1, dev, "faults"), _kv_stream(stream, dev))
    if rc:
        _kv_check(rc)


def flame_kvq_extend(cfg, cache, q, q_offsets, kv_lens, out, workspace=None, faults=None, stream=None) -> None:
    """flame_kv_extend over a cache of pack_kvq_cache (workspace: flame_kv_workspace_bytes)."""
    n_seqs, n, dev = len(kv_lens), len(q), torch.cuda.current_device()
    if len(out) != n:
        raise ValueError("out must have the rows of q")
    wp, wb = _kv_workspace(workspace, dev)
    rc = _lib.flame_kvq_extend(cfg, _kv_cache_for(cfg, cache, n_seqs, dev), _kv_rows(cfg, q, cfg.n_q_heads, dev, "q"), _kv_ints(q_offsets, n_seqs + 1, dev, "q_offsets"),
                               _kv_ints(kv_lens, n_seqs, dev, "kv_lens"), n_seqs, n, _kv_rows(cfg, out, cfg.n_q_heads, dev, "out", True), wp, wb,
                               None if faults is None else _kv_ints(faults, 1, dev, "faults"), _kv_stream(stream, dev))
    if rc:
        _kv_check(rc)


def flame_kvq_decode(cfg, cache, q, kv_lens, out, workspace=None, faults=None, stream=None) -> None:
    """flame_kv_decode over a cache of pack_kvq_cache (workspace: flame_kv_workspace_bytes)."""
    n_seqs, dev = len(kv_lens), torch.cuda.current_device()
    if len(q) != n_seqs or len(out) != n_seqs:
        raise ValueError("q and out must have one row per sequence")
    wp, wb = _kv_workspace(workspace, dev)
    rc = _lib.flame_kvq_decode(cfg, _kv_cache_for(cfg, cache, n_seqs, dev), _kv_rows(cfg, q, cfg.n_q_heads, dev, "q"), _kv_ints(kv_lens, n_seqs, dev, "kv_lens"), n_seqs,
                               _kv_rows(cfg, out, cfg.n_q_heads, dev, "out", True), wp, wb, None if faults is None else _kv_ints(faults, 1, dev, "faults"), _kv_stream(stream, dev))
    if rc:
        _kv_check(rc)


def flame_kvq_shared(cfg, cache, q, q_offsets, kv_lens, group_offsets, prefix_lens, out, workspace=None, faults=None, stream=None) -> None:
    """flame_kv_shared over a cache of pack_kvq_cache."""
    _kv_shared(_lib.flame_kvq_shared, cfg, _kv_cache_for(cfg, cache, len(kv_lens), torch.cuda.current_device()), q, q_offsets, kv_lens, group_offsets, prefix_lens, out, workspace, faults, stream)


# ---------------------------------------------------------------------------------------------
# marshalling of a numpy workload into device tensors
# ---------------------------------------------------------------------------------------------
def to_device(workload, device="cuda:0"):
    """Upload a workloads.Workload: returns (cfg struct fields dict, weights dict, hist, cand) as
    torch tensors of the workload's storage dtype (bf16 values are already exactly representable)."""
    dt = torch.bfloat16 if workload.cfg.dtype == "bf16" else torch.float32

    def up(a, dtype=dt):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device=device, dtype=dtype)

    w = workload.weights
    dw = {k: up(w[k]) for k in ("w1", "b1", "ln_g", "ln_b", "w2", "b2", "w_s")}
    dw["rab"] = up(w["rab"], torch.float32)
    dw["b_s"] = float(w["b_s"])
    if "temperature" in w:
        dw["temperature"] = up(w["temperature"], torch.float32)
    return dw, up(workload.history_emb), up(workload.cand_emb)


def config_for(workload, *, n_streams=0, max_seq_tokens=0, slack_requests=0, kv_cache=0, slack_tokens=0,
               latency_mode=0, weights_static=0) -> flame_gr_config:
    c = workload.cfg
    tot = int(workload.history_offsets[-1]) + int(workload.cand_offsets[-1])
    return make_config(c.n_layers, c.d_model, c.n_heads, c.n_buckets, c.max_rel_dist, c.dtype,
                       ln_eps=c.ln_eps, attn_scale=c.attn_scale,
                       max_requests=workload.n_requests + slack_requests, max_total_tokens=tot + slack_tokens,
                       max_seq_tokens=max_seq_tokens, n_streams=n_streams, kv_cache=kv_cache,
                       attn_kind=getattr(c, "attn_kind", "silu"), latency_mode=latency_mode, weights_static=weights_static)
