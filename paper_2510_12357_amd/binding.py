"""ctypes front end of ``libmobile_moe.so`` -- argument marshalling only.

Every function has the name and argument order of its C entry point in
``include/mobile_moe.h``; tensors are torch tensors (device memory and streams are all that
torch is used for) and are passed down as raw pointers.  Nothing is computed in Python, and
there is no fallback: if the HIP library is missing, loading fails with an error.
"""
from __future__ import annotations

import ctypes
import math
import os
import threading
from typing import Optional, Sequence

import torch

from .workloads import LayerConfig

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmobile_moe.so")

MOE_BF16, MOE_FP32, MOE_BF16_W8, MOE_BF16_MXFP4 = 0, 1, 2, 3
MOE_FETCH_DEMAND, MOE_FETCH_PREFETCH = 0, 1
MOE_MAX_SHARED = 4
MOE_INT8_MAX_K, MOE_MAX_ALTERNATIVES, MOE_MAX_GIVEN = 131071, 32, 64
MOE_E4M3 = 4
MOE_ROPE_HALF, MOE_ROPE_INTERLEAVED = 0, 1
MOE_MAX_HEAD_DIM, MOE_ATTENTION_COUNTERS = 256, 16384
MOE_OK = 0
ERRORS = {-1: "MOE_E_BADARG", -2: "MOE_E_SHAPE", -3: "MOE_E_UNSUPPORTED", -4: "MOE_E_HIP",
          -5: "MOE_E_CACHE_FULL", -6: "MOE_E_WORKSPACE"}

EXPORTS = ("moe_last_error", "moe_device_info", "moe_profile_enable", "moe_profile_read", "moe_profile_plain_read", "moe_profile_expert_ffn", "moe_profile_expert_ffn_kernel", "moe_route",
           "moe_token_confidence", "moe_dispatch_workspace_bytes", "moe_dispatch", "moe_dispatch_from", "moe_combine_add",
           "moe_expert_ffn_workspace_bytes", "moe_expert_blob_bytes",
           "moe_shared_out_slabs", "moe_layer_decode_workspace_bytes", "moe_layer_decode_init",
           "moe_layer_decode_status", "moe_layer_decode", "moe_layer_step", "moe_layer_fallback", "moe_expert_ffn", "moe_expert_ffn_static", "moe_expert_ffn_static_max_bytes",
           "moe_combine", "moe_cache_create", "moe_cache_destroy",
           "moe_cache_expert_table", "expert_cache_fetch", "moe_expert_ffn_cached", "moe_cache_snapshot", "moe_cache_sync",
           "moe_cache_set_prefetch_limit", "moe_cache_emulate_link", "moe_prefetcher_create", "moe_prefetcher_destroy",
           "moe_prefetcher_set_in_flight_limit", "moe_prefetcher_set_yield_to_demand", "moe_prefetcher_predict", "moe_prefetcher_predicted",
           "moe_prefetcher_advance", "moe_quantize_rows", "moe_matmul_int8", "moe_linear_int8_workspace_bytes", "moe_linear_int8",
           "moe_token_logprobs_workspace_bytes", "moe_token_logprobs", "moe_rope", "moe_kv_append",
           "moe_paged_attention_workspace_bytes", "moe_paged_attention")


class MoeError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERRORS.get(code, code)}: {msg}")
        self.code = code


class moe_config(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("H", ctypes.c_int32), ("E", ctypes.c_int32),
                ("I", ctypes.c_int32), ("k_big", ctypes.c_int32), ("k_little", ctypes.c_int32),
                ("n_shared", ctypes.c_int32), ("shared_I", ctypes.c_int32 * MOE_MAX_SHARED),
                ("dtype", ctypes.c_int32), ("renorm", ctypes.c_int32), ("gamma", ctypes.c_float)]


class moe_step_buffers(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("logits", "topk_idx", "topk_w", "important", "k_t", "expert_offsets", "sorted_token",
                                               "sorted_rank", "inv_pos", "y", "shared_out", "out")] + [
        ("dispatch_ws", ctypes.c_void_p), ("dispatch_ws_bytes", ctypes.c_size_t),
        ("ffn_ws", ctypes.c_void_p), ("ffn_ws_bytes", ctypes.c_size_t)]


class moe_int8_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "N", "K", "x_dtype", "out_dtype", "reserved")] + [
        (n, ctypes.c_int64) for n in ("ldx", "ldw", "ldo")]


class moe_logprobs_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "V", "dtype", "n_given", "n_top", "reserved")] + [("ld", ctypes.c_int64)]


class moe_rope_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "heads", "D", "rotary_dim", "dtype", "layout", "inverse")] + [("mscale", ctypes.c_float)] + [
        (n, ctypes.c_int64) for n in ("x_token", "x_head", "out_token", "out_head")]


class moe_kv_cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "heads", "D", "dtype", "reserved")] + [
        (n, ctypes.c_int64) for n in ("page", "head", "row")] + [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")]


class moe_append_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "heads", "rotary_dim", "dtype", "layout", "n_seqs", "table_len")] + [("mscale", ctypes.c_float)] + [
        (n, ctypes.c_int64) for n in ("table_ld", "q_token", "q_head", "k_token", "k_head", "v_token", "v_head", "out_token", "out_head")]


class moe_attention_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "heads", "dtype", "max_len", "window", "table_len")] + [
        ("scale", ctypes.c_float), ("softcap", ctypes.c_float)] + [(n, ctypes.c_int64) for n in ("table_ld", "q_token", "q_head", "out_token", "out_head")]


class moe_fetch_stats(ctypes.Structure):
    _fields_ = [("hits", ctypes.c_int32), ("misses", ctypes.c_int32), ("dropped", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("bytes_h2d", ctypes.c_uint64)]


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads the HIP library; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2510_12357_amd.build` (hipcc, gfx950)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    cfgp = ctypes.POINTER(moe_config)
    lib.moe_last_error.restype = ctypes.c_char_p
    lib.moe_last_error.argtypes = []
    lib.moe_device_info.argtypes = [ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.moe_profile_enable.argtypes = [ctypes.c_int]
    lib.moe_profile_read.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_int64),
                                     ctypes.POINTER(ctypes.c_double)]
    lib.moe_profile_plain_read.argtypes = [vp, sz, vp, vp]
    lib.moe_profile_expert_ffn.argtypes = [cfgp, ctypes.c_int, ctypes.c_int, vp, vp, vp, vp, ctypes.POINTER(vp), ctypes.c_int,
                                           ctypes.c_int, vp, vp, vp, sz, vp]
    lib.moe_profile_expert_ffn.restype = ctypes.c_int
    lib.moe_profile_expert_ffn_kernel.argtypes = [cfgp, ctypes.c_int, ctypes.c_int]
    lib.moe_profile_expert_ffn_kernel.restype = ctypes.c_int
    lib.moe_route.argtypes = [cfgp, vp, vp, vp, vp, vp, ctypes.c_int, vp, vp, vp, vp, vp]
    lib.moe_token_confidence.argtypes = [vp, i32, i32, vp, vp]
    lib.moe_dispatch_workspace_bytes.argtypes = [cfgp]
    lib.moe_dispatch_workspace_bytes.restype = sz
    lib.moe_dispatch.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.moe_dispatch_from.argtypes = [cfgp, vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.moe_combine_add.argtypes = [cfgp, vp, vp, vp, vp, i32, vp, vp]
    lib.moe_expert_ffn_workspace_bytes.argtypes = [cfgp]
    lib.moe_expert_ffn_workspace_bytes.restype = sz
    lib.moe_expert_blob_bytes.argtypes = [cfgp, i32]
    lib.moe_expert_blob_bytes.restype = sz
    lib.moe_shared_out_slabs.argtypes = [cfgp]
    lib.moe_shared_out_slabs.restype = i32
    lib.moe_expert_ffn.argtypes = [cfgp, vp, vp, vp, vp, ctypes.POINTER(vp), ctypes.c_int,
                                   ctypes.c_int, vp, vp, vp, sz, vp]
    lib.moe_layer_decode_workspace_bytes.argtypes = [cfgp]
    lib.moe_layer_decode_workspace_bytes.restype = sz
    lib.moe_layer_decode_init.argtypes = [vp, sz, vp]
    lib.moe_layer_decode_init.restype = ctypes.c_int
    lib.moe_layer_decode_status.argtypes = [vp, ctypes.POINTER(i32)]
    lib.moe_layer_decode_status.restype = ctypes.c_int
    lib.moe_layer_decode.argtypes = [cfgp, vp, vp, vp, vp, vp, ctypes.POINTER(vp), vp, ctypes.c_int] + [vp] * 11 + [
        vp, sz, vp]
    lib.moe_layer_decode.restype = ctypes.c_int
    lib.moe_layer_step.argtypes = [cfgp, vp, vp, vp, vp, vp, ctypes.POINTER(vp), ctypes.c_int, ctypes.POINTER(moe_step_buffers), vp]
    lib.moe_layer_step.restype = ctypes.c_int
    lib.moe_layer_fallback.argtypes = [cfgp, vp, vp, vp, ctypes.POINTER(moe_step_buffers), vp]
    lib.moe_layer_fallback.restype = ctypes.c_int
    lib.moe_expert_ffn_static.argtypes = [cfgp, vp, vp, vp, vp, ctypes.POINTER(vp), ctypes.c_int,
                                          ctypes.c_int, vp, vp, vp]
    lib.moe_expert_ffn_static.restype = ctypes.c_int
    lib.moe_expert_ffn_static_max_bytes.argtypes = []
    lib.moe_expert_ffn_static_max_bytes.restype = sz
    lib.moe_combine.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp]
    lib.moe_cache_create.argtypes = [i32, sz, i32, vp, vp]
    lib.moe_cache_create.restype = vp
    lib.moe_cache_destroy.argtypes = [vp]
    lib.moe_cache_destroy.restype = None
    lib.moe_cache_expert_table.argtypes = [vp]
    lib.moe_cache_expert_table.restype = vp
    lib.expert_cache_fetch.argtypes = [vp, ctypes.POINTER(i32), i32, i32, ctypes.POINTER(i32),
                                       ctypes.POINTER(moe_fetch_stats), vp]
    lib.moe_expert_ffn_cached.argtypes = [cfgp, vp, vp, vp, vp, ctypes.POINTER(vp), vp, vp, vp, sz,
                                          ctypes.POINTER(moe_fetch_stats), ctypes.POINTER(i32), vp]
    lib.moe_cache_snapshot.argtypes = [vp, ctypes.POINTER(i32)]
    lib.moe_cache_sync.argtypes = [vp]
    lib.moe_cache_set_prefetch_limit.argtypes = [vp, i32]
    lib.moe_cache_emulate_link.argtypes = [vp, ctypes.c_double]
    lib.moe_prefetcher_create.argtypes = [i32, ctypes.POINTER(vp), i32]
    lib.moe_prefetcher_create.restype = vp
    lib.moe_prefetcher_destroy.argtypes = [vp]
    lib.moe_prefetcher_destroy.restype = None
    lib.moe_prefetcher_set_in_flight_limit.argtypes = [vp, i32]
    lib.moe_prefetcher_set_yield_to_demand.argtypes = [vp, i32]
    lib.moe_prefetcher_predict.argtypes = [vp, ctypes.POINTER(vp), i32, ctypes.POINTER(i32), i32, vp]
    lib.moe_prefetcher_predicted.argtypes = [vp, i32, ctypes.POINTER(i32)]
    lib.moe_prefetcher_advance.argtypes = [vp, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32),
                                           ctypes.POINTER(moe_fetch_stats), vp]
    for name in ("moe_prefetcher_set_in_flight_limit", "moe_prefetcher_set_yield_to_demand", "moe_prefetcher_predict", "moe_prefetcher_predicted",
                 "moe_prefetcher_advance"):
        getattr(lib, name).restype = ctypes.c_int
    for name in ("moe_device_info", "moe_profile_enable", "moe_profile_read", "moe_profile_plain_read", "moe_route", "moe_token_confidence", "moe_dispatch",
                 "moe_dispatch_from", "moe_combine_add",
                 "moe_expert_ffn", "moe_combine", "expert_cache_fetch", "moe_expert_ffn_cached", "moe_cache_snapshot",
                 "moe_cache_sync", "moe_cache_set_prefetch_limit", "moe_cache_emulate_link"):
        getattr(lib, name).restype = ctypes.c_int
    i64 = ctypes.c_int64
    lib.moe_quantize_rows.argtypes = [vp, i32, i32, i32, i64, vp, i64, vp, vp]
    lib.moe_matmul_int8.argtypes = [ctypes.POINTER(moe_int8_config), vp, vp, vp, vp, vp, vp, vp]
    lib.moe_linear_int8_workspace_bytes.argtypes = [ctypes.POINTER(moe_int8_config)]
    lib.moe_linear_int8_workspace_bytes.restype = sz
    lib.moe_linear_int8.argtypes = [ctypes.POINTER(moe_int8_config), vp, vp, vp, vp, vp, vp, sz, vp]
    lib.moe_token_logprobs_workspace_bytes.argtypes = [ctypes.POINTER(moe_logprobs_config)]
    lib.moe_token_logprobs_workspace_bytes.restype = sz
    lib.moe_token_logprobs.argtypes = [ctypes.POINTER(moe_logprobs_config)] + [vp] * 8 + [sz, vp]
    kvp = ctypes.POINTER(moe_kv_cache)
    lib.moe_rope.argtypes = [ctypes.POINTER(moe_rope_config)] + [vp] * 5
    lib.moe_kv_append.argtypes = [ctypes.POINTER(moe_append_config), kvp] + [vp] * 9
    lib.moe_paged_attention_workspace_bytes.argtypes = [ctypes.POINTER(moe_attention_config), kvp]
    lib.moe_paged_attention_workspace_bytes.restype = sz
    lib.moe_paged_attention.argtypes = [ctypes.POINTER(moe_attention_config), kvp] + [vp] * 6 + [sz, vp, vp]
    for name in ("moe_quantize_rows", "moe_matmul_int8", "moe_linear_int8", "moe_token_logprobs", "moe_rope", "moe_kv_append", "moe_paged_attention"):
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _check(rc: int) -> None:
    if rc != MOE_OK:
        raise MoeError(rc, load_library().moe_last_error().decode())


def make_config(cfg: LayerConfig, T: Optional[int] = None) -> moe_config:
    c = moe_config()
    c.T = cfg.T if T is None else T
    c.H, c.E, c.I, c.k_big, c.k_little = cfg.H, cfg.E, cfg.I, cfg.k_big, cfg.k_little
    c.n_shared = len(cfg.shared_I)
    for i, v in enumerate(cfg.shared_I):
        c.shared_I[i] = v
    c.dtype = {"bf16": MOE_BF16, "fp32": MOE_FP32, "bf16w8": MOE_BF16_W8, "bf16mx4": MOE_BF16_MXFP4}[cfg.dtype]
    c.renorm = int(cfg.renorm)
    c.gamma = cfg.gamma
    return c


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_contiguous(), "tensors passed to the C ABI must be dense"
    return ctypes.c_void_p(t.data_ptr())


def _addr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_contiguous(), "tensors passed to the C ABI must be dense"
    return t.data_ptr()


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    if isinstance(stream, torch.cuda.Stream):
        return ctypes.c_void_p(stream.cuda_stream)
    return ctypes.c_void_p(int(stream))


# ------------------------------------------------------------------------------ entry points
def moe_last_error() -> str:
    return load_library().moe_last_error().decode()


def moe_device_info():
    n_cu, is950 = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(load_library().moe_device_info(ctypes.byref(n_cu), ctypes.byref(is950)))
    return n_cu.value, bool(is950.value)


PROFILE_KINDS = ("router_gemm", "route_topk", "dispatch", "ffn_gate_up", "ffn_down", "combine",
                 "token_confidence", "decode_step", "quantize_rows", "int8_product", "token_logprobs")


def moe_profile_enable(on: bool) -> None:
    _check(load_library().moe_profile_enable(int(bool(on))))


def moe_profile_plain_read(buf, sink) -> None:
    """One plain streaming read of the tensor `buf` on the current stream (measurement aid)."""
    _check(load_library().moe_profile_plain_read(buf.data_ptr(), buf.numel() * buf.element_size(), sink.data_ptr(), _stream(None)))


def moe_profile_read(kind: int):
    """-> (launch sites recorded, summed duration in ms) of one kernel kind"""
    n, ms = ctypes.c_int64(0), ctypes.c_double(0.0)
    _check(load_library().moe_profile_read(kind, ctypes.byref(n), ctypes.byref(ms)))
    return n.value, ms.value


def moe_route(cfg: moe_config, x, Wg, gate_bias, conf, logits, logits_given, topk_idx, topk_w,
              important, k_t, stream=None) -> None:
    _check(load_library().moe_route(ctypes.byref(cfg), _ptr(x), _ptr(Wg), _ptr(gate_bias), _ptr(conf),
                                    _ptr(logits), int(bool(logits_given)), _ptr(topk_idx),
                                    _ptr(topk_w), _ptr(important), _ptr(k_t), _stream(stream)))


def moe_token_confidence(lm_logits, T: int, V: int, conf, stream=None) -> None:
    _check(load_library().moe_token_confidence(_ptr(lm_logits), T, V, _ptr(conf), _stream(stream)))


def moe_dispatch_workspace_bytes(cfg: moe_config) -> int:
    return int(load_library().moe_dispatch_workspace_bytes(ctypes.byref(cfg)))


def moe_dispatch(cfg: moe_config, topk_idx, k_t, expert_offsets, sorted_token, sorted_rank,
                 inv_pos, ws, ws_bytes: int, stream=None) -> None:
    _check(load_library().moe_dispatch(ctypes.byref(cfg), _ptr(topk_idx), _ptr(k_t),
                                       _ptr(expert_offsets), _ptr(sorted_token), _ptr(sorted_rank),
                                       _ptr(inv_pos), _ptr(ws), ws_bytes, _stream(stream)))


def moe_dispatch_from(cfg: moe_config, topk_idx, k_t, j_lo: int, expert_offsets, sorted_token, sorted_rank,
                      inv_pos, ws, ws_bytes: int, stream=None) -> None:
    _check(load_library().moe_dispatch_from(ctypes.byref(cfg), _ptr(topk_idx), _ptr(k_t), int(j_lo),
                                            _ptr(expert_offsets), _ptr(sorted_token), _ptr(sorted_rank),
                                            _ptr(inv_pos), _ptr(ws), ws_bytes, _stream(stream)))


def moe_combine_add(cfg: moe_config, y, topk_w, inv_pos, k_t, j_lo: int, out, stream=None) -> None:
    _check(load_library().moe_combine_add(ctypes.byref(cfg), _ptr(y), _ptr(topk_w), _ptr(inv_pos), _ptr(k_t),
                                          int(j_lo), _ptr(out), _stream(stream)))


def moe_expert_ffn_workspace_bytes(cfg: moe_config) -> int:
    return int(load_library().moe_expert_ffn_workspace_bytes(ctypes.byref(cfg)))


def moe_expert_blob_bytes(cfg: moe_config, I: int) -> int:
    return int(load_library().moe_expert_blob_bytes(ctypes.byref(cfg), I))


def moe_shared_out_slabs(cfg: moe_config) -> int:
    return int(load_library().moe_shared_out_slabs(ctypes.byref(cfg)))


def moe_expert_ffn(cfg: moe_config, x, expert_offsets, sorted_token, expert_w, shared_w: Sequence,
                   run_routed, run_shared, y, shared_out, ws, ws_bytes: int, stream=None) -> None:
    """expert_w: device int64 tensor [E] of blob addresses, or a raw device address (int);
    shared_w: sequence of device tensors (their addresses form the host pointer array)."""
    sw = (ctypes.c_void_p * max(1, len(shared_w)))(*[t.data_ptr() for t in shared_w])
    ew = ctypes.c_void_p(expert_w) if isinstance(expert_w, int) else _ptr(expert_w)
    _check(load_library().moe_expert_ffn(ctypes.byref(cfg), _ptr(x), _ptr(expert_offsets),
                                         _ptr(sorted_token), ew, sw, int(bool(run_routed)),
                                         int(bool(run_shared)), _ptr(y), _ptr(shared_out), _ptr(ws),
                                         ws_bytes, _stream(stream)))


def moe_profile_expert_ffn(cfg: moe_config, kernel: int, variant: int, x, expert_offsets, sorted_token, expert_w,
                           shared_w: Sequence, run_routed, run_shared, y, shared_out, ws, ws_bytes: int, stream=None) -> None:
    """moe_expert_ffn on a given kernel: 0 streamed (variant: token tiles per wave; 4, 5: rows of its own per wave, one or two tiles of them), 1 tiles of 128 x 256, 2 of
    256 x 256 (variant 1: by rows; on 1, narrow weights then in whole lines, and 2, 3: the same with bf16 weights past the caches and tiles that fill their rounds)."""
    sw = (ctypes.c_void_p * max(1, len(shared_w)))(*[t.data_ptr() for t in shared_w])
    ew = ctypes.c_void_p(expert_w) if isinstance(expert_w, int) else _ptr(expert_w)
    _check(load_library().moe_profile_expert_ffn(ctypes.byref(cfg), kernel, variant, _ptr(x), _ptr(expert_offsets),
                                                 _ptr(sorted_token), ew, sw, int(bool(run_routed)), int(bool(run_shared)),
                                                 _ptr(y), _ptr(shared_out), _ptr(ws), ws_bytes, _stream(stream)))


def moe_profile_expert_ffn_kernel(cfg: moe_config, run_routed=True, run_shared=True) -> int:
    rc = load_library().moe_profile_expert_ffn_kernel(ctypes.byref(cfg), int(bool(run_routed)), int(bool(run_shared)))
    if rc < 0:
        _check(rc)
    return rc


def moe_layer_decode_workspace_bytes(cfg: moe_config) -> int:
    return int(load_library().moe_layer_decode_workspace_bytes(ctypes.byref(cfg)))


def moe_layer_decode_init(ws, ws_bytes: int, stream=None) -> None:
    _check(load_library().moe_layer_decode_init(_ptr(ws), ws_bytes, _stream(stream)))


def moe_layer_decode_status(ws) -> int:
    """-> number of waits inside the kernel that have ever given up on this workspace (synchronises)"""
    n = ctypes.c_int32(0)
    _check(load_library().moe_layer_decode_status(_ptr(ws), ctypes.byref(n)))
    return n.value


def moe_layer_decode(cfg: moe_config, x, Wg, gate_bias, conf, expert_w, shared_w: Sequence, logits, logits_given,
                     topk_idx, topk_w, important, k_t, expert_offsets, sorted_token, sorted_rank, inv_pos, y,
                     shared_out, out, ws, ws_bytes: int, stream=None) -> None:
    sw = (ctypes.c_void_p * max(1, len(shared_w)))(*[t.data_ptr() for t in shared_w])
    ew = ctypes.c_void_p(expert_w) if isinstance(expert_w, int) else _ptr(expert_w)
    _check(load_library().moe_layer_decode(ctypes.byref(cfg), _ptr(x), _ptr(Wg), _ptr(gate_bias), _ptr(conf), ew, sw,
                                           _ptr(logits), int(bool(logits_given)), _ptr(topk_idx), _ptr(topk_w),
                                           _ptr(important), _ptr(k_t), _ptr(expert_offsets), _ptr(sorted_token),
                                           _ptr(sorted_rank), _ptr(inv_pos), _ptr(y), _ptr(shared_out), _ptr(out),
                                           _ptr(ws), ws_bytes, _stream(stream)))


def moe_expert_ffn_static_max_bytes() -> int:
    return int(load_library().moe_expert_ffn_static_max_bytes())


def moe_expert_ffn_static(cfg: moe_config, x, expert_offsets, sorted_token, expert_w, shared_w: Sequence,
                          run_routed, run_shared, y, shared_out, stream=None) -> None:
    """moe_expert_ffn without a workspace argument (the library's built-in scratch buffer)."""
    sw = (ctypes.c_void_p * max(1, len(shared_w)))(*[t.data_ptr() for t in shared_w])
    ew = ctypes.c_void_p(expert_w) if isinstance(expert_w, int) else _ptr(expert_w)
    _check(load_library().moe_expert_ffn_static(ctypes.byref(cfg), _ptr(x), _ptr(expert_offsets),
                                                _ptr(sorted_token), ew, sw, int(bool(run_routed)),
                                                int(bool(run_shared)), _ptr(y), _ptr(shared_out),
                                                _stream(stream)))


def moe_combine(cfg: moe_config, y, topk_w, inv_pos, k_t, shared_out, out, stream=None) -> None:
    _check(load_library().moe_combine(ctypes.byref(cfg), _ptr(y), _ptr(topk_w), _ptr(inv_pos),
                                      _ptr(k_t), _ptr(shared_out), _ptr(out), _stream(stream)))


def moe_layer_step(cfg: moe_config, x, Wg, gate_bias, conf, expert_w, shared_w: Sequence, logits_given, buffers: moe_step_buffers,
                   stream=None) -> None:
    sw = (ctypes.c_void_p * max(1, len(shared_w)))(*[t.data_ptr() for t in shared_w])
    ew = ctypes.c_void_p(expert_w) if isinstance(expert_w, int) else _ptr(expert_w)
    _check(load_library().moe_layer_step(ctypes.byref(cfg), _ptr(x), _ptr(Wg), _ptr(gate_bias), _ptr(conf), ew, sw,
                                         int(bool(logits_given)), ctypes.byref(buffers), _stream(stream)))


def moe_layer_fallback(cfg: moe_config, x, conf, expert_w, buffers: moe_step_buffers, stream=None) -> None:
    ew = ctypes.c_void_p(expert_w) if isinstance(expert_w, int) else _ptr(expert_w)
    _check(load_library().moe_layer_fallback(ctypes.byref(cfg), _ptr(x), _ptr(conf), ew, ctypes.byref(buffers), _stream(stream)))


def moe_cache_create(E: int, blob_bytes: int, n_slots: int, host_blobs: torch.Tensor,
                     device_slots: torch.Tensor) -> int:
    assert host_blobs.is_pinned(), "host arena must be pinned memory"
    h = load_library().moe_cache_create(E, blob_bytes, n_slots, _ptr(host_blobs), _ptr(device_slots))
    if not h:
        raise MoeError(-1, moe_last_error())
    return h


def moe_cache_destroy(cache: int) -> None:
    load_library().moe_cache_destroy(ctypes.c_void_p(cache))


def moe_cache_expert_table(cache: int) -> int:
    return int(load_library().moe_cache_expert_table(ctypes.c_void_p(cache)))


def expert_cache_fetch(cache: int, expert_ids: Sequence[int], mode: int, stream=None):
    """-> (slot_of list, moe_fetch_stats)"""
    n = len(expert_ids)
    ids = (ctypes.c_int32 * max(1, n))(*expert_ids)
    slots = (ctypes.c_int32 * max(1, n))()
    st = moe_fetch_stats()
    _check(load_library().expert_cache_fetch(ctypes.c_void_p(cache), ids, n, mode, slots,
                                             ctypes.byref(st), _stream(stream)))
    return list(slots[:n]), st


def moe_expert_ffn_cached(cfg: moe_config, cache: int, x, expert_offsets, sorted_token, shared_w: Sequence,
                          y, shared_out, ws, ws_bytes: int, stream=None):
    """-> (summed moe_fetch_stats, number of waves)"""
    sw = (ctypes.c_void_p * max(1, len(shared_w)))(*[t.data_ptr() for t in shared_w])
    st, nw = moe_fetch_stats(), ctypes.c_int32(0)
    _check(load_library().moe_expert_ffn_cached(ctypes.byref(cfg), ctypes.c_void_p(cache), _ptr(x),
                                                _ptr(expert_offsets), _ptr(sorted_token), sw, _ptr(y),
                                                _ptr(shared_out), _ptr(ws), ws_bytes, ctypes.byref(st),
                                                ctypes.byref(nw), _stream(stream)))
    return st, nw.value


def moe_cache_snapshot(cache: int, n_slots: int):
    out = (ctypes.c_int32 * n_slots)()
    rc = load_library().moe_cache_snapshot(ctypes.c_void_p(cache), out)
    if rc < 0:
        _check(rc)
    return list(out)


def moe_cache_sync(cache: int) -> None:
    _check(load_library().moe_cache_sync(ctypes.c_void_p(cache)))


def moe_cache_set_prefetch_limit(cache: int, max_copies_per_call: int) -> None:
    _check(load_library().moe_cache_set_prefetch_limit(ctypes.c_void_p(cache), int(max_copies_per_call)))


def moe_cache_emulate_link(cache: int, gb_per_s: float) -> None:
    _check(load_library().moe_cache_emulate_link(ctypes.c_void_p(cache), float(gb_per_s)))


def moe_prefetcher_create(caches: Sequence[int], k_big: int) -> int:
    arr = (ctypes.c_void_p * max(1, len(caches)))(*caches)
    h = load_library().moe_prefetcher_create(len(caches), arr, int(k_big))
    if not h:
        raise MoeError(-1, moe_last_error())
    return int(h)


def moe_prefetcher_destroy(p: int) -> None:
    load_library().moe_prefetcher_destroy(ctypes.c_void_p(p))


def moe_prefetcher_set_in_flight_limit(p: int, max_copies_in_flight: int) -> None:
    _check(load_library().moe_prefetcher_set_in_flight_limit(ctypes.c_void_p(p), int(max_copies_in_flight)))


def moe_prefetcher_set_yield_to_demand(p: int, on: bool) -> None:
    _check(load_library().moe_prefetcher_set_yield_to_demand(ctypes.c_void_p(p), 1 if on else 0))


def moe_prefetcher_predict(p: int, layer_logits: Sequence, T: int, rejected: Sequence[int], stream=None) -> None:
    """layer_logits: one device tensor [T, E] fp32 per layer."""
    ptrs = (ctypes.c_void_p * max(1, len(layer_logits)))(*[t.data_ptr() for t in layer_logits])
    n = len(rejected)
    rej = (ctypes.c_int32 * max(1, n))(*rejected)
    _check(load_library().moe_prefetcher_predict(ctypes.c_void_p(p), ptrs, int(T), rej, n, _stream(stream)))


def moe_prefetcher_predicted(p: int, layer: int, n_experts: int):
    out = (ctypes.c_int32 * n_experts)()
    rc = load_library().moe_prefetcher_predicted(ctypes.c_void_p(p), int(layer), out)
    if rc < 0:
        _check(rc)
    return list(out[:rc])


def moe_prefetcher_advance(p: int, layer: int, distance: int, n_layers: int, stream=None):
    """-> [(layer, limit the request ran under, moe_fetch_stats), ...] of the requests made"""
    ls, lim = (ctypes.c_int32 * n_layers)(), (ctypes.c_int32 * n_layers)()
    st = (moe_fetch_stats * n_layers)()
    rc = load_library().moe_prefetcher_advance(ctypes.c_void_p(p), int(layer), int(distance), ls, lim, st,
                                               _stream(stream))
    if rc < 0:
        _check(rc)
    return [(int(ls[i]), int(lim[i]), st[i]) for i in range(rc)]


def moe_quantize_rows(x, q, scale, stream=None) -> None:
    """x: [rows, K] float rows; q: int8 [rows, ldq] whole rows, ldq >= K a multiple of 16; scale: [rows] fp32."""
    if q.dim() != 2 or q.shape[0] != x.shape[0] or q.dtype != torch.int8 or not q.is_contiguous():
        raise ValueError("codes: int8 [rows, ldq], dense")
    if scale.dtype != torch.float32 or scale.numel() != x.shape[0]:
        raise ValueError("scales: fp32 [rows]")
    _ld(x), _on_one_gpu(x, q, scale)
    x = _near_rows(x, stream)
    args = _rows(x), _float_type(x), x.shape[0], x.shape[1], _ld(x), _ptr(q), q.shape[1], _ptr(scale)
    _check(load_library().moe_quantize_rows(*args, _stream(stream)))


def moe_matmul_int8(cfg: moe_int8_config, x, x_scale, w, w_scale, bias, out, stream=None) -> None:
    _on_one_gpu(x, x_scale, w, w_scale, bias, out)
    _check(load_library().moe_matmul_int8(ctypes.byref(cfg), _rows(x), _ptr(x_scale), _rows(w), _ptr(w_scale), _ptr(bias), _rows(out),
                                          _stream(stream)))


def moe_linear_int8_workspace_bytes(cfg: moe_int8_config) -> int:
    return int(load_library().moe_linear_int8_workspace_bytes(ctypes.byref(cfg)))


def moe_linear_int8(cfg: moe_int8_config, x, w, w_scale, bias, out, ws, ws_bytes: int, stream=None) -> None:
    _on_one_gpu(x, w, w_scale, bias, out, ws)
    _check(load_library().moe_linear_int8(ctypes.byref(cfg), _rows(x), _rows(w), _ptr(w_scale), _ptr(bias), _rows(out), _ptr(ws),
                                          ws_bytes, _stream(stream)))


def moe_token_logprobs_workspace_bytes(cfg: moe_logprobs_config) -> int:
    return int(load_library().moe_token_logprobs_workspace_bytes(ctypes.byref(cfg)))


def moe_token_logprobs(cfg: moe_logprobs_config, logits, tokens, token_logp, entropy, conf, top_idx, top_logp, ws, ws_bytes: int,
                       stream=None) -> None:
    _on_one_gpu(logits, tokens, token_logp, entropy, conf, top_idx, top_logp, ws)
    _check(load_library().moe_token_logprobs(ctypes.byref(cfg), _rows(logits), _ptr(tokens), _ptr(token_logp), _ptr(entropy), _ptr(conf),
                                             _ptr(top_idx), _ptr(top_logp), _ptr(ws), ws_bytes, _stream(stream)))


def moe_rope(cfg: moe_rope_config, x, pos, freq, out, stream=None) -> None:
    _on_one_gpu(x, pos, freq, out)
    _check(load_library().moe_rope(ctypes.byref(cfg), _heads_ptr(x), _ptr(pos), _ptr(freq), _heads_ptr(out), _stream(stream)))


def moe_kv_append(cfg: moe_append_config, cache: moe_kv_cache, q, k, v, pos, seq, table, freq, q_out, stream=None) -> None:
    _on_one_gpu(q, k, v, pos, seq, table, freq, q_out)
    _check(load_library().moe_kv_append(ctypes.byref(cfg), ctypes.byref(cache), _heads_ptr(q), _heads_ptr(k), _heads_ptr(v), _ptr(pos), _ptr(seq),
                                        _rows(table), _ptr(freq), _heads_ptr(q_out), _stream(stream)))


def moe_paged_attention_workspace_bytes(cfg: moe_attention_config, cache: moe_kv_cache) -> int:
    return int(load_library().moe_paged_attention_workspace_bytes(ctypes.byref(cfg), ctypes.byref(cache)))


def moe_paged_attention(cfg: moe_attention_config, cache: moe_kv_cache, q, table, lengths, out, lse, ws, ws_bytes: int, counters=None, stream=None) -> None:
    _on_one_gpu(q, table, lengths, out, lse, ws, counters)
    _check(load_library().moe_paged_attention(ctypes.byref(cfg), ctypes.byref(cache), _heads_ptr(q), _rows(table), _ptr(lengths), _heads_ptr(out),
                                              _ptr(lse), _ptr(ws), ws_bytes, _ptr(counters), _stream(stream)))


# ------------------------------------------------------------------------------ plumbing helpers
def _heads_ptr(t: Optional[torch.Tensor]):
    """Address of [tokens, heads, channels] whose channels are dense."""
    if t is None:
        return None
    assert t.dim() == 3 and (t.shape[2] <= 1 or t.stride(2) == 1), "channels passed to the C ABI must be dense"
    return ctypes.c_void_p(t.data_ptr())


def _rows(t: Optional[torch.Tensor]):
    """Address of a matrix whose rows are dense and may lie apart."""
    if t is None:
        return None
    assert t.dim() == 2 and (t.shape[1] <= 1 or t.stride(1) == 1), "rows passed to the C ABI must be dense"
    return ctypes.c_void_p(t.data_ptr())


_DEVICES = "tensors on more than one device, or not on a GPU"


def _on_one_gpu(*tensors: Optional[torch.Tensor]) -> None:
    """The kernels take addresses as they are."""
    devices = {t.device for t in tensors if t is not None}
    if len(devices) != 1 or devices.pop().type != "cuda":
        raise ValueError(_DEVICES)


# an expanded tensor's rows are 0 elements apart, which to the C ABI means dense rows
_SHARED_ROWS = "rows share memory: make them dense with contiguous()"
_MAX_LD = 1 << 22                                            # distances of rows that most calls stay below


def _ld(t: torch.Tensor) -> int:
    step, n = int(t.stride(0)), int(t.shape[1])
    if t.shape[0] <= 1:                                      # there is no next row: torch gives such a dimension any stride
        return max(step, n) if step < _MAX_LD else (n + 15) // 16 * 16
    if step < n:
        raise ValueError(_SHARED_ROWS)
    return step


def _near_rows(t: torch.Tensor, stream) -> torch.Tensor:
    """Rows that lie too far apart for a call (logits[:, -1] of a batch of prompts) as a dense copy, made on the stream that reads it."""
    if t.shape[0] <= 1 or t.stride(0) < _MAX_LD:
        return t
    with torch.cuda.stream(_torch_stream(stream)):
        return t.contiguous()


def _float_type(t: torch.Tensor) -> int:
    return {torch.bfloat16: MOE_BF16, torch.float32: MOE_FP32}[t.dtype]


def int8_config(x: torch.Tensor, w: torch.Tensor, out: torch.Tensor) -> moe_int8_config:
    """The description of out[T, N] = x[T, K] w[N, K]^T by the tensors' shapes, types and strides."""
    c = moe_int8_config()
    (c.T, c.K), c.N = x.shape, w.shape[0]
    assert w.shape[1] == c.K and tuple(out.shape) == (c.T, c.N), "shapes of x, w and out do not fit"
    c.x_dtype = MOE_BF16 if x.dtype == torch.int8 else _float_type(x)
    c.out_dtype = _float_type(out)
    c.ldx, c.ldw, c.ldo = _ld(x), _ld(w), _ld(out)
    return c


def quantize_rows(x: torch.Tensor, stream=None):
    """-> (codes int8 [rows, K], a view of rows padded to 16 bytes; scales fp32 [rows]) of float rows [rows, K].  They belong to `stream`: what reads
    them on another one has to be ordered behind it."""
    rows, K = x.shape
    _on_one_gpu(x)
    with torch.cuda.stream(_torch_stream(stream)):
        q = torch.empty((rows, (K + 15) // 16 * 16), dtype=torch.int8, device=x.device)
        scale = torch.empty((rows,), dtype=torch.float32, device=x.device)
    moe_quantize_rows(x, q, scale, stream)
    return q[:, :K], scale


def _torch_stream(stream, device: Optional[torch.device] = None) -> torch.cuda.Stream:
    """The stream as torch has it; None: the current one; of the current device or of the tensors' one."""
    if device is not None and device.type != "cuda":         # of the host: refused later
        device = None
    if stream is None:
        return torch.cuda.current_stream(device)
    return stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream), device=device)


def _raw_stream(stream, device: int) -> int:
    """The stream's handle as a number; None: torch's current stream of the device."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device)
    return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else int(stream)


class Int8Linear:
    """A projection with 8-bit weights: codes w [N, K] (rows padded to 16 bytes, as quantize_rows makes them), w_scale [N] and
    an optional bias [N] in fp32.  Calling it enqueues one product on `stream`; the workspace for float tokens is kept and
    grows with the largest call, so calls that may overlap (streams without order between them, a graph's replay among them) need
    an object each.  A captured graph reads the weights and a workspace of its object, which has to live as long as the graph; larger
    calls in between do not matter to it."""

    def __init__(self, w: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None):
        load_library()
        _rows(w)
        for name, t in (("w_scale", w_scale), ("bias", bias)):
            assert t is None or (t.dtype == torch.float32 and tuple(t.shape) == (w.shape[0],) and t.is_contiguous()), f"{name}: [N] fp32"
        assert w.dtype == torch.int8 and all(t is None or t.device == w.device for t in (w_scale, bias)), "int8 codes, all on one device"
        self._w, self._w_scale, self._bias = w, w_scale, bias
        self.ws = None
        self._streams = set()
        self._outgrown = []                                  # workspaces of smaller calls: captured graphs have their addresses
        self._calls = {}                                     # of each form of tokens and outputs: its description, workspace bytes

    w, w_scale, bias = property(lambda self: self._w), property(lambda self: self._w_scale), property(lambda self: self._bias)

    @classmethod
    def quantize(cls, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, stream=None) -> "Int8Linear":
        """From a float weight [N, K]."""
        return cls(*quantize_rows(weight, stream), bias)

    def _workspace(self, need: int, stream) -> int:
        if self.ws is None or self.ws.numel() < need:
            if self.ws is not None:                          # twice as large at least: what is kept stays below the one in use
                need = max(need, 2 * self.ws.numel())
                self._outgrown.append(self.ws)
            with torch.cuda.stream(_torch_stream(stream)):
                self.ws = torch.empty((need,), dtype=torch.uint8, device=self._w.device)
            self._streams.clear()
        return self.ws.data_ptr()

    def _used_on(self, stream, handle: int) -> None:
        """Memory belongs to the stream it was taken on: its reuse after the object's end waits for every other one that was here."""
        if handle not in self._streams:
            for t in (self._w, self._w_scale, self._bias, self.ws):
                if t is not None:
                    t.record_stream(_torch_stream(stream))
            self._streams.add(handle)

    def _call(self, x: torch.Tensor, out: torch.Tensor):
        """-> (description, workspace bytes) of a call with such tokens and outputs: the checks that their shapes, types and strides need."""
        _rows(x), _rows(out)
        _on_one_gpu(x, out, self._w)
        c = int8_config(x, self._w, out)
        need = 0 if x.dtype == torch.int8 else moe_linear_int8_workspace_bytes(c)
        if len(self._calls) > 256:                           # a server's batches are of any size
            self._calls.clear()
        return c, ctypes.byref(c), need

    def __call__(self, x: torch.Tensor, x_scale: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
        """x: float tokens [T, K], or their codes with x_scale [T].  out: [T, N] bf16 or fp32 (default: a new fp32 tensor)."""
        if out is None:
            with torch.cuda.stream(_torch_stream(stream)):
                out = torch.empty((x.shape[0], self._w.shape[0]), dtype=torch.float32, device=x.device)
        key = (x.shape, x.stride(), x.dtype, x.get_device(), out.shape, out.stride(), out.dtype, out.get_device())
        call = self._calls.get(key)
        if call is None:
            call = self._call(x, out)
            self._calls[key] = call
        _, c, need = call
        s = _raw_stream(stream, key[3])
        bias = None if self._bias is None else self._bias.data_ptr()
        ws = None if x.dtype is torch.int8 else self._workspace(need, stream)
        if s not in self._streams:
            self._used_on(stream, s)
        if x.dtype is torch.int8:
            assert x_scale is not None and x_scale.dtype is torch.float32 and x_scale.numel() == x.shape[0] and x_scale.is_contiguous(), \
                "codes come with their scales, [T] fp32"
            if x_scale.get_device() != key[3]:
                raise ValueError(_DEVICES)
            rc = _lib.moe_matmul_int8(c, x.data_ptr(), x_scale.data_ptr(), self._w.data_ptr(), self._w_scale.data_ptr(), bias, out.data_ptr(), s)
        else:
            rc = _lib.moe_linear_int8(c, x.data_ptr(), self._w.data_ptr(), self._w_scale.data_ptr(), bias, out.data_ptr(), ws, self.ws.numel(), s)
        if rc:
            _check(rc)
        return out


class LogprobBuffers:
    """Device buffers of moe_token_logprobs for T rows of V logits."""

    def __init__(self, T: int, n_given: int, n_top: int, V: int, device="cuda"):
        f32 = dict(dtype=torch.float32, device=device)
        self.T, self.V, self.n_given, self.n_top = T, V, n_given, n_top
        self.token_logp = torch.empty((T, n_given), **f32)
        self.entropy, self.conf = torch.empty((T,), **f32), torch.empty((T,), **f32)
        self.top_idx = torch.empty((T, n_top), dtype=torch.int32, device=device)
        self.top_logp = torch.empty((T, n_top), **f32)
        self.c = {}
        need = 0
        for dtype in (MOE_BF16, MOE_FP32):
            c = self.c[dtype] = moe_logprobs_config()
            c.T, c.V, c.dtype, c.n_given, c.n_top, c.ld = T, V, dtype, n_given, n_top, V
            need = max(need, moe_token_logprobs_workspace_bytes(c))
        self._configs = {torch.bfloat16: (self.c[MOE_BF16], ctypes.byref(self.c[MOE_BF16])),
                         torch.float32: (self.c[MOE_FP32], ctypes.byref(self.c[MOE_FP32]))}
        self.ws = torch.empty((need,), dtype=torch.uint8, device=device)
        self._device = self.ws.get_device()                  # -1: not a GPU's
        self._streams = set()

    def _used_on(self, stream, handle: int) -> None:
        """Memory belongs to the stream it was taken on: its reuse after the object's end waits for every other one that was here."""
        if handle not in self._streams:
            for t in (self.token_logp, self.entropy, self.conf, self.top_idx, self.top_logp, self.ws):
                t.record_stream(_torch_stream(stream))
            self._streams.add(handle)

    def run(self, logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, stream=None) -> "LogprobBuffers":
        """logits [T, V] bf16 or fp32, tokens int32 [T, n_given]."""
        T, V = logits.shape
        assert T == self.T and V == self.V, "logits do not fit the buffers"
        step, inner = logits.stride()
        assert inner == 1 or V == 1, "rows passed to the C ABI must be dense"
        given, device = None, logits.get_device()
        if self.n_given:
            if tokens is None:
                raise ValueError("the buffers are for given tokens, of which there are none")
            assert tokens.dtype is torch.int32 and tokens.shape == self.token_logp.shape and tokens.is_contiguous(), "tokens: int32 [T, n_given]"
            given = tokens.data_ptr()
        c, ref = self._configs[logits.dtype]
        if T <= 1:
            step = V                                         # there is no next row: torch gives such a dimension any stride
        elif step < V:
            raise ValueError(_SHARED_ROWS)
        if device < 0 or device != self._device or (given is not None and tokens.get_device() != device):
            raise ValueError(_DEVICES)
        if step >= _MAX_LD:
            logits, step = _near_rows(logits, stream), V
        c.ld = step
        s = _raw_stream(stream, device)
        if s not in self._streams:
            self._used_on(stream, s)
        rc = _lib.moe_token_logprobs(ref, logits.data_ptr(), given, self.token_logp.data_ptr(), self.entropy.data_ptr(), self.conf.data_ptr(),
                                     self.top_idx.data_ptr(), self.top_logp.data_ptr(), self.ws.data_ptr(), self.ws.numel(), s)
        if rc:
            _check(rc)
        return self


# ------------------------------------------------------------------------------ the attention step
def _strides(t: torch.Tensor, what: str):
    """Strides of [tokens, heads, channels] as the C ABI takes them: 0 (dense) where there is no next one, whose stride torch leaves open."""
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{what}: [tokens, heads, channels] with dense channels")
    token, head = (0 if n <= 1 else s for n, s in zip(t.shape[:2], t.stride()[:2]))
    if (t.shape[0] > 1 and token == 0) or (t.shape[1] > 1 and head == 0):
        raise ValueError(f"{what}: {_SHARED_ROWS}")
    return token, head


def _integers(t: torch.Tensor, what: str, shape) -> None:
    if t.dtype is torch.int32 and t.shape == shape and t.is_contiguous():        # as nearly every call has them
        return
    if t.dtype is not torch.int32 or t.dim() != len(shape) or any(n >= 0 and n != m for n, m in zip(shape, t.shape)):
        raise ValueError(f"{what}: int32 {[('any' if n < 0 else n) for n in shape]}")
    if (not t.is_contiguous()) if len(shape) == 1 else (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: dense rows")


def _table_ld(table: torch.Tensor) -> int:
    if table.shape[0] <= 1:
        return 0
    if table.stride(0) < table.shape[1]:
        raise ValueError(f"table: {_SHARED_ROWS}")
    return table.stride(0)


class _Owner:
    """Of device memory: its reuse after the object's end waits for every stream that used it."""

    def __init__(self):
        self._streams = set()

    def _memory(self):
        return ()

    def _used_on(self, stream, handle: int) -> None:
        streams = self._streams                              # of the memory that is recorded: another thread may put a larger one in its place
        if handle not in streams:
            for t in self._memory():
                if t is not None:
                    t.record_stream(_torch_stream(stream, t.device))
            streams.add(handle)


def _call_on(device: int, function, *args) -> None:
    """A C call with the tensors' device as the current one."""
    if torch._C._cuda_getDevice() == device:
        rc = function(*args)
    else:
        with torch.cuda.device(device):
            rc = function(*args)
    if rc:
        _check(rc)


class Rotary(_Owner):
    """Rotary positions: freq is fp64 [rotary_dim / 2] on the GPU, radians per position of each pair of channels; layout "half" (pairs i, i + rotary_dim / 2)
    or "interleaved" (pairs 2i, 2i + 1); mscale multiplies what is turned."""

    LAYOUTS = {"half": MOE_ROPE_HALF, "interleaved": MOE_ROPE_INTERLEAVED}

    def __init__(self, freq: torch.Tensor, layout: str = "half", mscale: float = 1.0):
        super().__init__()
        load_library()
        if freq.dtype != torch.float64 or freq.dim() != 1 or not freq.is_contiguous() or freq.numel() == 0:
            raise ValueError("freq: fp64 [rotary_dim / 2], dense")
        if layout not in self.LAYOUTS:
            raise ValueError(f"layout {layout!r}: one of {sorted(self.LAYOUTS)}")
        _on_one_gpu(freq)
        self._freq, self._layout = freq, layout
        self._key = (2 * freq.numel(), self.LAYOUTS[layout], float(mscale))
        self._calls = {}

    freq, layout = property(lambda self: self._freq), property(lambda self: self._layout)
    rotary_dim, mscale = property(lambda self: self._key[0]), property(lambda self: self._key[2])

    @classmethod
    def scaled(cls, rotary_dim: int, base: float = 10000.0, layout: str = "half", factor: float = 1.0, trained: int = 0, slow: float = 1.0,
               fast: float = 32.0, mscale: float = 1.0, device="cuda") -> "Rotary":
        """Frequencies base^(-2i / rotary_dim), slowed for contexts `factor` times as long: all of them, or with `trained` positions those that turn at
        most `slow` times over them, those between `slow` and `fast` in proportion, faster ones not."""
        if rotary_dim < 2 or rotary_dim % 2 or not factor > 0 or trained < 0 or not fast > slow:
            raise ValueError(f"rotary_dim={rotary_dim} factor={factor} trained={trained} slow={slow} fast={fast}")
        freq = []
        for i in range(rotary_dim // 2):
            f = base ** (-2.0 * i / rotary_dim)
            keep = 0.0 if not trained else min(1.0, max(0.0, (trained * f / (2.0 * math.pi) - slow) / (fast - slow)))
            freq.append(f if factor == 1.0 else f * (keep + (1.0 - keep) / factor))
        return cls(torch.tensor(freq, dtype=torch.float64, device=device), layout, mscale)

    def _memory(self):
        return (self._freq,)

    def _call(self, x: torch.Tensor, out: torch.Tensor, inverse: bool):
        c = moe_rope_config()
        if x.shape != out.shape or x.dtype != out.dtype:
            raise ValueError("out: shape and type of x")
        (c.x_token, c.x_head), (c.out_token, c.out_head) = _strides(x, "x"), _strides(out, "out")
        c.T, c.heads, c.D = x.shape
        c.rotary_dim, c.layout, c.mscale = self._key
        c.dtype, c.inverse = _float_type(x), 1 if inverse else 0
        if len(self._calls) > 256:                           # a server's batches are of any size
            self._calls.clear()
        return ctypes.byref(c)

    def __call__(self, x: torch.Tensor, pos: torch.Tensor, out: Optional[torch.Tensor] = None, inverse: bool = False, stream=None) -> torch.Tensor:
        """x [tokens, heads, channels] bf16 or fp32 at positions pos int32 [tokens] -> out (default: a new tensor; x itself: in place).  inverse: turned back."""
        if out is None:
            with torch.cuda.stream(_torch_stream(stream, x.device)):
                out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        # another thread may call while the C call reads its description, which nobody writes any more
        key = (x.shape, x.stride(), x.dtype, out.shape, out.stride(), out.dtype, bool(inverse))
        ref = self._calls.get(key)
        if ref is None:
            ref = self._calls[key] = self._call(x, out, inverse)
        device = x.get_device()
        if device < 0 or device != self._freq.get_device() or device != out.get_device() or device != pos.get_device():
            raise ValueError(_DEVICES)
        _integers(pos, "pos", x.shape[:1])
        s = _raw_stream(stream, device)
        if s not in self._streams:
            self._used_on(stream, s)
        _call_on(device, _lib.moe_rope, ref, x.data_ptr(), pos.data_ptr(), self._freq.data_ptr(), out.data_ptr(), s)
        return out


class KvCache(_Owner):
    """The paged keys and values of one layer: k, v [pages, key heads, positions of a page, channels] bf16, fp32 or, with scales [pages, key heads, positions]
    fp32, float8_e4m3fn.  Which pages a sequence has is in the page table of each call: int32 [sequences, entries], positions p of a sequence in
    page table[s, p // page_size]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None):
        super().__init__()
        load_library()
        kinds = {torch.bfloat16: MOE_BF16, torch.float32: MOE_FP32, torch.float8_e4m3fn: MOE_E4M3}
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.dtype not in kinds or k.stride(3) != 1 or v.stride(3) != 1:
            raise ValueError("k, v: [pages, key heads, positions, channels] of one type (bf16, fp32, float8_e4m3fn), with dense channels")
        steps = [0 if n <= 1 else s for n, s in zip(k.shape[:3], k.stride())]
        if steps != [0 if n <= 1 else s for n, s in zip(v.shape[:3], v.stride())]:
            raise ValueError("k and v have different strides")
        if any(n > 1 and s == 0 for n, s in zip(k.shape[:3], steps)):
            raise ValueError(_SHARED_ROWS)
        codes = k.dtype is torch.float8_e4m3fn
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            if codes != (t is not None) or (codes and (t.dtype != torch.float32 or t.shape != k.shape[:3] or not t.is_contiguous())):
                raise ValueError(f"{name}: fp32 [pages, key heads, positions] with float8_e4m3fn rows, None with others")
        _on_one_gpu(k, v, k_scale, v_scale)
        self._k, self._v, self._k_scale, self._v_scale = k, v, k_scale, v_scale
        self.n_pages, self.n_heads, self.page_size, self.head_dim = k.shape
        self._device = k.get_device()
        c = self.c = moe_kv_cache()
        c.n_pages, c.heads, c.page_size, c.D = k.shape
        c.dtype = kinds[k.dtype]
        c.page, c.head, c.row = steps
        c.k, c.v = k.data_ptr(), v.data_ptr()
        if codes:
            c.k_scale, c.v_scale = k_scale.data_ptr(), v_scale.data_ptr()
        self._ref = ctypes.byref(c)
        self._calls = {}

    k, v = property(lambda self: self._k), property(lambda self: self._v)
    k_scale, v_scale = property(lambda self: self._k_scale), property(lambda self: self._v_scale)

    @classmethod
    def empty(cls, n_pages: int, page_size: int, n_heads: int, head_dim: int, dtype: torch.dtype = torch.bfloat16, device="cuda") -> "KvCache":
        """A cache of dense pages; what is in them does not matter until it is written."""
        k, v = (torch.empty((n_pages, n_heads, page_size, head_dim), dtype=dtype, device=device) for _ in range(2))
        if dtype is not torch.float8_e4m3fn:
            return cls(k, v)
        return cls(k, v, *(torch.empty((n_pages, n_heads, page_size), dtype=torch.float32, device=device) for _ in range(2)))

    def _memory(self):
        return self._k, self._v, self._k_scale, self._v_scale

    def _call(self, k, v, q, q_out, table, rotary):
        c = moe_append_config()
        if k.dim() != 3 or k.shape != v.shape or k.dtype != v.dtype or tuple(k.shape[1:]) != (self.n_heads, self.head_dim):
            raise ValueError(f"k, v: [tokens, {self.n_heads}, {self.head_dim}] of one type")
        (c.k_token, c.k_head), (c.v_token, c.v_head) = _strides(k, "k"), _strides(v, "v")
        c.T, c.dtype = k.shape[0], _float_type(k)
        if q is not None:
            if q.dim() != 3 or q.shape[0] != k.shape[0] or q.shape[2] != self.head_dim or q.dtype != k.dtype or q_out.shape != q.shape or q_out.dtype != q.dtype:
                raise ValueError(f"q, q_out: [tokens, heads, {self.head_dim}] of the keys' type")
            (c.q_token, c.q_head), (c.out_token, c.out_head) = _strides(q, "q"), _strides(q_out, "q_out")
            c.heads = q.shape[1]
        _integers(table, "table", (-1, -1))
        c.n_seqs, c.table_len = table.shape
        c.table_ld = _table_ld(table)
        c.mscale = 1.0
        if rotary is not None:
            c.rotary_dim, c.layout, c.mscale = rotary._key
        if len(self._calls) > 256:                           # a server's batches are of any size
            self._calls.clear()
        return c, ctypes.byref(c)

    def append(self, k: torch.Tensor, v: torch.Tensor, pos: torch.Tensor, table: torch.Tensor, seq: Optional[torch.Tensor] = None,
               rotary: Optional[Rotary] = None, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
               stream=None) -> Optional[torch.Tensor]:
        """Stores keys (turned, with `rotary`) and values [tokens, key heads, channels] at positions pos int32 [tokens] of sequences seq int32 [tokens] (None:
        token t is of sequence t); positions below 0 are padding.  With queries q [tokens, heads, channels]: -> q_out (default: a new tensor; q itself: in
        place), turned."""
        if q is None:
            if q_out is not None:
                raise ValueError("q_out without q")
            key = (k.shape, k.stride(), k.dtype, v.shape, v.stride(), v.dtype, table.shape, table.stride(), table.dtype, rotary and rotary._key)
        else:
            if q_out is None:
                with torch.cuda.stream(_torch_stream(stream, q.device)):
                    q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            key = (k.shape, k.stride(), k.dtype, v.shape, v.stride(), v.dtype, table.shape, table.stride(), table.dtype, rotary and rotary._key,
                   q.shape, q.stride(), q.dtype, q_out.shape, q_out.stride(), q_out.dtype)
        call = self._calls.get(key)
        if call is None:
            call = self._calls[key] = self._call(k, v, q, q_out, table, rotary)
        device = self._device
        for t in (k, v, pos, table):
            if t.get_device() != device:
                raise ValueError(_DEVICES)
        for t in (seq, q, q_out, rotary and rotary._freq):
            if t is not None and t.get_device() != device:
                raise ValueError(_DEVICES)
        _integers(pos, "pos", k.shape[:1])
        if seq is not None:
            _integers(seq, "seq", k.shape[:1])
        s = _raw_stream(stream, device)
        if s not in self._streams:
            self._used_on(stream, s)
        if rotary is not None and s not in rotary._streams:
            rotary._used_on(stream, s)
        _call_on(device, _lib.moe_kv_append, call[1], self._ref, None if q is None else q.data_ptr(), k.data_ptr(), v.data_ptr(), pos.data_ptr(),
                 None if seq is None else seq.data_ptr(), table.data_ptr(), None if rotary is None else rotary._freq.data_ptr(),
                 None if q is None else q_out.data_ptr(), s)
        return q_out


class DecodeAttention(_Owner):
    """Attention of one new token per sequence over a cache.  Calling it enqueues it on `stream`; its workspace is kept and grows with the largest call, so
    calls that may overlap (streams without order between them, a graph's replay among them) need an object each.  A captured graph reads the cache and a
    workspace of its object, which has to live as long as the graph; larger calls in between do not matter to it."""

    def __init__(self, cache: KvCache, n_heads: int, scale: Optional[float] = None, window: int = 0, softcap: float = 0.0):
        super().__init__()
        if n_heads <= 0 or n_heads % cache.n_heads:
            raise ValueError(f"{n_heads} query heads on {cache.n_heads} key heads")
        self._cache, self._n_heads = cache, n_heads
        self._scale = 1.0 / math.sqrt(cache.head_dim) if scale is None else float(scale)
        self._window, self._softcap = int(window), float(softcap)
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("made while a graph is captured: its counters have to be zero before")
        # zero before any stream's first call, and after each call again
        self.counters = torch.zeros((MOE_ATTENTION_COUNTERS // 4,), dtype=torch.int32, device=cache.k.device)
        torch.cuda.current_stream(cache.k.device).synchronize()
        self.ws = None
        self._outgrown = []                                  # workspaces of smaller calls: captured graphs have their addresses
        self._growing = threading.Lock()
        self._calls = {}

    cache, n_heads = property(lambda self: self._cache), property(lambda self: self._n_heads)
    scale, window, softcap = property(lambda self: self._scale), property(lambda self: self._window), property(lambda self: self._softcap)

    def _memory(self):
        return self.ws, self.counters, *self._outgrown

    def _workspace(self, need: int, stream) -> torch.Tensor:
        """One that is large enough; a call stays with the one that it was given, whatever other threads' calls need."""
        with self._growing:
            ws = self.ws
            if ws is None or ws.numel() < need:
                if ws is not None:                           # twice as large at least: what is kept stays below the one in use
                    need = max(need, 2 * ws.numel())
                with torch.cuda.stream(_torch_stream(stream, self.cache.k.device)):
                    larger = torch.empty((need,), dtype=torch.uint8, device=self.cache.k.device)
                if ws is not None:
                    self._outgrown.append(ws)
                self._streams = set()                        # in front of the workspace, which no stream in it has used
                ws = self.ws = larger
            return ws

    def _call(self, q, out, table, max_len: int):
        """-> (description, its bound, workspace bytes) of a call with such tensors: nobody writes it any more, since another thread may call while the C call reads it."""
        c = moe_attention_config()
        if q.dim() != 3 or tuple(q.shape[1:]) != (self.n_heads, self.cache.head_dim) or out.shape != q.shape or out.dtype != q.dtype:
            raise ValueError(f"q, out: [sequences, {self.n_heads}, {self.cache.head_dim}] of one type")
        (c.q_token, c.q_head), (c.out_token, c.out_head) = _strides(q, "q"), _strides(out, "out")
        c.B, c.heads, c.dtype = q.shape[0], self.n_heads, _float_type(q)
        _integers(table, "table", (q.shape[0], -1))
        c.table_len, c.table_ld = table.shape[1], _table_ld(table)
        c.window, c.scale, c.softcap = self.window, self.scale, self.softcap
        if len(self._calls) > 256:                           # a server's batches are of any size
            self._calls.clear()
        return self._bounded(c, max_len)

    def _bounded(self, c, max_len: int):
        """With this bound: a batch that generates has another one in every step."""
        if not 0 <= max_len < 2 ** 31:
            raise ValueError(f"max_len {max_len}")
        c = moe_attention_config.from_buffer_copy(c)
        c.max_len = max_len
        ref = ctypes.byref(c)
        return ref, c.max_len, int(_lib.moe_paged_attention_workspace_bytes(ref, self.cache._ref))

    def __call__(self, q: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, max_len: int, out: Optional[torch.Tensor] = None,
                 lse: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """q [sequences, heads, channels] bf16 or fp32, lengths int32 [sequences] (the new token's position is length - 1) of at most max_len -> out (default: a new
        tensor); lse: fp32 [sequences, heads], filled where it is given."""
        if out is None:
            with torch.cuda.stream(_torch_stream(stream, q.device)):
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        key = (q.shape, q.stride(), q.dtype, out.shape, out.stride(), out.dtype, table.shape, table.stride(), table.dtype)
        call = self._calls.get(key)
        if call is None:
            call = self._calls[key] = self._call(q, out, table, max_len)
        elif call[1] != max_len:
            call = self._calls[key] = self._bounded(call[0]._obj, max_len)
        ref, _, need = call
        cache = self._cache
        device = cache._device
        for t in (q, table, lengths, out):
            if t.get_device() != device:
                raise ValueError(_DEVICES)
        _integers(lengths, "lengths", q.shape[:1])
        if lse is not None:
            if lse.get_device() != device:
                raise ValueError(_DEVICES)
            if lse.dtype is not torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous():
                raise ValueError("lse: fp32 [sequences, heads], dense")
        ws = self.ws
        if need and (ws is None or ws.numel() < need):
            ws = self._workspace(need, stream)
        s = _raw_stream(stream, device)
        if s not in self._streams:
            self._used_on(stream, s)
        if s not in cache._streams:
            cache._used_on(stream, s)
        _call_on(device, _lib.moe_paged_attention, ref, cache._ref, q.data_ptr(), table.data_ptr(), lengths.data_ptr(), out.data_ptr(),
                 None if lse is None else lse.data_ptr(), None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(), self.counters.data_ptr(), s)
        return out


def torch_dtype(cfg: LayerConfig):
    return torch.float32 if cfg.dtype == "fp32" else torch.bfloat16


def to_device(a, cfg: LayerConfig, device="cuda") -> torch.Tensor:
    """Uploads a stored host tensor (float32, or uint16 holding bf16 bits) without changing bits."""
    import numpy as np
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(a).to(device)


class StepBuffers:
    """Device buffers of one layer step (allocation only; the step itself is the C calls)."""

    def __init__(self, cfg: LayerConfig, T: Optional[int] = None, device="cuda"):
        T = cfg.T if T is None else T
        self.cfg, self.T = cfg, T
        self.c = make_config(cfg, T)
        K, E, H = cfg.k_big, cfg.E, cfg.H
        i32 = dict(dtype=torch.int32, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        self.logits = torch.empty((T, E), **f32)
        self.topk_idx = torch.empty((T, K), **i32)
        self.topk_w = torch.empty((T, K), **f32)
        self.important = torch.empty((T,), dtype=torch.uint8, device=device)
        self.k_t = torch.empty((T,), **i32)
        self.expert_offsets = torch.empty((E + 1,), **i32)
        self.sorted_token = torch.empty((T * K,), **i32)
        self.sorted_rank = torch.empty((T * K,), **i32)
        self.inv_pos = torch.empty((T, K), **i32)
        self.y = torch.zeros((T * K, H), **f32)
        ns = moe_shared_out_slabs(self.c)
        self.shared_out = torch.zeros((ns, T, H), **f32) if ns > 0 else None
        self.out = torch.empty((T, H), dtype=torch_dtype(cfg), device=device)
        self.dws_bytes = moe_dispatch_workspace_bytes(self.c)
        self.dws = torch.empty((self.dws_bytes,), dtype=torch.uint8, device=device)
        self.fws_bytes = moe_expert_ffn_workspace_bytes(self.c)
        self.fws = torch.empty((self.fws_bytes,), dtype=torch.uint8, device=device)
        self.ev_in, self.ev_shared = torch.cuda.Event(), torch.cuda.Event()
        # workspace of moe_layer_decode (steps of at most 64 tokens, bf16 activations), cleared once
        self.lws_bytes = moe_layer_decode_workspace_bytes(self.c) if 0 < T <= 64 and cfg.dtype in ("bf16", "bf16w8") else 0
        self.lws = None
        if self.lws_bytes:
            self.lws = torch.empty((self.lws_bytes,), dtype=torch.uint8, device=device)
            moe_layer_decode_init(self.lws, self.lws_bytes)


    def as_struct(self) -> moe_step_buffers:
        """The buffers as the one-call entry points take them, with the addresses of this moment."""
        return moe_step_buffers(_addr(self.logits), _addr(self.topk_idx), _addr(self.topk_w), _addr(self.important), _addr(self.k_t),
                                _addr(self.expert_offsets), _addr(self.sorted_token), _addr(self.sorted_rank), _addr(self.inv_pos),
                                _addr(self.y), _addr(self.shared_out), _addr(self.out), _addr(self.dws), self.dws_bytes,
                                _addr(self.fws), self.fws_bytes)


def layer_step(b: StepBuffers, x, Wg, gate_bias, conf, expert_table, shared_w, logits_given=False,
               stream=None, side_stream=None) -> torch.Tensor:
    """One step of the layer with all experts resident: one C call on `stream`.

    With `side_stream` (a second torch stream of default priority) the separate calls: the shared experts, which do not
    depend on the router, are enqueued there first and run under the router, selection and dispatch
    kernels; the combine waits for them.  Only stream plumbing is added; the results are the same."""
    if side_stream is None or b.shared_out is None:
        moe_layer_step(b.c, x, Wg, gate_bias, conf, expert_table, shared_w, logits_given, b.as_struct(), stream)
        return b.out
    main = stream if stream is not None else torch.cuda.current_stream()
    b.ev_in.record(main)                         # x is ready; the previous combine has read shared_out
    side_stream.wait_event(b.ev_in)
    moe_expert_ffn(b.c, x, b.expert_offsets, b.sorted_token, None, shared_w, False, True, b.y,
                   b.shared_out, b.fws, b.fws_bytes, side_stream)
    b.ev_shared.record(side_stream)
    moe_route(b.c, x, Wg, gate_bias, conf, b.logits, logits_given, b.topk_idx, b.topk_w, b.important,
              b.k_t, stream)
    moe_dispatch(b.c, b.topk_idx, b.k_t, b.expert_offsets, b.sorted_token, b.sorted_rank, b.inv_pos,
                 b.dws, b.dws_bytes, stream)
    moe_expert_ffn(b.c, x, b.expert_offsets, b.sorted_token, expert_table, shared_w, True, False, b.y,
                   b.shared_out, b.fws, b.fws_bytes, stream)
    main.wait_event(b.ev_shared)
    moe_combine(b.c, b.y, b.topk_w, b.inv_pos, b.k_t, b.shared_out, b.out, stream)
    return b.out


def layer_decode_step(b: StepBuffers, x, Wg, gate_bias, conf, expert_table, shared_w, logits_given=False,
                      stream=None) -> torch.Tensor:
    """One decode step (at most 64 tokens) of the layer: a single C call."""
    moe_layer_decode(b.c, x, Wg, gate_bias, conf, expert_table, shared_w, b.logits, logits_given, b.topk_idx,
                     b.topk_w, b.important, b.k_t, b.expert_offsets, b.sorted_token, b.sorted_rank, b.inv_pos, b.y,
                     b.shared_out, b.out, b.lws, b.lws_bytes, stream)
    return b.out


def fallback_step(b: StepBuffers, x, conf, expert_table, stream=None) -> torch.Tensor:
    """Second pass of Alg. 1 on the buffers of a little pass (layer_step with a confidence above gamma
    for every token, which leaves the router logits in b.logits and the little output in b.out): the
    tokens rejected by `conf` get the experts of ranks k_little .. k_big-1 added.  One C call."""
    moe_layer_fallback(b.c, x, conf, expert_table, b.as_struct(), stream)
    return b.out


def layer_step_cached(b: StepBuffers, x, Wg, gate_bias, conf, cache: int, shared_w, stream=None):
    """One step of the layer whose routed experts live in pinned host memory behind `cache`
    (Sec. II-B): router and dispatch as in layer_step, then the execution stage through the cache
    (the host waits once for the router's decision).  -> (b.out, summed fetch statistics, waves)."""
    moe_route(b.c, x, Wg, gate_bias, conf, b.logits, False, b.topk_idx, b.topk_w, b.important, b.k_t, stream)
    moe_dispatch(b.c, b.topk_idx, b.k_t, b.expert_offsets, b.sorted_token, b.sorted_rank, b.inv_pos,
                 b.dws, b.dws_bytes, stream)
    st, waves = moe_expert_ffn_cached(b.c, cache, x, b.expert_offsets, b.sorted_token, shared_w, b.y,
                                      b.shared_out, b.fws, b.fws_bytes, stream)
    moe_combine(b.c, b.y, b.topk_w, b.inv_pos, b.k_t, b.shared_out, b.out, stream)
    return b.out, st, waves
