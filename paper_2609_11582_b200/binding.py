"""Thin ctypes binding of the okq C ABI (argument marshalling only).

PyTorch is used for device memory and streams; every step of the path runs in the CUDA
library.  If the library is missing this module raises: there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libokq.so")

HEAD_DIM, WINDOW, RECORD_BYTES, MAX_GROUP = 128, 32, 2688, 8
RECORD_BYTES_MX, MX_META_BYTES = 2312, 136
META_FP16, META_MXFP4 = 0, 1
SCHEDULE_WINDOW, SCHEDULE_CAPTION = 0, 1

PLAN_PAIR_QUARTER, PLAN_PAIR_ONE, PLAN_PAIR_FOUR = -1, -2, -3

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_ALIGNMENT, ERR_CAPACITY, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(8)


class okq_cache(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("batch", C.c_int32), ("n_kv_heads", C.c_int32), ("n_q_heads", C.c_int32),
                ("head_dim", C.c_int32), ("window", C.c_int32), ("capacity", C.c_int32), ("meta_format", C.c_int32),
                ("schedule", C.c_int32), ("reserved", C.c_int32),
                ("records", C.c_void_p), ("modality", C.c_void_p), ("k_tail", C.c_void_p), ("v_tail", C.c_void_p),
                ("seq_len", C.c_void_p), ("status", C.c_void_p)]


class okq_ladder_cache(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_kv_heads", C.c_int32), ("n_q_heads", C.c_int32), ("capacity", C.c_int32),
                ("bits", C.c_int32), ("reserved", C.c_int32),
                ("k_codes", C.c_void_p), ("k_norm", C.c_void_p), ("k_meta", C.c_void_p), ("v_codes", C.c_void_p),
                ("v_norm", C.c_void_p), ("modality", C.c_void_p)]


class okq_paged(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("batch", C.c_int32), ("n_kv_heads", C.c_int32), ("n_q_heads", C.c_int32),
                ("page_tokens", C.c_int32), ("n_pages", C.c_int32), ("max_pages", C.c_int32), ("dtype", C.c_int32),
                ("codes", C.c_void_p), ("scales", C.c_void_p), ("raw", C.c_void_p), ("table", C.c_void_p), ("refs", C.c_void_p),
                ("seq_len", C.c_void_p), ("status", C.c_void_p)]


class okq_rope(C.Structure):
    _fields_ = [("sections", C.c_int32 * 3), ("interleaved", C.c_int32), ("freq", C.c_void_p), ("positions", C.c_void_p)]


class okq_rope_tensor(C.Structure):
    _fields_ = [("in_", C.c_void_p), ("out", C.c_void_p), ("in_strides", C.c_int64 * 3), ("out_strides", C.c_int64 * 3),
                ("heads", C.c_int32)]


class okq_norm_tensor(C.Structure):
    _fields_ = [("in_", C.c_void_p), ("grad_out", C.c_void_p), ("out", C.c_void_p), ("in_strides", C.c_int64 * 3), ("grad_strides", C.c_int64 * 3),
                ("out_strides", C.c_int64 * 3), ("weight", C.c_void_p), ("weight_grad", C.c_void_p), ("weight_dtype", C.c_int32), ("heads", C.c_int32)]


class OkqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().okq_status_string(status).decode()
        if status == ERR_CUDA:
            msg += f" (cudaError {lib().okq_last_cuda_error()})"
        super().__init__(f"{where}: {msg}")


_lib = None


def lib():
    """Load libokq.so (built in-tree by `python -m paper_2609_11582_b200.build`)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_11582_b200.build` "
                               "(the okq path has no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        L.okq_status_string.restype = C.c_char_p
        L.okq_status_string.argtypes = [C.c_int]
        L.okq_last_cuda_error.restype = C.c_int
        L.okq_cache_sizes.restype = C.c_int
        L.okq_cache_sizes.argtypes = [C.POINTER(okq_cache), C.POINTER(C.c_size_t)]
        L.okq_decode_workspace_bytes.restype = C.c_size_t
        L.okq_decode_workspace_bytes.argtypes = [C.POINTER(okq_cache), C.c_int32, C.c_int32]
        L.okq_quantize_keys.restype = C.c_int
        L.okq_quantize_keys.argtypes = [C.POINTER(okq_cache), C.c_int32, C.c_void_p, C.POINTER(C.c_int64), C.c_int32,
                                        C.c_void_p, C.c_void_p]
        L.okq_quantize_values.restype = C.c_int
        L.okq_quantize_values.argtypes = [C.POINTER(okq_cache), C.c_int32, C.c_void_p, C.POINTER(C.c_int64), C.c_int32,
                                          C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.okq_quantize_values_bulk.restype = C.c_int
        L.okq_quantize_values_bulk.argtypes = L.okq_quantize_values.argtypes
        L.okq_debug_bulk_timeout.restype = C.c_int
        L.okq_debug_bulk_timeout.argtypes = list(L.okq_quantize_values.argtypes[:-1]) + [C.c_int64, C.c_void_p]
        L.okq_append.restype = C.c_int
        L.okq_append.argtypes = [C.POINTER(okq_cache), C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                 C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.okq_decode_attention.restype = C.c_int
        L.okq_decode_attention.argtypes = [C.POINTER(okq_cache), C.c_int32, C.c_int32, C.c_void_p, C.c_float,
                                           C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_size_t, C.c_int32,
                                           C.c_void_p, C.c_void_p]
        L.okq_decode_attention_simt.restype = C.c_int
        L.okq_decode_attention_simt.argtypes = L.okq_decode_attention.argtypes
        L.okq_decode_attention_noalloc.restype = C.c_int
        L.okq_decode_attention_noalloc.argtypes = [C.POINTER(okq_cache), C.c_int32, C.c_int32, C.c_void_p, C.c_float,
                                                   C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        L.okq_debug_decode_plan.restype = C.c_int32
        L.okq_debug_decode_plan.argtypes = [C.POINTER(okq_cache), C.c_int32, C.c_int32, C.c_size_t]
        L.okq_decode_select.restype = C.c_int32
        L.okq_decode_select.argtypes = [C.c_int32]
        L.okq_profile_events.restype = None
        L.okq_profile_events.argtypes = [C.c_void_p, C.c_void_p]
        L.okq_cache_export.restype = C.c_int
        L.okq_cache_export.argtypes = [C.POINTER(okq_cache), C.c_int32] + [C.c_void_p] * 6
        L.okq_cache_export_mx.restype = C.c_int
        L.okq_cache_export_mx.argtypes = [C.POINTER(okq_cache), C.c_int32] + [C.c_void_p] * 7
        L.okq_calib_workspace_bytes.restype = C.c_size_t
        L.okq_calib_workspace_bytes.argtypes = [C.c_int32, C.c_int32]
        L.okq_calib_attention_weights.restype = C.c_int
        L.okq_calib_attention_weights.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_int32,
                                                  C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.okq_debug_calib_timeout.restype = C.c_int
        L.okq_debug_calib_timeout.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p,
                                              C.c_int64, C.c_void_p]
        L.okq_debug_calib_direct.restype = C.c_int
        L.okq_debug_calib_direct.argtypes = [C.c_void_p] * 6
        L.okq_calib_moments.restype = C.c_int
        L.okq_calib_moments.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_size_t,
                                        C.c_void_p, C.c_void_p]
        L.okq_calib_rotation.restype = C.c_int
        L.okq_calib_rotation.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.c_void_p]
        L.okq_cache_import.restype = C.c_int
        L.okq_cache_import.argtypes = [C.POINTER(okq_cache), C.c_int32] + [C.c_void_p] * 6
        L.okq_ladder_codebook.restype = C.c_int32
        L.okq_ladder_codebook.argtypes = [C.c_int32, C.POINTER(C.c_float), C.POINTER(C.c_float)]
        L.okq_ladder_quantize_keys.restype = C.c_int
        L.okq_ladder_quantize_keys.argtypes = [C.POINTER(okq_ladder_cache), C.c_void_p, C.POINTER(C.c_int64), C.c_int32,
                                               C.c_void_p, C.c_void_p]
        L.okq_ladder_quantize_values.restype = C.c_int
        L.okq_ladder_quantize_values.argtypes = [C.POINTER(okq_ladder_cache), C.c_void_p, C.POINTER(C.c_int64), C.c_int32,
                                                 C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.okq_debug_ladder_timeout.restype = C.c_int
        L.okq_debug_ladder_timeout.argtypes = list(L.okq_ladder_quantize_values.argtypes[:-1]) + [C.c_int64, C.c_void_p]
        L.okq_ladder_decode_attention.restype = C.c_int
        L.okq_ladder_decode_attention.argtypes = [C.POINTER(okq_ladder_cache), C.c_int32, C.c_void_p, C.c_float, C.c_void_p,
                                                  C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
        L.okq_turboquant_encode.restype = C.c_int
        L.okq_turboquant_encode.argtypes = [C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.okq_turboquant_decode.restype = C.c_int
        L.okq_turboquant_decode.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        paged, i32, ptr = C.POINTER(okq_paged), C.c_int32, C.c_void_p   # (ptr: also strides and small structs, as packed bytes)
        L.okq_paged_sizes.restype = C.c_int
        L.okq_paged_sizes.argtypes = [paged, C.POINTER(C.c_size_t)]
        L.okq_paged_workspace_bytes.restype = C.c_size_t
        L.okq_paged_workspace_bytes.argtypes = [paged, i32, i32]
        L.okq_rope_apply.restype = C.c_int
        L.okq_rope_apply.argtypes = [ptr, i32, i32, i32, ptr, ptr, i32, ptr]
        L.okq_norm_rope_apply.restype = C.c_int
        L.okq_norm_rope_apply.argtypes = [ptr, C.c_float, i32, i32, i32, ptr, ptr, ptr]
        L.okq_norm_rope_grad.restype = C.c_int
        L.okq_norm_rope_grad.argtypes = [ptr, C.c_float, i32, i32, i32, ptr, ptr, ptr, C.c_size_t, ptr]
        L.okq_norm_rope_workspace_bytes.restype = C.c_size_t
        L.okq_norm_rope_workspace_bytes.argtypes = [i32, i32, i32, i32]
        L.okq_paged_append.restype = C.c_int
        L.okq_paged_append.argtypes = [paged, i32, i32, ptr, ptr, ptr, ptr, i32, ptr, ptr, ptr]
        L.okq_paged_read.restype = C.c_int
        L.okq_paged_read.argtypes = [paged, i32, i32, i32, i32, ptr, ptr, ptr]
        L.okq_paged_attention.restype = C.c_int
        L.okq_paged_attention.argtypes = [paged, i32, i32, ptr, ptr, i32, ptr, ptr, C.c_float, ptr, C.c_size_t, ptr, ptr, ptr]
        L.okq_debug_paged_timeout.restype = C.c_int
        L.okq_debug_paged_timeout.argtypes = [paged, i32, i32, ptr, ptr, i32, ptr, C.c_size_t, ptr, ptr, C.c_int64, ptr]
        L.okq_debug_paged_timeout_sight.restype = C.c_int
        L.okq_debug_paged_timeout_sight.argtypes = [paged, i32, i32, ptr, ptr, i32, i32, i32, ptr, ptr, C.c_size_t, ptr, ptr, C.c_int64, ptr]
        L.okq_debug_paged_plan.restype = i32
        L.okq_debug_paged_plan.argtypes = [paged, i32, i32]
        L.okq_paged_attention_window.restype = C.c_int
        L.okq_paged_attention_window.argtypes = [paged, i32, i32, ptr, ptr, i32, ptr, ptr, C.c_float, i32, i32, ptr, C.c_size_t, ptr, ptr, ptr]
        L.okq_paged_attention_tree.restype = C.c_int
        L.okq_paged_attention_tree.argtypes = [paged, i32, i32, ptr, ptr, i32, ptr, ptr, C.c_float, ptr, ptr, C.c_size_t, ptr, ptr, ptr]
        L.okq_tree_ancestors.restype = C.c_int
        L.okq_tree_ancestors.argtypes = [paged, ptr, i32, ptr, ptr, ptr, ptr]
        L.okq_debug_paged_plan_window.restype = i32
        L.okq_debug_paged_plan_window.argtypes = [paged, i32, i32, i32, i32]
        L.okq_pages_slide.restype = C.c_int
        L.okq_pages_slide.argtypes = [paged, i32, i32, ptr, ptr]
        L.okq_pages_reserve.restype = C.c_int
        L.okq_pages_reserve.argtypes = [paged, ptr, ptr]
        L.okq_pages_fork.restype = C.c_int
        L.okq_pages_fork.argtypes = [paged, ptr, ptr, i32, ptr, C.c_size_t, ptr]
        L.okq_pages_release.restype = C.c_int
        L.okq_pages_release.argtypes = [paged, ptr, i32, ptr]
        L.okq_pages_copy.restype = C.c_int
        L.okq_pages_copy.argtypes = [paged, ptr, ptr, i32, ptr]
        L.okq_pages_compact.restype = C.c_int
        L.okq_pages_compact.argtypes = [paged, ptr, ptr, C.c_size_t, ptr]
        _lib = L
    return _lib


def exported_symbols():
    return ["okq_status_string", "okq_last_cuda_error", "okq_cache_sizes", "okq_decode_workspace_bytes",
            "okq_quantize_keys", "okq_quantize_values", "okq_append", "okq_decode_attention", "okq_cache_export",
            "okq_cache_import", "okq_profile_events", "okq_decode_select", "okq_debug_decode_plan", "okq_decode_attention_simt",
            "okq_decode_attention_noalloc", "okq_quantize_values_bulk", "okq_debug_bulk_timeout", "okq_cache_export_mx",
            "okq_calib_workspace_bytes", "okq_calib_attention_weights", "okq_debug_calib_timeout", "okq_debug_calib_direct",
            "okq_calib_moments", "okq_calib_rotation",
            "okq_ladder_codebook", "okq_ladder_quantize_keys", "okq_ladder_quantize_values",
            "okq_debug_ladder_timeout", "okq_ladder_decode_attention", "okq_turboquant_encode", "okq_turboquant_decode",
            "okq_paged_sizes", "okq_paged_workspace_bytes", "okq_rope_apply",
            "okq_norm_rope_apply", "okq_norm_rope_grad", "okq_norm_rope_workspace_bytes", "okq_paged_append", "okq_paged_read",
            "okq_paged_attention", "okq_debug_paged_timeout", "okq_debug_paged_plan", "okq_pages_reserve", "okq_pages_fork", "okq_pages_release", "okq_pages_copy",
            "okq_pages_compact", "okq_pages_slide", "okq_paged_attention_window", "okq_paged_attention_tree", "okq_tree_ancestors",
            "okq_debug_paged_plan_window", "okq_debug_paged_timeout_sight"]


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


# The current stream's handle without building a torch.cuda.Stream object around it (0.2 us instead of 3 us per call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device_index = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _device_index is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device_index())


def _check(st: int, where: str):
    if st != OK:
        raise OkqError(st, where)


def cache_sizes(n_layers, batch, n_kv_heads, n_q_heads, capacity, head_dim=HEAD_DIM, window=WINDOW,
                meta_format=META_FP16, schedule=SCHEDULE_WINDOW):
    shape = okq_cache(n_layers, batch, n_kv_heads, n_q_heads, head_dim, window, capacity, meta_format, schedule, 0)
    out = (C.c_size_t * 6)()
    _check(lib().okq_cache_sizes(C.byref(shape), out), "okq_cache_sizes")
    return list(out)


class Cache:
    """Device buffers of a 2-bit KV cache plus the C struct that describes them."""

    def __init__(self, n_layers, batch, n_kv_heads, n_q_heads, capacity, device="cuda", meta_format=META_FP16,
                 schedule=SCHEDULE_WINDOW):
        sizes = cache_sizes(n_layers, batch, n_kv_heads, n_q_heads, capacity, meta_format=meta_format, schedule=schedule)
        self.meta_format, self.schedule = meta_format, schedule
        self.n_layers, self.batch, self.n_kv_heads, self.n_q_heads, self.capacity = (
            n_layers, batch, n_kv_heads, n_q_heads, capacity)
        self.device = torch.device(device)
        self.records = torch.zeros(sizes[0], dtype=torch.uint8, device=device)
        self.modality = torch.zeros(sizes[1], dtype=torch.uint8, device=device)
        self.k_tail = torch.zeros(sizes[2] // 2, dtype=torch.float16, device=device)
        self.v_tail = torch.zeros(sizes[3] // 2, dtype=torch.float16, device=device)
        self.seq_len = torch.zeros(n_layers * batch, dtype=torch.int32, device=device)
        self.status = torch.zeros(4, dtype=torch.int32, device=device)
        self.c = okq_cache(n_layers, batch, n_kv_heads, n_q_heads, HEAD_DIM, WINDOW, capacity, meta_format, schedule, 0,
                           self.records.data_ptr(), self.modality.data_ptr(), self.k_tail.data_ptr(),
                           self.v_tail.data_ptr(), self.seq_len.data_ptr(), self.status.data_ptr())
        self.ref = C.byref(self.c)   # what the calls are handed, built once

    @property
    def group(self):
        return self.n_q_heads // self.n_kv_heads

    def packed_bytes(self, n_tokens):
        """Bytes of packed records a decode step over n_tokens per sequence must read."""
        return self.n_layers * self.batch * self.n_kv_heads * (n_tokens // WINDOW) * (
            RECORD_BYTES_MX if self.meta_format == META_MXFP4 else RECORD_BYTES)

    def device_status(self) -> int:
        return int(self.status[0].item())


def quantize_keys(cache: Cache, layer: int, k: torch.Tensor, signs: torch.Tensor, n_tokens=None, stream=None):
    """k: fp16 [batch, n_kv_heads, n, 128] (last dim contiguous); signs: float32 [128]."""
    assert k.dtype == torch.float16 and k.stride(3) == 1
    n = k.shape[2] if n_tokens is None else n_tokens
    strides = (C.c_int64 * 3)(k.stride(0), k.stride(1), k.stride(2))
    _check(lib().okq_quantize_keys(C.byref(cache.c), layer, _ptr(k), strides, n, _ptr(signs), _stream(stream)),
           "okq_quantize_keys")


def quantize_values(cache: Cache, layer: int, v: torch.Tensor, modality: torch.Tensor, R: torch.Tensor,
                    n_tokens=None, stream=None, bulk=False):
    """v: fp16 [batch, n_kv_heads, n, 128]; modality: uint8 [batch, n]; R: float32 [n_R, 3, 128, 128].
    bulk=True calls okq_quantize_values_bulk (tensor-core rotation)."""
    assert v.dtype == torch.float16 and v.stride(3) == 1 and modality.dtype == torch.uint8 and modality.is_contiguous()
    n = v.shape[2] if n_tokens is None else n_tokens
    assert modality.shape[-1] == n
    strides = (C.c_int64 * 3)(v.stride(0), v.stride(1), v.stride(2))
    n_R = R.shape[0] if R.dim() == 4 else 1
    fn = lib().okq_quantize_values_bulk if bulk else lib().okq_quantize_values
    _check(fn(C.byref(cache.c), layer, _ptr(v), strides, n, _ptr(modality), _ptr(R), n_R, _stream(stream)),
           "okq_quantize_values_bulk" if bulk else "okq_quantize_values")


def debug_bulk_timeout(cache: Cache, layer: int, v: torch.Tensor, modality: torch.Tensor, R: torch.Tensor,
                       limit_clocks: int = 20_000_000, stream=None):
    """okq_debug_bulk_timeout: the bulk value quantiser with its first tile withheld and every wait limited to
    `limit_clocks` SM clocks; the device status word becomes ERR_TIMEOUT (testing aid)."""
    strides = (C.c_int64 * 3)(v.stride(0), v.stride(1), v.stride(2))
    n_R = R.shape[0] if R.dim() == 4 else 1
    _check(lib().okq_debug_bulk_timeout(C.byref(cache.c), layer, _ptr(v), strides, v.shape[2], _ptr(modality), _ptr(R), n_R,
                                        limit_clocks, _stream(stream)), "okq_debug_bulk_timeout")


def append(cache: Cache, layer: int, layer_count: int, k_new, v_new, modality_new, signs, R, n_R=1, stream=None):
    st = (_lib or lib()).okq_append(cache.ref, layer, layer_count, _ptr(k_new), _ptr(v_new), _ptr(modality_new), _ptr(signs),
                                    _ptr(R), n_R, _stream(stream))
    if st != OK:
        raise OkqError(st, "okq_append")


def decode_workspace_bytes(cache: Cache, layer_count: int, num_splits: int = 0) -> int:
    return lib().okq_decode_workspace_bytes(C.byref(cache.c), layer_count, num_splits)


def decode_attention(cache: Cache, layer: int, layer_count: int, q, signs, R, workspace, out, n_R=1,
                     sm_scale=None, num_splits=0, stream=None, simt=False):
    """q: fp16 [layer_count, batch, n_q_heads, 128]; out: float32 same shape; workspace: uint8 device tensor.
    simt=True calls okq_decode_attention_simt (CUDA-core cross-check) instead."""
    L = _lib or lib()
    fn = L.okq_decode_attention_simt if simt else L.okq_decode_attention
    st = fn(cache.ref, layer, layer_count, _ptr(q), HEAD_DIM ** -0.5 if sm_scale is None else sm_scale, _ptr(signs), _ptr(R),
            n_R, _ptr(workspace), 0 if workspace is None else workspace.nbytes, num_splits, _ptr(out), _stream(stream))
    if st != OK:
        raise OkqError(st, "okq_decode_attention")


def decode_attention_noalloc(cache: Cache, layer: int, layer_count: int, q, signs, R, out, n_R=1, sm_scale=None,
                             num_splits=0, stream=None):
    """okq_decode_attention_noalloc: decode_attention (bit for bit where the same kernel takes the call), scratch held inside the library
    (64 MiB per GPU, shared by all calls on that GPU; overlapping calls race).  Allocates nothing."""
    scale = HEAD_DIM ** -0.5 if sm_scale is None else sm_scale
    _check(lib().okq_decode_attention_noalloc(C.byref(cache.c), layer, layer_count, _ptr(q), scale, _ptr(signs),
                                              _ptr(R), n_R, num_splits, _ptr(out), _stream(stream)),
           "okq_decode_attention_noalloc")


def decode_plan(c: okq_cache, layer_count: int, num_splits=0, workspace_bytes=0) -> int:
    """okq_debug_decode_plan: which kernels a decode call on a cache of these sizes would take."""
    return lib().okq_debug_decode_plan(C.byref(c), layer_count, num_splits, workspace_bytes)


def decode_select(impl: int) -> int:
    """Choose the split-K kernel of later decode calls (0: tcgen05, 1: mma.sync, the default); returns the previous choice."""
    return lib().okq_decode_select(impl)


def profile_events(before=None, after=None):
    """Record two torch.cuda.Event objects around the split-K kernel of later decode calls, or around all of a call that takes
    one launch (None clears)."""
    lib().okq_profile_events(None if before is None else before.cuda_event, None if after is None else after.cuda_event)


def cache_export(cache: Cache, layer: int, stream=None):
    """Canonical arrays of one layer as a dict of device tensors."""
    B, H, cap, dev = cache.batch, cache.n_kv_heads, cache.capacity, cache.device
    out = {"k_codes": torch.empty(B, H, cap, 32, dtype=torch.uint8, device=dev),
           "k_norm": torch.empty(B, H, cap, dtype=torch.float16, device=dev),
           "k_meta": torch.empty(B, H, cap // WINDOW, HEAD_DIM, 2, dtype=torch.float16, device=dev),
           "v_codes": torch.empty(B, H, cap, 32, dtype=torch.uint8, device=dev),
           "v_norm": torch.empty(B, H, cap, dtype=torch.float16, device=dev)}
    if cache.meta_format == META_MXFP4:   # k_meta = decoded pairs, k_mx = the stored bytes
        out["k_mx"] = torch.empty(B, H, cap // WINDOW, MX_META_BYTES, dtype=torch.uint8, device=dev)
        _check(lib().okq_cache_export_mx(C.byref(cache.c), layer, _ptr(out["k_codes"]), _ptr(out["k_norm"]),
                                         _ptr(out["k_meta"]), _ptr(out["k_mx"]), _ptr(out["v_codes"]),
                                         _ptr(out["v_norm"]), _stream(stream)), "okq_cache_export_mx")
        return out
    _check(lib().okq_cache_export(C.byref(cache.c), layer, _ptr(out["k_codes"]), _ptr(out["k_norm"]),
                                  _ptr(out["k_meta"]), _ptr(out["v_codes"]), _ptr(out["v_norm"]), _stream(stream)),
           "okq_cache_export")
    return out


def cache_import(cache: Cache, layer: int, arrays: dict, stream=None):
    a = {k: v.contiguous() for k, v in arrays.items()}
    _check(lib().okq_cache_import(C.byref(cache.c), layer, _ptr(a["k_codes"]), _ptr(a["k_norm"]), _ptr(a["k_meta"]),
                                  _ptr(a["v_codes"]), _ptr(a["v_norm"]), _stream(stream)), "okq_cache_import")


# ---- offline calibration of the value rotations (okq_calib.h)

def calib_workspace(group: int, n: int, device="cuda") -> torch.Tensor:
    return torch.empty(lib().okq_calib_workspace_bytes(group, n), dtype=torch.uint8, device=device)


def calib_attention_weights(q, k, workspace, sm_scale=None, causal=True, stream=None):
    """q: fp16 [group, n, 128], k: fp16 [n, 128] (contiguous) -> w float32 [n]."""
    assert q.dtype == torch.float16 and k.dtype == torch.float16 and q.is_contiguous() and k.is_contiguous()
    group, n = q.shape[0], q.shape[1]
    w = torch.empty(n, dtype=torch.float32, device=q.device)
    scale = HEAD_DIM ** -0.5 if sm_scale is None else sm_scale
    _check(lib().okq_calib_attention_weights(_ptr(q), _ptr(k), group, n, scale, 1 if causal else 0, _ptr(workspace),
                                             workspace.numel(), _ptr(w), _stream(stream)), "okq_calib_attention_weights")
    return w


def debug_calib_timeout(q, k, workspace, limit_clocks, stream=None):
    """okq_debug_calib_timeout: the attention weights with every block's first tile withheld and waits limited to
    `limit_clocks` SM clocks."""
    w = torch.empty(q.shape[1], dtype=torch.float32, device=q.device)
    _check(lib().okq_debug_calib_timeout(_ptr(q), _ptr(k), q.shape[0], q.shape[1], _ptr(workspace), workspace.numel(), _ptr(w),
                                         limit_clocks, _stream(stream)), "okq_debug_calib_timeout")
    return w


def calib_moments(v, w, modality, workspace, stream=None):
    """v: fp16 [n, 128], w: float32 [n], modality: uint8 [n] -> C float32 [3, 128, 128]."""
    assert v.dtype == torch.float16 and v.is_contiguous() and w.dtype == torch.float32 and modality.dtype == torch.uint8
    Cm = torch.empty(3, HEAD_DIM, HEAD_DIM, dtype=torch.float32, device=v.device)
    _check(lib().okq_calib_moments(_ptr(v), _ptr(w), _ptr(modality), v.shape[0], _ptr(workspace), workspace.numel(),
                                   _ptr(Cm), _stream(stream)), "okq_calib_moments")
    return Cm


def calib_rotation(Cm, signs, workspace, stream=None):
    """Cm: float32 [128, 128] symmetric, signs: float32 [128] -> (R float32 [128, 128], eigenvalues [128], sweeps)."""
    assert Cm.dtype == torch.float32 and Cm.is_contiguous() and signs.dtype == torch.float32
    R = torch.empty(HEAD_DIM, HEAD_DIM, dtype=torch.float32, device=Cm.device)
    lam = torch.empty(HEAD_DIM, dtype=torch.float32, device=Cm.device)
    sweeps = torch.zeros(1, dtype=torch.int32, device=Cm.device)
    _check(lib().okq_calib_rotation(_ptr(Cm), _ptr(signs), _ptr(workspace), workspace.numel(), _ptr(R), _ptr(lam),
                                    _ptr(sweeps), _stream(stream)), "okq_calib_rotation")
    return R, lam, sweeps


def debug_calib_direct(Cm, signs, stream=None):
    """okq_debug_calib_direct: as calib_rotation, by the direct solver alone; eigenvalue 0 is NaN for a matrix that it leaves."""
    R, lam = torch.empty_like(Cm), torch.empty(HEAD_DIM, dtype=torch.float32, device=Cm.device)
    sweeps = torch.zeros(1, dtype=torch.int32, device=Cm.device)
    _check(lib().okq_debug_calib_direct(_ptr(Cm), _ptr(signs), _ptr(R), _ptr(lam), _ptr(sweeps), _stream(stream)), "okq_debug_calib_direct")
    return R, lam, sweeps


# ---------------------------------------------------------------- bit-width ladder (okq_ladder.h)
class LadderCache:
    """Device buffers of an okq_ladder_cache at `bits` bits per code (canonical layout, one layer)."""

    def __init__(self, batch, n_kv_heads, n_q_heads, capacity, bits, device="cuda"):
        self.bits, self.capacity = bits, capacity
        dev = torch.device(device)
        rows = (batch, n_kv_heads, capacity)
        self.k_codes = torch.zeros(rows + (16 * bits,), dtype=torch.uint8, device=dev)
        self.v_codes = torch.zeros(rows + (16 * bits,), dtype=torch.uint8, device=dev)
        self.k_norm = torch.zeros(rows, dtype=torch.float16, device=dev)
        self.v_norm = torch.zeros(rows, dtype=torch.float16, device=dev)
        self.k_meta = torch.zeros((batch, n_kv_heads, capacity // WINDOW, HEAD_DIM, 2), dtype=torch.float16, device=dev)
        self.modality = torch.zeros((batch, capacity), dtype=torch.uint8, device=dev)
        self.c = okq_ladder_cache(batch, n_kv_heads, n_q_heads, capacity, bits, 0, _ptr(self.k_codes), _ptr(self.k_norm),
                                  _ptr(self.k_meta), _ptr(self.v_codes), _ptr(self.v_norm), _ptr(self.modality))


def ladder_codebook(bits: int):
    """(levels, thresholds) the kernels hold for `bits`, as Python lists of floats."""
    lv, th = (C.c_float * 16)(), (C.c_float * 15)()
    n = lib().okq_ladder_codebook(bits, lv, th)
    if n == 0:
        raise OkqError(ERR_UNSUPPORTED, "okq_ladder_codebook")
    return list(lv)[:n], list(th)[:n - 1]


def ladder_quantize_keys(cache: LadderCache, k: torch.Tensor, signs: torch.Tensor, stream=None):
    assert k.dtype == torch.float16 and k.stride(3) == 1
    strides = (C.c_int64 * 3)(k.stride(0), k.stride(1), k.stride(2))
    _check(lib().okq_ladder_quantize_keys(C.byref(cache.c), _ptr(k), strides, k.shape[2], _ptr(signs), _stream(stream)),
           "okq_ladder_quantize_keys")


def ladder_quantize_values(cache: LadderCache, v: torch.Tensor, modality: torch.Tensor, R: torch.Tensor, stream=None):
    assert v.dtype == torch.float16 and v.stride(3) == 1 and modality.dtype == torch.uint8 and modality.is_contiguous()
    strides = (C.c_int64 * 3)(v.stride(0), v.stride(1), v.stride(2))
    n_R = R.shape[0] if R.dim() == 4 else 1
    _check(lib().okq_ladder_quantize_values(C.byref(cache.c), _ptr(v), strides, v.shape[2], _ptr(modality), _ptr(R), n_R,
                                            _stream(stream)), "okq_ladder_quantize_values")


def debug_ladder_timeout(cache: LadderCache, v: torch.Tensor, modality: torch.Tensor, R: torch.Tensor,
                         limit_clocks: int = 20_000_000, stream=None):
    """okq_debug_ladder_timeout: the ladder's value quantiser with its first tile withheld and every wait limited to
    `limit_clocks` SM clocks; the norms of the tokens concerned become NaN (testing aid)."""
    strides = (C.c_int64 * 3)(v.stride(0), v.stride(1), v.stride(2))
    n_R = R.shape[0] if R.dim() == 4 else 1
    _check(lib().okq_debug_ladder_timeout(C.byref(cache.c), _ptr(v), strides, v.shape[2], _ptr(modality), _ptr(R), n_R, limit_clocks,
                                          _stream(stream)), "okq_debug_ladder_timeout")


def ladder_decode_attention(cache: LadderCache, n_tokens: int, q, signs, R, out, sm_scale=None, stream=None):
    """q: fp16 [batch, n_q_heads, 128]; out: float32 [batch, n_q_heads, 128]."""
    n_R = R.shape[0] if R.dim() == 4 else 1
    scale = HEAD_DIM ** -0.5 if sm_scale is None else sm_scale
    _check(lib().okq_ladder_decode_attention(C.byref(cache.c), n_tokens, _ptr(q), scale, _ptr(signs), _ptr(R), n_R,
                                             _ptr(out), _stream(stream)), "okq_ladder_decode_attention")


def turboquant_encode(x: torch.Tensor, signs: torch.Tensor, bits: int, stream=None):
    """x: fp16 [n, 128] contiguous -> (codes uint8 [n, 16 * bits], norms fp16 [n])."""
    assert x.dtype == torch.float16 and x.is_contiguous() and x.shape[-1] == HEAD_DIM
    n = x.numel() // HEAD_DIM
    codes = torch.empty((n, 16 * bits), dtype=torch.uint8, device=x.device)
    norms = torch.empty((n,), dtype=torch.float16, device=x.device)
    _check(lib().okq_turboquant_encode(_ptr(x), n, bits, _ptr(signs), _ptr(codes), _ptr(norms), _stream(stream)),
           "okq_turboquant_encode")
    return codes, norms


def turboquant_decode(codes: torch.Tensor, norms: torch.Tensor, signs: torch.Tensor, bits: int, stream=None):
    n = norms.numel()
    x_hat = torch.empty((n, HEAD_DIM), dtype=torch.float32, device=codes.device)
    _check(lib().okq_turboquant_decode(_ptr(codes), _ptr(norms), n, bits, _ptr(signs), _ptr(x_hat), _stream(stream)),
           "okq_turboquant_decode")
    return x_hat


# ---------------------------------------------------------------- 8-bit paged cache and rotary positions (okq_paged.h)
DTYPE_CODES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
_strides4 = struct.Struct("4q").pack                 # int64_t[4]
_rope_struct = struct.Struct("4i2Q").pack            # okq_rope
_rope_tensor_struct = struct.Struct("2Q6qi4x").pack  # okq_rope_tensor
_norm_tensor_struct = struct.Struct("3Q9q2Q2i").pack  # okq_norm_tensor


def _here(*tensors):
    """Refuses tensors that do not lie on the current device, where the call is going to run."""
    dev = torch.cuda.current_device() if _device_index is None or not torch.cuda.is_initialized() else _device_index()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"a tensor lies on {t.device}, the call runs on cuda:{dev}")


def paged_sizes(n_layers, batch, n_kv_heads, n_q_heads, n_pages, max_pages, page_tokens=64, dtype=torch.float16):
    """Bytes of codes, scales, raw, table, refs, seq_len and status."""
    shape = okq_paged(n_layers, batch, n_kv_heads, n_q_heads, page_tokens, n_pages, max_pages, DTYPE_CODES[dtype])
    out = (C.c_size_t * 7)()
    _check(lib().okq_paged_sizes(C.byref(shape), out), "okq_paged_sizes")
    return list(out)


class PagedCache:
    """Device buffers of an 8-bit paged cache plus the C struct that describes them.  `buffers`: a dict with codes, scales, raw,
    table, refs and seq_len of the caller's own (shapes as in okq_paged.h); without it an empty cache is made."""

    def __init__(self, n_layers, batch, n_kv_heads, n_q_heads, n_pages=None, max_pages=None, page_tokens=64, dtype=torch.float16,
                 device="cuda", buffers=None):
        if buffers is None:
            paged_sizes(n_layers, batch, n_kv_heads, n_q_heads, n_pages, max_pages, page_tokens, dtype)   # refuses bad shapes
            dev = torch.device(device)
            buffers = {"codes": torch.zeros(n_layers, n_pages, n_kv_heads, 2, page_tokens, HEAD_DIM, dtype=torch.int8, device=dev),
                       "scales": torch.zeros(n_layers, n_pages, n_kv_heads, 2, page_tokens // WINDOW, device=dev),
                       "raw": torch.zeros(n_layers, batch, n_kv_heads, 2, WINDOW, HEAD_DIM, dtype=dtype, device=dev),
                       "table": torch.full((batch, max_pages), -1, dtype=torch.int32, device=dev),
                       "refs": torch.zeros(n_pages, dtype=torch.int32, device=dev),
                       "seq_len": torch.zeros(n_layers, batch, dtype=torch.int32, device=dev)}
        b = buffers
        n_pages, max_pages = b["refs"].numel(), b["table"].shape[1]
        want = {"codes": ((n_layers, n_pages, n_kv_heads, 2, page_tokens, HEAD_DIM), torch.int8),
                "scales": ((n_layers, n_pages, n_kv_heads, 2, page_tokens // WINDOW), torch.float32),
                "raw": ((n_layers, batch, n_kv_heads, 2, WINDOW, HEAD_DIM), dtype), "table": ((batch, max_pages), torch.int32),
                "refs": ((n_pages,), torch.int32), "seq_len": ((n_layers, batch), torch.int32)}
        for name, (shape, dt) in want.items():
            assert tuple(b[name].shape) == shape and b[name].dtype == dt and b[name].is_contiguous(), name
            if b[name].device != b["codes"].device:
                raise ValueError(f"codes on {b['codes'].device}, {name} on {b[name].device}")
        self.codes, self.scales, self.raw, self.table, self.refs, self.seq_len = (b[n] for n in want)
        self.n_layers, self.batch, self.n_kv_heads, self.n_q_heads = n_layers, batch, n_kv_heads, n_q_heads
        self.n_pages, self.max_pages, self.page_tokens, self.dtype, self.device = n_pages, max_pages, page_tokens, dtype, self.codes.device
        self.status = torch.zeros(4, dtype=torch.int32, device=self.device)
        self.c = okq_paged(n_layers, batch, n_kv_heads, n_q_heads, page_tokens, n_pages, max_pages, DTYPE_CODES[dtype],
                           *(t.data_ptr() for t in (self.codes, self.scales, self.raw, self.table, self.refs, self.seq_len, self.status)))
        self.ref = C.byref(self.c)   # what the calls are handed, built once
        _check(lib().okq_paged_sizes(self.ref, (C.c_size_t * 7)()), "PagedCache")

    def device_status(self) -> int:
        return int(self.status[0].item())


def rope_frequencies(theta: float, pairs: int, device="cuda") -> torch.Tensor:
    """float64 [pairs]: theta^(-c / pairs), the usual choice."""
    return (float(theta) ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).to(device)


class Rope:
    """Rotary positions of one call: positions int32 [3, batch, n], freq float64 [pairs] (contiguous, on the device; kept alive here)."""

    def __init__(self, positions, freq, sections, interleaved=False):
        axes, self.batch, self.n = positions.shape
        assert positions.dtype == torch.int32 and axes == 3 and positions.is_contiguous()
        assert freq.dtype == torch.float64 and freq.numel() == sum(sections) and freq.is_contiguous()
        index = freq.get_device()
        if index != positions.get_device() or (index < 0 and freq.device != positions.device):
            raise ValueError(f"positions on {positions.device}, freq on {freq.device}")
        self.positions, self.freq = positions, freq
        self.ref = _rope_struct(*sections, 1 if interleaved else 0, freq.data_ptr(), positions.data_ptr())


def _rope_ref(rope, batch, n):
    if rope is None:
        return None
    assert (rope.batch, rope.n) == (batch, n), "positions are [3, batch, n] of the call's own tokens"
    return rope.ref


def _rope_tensor(x, out, dtype, shape):
    xs, os = x.stride(), out.stride()
    assert x.shape == out.shape == shape and x.dtype == out.dtype == dtype and xs[3] == os[3] == 1
    return _rope_tensor_struct(x.data_ptr(), out.data_ptr(), xs[0], xs[1], xs[2], os[0], os[1], os[2], shape[1])


def rope_apply(rope: Rope, q, q_out, k=None, k_out=None, inverse=False, stream=None):
    """Rotates q and k, [batch, heads, n, 128] of fp16, bf16 or fp32 (last dim contiguous, any other strides), into q_out and k_out
    (which may be the inputs).  inverse=True is the transpose: gradients of the outputs in, gradients of the inputs out."""
    _here(q, q_out, k, k_out, rope.positions, rope.freq)
    batch, heads, n, _ = q.shape
    dtype = q.dtype
    assert (rope.batch, rope.n) == (batch, n), "positions are [3, batch, n] of the call's own tokens"
    q_ref = _rope_tensor(q, q_out, dtype, (batch, heads, n, HEAD_DIM))
    k_ref = None if k is None else _rope_tensor(k, k_out, dtype, (batch, k.shape[1], n, HEAD_DIM))
    st = (_lib or lib()).okq_rope_apply(rope.ref, DTYPE_CODES[dtype], batch, n, q_ref, k_ref, 1 if inverse else 0, _stream(stream))
    if st != OK:
        raise OkqError(st, "okq_rope_apply")


def _norm_tensor(x, up, out, weight, weight_grad, shape):
    """okq_norm_tensor of one side; checks what the C call cannot see."""
    dtype, (x0, x1, x2, x3), (o0, o1, o2, o3) = x.dtype, x.stride(), out.stride()
    assert out.shape == shape and out.dtype == dtype and x3 == 1 and o3 == 1 and shape[3] == HEAD_DIM
    up_ptr, u0, u1, u2 = 0, 0, 0, 0
    if up is not None:
        up_ptr, (u0, u1, u2, u3) = up.data_ptr(), up.stride()
        assert up.shape == shape and up.dtype == dtype and u3 == 1
    weight_ptr = grad_ptr = 0
    code = 2
    if weight is not None:
        weight_ptr, code = weight.data_ptr(), DTYPE_CODES[weight.dtype]
        assert weight.numel() == HEAD_DIM and weight.is_contiguous()
    if weight_grad is not None:
        grad_ptr = weight_grad.data_ptr()
        assert weight_grad.numel() == HEAD_DIM and weight_grad.is_contiguous() and weight_grad.dtype == torch.float32
    return _norm_tensor_struct(x.data_ptr(), up_ptr, out.data_ptr(), x0, x1, x2, u0, u1, u2, o0, o1, o2, weight_ptr, grad_ptr, code, shape[1])


def _norm_sides(rope, q, k):
    """(batch, n, shapes of q and k, the rotation's struct)"""
    shape = q.shape
    batch, n = shape[0], shape[2]
    k_shape = None
    if k is not None:
        k_shape = k.shape
        assert k_shape[0] == batch and k_shape[2] == n and k.dtype == q.dtype
    if rope is None:
        return batch, n, shape, k_shape, None
    assert rope.batch == batch and rope.n == n, "positions are [3, batch, n] of the call's own tokens"
    return batch, n, shape, k_shape, rope.ref


def norm_rope_apply(rope, q, q_out, q_weight=None, k=None, k_out=None, k_weight=None, eps=1e-6, stream=None):
    """Norm of every head of q and k, [batch, heads, n, 128] of fp16, bf16 or fp32 (last dim contiguous, any other strides), with its weight
    ([128] of any of the three types, ones without it), then the rotation (none with rope=None), into q_out and k_out (which may be the
    inputs)."""
    if rope is None:
        _here(q, q_out, q_weight, k, k_out, k_weight)
    else:
        _here(q, q_out, q_weight, k, k_out, k_weight, rope.positions)
    batch, n, shape, k_shape, ref = _norm_sides(rope, q, k)
    st = (_lib or lib()).okq_norm_rope_apply(ref, eps, DTYPE_CODES[q.dtype], batch, n, _norm_tensor(q, None, q_out, q_weight, None, shape),
                                             None if k is None else _norm_tensor(k, None, k_out, k_weight, None, k_shape), _stream(stream))
    if st != OK:
        raise OkqError(st, "okq_norm_rope_apply")


def norm_rope_workspace_bytes(batch: int, n: int, q_heads: int, k_heads: int = 0) -> int:
    return lib().okq_norm_rope_workspace_bytes(batch, n, q_heads, k_heads)


def norm_rope_grad(rope, q, q_up, q_grad, workspace=None, q_weight=None, q_weight_grad=None, k=None, k_up=None, k_grad=None, k_weight=None,
                   k_weight_grad=None, eps=1e-6, stream=None):
    """The gradients of norm_rope_apply's inputs into q_grad and k_grad (which may be q_up and k_up, the gradients of its results) and, where
    q_weight_grad and k_weight_grad (float32 [128], overwritten) are given, those of its weights; q and k as they were before the norm."""
    _here(q, q_up, q_grad, workspace, q_weight, q_weight_grad, k, k_up, k_grad, k_weight, k_weight_grad, None if rope is None else rope.positions)
    assert k is not None or (k_up is None and k_grad is None and k_weight_grad is None), "gradients of keys that were not given"
    batch, n, shape, k_shape, ref = _norm_sides(rope, q, k)
    st = (_lib or lib()).okq_norm_rope_grad(ref, eps, DTYPE_CODES[q.dtype], batch, n, _norm_tensor(q, q_up, q_grad, q_weight, q_weight_grad, shape),
                                            None if k is None else _norm_tensor(k, k_up, k_grad, k_weight, k_weight_grad, k_shape), _ptr(workspace),
                                            0 if workspace is None else workspace.nbytes, _stream(stream))
    if st != OK:
        raise OkqError(st, "okq_norm_rope_grad")


def _rows(cache, x, layer_count, heads, n):
    """Strides of a [layer_count, batch, heads, n, 128] tensor of the cache's dtype."""
    s = x.stride()
    assert x.dtype == cache.dtype and x.shape == (layer_count, cache.batch, heads, n, HEAD_DIM) and s[4] == 1
    return _strides4(s[0], s[1], s[2], s[3])


def paged_append(cache: PagedCache, layer: int, layer_count: int, k, v, new_len=None, rope=None, stream=None):
    """k, v: [layer_count, batch, n_kv_heads, n_new, 128]; new_len: int32 [batch], new tokens of each sequence (all n_new without it);
    rope: a Rope of [3, batch, n_new] positions that the keys are given first."""
    _here(cache.codes, k, v, new_len, None if rope is None else rope.positions)
    n = k.shape[3]
    assert new_len is None or (new_len.dtype == torch.int32 and new_len.is_contiguous() and new_len.numel() == cache.batch)
    st = (_lib or lib()).okq_paged_append(cache.ref, layer, layer_count, k.data_ptr(), _rows(cache, k, layer_count, cache.n_kv_heads, n),
                                          v.data_ptr(), _rows(cache, v, layer_count, cache.n_kv_heads, n), n, _ptr(new_len),
                                          _rope_ref(rope, cache.batch, n), _stream(stream))
    if st != OK:
        raise OkqError(st, "okq_paged_append")


def paged_read(cache: PagedCache, layer: int, layer_count: int, begin: int, k_out, v_out, stream=None):
    """Values of tokens [begin, begin + n) of every sequence into k_out, v_out: [layer_count, batch, n_kv_heads, n, 128], contiguous."""
    _here(cache.codes, k_out, v_out)
    assert k_out.shape == v_out.shape and k_out.is_contiguous() and v_out.is_contiguous() and k_out.dtype == v_out.dtype == cache.dtype
    assert k_out.shape[:3] == (layer_count, cache.batch, cache.n_kv_heads) and k_out.shape[4] == HEAD_DIM
    _check((_lib or lib()).okq_paged_read(cache.ref, layer, layer_count, begin, k_out.shape[3], k_out.data_ptr(), v_out.data_ptr(),
                                          _stream(stream)), "okq_paged_read")


def paged_workspace_bytes(cache: PagedCache, layer_count: int, n_new: int = 1) -> int:
    return lib().okq_paged_workspace_bytes(cache.ref, layer_count, n_new)


def paged_attention(cache: PagedCache, layer: int, layer_count: int, q, workspace, out, q_len=None, rope=None, sm_scale=None, stream=None):
    """q, out: [layer_count, batch, n_q_heads, n_new, 128] of the cache's dtype (last dim contiguous); the queries are those of each
    sequence's newest n_new (q_len[b] with q_len, int32 [batch]) tokens; rope: a Rope that the queries are given first."""
    _here(cache.codes, q, workspace, out, q_len, None if rope is None else rope.positions)
    n = q.shape[3]
    assert q_len is None or (q_len.dtype == torch.int32 and q_len.is_contiguous() and q_len.numel() == cache.batch)
    st = (_lib or lib()).okq_paged_attention(cache.ref, layer, layer_count, q.data_ptr(), _rows(cache, q, layer_count, cache.n_q_heads, n), n,
                                             _ptr(q_len), _rope_ref(rope, cache.batch, n), HEAD_DIM ** -0.5 if sm_scale is None else sm_scale,
                                             _ptr(workspace), 0 if workspace is None else workspace.nbytes, out.data_ptr(),
                                             _rows(cache, out, layer_count, cache.n_q_heads, n), _stream(stream))
    if st != OK:
        raise OkqError(st, "okq_paged_attention")


def paged_attention_window(cache: PagedCache, layer: int, layer_count: int, q, workspace, out, window: int, sinks: int = 0, q_len=None, rope=None,
                           sm_scale=None, stream=None):
    """paged_attention in which a query of token p sees token t <= p where p - t < window or t < sinks."""
    _here(cache.codes, q, workspace, out, q_len, None if rope is None else rope.positions)
    n = q.shape[3]
    assert q_len is None or (q_len.dtype == torch.int32 and q_len.is_contiguous() and q_len.numel() == cache.batch)
    st = (_lib or lib()).okq_paged_attention_window(
        cache.ref, layer, layer_count, q.data_ptr(), _rows(cache, q, layer_count, cache.n_q_heads, n), n, _ptr(q_len), _rope_ref(rope, cache.batch, n),
        HEAD_DIM ** -0.5 if sm_scale is None else sm_scale, window, sinks, _ptr(workspace), 0 if workspace is None else workspace.nbytes,
        out.data_ptr(), _rows(cache, out, layer_count, cache.n_q_heads, n), _stream(stream))
    if st != OK:
        raise OkqError(st, "okq_paged_attention_window")


def _seen(cache, seen, n):
    assert seen.dtype in (torch.int64, torch.uint64) and seen.shape == (cache.batch, n, (n + 63) // 64) and seen.is_contiguous()
    return seen.data_ptr()


def paged_attention_tree(cache: PagedCache, layer: int, layer_count: int, q, workspace, out, seen, q_len=None, rope=None, sm_scale=None, stream=None):
    """paged_attention of each sequence's newest n_new (q_len[b]) tokens as nodes of a tree: query i sees what was there before the nodes, and
    node j where bit j % 64 of seen[b, i, j // 64] is set.  seen: int64 [batch, n_new, ceil(n_new / 64)], as tree_ancestors makes it."""
    _here(cache.codes, q, workspace, out, seen, q_len, None if rope is None else rope.positions)
    n = q.shape[3]
    assert q_len is None or (q_len.dtype == torch.int32 and q_len.is_contiguous() and q_len.numel() == cache.batch)
    st = (_lib or lib()).okq_paged_attention_tree(
        cache.ref, layer, layer_count, q.data_ptr(), _rows(cache, q, layer_count, cache.n_q_heads, n), n, _ptr(q_len), _rope_ref(rope, cache.batch, n),
        HEAD_DIM ** -0.5 if sm_scale is None else sm_scale, _seen(cache, seen, n), _ptr(workspace), 0 if workspace is None else workspace.nbytes,
        out.data_ptr(), _rows(cache, out, layer_count, cache.n_q_heads, n), _stream(stream))
    if st != OK:
        raise OkqError(st, "okq_paged_attention_tree")


def tree_ancestors(cache: PagedCache, parents, seen, depth=None, q_len=None, stream=None):
    """parents: int32 [batch, n_new], each a node before its own or -1.  Writes the bits of every node's ancestors and its own into seen
    (int64 [batch, n_new, ceil(n_new / 64)]) and the number of its ancestors into depth (int32 [batch, n_new])."""
    _here(cache.codes, parents, seen, depth, q_len)
    n = parents.shape[1]
    assert parents.shape[0] == cache.batch and (depth is None or (depth.shape == parents.shape and depth.dtype == torch.int32 and depth.is_contiguous()))
    assert q_len is None or (q_len.dtype == torch.int32 and q_len.is_contiguous() and q_len.numel() == cache.batch)
    _check((_lib or lib()).okq_tree_ancestors(cache.ref, _indices(parents), n, _ptr(q_len), _seen(cache, seen, n), _ptr(depth), _stream(stream)),
           "okq_tree_ancestors")


def debug_paged_timeout(cache: PagedCache, layer: int, layer_count: int, q, workspace, out, limit_clocks: int = 20_000_000, stream=None):
    """okq_debug_paged_timeout: paged_attention with nothing delivered and waits limited to `limit_clocks` SM clocks (testing aid)."""
    _here(cache.codes, q, workspace, out)
    n = q.shape[3]
    _check(lib().okq_debug_paged_timeout(cache.ref, layer, layer_count, q.data_ptr(), _rows(cache, q, layer_count, cache.n_q_heads, n), n,
                                         _ptr(workspace), workspace.nbytes, out.data_ptr(), _rows(cache, out, layer_count, cache.n_q_heads, n),
                                         limit_clocks, _stream(stream)), "okq_debug_paged_timeout")


PLAN_LINE, PLAN_PROMPT = -1, -2


def debug_paged_timeout_sight(cache: PagedCache, layer: int, layer_count: int, q, workspace, out, window: int = 0, sinks: int = 0, seen=None,
                              limit_clocks: int = 20_000_000, stream=None):
    """okq_debug_paged_timeout_sight: the same for paged_attention_window or, with `seen`, paged_attention_tree (testing aid)."""
    _here(cache.codes, q, workspace, out, seen)
    n = q.shape[3]
    _check(lib().okq_debug_paged_timeout_sight(cache.ref, layer, layer_count, q.data_ptr(), _rows(cache, q, layer_count, cache.n_q_heads, n), n,
                                               window, sinks, 0 if seen is None else _seen(cache, seen, n), _ptr(workspace),
                                               0 if workspace is None else workspace.nbytes, out.data_ptr(),
                                               _rows(cache, out, layer_count, cache.n_q_heads, n), limit_clocks, _stream(stream)),
           "okq_debug_paged_timeout_sight")


def paged_plan(cache: PagedCache, layer_count: int, n_new: int = 1) -> int:
    """okq_debug_paged_plan: which kernel a paged_attention call would take."""
    return lib().okq_debug_paged_plan(cache.ref, layer_count, n_new)


def paged_plan_window(cache: PagedCache, layer_count: int, n_new: int, window: int, sinks: int = 0) -> int:
    """okq_debug_paged_plan_window: as paged_plan, for paged_attention_window."""
    return lib().okq_debug_paged_plan_window(cache.ref, layer_count, n_new, window, sinks)


def _indices(x, n=None):
    assert x.dtype == torch.int32 and x.is_contiguous() and (n is None or x.numel() == n)
    return x.data_ptr()


def pages_reserve(cache: PagedCache, tokens, stream=None):
    """tokens: int32 [batch]; gives every sequence pages for at least so many tokens."""
    _here(cache.codes, tokens)
    _check(lib().okq_pages_reserve(cache.ref, _indices(tokens, cache.batch), _stream(stream)), "okq_pages_reserve")


def pages_fork(cache: PagedCache, src, dst, workspace, stream=None):
    """src, dst: int32 [count]; sequence dst[i], empty, becomes a copy of sequence src[i] that shares its full pages."""
    _here(cache.codes, src, dst, workspace)
    _check(lib().okq_pages_fork(cache.ref, _indices(src), _indices(dst, src.numel()), src.numel(), _ptr(workspace),
                                0 if workspace is None else workspace.nbytes, _stream(stream)), "okq_pages_fork")


def pages_release(cache: PagedCache, seqs, stream=None):
    """seqs: int32 [count]; the sequences become empty, pages that no other shares become free."""
    _here(cache.codes, seqs)
    _check(lib().okq_pages_release(cache.ref, _indices(seqs), seqs.numel(), _stream(stream)), "okq_pages_release")


def pages_slide(cache: PagedCache, window: int, sinks: int = 0, dropped=None, stream=None):
    """Gives back the pages that no coming token sees with this window and these sinks; dropped: int32 [batch], tokens that each sequence lost."""
    _here(cache.codes, dropped)
    _check((_lib or lib()).okq_pages_slide(cache.ref, window, sinks, 0 if dropped is None else _indices(dropped, cache.batch), _stream(stream)), "okq_pages_slide")


def pages_copy(cache: PagedCache, src, dst, stream=None):
    """src, dst: int32 [count] pages; codes and scales of src[i] go to dst[i]."""
    _here(cache.codes, src, dst)
    _check(lib().okq_pages_copy(cache.ref, _indices(src), _indices(dst, src.numel()), src.numel(), _stream(stream)), "okq_pages_copy")


def pages_compact(cache: PagedCache, workspace, n_live=None, stream=None):
    """Moves the pages in use to the front of the pool; n_live: int32 [1], receives their number."""
    _here(cache.codes, workspace, n_live)
    _check(lib().okq_pages_compact(cache.ref, 0 if n_live is None else _indices(n_live, 1), _ptr(workspace),
                                   0 if workspace is None else workspace.nbytes, _stream(stream)), "okq_pages_compact")
