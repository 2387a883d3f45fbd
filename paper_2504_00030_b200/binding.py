"""ctypes binding of libspecverify.so -- argument marshalling only.

Every function here has the name and the arguments of the C entry point it
calls (``include/specverify.h``); torch tensors stand in for device pointers.
Nothing is computed in Python, and there is no fallback: if the shared library
has not been built the first call raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspecverify.so")

SV_OK, SV_EINVAL, SV_EUNSUPPORTED, SV_EALIGN, SV_ECUDA, SV_EWORKSPACE = 0, -1, -2, -3, -4, -5
SV_DEV_BAD_GAMMA, SV_DEV_BAD_PAGE, SV_DEV_BAD_TOKEN = 1, 2, 4
SV_DEV_NONFINITE, SV_DEV_TIMEOUT, SV_DEV_BAD_LEN, SV_DEV_NO_PAGES = 8, 16, 32, 64
SV_GT_FIXED, SV_GT_PROPOSED, SV_GT_LITERAL = 0, 1, 2

EXPORTS = (
    "sv_status_str", "sv_launch_count", "spec_kv_pool_register", "spec_kv_pool_release",
    "spec_verify_attn_workspace_bytes", "spec_verify_attn", "spec_accept_sample_workspace_bytes",
    "spec_accept_sample", "spec_accept_sample_static", "gamma_tune_update", "gamma_tune_init",
    "spec_verify_step_host", "spec_draft_stop_workspace_bytes", "spec_draft_stop", "spec_kv_append",
    "sv_selftest_wait_expiry", "spec_verify_attn_layers", "spec_draft_step_workspace_bytes", "spec_draft_step",
    "spec_kv_pages_update", "spec_rope_append", "spec_logits_adjust", "spec_token_counts_update",
    "spec_page_bounds_update", "spec_page_select", "spec_page_select_workspace_bytes", "spec_verify_attn_pages",
    "spec_verify_attn_pages_workspace_bytes", "spec_verify_attn_prefix", "spec_verify_attn_prefix_workspace_bytes",
)


class SpecVerifyError(RuntimeError):
    def __init__(self, where: str, status: int):
        self.status = status
        super().__init__(f"{where}: {status_str(status)} ({status})")


class AttnParams(C.Structure):
    _fields_ = [("q", C.c_void_p), ("o", C.c_void_p), ("lse", C.c_void_p), ("pool", C.c_void_p),
                ("block_table", C.c_void_p), ("block_table_stride", C.c_int64),
                ("seq_len", C.c_void_p), ("gamma", C.c_void_p), ("cu_q", C.c_void_p),
                ("batch", C.c_int32), ("gamma_max", C.c_int32), ("hq", C.c_int32),
                ("hkv", C.c_int32), ("head_dim", C.c_int32), ("max_seq_len", C.c_int32),
                ("sm_scale", C.c_float), ("device_status", C.c_void_p)]


class AttnLayersParams(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("pools", C.POINTER(C.c_void_p)), ("q", C.POINTER(C.c_void_p)),
                ("o", C.POINTER(C.c_void_p)), ("lse", C.POINTER(C.c_void_p)), ("k_new", C.POINTER(C.c_void_p)),
                ("v_new", C.POINTER(C.c_void_p)), ("shared", AttnParams)]


class KvAppendParams(C.Structure):
    _fields_ = [("k_new", C.c_void_p), ("v_new", C.c_void_p), ("pool", C.c_void_p),
                ("block_table", C.c_void_p), ("block_table_stride", C.c_int64),
                ("seq_len", C.c_void_p), ("gamma", C.c_void_p), ("cu_q", C.c_void_p),
                ("batch", C.c_int32), ("gamma_max", C.c_int32), ("device_status", C.c_void_p)]


class KvPagesParams(C.Structure):
    _fields_ = [("seq_len", C.c_void_p), ("batch", C.c_int32), ("block_table", C.c_void_p),
                ("block_table_stride", C.c_int64), ("n_held", C.c_void_p), ("free_list", C.c_void_p),
                ("n_free", C.c_void_p), ("n_pages", C.c_int64), ("page_size", C.c_int32),
                ("gamma", C.c_void_p), ("cu_q", C.c_void_p), ("gamma_max", C.c_int32),
                ("slot_map", C.c_void_p), ("positions", C.c_void_p), ("n_rows", C.c_int64),
                ("device_status", C.c_void_p)]


class RopeAppendParams(C.Structure):
    _fields_ = [("q", C.c_void_p), ("q_stride", C.c_int64), ("k_new", C.c_void_p), ("k_stride", C.c_int64),
                ("v_new", C.c_void_p), ("v_stride", C.c_int64), ("q_out", C.c_void_p), ("pool", C.c_void_p),
                ("hq", C.c_int32), ("n_rows", C.c_int64), ("slot_map", C.c_void_p), ("positions", C.c_void_p),
                ("n_axes", C.c_int32), ("freq_axis", C.c_void_p), ("inv_freq", C.c_void_p), ("rot_dim", C.c_int32),
                ("interleaved", C.c_int32), ("rope_scale", C.c_float), ("q_weight", C.c_void_p),
                ("k_weight", C.c_void_p), ("weights_f32", C.c_int32), ("eps", C.c_float),
                ("device_status", C.c_void_p)]


class LogitsAdjustParams(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("out", C.c_void_p), ("row_stride", C.c_int64), ("out_stride", C.c_int64),
                ("n_rows", C.c_int64), ("vocab", C.c_int32), ("logits_bf16", C.c_int32), ("batch", C.c_int32),
                ("gamma_max", C.c_int32), ("gamma", C.c_void_p), ("cu_q", C.c_void_p), ("cu_d", C.c_void_p),
                ("n_drafted", C.c_void_p), ("active", C.c_void_p), ("draft_tokens", C.c_void_p),
                ("n_d_rows", C.c_int64), ("token_counts", C.c_void_p), ("count_stride", C.c_int64),
                ("repetition", C.c_void_p), ("frequency", C.c_void_p), ("presence", C.c_void_p),
                ("bias_tokens", C.c_void_p), ("bias_values", C.c_void_p), ("n_bias", C.c_void_p),
                ("bias_stride", C.c_int32), ("mask", C.c_void_p), ("mask_stride", C.c_int64),
                ("device_status", C.c_void_p)]


class TokenCountsParams(C.Structure):
    _fields_ = [("token_counts", C.c_void_p), ("count_stride", C.c_int64), ("vocab", C.c_int32),
                ("batch", C.c_int32), ("tokens", C.c_void_p), ("token_stride", C.c_int64),
                ("cu_tokens", C.c_void_p), ("n_tokens", C.c_int64), ("max_tokens", C.c_int32),
                ("reset", C.c_void_p), ("prompt", C.c_int32), ("device_status", C.c_void_p)]


class PageBoundsParams(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("bounds", C.c_void_p), ("scales", C.c_void_p), ("block_table", C.c_void_p),
                ("block_table_stride", C.c_int64), ("seq_len", C.c_void_p), ("gamma", C.c_void_p),
                ("first", C.c_void_p), ("batch", C.c_int32), ("max_new", C.c_int32), ("device_status", C.c_void_p)]


class PageSelectParams(C.Structure):
    _fields_ = [("q", C.c_void_p), ("bounds", C.c_void_p), ("scales", C.c_void_p), ("n_pages", C.c_int64),
                ("block_table", C.c_void_p), ("block_table_stride", C.c_int64), ("seq_len", C.c_void_p),
                ("gamma", C.c_void_p), ("cu_q", C.c_void_p), ("batch", C.c_int32), ("gamma_max", C.c_int32),
                ("hq", C.c_int32), ("hkv", C.c_int32), ("head_dim", C.c_int32), ("max_seq_len", C.c_int32),
                ("n_select", C.c_int32), ("n_first", C.c_int32), ("n_last", C.c_int32), ("page_list", C.c_void_p),
                ("row_mask", C.c_void_p), ("n_list", C.c_void_p), ("list_stride", C.c_int64),
                ("device_status", C.c_void_p)]


class AttnPagesParams(C.Structure):
    _fields_ = [("attn", AttnParams), ("page_list", C.c_void_p), ("row_mask", C.c_void_p), ("n_list", C.c_void_p),
                ("list_stride", C.c_int64)]


class AttnPrefixParams(C.Structure):
    _fields_ = [("attn", AttnParams), ("group", C.c_void_p), ("prefix_len", C.c_void_p), ("n_groups", C.c_int32)]


class AcceptParams(C.Structure):
    _fields_ = [("target_logits", C.c_void_p), ("draft_logits", C.c_void_p),
                ("row_stride", C.c_int64), ("vocab", C.c_int32), ("draft_tokens", C.c_void_p),
                ("u_accept", C.c_void_p), ("u_sample", C.c_void_p), ("temperature", C.c_float),
                ("temperature_per_seq", C.c_void_p), ("gamma", C.c_void_p), ("cu_q", C.c_void_p),
                ("cu_d", C.c_void_p), ("batch", C.c_int32), ("gamma_max", C.c_int32),
                ("n_accepted", C.c_void_p), ("out_tokens", C.c_void_p), ("ratio", C.c_void_p),
                ("logZ_p", C.c_void_p), ("logZ_q", C.c_void_p), ("flag_count", C.c_void_p),
                ("device_status", C.c_void_p), ("logits_bf16", C.c_int32)]


class GammaConfigC(C.Structure):
    _fields_ = [("eta", C.c_double), ("delta", C.c_double), ("gamma_min", C.c_int32),
                ("gamma_max", C.c_int32), ("mode", C.c_int32), ("padded_rows", C.c_int32)]


class GammaParams(C.Structure):
    _fields_ = [("n_accepted", C.c_void_p), ("gamma_bar", C.c_void_p), ("gamma", C.c_void_p),
                ("seq_len", C.c_void_p), ("cu_q", C.c_void_p), ("cu_d", C.c_void_p),
                ("batch", C.c_int32), ("config", GammaConfigC), ("trajectory", C.c_void_p),
                ("accepted_log", C.c_void_p), ("step", C.c_int32), ("device_status", C.c_void_p),
                ("n_drafted", C.c_void_p)]


class DraftStopParams(C.Structure):
    _fields_ = [("draft_logits", C.c_void_p), ("row_stride", C.c_int64), ("vocab", C.c_int32),
                ("temperature", C.c_float), ("temperature_per_seq", C.c_void_p), ("tau", C.c_float),
                ("gamma", C.c_void_p), ("cu_d", C.c_void_p), ("batch", C.c_int32), ("gamma_max", C.c_int32),
                ("n_drafted", C.c_void_p), ("top_prob", C.c_void_p), ("device_status", C.c_void_p),
                ("logits_bf16", C.c_int32)]


class DraftStepParams(C.Structure):
    _fields_ = [("draft_logits", C.c_void_p), ("row_stride", C.c_int64), ("vocab", C.c_int32),
                ("temperature", C.c_float), ("temperature_per_seq", C.c_void_p), ("tau", C.c_float),
                ("u_sample", C.c_void_p), ("gamma", C.c_void_p), ("cu_d", C.c_void_p), ("batch", C.c_int32),
                ("gamma_max", C.c_int32), ("n_drafted", C.c_void_p), ("active", C.c_void_p),
                ("draft_tokens", C.c_void_p), ("top_prob", C.c_void_p), ("device_status", C.c_void_p),
                ("logits_bf16", C.c_int32)]


class StepHostIO(C.Structure):
    _fields_ = [("q_host", C.c_void_p), ("target_logits_host", C.c_void_p),
                ("draft_logits_host", C.c_void_p), ("draft_tokens_host", C.c_void_p),
                ("u_accept_host", C.c_void_p), ("u_sample_host", C.c_void_p),
                ("n_q_rows", C.c_int64), ("n_d_rows", C.c_int64), ("n_accepted_host", C.c_void_p),
                ("out_tokens_host", C.c_void_p), ("gamma_next_host", C.c_void_p),
                ("o_host", C.c_void_p)]


_lib = None


def load():
    """Load libspecverify.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2504_00030_b200.build` "
                "(there is no fallback path)")
        lib = C.CDLL(LIB_PATH)
        lib.sv_status_str.restype = C.c_char_p
        lib.sv_status_str.argtypes = [C.c_int32]
        lib.sv_launch_count.restype = C.c_uint64
        lib.spec_kv_pool_register.restype = C.c_int32
        lib.spec_kv_pool_register.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_int32,
                                              C.c_int32, C.POINTER(C.c_int64), C.POINTER(C.c_void_p)]
        lib.spec_kv_pool_release.restype = C.c_int32
        lib.spec_kv_pool_release.argtypes = [C.c_void_p]
        lib.spec_verify_attn_workspace_bytes.restype = C.c_size_t
        lib.spec_verify_attn_workspace_bytes.argtypes = [C.c_int32] * 6
        lib.spec_accept_sample_workspace_bytes.restype = C.c_size_t
        lib.spec_accept_sample_workspace_bytes.argtypes = [C.c_int32] * 3
        lib.spec_verify_attn.restype = C.c_int32
        lib.spec_verify_attn.argtypes = [C.POINTER(AttnParams), C.c_void_p, C.c_size_t, C.c_void_p]
        lib.spec_accept_sample.restype = C.c_int32
        lib.spec_accept_sample.argtypes = [C.POINTER(AcceptParams), C.c_void_p, C.c_size_t, C.c_void_p]
        lib.spec_accept_sample_static.restype = C.c_int32
        lib.spec_accept_sample_static.argtypes = [C.POINTER(AcceptParams), C.c_void_p]
        lib.gamma_tune_update.restype = C.c_int32
        lib.gamma_tune_update.argtypes = [C.POINTER(GammaParams), C.c_void_p]
        lib.gamma_tune_init.restype = C.c_int32
        lib.gamma_tune_init.argtypes = [C.POINTER(GammaParams), C.c_int32, C.c_void_p]
        lib.spec_verify_attn_layers.restype = C.c_int32
        lib.spec_verify_attn_layers.argtypes = [C.POINTER(AttnLayersParams), C.c_void_p, C.c_size_t, C.c_void_p]
        lib.sv_selftest_wait_expiry.restype = C.c_int32
        lib.sv_selftest_wait_expiry.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
        lib.spec_draft_stop_workspace_bytes.restype = C.c_size_t
        lib.spec_draft_stop_workspace_bytes.argtypes = [C.c_int32] * 3
        lib.spec_draft_stop.restype = C.c_int32
        lib.spec_draft_stop.argtypes = [C.POINTER(DraftStopParams), C.c_void_p, C.c_size_t, C.c_void_p]
        lib.spec_draft_step_workspace_bytes.restype = C.c_size_t
        lib.spec_draft_step_workspace_bytes.argtypes = [C.c_int32] * 2
        lib.spec_kv_pages_update.restype = C.c_int32
        lib.spec_kv_pages_update.argtypes = [C.c_void_p, C.c_void_p]      # KvPagesParams, or its bytes
        lib.spec_rope_append.restype = C.c_int32
        lib.spec_rope_append.argtypes = [C.c_void_p, C.c_void_p]      # RopeAppendParams, or its bytes
        lib.spec_logits_adjust.restype = C.c_int32
        lib.spec_logits_adjust.argtypes = [C.c_void_p, C.c_void_p]      # LogitsAdjustParams, or its bytes
        lib.spec_token_counts_update.restype = C.c_int32
        lib.spec_token_counts_update.argtypes = [C.c_void_p, C.c_void_p]      # TokenCountsParams, or its bytes
        lib.spec_page_bounds_update.restype = C.c_int32
        lib.spec_page_bounds_update.argtypes = [C.c_void_p, C.c_void_p]      # PageBoundsParams, or its bytes
        lib.spec_page_select_workspace_bytes.restype = C.c_size_t
        lib.spec_page_select_workspace_bytes.argtypes = [C.c_int32] * 4
        lib.spec_page_select.restype = C.c_int32
        lib.spec_page_select.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]      # PageSelectParams, or its bytes
        lib.spec_verify_attn_pages_workspace_bytes.restype = C.c_size_t
        lib.spec_verify_attn_pages_workspace_bytes.argtypes = [C.c_int32] * 5
        lib.spec_verify_attn_pages.restype = C.c_int32
        lib.spec_verify_attn_pages.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]      # AttnPagesParams, or its bytes
        lib.spec_verify_attn_prefix_workspace_bytes.restype = C.c_size_t
        lib.spec_verify_attn_prefix_workspace_bytes.argtypes = [C.c_int32] * 6
        lib.spec_verify_attn_prefix.restype = C.c_int32
        lib.spec_verify_attn_prefix.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]      # AttnPrefixParams, or its bytes
        lib.spec_draft_step.restype = C.c_int32
        lib.spec_draft_step.argtypes = [C.POINTER(DraftStepParams), C.c_void_p, C.c_size_t, C.c_void_p]
        lib.spec_verify_step_host.restype = C.c_int32
        lib.spec_verify_step_host.argtypes = [C.POINTER(StepHostIO), C.POINTER(AttnParams), C.c_void_p,
                                              C.c_size_t, C.POINTER(AcceptParams), C.c_void_p,
                                              C.c_size_t, C.POINTER(GammaParams), C.c_void_p]
        _lib = lib
    return _lib


def status_str(status: int) -> str:
    return load().sv_status_str(int(status)).decode()


def sv_launch_count() -> int:
    return int(load().sv_launch_count())


def _check(where: str, status: int):
    if status != SV_OK:
        raise SpecVerifyError(where, status)


def _dev(t, dtype, name, allow_none=False):
    """Device pointer of a CUDA tensor (dtype and contiguity checked)."""
    if t is None:
        if allow_none:
            return None
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _dev_rows(t, dtype, name):
    """Device pointer of a 2-D CUDA tensor whose rows are contiguous; the rows may be strided."""
    if t is None or not t.is_cuda or t.dtype != dtype or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be a 2-D CUDA tensor of {dtype} with contiguous rows")
    return t.data_ptr()


def _host(t, dtype, name, allow_none=False):
    if t is None:
        if allow_none:
            return None
        raise ValueError(f"{name} is required")
    if t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous host tensor of {dtype}")
    return t.data_ptr()


def _launch_at(stream, first, name):
    """Device index and raw stream of a launch: the current device, where the tensors have to be.  (The raw stream of
    the current device is asked for by index: building a Stream object costs more than the launch.)"""
    if not first.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    index = torch._C._cuda_getDevice()                         # there is a CUDA tensor, so CUDA has been initialised
    if stream is None:
        return index, torch._C._cuda_getCurrentRawStream(index)
    if stream.device.index != index:
        raise ValueError(f"the stream is on {stream.device}, the current device is cuda:{index}")
    return index, stream.cuda_stream


def _on(t, dtype, name, index, n=-1):
    """Device pointer of a contiguous tensor of `dtype` (and `n` entries) on CUDA device `index`; 0 for None."""
    if t is None:
        return 0
    if t.get_device() == index and t.dtype is dtype and t.is_contiguous() and (n < 0 or t.numel() == n):
        return t.data_ptr()
    _dev(t, dtype, name)
    if n >= 0 and t.numel() != n:
        raise ValueError(f"{name} must have {n} entries, got {t.numel()}")
    raise ValueError(f"{name} is on {t.device}, the current device is cuda:{index}")


def _rows_on(t, dtype, name, index):
    """Device pointer, row stride and shape of a 2-D tensor on the device `index` with contiguous rows."""
    if t.get_device() == index and t.dtype is dtype and t.dim() == 2:
        rows, cols = t.shape
        s0, s1 = t.stride()
        if s1 == 1 or cols <= 1:
            return t.data_ptr(), s0 if rows > 1 else max(cols, s0), rows, cols
    raise ValueError(f"{name} must be a 2-D tensor of {dtype} with contiguous rows on the current device (cuda:{index})")


def _packer(cls):
    """Packs field values as the C struct of a ctypes Structure has them: a third of the time that its constructor takes."""
    codes = {C.c_void_p: "P", C.c_int64: "q", C.c_int32: "i", C.c_float: "f"}

    def of(c):      # a nested struct's fields in its place: it is aligned as its first field, a pointer, is, and padded to one
        return "".join(of(ty) + "0q" if issubclass(ty, C.Structure) else codes[ty] for _, ty in c._fields_)

    return struct.Struct("@" + of(cls) + "0q").pack


def _nbytes(t) -> int:
    return t.numel() * t.element_size()


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


# --------------------------------------------------------------------------- KV pool
class KVPool:
    """Handle of a registered paged KV pool (keeps the tensors alive)."""

    def __init__(self, k_pool: torch.Tensor, v_pool: torch.Tensor, strides=None):
        if k_pool.dim() != 4 or k_pool.shape != v_pool.shape:
            raise ValueError("pools must be 4-D [n_pages, hkv, page_size, head_dim] and alike")
        n_pages, hkv, page_size, head_dim = k_pool.shape
        if strides is None:
            strides = k_pool.stride()
            if tuple(v_pool.stride()) != tuple(strides):
                raise ValueError("K and V pools must share their strides")
        if not (k_pool.is_cuda and v_pool.is_cuda and k_pool.dtype == torch.bfloat16 and
                v_pool.dtype == torch.bfloat16):
            raise ValueError("pools must be CUDA bf16 tensors")
        self.k_pool, self.v_pool = k_pool, v_pool
        self.n_pages, self.hkv, self.page_size, self.head_dim = n_pages, hkv, page_size, head_dim
        st = (C.c_int64 * 4)(*[int(s) for s in strides])
        handle = C.c_void_p()
        self.handle = None
        _check("spec_kv_pool_register",
               load().spec_kv_pool_register(k_pool.data_ptr(), v_pool.data_ptr(), n_pages, page_size,
                                            hkv, head_dim, st, C.byref(handle)))
        self.handle = handle

    def release(self):
        if self.handle is not None and self.handle.value:
            load().spec_kv_pool_release(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.release()
        except Exception:
            pass


def spec_kv_pool_register(k_pool, v_pool, strides=None) -> KVPool:
    return KVPool(k_pool, v_pool, strides)


# --------------------------------------------------------------------------- attention
def spec_verify_attn_workspace_bytes(batch, gamma_max, hq, hkv, head_dim, max_seq_len) -> int:
    return int(load().spec_verify_attn_workspace_bytes(batch, gamma_max, hq, hkv, head_dim, max_seq_len))


def attn_params(q, o, pool: KVPool, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len,
                sm_scale=None, lse=None, device_status=None) -> AttnParams:
    n_rows, hq, head_dim = q.shape
    p = AttnParams()
    p.q = _dev(q, torch.bfloat16, "q")
    p.o = _dev(o, torch.bfloat16, "o")
    p.lse = _dev(lse, torch.float32, "lse", True)
    p.pool = pool.handle
    p.block_table = _dev(block_table, torch.int32, "block_table")
    p.block_table_stride = block_table.shape[1]
    p.seq_len = _dev(seq_len, torch.int32, "seq_len")
    p.gamma = _dev(gamma, torch.int32, "gamma")
    p.cu_q = _dev(cu_q, torch.int32, "cu_q")
    p.batch = seq_len.shape[0]
    p.gamma_max = gamma_max
    p.hq, p.hkv, p.head_dim = hq, pool.hkv, head_dim
    p.max_seq_len = max_seq_len
    p.sm_scale = float(sm_scale) if sm_scale is not None else head_dim ** -0.5
    p.device_status = _dev(device_status, torch.int32, "device_status", True)
    return p


def spec_verify_attn(q, o, pool, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len,
                     workspace, sm_scale=None, lse=None, device_status=None, stream=None):
    """Attention of the draft block against the paged KV cache (asynchronous)."""
    p = attn_params(q, o, pool, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len,
                    sm_scale, lse, device_status)
    _check("spec_verify_attn",
           load().spec_verify_attn(C.byref(p), workspace.data_ptr(), _nbytes(workspace), _stream(stream)))


def kv_append_params(k_new, v_new, pool, block_table, seq_len, gamma, cu_q, gamma_max,
                     device_status=None) -> KvAppendParams:
    p = KvAppendParams()
    p.k_new = _dev(k_new, torch.bfloat16, "k_new")
    p.v_new = _dev(v_new, torch.bfloat16, "v_new")
    if tuple(k_new.shape) != tuple(v_new.shape) or k_new.dim() != 3:
        raise ValueError("k_new and v_new must both be [n_rows, hkv, head_dim]")
    if tuple(k_new.shape[1:]) != (pool.hkv, pool.head_dim):
        raise ValueError("k_new rows do not match the pool's heads and head_dim")
    p.pool = pool.handle
    p.block_table = _dev(block_table, torch.int32, "block_table")
    p.block_table_stride = block_table.shape[1]
    p.seq_len = _dev(seq_len, torch.int32, "seq_len")
    p.gamma = _dev(gamma, torch.int32, "gamma")
    p.cu_q = _dev(cu_q, torch.int32, "cu_q")
    p.batch = gamma.shape[0]
    p.gamma_max = gamma_max
    p.device_status = _dev(device_status, torch.int32, "device_status", True)
    return p


def spec_kv_append(k_new, v_new, pool, block_table, seq_len, gamma, cu_q, gamma_max, device_status=None,
                   stream=None):
    """Write the draft block's keys and values behind each sequence's context (asynchronous)."""
    p = kv_append_params(k_new, v_new, pool, block_table, seq_len, gamma, cu_q, gamma_max, device_status)
    _check("spec_kv_append", load().spec_kv_append(C.byref(p), _stream(stream)))


# --------------------------------------------------------------------------- block tables and slot maps
def _kv_pages_args(index, seq_len, block_table, n_held, free_list, n_free, gamma=None, cu_q=None, gamma_max=0,
                   slot_map=None, positions=None, device_status=None):
    i32, batch = torch.int32, seq_len.numel()
    if block_table.dim() != 2 or block_table.shape[0] != batch:
        raise ValueError("block_table must have one row per sequence")
    n_rows = slot_map.numel() if slot_map is not None else positions.numel() if positions is not None else 0
    return (_on(seq_len, i32, "seq_len", index), batch, _on(block_table, i32, "block_table", index), block_table.shape[1],
            _on(n_held, i32, "n_held", index, batch), _on(free_list, i32, "free_list", index),
            _on(n_free, i32, "n_free", index, 1), free_list.numel(), 16, _on(gamma, i32, "gamma", index, batch),
            _on(cu_q, i32, "cu_q", index, batch + 1), gamma_max, _on(slot_map, torch.int64, "slot_map", index),
            _on(positions, i32, "positions", index, n_rows), n_rows, _on(device_status, i32, "device_status", index))


def kv_pages_params(*args, **kwargs) -> KvPagesParams:
    """Arguments of spec_kv_pages_update (without stream)."""
    return KvPagesParams(*_kv_pages_args(torch.cuda.current_device(), *args, **kwargs))


_pack_kv_pages = _packer(KvPagesParams)


def spec_kv_pages_update(seq_len, block_table, n_held, free_list, n_free, gamma=None, cu_q=None, gamma_max=0,
                         slot_map=None, positions=None, device_status=None, stream=None):
    """Block table, held pages and free stack brought to the lengths of the coming step, and the cache slot and
    position of each of its rows (asynchronous)."""
    index, raw = _launch_at(stream, seq_len, "seq_len")
    p = _pack_kv_pages(*_kv_pages_args(index, seq_len, block_table, n_held, free_list, n_free, gamma, cu_q, gamma_max,
                                       slot_map, positions, device_status))
    _check("spec_kv_pages_update", load().spec_kv_pages_update(p, raw))


# --------------------------------------------------------------------------- norm, rotation and append in one pass
def _head_rows(t, heads, head_dim, n_rows, name, index):
    """Device pointer and row stride of [n_rows, heads, head_dim] bf16 heads; the rows may be strided."""
    if t.get_device() != index or t.dtype != torch.bfloat16:
        raise ValueError(f"{name} must be a bf16 tensor on the current device (cuda:{index})")
    if t.shape != (n_rows, heads, head_dim):
        raise ValueError(f"{name} must be [{n_rows}, {heads}, {head_dim}], got {tuple(t.shape)}")
    s0, s1, s2 = t.stride()
    if s2 != 1 or (s1 != head_dim and heads > 1):
        raise ValueError(f"the heads of a row of {name} must be contiguous")
    return t.data_ptr(), s0 if n_rows > 1 else heads * head_dim


def _rope_append_args(index, q, k_new, v_new, q_out, pool, positions, slot_map, inv_freq, q_weight=None, k_weight=None,
                      eps=1e-6, interleaved=False, freq_axis=None, rope_scale=1.0, device_status=None):
    if q.dim() != 3:
        raise ValueError("q must be [n_rows, hq, head_dim]")
    n_rows, hq, head_dim = q.shape
    if head_dim != pool.head_dim:
        raise ValueError("q's head_dim is not the pool's")
    if pool.handle is None:
        raise ValueError("the pool has been released")
    if pool.k_pool.get_device() != index or pool.v_pool.get_device() != index:
        raise ValueError(f"the pool's memory is not on the current device (cuda:{index})")
    qp, qs = _head_rows(q, hq, head_dim, n_rows, "q", index)
    kp, ks = _head_rows(k_new, pool.hkv, head_dim, n_rows, "k_new", index)
    vp, vs = _head_rows(v_new, pool.hkv, head_dim, n_rows, "v_new", index)
    if q_out.shape != q.shape:
        raise ValueError("q_out must have q's shape")
    axes = positions.shape[0] if positions.dim() == 2 else 1
    nf = inv_freq.numel() if inv_freq is not None else 0
    w = q_weight if q_weight is not None else k_weight
    wt = torch.float32 if w is not None and w.dtype == torch.float32 else torch.bfloat16      # float32 or bf16 weights
    return (qp, qs, kp, ks, vp, vs, _on(q_out, torch.bfloat16, "q_out", index), pool.handle.value, hq, n_rows,
            _on(slot_map, torch.int64, "slot_map", index, n_rows), _on(positions, torch.int32, "positions", index, axes * n_rows),
            axes, _on(freq_axis, torch.uint8, "freq_axis", index, nf), _on(inv_freq, torch.float64, "inv_freq", index), 2 * nf,
            1 if interleaved else 0, rope_scale, _on(q_weight, wt, "q_weight", index, head_dim),
            _on(k_weight, wt, "k_weight", index, head_dim), 1 if wt == torch.float32 else 0, eps,
            _on(device_status, torch.int32, "device_status", index))


def rope_append_params(*args, **kwargs) -> RopeAppendParams:
    """Arguments of spec_rope_append (without stream)."""
    return RopeAppendParams(*_rope_append_args(torch.cuda.current_device(), *args, **kwargs))


_pack_rope_append = _packer(RopeAppendParams)


def spec_rope_append(q, k_new, v_new, q_out, pool, positions, slot_map, inv_freq, q_weight=None, k_weight=None,
                     eps=1e-6, interleaved=False, freq_axis=None, rope_scale=1.0, device_status=None, stream=None):
    """Per-head norm of queries and keys, position rotation, and keys and values written into the paged cache by slot
    (asynchronous).  q, k_new and v_new may be views of one projection's output."""
    index, raw = _launch_at(stream, q, "q")
    p = _pack_rope_append(*_rope_append_args(index, q, k_new, v_new, q_out, pool, positions, slot_map, inv_freq, q_weight,
                                             k_weight, eps, interleaved, freq_axis, rope_scale, device_status))
    _check("spec_rope_append", load().spec_rope_append(p, raw))


# --------------------------------------------------------------------------- penalties, biases and grammar masks
def _logits_adjust_args(index, logits, out, gamma, cu_q, cu_d, gamma_max, draft_tokens=None, token_counts=None, repetition=None,
                        frequency=None, presence=None, bias_tokens=None, bias_values=None, n_bias=None, mask=None,
                        n_drafted=None, active=None, device_status=None):
    i32, f32 = torch.int32, torch.float32
    bf16 = logits.dtype == torch.bfloat16                                         # float32 or bf16 logits
    ldt = torch.bfloat16 if bf16 else f32
    lp, ls, n_rows, vocab = _rows_on(logits, ldt, "logits", index)
    op, os_ = lp, ls
    if out is not logits:
        op, os_, o_rows, o_cols = _rows_on(out, ldt, "out", index)
        if o_rows != n_rows or o_cols != vocab:
            raise ValueError("out must have the shape of logits")
    batch = (n_drafted if n_drafted is not None else gamma).numel()
    if n_drafted is not None and n_rows != batch:
        raise ValueError("draft rows: one row of logits per sequence")
    cp = cs = mp = ms = width = n_d_rows = 0
    if token_counts is not None:
        cp, cs, c_rows, c_cols = _rows_on(token_counts, torch.int16, "token_counts", index)
        if c_rows != batch or c_cols < vocab:
            raise ValueError("token_counts must have a row of at least vocab entries per sequence")
    if bias_tokens is not None:
        width = bias_tokens.shape[-1]
        if bias_tokens.dim() != 2 or bias_values is None or bias_values.shape != bias_tokens.shape:
            raise ValueError("bias_tokens and bias_values must be [batch, entries]")
    if mask is not None:
        mp, ms, m_rows, m_cols = _rows_on(mask, i32, "mask", index)
        if m_rows != n_rows or 32 * m_cols < vocab:
            raise ValueError("mask must have a row of at least vocab bits per row of logits")
    if draft_tokens is not None:
        n_d_rows = draft_tokens.numel()
    return (lp, op, ls, os_, n_rows, vocab, 1 if bf16 else 0, batch, gamma_max, _on(gamma, i32, "gamma", index, batch),
            _on(cu_q, i32, "cu_q", index, batch + 1), _on(cu_d, i32, "cu_d", index, batch + 1),
            _on(n_drafted, i32, "n_drafted", index), _on(active, i32, "active", index, batch),
            _on(draft_tokens, i32, "draft_tokens", index), n_d_rows, cp, cs, _on(repetition, f32, "repetition", index, batch),
            _on(frequency, f32, "frequency", index, batch), _on(presence, f32, "presence", index, batch),
            _on(bias_tokens, i32, "bias_tokens", index, batch * width),
            _on(bias_values, f32, "bias_values", index), _on(n_bias, i32, "n_bias", index, batch), width, mp, ms,
            _on(device_status, i32, "device_status", index))


def logits_adjust_params(*args, **kwargs) -> LogitsAdjustParams:
    """Arguments of spec_logits_adjust (without stream)."""
    return LogitsAdjustParams(*_logits_adjust_args(torch.cuda.current_device(), *args, **kwargs))


_pack_logits_adjust = _packer(LogitsAdjustParams)


def spec_logits_adjust(logits, out, gamma, cu_q, cu_d, gamma_max, draft_tokens=None, token_counts=None, repetition=None,
                       frequency=None, presence=None, bias_tokens=None, bias_values=None, n_bias=None, mask=None,
                       n_drafted=None, active=None, device_status=None, stream=None):
    """Penalties, biases and grammar masks on the target rows of every block, or, with n_drafted, on one draft row per
    sequence (asynchronous).  out may be logits itself.  mask: int32 [n_rows, words], a set bit allows its token."""
    index, raw = _launch_at(stream, logits, "logits")
    p = _pack_logits_adjust(*_logits_adjust_args(index, logits, out, gamma, cu_q, cu_d, gamma_max, draft_tokens, token_counts,
                                                 repetition, frequency, presence, bias_tokens, bias_values, n_bias, mask,
                                                 n_drafted, active, device_status))
    _check("spec_logits_adjust", load().spec_logits_adjust(p, raw))


def _token_counts_args(index, token_counts, vocab, tokens=None, cu_tokens=None, max_tokens=None, reset=None, prompt=False,
                       device_status=None):
    i32 = torch.int32
    cp, cs, batch, cols = _rows_on(token_counts, torch.int16, "token_counts", index)
    if cols < vocab:
        raise ValueError("token_counts must have at least vocab entries per row")
    tp = ts = n_tokens = 0
    if tokens is not None:
        if cu_tokens is None:
            tp, ts, t_rows, t_cols = _rows_on(tokens, i32, "tokens", index)
            max_tokens = t_cols if max_tokens is None else max_tokens
            if t_rows != batch or max_tokens > t_cols:
                raise ValueError("tokens must have one row per sequence, of at least max_tokens columns")
        else:
            tp, n_tokens = _on(tokens, i32, "tokens", index), tokens.numel()
            max_tokens = n_tokens if max_tokens is None else max_tokens
    return (cp, cs, vocab, batch, tp, ts, _on(cu_tokens, i32, "cu_tokens", index, batch + 1), n_tokens, max_tokens or 0,
            _on(reset, i32, "reset", index, batch), 1 if prompt else 0, _on(device_status, i32, "device_status", index))


def token_counts_params(*args, **kwargs) -> TokenCountsParams:
    """Arguments of spec_token_counts_update (without stream)."""
    return TokenCountsParams(*_token_counts_args(torch.cuda.current_device(), *args, **kwargs))


_pack_token_counts = _packer(TokenCountsParams)


def spec_token_counts_update(token_counts, vocab, tokens=None, cu_tokens=None, max_tokens=None, reset=None, prompt=False,
                             device_status=None, stream=None):
    """Count generated tokens (or mark prompt tokens) in the int16 state behind the penalties, after clearing the rows
    of newly admitted sequences (asynchronous).  tokens: [batch, columns] padded with -1, or packed with cu_tokens.
    max_tokens: the most that a sequence has; it sizes the grid, and with cu_tokens it should be given: where it is
    left out it is the number of all tokens, for each sequence (128 prompts of 8192 marked without reset: 404 us, not 9)."""
    index, raw = _launch_at(stream, token_counts, "token_counts")
    p = _pack_token_counts(*_token_counts_args(index, token_counts, vocab, tokens, cu_tokens, max_tokens, reset, prompt,
                                               device_status))
    _check("spec_token_counts_update", load().spec_token_counts_update(p, raw))


# --------------------------------------------------------------------------- long contexts: pages that matter, shared prefixes
def _pool_on(pool, index):
    """Handle of a registered pool whose memory is on the current device."""
    if pool.handle is None:
        raise ValueError("the pool has been released")
    if pool.k_pool.get_device() != index or pool.v_pool.get_device() != index:
        raise ValueError(f"the pool's memory is not on the current device (cuda:{index})")
    return pool.handle.value


def _workspace_on(workspace, index):
    if workspace is None or workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on the current device (cuda:{index})")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _table_on(block_table, batch, index):
    if block_table.dim() != 2 or block_table.shape[0] != batch:
        raise ValueError("block_table must have one row per sequence")
    return _on(block_table, torch.int32, "block_table", index), block_table.shape[1]


def _bounds_on(bounds, scales, shape, index):
    if tuple(bounds.shape) != shape:
        raise ValueError(f"bounds must be {list(shape)}, got {list(bounds.shape)}")
    return _on(bounds, torch.int8, "bounds", index), _on(scales, torch.float32, "scales", index, shape[0] * shape[1])


def _page_bounds_args(index, pool, bounds, scales, block_table, seq_len, gamma=None, first=None, max_new=1, device_status=None):
    i32, batch = torch.int32, seq_len.numel()
    bp, sp = _bounds_on(bounds, scales, (pool.n_pages, pool.hkv, 2, pool.head_dim), index)
    tp, ts = _table_on(block_table, batch, index)
    return (_pool_on(pool, index), bp, sp, tp, ts, _on(seq_len, i32, "seq_len", index), _on(gamma, i32, "gamma", index, batch),
            _on(first, i32, "first", index, batch), batch, max_new, _on(device_status, i32, "device_status", index))


def page_bounds_params(*args, **kwargs) -> PageBoundsParams:
    """Arguments of spec_page_bounds_update (without stream)."""
    return PageBoundsParams(*_page_bounds_args(torch.cuda.current_device(), *args, **kwargs))


_pack_page_bounds = _packer(PageBoundsParams)


def spec_page_bounds_update(pool, bounds, scales, block_table, seq_len, gamma=None, first=None, max_new=1, device_status=None,
                            stream=None):
    """Bounds of the keys of every page that holds a new position, in 8 bits with a scale per page and kv head
    (asynchronous).  New are the gamma+1 positions of the draft block, or those from first on; max_new bounds their number."""
    index, raw = _launch_at(stream, seq_len, "seq_len")
    p = _pack_page_bounds(*_page_bounds_args(index, pool, bounds, scales, block_table, seq_len, gamma, first, max_new, device_status))
    _check("spec_page_bounds_update", load().spec_page_bounds_update(p, raw))


def spec_page_select_workspace_bytes(batch, gamma_max, hkv, max_seq_len) -> int:
    return int(load().spec_page_select_workspace_bytes(batch, gamma_max, hkv, max_seq_len))


def _lists_on(page_list, row_mask, n_list, batch, hkv, index):
    if page_list.dim() != 3 or page_list.shape[0] != batch or page_list.shape[1] != hkv or row_mask.shape != page_list.shape:
        raise ValueError("page_list and row_mask must be [batch, hkv, entries]")
    return (_on(page_list, torch.int32, "page_list", index), _on(row_mask, torch.int64, "row_mask", index),
            _on(n_list, torch.int32, "n_list", index, batch * hkv), page_list.shape[2])


def _page_select_args(index, q, bounds, scales, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len, n_select, n_first, n_last,
                      page_list, row_mask, n_list, device_status=None):
    i32, batch = torch.int32, seq_len.numel()
    if q.dim() != 3 or bounds.dim() != 4:
        raise ValueError("q must be [n_rows, hq, head_dim] and bounds [n_pages, hkv, 2, head_dim]")
    _, hq, head_dim = q.shape
    n_pages, hkv = bounds.shape[:2]
    bp, sp = _bounds_on(bounds, scales, (n_pages, hkv, 2, head_dim), index)
    tp, ts = _table_on(block_table, batch, index)
    lp, mp, np_, width = _lists_on(page_list, row_mask, n_list, batch, hkv, index)
    return (_on(q, torch.bfloat16, "q", index), bp, sp, n_pages, tp, ts, _on(seq_len, i32, "seq_len", index),
            _on(gamma, i32, "gamma", index, batch), _on(cu_q, i32, "cu_q", index, batch + 1), batch, gamma_max, hq, hkv, head_dim,
            max_seq_len, n_select, n_first, n_last, lp, mp, np_, width, _on(device_status, i32, "device_status", index))


def page_select_params(*args, **kwargs) -> PageSelectParams:
    """Arguments of spec_page_select (without workspace and stream)."""
    return PageSelectParams(*_page_select_args(torch.cuda.current_device(), *args, **kwargs))


_pack_page_select = _packer(PageSelectParams)


def spec_page_select(q, bounds, scales, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len, n_select, n_first, n_last,
                     page_list, row_mask, n_list, workspace, device_status=None, stream=None):
    """The n_select pages that each row of a block reads, by a score on the pages' bounds, as one list per sequence and kv
    head with a mask of the rows that read each page (asynchronous).  row_mask: int64, bit i for row i."""
    index, raw = _launch_at(stream, q, "q")
    p = _pack_page_select(*_page_select_args(index, q, bounds, scales, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len,
                                             n_select, n_first, n_last, page_list, row_mask, n_list, device_status))
    _check("spec_page_select", load().spec_page_select(p, *_workspace_on(workspace, index), raw))


def _attn_args(index, q, o, pool, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len, sm_scale=None, lse=None,
               device_status=None):
    i32, batch = torch.int32, seq_len.numel()
    if q.dim() != 3 or o.shape != q.shape:
        raise ValueError("q and o must be [n_rows, hq, head_dim]")
    n_rows, hq, head_dim = q.shape
    tp, ts = _table_on(block_table, batch, index)
    return (_on(q, torch.bfloat16, "q", index), _on(o, torch.bfloat16, "o", index), _on(lse, torch.float32, "lse", index, n_rows * hq),
            _pool_on(pool, index), tp, ts, _on(seq_len, i32, "seq_len", index), _on(gamma, i32, "gamma", index, batch),
            _on(cu_q, i32, "cu_q", index, batch + 1), batch, gamma_max, hq, pool.hkv, head_dim, max_seq_len,
            sm_scale if sm_scale is not None else head_dim ** -0.5, _on(device_status, i32, "device_status", index))


def spec_verify_attn_pages_workspace_bytes(batch, gamma_max, hq, hkv, head_dim) -> int:
    return int(load().spec_verify_attn_pages_workspace_bytes(batch, gamma_max, hq, hkv, head_dim))


_pack_attn_pages = _packer(AttnPagesParams)


def spec_verify_attn_pages(q, o, pool, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len, page_list, row_mask, n_list,
                           workspace, sm_scale=None, lse=None, device_status=None, stream=None):
    """Attention of the draft block over the listed pages, each row over those whose mask names it (asynchronous)."""
    index, raw = _launch_at(stream, q, "q")
    lists = _lists_on(page_list, row_mask, n_list, seq_len.numel(), pool.hkv, index)
    p = _pack_attn_pages(*_attn_args(index, q, o, pool, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len, sm_scale, lse,
                                     device_status), *lists)
    _check("spec_verify_attn_pages", load().spec_verify_attn_pages(p, *_workspace_on(workspace, index), raw))


def spec_verify_attn_prefix_workspace_bytes(batch, gamma_max, hq, hkv, head_dim, n_groups) -> int:
    return int(load().spec_verify_attn_prefix_workspace_bytes(batch, gamma_max, hq, hkv, head_dim, n_groups))


_pack_attn_prefix = _packer(AttnPrefixParams)


def spec_verify_attn_prefix(q, o, pool, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len, group, prefix_len, workspace,
                            sm_scale=None, lse=None, device_status=None, stream=None):
    """Attention of the draft block against the paged KV cache of a batch in which the sequences of a group share the pages
    of their first prefix_len[group] tokens: those are read once per group (asynchronous).  group[b] = -1: none."""
    index, raw = _launch_at(stream, q, "q")
    p = _pack_attn_prefix(*_attn_args(index, q, o, pool, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len, sm_scale, lse,
                                      device_status),
                          _on(group, torch.int32, "group", index, seq_len.numel()), _on(prefix_len, torch.int32, "prefix_len", index),
                          prefix_len.numel())
    _check("spec_verify_attn_prefix", load().spec_verify_attn_prefix(p, *_workspace_on(workspace, index), raw))


# --------------------------------------------------------------------------- accept / resample
def spec_accept_sample_workspace_bytes(batch, gamma_max, vocab) -> int:
    return int(load().spec_accept_sample_workspace_bytes(batch, gamma_max, vocab))


def accept_params(target_logits, draft_logits, draft_tokens, u_accept, u_sample, temperature, gamma,
                  cu_q, cu_d, gamma_max, n_accepted, out_tokens, ratio=None, logZ_p=None,
                  logZ_q=None, flag_count=None, device_status=None,
                  temperature_per_seq=None) -> AcceptParams:
    p = AcceptParams()
    ldt = target_logits.dtype if target_logits.dtype == torch.bfloat16 else torch.float32     # float32 or bf16 logits
    p.logits_bf16 = int(ldt == torch.bfloat16)
    p.target_logits = _dev(target_logits, ldt, "target_logits")
    p.draft_logits = _dev(draft_logits, ldt, "draft_logits", True)
    p.row_stride = target_logits.stride(0)
    p.vocab = target_logits.shape[-1]
    p.draft_tokens = _dev(draft_tokens, torch.int32, "draft_tokens", True)
    p.u_accept = _dev(u_accept, torch.float32, "u_accept", True)
    p.u_sample = _dev(u_sample, torch.float32, "u_sample", True)
    p.temperature = float(temperature)
    p.temperature_per_seq = _dev(temperature_per_seq, torch.float32, "temperature_per_seq", True)
    p.gamma = _dev(gamma, torch.int32, "gamma")
    p.cu_q = _dev(cu_q, torch.int32, "cu_q")
    p.cu_d = _dev(cu_d, torch.int32, "cu_d")
    p.batch = gamma.shape[0]
    p.gamma_max = gamma_max
    p.n_accepted = _dev(n_accepted, torch.int32, "n_accepted")
    p.out_tokens = _dev(out_tokens, torch.int32, "out_tokens")
    p.ratio = _dev(ratio, torch.float64, "ratio", True)
    p.logZ_p = _dev(logZ_p, torch.float64, "logZ_p", True)
    p.logZ_q = _dev(logZ_q, torch.float64, "logZ_q", True)
    p.flag_count = _dev(flag_count, torch.int32, "flag_count", True)
    p.device_status = _dev(device_status, torch.int32, "device_status", True)
    return p


def spec_accept_sample(target_logits, draft_logits, draft_tokens, u_accept, u_sample, temperature,
                       gamma, cu_q, cu_d, gamma_max, n_accepted, out_tokens, workspace, ratio=None,
                       logZ_p=None, logZ_q=None, flag_count=None, device_status=None,
                       temperature_per_seq=None, stream=None):
    """Accept / reject the drafts and draw the next token (asynchronous)."""
    p = accept_params(target_logits, draft_logits, draft_tokens, u_accept, u_sample, temperature,
                      gamma, cu_q, cu_d, gamma_max, n_accepted, out_tokens, ratio, logZ_p, logZ_q,
                      flag_count, device_status, temperature_per_seq)
    _check("spec_accept_sample",
           load().spec_accept_sample(C.byref(p), workspace.data_ptr(), _nbytes(workspace),
                                     _stream(stream)))


SV_ACCEPT_STATIC_SCRATCH_BYTES = 8 << 20


def spec_accept_sample_static(target_logits, draft_logits, draft_tokens, u_accept, u_sample, temperature,
                              gamma, cu_q, cu_d, gamma_max, n_accepted, out_tokens, ratio=None,
                              logZ_p=None, logZ_q=None, flag_count=None, device_status=None,
                              temperature_per_seq=None, stream=None):
    """spec_accept_sample for callers that cannot hand over scratch memory (no workspace
    argument; the library's built-in array is used).  Problems beyond that array's size raise
    SpecVerifyError with SV_EWORKSPACE.  Calls on one device must not overlap on the GPU."""
    p = accept_params(target_logits, draft_logits, draft_tokens, u_accept, u_sample, temperature,
                      gamma, cu_q, cu_d, gamma_max, n_accepted, out_tokens, ratio, logZ_p, logZ_q,
                      flag_count, device_status, temperature_per_seq)
    _check("spec_accept_sample_static", load().spec_accept_sample_static(C.byref(p), _stream(stream)))


# --------------------------------------------------------------------------- GammaTune
@dataclass
class GammaConfig:
    eta: float = 0.5
    delta: float = 2.0
    gamma_min: int = 1
    gamma_max: int = 8
    mode: int = SV_GT_PROPOSED
    padded_rows: bool = False


def gamma_params(n_accepted, gamma_bar, gamma, seq_len, cu_q, cu_d, config: GammaConfig,
                 trajectory=None, accepted_log=None, step=0, device_status=None, n_drafted=None) -> GammaParams:
    p = GammaParams()
    p.n_accepted = _dev(n_accepted, torch.int32, "n_accepted", True)
    p.gamma_bar = _dev(gamma_bar, torch.float64, "gamma_bar")
    p.gamma = _dev(gamma, torch.int32, "gamma")
    p.seq_len = _dev(seq_len, torch.int32, "seq_len", True)
    p.cu_q = _dev(cu_q, torch.int32, "cu_q")
    p.cu_d = _dev(cu_d, torch.int32, "cu_d")
    p.batch = gamma.shape[0]
    p.config = GammaConfigC(config.eta, config.delta, config.gamma_min, config.gamma_max,
                            config.mode, int(config.padded_rows))
    p.trajectory = _dev(trajectory, torch.int32, "trajectory", True)
    p.accepted_log = _dev(accepted_log, torch.int32, "accepted_log", True)
    p.step = step
    p.device_status = _dev(device_status, torch.int32, "device_status", True)
    p.n_drafted = _dev(n_drafted, torch.int32, "n_drafted", True)
    return p


def gamma_tune_update(n_accepted, gamma_bar, gamma, seq_len, cu_q, cu_d, config: GammaConfig,
                      trajectory=None, accepted_log=None, step=0, device_status=None, stream=None,
                      n_drafted=None):
    """One GammaTune update of every sequence's (gamma_bar, gamma) on the device (asynchronous)."""
    p = gamma_params(n_accepted, gamma_bar, gamma, seq_len, cu_q, cu_d, config, trajectory,
                     accepted_log, step, device_status, n_drafted)
    _check("gamma_tune_update", load().gamma_tune_update(C.byref(p), _stream(stream)))


# --------------------------------------------------------------------------- GammaTune+ early stop
def spec_draft_stop_workspace_bytes(batch, gamma_max, vocab) -> int:
    return int(load().spec_draft_stop_workspace_bytes(batch, gamma_max, vocab))


def draft_stop_params(draft_logits, temperature, tau, gamma, cu_d, gamma_max, n_drafted, top_prob=None,
                      device_status=None, temperature_per_seq=None) -> DraftStopParams:
    p = DraftStopParams()
    ldt = draft_logits.dtype if draft_logits.dtype == torch.bfloat16 else torch.float32       # float32 or bf16 logits
    p.logits_bf16 = int(ldt == torch.bfloat16)
    p.draft_logits = _dev(draft_logits, ldt, "draft_logits")
    p.row_stride = draft_logits.stride(0)
    p.vocab = draft_logits.shape[-1]
    p.temperature = float(temperature)
    p.temperature_per_seq = _dev(temperature_per_seq, torch.float32, "temperature_per_seq", True)
    p.tau = float(tau)
    p.gamma = _dev(gamma, torch.int32, "gamma")
    p.cu_d = _dev(cu_d, torch.int32, "cu_d")
    p.batch = gamma.shape[0]
    p.gamma_max = gamma_max
    p.n_drafted = _dev(n_drafted, torch.int32, "n_drafted")
    p.top_prob = _dev(top_prob, torch.float64, "top_prob", True)
    p.device_status = _dev(device_status, torch.int32, "device_status", True)
    return p


def spec_draft_stop(draft_logits, temperature, tau, gamma, cu_d, gamma_max, n_drafted, workspace,
                    top_prob=None, device_status=None, temperature_per_seq=None, stream=None):
    """GammaTune+ early stop of drafting: n_drafted per sequence (asynchronous)."""
    p = draft_stop_params(draft_logits, temperature, tau, gamma, cu_d, gamma_max, n_drafted, top_prob,
                          device_status, temperature_per_seq)
    _check("spec_draft_stop",
           load().spec_draft_stop(C.byref(p), workspace.data_ptr(), _nbytes(workspace), _stream(stream)))


# --------------------------------------------------------------------------- GammaTune+ drafting step
def spec_draft_step_workspace_bytes(batch, vocab) -> int:
    return int(load().spec_draft_step_workspace_bytes(batch, vocab))


def draft_step_params(draft_logits, temperature, tau, u_sample, gamma, cu_d, gamma_max, n_drafted, active,
                      draft_tokens, top_prob=None, device_status=None, temperature_per_seq=None) -> DraftStepParams:
    p = DraftStepParams()
    ldt = draft_logits.dtype if draft_logits.dtype == torch.bfloat16 else torch.float32       # float32 or bf16 logits
    p.logits_bf16 = int(ldt == torch.bfloat16)
    p.draft_logits = _dev_rows(draft_logits, ldt, "draft_logits")     # e.g. position i of every block
    p.row_stride = draft_logits.stride(0)
    p.vocab = draft_logits.shape[-1]
    p.temperature = float(temperature)
    p.temperature_per_seq = _dev(temperature_per_seq, torch.float32, "temperature_per_seq", True)
    p.tau = float(tau)
    p.u_sample = _dev(u_sample, torch.float32, "u_sample", True)
    p.gamma = _dev(gamma, torch.int32, "gamma")
    p.cu_d = _dev(cu_d, torch.int32, "cu_d")
    p.batch = gamma.shape[0]
    p.gamma_max = gamma_max
    p.n_drafted = _dev(n_drafted, torch.int32, "n_drafted")
    p.active = _dev(active, torch.int32, "active")
    p.draft_tokens = _dev(draft_tokens, torch.int32, "draft_tokens")
    p.top_prob = _dev(top_prob, torch.float64, "top_prob", True)
    p.device_status = _dev(device_status, torch.int32, "device_status", True)
    return p


def spec_draft_step(draft_logits, temperature, tau, u_sample, gamma, cu_d, gamma_max, n_drafted, active,
                    draft_tokens, workspace, top_prob=None, device_status=None, temperature_per_seq=None,
                    stream=None):
    """One drafting step with the confidence stop (asynchronous): token, top probability, n_drafted, active."""
    p = draft_step_params(draft_logits, temperature, tau, u_sample, gamma, cu_d, gamma_max, n_drafted, active,
                          draft_tokens, top_prob, device_status, temperature_per_seq)
    _check("spec_draft_step",
           load().spec_draft_step(C.byref(p), workspace.data_ptr(), _nbytes(workspace), _stream(stream)))


def gamma_tune_init(gamma_bar, gamma, cu_q, cu_d, config: GammaConfig, gamma0: int, stream=None):
    p = gamma_params(None, gamma_bar, gamma, None, cu_q, cu_d, config)
    _check("gamma_tune_init", load().gamma_tune_init(C.byref(p), int(gamma0), _stream(stream)))


# --------------------------------------------------------------------------- step from host buffers
def spec_verify_step_host(io: StepHostIO, attn: AttnParams, attn_workspace, accept: AcceptParams,
                          accept_workspace, gamma: GammaParams, stream=None):
    """One whole verify step whose per-step inputs start in (pinned) host memory."""
    _check("spec_verify_step_host",
           load().spec_verify_step_host(
               C.byref(io), C.byref(attn), attn_workspace.data_ptr(), _nbytes(attn_workspace),
               C.byref(accept), accept_workspace.data_ptr(), _nbytes(accept_workspace),
               C.byref(gamma), _stream(stream)))


def step_host_io(q_host, target_logits_host, draft_logits_host, draft_tokens_host, u_accept_host,
                 u_sample_host, n_q_rows, n_d_rows, n_accepted_host, out_tokens_host,
                 gamma_next_host, o_host=None) -> StepHostIO:
    io = StepHostIO()
    io.q_host = _host(q_host, torch.bfloat16, "q_host")
    io.target_logits_host = _host(target_logits_host, torch.float32, "target_logits_host")
    io.draft_logits_host = _host(draft_logits_host, torch.float32, "draft_logits_host", True)
    io.draft_tokens_host = _host(draft_tokens_host, torch.int32, "draft_tokens_host", True)
    io.u_accept_host = _host(u_accept_host, torch.float32, "u_accept_host", True)
    io.u_sample_host = _host(u_sample_host, torch.float32, "u_sample_host", True)
    io.n_q_rows, io.n_d_rows = int(n_q_rows), int(n_d_rows)
    io.n_accepted_host = _host(n_accepted_host, torch.int32, "n_accepted_host")
    io.out_tokens_host = _host(out_tokens_host, torch.int32, "out_tokens_host")
    io.gamma_next_host = _host(gamma_next_host, torch.int32, "gamma_next_host")
    io.o_host = _host(o_host, torch.bfloat16, "o_host", True)
    return io


# --------------------------------------------------------------------------- all layers of a step
def attn_layers_params(qs, os_, pools, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len, k_new=None,
                       v_new=None, lses=None, sm_scale=None, device_status=None) -> AttnLayersParams:
    """Arguments of spec_verify_attn_layers: lists with one entry per layer, the rest shared.  The returned
    struct keeps the pointer arrays alive."""
    n = len(pools)
    if not (len(qs) == n and len(os_) == n):
        raise ValueError("one q, o and pool per layer")
    p = AttnLayersParams()
    p.n_layers = n
    p.shared = attn_params(qs[0], os_[0], pools[0], block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len,
                           sm_scale, None, device_status)

    def arr(ptrs):
        a = (C.c_void_p * n)(*ptrs)
        return a

    p._keep = [arr([pl.handle.value for pl in pools]), arr([_dev(t, torch.bfloat16, "q") for t in qs]),
               arr([_dev(t, torch.bfloat16, "o") for t in os_])]
    p.pools, p.q, p.o = (C.cast(a, C.POINTER(C.c_void_p)) for a in p._keep)
    if lses is not None:
        a = arr([_dev(t, torch.float32, "lse") for t in lses])
        p._keep.append(a)
        p.lse = C.cast(a, C.POINTER(C.c_void_p))
    if k_new is not None:
        ak = arr([_dev(t, torch.bfloat16, "k_new") for t in k_new])
        av = arr([_dev(t, torch.bfloat16, "v_new") for t in v_new])
        p._keep += [ak, av]
        p.k_new, p.v_new = C.cast(ak, C.POINTER(C.c_void_p)), C.cast(av, C.POINTER(C.c_void_p))
    return p


def spec_verify_attn_layers(qs, os_, pools, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len, workspace,
                            k_new=None, v_new=None, lses=None, sm_scale=None, device_status=None, stream=None):
    """Cache append (one launch for all layers) and verify attention of every layer's cache (asynchronous)."""
    p = attn_layers_params(qs, os_, pools, block_table, seq_len, gamma, cu_q, gamma_max, max_seq_len, k_new, v_new,
                           lses, sm_scale, device_status)
    _check("spec_verify_attn_layers",
           load().spec_verify_attn_layers(C.byref(p), workspace.data_ptr(), _nbytes(workspace), _stream(stream)))


# --------------------------------------------------------------------------- self-test
def sv_selftest_wait_expiry(device_status, device_result, limit_cycles, stream=None):
    """One thread block waits, with a budget of `limit_cycles`, on a barrier nothing arrives at."""
    _check("sv_selftest_wait_expiry",
           load().sv_selftest_wait_expiry(_dev(device_status, torch.int32, "device_status"),
                                          _dev(device_result, torch.int32, "device_result"),
                                          int(limit_cycles), _stream(stream)))
