"""ctypes binding of librespec.so: argument marshalling only.

Same names as the C boundary (``include/respec.h``).  Torch tensors are used for device
memory and the current stream; every step of the verify path runs in the HIP kernels.
There is no CPU fallback: a missing library or a non-CUDA tensor is an error.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

from . import build as _build

RESPEC_F32 = 0
RESPEC_BF16 = 1
RESPEC_E4M3 = 2

_lib = None


class RespecError(RuntimeError):
    def __init__(self, status: int, text: str, detail: str):
        super().__init__(f"librespec status {status} ({text}): {detail}")
        self.status = status


def library_path() -> str:
    """Path of librespec.so; RESPEC_LIBRARY_PATH points at another build of it (experiments)."""
    return os.environ.get("RESPEC_LIBRARY_PATH") or _build.LIB_PATH


def load():
    """Load librespec.so (building it first only if it has never been built)."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        _build.build()
    if not os.path.exists(path):
        raise RuntimeError(f"librespec.so not found at {path}; run python -m paper_2510_26475_amd.build")
    lib = ctypes.CDLL(path)
    c = ctypes
    lib.respec_status_string.restype = c.c_char_p
    lib.respec_status_string.argtypes = [c.c_int]
    lib.respec_last_error.restype = c.c_char_p
    lib.respec_last_error.argtypes = []
    lib.respec_version.restype = c.c_int
    lib.respec_version.argtypes = []
    lib.respec_verify_attention_workspace_bytes.restype = c.c_size_t
    lib.respec_verify_attention_workspace_bytes.argtypes = [
        c.c_int32, c.c_int32, c.c_int64, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32,
        c.c_int]
    lib.respec_verify_attention.restype = c.c_int
    lib.respec_verify_attention.argtypes = [
        c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
        c.c_int32, c.c_int32, c.c_int64, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32,
        c.c_float, c.c_int, c.c_void_p, c.c_size_t, c.c_void_p]
    lib.respec_verify_attention_tree.restype = c.c_int
    lib.respec_verify_attention_tree.argtypes = [
        c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
        c.c_int32, c.c_int32, c.c_int64, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32,
        c.c_float, c.c_int, c.c_void_p, c.c_size_t, c.c_void_p]
    lib.respec_verify_attention_next_layer.restype = c.c_int
    lib.respec_verify_attention_next_layer.argtypes = lib.respec_verify_attention_tree.argtypes
    lib.respec_static_scratch_bytes.restype = c.c_size_t
    lib.respec_static_scratch_bytes.argtypes = []
    lib.respec_static_scratch_init.restype = c.c_int
    lib.respec_static_scratch_init.argtypes = []
    lib.respec_verify_attention_static.restype = c.c_int
    lib.respec_verify_attention_static.argtypes = [
        c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
        c.c_int32, c.c_int32, c.c_int64, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32,
        c.c_float, c.c_int, c.c_void_p]
    lib.respec_reload_knobs.restype = None
    lib.respec_reload_knobs.argtypes = []
    lib.respec_profile_mark_main.restype = None
    lib.respec_profile_mark_main.argtypes = [c.c_void_p, c.c_void_p]
    lib.respec_rejection_sample_workspace_bytes.restype = c.c_size_t
    lib.respec_rejection_sample_workspace_bytes.argtypes = [c.c_int32, c.c_int32, c.c_int32, c.c_int]
    lib.respec_rejection_sample.restype = c.c_int
    lib.respec_rejection_sample.argtypes = [
        c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
        c.c_void_p, c.c_void_p, c.c_void_p,
        c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int64, c.c_int64,
        c.c_float, c.c_int, c.c_void_p, c.c_size_t, c.c_void_p]
    lib.respec_rejection_sample_per_seq.restype = c.c_int
    lib.respec_rejection_sample_per_seq.argtypes = [
        c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
        c.c_void_p, c.c_void_p, c.c_void_p,
        c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int64, c.c_int64, c.c_int, c.c_void_p]
    lib.respec_tree_rejection_sample.restype = c.c_int
    lib.respec_tree_rejection_sample.argtypes = [
        c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
        c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
        c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int64, c.c_int64,
        c.c_float, c.c_int, c.c_void_p]
    lib.respec_verify_attention_paged.restype = c.c_int
    lib.respec_verify_attention_paged.argtypes = [
        c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
        c.c_void_p, c.c_void_p,
        c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32,
        c.c_int32, c.c_float, c.c_int, c.c_void_p, c.c_size_t, c.c_void_p]
    lib.respec_verify_attention_paged_next_layer.restype = c.c_int
    lib.respec_verify_attention_paged_next_layer.argtypes = lib.respec_verify_attention_paged.argtypes
    lib.respec_commit_accepted_paged.restype = c.c_int
    lib.respec_commit_accepted_paged.argtypes = [
        c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_int32,
        c.c_void_p, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32, c.c_int32,
        c.c_int, c.c_void_p]
    lib.respec_kd_rows_workspace_bytes.restype = c.c_size_t
    lib.respec_kd_rows_workspace_bytes.argtypes = [c.c_int32, c.c_int32, c.c_int]
    lib.respec_kd_rows.restype = c.c_int
    lib.respec_kd_rows.argtypes = [
        c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
        c.c_int32, c.c_int32, c.c_int64, c.c_int64, c.c_int64, c.c_int, c.c_void_p, c.c_size_t, c.c_void_p]
    lib.respec_validate_batch_workspace_bytes.restype = c.c_size_t
    lib.respec_validate_batch_workspace_bytes.argtypes = [c.c_int32]
    lib.respec_validate_batch.restype = c.c_int
    lib.respec_validate_batch.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_int32, c.c_int32, c.c_int64,
                                          c.c_int32, c.c_int32, c.c_int32, c.c_void_p, c.c_size_t, c.c_void_p]
    lib.respec_solver_pick.restype = c.c_int
    lib.respec_solver_pick.argtypes = [c.c_void_p, c.c_int32, c.c_int32, c.c_double, c.c_double,
                                       c.POINTER(c.c_int32), c.POINTER(c.c_double), c.POINTER(c.c_double)]
    ptr, i32, i64, f32, size = c.c_void_p, c.c_int32, c.c_int64, c.c_float, c.c_size_t
    for name, result, args in (
            ("respec_prompt_attention_workspace_bytes", size, [i32, i32, i64] + [i32] * 5 + [c.c_int]),
            ("respec_prompt_attention", c.c_int,
             [ptr] * 7 + [i32, i32, i64] + [i32] * 5 + [i64] * 3 + [f32, c.c_int, ptr, size, ptr]),
            ("respec_prompt_attention_paged", c.c_int, [ptr] * 9 + [i32] * 10 + [i64, f32, c.c_int, ptr, size, ptr]),
            ("respec_append_paged", c.c_int, [ptr] * 8 + [i32] * 8 + [i64, c.c_int, ptr]),
            ("respec_pages_workspace_bytes", size, [i32, i32]),
            ("respec_pages_resize", c.c_int, [ptr] * 9 + [i32] * 4 + [ptr, size, ptr]),
            ("respec_pages_fork", c.c_int, [ptr] * 7 + [i32] * 3 + [ptr]),
            ("respec_pages_compact", c.c_int, [ptr] * 7 + [i32] * 3 + [ptr, size, ptr]),
            ("respec_pages_copy", c.c_int, [ptr] * 4 + [i32] * 5 + [c.c_int, ptr]),
            ("respec_norm_rope_append_paged", c.c_int, [ptr] * 16 + [i32] * 11 + [i64] * 4 + [f32, c.c_int, c.c_int, ptr]),
            ("respec_read_paged_quantised", c.c_int, [ptr] * 10 + [i32, i64] + [i32] * 6 + [c.c_int, ptr]),
            ("respec_commit_accepted_paged_quantised", c.c_int, [ptr] * 9 + [i32, ptr] + [i32] * 8 + [ptr]),
            ("respec_pages_copy_quantised", c.c_int, [ptr] * 6 + [i32] * 5 + [ptr]),
            ("respec_verify_attention_shared_workspace_bytes", size, [i32] * 8 + [c.c_int]),
            ("respec_verify_attention_shared", c.c_int, [ptr] * 14 + [i32] * 11 + [f32, c.c_int, c.c_int, ptr, size, ptr]),
            ("respec_verify_attention_shared_next_layer", c.c_int, [ptr] * 14 + [i32] * 11 + [f32, c.c_int, c.c_int, ptr, size, ptr]),
            ("respec_verify_attention_paged_quantised", c.c_int, [ptr] * 12 + [i32] * 10 + [f32, c.c_int, ptr, size, ptr]),
            ("respec_token_logprobs_workspace_bytes", size, [i32] * 3 + [c.c_int]),
            ("respec_token_logprobs", c.c_int, [ptr] * 8 + [i32, i32, i64, i32, f32, c.c_int, ptr, size, ptr]),
            ("respec_token_logprobs_grad", c.c_int, [ptr] * 8 + [i32, i32, i64, i64, f32, c.c_int, ptr])):
        entry = getattr(lib, name)
        entry.restype, entry.argtypes = result, args
    _lib = lib
    return lib


class ProfilePoint(ctypes.Structure):
    """respec_profile_point_t"""
    _fields_ = [("batch", ctypes.c_int32), ("k", ctypes.c_int32), ("step_us", ctypes.c_double),
                ("emitted_per_seq", ctypes.c_double)]


EXPORTED_SYMBOLS = [
    "respec_status_string", "respec_last_error", "respec_version",
    "respec_verify_attention_workspace_bytes", "respec_verify_attention", "respec_verify_attention_tree",
    "respec_verify_attention_next_layer", "respec_verify_attention_paged_next_layer",
    "respec_rejection_sample_workspace_bytes", "respec_rejection_sample", "respec_rejection_sample_per_seq",
    "respec_tree_rejection_sample", "respec_verify_attention_paged", "respec_commit_accepted_paged",
    "respec_kd_rows_workspace_bytes", "respec_kd_rows", "respec_solver_pick",
    "respec_validate_batch_workspace_bytes", "respec_validate_batch",
    "respec_profile_mark_main",
    "respec_static_scratch_bytes", "respec_static_scratch_init", "respec_verify_attention_static",
    "respec_reload_knobs",
    "respec_prompt_attention_workspace_bytes", "respec_prompt_attention", "respec_prompt_attention_paged", "respec_append_paged",
    "respec_pages_workspace_bytes", "respec_pages_resize", "respec_pages_fork", "respec_pages_compact", "respec_pages_copy",
    "respec_token_logprobs_workspace_bytes", "respec_token_logprobs", "respec_token_logprobs_grad",
    "respec_norm_rope_append_paged", "respec_read_paged_quantised", "respec_commit_accepted_paged_quantised", "respec_pages_copy_quantised",
    "respec_verify_attention_shared_workspace_bytes", "respec_verify_attention_shared", "respec_verify_attention_shared_next_layer",
    "respec_verify_attention_paged_quantised",
]


def _check(status: int):
    if status != 0:
        lib = load()
        raise RespecError(status, lib.respec_status_string(status).decode(),
                          lib.respec_last_error().decode())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return RESPEC_F32
    if t.dtype == torch.bfloat16:
        return RESPEC_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _dev_ptr(t: Optional[torch.Tensor], name: str):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU (got {t.device})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


# (A small step is bound by this module: its calls enqueue in about the time that its kernels take.  A
# stream object made for its handle takes 2.7 us of the 9 to 12 us that a call needs here, the handle
# alone 0.3: the fp32 step of 4 sequences 19.4 -> 14.9 us.  The function is not part of torch's public
# interface: without it a stream object is made.)
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream: Optional[torch.cuda.Stream]):
    if stream is not None:
        return stream.cuda_stream
    if _current_raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _current_raw_stream(torch.cuda.current_device())


def respec_reload_knobs():
    """Have the library read its RESPEC_* environment knobs again (tests and sweeps)."""
    load().respec_reload_knobs()


def respec_version() -> int:
    return int(load().respec_version())


def respec_verify_attention_workspace_bytes(B, total_q, total_kv, max_q_per_seq, max_kv_len, Hq,
                                            Hkv, D, dt) -> int:
    return int(load().respec_verify_attention_workspace_bytes(
        B, total_q, total_kv, max_q_per_seq, max_kv_len, Hq, Hkv, D, dt))


def respec_verify_attention(q, k_cache, v_cache, q_indptr, kv_indptr, out, lse, max_q_per_seq,
                            max_kv_len, sm_scale, workspace, stream=None):
    """q/out [total_q,Hq,D], k_cache/v_cache [total_kv,Hkv,D], q_indptr int32, kv_indptr int64."""
    lib = load()
    total_q, Hq, D = q.shape
    total_kv, Hkv, _ = k_cache.shape
    B = q_indptr.numel() - 1
    if q_indptr.dtype != torch.int32 or kv_indptr.dtype != torch.int64:
        raise TypeError("q_indptr must be int32 and kv_indptr int64")
    if lse is not None and lse.dtype != torch.float32:
        raise TypeError("lse must be float32")
    if out.dtype != q.dtype or k_cache.dtype != q.dtype or v_cache.dtype != q.dtype:
        raise TypeError("q, k_cache, v_cache and out must share one dtype")
    ws_ptr = _dev_ptr(workspace, "workspace") if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib.respec_verify_attention(
        _dev_ptr(q, "q"), _dev_ptr(k_cache, "k_cache"), _dev_ptr(v_cache, "v_cache"),
        _dev_ptr(q_indptr, "q_indptr"), _dev_ptr(kv_indptr, "kv_indptr"), _dev_ptr(out, "out"),
        _dev_ptr(lse, "lse"), B, total_q, total_kv, max_q_per_seq, max_kv_len, Hq, Hkv, D,
        float(sm_scale), _dtype_code(q), ws_ptr, ws_bytes, _stream_ptr(stream)))


def respec_static_scratch_bytes() -> int:
    return int(load().respec_static_scratch_bytes())


def respec_static_scratch_init():
    _check(load().respec_static_scratch_init())


def respec_verify_attention_static(q, k_cache, v_cache, q_indptr, kv_indptr, out, lse, max_q_per_seq,
                                   max_kv_len, sm_scale, stream=None):
    """respec_verify_attention without a workspace: the scratch is the library's built-in buffer."""
    lib = load()
    total_q, Hq, D = q.shape
    total_kv, Hkv, _ = k_cache.shape
    B = q_indptr.numel() - 1
    if q_indptr.dtype != torch.int32 or kv_indptr.dtype != torch.int64:
        raise TypeError("q_indptr must be int32 and kv_indptr int64")
    if lse is not None and lse.dtype != torch.float32:
        raise TypeError("lse must be float32")
    if out.dtype != q.dtype or k_cache.dtype != q.dtype or v_cache.dtype != q.dtype:
        raise TypeError("q, k_cache, v_cache and out must share one dtype")
    _check(lib.respec_verify_attention_static(
        _dev_ptr(q, "q"), _dev_ptr(k_cache, "k_cache"), _dev_ptr(v_cache, "v_cache"),
        _dev_ptr(q_indptr, "q_indptr"), _dev_ptr(kv_indptr, "kv_indptr"), _dev_ptr(out, "out"),
        _dev_ptr(lse, "lse"), B, total_q, total_kv, max_q_per_seq, max_kv_len, Hq, Hkv, D,
        float(sm_scale), _dtype_code(q), _stream_ptr(stream)))


def respec_verify_attention_next_layer(q, k_cache, v_cache, q_indptr, kv_indptr, out, lse, max_q_per_seq,
                                       max_kv_len, sm_scale, workspace, tree_mask=None, stream=None):
    """Another layer of the same forward: same index arrays and sizes as the previous call on this
    workspace, other q / caches / out.  Reuses the set-up the workspace holds."""
    lib = load()
    total_q, Hq, D = q.shape
    total_kv, Hkv, _ = k_cache.shape
    B = q_indptr.numel() - 1
    if q_indptr.dtype != torch.int32 or kv_indptr.dtype != torch.int64:
        raise TypeError("q_indptr must be int32 and kv_indptr int64")
    if tree_mask is not None and (tree_mask.element_size() != 8 or tree_mask.numel() != total_q):
        raise TypeError("tree_mask must hold one 64-bit word per query row")
    if lse is not None and lse.dtype != torch.float32:
        raise TypeError("lse must be float32")
    if out.dtype != q.dtype or k_cache.dtype != q.dtype or v_cache.dtype != q.dtype:
        raise TypeError("q, k_cache, v_cache and out must share one dtype")
    ws_ptr = _dev_ptr(workspace, "workspace") if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib.respec_verify_attention_next_layer(
        _dev_ptr(q, "q"), _dev_ptr(k_cache, "k_cache"), _dev_ptr(v_cache, "v_cache"),
        _dev_ptr(q_indptr, "q_indptr"), _dev_ptr(kv_indptr, "kv_indptr"), _dev_ptr(tree_mask, "tree_mask"),
        _dev_ptr(out, "out"), _dev_ptr(lse, "lse"), B, total_q, total_kv, max_q_per_seq, max_kv_len, Hq, Hkv, D,
        float(sm_scale), _dtype_code(q), ws_ptr, ws_bytes, _stream_ptr(stream)))


def respec_verify_attention_tree(q, k_cache, v_cache, q_indptr, kv_indptr, tree_mask, out, lse,
                                 max_q_per_seq, max_kv_len, sm_scale, workspace, stream=None):
    """As respec_verify_attention; tree_mask [total_q] int64 (or uint64) holding the 64 mask bits."""
    lib = load()
    total_q, Hq, D = q.shape
    total_kv, Hkv, _ = k_cache.shape
    B = q_indptr.numel() - 1
    if q_indptr.dtype != torch.int32 or kv_indptr.dtype != torch.int64:
        raise TypeError("q_indptr must be int32 and kv_indptr int64")
    if tree_mask.element_size() != 8 or tree_mask.numel() != total_q:
        raise TypeError("tree_mask must hold one 64-bit word per query row")
    if lse is not None and lse.dtype != torch.float32:
        raise TypeError("lse must be float32")
    if out.dtype != q.dtype or k_cache.dtype != q.dtype or v_cache.dtype != q.dtype:
        raise TypeError("q, k_cache, v_cache and out must share one dtype")
    ws_ptr = _dev_ptr(workspace, "workspace") if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib.respec_verify_attention_tree(
        _dev_ptr(q, "q"), _dev_ptr(k_cache, "k_cache"), _dev_ptr(v_cache, "v_cache"),
        _dev_ptr(q_indptr, "q_indptr"), _dev_ptr(kv_indptr, "kv_indptr"), _dev_ptr(tree_mask, "tree_mask"),
        _dev_ptr(out, "out"), _dev_ptr(lse, "lse"), B, total_q, total_kv, max_q_per_seq, max_kv_len, Hq,
        Hkv, D, float(sm_scale), _dtype_code(q), ws_ptr, ws_bytes, _stream_ptr(stream)))


def respec_profile_mark_main(before: Optional[torch.cuda.Event], after: Optional[torch.cuda.Event]):
    """Have the next respec_verify_attention record the two events around its main kernel."""
    def handle(ev):
        if ev is None:
            return None
        if not ev.cuda_event:
            raise ValueError("the event must have been created (record it once first)")
        return ctypes.c_void_p(ev.cuda_event)
    load().respec_profile_mark_main(handle(before), handle(after))


def respec_rejection_sample_workspace_bytes(B, total_q, V, logits_dt) -> int:
    return int(load().respec_rejection_sample_workspace_bytes(B, total_q, V, logits_dt))


def respec_rejection_sample(target_logits, draft_logits, draft_tokens, q_indptr, u_accept, u_final,
                            out_tokens, out_num_accepted, out_flags, max_k, temperature,
                            workspace=None, stream=None):
    """target_logits [total_q,V], draft_logits [total_q-B,V]; outputs are written in place."""
    lib = load()
    total_q, V = target_logits.shape
    B = q_indptr.numel() - 1
    if q_indptr.dtype != torch.int32:
        raise TypeError("q_indptr must be int32")
    if out_tokens.dtype != torch.int32 or out_num_accepted.dtype != torch.int32:
        raise TypeError("out_tokens and out_num_accepted must be int32")
    if tuple(out_tokens.shape) != (B, max_k + 1) or out_num_accepted.numel() != B:
        raise ValueError("out_tokens must be [B, max_k+1] and out_num_accepted [B]")
    if u_final.dtype != torch.float32 or u_final.numel() != B:
        raise TypeError("u_final must be float32 [B]")
    n_draft = total_q - B
    if n_draft > 0:
        if draft_logits.dtype != target_logits.dtype or tuple(draft_logits.shape) != (n_draft, V):
            raise ValueError("draft_logits must be [total_q-B, V] in the target's dtype")
        if draft_tokens.dtype != torch.int32 or draft_tokens.numel() != n_draft:
            raise TypeError("draft_tokens must be int32 [total_q-B]")
        if u_accept.dtype != torch.float32 or u_accept.numel() != n_draft:
            raise TypeError("u_accept must be float32 [total_q-B]")
        ld_d = draft_logits.stride(0)
    else:
        draft_logits = draft_tokens = u_accept = None
        ld_d = V
    if target_logits.stride(1) != 1:
        raise ValueError("logits rows must be unit-stride")
    ws_ptr = _dev_ptr(workspace, "workspace") if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0

    def row_ptr(t, name):
        if t is None:
            return None
        if not t.is_cuda:
            raise ValueError(f"{name} must live on the GPU")
        return t.data_ptr()

    _check(lib.respec_rejection_sample(
        row_ptr(target_logits, "target_logits"), row_ptr(draft_logits, "draft_logits"),
        _dev_ptr(draft_tokens, "draft_tokens"), _dev_ptr(q_indptr, "q_indptr"),
        _dev_ptr(u_accept, "u_accept"), _dev_ptr(u_final, "u_final"),
        _dev_ptr(out_tokens, "out_tokens"), _dev_ptr(out_num_accepted, "out_num_accepted"),
        _dev_ptr(out_flags, "out_flags"), B, total_q, max_k, V, target_logits.stride(0), ld_d,
        float(temperature), _dtype_code(target_logits), ws_ptr, ws_bytes, _stream_ptr(stream)))


def respec_rejection_sample_per_seq(target_logits, draft_logits, draft_tokens, q_indptr, u_accept, u_final,
                                    temperatures, out_tokens, out_num_accepted, out_flags, max_k, stream=None):
    """respec_rejection_sample with temperatures [B] float32 on the device (0 = greedy).
    draft_logits and u_accept may be None when every sequence that has drafts is greedy."""
    lib = load()
    total_q, V = target_logits.shape
    B = q_indptr.numel() - 1
    if q_indptr.dtype != torch.int32:
        raise TypeError("q_indptr must be int32")
    if out_tokens.dtype != torch.int32 or out_num_accepted.dtype != torch.int32:
        raise TypeError("out_tokens and out_num_accepted must be int32")
    if tuple(out_tokens.shape) != (B, max_k + 1) or out_num_accepted.numel() != B:
        raise ValueError("out_tokens must be [B, max_k+1] and out_num_accepted [B]")
    if u_final.dtype != torch.float32 or u_final.numel() != B:
        raise TypeError("u_final must be float32 [B]")
    if temperatures.dtype != torch.float32 or temperatures.numel() != B:
        raise TypeError("temperatures must be float32 [B]")
    n_draft = total_q - B
    ld_d = V
    if n_draft > 0:
        if draft_tokens.dtype != torch.int32 or draft_tokens.numel() != n_draft:
            raise TypeError("draft_tokens must be int32 [total_q-B]")
        if draft_logits is not None:
            if draft_logits.dtype != target_logits.dtype or tuple(draft_logits.shape) != (n_draft, V):
                raise ValueError("draft_logits must be [total_q-B, V] in the target's dtype")
            ld_d = draft_logits.stride(0)
        if u_accept is not None and (u_accept.dtype != torch.float32 or u_accept.numel() != n_draft):
            raise TypeError("u_accept must be float32 [total_q-B]")
    else:
        draft_logits = draft_tokens = u_accept = None
    if target_logits.stride(1) != 1:
        raise ValueError("logits rows must be unit-stride")

    def row_ptr(t, name):
        if t is None:
            return None
        if not t.is_cuda:
            raise ValueError(f"{name} must live on the GPU")
        return t.data_ptr()

    _check(lib.respec_rejection_sample_per_seq(
        row_ptr(target_logits, "target_logits"), row_ptr(draft_logits, "draft_logits"),
        _dev_ptr(draft_tokens, "draft_tokens"), _dev_ptr(q_indptr, "q_indptr"),
        _dev_ptr(u_accept, "u_accept"), _dev_ptr(u_final, "u_final"), _dev_ptr(temperatures, "temperatures"),
        _dev_ptr(out_tokens, "out_tokens"), _dev_ptr(out_num_accepted, "out_num_accepted"),
        _dev_ptr(out_flags, "out_flags"), B, total_q, max_k, V, target_logits.stride(0), ld_d,
        _dtype_code(target_logits), _stream_ptr(stream)))


def respec_tree_rejection_sample(target_logits, draft_logits, node_tokens, parent, q_indptr, u_accept,
                                 u_final, out_tokens, out_path, out_num_accepted, out_flags,
                                 max_q_per_seq, max_depth, temperature, stream=None):
    """target_logits and draft_logits [total_q,V] (one row per tree node); outputs are written in place."""
    lib = load()
    total_q, V = target_logits.shape
    B = q_indptr.numel() - 1
    if q_indptr.dtype != torch.int32:
        raise TypeError("q_indptr must be int32")
    if draft_logits.dtype != target_logits.dtype or tuple(draft_logits.shape) != (total_q, V):
        raise ValueError("draft_logits must be [total_q, V] in the target's dtype")
    for t, name in ((node_tokens, "node_tokens"), (parent, "parent")):
        if t.dtype != torch.int32 or t.numel() != total_q:
            raise TypeError(f"{name} must be int32 [total_q]")
    if u_accept.dtype != torch.float32 or u_accept.numel() != total_q:
        raise TypeError("u_accept must be float32 [total_q]")
    if u_final.dtype != torch.float32 or u_final.numel() != B:
        raise TypeError("u_final must be float32 [B]")
    for t, name in ((out_tokens, "out_tokens"), (out_path, "out_path"), (out_num_accepted, "out_num_accepted")):
        if t.dtype != torch.int32:
            raise TypeError(f"{name} must be int32")
    if tuple(out_tokens.shape) != (B, max_depth + 1) or tuple(out_path.shape) != (B, max(max_depth, 1)):
        raise ValueError("out_tokens must be [B, max_depth+1] and out_path [B, max(max_depth,1)]")
    if out_num_accepted.numel() != B:
        raise ValueError("out_num_accepted must be [B]")
    if target_logits.stride(1) != 1 or draft_logits.stride(1) != 1:
        raise ValueError("logits rows must be unit-stride")
    for t, name in ((target_logits, "target_logits"), (draft_logits, "draft_logits")):
        if not t.is_cuda:
            raise ValueError(f"{name} must live on the GPU")
    _check(lib.respec_tree_rejection_sample(
        target_logits.data_ptr(), draft_logits.data_ptr(),
        _dev_ptr(node_tokens, "node_tokens"), _dev_ptr(parent, "parent"), _dev_ptr(q_indptr, "q_indptr"),
        _dev_ptr(u_accept, "u_accept"), _dev_ptr(u_final, "u_final"), _dev_ptr(out_tokens, "out_tokens"),
        _dev_ptr(out_path, "out_path"), _dev_ptr(out_num_accepted, "out_num_accepted"),
        _dev_ptr(out_flags, "out_flags"), B, total_q, max_q_per_seq, max_depth, V,
        target_logits.stride(0), draft_logits.stride(0), float(temperature), _dtype_code(target_logits),
        _stream_ptr(stream)))


def respec_verify_attention_paged_next_layer(q, k_pages, v_pages, q_indptr, page_indptr, page_table, kv_len, out,
                                             lse, max_q_per_seq, max_kv_len, sm_scale, workspace, tree_mask=None,
                                             stream=None):
    """Another layer's pools behind the same page table: reuses the set-up in the workspace."""
    respec_verify_attention_paged(q, k_pages, v_pages, q_indptr, page_indptr, page_table, kv_len, out, lse,
                                  max_q_per_seq, max_kv_len, sm_scale, workspace, tree_mask=tree_mask, stream=stream,
                                  _entry="respec_verify_attention_paged_next_layer")


def respec_verify_attention_paged(q, k_pages, v_pages, q_indptr, page_indptr, page_table, kv_len, out, lse,
                                  max_q_per_seq, max_kv_len, sm_scale, workspace, tree_mask=None, stream=None,
                                  _entry="respec_verify_attention_paged"):
    """k_pages, v_pages [num_pages, page_size, Hkv, D]; out is written in place."""
    lib = load()
    total_q, Hq, D = q.shape
    num_pages, page_size, Hkv, Dk = k_pages.shape
    if Dk != D or tuple(v_pages.shape) != tuple(k_pages.shape):
        raise ValueError("k_pages and v_pages must be [num_pages, page_size, Hkv, D] with q's D")
    if k_pages.dtype != q.dtype or v_pages.dtype != q.dtype or out.dtype != q.dtype:
        raise TypeError("q, k_pages, v_pages and out must share one dtype")
    if tuple(out.shape) != tuple(q.shape):
        raise ValueError("out must have q's shape")
    B = q_indptr.numel() - 1
    for t, name, n in ((q_indptr, "q_indptr", B + 1), (page_indptr, "page_indptr", B + 1), (kv_len, "kv_len", B)):
        if t.dtype != torch.int32 or t.numel() != n:
            raise TypeError(f"{name} must be int32 [{n}]")
    if page_table.dtype != torch.int32:
        raise TypeError("page_table must be int32")
    if tree_mask is not None and (tree_mask.dtype != torch.int64 or tree_mask.numel() != total_q):
        raise TypeError("tree_mask must be int64 [total_q] (the bits of a uint64 per row)")
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (total_q, Hq)):
        raise TypeError("lse must be float32 [total_q, Hq]")
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(getattr(lib, _entry)(
        _dev_ptr(q, "q"), _dev_ptr(k_pages, "k_pages"), _dev_ptr(v_pages, "v_pages"), _dev_ptr(q_indptr, "q_indptr"),
        _dev_ptr(page_indptr, "page_indptr"), _dev_ptr(page_table, "page_table"), _dev_ptr(kv_len, "kv_len"),
        _dev_ptr(tree_mask, "tree_mask"), _dev_ptr(out, "out"), _dev_ptr(lse, "lse"), B, total_q, num_pages,
        page_table.numel(), page_size, max_q_per_seq, max_kv_len, Hq, Hkv, D, float(sm_scale), _dtype_code(q),
        _dev_ptr(workspace, "workspace"), ws_bytes, _stream_ptr(stream)))


def respec_commit_accepted_paged(k_pages, v_pages, q_indptr, page_indptr, page_table, kv_len, num_accepted,
                                 total_q, max_q_per_seq, path=None, stream=None):
    """Moves the K/V of the accepted rows behind the last committed token; k_pages, v_pages and
    kv_len are changed in place."""
    lib = load()
    num_pages, page_size, Hkv, D = k_pages.shape
    if tuple(v_pages.shape) != tuple(k_pages.shape) or v_pages.dtype != k_pages.dtype:
        raise ValueError("k_pages and v_pages must have one shape and dtype")
    B = q_indptr.numel() - 1
    for t, name, n in ((q_indptr, "q_indptr", B + 1), (page_indptr, "page_indptr", B + 1), (kv_len, "kv_len", B),
                       (num_accepted, "num_accepted", B)):
        if t.dtype != torch.int32 or t.numel() != n:
            raise TypeError(f"{name} must be int32 [{n}]")
    if page_table.dtype != torch.int32:
        raise TypeError("page_table must be int32")
    stride = 0
    if path is not None:
        if path.dtype != torch.int32 or path.dim() != 2 or path.shape[0] != B:
            raise TypeError("path must be int32 [B, stride]")
        stride = path.shape[1]
    _check(lib.respec_commit_accepted_paged(
        _dev_ptr(k_pages, "k_pages"), _dev_ptr(v_pages, "v_pages"), _dev_ptr(q_indptr, "q_indptr"),
        _dev_ptr(page_indptr, "page_indptr"), _dev_ptr(page_table, "page_table"), _dev_ptr(kv_len, "kv_len"),
        _dev_ptr(path, "path"), stride, _dev_ptr(num_accepted, "num_accepted"), B, total_q, max_q_per_seq,
        num_pages, page_table.numel(), page_size, Hkv, D, _dtype_code(k_pages), _stream_ptr(stream)))


def respec_kd_rows_workspace_bytes(rows, V, dt) -> int:
    return int(load().respec_kd_rows_workspace_bytes(rows, V, dt))


def respec_kd_rows(target_logits, draft_logits, row_weight, grad, row_loss, total_loss, workspace, stream=None):
    """target_logits, draft_logits, grad [rows, V]; row_weight, row_loss [rows] f32; total_loss [1] f64 or None."""
    lib = load()
    rows, V = target_logits.shape
    for t, name in ((draft_logits, "draft_logits"), (grad, "grad")):
        if tuple(t.shape) != (rows, V) or t.dtype != target_logits.dtype or t.stride(1) != 1:
            raise ValueError(f"{name} must be [rows, V] in the target's dtype with unit-stride rows")
    if target_logits.stride(1) != 1:
        raise ValueError("logits rows must be unit-stride")
    for t, name in ((row_weight, "row_weight"), (row_loss, "row_loss")):
        if t.dtype != torch.float32 or t.numel() != rows:
            raise TypeError(f"{name} must be float32 [rows]")
    if total_loss is not None and (total_loss.dtype != torch.float64 or total_loss.numel() != 1):
        raise TypeError("total_loss must be float64 [1]")
    for t, name in ((target_logits, "target_logits"), (draft_logits, "draft_logits"), (grad, "grad")):
        if not t.is_cuda:
            raise ValueError(f"{name} must live on the GPU")
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib.respec_kd_rows(
        target_logits.data_ptr(), draft_logits.data_ptr(),
        _dev_ptr(row_weight, "row_weight"), grad.data_ptr(), _dev_ptr(row_loss, "row_loss"),
        _dev_ptr(total_loss, "total_loss"), rows, V, target_logits.stride(0), draft_logits.stride(0),
        grad.stride(0), _dtype_code(target_logits), _dev_ptr(workspace, "workspace"), ws_bytes,
        _stream_ptr(stream)))


# (As above: torch.cuda.current_device() takes 0.5 us of a call's 6 to 10, this 0.1.)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _here(first, *others):
    """The index of the current GPU, on which `first` and the others (None: absent) have to live: the stream is its."""
    index = first.get_device()
    if index < 0 or index != _current_device():
        raise ValueError(f"tensors must live on the current GPU (got {first.device})")
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError(f"all tensors must live on {first.device} (got one on {t.device})")
    return index


def _stream_on(index, stream):
    if stream is not None or _current_raw_stream is None:
        return _stream_ptr(stream)
    return _current_raw_stream(index)


_INT32, _FLOAT32 = torch.int32, torch.float32


def _ints(n, names, *tensors):
    """Contiguous int32 tensors of n elements (None: any number)."""
    for t in tensors:
        if t.dtype is not _INT32 or (n is not None and t.numel() != n) or not t.is_contiguous():
            name = names.split()[[x is t for x in tensors].index(True)]
            raise TypeError(f"{name} must be contiguous int32" + ("" if n is None else f" [{n}]"))


def _floats(n, names, *tensors):
    """Contiguous float32 tensors of n elements; None may stand for an absent one."""
    for t in tensors:
        if t is not None and (t.dtype is not _FLOAT32 or t.numel() != n or not t.is_contiguous()):
            name = names.split()[[x is t for x in tensors].index(True)]
            raise TypeError(f"{name} must be contiguous float32 [{n}]")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _room(workspace):
    """Address and size of a workspace (None: absent)."""
    if workspace is None:
        return None, 0
    return _dev_ptr(workspace, "workspace"), workspace.numel() * workspace.element_size()


def _token_stride(t, tokens, heads, D, name):
    """Elements between the tokens of a [tokens, heads, D] tensor whose tokens are contiguous in themselves."""
    token, head, one = t.stride()
    if one != 1 or (head != D and heads > 1):
        raise ValueError(f"{name} must be [tokens, heads, D] with contiguous tokens")
    return token if tokens > 1 else heads * D


def _three(t, name):
    if t.dim() != 3:
        raise ValueError(f"{name} must be [tokens, heads, D]")
    return t.shape


def respec_prompt_attention_workspace_bytes(B, total_q, total_kv, max_q_per_seq, max_kv_len, Hq, Hkv, D, dt) -> int:
    return int(load().respec_prompt_attention_workspace_bytes(B, total_q, total_kv, max_q_per_seq, max_kv_len, Hq, Hkv, D, dt))


def respec_prompt_attention(q, k, v, q_indptr, kv_indptr, out, lse, max_q_per_seq, max_kv_len, sm_scale, workspace, stream=None):
    """q [total_q,Hq,D], k and v [total_kv,Hkv,D] (slices along the token stride are fine), out contiguous; q_indptr int32,
    kv_indptr int64."""
    total_q, Hq, D = shape = _three(q, "q")
    total_kv, Hkv, Dk = kv_shape = _three(k, "k")
    B, dtype = q_indptr.numel() - 1, q.dtype
    index = _here(q, k, v, q_indptr, kv_indptr, out, lse, workspace)
    _ints(B + 1, "q_indptr", q_indptr)
    if kv_indptr.dtype is not torch.int64 or kv_indptr.numel() != B + 1 or not kv_indptr.is_contiguous():
        raise TypeError(f"kv_indptr must be contiguous int64 [{B + 1}]")
    if k.dtype is not dtype or v.dtype is not dtype or out.dtype is not dtype:
        raise TypeError("q, k, v and out must share one dtype")
    if Dk != D or v.shape != kv_shape or out.shape != shape or not out.is_contiguous():
        raise ValueError("k and v must be [total_kv, Hkv, D] with q's D, and out contiguous in q's shape")
    _floats(total_q * Hq, "lse", lse)
    _check(load().respec_prompt_attention(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), q_indptr.data_ptr(), kv_indptr.data_ptr(), out.data_ptr(), _ptr(lse), B, total_q,
        total_kv, max_q_per_seq, max_kv_len, Hq, Hkv, D, _token_stride(q, total_q, Hq, D, "q"), _token_stride(k, total_kv, Hkv, D, "k"),
        _token_stride(v, total_kv, Hkv, D, "v"), float(sm_scale), _dtype_code(q), *_room(workspace), _stream_on(index, stream)))


def _pools(k_pages, v_pages):
    shape = k_pages.shape
    if len(shape) != 4 or v_pages.shape != shape or v_pages.dtype is not k_pages.dtype or not (
            k_pages.is_contiguous() and v_pages.is_contiguous()):
        raise ValueError("k_pages and v_pages must be contiguous [num_pages, page_size, Hkv, D] of one shape and dtype")
    return shape


def respec_prompt_attention_paged(q, k_pages, v_pages, q_indptr, page_indptr, page_table, kv_len, out, lse, max_q_per_seq,
                                  max_kv_len, sm_scale, workspace, stream=None):
    """q [total_q,Hq,D] (token stride), k_pages and v_pages [num_pages, page_size, Hkv, D]; out is written in place."""
    total_q, Hq, D = shape = _three(q, "q")
    num_pages, page_size, Hkv, Dk = _pools(k_pages, v_pages)
    B, dtype = q_indptr.numel() - 1, q.dtype
    index = _here(q, k_pages, v_pages, q_indptr, page_indptr, page_table, kv_len, out, lse, workspace)
    _ints(B + 1, "q_indptr page_indptr", q_indptr, page_indptr)
    _ints(B, "kv_len", kv_len)
    _ints(None, "page_table", page_table)
    if k_pages.dtype is not dtype or out.dtype is not dtype:
        raise TypeError("q, k_pages, v_pages and out must share one dtype")
    if Dk != D or out.shape != shape or not out.is_contiguous():
        raise ValueError("k_pages and v_pages must have q's D, and out must be contiguous in q's shape")
    _floats(total_q * Hq, "lse", lse)
    _check(load().respec_prompt_attention_paged(
        q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), q_indptr.data_ptr(), page_indptr.data_ptr(), page_table.data_ptr(),
        kv_len.data_ptr(), out.data_ptr(), _ptr(lse), B, total_q, num_pages, page_table.numel(), page_size, max_q_per_seq, max_kv_len,
        Hq, Hkv, D, _token_stride(q, total_q, Hq, D, "q"), float(sm_scale), _dtype_code(q), *_room(workspace), _stream_on(index, stream)))


def respec_append_paged(k_new, v_new, k_pages, v_pages, q_indptr, page_indptr, page_table, kv_len, max_q_per_seq, stream=None):
    """k_new, v_new [total_q, Hkv, D] (one token stride) into the last R_b of every sequence's kv_len tokens; the pools are
    changed in place."""
    num_pages, page_size, Hkv, D = _pools(k_pages, v_pages)
    total_q, H, Dn = shape = _three(k_new, "k_new")
    B, dtype = q_indptr.numel() - 1, k_pages.dtype
    index = _here(k_new, v_new, k_pages, v_pages, q_indptr, page_indptr, page_table, kv_len)
    _ints(B + 1, "q_indptr page_indptr", q_indptr, page_indptr)
    _ints(B, "kv_len", kv_len)
    _ints(None, "page_table", page_table)
    if k_new.dtype is not dtype or v_new.dtype is not dtype:
        raise TypeError("the new tokens must have the pools' dtype")
    if H != Hkv or Dn != D or v_new.shape != shape:
        raise ValueError("k_new and v_new must be [total_q, Hkv, D]")
    ld = _token_stride(k_new, total_q, H, D, "k_new")
    if _token_stride(v_new, total_q, H, D, "v_new") != ld:
        raise ValueError("k_new and v_new must have one token stride")
    _check(load().respec_append_paged(
        k_new.data_ptr(), v_new.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), q_indptr.data_ptr(), page_indptr.data_ptr(),
        page_table.data_ptr(), kv_len.data_ptr(), B, total_q, max_q_per_seq, num_pages, page_table.numel(), page_size, Hkv, D, ld,
        _dtype_code(k_pages), _stream_on(index, stream)))


def respec_pages_workspace_bytes(B, num_pages) -> int:
    return int(load().respec_pages_workspace_bytes(B, num_pages))


def respec_pages_resize(want_tokens, page_indptr, page_table, page_count, kv_len, page_refs, copy_src, copy_dst, out_missing, page_size,
                        workspace, stream=None):
    """want_tokens [B] (negative: leave the sequence alone); the state and the outputs are changed in place."""
    B = want_tokens.numel()
    index = _here(want_tokens, page_indptr, page_table, page_count, kv_len, page_refs, copy_src, copy_dst, out_missing, workspace)
    _ints(B + 1, "page_indptr", page_indptr)
    _ints(B, "want_tokens page_count kv_len copy_src copy_dst out_missing", want_tokens, page_count, kv_len, copy_src, copy_dst, out_missing)
    _ints(None, "page_table page_refs", page_table, page_refs)
    _check(load().respec_pages_resize(
        want_tokens.data_ptr(), page_indptr.data_ptr(), page_table.data_ptr(), page_count.data_ptr(), kv_len.data_ptr(),
        page_refs.data_ptr(), copy_src.data_ptr(), copy_dst.data_ptr(), out_missing.data_ptr(), B, page_table.numel(), page_refs.numel(),
        page_size, *_room(workspace), _stream_on(index, stream)))


def respec_pages_fork(parent, page_indptr, page_table, page_count, kv_len, page_refs, out_missing, stream=None):
    """parent [B] (negative: leave the sequence alone); the state and out_missing are changed in place."""
    B = parent.numel()
    index = _here(parent, page_indptr, page_table, page_count, kv_len, page_refs, out_missing)
    _ints(B + 1, "page_indptr", page_indptr)
    _ints(B, "parent page_count kv_len out_missing", parent, page_count, kv_len, out_missing)
    _ints(None, "page_table page_refs", page_table, page_refs)
    _check(load().respec_pages_fork(
        parent.data_ptr(), page_indptr.data_ptr(), page_table.data_ptr(), page_count.data_ptr(), kv_len.data_ptr(), page_refs.data_ptr(),
        out_missing.data_ptr(), B, page_table.numel(), page_refs.numel(), _stream_on(index, stream)))


def respec_pages_compact(page_table, page_refs, new_page_table, new_page_refs, copy_src, copy_dst, out_pages_end, workspace, stream=None):
    """At most copy_src.numel() moves; new_page_table and new_page_refs may be the old ones."""
    index = _here(page_table, page_refs, new_page_table, new_page_refs, copy_src, copy_dst, out_pages_end, workspace)
    _ints(None, "page_table page_refs copy_src", page_table, page_refs, copy_src)
    _ints(page_table.numel(), "new_page_table", new_page_table)
    _ints(page_refs.numel(), "new_page_refs", new_page_refs)
    _ints(copy_src.numel(), "copy_dst", copy_dst)
    _ints(1, "out_pages_end", out_pages_end)
    _check(load().respec_pages_compact(
        page_table.data_ptr(), page_refs.data_ptr(), new_page_table.data_ptr(), new_page_refs.data_ptr(), copy_src.data_ptr(),
        copy_dst.data_ptr(), out_pages_end.data_ptr(), page_table.numel(), page_refs.numel(), copy_src.numel(), *_room(workspace),
        _stream_on(index, stream)))


def respec_pages_copy(k_pages, v_pages, copy_src, copy_dst, stream=None):
    """Pages copy_src[i] -> copy_dst[i] of one layer's pools (-1: none)."""
    num_pages, page_size, Hkv, D = _pools(k_pages, v_pages)
    index = _here(k_pages, v_pages, copy_src, copy_dst)
    _ints(None, "copy_src", copy_src)
    _ints(copy_src.numel(), "copy_dst", copy_dst)
    _check(load().respec_pages_copy(
        k_pages.data_ptr(), v_pages.data_ptr(), copy_src.data_ptr(), copy_dst.data_ptr(), copy_src.numel(), num_pages, page_size, Hkv, D,
        _dtype_code(k_pages), _stream_on(index, stream)))


def _rows_of(logits):
    rows, V = logits.shape
    row, one = logits.stride()
    if one != 1 and V > 1:
        raise ValueError("logits rows must be unit-stride")
    return rows, V, row if rows > 1 else V


def respec_token_logprobs_workspace_bytes(rows, V, top_n, dt) -> int:
    return int(load().respec_token_logprobs_workspace_bytes(rows, V, top_n, dt))


def respec_token_logprobs(logits, tokens, logprob, lse, entropy, top_tokens, top_logprobs, temperature, workspace, row_temperature=None,
                          stream=None):
    """logits [rows,V], tokens [rows] int32 (outside [0,V): an unused row); logprob, lse, entropy (or None) [rows] float32;
    top_tokens int32 and top_logprobs float32 [rows,n] or both None.  row_temperature [rows] takes the place of temperature."""
    rows, V, ld = _rows_of(logits)
    index = _here(logits, tokens, logprob, lse, entropy, top_tokens, top_logprobs, workspace, row_temperature)
    _ints(rows, "tokens", tokens)
    _floats(rows, "logprob lse entropy row_temperature", logprob, lse, entropy, row_temperature)
    if (top_tokens is None) != (top_logprobs is None):
        raise ValueError("top_tokens and top_logprobs go together")
    n = 0
    if top_tokens is not None:
        shape = top_tokens.shape
        if len(shape) != 2 or shape[0] != rows:
            raise ValueError("top_tokens must be [rows, n]")
        n = shape[1]
        _ints(rows * n, "top_tokens", top_tokens)
        _floats(rows * n, "top_logprobs", top_logprobs)
    _check(load().respec_token_logprobs(
        logits.data_ptr(), tokens.data_ptr(), _ptr(row_temperature), logprob.data_ptr(), lse.data_ptr(), _ptr(entropy), _ptr(top_tokens),
        _ptr(top_logprobs), rows, V, ld, n, float(temperature), _dtype_code(logits), *_room(workspace), _stream_on(index, stream)))


def respec_token_logprobs_grad(logits, tokens, lse, entropy, grad_logprob, grad_entropy, grad_logits, temperature, row_temperature=None,
                               stream=None):
    """The gradient in the logits from what respec_token_logprobs wrote; grad_logprob or grad_entropy may be None."""
    rows, V, ld = _rows_of(logits)
    index = _here(logits, tokens, lse, entropy, grad_logprob, grad_entropy, grad_logits, row_temperature)
    _ints(rows, "tokens", tokens)
    _floats(rows, "lse entropy grad_logprob grad_entropy row_temperature", lse, entropy, grad_logprob, grad_entropy, row_temperature)
    rows_g, V_g, ld_g = _rows_of(grad_logits)
    if rows_g != rows or V_g != V or grad_logits.dtype is not logits.dtype:
        raise ValueError("grad_logits must have the logits' shape and dtype")
    _check(load().respec_token_logprobs_grad(
        logits.data_ptr(), tokens.data_ptr(), _ptr(row_temperature), lse.data_ptr(), _ptr(entropy), _ptr(grad_logprob),
        _ptr(grad_entropy), grad_logits.data_ptr(), rows, V, ld, ld_g, float(temperature), _dtype_code(logits), _stream_on(index, stream)))


_E4M3_TYPES = (torch.float8_e4m3fn, torch.uint8)


def _scaled_pools(k_pages, v_pages, k_scale, v_scale):
    """Shape and type code of pools that may be of 8 bits: these come with scales [num_pages, Hkv, page_size]."""
    num_pages, page_size, Hkv, D = shape = _pools(k_pages, v_pages)
    if k_scale is None and v_scale is None:
        return shape, _dtype_code(k_pages)
    if k_pages.dtype not in _E4M3_TYPES:
        raise TypeError("pools with scales must hold e4m3 codes (float8_e4m3fn or uint8)")
    for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
        if t is None or t.dtype is not torch.uint8 or tuple(t.shape) != (num_pages, Hkv, page_size) or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous uint8 [num_pages, Hkv, page_size]")
    return shape, RESPEC_E4M3


def respec_norm_rope_append_paged(q, k, v, q_weight, k_weight, inv_freq, positions, q_out, k_pages, v_pages, k_scale, v_scale, q_indptr,
                                  page_indptr, page_table, kv_len, max_q_per_seq, eps, interleaved=False, stream=None):
    """q, q_out [total_q,Hq,D] (both None: K and V only), k, v [total_q,Hkv,D], each with a token stride of its own; weights [D] and inv_freq
    [rotary_dim/2] float32 or None, positions [total_q] int32 or None; pools in k's dtype, or e4m3 codes with k_scale and v_scale."""
    (num_pages, page_size, Hkv, D), pool = _scaled_pools(k_pages, v_pages, k_scale, v_scale)
    total_q, H, Dk = shape = _three(k, "k")
    B, dtype, Hq = q_indptr.numel() - 1, k.dtype, Hkv
    index = _here(k, q, v, q_weight, k_weight, inv_freq, positions, q_out, k_pages, v_pages, k_scale, v_scale, q_indptr, page_indptr, page_table,
                  kv_len)
    _ints(B + 1, "q_indptr page_indptr", q_indptr, page_indptr)
    _ints(B, "kv_len", kv_len)
    _ints(None, "page_table", page_table)
    if positions is not None:
        _ints(total_q, "positions", positions)
    _floats(D, "q_weight k_weight", q_weight, k_weight)
    if v.dtype is not dtype or (pool != RESPEC_E4M3 and k_pages.dtype is not dtype):
        raise TypeError("k, v and pools without scales must share one dtype")
    if H != Hkv or Dk != D or v.shape != shape:
        raise ValueError("k and v must be [total_q, Hkv, D]")
    ld_q = ld_out = 0
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    if q is not None:
        n, Hq, Dq = _three(q, "q")
        if n != total_q or Dq != D or q_out.shape != q.shape or q.dtype is not dtype or q_out.dtype is not dtype:
            raise ValueError("q and q_out must be [total_q, Hq, D] in k's dtype")
        ld_q, ld_out = _token_stride(q, n, Hq, D, "q"), _token_stride(q_out, n, Hq, D, "q_out")
    rotary = 0
    if inv_freq is not None:
        rotary = 2 * inv_freq.numel()
        _floats(rotary // 2, "inv_freq", inv_freq)
    _check(load().respec_norm_rope_append_paged(
        _ptr(q), k.data_ptr(), v.data_ptr(), _ptr(q_weight), _ptr(k_weight), _ptr(inv_freq), _ptr(positions), _ptr(q_out), k_pages.data_ptr(),
        v_pages.data_ptr(), _ptr(k_scale), _ptr(v_scale), q_indptr.data_ptr(), page_indptr.data_ptr(), page_table.data_ptr(), kv_len.data_ptr(),
        B, total_q, max_q_per_seq, num_pages, page_table.numel(), page_size, Hq, Hkv, D, rotary, int(interleaved), ld_q,
        _token_stride(k, total_q, H, D, "k"), _token_stride(v, total_q, H, D, "v"), ld_out, float(eps), _dtype_code(k), pool,
        _stream_on(index, stream)))


def _quantised_pools(k_pages, v_pages, k_scale, v_scale):
    if k_scale is None or v_scale is None:
        raise ValueError("a cache of 8 bits has k_scale and v_scale")
    return _scaled_pools(k_pages, v_pages, k_scale, v_scale)[0]


def respec_read_paged_quantised(k_pages, v_pages, k_scale, v_scale, page_indptr, page_table, kv_len, kv_indptr, k_out, v_out, max_kv_len, stream=None):
    """What the tokens of every sequence stand for to rows kv_indptr[b] on of k_out and v_out [total_kv, Hkv, D] (bf16 or float32)."""
    num_pages, page_size, Hkv, D = _quantised_pools(k_pages, v_pages, k_scale, v_scale)
    total_kv, H, Dk = shape = _three(k_out, "k_out")
    B = page_indptr.numel() - 1
    index = _here(k_pages, v_pages, k_scale, v_scale, page_indptr, page_table, kv_len, kv_indptr, k_out, v_out)
    _ints(B, "kv_len", kv_len)
    _ints(None, "page_indptr page_table", page_indptr, page_table)
    if kv_indptr.dtype is not torch.int64 or kv_indptr.numel() != B + 1 or not kv_indptr.is_contiguous():
        raise TypeError(f"kv_indptr must be contiguous int64 [{B + 1}]")
    if H != Hkv or Dk != D or v_out.shape != shape or v_out.dtype is not k_out.dtype or not (k_out.is_contiguous() and v_out.is_contiguous()):
        raise ValueError("k_out and v_out must be contiguous [total_kv, Hkv, D] of one dtype")
    _check(load().respec_read_paged_quantised(
        k_pages.data_ptr(), v_pages.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), page_indptr.data_ptr(), page_table.data_ptr(),
        kv_len.data_ptr(), kv_indptr.data_ptr(), k_out.data_ptr(), v_out.data_ptr(), B, total_kv, max_kv_len, num_pages, page_table.numel(), page_size,
        Hkv, D, _dtype_code(k_out), _stream_on(index, stream)))


def respec_commit_accepted_paged_quantised(k_pages, v_pages, k_scale, v_scale, q_indptr, page_indptr, page_table, kv_len, num_accepted, total_q,
                                           max_q_per_seq, path=None, stream=None):
    """respec_commit_accepted_paged for a cache of 8 bits; pools, scales and kv_len are changed in place."""
    num_pages, page_size, Hkv, D = _quantised_pools(k_pages, v_pages, k_scale, v_scale)
    B = q_indptr.numel() - 1
    index = _here(k_pages, v_pages, k_scale, v_scale, q_indptr, page_indptr, page_table, kv_len, num_accepted, path)
    _ints(B + 1, "q_indptr page_indptr", q_indptr, page_indptr)
    _ints(B, "kv_len num_accepted", kv_len, num_accepted)
    _ints(None, "page_table", page_table)
    stride = 0
    if path is not None:
        if path.dim() != 2 or path.shape[0] != B:
            raise ValueError("path must be [B, stride]")
        stride = path.shape[1]
        _ints(None, "path", path)
    _check(load().respec_commit_accepted_paged_quantised(
        k_pages.data_ptr(), v_pages.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), q_indptr.data_ptr(), page_indptr.data_ptr(),
        page_table.data_ptr(), kv_len.data_ptr(), _ptr(path), stride, num_accepted.data_ptr(), B, total_q, max_q_per_seq, num_pages,
        page_table.numel(), page_size, Hkv, D, _stream_on(index, stream)))


def respec_pages_copy_quantised(k_pages, v_pages, k_scale, v_scale, copy_src, copy_dst, stream=None):
    """Pages copy_src[i] -> copy_dst[i] of one layer's codes and scales (-1: none)."""
    num_pages, page_size, Hkv, D = _quantised_pools(k_pages, v_pages, k_scale, v_scale)
    index = _here(k_pages, v_pages, k_scale, v_scale, copy_src, copy_dst)
    _ints(None, "copy_src", copy_src)
    _ints(copy_src.numel(), "copy_dst", copy_dst)
    _check(load().respec_pages_copy_quantised(
        k_pages.data_ptr(), v_pages.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), copy_src.data_ptr(), copy_dst.data_ptr(), copy_src.numel(),
        num_pages, page_size, Hkv, D, _stream_on(index, stream)))


def respec_verify_attention_shared_workspace_bytes(B, total_q, num_groups, max_q_per_seq, max_kv_len, Hq, Hkv, D, dt) -> int:
    return int(load().respec_verify_attention_shared_workspace_bytes(B, total_q, num_groups, max_q_per_seq, max_kv_len, Hq, Hkv, D, dt))


def respec_verify_attention_shared(q, k_pages, v_pages, k_scale, v_scale, q_indptr, page_indptr, page_table, kv_len, group_indptr, shared_len,
                                   tree_mask, out, lse, max_q_per_seq, max_kv_len, sm_scale, workspace, stream=None,
                                   _entry="respec_verify_attention_shared"):
    """q, out [total_q,Hq,D] contiguous, pools in q's dtype, or e4m3 codes with k_scale and v_scale (q bf16); group_indptr [num_groups+1] and shared_len
    [num_groups] int32, or both None; tree_mask [total_q] int64 or None."""
    (num_pages, page_size, Hkv, Dk), pool = _scaled_pools(k_pages, v_pages, k_scale, v_scale)
    total_q, Hq, D = shape = _three(q, "q")
    B, dtype = q_indptr.numel() - 1, q.dtype
    index = _here(q, k_pages, v_pages, k_scale, v_scale, q_indptr, page_indptr, page_table, kv_len, group_indptr, shared_len, tree_mask, out, lse,
                  workspace)
    _ints(B + 1, "q_indptr page_indptr", q_indptr, page_indptr)
    _ints(B, "kv_len", kv_len)
    _ints(None, "page_table", page_table)
    if (group_indptr is None) != (shared_len is None):
        raise ValueError("group_indptr and shared_len go together")
    groups = 0
    if shared_len is not None:
        groups = shared_len.numel()
        _ints(groups, "shared_len", shared_len)
        _ints(groups + 1, "group_indptr", group_indptr)
    if tree_mask is not None and (tree_mask.dtype is not torch.int64 or tree_mask.numel() != total_q or not tree_mask.is_contiguous()):
        raise TypeError("tree_mask must be contiguous int64 [total_q] (the bits of a uint64 per row)")
    if out.dtype is not dtype or (pool != RESPEC_E4M3 and k_pages.dtype is not dtype):
        raise TypeError("q, out and pools without scales must share one dtype")
    if Dk != D or out.shape != shape or not (out.is_contiguous() and q.is_contiguous()):
        raise ValueError("q and out must be contiguous [total_q, Hq, D] with the pools' D")
    _floats(total_q * Hq, "lse", lse)
    _check(getattr(load(), _entry)(
        q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_scale), _ptr(v_scale), q_indptr.data_ptr(), page_indptr.data_ptr(),
        page_table.data_ptr(), kv_len.data_ptr(), _ptr(group_indptr), _ptr(shared_len), _ptr(tree_mask), out.data_ptr(), _ptr(lse), B, total_q, groups,
        num_pages, page_table.numel(), page_size, max_q_per_seq, max_kv_len, Hq, Hkv, D, float(sm_scale), _dtype_code(q), pool, *_room(workspace),
        _stream_on(index, stream)))


def respec_verify_attention_shared_next_layer(*args, **kwargs):
    """Another layer of the same forward: respec_verify_attention_shared with the set-up that its workspace holds."""
    respec_verify_attention_shared(*args, **kwargs, _entry="respec_verify_attention_shared_next_layer")


def respec_verify_attention_paged_quantised(q, k_pages, v_pages, k_scale, v_scale, q_indptr, page_indptr, page_table, kv_len, out, lse,
                                            max_q_per_seq, max_kv_len, sm_scale, workspace, tree_mask=None, stream=None):
    """respec_verify_attention_paged over a cache of 8 bits; the workspace is that of respec_verify_attention_shared without groups."""
    num_pages, page_size, Hkv, Dk = _quantised_pools(k_pages, v_pages, k_scale, v_scale)
    total_q, Hq, D = shape = _three(q, "q")
    B = q_indptr.numel() - 1
    index = _here(q, k_pages, v_pages, k_scale, v_scale, q_indptr, page_indptr, page_table, kv_len, tree_mask, out, lse, workspace)
    _ints(B + 1, "q_indptr page_indptr", q_indptr, page_indptr)
    _ints(B, "kv_len", kv_len)
    _ints(None, "page_table", page_table)
    if tree_mask is not None and (tree_mask.dtype is not torch.int64 or tree_mask.numel() != total_q or not tree_mask.is_contiguous()):
        raise TypeError("tree_mask must be contiguous int64 [total_q] (the bits of a uint64 per row)")
    if out.dtype is not q.dtype:
        raise TypeError("q and out must share one dtype")
    if Dk != D or out.shape != shape or not (out.is_contiguous() and q.is_contiguous()):
        raise ValueError("q and out must be contiguous [total_q, Hq, D] with the pools' D")
    _floats(total_q * Hq, "lse", lse)
    _check(load().respec_verify_attention_paged_quantised(
        q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), q_indptr.data_ptr(), page_indptr.data_ptr(),
        page_table.data_ptr(), kv_len.data_ptr(), _ptr(tree_mask), out.data_ptr(), _ptr(lse), B, total_q, num_pages, page_table.numel(), page_size,
        max_q_per_seq, max_kv_len, Hq, Hkv, D, float(sm_scale), _dtype_code(q), *_room(workspace), _stream_on(index, stream)))


def respec_solver_pick(points, active_batch, draft_us_fixed, draft_us_per_seq):
    """points: iterable of (batch, k, step_us, emitted_per_seq), host numbers.
    Returns (best_k, speedup, cost_us)."""
    lib = load()
    pts = list(points)
    arr = (ProfilePoint * max(len(pts), 1))()
    for i, (B, k, t, e) in enumerate(pts):
        arr[i] = ProfilePoint(int(B), int(k), float(t), float(e))
    best, speedup, cost = ctypes.c_int32(-1), ctypes.c_double(0.0), ctypes.c_double(0.0)
    _check(lib.respec_solver_pick(ctypes.cast(arr, ctypes.c_void_p) if pts else None, len(pts), int(active_batch),
                                  float(draft_us_fixed), float(draft_us_per_seq), ctypes.byref(best),
                                  ctypes.byref(speedup), ctypes.byref(cost)))
    return best.value, speedup.value, cost.value


def respec_validate_batch(q_indptr, kv_indptr, draft_tokens, total_q, total_kv, max_q_per_seq, max_kv_len, V,
                          stream=None):
    """Debug check of a batch's index arrays and drafted tokens; raises RespecError naming the
    first bad sequence.  Synchronises the stream."""
    lib = load()
    B = q_indptr.numel() - 1
    if q_indptr.dtype != torch.int32 or (kv_indptr is not None and kv_indptr.dtype != torch.int64):
        raise TypeError("q_indptr must be int32 and kv_indptr int64")
    if draft_tokens is not None and draft_tokens.dtype != torch.int32:
        raise TypeError("draft_tokens must be int32")
    ws = torch.empty(int(lib.respec_validate_batch_workspace_bytes(B)), dtype=torch.uint8, device=q_indptr.device)
    _check(lib.respec_validate_batch(_dev_ptr(q_indptr, "q_indptr"), _dev_ptr(kv_indptr, "kv_indptr"),
                                     _dev_ptr(draft_tokens, "draft_tokens"), B, int(total_q), int(total_kv),
                                     int(max_q_per_seq), int(max_kv_len), int(V), _dev_ptr(ws, "workspace"),
                                     ws.numel(), _stream_ptr(stream)))
