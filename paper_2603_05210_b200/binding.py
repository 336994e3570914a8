"""Python binding of ``libvt.so``: argument marshalling only.

Each function has the name of the C entry point it calls (``include/vt.h``) and passes torch
tensors' device pointers and the current CUDA stream through ctypes.  PyTorch provides device
memory and streams; every step of the head runs inside the library's kernels.  There is no
fallback: if the library cannot be loaded the call raises.
"""
from __future__ import annotations

import ctypes
import importlib
import math
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvt.so")
MARSHAL_PATH = os.path.join(_HERE, "_vt_torch.so")

VT_OK = 0
VT_ERR_NULL, VT_ERR_SHAPE, VT_ERR_ALIGN, VT_ERR_RANGE, VT_ERR_DUP = 1, 2, 3, 4, 5
VT_ERR_EMPTY, VT_ERR_WORKSPACE, VT_ERR_TIMEOUT, VT_ERR_CUDA, VT_ERR_UNSUPPORTED = 6, 7, 8, 9, 10
VT_MAX_K = 64
VT_PATH_AUTO, VT_PATH_GEMV, VT_PATH_MMA, VT_PATH_MMA_SMALL = 0, 1, 2, 3
VT_HEAD_STATIC_WEIGHTS, VT_HEAD_D2T_OFFSETS = 0x100, 0x200
VT_ACT_SILU, VT_ACT_GELU = 0, 1
VT_ROPE_NONE, VT_ROPE_LINEAR, VT_ROPE_BASE, VT_ROPE_WAVELENGTH, VT_ROPE_RAMP = 0, 1, 2, 3, 4
VT_ROPE_INTERLEAVED, VT_ROPE_INVERSE = 1, 2

# every symbol include/vt.h declares: name -> (restype, argtypes)
_p, _i, _i64, _sz, _f = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
SYMBOLS = {
    "vt_strerror": (ctypes.c_char_p, [_i]),
    "vt_last_cuda_error": (_i, []),
    "vt_compact_head": (_i, [_p, _i, _i, _p, _i, _p, _p]),
    "vt_coverage_workspace_bytes": (_sz, [_i]),
    "vt_validate_keep_ids": (_i, [_p, _i, _i, _p, _sz, _p]),
    "vt_workspace_bytes": (_sz, [_i, _i]),
    "vt_workspace_init": (_i, [_p, _sz, _p]),
    "vt_draft_head": (_i, [_p, _p, _p, _i, _i, _i, _i, _p, _p, _p, _p, _p, _sz, _p]),
    "vt_draft_head_path": (_i, [_p, _p, _p, _i, _i, _i, _i, _p, _p, _p, _p, _p, _sz, _p, _i]),
    "vt_host_workspace_bytes": (_sz, [_i, _i, _i]),
    "vt_draft_head_host": (_i, [_p, _p, _p, _i, _i, _i, _i, _p, _p, _p, _sz, _p]),
    "vt_last_status": (_i, [_p, _p]),
    "vt_coverage": (_i, [_p, _i64, _p, _i, _i, _p, _p, _p, _sz, _p]),
    "vt_coverage_enqueue": (_i, [_p, _i64, _p, _i, _i, _p, _sz, _p]),
    "vt_coverage_result": (_i, [_p, _i64, _p, _p, _p]),
    "vt_select_workspace_bytes": (_sz, [_i]),
    "vt_select_vocab": (_i, [_p, _i64, _i, _i, ctypes.c_double, ctypes.c_double, ctypes.c_double, _i, _i, _p, _p, _p, _p, _p,
                            _p, _p, _p, _sz, _p]),
    "vt_coverage_static": (_i, [_p, _i64, _p, _i, _i, _p, _p, _p]),
    "vt_debug_logits": (_i, [_p, _p, _i, _i, _i, _p, _p, _sz, _p, _i]),
    "vt_fuse_features": (_i, [_p, _p, _i, _i, _i, _p, _p, _sz, _p]),
    "vt_tree_select": (_i, [_p, _p, _p, _i, _i, _i, _p, _p, _p, _p, _p]),
    "vt_score_workspace_bytes": (_sz, [_i, _i, _i, _i]),
    "vt_score_tokens": (_i, [_p, _i64, _p, _p, _i, _i, _i, _f, _i, _p, _p, _p, _p, _p, _p, _sz, _p]),
    "vt_score_backward_workspace_bytes": (_sz, [_i, _i, _i]),
    "vt_score_tokens_backward": (_i, [_p, _i64, _p, _p, _p, _p, _p, _p, _i, _i, _i, _f, _p, _p, _p, _sz, _p]),
    "vt_gated_ffn_workspace_bytes": (_sz, [_i, _i, _i]),
    "vt_gated_ffn": (_i, [_p, _i64, _p, _p, _p, _i, _i, _i, _i, _p, _p, _p, _sz, _p]),
    "vt_gated_ffn_backward_workspace_bytes": (_sz, [_i, _i, _i]),
    "vt_gated_ffn_backward": (_i, [_p, _i64, _p, _p, _p, _p, _p, _i64, _i, _i, _i, _i, _p, _p, _p, _p, _p, _sz, _p]),
    "vt_rope_table": (_i, [_p, _i, ctypes.c_double, _i, ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_double, _p]),
    "vt_rope": (_i, [_p, _p, _p, _p, _i, _i, _i, _i, _i, _f, _i, _p, _p, _p]),
    "vt_rope_append": (_i, [_p, _p, _p, _p, _p, _p, _i, _i, _i, _f, _i, _p, _p, _p]),
    "vt_tree_attention_workspace_bytes": (_sz, [_i, _i, _i, _i]),
    "vt_tree_attention": (_i, [_p, _p, _p, _p, _i, _i, _i, _i, _f, _p, _p, _p, _sz, _p]),
    "vt_tree_mask": (_i, [_p, _p, _p, _i, _i, _p, _i, _p, _p]),
    "vt_verify_tokens": (_i, [_p, _i64, _p, _p, _p, _p, _p, _p, _i64, _p, _p, _i, _i, _i, _i, _i, _p, _p, _p, _p]),
    "vt_remap": (_i, [_p, _p, _i64, _i, _p, _p]),
    "vt_vocab_maps": (_i, [_p, _i, _i, _p, _p, _p]),
    "vt_last_launch_count": (_i, []),
    "vt_test_timeout_probe": (_i, [_p, _i, _p]),
    "vt_test_late_copy": (_i, [_p, _p, _sz, _i, _p]),
    "vt_test_withhold_copies": (_i, [_i]),
    "vt_test_products": (_i, [_p, _i]),
}

_lib = None
_fast = None         # the compiled marshalling of the decode step's calls (csrc/vt_torch.cpp)


class VtError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = int(status)
        text = lib().vt_strerror(self.status).decode()
        extra = f" (CUDA error {lib().vt_last_cuda_error()})" if self.status == VT_ERR_CUDA else ""
        super().__init__(f"{what}: status {self.status}: {text}{extra}")


def lib() -> ctypes.CDLL:
    """Load ``libvt.so`` from the package directory, building it with nvcc first if it is absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            from .build import build_library
            build_library()
        cd = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SYMBOLS.items():
            fn = getattr(cd, name)     # AttributeError if the library lacks a declared symbol
            fn.restype, fn.argtypes = res, args
        _lib = cd
    return _lib


def _marshal():
    """The compiled marshalling, told where the library's entry points are; built first if it is absent, or was built against another PyTorch."""
    global _fast
    if _fast is None:
        cd = lib()
        from .build import build_marshal
        if not os.path.exists(MARSHAL_PATH):
            build_marshal()
        importlib.invalidate_caches()
        try:
            fast = importlib.import_module("._vt_torch", __package__)
        except ImportError:
            build_marshal(force=True)
            fast = importlib.import_module("._vt_torch", __package__)
        fast.init(*(ctypes.cast(getattr(cd, n), _p).value for n in (
            "vt_rope", "vt_rope_append", "vt_tree_mask", "vt_tree_attention", "vt_tree_attention_workspace_bytes", "vt_verify_tokens")))
        _fast = fast
    return _fast


def _check(status: int, what: str):
    if status != VT_OK:
        raise VtError(status, what)


def _stream() -> int:
    # the handle alone: building a Stream object around it takes longer than a launch's other host work together
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _bf16(t: torch.Tensor, name: str) -> torch.Tensor:
    if t.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
        raise TypeError(f"{name}: expected bf16 data (torch.bfloat16 or a 16-bit integer view), got {t.dtype}")
    if not t.is_cuda or not t.is_contiguous() or t.dim() != 2:
        raise ValueError(f"{name}: expected a contiguous 2-D CUDA tensor")
    return t


def _i32(t: torch.Tensor, name: str) -> torch.Tensor:
    if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous int32 CUDA tensor")
    return t


def _bf16_rows(t: torch.Tensor, name: str) -> torch.Tensor:
    """bf16 rows that may lie further apart than they are long (a slice of a wider buffer)."""
    if t.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
        raise TypeError(f"{name}: expected bf16 data (torch.bfloat16 or a 16-bit integer view), got {t.dtype}")
    if not t.is_cuda or t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{name}: expected a 2-D CUDA tensor with contiguous rows")
    return t


def _ld(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _f32(t: torch.Tensor, name: str, shape: tuple) -> torch.Tensor:
    if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != shape:
        raise ValueError(f"{name}: expected a contiguous float32 CUDA tensor of shape {shape}")
    return t


def _out(t: torch.Tensor | None, name: str, shape: tuple, dtype: torch.dtype, like: torch.Tensor) -> torch.Tensor:
    """An output given by the caller, checked, or a new one on the device of `like` (of its shape and type: the cheapest way)."""
    if t is None:
        if like.dtype == dtype and like.shape == shape and like.is_contiguous():
            return torch.empty_like(like)
        return like.new_empty(shape, dtype=dtype)
    if t.dtype != dtype or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != shape:
        raise ValueError(f"{name}: expected a contiguous {dtype} CUDA tensor of shape {shape}")
    return t


def _scratch(workspace: torch.Tensor | None, nbytes, *sizes, device) -> torch.Tensor:
    """The caller's workspace, which must be on the device, or a new one of nbytes(*sizes)."""
    if workspace is None:
        return torch.empty(max(nbytes(*sizes), 256), dtype=torch.uint8, device=device)
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace: expected a contiguous CUDA tensor")
    return workspace


def vt_workspace_bytes(M: int, k: int) -> int:
    return int(lib().vt_workspace_bytes(M, k))


def vt_host_workspace_bytes(M: int, d: int, k: int) -> int:
    return int(lib().vt_host_workspace_bytes(M, d, k))


def vt_coverage_workspace_bytes(V_full: int) -> int:
    return int(lib().vt_coverage_workspace_bytes(V_full))


def vt_workspace_init(workspace: torch.Tensor) -> torch.Tensor:
    _check(lib().vt_workspace_init(workspace.data_ptr(), workspace.numel(), _stream()), "vt_workspace_init")
    return workspace


def new_workspace(nbytes: int, device=None) -> torch.Tensor:
    """A zero-initialised byte buffer of the caller's (torch's caching allocator is 512-byte aligned)."""
    ws = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device or "cuda")
    return vt_workspace_init(ws)


def vt_compact_head(W_full: torch.Tensor, keep_ids: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    W_full = _bf16(W_full, "W_full")
    keep_ids = _i32(keep_ids, "keep_ids")
    V, d = W_full.shape
    Vt = keep_ids.numel()
    if out is None:
        out = torch.empty((Vt, d), dtype=W_full.dtype, device=W_full.device)
    _check(lib().vt_compact_head(W_full.data_ptr(), V, d, keep_ids.data_ptr(), Vt, out.data_ptr(), _stream()),
           "vt_compact_head")
    return out


def vt_validate_keep_ids(keep_ids: torch.Tensor, V_full: int, workspace: torch.Tensor | None = None) -> int:
    """Returns the status (VT_OK, VT_ERR_RANGE or VT_ERR_DUP) instead of raising for those two."""
    keep_ids = _i32(keep_ids, "keep_ids")
    if workspace is None:
        workspace = torch.empty(vt_coverage_workspace_bytes(V_full), dtype=torch.uint8, device=keep_ids.device)
    st = lib().vt_validate_keep_ids(keep_ids.data_ptr(), keep_ids.numel(), V_full, workspace.data_ptr(),
                                    workspace.numel(), _stream())
    if st not in (VT_OK, VT_ERR_RANGE, VT_ERR_DUP):
        raise VtError(st, "vt_validate_keep_ids")
    return st


def vt_draft_head(h: torch.Tensor, W_trim: torch.Tensor, d2t: torch.Tensor, k: int, *,
                  workspace: torch.Tensor | None = None, path: int = VT_PATH_AUTO,
                  target_ids: torch.Tensor | None = None, logprobs: torch.Tensor | None = None,
                  draft_ids: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                  static_weights: bool = False, d2t_offsets: bool = False):
    """(target_ids [M,k] int32, logprobs [M,k] float32); pass ``draft_ids`` / ``lse`` tensors to receive those too.

    ``static_weights`` sets VT_HEAD_STATIC_WEIGHTS, ``d2t_offsets`` sets VT_HEAD_D2T_OFFSETS (see ``include/vt.h``)."""
    h = _bf16(h, "h")
    W_trim = _bf16(W_trim, "W_trim")
    d2t = _i32(d2t, "d2t")
    M, d = h.shape
    Vt, d2 = W_trim.shape
    if d2 != d or d2t.numel() != Vt:
        raise ValueError("h, W_trim and d2t disagree on d or V_trim")
    if workspace is None:
        workspace = new_workspace(vt_workspace_bytes(M, min(max(k, 1), VT_MAX_K)), h.device)
    if target_ids is None:
        target_ids = torch.empty((M, k), dtype=torch.int32, device=h.device)
    if logprobs is None:
        logprobs = torch.empty((M, k), dtype=torch.float32, device=h.device)
    _check(lib().vt_draft_head_path(h.data_ptr(), W_trim.data_ptr(), d2t.data_ptr(), M, d, Vt, k,
                                    target_ids.data_ptr(), logprobs.data_ptr(), _ptr(draft_ids), _ptr(lse),
                                    workspace.data_ptr(), workspace.numel(), _stream(),
                                    path | (VT_HEAD_STATIC_WEIGHTS if static_weights else 0)
                                    | (VT_HEAD_D2T_OFFSETS if d2t_offsets else 0)), "vt_draft_head")
    return target_ids, logprobs


def vt_draft_head_host(h_host: torch.Tensor, W_trim: torch.Tensor, d2t: torch.Tensor, k: int,
                       target_ids_host: torch.Tensor, logprobs_host: torch.Tensor, workspace: torch.Tensor):
    """Host-buffer form: ``h_host`` and both outputs are CPU tensors (pinned for speed); synchronises."""
    M, d = h_host.shape
    Vt = W_trim.shape[0]
    if h_host.is_cuda or target_ids_host.is_cuda or logprobs_host.is_cuda:
        raise ValueError("vt_draft_head_host takes host tensors for h and the outputs")
    _check(lib().vt_draft_head_host(h_host.data_ptr(), W_trim.data_ptr(), d2t.data_ptr(), M, d, Vt, k,
                                    target_ids_host.data_ptr(), logprobs_host.data_ptr(),
                                    workspace.data_ptr(), workspace.numel(), _stream()), "vt_draft_head_host")
    return target_ids_host, logprobs_host


def vt_last_status(workspace: torch.Tensor) -> int:
    return int(lib().vt_last_status(workspace.data_ptr(), _stream()))


def vt_coverage(token_ids: torch.Tensor, keep_ids: torch.Tensor, V_full: int,
                workspace: torch.Tensor | None = None) -> tuple[int, float]:
    token_ids = _i32(token_ids, "token_ids")
    keep_ids = _i32(keep_ids, "keep_ids")
    if workspace is None:
        workspace = torch.empty(vt_coverage_workspace_bytes(V_full), dtype=torch.uint8, device=keep_ids.device)
    covered = ctypes.c_uint64(0)
    frac = ctypes.c_double(0.0)
    _check(lib().vt_coverage(token_ids.data_ptr() if token_ids.numel() else None, token_ids.numel(),
                             keep_ids.data_ptr(), keep_ids.numel(), V_full,
                             ctypes.addressof(covered), ctypes.addressof(frac),
                             workspace.data_ptr(), workspace.numel(), _stream()), "vt_coverage")
    return int(covered.value), float(frac.value)


def vt_coverage_enqueue(token_ids: torch.Tensor, keep_ids: torch.Tensor, V_full: int, workspace: torch.Tensor) -> None:
    token_ids = _i32(token_ids, "token_ids")
    keep_ids = _i32(keep_ids, "keep_ids")
    _check(lib().vt_coverage_enqueue(token_ids.data_ptr() if token_ids.numel() else None, token_ids.numel(),
                                     keep_ids.data_ptr(), keep_ids.numel(), V_full,
                                     workspace.data_ptr(), workspace.numel(), _stream()), "vt_coverage_enqueue")


def vt_coverage_result(workspace: torch.Tensor, N: int) -> tuple[int, float]:
    covered = ctypes.c_uint64(0)
    frac = ctypes.c_double(0.0)
    _check(lib().vt_coverage_result(workspace.data_ptr(), int(N), ctypes.addressof(covered), ctypes.addressof(frac),
                                    _stream()), "vt_coverage_result")
    return int(covered.value), float(frac.value)


def vt_select_workspace_bytes(V_full: int) -> int:
    return int(lib().vt_select_workspace_bytes(V_full))


def vt_select_vocab(token_ids: torch.Tensor, V_full: int, d: int, F_fixed: float, alpha: float, c_min: float,
                    k_min: int, k_max: int, *, want_cum: bool = False, workspace: torch.Tensor | None = None) -> dict:
    """k* and the frequency ranking (Eq. 1-5).  Returns k_star, C, R, U (at k*), ranked_ids [V_full] and, if asked, cum_counts."""
    token_ids = _i32(token_ids, "token_ids")
    dev = token_ids.device
    ranked = torch.empty(V_full, dtype=torch.int32, device=dev)
    cum = torch.empty(V_full, dtype=torch.int64, device=dev) if want_cum else None
    if workspace is None:
        workspace = torch.empty(vt_select_workspace_bytes(V_full), dtype=torch.uint8, device=dev)
    k_star = ctypes.c_int(0)
    C, R, U, uq = ctypes.c_double(0), ctypes.c_double(0), ctypes.c_double(0), ctypes.c_double(0)
    _check(lib().vt_select_vocab(token_ids.data_ptr() if token_ids.numel() else None, token_ids.numel(), V_full, d,
                                 float(F_fixed), float(alpha), float(c_min), k_min, k_max, ranked.data_ptr(), _ptr(cum),
                                 ctypes.addressof(k_star), ctypes.addressof(C), ctypes.addressof(R), ctypes.addressof(U),
                                 ctypes.addressof(uq), workspace.data_ptr(), workspace.numel(), _stream()), "vt_select_vocab")
    out = {"k_star": int(k_star.value), "C": float(C.value), "R": float(R.value), "U": float(U.value),
           "unique": float(uq.value), "ranked_ids": ranked}
    if want_cum:
        out["cum_counts"] = cum
    return out


def vt_coverage_static(token_ids: torch.Tensor, keep_ids: torch.Tensor, V_full: int) -> tuple[int, float]:
    """``vt_coverage`` without a workspace: the library's built-in scratch is used and nothing is allocated
    here or in the library (for callers that may not allocate; V_full <= 262,144; calls must not overlap)."""
    token_ids = _i32(token_ids, "token_ids")
    keep_ids = _i32(keep_ids, "keep_ids")
    covered = ctypes.c_uint64(0)
    frac = ctypes.c_double(0.0)
    _check(lib().vt_coverage_static(token_ids.data_ptr() if token_ids.numel() else None, token_ids.numel(),
                                    keep_ids.data_ptr(), keep_ids.numel(), V_full,
                                    ctypes.addressof(covered), ctypes.addressof(frac), _stream()),
           "vt_coverage_static")
    return int(covered.value), float(frac.value)


def vt_debug_logits(h: torch.Tensor, W_trim: torch.Tensor, path: int = VT_PATH_AUTO) -> torch.Tensor:
    h = _bf16(h, "h")
    W_trim = _bf16(W_trim, "W_trim")
    M, d = h.shape
    Vt = W_trim.shape[0]
    logits = torch.empty((M, Vt), dtype=torch.float32, device=h.device)
    ws = new_workspace(vt_workspace_bytes(M, 2), h.device)
    _check(lib().vt_debug_logits(h.data_ptr(), W_trim.data_ptr(), M, d, Vt, logits.data_ptr(), ws.data_ptr(),
                                 ws.numel(), _stream(), path), "vt_debug_logits")
    return logits


def vt_fuse_features(h3: torch.Tensor, W_fuse: torch.Tensor, *, out: torch.Tensor | None = None,
                     workspace: torch.Tensor | None = None) -> torch.Tensor:
    """fused [M, d_out] bf16 = h3 [M, d_in] x W_fuse[d_out, d_in]^T, fp32 accumulation, one rounding to bf16."""
    h3 = _bf16(h3, "h3")
    W_fuse = _bf16(W_fuse, "W_fuse")
    M, d_in = h3.shape
    d_out, d2 = W_fuse.shape
    if d2 != d_in:
        raise ValueError("h3 and W_fuse disagree on d_in")
    if out is None:
        out = torch.empty((M, d_out), dtype=h3.dtype, device=h3.device)
    if workspace is None:
        workspace = new_workspace(vt_workspace_bytes(M, 1), h3.device)
    _check(lib().vt_fuse_features(h3.data_ptr(), W_fuse.data_ptr(), M, d_in, d_out, out.data_ptr(), workspace.data_ptr(),
                                  workspace.numel(), _stream()), "vt_fuse_features")
    return out


def vt_tree_select(logprobs: torch.Tensor, target_ids: torch.Tensor, parent_scores: torch.Tensor, T: int):
    """The T best (row, slot) pairs by parent score + log-prob: (rows, slots, tokens, scores), each [T]."""
    M, k = logprobs.shape
    if logprobs.dtype != torch.float32 or parent_scores.dtype != torch.float32 or not logprobs.is_contiguous():
        raise ValueError("logprobs and parent_scores must be contiguous float32 CUDA tensors")
    target_ids = _i32(target_ids, "target_ids")
    dev = logprobs.device
    rows = torch.empty(T, dtype=torch.int32, device=dev)
    slots = torch.empty(T, dtype=torch.int32, device=dev)
    tokens = torch.empty(T, dtype=torch.int32, device=dev)
    scores = torch.empty(T, dtype=torch.float32, device=dev)
    _check(lib().vt_tree_select(logprobs.data_ptr(), target_ids.data_ptr(), parent_scores.data_ptr(), M, k, T,
                                rows.data_ptr(), slots.data_ptr(), tokens.data_ptr(), scores.data_ptr(), _stream()),
           "vt_tree_select")
    return rows, slots, tokens, scores


class VtScores(NamedTuple):
    """What ``vt_score_tokens`` returns: [M] float32 each, and [M, k] for the alternatives (None for k = 0)."""
    logprobs: torch.Tensor | None
    entropy: torch.Tensor
    lse: torch.Tensor
    top_ids: torch.Tensor | None
    top_logprobs: torch.Tensor | None


def vt_score_workspace_bytes(M: int, d: int, V: int, k: int) -> int:
    return int(lib().vt_score_workspace_bytes(M, d, V, k))


def vt_score_backward_workspace_bytes(M: int, d: int, V: int) -> int:
    return int(lib().vt_score_backward_workspace_bytes(M, d, V))


def _score_inputs(h, W, tokens):
    h, W = _bf16_rows(h, "h"), _bf16(W, "W")
    if W.shape[1] != h.shape[1]:
        raise ValueError("h and W disagree on d")
    if tokens is not None and _i32(tokens, "tokens").shape != (h.shape[0],):
        raise ValueError("tokens must hold one id per row of h")
    return h, W


def vt_score_tokens(h: torch.Tensor, W: torch.Tensor, tokens: torch.Tensor | None, *, k: int = 0, scale: float = 1.0,
                    workspace: torch.Tensor | None = None, logprobs: torch.Tensor | None = None,
                    entropy: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                    top_ids: torch.Tensor | None = None, top_logprobs: torch.Tensor | None = None) -> VtScores:
    """Log probabilities of ``tokens`` [M] under the head ``W`` [V, d], with entropy, log-sum-exp and the k best alternatives.

    Rows whose token lies outside [0, V) are not scored (zeros, top_ids -1); ``tokens=None`` scores every row without a
    given token.  Pass tensors for outputs and workspace to have them reused.  A device-side wait that runs out leaves
    invalid results and is only seen by ``vt_last_status`` of a workspace of the caller's (from ``new_workspace``)."""
    h, W = _score_inputs(h, W, tokens)
    (M, d), V, dev = h.shape, W.shape[0], h.device
    if tokens is None and logprobs is not None:
        raise ValueError("logprobs needs tokens")
    if logprobs is None and entropy is None and lse is None and top_ids is None and top_logprobs is None:
        # one allocation cut up: five of them, and checking them, take as long as the call itself
        if k > 0:
            logprobs, entropy, lse, top_ids, top_logprobs = h.new_empty((M * (3 + 2 * k),), dtype=torch.float32).split_with_sizes(
                (M, M, M, M * k, M * k))
            top_ids, top_logprobs = top_ids.view(torch.int32).view(M, k), top_logprobs.view(M, k)
        else:
            logprobs, entropy, lse = h.new_empty((M * 3,), dtype=torch.float32).split_with_sizes((M, M, M))
        if tokens is None:
            logprobs = None
    else:
        logprobs = None if tokens is None else _out(logprobs, "logprobs", (M,), torch.float32, h)
        entropy = _out(entropy, "entropy", (M,), torch.float32, h)
        lse = _out(lse, "lse", (M,), torch.float32, h)
        if k > 0:
            top_ids = _out(top_ids, "top_ids", (M, k), torch.int32, h)
            top_logprobs = _out(top_logprobs, "top_logprobs", (M, k), torch.float32, h)
        else:
            top_ids = top_logprobs = None
    workspace = _scratch(workspace, vt_score_workspace_bytes, M, d, V, k, device=dev)
    _check(lib().vt_score_tokens(h.data_ptr(), _ld(h), W.data_ptr(), _ptr(tokens), M, d, V, scale, k, _ptr(logprobs),
                                 entropy.data_ptr(), lse.data_ptr(), _ptr(top_ids), _ptr(top_logprobs),
                                 workspace.data_ptr(), workspace.nbytes, _stream()), "vt_score_tokens")
    return VtScores(logprobs, entropy, lse, top_ids, top_logprobs)


def vt_score_tokens_backward(h: torch.Tensor, W: torch.Tensor, tokens: torch.Tensor, lse: torch.Tensor,
                             entropy: torch.Tensor | None, grad_logprobs: torch.Tensor,
                             grad_entropy: torch.Tensor | None = None, *, scale: float = 1.0,
                             workspace: torch.Tensor | None = None, grad_h: torch.Tensor | None = None,
                             grad_W: torch.Tensor | None = None, want_h: bool = True, want_W: bool = True):
    """(grad_h [M, d], grad_W [V, d]) in bf16 from the forward call's ``lse`` and ``entropy``; one not wanted is None.

    Time-outs are only seen by ``vt_last_status`` of a workspace of the caller's (from ``new_workspace``)."""
    h, W = _score_inputs(h, W, tokens)
    (M, d), V, dev = h.shape, W.shape[0], h.device
    lse, grad_logprobs = _f32(lse, "lse", (M,)), _f32(grad_logprobs, "grad_logprobs", (M,))
    if grad_entropy is not None:
        if entropy is None:
            raise ValueError("grad_entropy needs the forward call's entropy")
        _f32(entropy, "entropy", (M,)), _f32(grad_entropy, "grad_entropy", (M,))
    grad_h = _out(grad_h, "grad_h", (M, d), torch.bfloat16, h) if want_h else None
    grad_W = _out(grad_W, "grad_W", (V, d), torch.bfloat16, W) if want_W else None
    workspace = _scratch(workspace, vt_score_backward_workspace_bytes, M, d, V, device=dev)
    _check(lib().vt_score_tokens_backward(h.data_ptr(), _ld(h), W.data_ptr(), _ptr(tokens), lse.data_ptr(), _ptr(entropy),
                                          grad_logprobs.data_ptr(), _ptr(grad_entropy), M, d, V, scale, _ptr(grad_h), _ptr(grad_W),
                                          workspace.data_ptr(), workspace.nbytes, _stream()), "vt_score_tokens_backward")
    return grad_h, grad_W


_ACTS = {"silu": VT_ACT_SILU, "gelu": VT_ACT_GELU, VT_ACT_SILU: VT_ACT_SILU, VT_ACT_GELU: VT_ACT_GELU}


def _act(act: str | int) -> int:
    if act not in _ACTS:
        raise ValueError(f"act: expected 'silu' or 'gelu' (or VT_ACT_SILU, VT_ACT_GELU), got {act!r}")
    return _ACTS[act]


def vt_gated_ffn_workspace_bytes(M: int, d: int, f: int) -> int:
    return int(lib().vt_gated_ffn_workspace_bytes(M, d, f))


def vt_gated_ffn_backward_workspace_bytes(M: int, d: int, f: int) -> int:
    return int(lib().vt_gated_ffn_backward_workspace_bytes(M, d, f))


def _ffn_inputs(x, W_gate, W_up, W_down):
    x = _bf16_rows(x, "x")
    _bf16(W_gate, "W_gate"), _bf16(W_up, "W_up"), _bf16(W_down, "W_down")
    d, f = x.shape[1], W_gate.shape[0]
    if W_gate.shape != (f, d) or W_up.shape != (f, d) or W_down.shape != (d, f):
        raise ValueError("x, W_gate, W_up and W_down disagree on d or f")
    return x, d, f


def vt_gated_ffn(x: torch.Tensor, W_gate: torch.Tensor, W_up: torch.Tensor, W_down: torch.Tensor, *, act: str | int = "silu",
                 out: torch.Tensor | None = None, saved: torch.Tensor | None = None,
                 workspace: torch.Tensor | None = None) -> torch.Tensor:
    """y [M, d] bf16 = (act(x W_gate^T) * (x W_up^T)) W_down^T, act "silu" or "gelu" (tanh form).

    Pass ``saved`` [M, 2 f] float32 to receive what ``vt_gated_ffn_backward`` needs (its layout is the library's own).
    Time-outs are only seen by ``vt_last_status`` of a workspace of the caller's (from ``new_workspace``)."""
    x, d, f = _ffn_inputs(x, W_gate, W_up, W_down)
    M = x.shape[0]
    out = _out(out, "out", (M, d), torch.bfloat16, x)
    if saved is not None:
        _f32(saved, "saved", (M, 2 * f))
    workspace = _scratch(workspace, vt_gated_ffn_workspace_bytes, M, d, f, device=x.device)
    _check(lib().vt_gated_ffn(x.data_ptr(), _ld(x), W_gate.data_ptr(), W_up.data_ptr(), W_down.data_ptr(), M, d, f,
                              _act(act), out.data_ptr(), _ptr(saved), workspace.data_ptr(), workspace.nbytes,
                              _stream()), "vt_gated_ffn")
    return out


def vt_gated_ffn_backward(x: torch.Tensor, W_gate: torch.Tensor, W_up: torch.Tensor, W_down: torch.Tensor, saved: torch.Tensor,
                          grad_y: torch.Tensor, *, act: str | int = "silu", workspace: torch.Tensor | None = None,
                          grad_x: torch.Tensor | None = None, grad_W_gate: torch.Tensor | None = None,
                          grad_W_up: torch.Tensor | None = None, grad_W_down: torch.Tensor | None = None):
    """(grad_x [M, d], grad_W_gate [f, d], grad_W_up [f, d], grad_W_down [d, f]) in bf16 from the forward call's ``saved``.

    Time-outs are only seen by ``vt_last_status`` of a workspace of the caller's (from ``new_workspace``)."""
    x, d, f = _ffn_inputs(x, W_gate, W_up, W_down)
    M, dev = x.shape[0], x.device
    _f32(saved, "saved", (M, 2 * f))
    if _bf16_rows(grad_y, "grad_y").shape != (M, d):
        raise ValueError("grad_y must have the shape of x")
    grad_x = _out(grad_x, "grad_x", (M, d), torch.bfloat16, x)
    grad_W_gate = _out(grad_W_gate, "grad_W_gate", (f, d), torch.bfloat16, W_gate)
    grad_W_up = _out(grad_W_up, "grad_W_up", (f, d), torch.bfloat16, W_up)
    grad_W_down = _out(grad_W_down, "grad_W_down", (d, f), torch.bfloat16, W_down)
    workspace = _scratch(workspace, vt_gated_ffn_backward_workspace_bytes, M, d, f, device=dev)
    _check(lib().vt_gated_ffn_backward(x.data_ptr(), _ld(x), W_gate.data_ptr(), W_up.data_ptr(), W_down.data_ptr(), saved.data_ptr(),
                                       grad_y.data_ptr(), _ld(grad_y), M, d, f, _act(act), grad_x.data_ptr(),
                                       grad_W_gate.data_ptr(), grad_W_up.data_ptr(), grad_W_down.data_ptr(), workspace.data_ptr(),
                                       workspace.nbytes, _stream()), "vt_gated_ffn_backward")
    return grad_x, grad_W_gate, grad_W_up, grad_W_down


class _VtHeads(ctypes.Structure):
    """``vt_heads``: a [tokens, heads, D] bf16 tensor."""
    _fields_ = [("ptr", _p), ("token_stride", _i64), ("head_stride", _i64)]


class _VtCacheStruct(ctypes.Structure):
    _fields_ = [("k", _p), ("v", _p), ("page_table", _p), ("lens", _p)] + \
        [(n, _i64) for n in ("k_page_stride", "k_token_stride", "k_head_stride", "v_page_stride", "v_token_stride", "v_head_stride",
                             "table_stride")] + \
        [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "heads", "head_dim", "B", "max_pages")]


class VtRope(NamedTuple):
    """Frequencies and layout of rotary positions, from ``vt_rope_table``."""
    table: torch.Tensor        # [rot_dim / 2] int64: turns per position, as fractions of 2^64
    rot_dim: int
    interleaved: bool
    amplitude: float


_ROPE_SCALINGS = {"none": VT_ROPE_NONE, "linear": VT_ROPE_LINEAR, "base": VT_ROPE_BASE, "wavelength": VT_ROPE_WAVELENGTH, "ramp": VT_ROPE_RAMP}


def vt_rope_table(rot_dim: int, *, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, low: float = 1.0,
                  high: float | None = None, original_len: float = 8192.0, interleaved: bool = False, amplitude: float | None = None,
                  device=None) -> VtRope:
    """The plan of rotary positions over a head's first ``rot_dim`` elements, pairs (i, i + rot_dim / 2) or, ``interleaved``, (2 i, 2 i + 1).

    ``scaling`` stretches positions for contexts longer than ``original_len``: "linear", "base", "wavelength" (``low`` and ``high`` turns,
    1 and 4) or "ramp" (1 and 32; the amplitude is then 0.1 log(factor) + 1, for factors above 1, unless it is given).  Formulas: ``include/vt.h``."""
    if scaling not in _ROPE_SCALINGS:
        raise ValueError(f"scaling: expected one of {', '.join(_ROPE_SCALINGS)}, got {scaling!r}")
    if high is None:
        high = 32.0 if scaling == "ramp" else 4.0
    if amplitude is None:
        amplitude = 0.1 * math.log(factor) + 1.0 if scaling == "ramp" and factor > 1 else 1.0
    table = torch.empty(max(int(rot_dim) // 2, 1), dtype=torch.int64, device=device or "cuda")
    if table.get_device() != torch.cuda.current_device():
        raise ValueError("device: expected the current CUDA device")
    _check(lib().vt_rope_table(table.data_ptr(), rot_dim, base, _ROPE_SCALINGS[scaling], factor, low, high, original_len, _stream()),
           "vt_rope_table")
    return VtRope(table, int(rot_dim), bool(interleaved), float(amplitude))


class VtCache:
    """A paged cache: ``k`` and ``v`` [pages, page_size, heads, D] bf16 (any strides that are multiples of 8, D in a row), ``page_table`` [B, n]
    int32 and ``lens`` [B] int32.  The tensors are the caller's: the table, the lengths and the cache itself may be written between
    calls; for other tensors make another ``VtCache``."""
    __slots__ = ("_k", "_v", "_table", "_lens", "_struct", "_ref", "_device")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor, lens: torch.Tensor):
        for name, t in (("k", k), ("v", v)):
            if t.dtype is not torch.bfloat16:
                raise TypeError(f"{name}: expected torch.bfloat16, got {t.dtype}")
            if t.dim() != 4 or not t.is_cuda or (t.stride(3) != 1 and t.shape[3] > 1) or t.shape != k.shape or t.device != k.device:
                raise ValueError(f"{name}: expected [pages, page_size, heads, D] with D in a row on one CUDA device, both alike")
        B = lens.shape[0] if lens.dim() == 1 else -1
        if lens.dtype is not torch.int32 or B < 1 or not lens.is_contiguous() or lens.device != k.device:
            raise ValueError("lens: expected a contiguous int32 vector on the cache's device")
        if page_table.dtype is not torch.int32 or page_table.dim() != 2 or page_table.shape[0] != B or page_table.device != k.device or \
                (page_table.stride(1) != 1 and page_table.shape[1] > 1):
            raise ValueError("page_table: expected int32 [len(lens), pages] with contiguous rows on the cache's device")
        if page_table.shape[1] < 1 or min(k.shape) < 1:
            raise ValueError("page_table, k: an empty cache")
        self._k, self._v, self._table, self._lens, self._device = k, v, page_table, lens, k.get_device()
        whole = k.numel()

        def strides(t):                # the stride of one alone says nothing
            return [s if n > 1 else (whole + 7) // 8 * 8 for s, n in zip(t.stride()[:3], t.shape)]

        self._struct = _VtCacheStruct(k.data_ptr(), v.data_ptr(), page_table.data_ptr(), lens.data_ptr(), *strides(k), *strides(v),
                                      page_table.stride(0), *k.shape, B, page_table.shape[1])
        self._ref = ctypes.addressof(self._struct)

    k = property(lambda self: self._k)
    v = property(lambda self: self._v)
    page_table = property(lambda self: self._table)
    lens = property(lambda self: self._lens)


def vt_rope(q: torch.Tensor, k: torch.Tensor | None, positions: torch.Tensor, rope: VtRope, *, inverse: bool = False,
            out_q: torch.Tensor | None = None, out_k: torch.Tensor | None = None):
    """(q, k) turned to their ``positions`` [N] int32; q [N, Hq, D], k [N, Hkv, D] or None.

    ``inverse`` turns back, which is the gradient's way: (grad_q, grad_k) = vt_rope(grad of q, grad of k, ..., inverse=True).  The outputs may
    be the inputs themselves."""
    r = (_fast or _marshal()).rope(q, k, positions, rope.table, rope.rot_dim, rope.amplitude,
                                   (VT_ROPE_INTERLEAVED if rope.interleaved else 0) | (VT_ROPE_INVERSE if inverse else 0), out_q, out_k)
    return r if type(r) is tuple else _check(r, "vt_rope")


def vt_rope_append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, cu_tokens: torch.Tensor, cache: VtCache,
                   rope: VtRope, *, out_q: torch.Tensor | None = None) -> torch.Tensor:
    """q [N, Hq, D] turned; k [N, heads, D] turned into the cache and v beside it, at places lens[b], lens[b] + 1, ... of each request.

    Request b has the tokens from ``cu_tokens``[b] to ``cu_tokens``[b + 1]; tokens outside all requests are padding, and left alone."""
    r = (_fast or _marshal()).rope_append(q, k, v, positions, cu_tokens, cache._ref, cache._device, rope.table, rope.rot_dim, rope.amplitude,
                                          VT_ROPE_INTERLEAVED if rope.interleaved else 0, out_q)
    return _check(r, "vt_rope_append") if type(r) is int else r


def vt_tree_mask(parents: torch.Tensor, cu_tokens: torch.Tensor, max_tokens: int, *, lens: torch.Tensor | None = None,
                 mask: torch.Tensor | None = None, positions: torch.Tensor | None = None):
    """(mask [N, ceil(max_tokens / 32)] int32, positions [N] int32) of drafted trees from ``parents`` [N] (index within the request, -1: none).

    A token's row has the bits of the tokens on its way up and its own; its position is lens[b] + its depth (without ``lens`` the depth)."""
    r = (_fast or _marshal()).tree_mask(parents, cu_tokens, (int(max_tokens) + 31) // 32, lens, mask, positions)
    return r if type(r) is tuple else _check(r, "vt_tree_mask")


def vt_tree_attention_workspace_bytes(Hq: int, heads: int, D: int, max_tokens: int) -> int:
    return int(lib().vt_tree_attention_workspace_bytes(Hq, heads, D, max_tokens))


def vt_tree_attention(q: torch.Tensor, cu_tokens: torch.Tensor, cache: VtCache, *, max_tokens: int, mask: torch.Tensor | None = None,
                      scale: float | None = None, out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor]:
    """(out [N, Hq, D] bf16, lse [N, Hq] float32): drafted tokens' attention over the cache, which holds their keys and values at its end.

    ``max_tokens`` bounds the tokens of a request.  ``mask`` [N, words] int32 (``vt_tree_mask``) says which drafted tokens each attends; without
    it a token attends itself and those before it.  ``scale`` is D^-0.5 unless it is given.  Rows outside all requests are left as they were.
    Time-outs and page ids outside the cache are only seen by ``vt_last_status`` of a workspace of the caller's (from ``new_workspace``)."""
    r = (_fast or _marshal()).tree_attention(q, cu_tokens, cache._ref, cache._device, mask, max_tokens, scale, out, lse, workspace)
    return r if type(r) is tuple else _check(r, "vt_tree_attention")


class VtVerified(NamedTuple):
    """What ``vt_verify_tokens`` returns, int32."""
    n_accepted: torch.Tensor   # [B]
    path: torch.Tensor         # [B, max_tokens]: accepted tokens as indices within the request, then -1
    tokens: torch.Tensor       # [B, max_tokens]: the accepted tokens, the one that follows them, then -1


def vt_verify_tokens(probs: torch.Tensor, tokens: torch.Tensor, parents: torch.Tensor, cu_tokens: torch.Tensor, u_accept: torch.Tensor,
                     u_sample: torch.Tensor, *, max_tokens: int, draft_probs: torch.Tensor | None = None,
                     draft_ids: torch.Tensor | None = None, d2t: torch.Tensor | None = None, out: VtVerified | None = None) -> VtVerified:
    """Which drafted tokens stay, given the target's ``probs`` [N, V] after each token and random numbers, and the token that follows them.

    Token 0 of a request is its root.  With ``draft_probs`` [N, Vd] the children of a token were drawn from its row (``draft_ids`` [N]: the tokens
    as draft indices, ``d2t`` [Vd] the draft-to-target map); without them they were picked without chance (``vt_tree_select``).  The result is
    distributed as if the target had generated alone; the rule is spelled out in ``include/vt.h``."""
    n_accepted, path, out_tokens = out or (None, None, None)
    r = (_fast or _marshal()).verify_tokens(probs, tokens, parents, cu_tokens, u_accept, u_sample, max_tokens, draft_probs, draft_ids, d2t,
                                            n_accepted, path, out_tokens)
    return VtVerified(*r) if type(r) is tuple else _check(r, "vt_verify_tokens")


def vt_remap(draft_ids: torch.Tensor, d2t: torch.Tensor) -> torch.Tensor:
    draft_ids = _i32(draft_ids, "draft_ids")
    d2t = _i32(d2t, "d2t")
    out = torch.empty_like(draft_ids)
    _check(lib().vt_remap(draft_ids.data_ptr(), d2t.data_ptr(), draft_ids.numel(), d2t.numel(), out.data_ptr(),
                          _stream()), "vt_remap")
    return out


def vt_vocab_maps(keep_ids: torch.Tensor, V_full: int) -> tuple[torch.Tensor, torch.Tensor]:
    """(d2t offsets [V_trim] int32, t2d membership mask [V_full] uint8) in the form EAGLE-3 checkpoints store."""
    keep_ids = _i32(keep_ids, "keep_ids")
    off = torch.empty_like(keep_ids)
    mask = torch.empty(V_full, dtype=torch.uint8, device=keep_ids.device)
    _check(lib().vt_vocab_maps(keep_ids.data_ptr(), keep_ids.numel(), V_full, off.data_ptr(), mask.data_ptr(), _stream()),
           "vt_vocab_maps")
    return off, mask


def vt_last_launch_count() -> int:
    return int(lib().vt_last_launch_count())


def vt_test_timeout_probe(workspace: torch.Tensor, limit_us: int) -> None:
    _check(lib().vt_test_timeout_probe(workspace.data_ptr(), int(limit_us), _stream()), "vt_test_timeout_probe")


def vt_test_products() -> list[tuple[int, ...]]:
    """(pair, NT, splits, items, at once) of each product this thread launched since the last call; see ``include/vt.h``."""
    rows = (ctypes.c_int * 80)()
    n = lib().vt_test_products(ctypes.addressof(rows), 16)
    return [tuple(rows[5 * i:5 * i + 5]) for i in range(n)]


def vt_test_withhold_copies(limit_us: int) -> None:
    """Products of this thread give up waiting after ``limit_us`` (0: back to normal); see ``include/vt.h``."""
    _check(lib().vt_test_withhold_copies(limit_us), "vt_test_withhold_copies")


def vt_test_late_copy(dst: torch.Tensor, src: torch.Tensor, delay_us: int) -> None:
    n = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != n:
        raise ValueError("dst and src differ in size")
    _check(lib().vt_test_late_copy(dst.data_ptr(), src.data_ptr(), n, int(delay_us), _stream()), "vt_test_late_copy")
