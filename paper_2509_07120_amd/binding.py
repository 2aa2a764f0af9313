"""ctypes binding of libbsga.so: argument marshalling only.

Every function here forwards to the C-ABI entry point of the same name with
device pointers taken from torch tensors and the current torch HIP stream.
Outputs and workspaces are torch tensors (torch is the device allocator and
stream provider, nothing else); all arithmetic happens in the HIP kernels.
There is no fallback path: if the library is missing or a call fails, an
exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from typing import Optional, Tuple

import torch

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libbsga.so")

BSGA_OK = 0
BSGA_ERR_INVALID_ARG = 1
BSGA_ERR_UNSUPPORTED = 2
BSGA_ERR_WORKSPACE = 3
BSGA_ERR_HIP = 4
BSGA_BF16 = 0
BSGA_FP32 = 1
BSGA_E4M3 = 2

EXPORTED_SYMBOLS = (
    "bsga_version",
    "bsga_last_error",
    "bsga_pool_qk",
    "bsga_pool_qk_split",
    "bsga_select_workspace_bytes",
    "bsga_select_blocks",
    "bsga_gather_tokens",
    "bsga_gather_pool",
    "bsga_split_heads",
    "bsga_merge_heads",
    "bsga_attn_workspace_bytes", "bsga_attn_fp32_parts_bytes",
    "bsga_sparse_attn",
    "bsga_sparse_attn_noalloc",
    "bsga_noalloc_scratch_bytes",
    "bsga_sparse_attn_qk",
    "bsga_sparse_attn_split",
    "bsga_dense_attn",
    "bsga_linear",
    "bsga_layer_norm",
    "bsga_probe_mfma",
    "bsga_cache_load",
    "bsga_paged_attn",
    "bsga_paged_attn_e4m3",
    "bsga_paged_attn_e4m3_workspace_bytes",
    "bsga_paged_attn_workspace_bytes",
    "bsga_prefix_attn",
    "bsga_prefix_attn_workspace_bytes",
    "bsga_qk_norm_rope",
    "bsga_qk_norm_rope_e4m3",
    "bsga_qk_norm_rope_bwd",
    "bsga_qk_norm_rope_bwd_workspace_bytes",
    "bsga_window_attn",
    "bsga_window_attn_bwd",
    "bsga_window_attn_bwd_workspace_bytes",
    "bsga_window_attn_workspace_bytes",
)


class BsgaError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"bsga error {code}: {message}")
        self.code = code
        self.message = message


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'` "
            "or `python paper_2509_07120_amd/build.py` first (there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    c_void_p, c_int, c_int64, c_double, c_float, c_size_t = (
        ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_double, ctypes.c_float, ctypes.c_size_t)
    lib.bsga_version.restype = c_int
    lib.bsga_version.argtypes = []
    lib.bsga_last_error.restype = ctypes.c_char_p
    lib.bsga_last_error.argtypes = []
    lib.bsga_pool_qk.restype = c_int
    lib.bsga_pool_qk.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int64, c_int, c_int, c_void_p, c_void_p, c_void_p]
    lib.bsga_pool_qk_split.restype = c_int
    lib.bsga_pool_qk_split.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int64, c_int64, c_int, c_int, c_void_p,
                                       c_void_p, c_void_p]
    lib.bsga_select_blocks.restype = c_int
    lib.bsga_select_blocks.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_double, c_double, c_double,
                                       c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_size_t,
                                       c_void_p]
    lib.bsga_select_workspace_bytes.restype = c_size_t
    lib.bsga_select_workspace_bytes.argtypes = [c_int, c_int, c_int]
    lib.bsga_gather_tokens.restype = c_int
    lib.bsga_gather_tokens.argtypes = [c_void_p, c_int, c_int, c_int64, c_int, c_void_p, c_int64, c_void_p, c_void_p]
    lib.bsga_gather_pool.restype = c_int
    lib.bsga_gather_pool.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int64, c_int, c_void_p, c_int64, c_int64, c_int,
                                     c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.bsga_split_heads.restype = c_int
    lib.bsga_split_heads.argtypes = [c_void_p, c_int, c_int64, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p]
    lib.bsga_merge_heads.restype = c_int
    lib.bsga_merge_heads.argtypes = [c_void_p, c_int, c_int, c_int64, c_int, c_void_p, c_void_p, c_void_p]
    lib.bsga_attn_workspace_bytes.restype = c_size_t
    lib.bsga_attn_workspace_bytes.argtypes = [c_int, c_int, c_int64, c_int]
    lib.bsga_attn_fp32_parts_bytes.restype = c_size_t
    lib.bsga_attn_fp32_parts_bytes.argtypes = [c_int, c_int64, c_int, c_double]
    lib.bsga_sparse_attn.restype = c_int
    lib.bsga_sparse_attn.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int64, c_int, c_int, c_float,
                                     c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.bsga_sparse_attn_noalloc.restype = c_int
    lib.bsga_sparse_attn_noalloc.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int64, c_int, c_int, c_float,
                                             c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p]
    lib.bsga_noalloc_scratch_bytes.restype = c_size_t
    lib.bsga_noalloc_scratch_bytes.argtypes = []
    lib.bsga_sparse_attn_qk.restype = c_int
    lib.bsga_sparse_attn_qk.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int64, c_int, c_int, c_int, c_float,
                                        c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.bsga_sparse_attn_split.restype = c_int
    lib.bsga_sparse_attn_split.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int64, c_int64, c_int, c_int,
                                           c_int, c_float, c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p,
                                           c_size_t, c_void_p]
    lib.bsga_dense_attn.restype = c_int
    lib.bsga_dense_attn.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int64, c_int, c_float,
                                    c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.bsga_linear.restype = c_int
    lib.bsga_linear.argtypes = [c_void_p, c_int, c_void_p, c_void_p, c_int64, c_int, c_int, c_int, c_void_p, c_void_p, c_int,
                                c_void_p, c_void_p]
    lib.bsga_layer_norm.restype = c_int
    lib.bsga_layer_norm.argtypes = [c_void_p, c_void_p, c_void_p, c_double, c_int64, c_int, c_void_p, c_void_p, c_void_p]
    lib.bsga_probe_mfma.restype = c_int
    lib.bsga_probe_mfma.argtypes = [c_int, c_int, c_int, c_void_p, c_size_t, ctypes.POINTER(c_double), c_void_p]
    strides = [c_int64] * 6
    norm = [c_int, c_double, c_void_p, c_void_p]
    lib.bsga_qk_norm_rope.restype = c_int
    lib.bsga_qk_norm_rope.argtypes = [c_void_p] * 3 + strides + [c_int, c_int64, c_int, c_int, c_int] + norm + [c_void_p] * 3 + [
        c_int, c_double, c_void_p, c_int64, c_int] + [c_void_p] * 4
    lib.bsga_qk_norm_rope_bwd.restype = c_int
    lib.bsga_qk_norm_rope_bwd.argtypes = [c_void_p] * 5 + [c_int64] * 4 + [c_int, c_int64, c_int, c_int, c_int] + norm + [
        c_void_p, c_int, c_double] + [c_void_p] * 3 + strides + [c_void_p, c_void_p, c_size_t, c_void_p]
    lib.bsga_qk_norm_rope_bwd_workspace_bytes.restype = c_size_t
    lib.bsga_qk_norm_rope_bwd_workspace_bytes.argtypes = [c_int64, c_int, c_int]
    seen = [c_int64] * 4
    lib.bsga_window_attn.restype = c_int
    lib.bsga_window_attn.argtypes = [c_void_p] * 3 + strides + [c_int, c_int, c_int, c_int64, c_int64, c_int, c_float] + seen + [
        c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.bsga_window_attn_workspace_bytes.restype = c_size_t
    lib.bsga_window_attn_workspace_bytes.argtypes = [c_int, c_int, c_int64, c_int64] + seen
    lib.bsga_window_attn_bwd.restype = c_int
    lib.bsga_window_attn_bwd.argtypes = [c_void_p] * 4 + strides + [c_void_p, c_void_p, c_int, c_int, c_int, c_int64, c_int64, c_int,
                                                                    c_float] + seen + [c_void_p] * 4 + [c_size_t, c_void_p]
    lib.bsga_window_attn_bwd_workspace_bytes.restype = c_size_t
    lib.bsga_window_attn_bwd_workspace_bytes.argtypes = [c_int, c_int, c_int, c_int64, c_int64] + seen
    lib.bsga_paged_attn.restype = c_int
    lib.bsga_paged_attn.argtypes = [c_void_p, c_int64, c_int64, c_void_p, c_void_p, c_int, c_int64, c_int, c_int, c_int, c_void_p, c_int64, c_void_p,
                                    c_int64, c_int, c_float, c_int64, c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.bsga_paged_attn_workspace_bytes.restype = c_size_t
    lib.bsga_paged_attn_workspace_bytes.argtypes = [c_int, c_int64, c_int, c_int, c_int64, c_int64, c_int] + [c_int64] * 3
    lib.bsga_paged_attn_e4m3.restype = c_int
    lib.bsga_paged_attn_e4m3.argtypes = [c_void_p, c_int64, c_int64] + [c_void_p] * 4 + [c_int, c_int64, c_int, c_int, c_int, c_void_p, c_int64, c_void_p,
                                                                                        c_int64, c_int, c_float, c_int64, c_int64, c_int64, c_void_p,
                                                                                        c_void_p, c_void_p, c_size_t, c_void_p]
    lib.bsga_paged_attn_e4m3_workspace_bytes.restype = c_size_t
    lib.bsga_paged_attn_e4m3_workspace_bytes.argtypes = lib.bsga_paged_attn_workspace_bytes.argtypes
    lib.bsga_qk_norm_rope_e4m3.restype = c_int
    lib.bsga_qk_norm_rope_e4m3.argtypes = [c_void_p] * 3 + strides + [c_int, c_int64, c_int, c_int, c_int] + norm + [c_void_p] * 3 + [
        c_int, c_double, c_void_p, c_int64, c_int] + [c_void_p] * 8
    lib.bsga_cache_load.restype = c_int
    lib.bsga_cache_load.argtypes = [c_void_p] * 4 + [c_int, c_int64, c_int, c_int, c_int, c_void_p, c_int64, c_int64, c_int64, c_int, c_void_p, c_void_p,
                                                     c_int64, c_int64, c_void_p]
    lib.bsga_prefix_attn.restype = c_int
    lib.bsga_prefix_attn.argtypes = [c_void_p, c_int64, c_int64] + [c_void_p] * 4 + [
        c_int, c_int, c_int64, c_int, c_int, c_int, c_void_p, c_int64, c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_int64, c_int64, c_int, c_float,
        c_int64, c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.bsga_prefix_attn_workspace_bytes.restype = c_size_t
    lib.bsga_prefix_attn_workspace_bytes.argtypes = [c_int, c_int, c_int64, c_int, c_int, c_int64, c_int64, c_int64, c_int64, c_int] + [c_int64] * 3
    return lib


lib = _load()


def _check(rc: int) -> None:
    if rc != BSGA_OK:
        raise BsgaError(rc, lib.bsga_last_error().decode())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# The current stream's handle without a Stream object around it (0.2 us instead of 1.9), where torch has it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t: torch.Tensor) -> int:
    if _raw_stream is not None:
        return _raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BSGA_BF16
    if t.dtype == torch.float32:
        return BSGA_FP32
    raise TypeError(f"unsupported dtype {t.dtype}: bsga takes bfloat16 or float32")


def _require(t: torch.Tensor, name: str, dtype=None) -> None:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")


def num_blocks(n_tokens: int, block: int) -> int:
    return (n_tokens + block - 1) // block


def bsga_pool_qk(q: torch.Tensor, k: torch.Tensor, block: int,
                 out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """q, k [H, N, 64] -> (q_pool, k_pool) [H, ceil(N/block), 64] float64 (written into `out` if given)."""
    _require(q, "q"); _require(k, "k", q.dtype)
    if q.shape != k.shape or q.dim() != 3:
        raise ValueError("q and k must both be [heads, n_tokens, head_dim]")
    H, N, d = q.shape
    nb = num_blocks(N, block)
    if out is None:
        q_pool = torch.empty((H, nb, d), dtype=torch.float64, device=q.device)
        k_pool = torch.empty_like(q_pool)
    else:
        q_pool, k_pool = out
        for t in (q_pool, k_pool):
            _require(t, "out", torch.float64)
            if tuple(t.shape) != (H, nb, d):
                raise ValueError(f"out tensors must be {(H, nb, d)}")
    _check(lib.bsga_pool_qk(_ptr(q), _ptr(k), _dtype_code(q), H, N, d, block, _ptr(q_pool), _ptr(k_pool), _stream(q)))
    return q_pool, k_pool


def split_blocks(n_tokens: int, n_first: int, block: int) -> int:
    """Blocks of a sequence whose parts [0, n_first) and [n_first, n_tokens) are blocked separately."""
    return num_blocks(n_first, block) + num_blocks(n_tokens - n_first, block)


def bsga_pool_qk_split(q: torch.Tensor, k: torch.Tensor, block: int, n_first: int,
                       out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """As bsga_pool_qk for a sequence split at token n_first: no block crosses n_first."""
    _require(q, "q"); _require(k, "k", q.dtype)
    if q.shape != k.shape or q.dim() != 3:
        raise ValueError("q and k must both be [heads, n_tokens, head_dim]")
    H, N, d = q.shape
    nb = split_blocks(N, n_first, block) if 0 <= n_first <= N else 1
    if out is None:
        q_pool = torch.empty((H, nb, d), dtype=torch.float64, device=q.device)
        k_pool = torch.empty_like(q_pool)
    else:
        q_pool, k_pool = out
        for t in (q_pool, k_pool):
            _require(t, "out", torch.float64)
            if tuple(t.shape) != (H, nb, d):
                raise ValueError(f"out tensors must be {(H, nb, d)}")
    _check(lib.bsga_pool_qk_split(_ptr(q), _ptr(k), _dtype_code(q), H, N, n_first, d, block, _ptr(q_pool),
                                  _ptr(k_pool), _stream(q)))
    return q_pool, k_pool


def bsga_pool(x: torch.Tensor, block: int) -> torch.Tensor:
    """x [H, N, 64] -> block means [H, ceil(N/block), 64] float64 (one tensor; for separate q / k block sizes)."""
    _require(x, "x")
    H, N, d = x.shape
    pooled = torch.empty((H, num_blocks(N, block), d), dtype=torch.float64, device=x.device)
    _check(lib.bsga_pool_qk(_ptr(x), None, _dtype_code(x), H, N, d, block, _ptr(pooled), None, _stream(x)))
    return pooled


def bsga_select_blocks(q_pool: torch.Tensor, k_pool: torch.Tensor, tau: float, rho: float = 1.0,
                       score_scale: Optional[float] = None, force_q: Optional[torch.Tensor] = None,
                       force_k: Optional[torch.Tensor] = None, want_bits: bool = True,
                       workspace: Optional[torch.Tensor] = None, out=None):
    """Pooled Q/K -> (mask_bits [H,nbq,ceil(nbk/32)] uint32-as-int32, kv_idx [H,nbq,nbk] int32, kv_cnt [H,nbq] int32).
    `workspace`: optional device byte buffer of bsga_select_workspace_bytes(H, nbq, nbk) bytes (allocated if absent).
    `out`: optional (mask_bits or None, kv_idx, kv_cnt) tensors of those shapes to write into."""
    _require(q_pool, "q_pool", torch.float64); _require(k_pool, "k_pool", torch.float64)
    H, nbq, d = q_pool.shape
    nbk = k_pool.shape[1]
    if score_scale is None:
        score_scale = 1.0 / math.sqrt(d)
    dev = q_pool.device
    words = (nbk + 31) // 32
    if out is None:
        # every word of every row is written by the kernel, so nothing needs to be cleared
        mask_bits = torch.empty((H, nbq, words), dtype=torch.int32, device=dev) if want_bits else None
        kv_idx = torch.empty((H, nbq, nbk), dtype=torch.int32, device=dev)
        kv_cnt = torch.empty((H, nbq), dtype=torch.int32, device=dev)
    else:
        mask_bits, kv_idx, kv_cnt = out
        for t, shape, name in ((mask_bits, (H, nbq, words), "mask_bits"), (kv_idx, (H, nbq, nbk), "kv_idx"),
                               (kv_cnt, (H, nbq), "kv_cnt")):
            if t is None and name == "mask_bits":
                continue
            _require(t, name, torch.int32)
            if tuple(t.shape) != shape:
                raise ValueError(f"{name} must be {shape}, got {tuple(t.shape)}")
    if force_q is not None:
        _require(force_q, "force_q", torch.uint8)
    if force_k is not None:
        _require(force_k, "force_k", torch.uint8)
    if workspace is None:
        workspace = torch.empty(bsga_select_workspace_bytes(H, nbq, nbk), dtype=torch.uint8, device=dev)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib.bsga_select_blocks(_ptr(q_pool), _ptr(k_pool), H, nbq, nbk, d, float(score_scale), float(tau),
                                  float(rho), _ptr(force_q), _ptr(force_k), _ptr(mask_bits), _ptr(kv_idx),
                                  _ptr(kv_cnt), nbk, _ptr(workspace), ws_bytes, _stream(q_pool)))
    return mask_bits, kv_idx, kv_cnt


def bsga_select_workspace_bytes(heads: int, nb_q: int, nb_k: int) -> int:
    return int(lib.bsga_select_workspace_bytes(heads, nb_q, nb_k))


def bsga_attn_workspace_bytes(dtype: torch.dtype, heads: int, n_tokens: int, head_dim: int = 64) -> int:
    code = BSGA_BF16 if dtype == torch.bfloat16 else BSGA_FP32
    return int(lib.bsga_attn_workspace_bytes(code, heads, n_tokens, head_dim))


def bsga_attn_fp32_parts_bytes(heads: int, n_tokens: int, head_dim: int = 64, kept: float = 1.0) -> int:
    return int(lib.bsga_attn_fp32_parts_bytes(heads, n_tokens, head_dim, float(kept)))


def _attn_bytes(code: int, heads: int, n_tokens: int, head_dim: int, kept: float) -> int:
    """Workspace that an attention call makes use of; `kept`: the share of the key blocks it is expected to keep."""
    if code == BSGA_FP32:
        return lib.bsga_attn_fp32_parts_bytes(heads, n_tokens, head_dim, kept)
    return lib.bsga_attn_workspace_bytes(code, heads, n_tokens, head_dim)


def _workspace(q: torch.Tensor, workspace: Optional[torch.Tensor], kept: float = 0.1) -> Tuple[Optional[torch.Tensor], int]:
    H, N, d = q.shape
    need = _attn_bytes(_dtype_code(q), H, N, d, kept) if workspace is None else 0
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    return workspace, nbytes


def bsga_sparse_attn(q, k, v, block: int, kv_idx: torch.Tensor, kv_cnt: torch.Tensor,
                     softmax_scale: Optional[float] = None, return_lse: bool = False,
                     out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                     ordered: bool = True, block_k: Optional[int] = None):
    """Attention of each query block over its kept key blocks; returns O (and lse).
    ordered = False passes no workspace: rows are launched in index order, not heaviest first.
    block_k: size of the key blocks the lists refer to when it differs from the query block size."""
    _require(q, "q"); _require(k, "k", q.dtype); _require(v, "v", q.dtype)
    _require(kv_idx, "kv_idx", torch.int32); _require(kv_cnt, "kv_cnt", torch.int32)
    H, N, d = q.shape
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(d)
    if out is None:
        out = torch.empty_like(q)
    lse = torch.empty((H, N), dtype=torch.float32, device=q.device) if return_lse else None
    workspace, ws_bytes = _workspace(q, workspace) if ordered else (None, 0)
    if block_k is None or block_k == block:
        _check(lib.bsga_sparse_attn(_ptr(q), _ptr(k), _ptr(v), _dtype_code(q), H, N, d, block, float(softmax_scale),
                                    _ptr(kv_idx), _ptr(kv_cnt), kv_idx.shape[-1], _ptr(out), _ptr(lse),
                                    _ptr(workspace), ws_bytes, _stream(q)))
    else:
        _check(lib.bsga_sparse_attn_qk(_ptr(q), _ptr(k), _ptr(v), _dtype_code(q), H, N, d, block, block_k,
                                       float(softmax_scale), _ptr(kv_idx), _ptr(kv_cnt), kv_idx.shape[-1], _ptr(out),
                                       _ptr(lse), _ptr(workspace), ws_bytes, _stream(q)))
    return (out, lse) if return_lse else out


def bsga_noalloc_scratch_bytes() -> int:
    return int(lib.bsga_noalloc_scratch_bytes())


def bsga_sparse_attn_noalloc(q, k, v, block: int, kv_idx: torch.Tensor, kv_cnt: torch.Tensor, out: torch.Tensor,
                             softmax_scale: Optional[float] = None, lse: Optional[torch.Tensor] = None):
    """bsga_sparse_attn on the library's built-in scratch: nothing is allocated here either (the
    caller passes `out`, and `lse` [H, N] float32 if wanted)."""
    _require(q, "q"); _require(k, "k", q.dtype); _require(v, "v", q.dtype); _require(out, "out", q.dtype)
    _require(kv_idx, "kv_idx", torch.int32); _require(kv_cnt, "kv_cnt", torch.int32)
    H, N, d = q.shape
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(d)
    _check(lib.bsga_sparse_attn_noalloc(_ptr(q), _ptr(k), _ptr(v), _dtype_code(q), H, N, d, block, float(softmax_scale),
                                        _ptr(kv_idx), _ptr(kv_cnt), kv_idx.shape[-1], _ptr(out), _ptr(lse), _stream(q)))
    return out


def bsga_sparse_attn_split(q, k, v, block: int, n_first: int, kv_idx: torch.Tensor, kv_cnt: torch.Tensor,
                           softmax_scale: Optional[float] = None, return_lse: bool = False,
                           out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                           block_k: Optional[int] = None):
    """As bsga_sparse_attn for a sequence split at token n_first (blocks as in bsga_pool_qk_split)."""
    _require(q, "q"); _require(k, "k", q.dtype); _require(v, "v", q.dtype)
    _require(kv_idx, "kv_idx", torch.int32); _require(kv_cnt, "kv_cnt", torch.int32)
    H, N, d = q.shape
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(d)
    if out is None:
        out = torch.empty_like(q)
    lse = torch.empty((H, N), dtype=torch.float32, device=q.device) if return_lse else None
    workspace, ws_bytes = _workspace(q, workspace)
    _check(lib.bsga_sparse_attn_split(_ptr(q), _ptr(k), _ptr(v), _dtype_code(q), H, N, n_first, d, block,
                                      block if block_k is None else block_k, float(softmax_scale), _ptr(kv_idx),
                                      _ptr(kv_cnt), kv_idx.shape[-1], _ptr(out), _ptr(lse), _ptr(workspace), ws_bytes,
                                      _stream(q)))
    return (out, lse) if return_lse else out


def bsga_dense_attn(q, k, v, softmax_scale: Optional[float] = None, return_lse: bool = False,
                    out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                    balanced: bool = True):
    """Dense softmax attention baseline; returns O (and lse).
    balanced = False passes no workspace: every row is then computed by the workgroup of its number
    instead of the last rows being handed out at run time."""
    _require(q, "q"); _require(k, "k", q.dtype); _require(v, "v", q.dtype)
    H, N, d = q.shape
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(d)
    if out is None:
        out = torch.empty_like(q)
    lse = torch.empty((H, N), dtype=torch.float32, device=q.device) if return_lse else None
    workspace, ws_bytes = _workspace(q, workspace, kept=1.0) if balanced else (None, 0)
    _check(lib.bsga_dense_attn(_ptr(q), _ptr(k), _ptr(v), _dtype_code(q), H, N, d, float(softmax_scale),
                               _ptr(out), _ptr(lse), _ptr(workspace), ws_bytes, _stream(q)))
    return (out, lse) if return_lse else out


def sparse_global_attention(q, k, v, block: int, tau: float, rho: float = 1.0,
                            score_scale: Optional[float] = None, softmax_scale: Optional[float] = None,
                            workspace: Optional[torch.Tensor] = None):
    """The whole layer: pool -> select -> block-sparse attention.  Returns (O, kv_idx, kv_cnt, mask_bits).

    A layer of one frame is bound by the host (40 us a pass when each stage was called by its own function),
    so the inputs are checked once and everything that does not outlive the call is one allocation: the pooled
    vectors, then the selection's logits, whose place the attention's workspace takes (the stages are ordered
    by the stream).  The logits of a long sequence are allocated apart and freed before the output is, so that the
    peak is the larger of the two (762 and 640 MB at 300 frames)."""
    _require(q, "q"); _require(k, "k", q.dtype); _require(v, "v", q.dtype)
    if q.shape != k.shape or q.dim() != 3:
        raise ValueError("q and k must both be [heads, n_tokens, head_dim]")
    H, N, d = q.shape
    dev, code, stream = q.device, _dtype_code(q), _stream(q)
    if block not in (64, 128) or d != 64:  # let the library say what is wrong
        bsga_pool_qk(q, k, block)
    nb = num_blocks(N, block)
    pool_bytes = H * nb * d * 8
    select_bytes = lib.bsga_select_workspace_bytes(H, nb, nb)
    # rows keep about tau of their blocks where the map is flat, and the top-k floor at least
    own = _attn_bytes(code, H, N, d, max(min(float(tau), 1.0), 1.0 - float(rho))) if workspace is None else 0
    together = max(select_bytes, own) <= 1 << 20
    scratch = torch.empty(2 * pool_bytes + (max(select_bytes, own) if together else 0), dtype=torch.uint8, device=dev)
    q_pool = scratch.data_ptr()
    k_pool = q_pool + pool_bytes
    logits = None if together else torch.empty(select_bytes, dtype=torch.uint8, device=dev)
    rest = k_pool + pool_bytes if together else logits.data_ptr()
    qp, kp = q.data_ptr(), k.data_ptr()
    _check(lib.bsga_pool_qk(qp, kp, code, H, N, d, block, q_pool, k_pool, stream))
    mask_bits = torch.empty((H, nb, (nb + 31) // 32), dtype=torch.int32, device=dev)
    kv_idx = torch.empty((H, nb, nb), dtype=torch.int32, device=dev)
    kv_cnt = torch.empty((H, nb), dtype=torch.int32, device=dev)
    scale = 1.0 / math.sqrt(d)
    idx, cnt = kv_idx.data_ptr(), kv_cnt.data_ptr()
    _check(lib.bsga_select_blocks(q_pool, k_pool, H, nb, nb, d, scale if score_scale is None else float(score_scale),
                                  float(tau), float(rho),
                                  None, None, mask_bits.data_ptr(), idx, cnt, nb, rest, select_bytes, stream))
    del logits
    out = torch.empty_like(q)
    if workspace is None and not together and own > 0:
        workspace = torch.empty(own, dtype=torch.uint8, device=dev)
    if workspace is None:
        ws, ws_bytes = (rest, own) if own > 0 else (None, 0)
    else:
        ws, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(lib.bsga_sparse_attn(qp, kp, v.data_ptr(), code, H, N, d, block,
                                scale if softmax_scale is None else float(softmax_scale), idx, cnt, nb, out.data_ptr(), None, ws,
                                ws_bytes, stream))
    return out, kv_idx, kv_cnt, mask_bits


def bsga_gather_tokens(x: torch.Tensor, index: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """out[h, i] = x[h, index[i]] for x [H, N, 64] and an int32 device index [n_out]."""
    _require(x, "x"); _require(index, "index", torch.int32)
    H, N, d = x.shape
    n_out = index.numel()
    if out is None:
        out = torch.empty((H, n_out, d), dtype=x.dtype, device=x.device)
    _check(lib.bsga_gather_tokens(_ptr(x), _dtype_code(x), H, N, d, _ptr(index), n_out, _ptr(out), _stream(x)))
    return out


def _require_order(index: Optional[torch.Tensor], x: torch.Tensor, n_tokens: int) -> None:
    if index is None:
        return
    _require(index, "index", torch.int32)
    if index.device != x.device:
        raise ValueError("index must be on the same device as x")
    if index.numel() != n_tokens:
        raise ValueError("index must have one entry per token")


def bsga_split_heads(x: torch.Tensor, parts: int, heads: int, index: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [N, parts * heads * 64] -> [parts, heads, N, 64], token i taken from row index[i] if an index is given."""
    _require(x, "x")
    N = x.shape[0]
    if x.dim() != 2 or x.shape[1] != parts * heads * 64:
        raise ValueError("x must be [n_tokens, parts * heads * 64]")
    _require_order(index, x, N)
    out = torch.empty((parts, heads, N, 64), dtype=x.dtype, device=x.device)
    _check(lib.bsga_split_heads(_ptr(x), _dtype_code(x), N, parts, heads, 64, _ptr(index), _ptr(out), _stream(x)))
    return out


def bsga_merge_heads(x: torch.Tensor, index: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [heads, N, 64] -> [N, heads * 64], row i taken from token index[i] if an index is given."""
    _require(x, "x")
    H, N, d = x.shape
    _require_order(index, x, N)
    out = torch.empty((N, H * d), dtype=x.dtype, device=x.device)
    _check(lib.bsga_merge_heads(_ptr(x), _dtype_code(x), H, N, d, _ptr(index), _ptr(out), _stream(x)))
    return out


def _require_beside(x: torch.Tensor, **others: Optional[torch.Tensor]) -> None:
    at = x.get_device()
    for name, t in others.items():
        if t is not None and t.get_device() != at:
            raise ValueError(f"{name} must be on the same device as x")


def bsga_layer_norm(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor, eps: float = 1e-5,
                    index: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Layer norm of x [N, D] (bfloat16, D a multiple of 8 up to 4096), row i of the result from row index[i] if an index is given."""
    _require(x, "x", torch.bfloat16); _require(weight, "weight", torch.bfloat16); _require(bias, "bias", torch.bfloat16)
    if x.dim() != 2 or tuple(weight.shape) != (x.shape[1],) or tuple(bias.shape) != (x.shape[1],):
        raise ValueError("x must be [n_tokens, features], weight and bias [features]")
    _require_beside(x, weight=weight, bias=bias)
    N, D = x.shape
    _require_order(index, x, N)
    out = torch.empty_like(x)
    _check(lib.bsga_layer_norm(_ptr(x), _ptr(weight), _ptr(bias), float(eps), N, D, _ptr(index), _ptr(out), _stream(x)))
    return out


def bsga_linear(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor, gelu: bool = False,
                residual: Optional[torch.Tensor] = None, row_index: Optional[torch.Tensor] = None,
                out_heads: bool = False) -> torch.Tensor:
    """weight x + bias in bfloat16 with its neighbours folded in (features are multiples of 64).  x is [N, K], or [K/64, N, 64]
    as the attention returns it.  gelu: applied to the fp32 sums; large calls round them to bf16 first, so a row's bits depend on how many
    tokens the call has.  row_index, residual: row i of the result is row row_index[i] of
    the output (a permutation) and has that row of the residual added.  out_heads: the output is [F/64, N, 64], not [N, F]."""
    _require(x, "x", torch.bfloat16); _require(weight, "weight", torch.bfloat16); _require(bias, "bias", torch.bfloat16)
    F_out, K = weight.shape
    heads = x.dim() == 3
    N = x.shape[1] if heads else x.shape[0]
    if tuple(x.shape) != ((K // 64, N, 64) if heads else (N, K)) or tuple(bias.shape) != (F_out,):
        raise ValueError("x must be [n_tokens, in_features] or [in_features / 64, n_tokens, 64], bias [out_features]")
    _require_order(row_index, x, N)
    if residual is not None:
        _require(residual, "residual", torch.bfloat16)
        if tuple(residual.shape) != (N, F_out):
            raise ValueError("residual must be [n_tokens, out_features]")
    _require_beside(x, weight=weight, bias=bias, residual=residual)
    out = torch.empty((F_out // 64, N, 64) if out_heads else (N, F_out), dtype=x.dtype, device=x.device)
    _check(lib.bsga_linear(_ptr(x), int(heads), _ptr(weight), _ptr(bias), N, K, F_out, int(gelu), _ptr(row_index),
                           _ptr(residual), int(out_heads), _ptr(out), _stream(x)))
    return out


class SpecialTokenPlan:
    """Index bookkeeping for the special-token split (Sec. 4.2), built once per sequence layout.

    The working order puts the patch tokens X_p first (in their original order) and the special
    tokens X_s last, and the two parts are blocked separately (the *_split entry points with
    n_first = N_p): blocks 0 .. n_patch_blocks-1, n_patch_blocks = ceil(N_p / block), hold every patch
    token and nothing else (the last of them may be ragged); they are the blocks the map is predicted
    on.  The blocks after them hold the special tokens, which attend and are attended densely:
    force_q = 1, force_k = 2 (kept, not ranked)."""

    def __init__(self, special: torch.Tensor, block: int, device):
        special = torch.as_tensor(special, dtype=torch.bool).cpu()
        n = special.numel()
        order = torch.cat([torch.nonzero(~special).flatten(), torch.nonzero(special).flatten()])
        inverse = torch.empty_like(order)
        inverse[order] = torch.arange(n)
        self.n_tokens = n
        self.block = block
        self.n_patch = int((~special).sum())
        self.n_patch_blocks = num_blocks(self.n_patch, block)
        nb = split_blocks(n, self.n_patch, block)
        self.n_blocks = nb
        dense = torch.arange(nb) >= self.n_patch_blocks
        self.perm = order.to(torch.int32).to(device)
        self.inverse = inverse.to(torch.int32).to(device)
        self.force_q = dense.to(torch.uint8).to(device)
        self.force_k = (dense.to(torch.uint8) * 2).to(device)


def _gather_pool(q, k, v, plan: SpecialTokenPlan):
    """q, k, v in working order and the pooled q and k of that."""
    perm, n = plan.perm, plan.perm.numel()
    alike = all(x.is_cuda and x.is_contiguous() and x.shape == q.shape and x.dtype == q.dtype and x.device == perm.device for x in (q, k, v))
    if not alike or q.dim() != 3 or q.shape[2] != 64 or q.shape[0] < 1 or q.shape[1] < 1 or n < 1:  # let the single steps say what is wrong
        qw, kw, vw = (bsga_gather_tokens(x, perm) for x in (q, k, v))
        return (qw, kw, vw) + bsga_pool_qk_split(qw, kw, plan.block, plan.n_patch)
    _require(perm, "index", torch.int32)
    H = q.shape[0]
    qw, kw, vw = (torch.empty((H, n, 64), dtype=q.dtype, device=q.device) for _ in range(3))
    nb = split_blocks(n, plan.n_patch, plan.block)
    q_pool, k_pool = (torch.empty((H, nb, 64), dtype=torch.float64, device=q.device) for _ in range(2))
    _check(lib.bsga_gather_pool(_ptr(q), _ptr(k), _ptr(v), _dtype_code(q), H, q.shape[1], 64, _ptr(perm), n, plan.n_patch, plan.block,
                                _ptr(qw), _ptr(kw), _ptr(vw), _ptr(q_pool), _ptr(k_pool), _stream(q)))
    return qw, kw, vw, q_pool, k_pool


def sparse_global_attention_special(q, k, v, plan: SpecialTokenPlan, tau: float, rho: float = 1.0,
                                    score_scale: Optional[float] = None, softmax_scale: Optional[float] = None):
    """The layer with the special-token split: gather into the working order, pool, select on the
    patch blocks only, block-sparse attention, gather back.  Returns (O in the caller's token order,
    kv_idx, kv_cnt, mask_bits); the lists refer to blocks of the working order."""
    qw, kw, vw, q_pool, k_pool = _gather_pool(q, k, v, plan)
    mask_bits, kv_idx, kv_cnt = bsga_select_blocks(q_pool, k_pool, tau, rho, score_scale, force_q=plan.force_q,
                                                   force_k=plan.force_k)
    ow = bsga_sparse_attn_split(qw, kw, vw, plan.block, plan.n_patch, kv_idx, kv_cnt, softmax_scale)
    return bsga_gather_tokens(ow, plan.inverse), kv_idx, kv_cnt, mask_bits


def bsga_probe_mfma(operands: int, softmax_mix: int, iters: int = 20000, repeats: int = 3) -> float:
    """Sustained TFLOP/s of the attention kernels' MFMA instruction with no memory traffic (see
    bsga_probe_mfma in the header).  Times `repeats` launches with events and returns the best."""
    dev = torch.device("cuda", torch.cuda.current_device())
    sink = torch.empty(2 * torch.cuda.get_device_properties(dev).multi_processor_count * 256, dtype=torch.float32, device=dev)
    flops = ctypes.c_double(0.0)
    stream = torch.cuda.current_stream(dev).cuda_stream
    best = 0.0
    for r in range(repeats + 1):  # the first launch is a warm-up
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        _check(lib.bsga_probe_mfma(int(operands), int(softmax_mix), int(iters), _ptr(sink), sink.numel() * 4,
                                   ctypes.byref(flops), stream))
        e1.record()
        torch.cuda.synchronize(dev)
        if r > 0:
            best = max(best, flops.value / (e0.elapsed_time(e1) * 1e-3) / 1e12)
    return best


NORMS = {None: 0, "none": 0, "rms": 1, "layer": 2}


def _wrong(t: torch.Tensor, name: str, dtype, at: int, beside: str) -> None:
    """Says what is wrong with a tensor that is not a contiguous one of this type on this device."""
    _require(t, name, dtype)
    if t.get_device() != at:
        raise ValueError(f"{name} must be on the same device as {beside}")


# (calls on few rows are bound by the host: one condition for what is right, and the words for what is not elsewhere)
def _rows(t: torch.Tensor, name: str, dtype, at: int, n_tokens: int, heads: Optional[int] = None) -> Tuple[int, int, int, int]:
    """Strides of the tokens and the heads of t [n_tokens, heads, d], whose rows are contiguous, the heads and d."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.get_device() != at:
        raise ValueError(f"{name} must be on the same device as the other tensors")
    shape = t.shape
    if len(shape) != 3 or shape[0] != n_tokens or (heads is not None and shape[1] != heads):
        raise ValueError(f"{name} must be [n_tokens, heads, 64] with as many tokens and heads as the tensors beside it, got {tuple(shape)}")
    st, sh, one = t.stride()
    if one != 1 and shape[2] > 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    return st, sh, shape[1], shape[2]


def _norm_weight(t: Optional[torch.Tensor], name: str, dtype, at: int, d: int) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or t.dtype != dtype or t.get_device() != at or not t.is_contiguous():
        _wrong(t, name, dtype, at, "the tensors")
    if t.numel() != d:
        raise ValueError(f"{name} must be [{d}]")
    return t.data_ptr()


def _norm_positions(positions: Optional[torch.Tensor], at: int, n_tokens: int) -> Tuple[Optional[int], int]:
    """Address and number of axes."""
    if positions is None:
        return None, 0
    if not positions.is_cuda or positions.dtype != torch.int32 or positions.get_device() != at or not positions.is_contiguous():
        _wrong(positions, "positions", torch.int32, at, "the tensors")
    shape = positions.shape
    if len(shape) not in (1, 2) or shape[0] != n_tokens:
        raise ValueError("positions must be [n_tokens] or [n_tokens, axes]")
    return positions.data_ptr(), 1 if len(shape) == 1 else shape[1]


def _norm_code(norm: Optional[str]) -> int:
    code = NORMS.get(norm, -1)
    if code < 0:
        raise ValueError(f"norm must be 'rms', 'layer' or None, got {norm!r}")
    return code


def bsga_qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: Optional[torch.Tensor] = None,
                      q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                      q_bias: Optional[torch.Tensor] = None, k_bias: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
                      norm: Optional[str] = "rms", eps: float = 1e-6, base: float = 10000.0, k_cache: Optional[torch.Tensor] = None,
                      v_cache: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None):
    """q [N, H, 64], k and v [N, Hkv, 64] (views of a projection's output are fine) -> (q [H, N, 64], k [Hkv, N, 64], v or None): queries
    and keys normed for each head ("rms", "layer" with weight and bias, or None) and turned by their position, v moved along.
    positions: int32 [N] or [N, 1] turn the pairs (j, j + 32) of a row by position * base^(-j/32); [N, 2] the pairs (j, j + 16) of
    its halves by the first and the second position.
    With slots (int32 [N]) keys and values go to these tokens of the caches [pages, Hkv, page, 64] instead (those outside are not
    written), and the caches are returned in their place."""
    dtype, at, N = q.dtype, q.get_device(), q.shape[0]
    code = _dtype_code(q)
    qt, qh, H, d = _rows(q, "q", dtype, at, N)
    kt, kh, K, kd = _rows(k, "k", dtype, at, N)
    vt, vh, _, vd = (0, 0, K, d) if v is None else _rows(v, "v", dtype, at, N, K)
    if kd != d or vd != d:
        raise ValueError("q, k and v must have the same head dimension")
    kind = _norm_code(norm)
    qw, kw = _norm_weight(q_weight, "q_weight", dtype, at, d), _norm_weight(k_weight, "k_weight", dtype, at, d)
    qb, kb = _norm_weight(q_bias, "q_bias", dtype, at, d), _norm_weight(k_bias, "k_bias", dtype, at, d)
    where, axes = _norm_positions(positions, at, N)
    q_out = q.new_empty((H, N, d))
    pages = page = 0
    slot = None
    if slots is None:
        if k_cache is not None or v_cache is not None:
            raise ValueError("caches go with slots")
        k_out = q.new_empty((K, N, d))
        v_out = None if v is None else q.new_empty((K, N, d))
    else:
        if not slots.is_cuda or slots.dtype != torch.int32 or slots.get_device() != at or not slots.is_contiguous():
            _wrong(slots, "slots", torch.int32, at, "the tensors")
        if slots.numel() != N:
            raise ValueError("slots must have one entry per token")
        if k_cache is None or (v is None) != (v_cache is None):
            raise ValueError("slots need the cache of the keys, and of the values with v")
        shape = k_cache.shape
        for name, t in (("k_cache", k_cache), ("v_cache", v_cache)):
            if t is not None:
                if not t.is_cuda or t.dtype != dtype or t.get_device() != at or not t.is_contiguous():
                    _wrong(t, name, dtype, at, "the tensors")
                if len(shape) != 4 or t.shape != shape or shape[1] != K or shape[3] != d:
                    raise ValueError(f"{name} must be [pages, kv_heads, page, 64]")
        pages, page = shape[0], shape[2]
        k_out, v_out, slot = k_cache, v_cache, slots.data_ptr()
    _check(lib.bsga_qk_norm_rope(q.data_ptr(), k.data_ptr(), _ptr(v), qt, qh, kt, kh, vt, vh, code, N, H, K, d, kind, eps, qw, qb, kw, kb, where, axes,
                                 base, slot, pages, page, q_out.data_ptr(), k_out.data_ptr(), _ptr(v_out), _stream(q)))
    return q_out, k_out, v_out


def bsga_qk_norm_rope_bwd(dq: torch.Tensor, dk: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                          positions: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
                          k_weight: Optional[torch.Tensor] = None, q_bias: Optional[torch.Tensor] = None,
                          k_bias: Optional[torch.Tensor] = None, dv: Optional[torch.Tensor] = None, norm: Optional[str] = "rms",
                          eps: float = 1e-6, base: float = 10000.0):
    """Gradient of bsga_qk_norm_rope (without slots): dq [H, N, 64], dk and dv [Hkv, N, 64] are the gradients of its outputs, the
    rest is what it was given (the biases say only whether their gradients are wanted).  Returns the gradients of (q, k, v, q_weight, k_weight,
    q_bias, k_bias), None for what was not given; those of q, k and v lie beside each other in one [N, H + 2 Hkv, 64] (without dv
    [N, H + Hkv, 64]), as a projection's output does, those of weights and biases are float32."""
    dtype, at, N = q.dtype, q.get_device(), q.shape[0]
    code = _dtype_code(q)
    qt, qh, H, d = _rows(q, "q", dtype, at, N)
    kt, kh, K, kd = _rows(k, "k", dtype, at, N)
    if kd != d:
        raise ValueError("q and k must have the same head dimension")
    for name, t, h in (("dq", dq, H), ("dk", dk, K), ("dv", dv, K)):
        if t is not None:
            if not t.is_cuda or t.dtype != dtype or t.get_device() != at or not t.is_contiguous():
                _wrong(t, name, dtype, at, "q")
            if t.shape != (h, N, d):
                raise ValueError(f"{name} must be {(h, N, d)}")
    kind = _norm_code(norm)
    qw, kw = _norm_weight(q_weight, "q_weight", dtype, at, d), _norm_weight(k_weight, "k_weight", dtype, at, d)
    _norm_weight(q_bias, "q_bias", dtype, at, d), _norm_weight(k_bias, "k_bias", dtype, at, d)
    where, axes = _norm_positions(positions, at, N)
    parts = (H, K) if dv is None else (H, K, K)
    dx = q.new_empty((N, sum(parts), d))
    row, size = dx.stride(0), dx.element_size() * d
    into = dx.data_ptr()  # (0 without tokens)
    wanted = q_weight is not None or k_weight is not None or q_bias is not None or k_bias is not None
    dw = work = None
    nbytes = 0
    if wanted:
        nbytes = lib.bsga_qk_norm_rope_bwd_workspace_bytes(N, H, K)
        dw = q.new_empty((4, d), dtype=torch.float32)  # of q's weight and bias, then of k's
        work = q.new_empty(nbytes, dtype=torch.uint8)
    _check(lib.bsga_qk_norm_rope_bwd(dq.data_ptr(), dk.data_ptr(), _ptr(dv), q.data_ptr(), k.data_ptr(), qt, qh, kt, kh, code, N, H, K, d, kind, eps, qw,
                                     kw, where, axes, base, into, into and into + H * size, None if dv is None else into and into + (H + K) * size, row, d, row,
                                     d, row, d,
                                     _ptr(dw), _ptr(work), nbytes, _stream(q)))
    dq_in, dk_in, *rest = dx.split(parts, 1)
    of = dw.unbind(0) if wanted else (None,) * 4
    return (dq_in, dk_in, None if dv is None else rest[0], None if q_weight is None else of[0], None if k_weight is None else of[2],
            None if q_bias is None else of[1], None if k_bias is None else of[3])


def _head_rows(t: torch.Tensor, name: str, like: torch.Tensor) -> Tuple[int, int]:
    """Strides of the tokens and the heads of t [heads, n_tokens, 64], whose rows are contiguous."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != like.dtype:
        raise TypeError(f"{name} must be {like.dtype}, got {t.dtype}")
    if t.get_device() != like.get_device():
        raise ValueError(f"{name} must be on the same device as q")
    strides = t.stride()
    if len(strides) != 3 or (strides[2] != 1 and t.shape[2] > 1):
        raise ValueError(f"{name} must be [heads, n_tokens, 64] with contiguous rows")
    return strides[1], strides[0]


def _window_args(q, k, v, window, sinks, frame, q_start, softmax_scale):
    """What both directions of the attention with a window check: strides, sizes and (q_start, frame, window, sinks)."""
    qs, ks, vs = _head_rows(q, "q", q), _head_rows(k, "k", q), _head_rows(v, "v", q)
    H, N, d = q.shape
    K, M, kd = k.shape
    if k.shape != v.shape or kd != d:
        raise ValueError("k and v must both be [kv_heads, n_k, head_dim]")
    if window is not None and window < 1:
        raise ValueError(f"window must be at least one frame, or None, got {window}")
    seen = (M - N if q_start is None else q_start, frame, 0 if window is None else window, sinks)
    scale = 1.0 / math.sqrt(d) if softmax_scale is None else float(softmax_scale)
    return qs + ks + vs, H, K, N, M, d, seen, scale


def bsga_window_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, window: Optional[int] = None, sinks: int = 0, frame: int = 1,
                     q_start: Optional[int] = None, softmax_scale: Optional[float] = None, return_lse: bool = False,
                     out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Attention of q [H, N, 64] over k, v [Hkv, M, 64] (views with contiguous rows are fine; H a multiple of Hkv) with a sliding window:
    the query at position p sees the keys of its own frame of `frame` tokens and of the window - 1 frames before it, and the first
    `sinks` tokens, never a later frame.  window = None: no limit.  q_start: position of the first query, by default M - N (the queries
    are the last tokens).  A query that sees nothing yields zeros and lse -inf.  Returns O [H, N, 64] (and lse [H, N] float32)."""
    code = _dtype_code(q)
    strides, H, K, N, M, d, seen, scale = _window_args(q, k, v, window, sinks, frame, q_start, softmax_scale)
    if out is None:
        out = q.new_empty((H, N, d))
    else:
        _require(out, "out", q.dtype)
        if tuple(out.shape) != (H, N, d) or out.get_device() != q.get_device():
            raise ValueError(f"out must be {(H, N, d)} on the same device as q")
    lse = q.new_empty((H, N), dtype=torch.float32) if return_lse else None
    if workspace is None:
        nbytes = lib.bsga_window_attn_workspace_bytes(code, H, N, M, *seen)
        if nbytes > 0:
            workspace = q.new_empty(nbytes, dtype=torch.uint8)
    else:
        nbytes = workspace.numel() * workspace.element_size()
    _check(lib.bsga_window_attn(_ptr(q), _ptr(k), _ptr(v), *strides, code, H, K, N, M, d, scale, *seen, _ptr(out), _ptr(lse),
                                _ptr(workspace), nbytes, _stream(q)))
    return (out, lse) if return_lse else out


def bsga_window_attn_bwd(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                         window: Optional[int] = None, sinks: int = 0, frame: int = 1, q_start: Optional[int] = None,
                         softmax_scale: Optional[float] = None, workspace: Optional[torch.Tensor] = None):
    """Gradients (dq [H, N, 64], dk and dv [Hkv, M, 64]) of bsga_window_attn: dout is that of its output, out and lse are what it returned for
    q, k, v and the same window."""
    code = _dtype_code(q)
    strides, H, K, N, M, d, seen, scale = _window_args(q, k, v, window, sinks, frame, q_start, softmax_scale)
    at = q.get_device()
    for name, t, dtype, shape in (("dout", dout, q.dtype, (H, N, d)), ("out", out, q.dtype, (H, N, d)), ("lse", lse, torch.float32, (H, N))):
        if not t.is_cuda or t.dtype != dtype or t.get_device() != at or not t.is_contiguous():
            _wrong(t, name, dtype, at, "q")
        if t.shape != shape:
            raise ValueError(f"{name} must be {shape}")
    dq, dk, dv = q.new_empty((H, N, d)), q.new_empty((K, M, d)), q.new_empty((K, M, d))
    if workspace is None:
        nbytes = lib.bsga_window_attn_bwd_workspace_bytes(code, H, K, N, M, *seen)
        workspace = q.new_empty(nbytes, dtype=torch.uint8) if nbytes > 0 else None
    else:
        nbytes = workspace.numel() * workspace.element_size()
    _check(lib.bsga_window_attn_bwd(_ptr(dout), _ptr(q), _ptr(k), _ptr(v), *strides, _ptr(out), _ptr(lse), code, H, K, N, M, d, scale, *seen,
                                    _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace), nbytes, _stream(q)))
    return dq, dk, dv


def bsga_paged_attn(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor,
                    window: Optional[int] = None, sinks: int = 0, frame: int = 1, softmax_scale: Optional[float] = None,
                    return_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """Attention of one new token for each sequence, q [B, H, 64] (a view with contiguous rows is fine), over the caches [pages, Hkv, page, 64]:
    key j of sequence b lies in row j % page of page page_table[b, j // page] (int32 [B, width]; entries are clamped to the pages there are).
    The query of sequence b stands at position lengths[b] - 1 (int32 [B]), its own key is in the cache already; it sees what
    bsga_window_attn's rule gives a query there (its own frame up to itself: later tokens are not there).  Returns O [B, H, 64] (and lse [B, H] float32); a sequence of length 0 yields zeros and -inf."""
    code = _dtype_code(q)
    if not q.is_cuda:
        raise ValueError("q must be a device tensor")
    strides = q.stride()
    if len(strides) != 3 or (strides[2] != 1 and q.shape[2] > 1):
        raise ValueError("q must be [batch, heads, 64] with contiguous rows")
    B, H, d = q.shape
    at = q.get_device()
    dtype, shape = q.dtype, k_cache.shape
    for name, t in (("k_cache", k_cache), ("v_cache", v_cache)):
        if not t.is_cuda or t.dtype != dtype or t.get_device() != at or not t.is_contiguous():
            _wrong(t, name, dtype, at, "q")
        if len(shape) != 4 or t.shape != shape or shape[3] != d:
            raise ValueError(f"{name} must be [pages, kv_heads, page, 64]")
    for name, t, dims in (("page_table", page_table, 2), ("lengths", lengths, 1)):
        if not t.is_cuda or t.dtype != torch.int32 or t.get_device() != at or not t.is_contiguous():
            _wrong(t, name, torch.int32, at, "q")
        if len(t.shape) != dims or t.shape[0] != B:
            raise ValueError(f"{name} must have a row for each sequence")
    if window is not None and window < 1:
        raise ValueError(f"window must be at least one frame, or None, got {window}")
    pages, K, page, _ = shape
    width = page_table.shape[1]
    seen = (frame, 0 if window is None else window, sinks)
    out = q.new_empty((B, H, d))
    lse = q.new_empty((B, H), dtype=torch.float32) if return_lse else None
    if workspace is None:
        nbytes = lib.bsga_paged_attn_workspace_bytes(code, B, H, K, width, pages, page, *seen)
        if nbytes > 0:
            workspace = q.new_empty(nbytes, dtype=torch.uint8)
    else:
        nbytes = workspace.numel() * workspace.element_size()
    _check(lib.bsga_paged_attn(_ptr(q), strides[0], strides[1], _ptr(k_cache), _ptr(v_cache), code, B, H, K, d, _ptr(page_table), width,
                               _ptr(lengths), pages, page, 1.0 / math.sqrt(d) if softmax_scale is None else float(softmax_scale), *seen,
                               _ptr(out), _ptr(lse), _ptr(workspace), nbytes, _stream(q)))
    return (out, lse) if return_lse else out


# (steps of a few sequences are bound by the host: one condition for what is right, and the words for what is not in a function of their own)
def _wrong_cache(name: str, t: torch.Tensor, dtype, at: int) -> None:
    if not t.is_cuda or t.dtype != dtype or t.get_device() != at or not t.is_contiguous():
        _wrong(t, name, dtype, at, "the tensors")
    raise ValueError(f"{name} must be [pages, kv_heads, page, 64]")


def _wrong_scale(name: str, t: Optional[torch.Tensor], at: int) -> None:
    if t is None:
        raise ValueError(f"a cache in 8 bits needs {name}")
    if not t.is_cuda or t.dtype != torch.uint8 or t.get_device() != at or not t.is_contiguous():
        _wrong(t, name, torch.uint8, at, "the tensors")
    raise ValueError(f"{name} must be [pages, kv_heads, page]")


def _cache_of(k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: Optional[torch.Tensor], v_scale: Optional[torch.Tensor], dtype, at: int, d: int,
              heads: Optional[int] = None):
    """Checks caches of this type, or in 8 bits with their scales, on device `at`: their type's code, pages, heads and page."""
    shape = k_cache.shape
    coded = k_cache.dtype is torch.float8_e4m3fn
    kind = torch.float8_e4m3fn if coded else dtype
    if len(shape) != 4 or k_cache.dtype is not kind or k_cache.get_device() != at or at < 0 or not k_cache.is_contiguous() or shape[3] != d or (
            heads is not None and shape[1] != heads):
        _wrong_cache("k_cache", k_cache, kind, at)
    if v_cache.dtype is not kind or v_cache.get_device() != at or not v_cache.is_contiguous() or v_cache.shape != shape:
        _wrong_cache("v_cache", v_cache, kind, at)
    pages, heads, page, _ = shape
    if coded:
        want = shape[:3]
        if k_scale is None or k_scale.dtype is not torch.uint8 or k_scale.get_device() != at or not k_scale.is_contiguous() or k_scale.shape != want:
            _wrong_scale("k_scale", k_scale, at)
        if v_scale is None or v_scale.dtype is not torch.uint8 or v_scale.get_device() != at or not v_scale.is_contiguous() or v_scale.shape != want:
            _wrong_scale("v_scale", v_scale, at)
        return BSGA_E4M3, pages, heads, page
    if k_scale is not None or v_scale is not None:
        raise ValueError("scales go with caches of torch.float8_e4m3fn")
    return _dtype_code(k_cache), pages, heads, page


def bsga_qk_norm_rope_e4m3(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                           k_scale: torch.Tensor, v_scale: torch.Tensor, slots: torch.Tensor, positions: Optional[torch.Tensor] = None,
                           q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, q_bias: Optional[torch.Tensor] = None,
                           k_bias: Optional[torch.Tensor] = None, norm: Optional[str] = "rms", eps: float = 1e-6, base: float = 10000.0,
                           return_rows: bool = False):
    """bsga_qk_norm_rope with slots, into caches in 8 bits: k_cache, v_cache [pages, Hkv, page, 64] of torch.float8_e4m3fn, k_scale, v_scale [pages, Hkv, page]
    uint8; a row stands for its numbers times 2^(scale - 127).  q [N, H, 64] or None, k and v [N, Hkv, 64], slots int32 [N], the rest as there.
    Returns (q [H, N, 64] or None, k, v): with return_rows the rows [Hkv, N, 64] as the caches hold them, of the tensors' type, else None."""
    dtype, at, N = k.dtype, k.get_device(), k.shape[0]
    code = _dtype_code(k)
    kt, kh, K, d = _rows(k, "k", dtype, at, N)
    qt, qh, H, qd = (0, 0, K, d) if q is None else _rows(q, "q", dtype, at, N)
    vt, vh, _, vd = _rows(v, "v", dtype, at, N, K)
    if qd != d or vd != d:
        raise ValueError("q, k and v must have the same head dimension")
    kind = _norm_code(norm)
    qw, kw = _norm_weight(q_weight, "q_weight", dtype, at, d), _norm_weight(k_weight, "k_weight", dtype, at, d)
    qb, kb = _norm_weight(q_bias, "q_bias", dtype, at, d), _norm_weight(k_bias, "k_bias", dtype, at, d)
    where, axes = _norm_positions(positions, at, N)
    if not slots.is_cuda or slots.dtype != torch.int32 or slots.get_device() != at or not slots.is_contiguous():
        _wrong(slots, "slots", torch.int32, at, "the tensors")
    if slots.numel() != N:
        raise ValueError("slots must have one entry per token")
    _, pages, _, page = _cache_of(k_cache, v_cache, k_scale, v_scale, torch.float8_e4m3fn, at, d, K)
    q_out = None if q is None else q.new_empty((H, N, d))
    k_rows = v_rows = None
    if return_rows:
        k_rows, v_rows = k.new_empty((K, N, d)), k.new_empty((K, N, d))
    _check(lib.bsga_qk_norm_rope_e4m3(_ptr(q), k.data_ptr(), v.data_ptr(), qt, qh, kt, kh, vt, vh, code, N, H, K, d, kind, eps, qw, qb, kw, kb, where, axes, base,
                                      slots.data_ptr(), pages, page, _ptr(q_out), _ptr(k_rows), _ptr(v_rows), k_cache.data_ptr(),
                                      v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), _stream_here(k)))
    return q_out, k_rows, v_rows


def bsga_cache_load(k_cache: torch.Tensor, v_cache: torch.Tensor, pages: torch.Tensor, n_tokens: int, first: int = 0,
                    k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None,
                    out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Tokens [first, first + n_tokens) of one sequence out of the caches [pages, Hkv, page, 64]: (k, v) [Hkv, n_tokens, 64].  pages (int32 [width]) is the
    sequence's row of a page table; tokens whose page does not exist are zeros.  Caches of torch.float8_e4m3fn come with their scales and are read as
    `dtype` (bfloat16 unless said otherwise), others as they are.  out: where to, each head's tokens one after the other (heads may be further apart)."""
    coded = k_cache.dtype == torch.float8_e4m3fn
    if out is not None:
        dtype = out[0].dtype if dtype is None else dtype
    if dtype is None:
        dtype = torch.bfloat16 if coded else k_cache.dtype
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype {dtype}: bsga takes bfloat16 or float32")
    at, d = k_cache.get_device(), 64
    if not coded and k_cache.dtype != dtype:
        raise TypeError(f"a cache that is not in 8 bits is read as it is, got {k_cache.dtype} and {dtype}")
    code, n_pages, K, page = _cache_of(k_cache, v_cache, k_scale, v_scale, dtype, at, d)
    if not pages.is_cuda or pages.dtype != torch.int32 or pages.get_device() != at or not pages.is_contiguous():
        _wrong(pages, "pages", torch.int32, at, "the caches")
    if pages.dim() != 1:
        raise ValueError("pages must be one sequence's row of a page table")
    if out is None:
        shape = (K, max(n_tokens, 0), d)
        k, v = k_cache.new_empty(shape, dtype=dtype), k_cache.new_empty(shape, dtype=dtype)
    else:
        k, v = out
        for name, t in (("out[0]", k), ("out[1]", v)):
            if t.dtype != dtype:
                raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
            if not t.is_cuda or t.get_device() != at:
                raise ValueError(f"{name} must be on the same device as the caches")
            if t.shape != (K, n_tokens, d) or (n_tokens > 0 and (t.stride(2) != 1 or (n_tokens > 1 and t.stride(1) != d))):
                raise ValueError(f"{name} must be {(K, n_tokens, d)}, each head's tokens one after the other")
    _check(lib.bsga_cache_load(_ptr(k_cache), _ptr(v_cache), _ptr(k_scale), _ptr(v_scale), code, n_pages, page, K, d, _ptr(pages), pages.shape[0], first,
                               n_tokens, BSGA_BF16 if dtype == torch.bfloat16 else BSGA_FP32, _ptr(k), _ptr(v), k.stride(0), v.stride(0), _stream_here(k_cache)))
    return k, v


# Kernels go to the current device's default stream where its handle is 0: tensors of another device would be read from there.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream_here(t: torch.Tensor) -> int:
    """The current stream of t's device, which must be the current one."""
    if t.get_device() != _current_device():
        raise ValueError(f"the tensors must be on the current device, got {t.device} (use torch.cuda.device)")
    return _stream(t)


def _scratch(workspace: torch.Tensor, at: int) -> int:
    """Bytes of a caller's workspace on device `at`."""
    if not workspace.is_cuda or workspace.get_device() != at or not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous and on the tensors' device")
    return workspace.numel() * workspace.element_size()


# (what a step's sizes ask for is the same from step to step)
@functools.lru_cache(maxsize=1024)
def _paged_bytes(*sizes: int) -> int:
    return lib.bsga_paged_attn_e4m3_workspace_bytes(*sizes)


@functools.lru_cache(maxsize=1024)
def _prefix_bytes(*sizes: int) -> int:
    return lib.bsga_prefix_attn_workspace_bytes(*sizes)


def _queries(q: torch.Tensor) -> Tuple[int, int]:
    """Strides of the sequences and heads of q [batch, heads, 64], whose rows are contiguous."""
    if not q.is_cuda:
        raise ValueError("q must be a device tensor")
    strides = q.stride()
    if len(strides) != 3 or (strides[2] != 1 and q.shape[2] > 1):
        raise ValueError("q must be [batch, heads, 64] with contiguous rows")
    return strides[0], strides[1]


def _numbers(name: str, t: torch.Tensor, at: int, n: int) -> int:
    """The address of an int32 tensor [n]."""
    if t.dtype is not torch.int32 or t.get_device() != at or not t.is_contiguous() or t.dim() != 1 or t.shape[0] != n:
        if not t.is_cuda or t.dtype != torch.int32 or t.get_device() != at or not t.is_contiguous():
            _wrong(t, name, torch.int32, at, "q")
        raise ValueError(f"{name} must be [{n}], got {tuple(t.shape)}")
    return t.data_ptr()


def _table(name: str, t: torch.Tensor, at: int, rows: Optional[int]) -> Tuple[int, int, int]:
    """The address, rows and width of an int32 tensor [rows, width]."""
    shape = t.shape
    if t.dtype is not torch.int32 or t.get_device() != at or not t.is_contiguous() or len(shape) != 2 or (rows is not None and shape[0] != rows):
        if not t.is_cuda or t.dtype != torch.int32 or t.get_device() != at or not t.is_contiguous():
            _wrong(t, name, torch.int32, at, "q")
        raise ValueError(f"{name} must be [{'any' if rows is None else rows}, width], got {tuple(shape)}")
    return t.data_ptr(), shape[0], shape[1]


def bsga_paged_attn_e4m3(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
                         page_table: torch.Tensor, lengths: torch.Tensor, window: Optional[int] = None, sinks: int = 0, frame: int = 1,
                         softmax_scale: Optional[float] = None, return_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """bsga_paged_attn over caches in 8 bits, as bsga_qk_norm_rope_e4m3 writes them: k_cache, v_cache [pages, Hkv, page, 64] of torch.float8_e4m3fn, k_scale,
    v_scale [pages, Hkv, page] uint8.  q and the result are bfloat16 or float32."""
    code = _dtype_code(q)
    strides = _queries(q)
    B, H, d = q.shape
    at = q.get_device()
    _, pages, K, page = _cache_of(k_cache, v_cache, k_scale, v_scale, torch.float8_e4m3fn, at, d)
    table, _, width = _table("page_table", page_table, at, B)
    many = _numbers("lengths", lengths, at, B)
    if window is not None and window < 1:
        raise ValueError(f"window must be at least one frame, or None, got {window}")
    seen = (frame, 0 if window is None else window, sinks)
    out = q.new_empty((B, H, d))
    lse = q.new_empty((B, H), dtype=torch.float32) if return_lse else None
    if workspace is None:
        nbytes = _paged_bytes(code, B, H, K, width, pages, page, *seen)
        if nbytes > 0:
            workspace = q.new_empty(nbytes, dtype=torch.uint8)
    else:
        nbytes = _scratch(workspace, at)
    _check(lib.bsga_paged_attn_e4m3(q.data_ptr(), *strides, k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), code, B, H, K, d, table,
                                    width, many, pages, page, 1.0 / math.sqrt(d) if softmax_scale is None else float(softmax_scale), *seen, out.data_ptr(),
                                    _ptr(lse), _ptr(workspace), nbytes, _stream_here(q)))
    return (out, lse) if return_lse else out


def bsga_prefix_attn(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor,
                     prefix_table: torch.Tensor, prefix_lengths: torch.Tensor, starts: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                     v_scale: Optional[torch.Tensor] = None, window: Optional[int] = None, sinks: int = 0, frame: int = 1,
                     softmax_scale: Optional[float] = None, return_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """bsga_paged_attn (or bsga_paged_attn_e4m3, with scales) where sequences begin with tokens that they share, which are read once for all: sequences
    starts[g] to starts[g + 1] - 1 (int32 [G + 1], not decreasing) see the prefix_lengths[g] (int32 [G]) tokens in the pages prefix_table[g] (int32 [G, prefix
    width]) and then the lengths[b] tokens of their own in the pages page_table[b]; sequences outside have none.  The query stands at the last of its tokens, and window,
    sinks and frame go by positions from the prefix's first token on.  Returns O [B, H, 64] (and lse [B, H] float32); a sequence without any token yields zeros and -inf."""
    code = _dtype_code(q)
    strides = _queries(q)
    B, H, d = q.shape
    at = q.get_device()
    kind, pages, K, page = _cache_of(k_cache, v_cache, k_scale, v_scale, q.dtype, at, d)
    table, _, width = _table("page_table", page_table, at, B)
    many = _numbers("lengths", lengths, at, B)
    prefix, G, prefix_width = _table("prefix_table", prefix_table, at, None)
    long, begin = _numbers("prefix_lengths", prefix_lengths, at, G), _numbers("starts", starts, at, G + 1)
    if window is not None and window < 1:
        raise ValueError(f"window must be at least one frame, or None, got {window}")
    seen = (frame, 0 if window is None else window, sinks)
    out = q.new_empty((B, H, d))
    lse = q.new_empty((B, H), dtype=torch.float32) if return_lse else None
    if workspace is None:
        nbytes = _prefix_bytes(code, kind, B, H, K, width, G, prefix_width, pages, page, *seen)
        if nbytes > 0:
            workspace = q.new_empty(nbytes, dtype=torch.uint8)
    else:
        nbytes = _scratch(workspace, at)
    _check(lib.bsga_prefix_attn(q.data_ptr(), *strides, k_cache.data_ptr(), v_cache.data_ptr(), _ptr(k_scale), _ptr(v_scale), code, kind, B, H, K, d, table, width,
                                many, prefix, prefix_width, long, begin, G, pages, page, 1.0 / math.sqrt(d) if softmax_scale is None else float(softmax_scale),
                                *seen, out.data_ptr(), _ptr(lse), _ptr(workspace), nbytes, _stream_here(q)))
    return (out, lse) if return_lse else out
