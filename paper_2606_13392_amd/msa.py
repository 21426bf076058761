"""Python binding of libmsa.so (argument marshalling only).

Each function checks dtypes, shapes and devices, takes device pointers and the
current torch stream, and calls the C ABI of ``include/msa.h`` under the same
name.  All work runs in the library's HIP kernels; there is no fallback: when
the library is not built, or a call returns an error, a RuntimeError is raised.
torch provides device memory (outputs, workspaces) and the stream.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional, Sequence

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmsa.so")

MSA_OK, MSA_ERR_INVALID, MSA_ERR_UNSUPPORTED, MSA_ERR_WORKSPACE, MSA_ERR_HIP = 0, -1, -2, -3, -4

EXPORTS = [
    "msa_strerror",
    "msa_index_topk_workspace_size", "msa_index_topk", "msa_index_topk_noalloc", "msa_block_topk",
    "msa_sparse_attn_prefill_workspace_size", "msa_sparse_attn_prefill",
    "msa_sparse_attn_decode_workspace_size", "msa_sparse_attn_decode",
    "msa_sparse_attn_prefill_fp8", "msa_sparse_attn_decode_fp8",
    "msa_dense_attn_workspace_size", "msa_dense_attn",
    "msa_dense_attn_paged_workspace_size", "msa_dense_attn_paged", "msa_dense_attn_paged_fp8",
    "msa_qk_norm_rope", "msa_qk_norm_rope_fp8",
    "msa_qk_norm_rope_backward_workspace_size", "msa_qk_norm_rope_backward",
    "msa_kv_append", "msa_kv_append_fp8",
    "msa_latent_append", "msa_latent_append_fp8",
    "msa_latent_attn_paged_workspace_size", "msa_latent_attn_paged", "msa_latent_attn_paged_fp8",
    "msa_latent_attn_workspace_size", "msa_latent_attn",
    "msa_latent_attn_backward_workspace_size", "msa_latent_attn_backward",
    "msa_sparse_attn_backward_workspace_size", "msa_sparse_attn_backward",
    "msa_sparse_kl_backward_workspace_size", "msa_sparse_kl_backward",
    "msa_profile_enable", "msa_profile_reset", "msa_profile_kernel_name", "msa_profile_read",
]


class MsaSeqsC(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32),
        ("total_q_rows", ctypes.c_int64),
        ("total_kv_rows", ctypes.c_int64),
        ("max_q_rows", ctypes.c_int32),
        ("max_kv_len", ctypes.c_int32),
        ("q_offsets", ctypes.c_void_p),
        ("kv_starts", ctypes.c_void_p),
        ("kv_lens", ctypes.c_void_p),
        ("block_table", ctypes.c_void_p),
        ("block_table_stride", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
    ]


class MsaRopeC(ctypes.Structure):
    _fields_ = [
        ("rot_dim", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("inv_freq", ctypes.c_void_p),
    ]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libmsa.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        P, S, I, Z, F = ctypes.c_void_p, ctypes.POINTER(MsaSeqsC), ctypes.c_int, ctypes.c_size_t, ctypes.c_float
        L.msa_strerror.argtypes = [I]
        L.msa_strerror.restype = ctypes.c_char_p
        L.msa_index_topk_workspace_size.argtypes = [S, I, I, I, I]
        L.msa_index_topk_workspace_size.restype = Z
        L.msa_index_topk.argtypes = [P, P, S, I, I, I, I, P, P, Z, P]
        L.msa_index_topk.restype = I
        L.msa_index_topk_noalloc.argtypes = [P, P, S, I, I, I, I, P, P]
        L.msa_index_topk_noalloc.restype = I
        L.msa_block_topk.argtypes = [P, ctypes.c_int64, I, ctypes.c_int64, I, P, P]
        L.msa_block_topk.restype = I
        for name in ("prefill", "decode"):
            ws = getattr(L, f"msa_sparse_attn_{name}_workspace_size")
            ws.argtypes = [S, I, I, I, I, I]
            ws.restype = Z
            fn = getattr(L, f"msa_sparse_attn_{name}")
            fn.argtypes = [P, P, P, P, S, I, I, I, I, I, F, P, P, P, Z, P]
            fn.restype = I
        for name in ("prefill", "decode"):
            fn = getattr(L, f"msa_sparse_attn_{name}_fp8")
            fn.argtypes = [P, P, P, F, F, F, P, S, I, I, I, I, I, F, P, P, P, Z, P]
            fn.restype = I
        L.msa_dense_attn_workspace_size.argtypes = [S, I, I, I]
        L.msa_dense_attn_workspace_size.restype = Z
        L.msa_dense_attn.argtypes = [P, P, P, S, I, I, I, F, P, P, P, Z, P]
        L.msa_dense_attn.restype = I
        L.msa_dense_attn_paged_workspace_size.argtypes = [S, I, I, I]
        L.msa_dense_attn_paged_workspace_size.restype = Z
        L.msa_dense_attn_paged.argtypes = [P, P, P, S, I, I, I, F, P, P, P, Z, P]
        L.msa_dense_attn_paged.restype = I
        L.msa_dense_attn_paged_fp8.argtypes = [P, P, P, F, F, F, S, I, I, I, F, P, P, P, Z, P]
        L.msa_dense_attn_paged_fp8.restype = I
        R, N = ctypes.POINTER(MsaRopeC), ctypes.c_int64
        L.msa_qk_norm_rope.argtypes = [P, N, P, N, S, I, I, I, P, P, F, R, P, P, P]
        L.msa_qk_norm_rope.restype = I
        L.msa_qk_norm_rope_fp8.argtypes = [P, N, P, N, F, F, S, I, I, I, P, P, F, R, P, P, P]
        L.msa_qk_norm_rope_fp8.restype = I
        L.msa_qk_norm_rope_backward_workspace_size.argtypes = [S, I, I, I]
        L.msa_qk_norm_rope_backward_workspace_size.restype = Z
        L.msa_qk_norm_rope_backward.argtypes = [P, N, P, N, P, P, S, I, I, I, P, P, F, R, P, N, P, N, P, P, P, Z, P]
        L.msa_qk_norm_rope_backward.restype = I
        L.msa_kv_append.argtypes = [P, N, P, N, P, N, S, I, I, I, P, P, F, R, R, P, P, P, P]
        L.msa_kv_append.restype = I
        L.msa_kv_append_fp8.argtypes = [P, N, P, N, F, F, P, N, S, I, I, I, P, P, F, R, R, P, P, P, P]
        L.msa_kv_append_fp8.restype = I
        L.msa_latent_append.argtypes = [P, N, P, N, S, I, P, F, R, P, P]
        L.msa_latent_append.restype = I
        L.msa_latent_append_fp8.argtypes = [P, N, P, N, F, S, I, P, F, R, P, P]
        L.msa_latent_append_fp8.restype = I
        L.msa_latent_attn_paged_workspace_size.argtypes = [S, I, I]
        L.msa_latent_attn_paged_workspace_size.restype = Z
        L.msa_latent_attn_paged.argtypes = [P, N, N, P, N, N, P, S, I, I, F, P, P, P, Z, P]
        L.msa_latent_attn_paged.restype = I
        L.msa_latent_attn_paged_fp8.argtypes = [P, N, N, P, N, N, P, F, S, I, I, F, P, P, P, Z, P]
        L.msa_latent_attn_paged_fp8.restype = I
        L.msa_latent_attn_workspace_size.argtypes = [S, I]
        L.msa_latent_attn_workspace_size.restype = Z
        L.msa_latent_attn.argtypes = [P, N, N, P, N, N, P, P, N, S, I, F, P, P, P, Z, P]
        L.msa_latent_attn.restype = I
        L.msa_latent_attn_backward_workspace_size.argtypes = [S, I]
        L.msa_latent_attn_backward_workspace_size.restype = Z
        L.msa_latent_attn_backward.argtypes = [P, N, N, P, N, N, P, P, N, P, P, P, S, I, F, P, N, N, P, N, N, P, P, N, P, Z, P]
        L.msa_latent_attn_backward.restype = I
        L.msa_sparse_attn_backward_workspace_size.argtypes = [S, I, I, I, I, I]
        L.msa_sparse_attn_backward_workspace_size.restype = Z
        L.msa_sparse_attn_backward.argtypes = [P, P, P, P, P, P, P, S, I, I, I, I, I, F, P, P, P, P, Z, P]
        L.msa_sparse_attn_backward.restype = I
        L.msa_sparse_kl_backward_workspace_size.argtypes = [S, I, I, I, I, I, I]
        L.msa_sparse_kl_backward_workspace_size.restype = Z
        L.msa_sparse_kl_backward.argtypes = [P, P, P, P, P, P, S, I, I, I, I, I, I, F, F, P, P, P, P, Z, P]
        L.msa_sparse_kl_backward.restype = I
        L.msa_profile_enable.argtypes = [I]
        L.msa_profile_enable.restype = I
        L.msa_profile_reset.argtypes = []
        L.msa_profile_reset.restype = I
        L.msa_profile_kernel_name.argtypes = [I]
        L.msa_profile_kernel_name.restype = ctypes.c_char_p
        L.msa_profile_read.argtypes = [ctypes.c_char_p, ctypes.POINTER(ctypes.c_int64),
                                       ctypes.POINTER(ctypes.c_double)]
        L.msa_profile_read.restype = I
        _lib = L
    return _lib


def _check(status: int, what: str):
    if status != MSA_OK:
        raise RuntimeError(f"{what} failed: {lib().msa_strerror(status).decode()} ({status})")


def _stream() -> int:
    # the handle itself: building a torch.cuda.Stream object took 2.8 us of a call
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _raw_stream(device: torch.device) -> int:
    return torch._C._cuda_getCurrentRawStream(device.index)


def _current(device: torch.device) -> bool:
    """Whether the GPU ``device`` is the current one (calls launch there)."""
    if device.type != "cuda":
        raise ValueError(f"expected tensors on a GPU, got {device}")
    return torch._C._cuda_getDevice() == device.index


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _need(t: torch.Tensor, name: str, dtype: torch.dtype, shape: Sequence[int], device):
    if t.dtype == dtype and t.shape == shape and t.is_contiguous() and t.device == device:
        return
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if t.device != device:
        raise ValueError(f"{name}: expected device {device}, got {t.device}")


class Seqs:
    """Sequence layout (see include/msa.h): device arrays plus host totals.

    ``block_table`` (int32 [num_seqs, max_blocks] on the device) makes the key
    side paged with pages of ``page_size`` rows; ``kv_starts`` is then unused."""

    def __init__(self, q_rows: Sequence[int], kv_lens: Sequence[int], kv_starts: Sequence[int],
                 total_kv_rows: int, device, block_table: Optional[torch.Tensor] = None, page_size: int = 0):
        assert len(q_rows) == len(kv_lens) == len(kv_starts) and len(q_rows) >= 1
        offs = [0]
        for r in q_rows:
            offs.append(offs[-1] + int(r))
        dev = torch.device(device)
        if dev.type == "cuda" and dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        self.device = dev
        self.q_offsets = torch.tensor(offs, dtype=torch.int32, device=self.device)
        self.kv_starts = torch.tensor([int(x) for x in kv_starts], dtype=torch.int64, device=self.device)
        self.kv_lens = torch.tensor([int(x) for x in kv_lens], dtype=torch.int32, device=self.device)
        self.num_seqs = len(q_rows)
        self.total_q_rows = offs[-1]
        self.total_kv_rows = int(total_kv_rows)
        self.max_q_rows = max(int(r) for r in q_rows)
        self.max_kv_len = max(int(x) for x in kv_lens)
        self.block_table = block_table
        if block_table is not None:
            _need(block_table, "block_table", torch.int32, (self.num_seqs, block_table.shape[1]), self.device)
        self.c = MsaSeqsC(self.num_seqs, self.total_q_rows, self.total_kv_rows, self.max_q_rows,
                          self.max_kv_len, self.q_offsets.data_ptr(), self.kv_starts.data_ptr(),
                          self.kv_lens.data_ptr(), None if block_table is None else block_table.data_ptr(),
                          0 if block_table is None else int(block_table.shape[1]), int(page_size))

    @classmethod
    def from_problem(cls, p, device) -> "Seqs":
        return cls(p.q_rows, p.kv_lens, p.kv_starts, p.total_kv_rows, device)

    def ref(self):
        return ctypes.byref(self.c)


def _workspace(nbytes: int, device, ws: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """The caller's workspace as given (a call runs in chunks sized to it and
    reports MSA_ERR_WORKSPACE below its minimum), else one of the queried size."""
    if ws is not None or nbytes == 0:
        return ws
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _need_workspace(ws: Optional[torch.Tensor], device) -> None:
    if ws is not None and (ws.device != device or not ws.is_contiguous()):
        raise ValueError(f"workspace: expected a contiguous tensor on {device}")


# ---------------------------------------------------------------- Index Branch
def index_topk_workspace_size(seqs: Seqs, num_kv_heads: int, d_idx: int, block_size: int, topk: int) -> int:
    return int(lib().msa_index_topk_workspace_size(seqs.ref(), num_kv_heads, d_idx, block_size, topk))


def index_topk(index_q: torch.Tensor, index_k: torch.Tensor, seqs: Seqs, block_size: int, topk: int,
               out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Block ids [total_q_rows, H_kv, topk] (int32, ascending, -1 padded)."""
    Tq, H_kv, d_idx = index_q.shape
    dev = seqs.device
    _need(index_q, "index_q", torch.bfloat16, (seqs.total_q_rows, H_kv, d_idx), dev)
    _need(index_k, "index_k", torch.bfloat16, (seqs.total_kv_rows, d_idx), dev)
    if out is None:
        out = torch.empty((Tq, H_kv, topk), dtype=torch.int32, device=dev)
    else:
        _need(out, "block_ids", torch.int32, (Tq, H_kv, topk), dev)
    nbytes = index_topk_workspace_size(seqs, H_kv, d_idx, block_size, topk)
    ws = _workspace(nbytes, dev, workspace)
    st = lib().msa_index_topk(_ptr(index_q), _ptr(index_k), seqs.ref(), H_kv, d_idx, block_size, topk,
                              _ptr(out), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(st, "msa_index_topk")
    return out


NOALLOC_MAX_BYTES = 64 << 20      # MSA_INDEX_TOPK_NOALLOC_MAX_BYTES


def index_topk_noalloc(index_q: torch.Tensor, index_k: torch.Tensor, seqs: Seqs, block_size: int, topk: int,
                       out: torch.Tensor) -> torch.Tensor:
    """msa_index_topk_noalloc: the Index Branch on the library's own scratch
    array; ``out`` (int32 [total_q_rows, H_kv, topk]) is caller-allocated."""
    Tq, H_kv, d_idx = index_q.shape
    dev = seqs.device
    _need(index_q, "index_q", torch.bfloat16, (seqs.total_q_rows, H_kv, d_idx), dev)
    _need(index_k, "index_k", torch.bfloat16, (seqs.total_kv_rows, d_idx), dev)
    _need(out, "block_ids", torch.int32, (Tq, H_kv, topk), dev)
    st = lib().msa_index_topk_noalloc(_ptr(index_q), _ptr(index_k), seqs.ref(), H_kv, d_idx, block_size, topk,
                                      _ptr(out), _stream())
    _check(st, "msa_index_topk_noalloc")
    return out


def block_topk(scores: torch.Tensor, k: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """msa_block_topk: the k best columns of each row of an fp32 [n_rows, n_cols]
    matrix (row stride taken from the tensor; unit column stride), int32
    [n_rows, k], ascending, -1 padded."""
    if scores.dim() != 2:
        raise ValueError("scores: expected a 2-d tensor")
    if scores.dtype != torch.float32:
        raise TypeError(f"scores: expected torch.float32, got {scores.dtype}")
    n_rows, n_cols = scores.shape
    if n_cols > 1 and scores.stride(1) != 1:
        raise ValueError("scores: columns must be contiguous")
    ld = scores.stride(0) if n_rows > 1 else max(n_cols, 1)
    dev = scores.device
    if out is None:
        out = torch.empty((n_rows, k), dtype=torch.int32, device=dev)
    else:
        _need(out, "ids", torch.int32, (n_rows, k), dev)
    st = lib().msa_block_topk(_ptr(scores), n_rows, n_cols, ld, k, _ptr(out), _stream())
    _check(st, "msa_block_topk")
    return out


# ---------------------------------------------------------------- Main Branch
def _attn(kind: str, q, k, v, block_ids, seqs: Seqs, block_size: int, softmax_scale, out, lse, workspace):
    Tq, H_q, d_h = q.shape
    H_kv = k.shape[1]
    topk = block_ids.shape[2]
    dev = seqs.device
    _need(q, "q", torch.bfloat16, (seqs.total_q_rows, H_q, d_h), dev)
    _need(k, "k", torch.bfloat16, (seqs.total_kv_rows, H_kv, d_h), dev)
    _need(v, "v", torch.bfloat16, (seqs.total_kv_rows, H_kv, d_h), dev)
    _need(block_ids, "block_ids", torch.int32, (Tq, H_kv, topk), dev)
    if out is None:
        out = torch.empty((Tq, H_q, d_h), dtype=torch.bfloat16, device=dev)
    else:
        _need(out, "o", torch.bfloat16, (Tq, H_q, d_h), dev)
    if lse is None:
        lse = torch.empty((Tq, H_q), dtype=torch.float32, device=dev)
    else:
        _need(lse, "lse", torch.float32, (Tq, H_q), dev)
    scale = 1.0 / math.sqrt(d_h) if softmax_scale is None else float(softmax_scale)
    L = lib()
    nbytes = int(getattr(L, f"msa_sparse_attn_{kind}_workspace_size")(seqs.ref(), H_q, H_kv, d_h, block_size, topk))
    ws = _workspace(nbytes, dev, workspace)
    st = getattr(L, f"msa_sparse_attn_{kind}")(
        _ptr(q), _ptr(k), _ptr(v), _ptr(block_ids), seqs.ref(), H_q, H_kv, d_h, block_size, topk, scale,
        _ptr(out), _ptr(lse), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(st, f"msa_sparse_attn_{kind}")
    return out, lse


def sparse_attn_prefill_workspace_size(seqs: Seqs, num_q_heads, num_kv_heads, head_dim, block_size, topk) -> int:
    return int(lib().msa_sparse_attn_prefill_workspace_size(seqs.ref(), num_q_heads, num_kv_heads, head_dim,
                                                             block_size, topk))


def sparse_attn_decode_workspace_size(seqs: Seqs, num_q_heads, num_kv_heads, head_dim, block_size, topk) -> int:
    return int(lib().msa_sparse_attn_decode_workspace_size(seqs.ref(), num_q_heads, num_kv_heads, head_dim,
                                                            block_size, topk))


def sparse_attn_prefill(q, k, v, block_ids, seqs: Seqs, block_size: int, softmax_scale=None,
                        out=None, lse=None, workspace=None):
    """O [Tq, H_q, d_h] bf16 and LSE [Tq, H_q] fp32 over the selected blocks."""
    return _attn("prefill", q, k, v, block_ids, seqs, block_size, softmax_scale, out, lse, workspace)


def sparse_attn_decode(q, k, v, block_ids, seqs: Seqs, block_size: int, softmax_scale=None,
                       out=None, lse=None, workspace=None):
    """Decode-shaped variant of sparse_attn_prefill (one query row per sequence)."""
    return _attn("decode", q, k, v, block_ids, seqs, block_size, softmax_scale, out, lse, workspace)


def _attn_fp8(kind: str, q, k, v, scales, block_ids, seqs: Seqs, block_size: int, softmax_scale, out, lse,
              workspace):
    Tq, H_q, d_h = q.shape
    H_kv = k.shape[1]
    topk = block_ids.shape[2]
    dev = seqs.device
    _need(q, "q", torch.uint8, (seqs.total_q_rows, H_q, d_h), dev)
    _need(k, "k", torch.uint8, (seqs.total_kv_rows, H_kv, d_h), dev)
    _need(v, "v", torch.uint8, (seqs.total_kv_rows, H_kv, d_h), dev)
    _need(block_ids, "block_ids", torch.int32, (Tq, H_kv, topk), dev)
    if out is None:
        out = torch.empty((Tq, H_q, d_h), dtype=torch.bfloat16, device=dev)
    else:
        _need(out, "o", torch.bfloat16, (Tq, H_q, d_h), dev)
    if lse is None:
        lse = torch.empty((Tq, H_q), dtype=torch.float32, device=dev)
    else:
        _need(lse, "lse", torch.float32, (Tq, H_q), dev)
    scale = 1.0 / math.sqrt(d_h) if softmax_scale is None else float(softmax_scale)
    L = lib()
    nbytes = int(getattr(L, f"msa_sparse_attn_{kind}_workspace_size")(seqs.ref(), H_q, H_kv, d_h, block_size, topk))
    ws = _workspace(nbytes, dev, workspace)
    qs, ks, vs = (float(x) for x in scales)
    st = getattr(L, f"msa_sparse_attn_{kind}_fp8")(
        _ptr(q), _ptr(k), _ptr(v), qs, ks, vs, _ptr(block_ids), seqs.ref(), H_q, H_kv, d_h, block_size, topk, scale,
        _ptr(out), _ptr(lse), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(st, f"msa_sparse_attn_{kind}_fp8")
    return out, lse


def sparse_attn_prefill_fp8(q, k, v, scales, block_ids, seqs: Seqs, block_size: int, softmax_scale=None,
                            out=None, lse=None, workspace=None):
    """Main Branch on e4m3 codes (uint8 tensors) with per-tensor scales (q, k, v)."""
    return _attn_fp8("prefill", q, k, v, scales, block_ids, seqs, block_size, softmax_scale, out, lse, workspace)


def sparse_attn_decode_fp8(q, k, v, scales, block_ids, seqs: Seqs, block_size: int, softmax_scale=None,
                           out=None, lse=None, workspace=None):
    return _attn_fp8("decode", q, k, v, scales, block_ids, seqs, block_size, softmax_scale, out, lse, workspace)


# ---------------------------------------------------------------- dense baseline
def dense_attn_workspace_size(seqs: Seqs, num_q_heads: int, num_kv_heads: int, head_dim: int = 128) -> int:
    return int(lib().msa_dense_attn_workspace_size(seqs.ref(), num_q_heads, num_kv_heads, head_dim))


def dense_attn(q, k, v, seqs: Seqs, softmax_scale=None, out=None, lse=None, workspace=None):
    """Dense causal GQA attention (the baseline): (O bf16 [Tq, H_q, d], LSE fp32 [Tq, H_q])."""
    Tq, H_q, d_h = q.shape
    H_kv = k.shape[1]
    dev = seqs.device
    _need(q, "q", torch.bfloat16, (seqs.total_q_rows, H_q, d_h), dev)
    _need(k, "k", torch.bfloat16, (seqs.total_kv_rows, H_kv, d_h), dev)
    _need(v, "v", torch.bfloat16, (seqs.total_kv_rows, H_kv, d_h), dev)
    if out is None:
        out = torch.empty((Tq, H_q, d_h), dtype=torch.bfloat16, device=dev)
    else:
        _need(out, "o", torch.bfloat16, (Tq, H_q, d_h), dev)
    if lse is None:
        lse = torch.empty((Tq, H_q), dtype=torch.float32, device=dev)
    else:
        _need(lse, "lse", torch.float32, (Tq, H_q), dev)
    scale = 1.0 / math.sqrt(d_h) if softmax_scale is None else float(softmax_scale)
    nbytes = dense_attn_workspace_size(seqs, H_q, H_kv, d_h)
    ws = _workspace(nbytes, dev, workspace)
    st = lib().msa_dense_attn(_ptr(q), _ptr(k), _ptr(v), seqs.ref(), H_q, H_kv, d_h, scale, _ptr(out), _ptr(lse),
                              _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(st, "msa_dense_attn")
    return out, lse


# ---------------------------------------------------------------- dense attention on a paged cache
def dense_attn_paged_workspace_size(seqs: Seqs, num_q_heads: int, num_kv_heads: int, head_dim: int = 128) -> int:
    return int(lib().msa_dense_attn_paged_workspace_size(seqs.ref(), num_q_heads, num_kv_heads, head_dim))


def _dense_paged(dtype, q, k, v, scales, seqs: Seqs, softmax_scale, out, lse, workspace):
    dev = seqs.device
    Tq, H_q, d_h = q.shape
    H_kv = k.shape[1]
    _need(q, "q", dtype, (seqs.total_q_rows, H_q, d_h), dev)
    _need(k, "k", dtype, (seqs.total_kv_rows, H_kv, d_h), dev)
    _need(v, "v", dtype, (seqs.total_kv_rows, H_kv, d_h), dev)
    _need_workspace(workspace, dev)
    if not _current(dev):
        with torch.cuda.device(dev):
            return _dense_paged(dtype, q, k, v, scales, seqs, softmax_scale, out, lse, workspace)
    if out is None:
        out = torch.empty(Tq, H_q, d_h, dtype=torch.bfloat16, device=dev)
    else:
        _need(out, "o", torch.bfloat16, (Tq, H_q, d_h), dev)
    if lse is None:
        lse = torch.empty(Tq, H_q, dtype=torch.float32, device=dev)
    else:
        _need(lse, "lse", torch.float32, (Tq, H_q), dev)
    scale = 1.0 / math.sqrt(d_h) if softmax_scale is None else float(softmax_scale)
    L, ref = lib(), seqs.ref()
    if workspace is None:
        workspace = _workspace(L.msa_dense_attn_paged_workspace_size(ref, H_q, H_kv, d_h), dev, None)
    ws, ws_bytes = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    if scales is None:
        st = L.msa_dense_attn_paged(q.data_ptr(), k.data_ptr(), v.data_ptr(), ref, H_q, H_kv, d_h, scale, out.data_ptr(),
                                    lse.data_ptr(), ws, ws_bytes, _raw_stream(dev))
    else:
        st = L.msa_dense_attn_paged_fp8(q.data_ptr(), k.data_ptr(), v.data_ptr(), *scales, ref, H_q, H_kv, d_h, scale,
                                        out.data_ptr(), lse.data_ptr(), ws, ws_bytes, _raw_stream(dev))
    _check(st, "msa_dense_attn_paged" if scales is None else "msa_dense_attn_paged_fp8")
    return out, lse


def dense_attn_paged(q, k, v, seqs: Seqs, softmax_scale=None, out=None, lse=None, workspace=None):
    """Dense causal attention of the new rows over a paged cache: (O bf16 [Tq, H_q, d], LSE fp32 [Tq, H_q])."""
    return _dense_paged(torch.bfloat16, q, k, v, None, seqs, softmax_scale, out, lse, workspace)


def dense_attn_paged_fp8(q, k, v, scales, seqs: Seqs, softmax_scale=None, out=None, lse=None, workspace=None):
    """The same on e4m3 codes (uint8 tensors) with per-tensor scales (q, k, v)."""
    qs, ks, vs = (float(x) for x in scales)
    return _dense_paged(torch.uint8, q, k, v, (qs, ks, vs), seqs, softmax_scale, out, lse, workspace)


# ---------------------------------------------------------------- norms, rotation, cache append
class Rope:
    """Rotation by position (struct msa_rope): ``inv_freq`` (radians per position
    of each pair, float64 on the device; its length is half the rotated
    dimensions), the pair layout and the factor of cosine and sine."""

    def __init__(self, inv_freq: torch.Tensor, interleaved: bool = False, scale: float = 1.0):
        if inv_freq.dim() != 1:
            raise ValueError("inv_freq: expected a 1-d tensor")
        _need(inv_freq, "inv_freq", torch.float64, tuple(inv_freq.shape), inv_freq.device)
        self.inv_freq = inv_freq
        self.c = MsaRopeC(2 * inv_freq.numel(), 1 if interleaved else 0, float(scale), inv_freq.data_ptr())
        self._ref = ctypes.byref(self.c)

    def ref(self):
        return self._ref


def rope_frequencies(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                     trained_len: int = 0, fast_turns: float = 32.0, slow_turns: float = 1.0):
    """(inv_freq as float64 CPU tensor, factor of cosine and sine) of rotary positions.

    ``scaling`` for contexts ``factor`` times as long as the trained ones:
      none       base^(-2i / rot_dim)
      linear     all divided by factor (positions interpolated)
      ntk        base * factor^(rot_dim / (rot_dim - 2)): the slowest pair is slowed
                 by factor, the fastest kept
      by_parts   a pair that turns r times over ``trained_len`` positions is kept for
                 r > ``fast_turns``, divided by factor for r < ``slow_turns``, and in
                 between mixed linearly in r (YaRN, arXiv 2309.00071, Sec. 3.2);
                 cosine and sine get 0.1 ln(factor) + 1 (Sec. 3.4)"""
    if rot_dim < 8 or rot_dim % 8 != 0:
        raise ValueError("rot_dim: expected a positive multiple of 8")
    if not base > 1.0 or not factor >= 1.0 or not math.isfinite(base * factor):
        raise ValueError("base must be above 1 and factor at least 1, both finite")
    i = torch.arange(rot_dim // 2, dtype=torch.float64)
    if scaling == "ntk":
        return (base * factor ** (rot_dim / (rot_dim - 2))) ** (-2.0 * i / rot_dim), 1.0
    f = base ** (-2.0 * i / rot_dim)
    if scaling == "none":
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling != "by_parts":
        raise ValueError(f"scaling: expected none, linear, ntk or by_parts, got {scaling!r}")
    if trained_len < 1 or not fast_turns > slow_turns > 0:
        raise ValueError("by_parts needs trained_len >= 1 and fast_turns > slow_turns > 0")
    keep = ((trained_len * f / (2 * math.pi) - slow_turns) / (fast_turns - slow_turns)).clamp(0.0, 1.0)
    return f * keep + f / factor * (1.0 - keep), 0.1 * math.log(factor) + 1.0


def _heads(t: torch.Tensor, name: str, rows: int, device):
    """(heads, head size, row stride) of a [rows, heads, dim] bf16 tensor whose rows may be apart (columns of a wider
    one)."""
    if t.dtype is torch.bfloat16 and t.dim() == 3 and t.device == device:
        n, h, d = t.shape
        if n == rows:
            sr, sh, sd = t.stride()
            if (sd == 1 or d == 1) and (sh == d or h == 1):
                return h, d, (sr if rows > 1 else h * d)
            raise ValueError(f"{name}: a row's heads must be contiguous")
    if t.dtype != torch.bfloat16:
        raise TypeError(f"{name}: expected torch.bfloat16, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name}: expected device {device}, got {t.device}")
    raise ValueError(f"{name}: expected shape ({rows}, heads, dim), got {tuple(t.shape)}")


def _weight(w: Optional[torch.Tensor], name: str, dim: int, device):
    if w is None:
        return None
    _need(w, name, torch.float32, (dim,), device)
    return w.data_ptr()


def _rope(rope: Optional[Rope], device):
    if rope is None:
        return None
    if rope.inv_freq.device != device:
        raise ValueError(f"rope: expected device {device}, got {rope.inv_freq.device}")
    return rope.ref()


def _norm_rope(scales, q, k, seqs: Seqs, rope, q_weight, k_weight, eps, q_out, k_out):
    dev, T = seqs.device, seqs.total_q_rows
    dtype = torch.bfloat16 if scales is None else torch.uint8
    H_q, d, q_stride = _heads(q, "q", T, dev)
    H_kv, k_stride, k_ptr, k_out_ptr = 0, 0, None, None
    if k is not None:
        H_kv, d_k, k_stride = _heads(k, "k", T, dev)
        if d_k != d:
            raise ValueError(f"k: expected head size {d}, got {d_k}")
    elif k_out is not None:
        raise ValueError("k_out: given without k")
    qw, kw = _weight(q_weight, "q_weight", d, dev), _weight(k_weight, "k_weight", d, dev)
    if q_out is not None:
        _need(q_out, "q_out", dtype, (T, H_q, d), dev)
    if k_out is not None:
        _need(k_out, "k_out", dtype, (T, H_kv, d), dev)
    if not _current(dev):
        with torch.cuda.device(dev):
            return _norm_rope(scales, q, k, seqs, rope, q_weight, k_weight, eps, q_out, k_out)
    if q_out is None:
        q_out = torch.empty(T, H_q, d, dtype=dtype, device=dev)
    if k is not None:
        if k_out is None:
            k_out = torch.empty(T, H_kv, d, dtype=dtype, device=dev)
        k_ptr, k_out_ptr = k.data_ptr(), k_out.data_ptr()
    if scales is None:
        st = lib().msa_qk_norm_rope(q.data_ptr(), q_stride, k_ptr, k_stride, seqs.ref(), H_q, H_kv, d, qw, kw, float(eps),
                                    _rope(rope, dev), q_out.data_ptr(), k_out_ptr, _raw_stream(dev))
    else:
        q_scale, k_scale = scales
        st = lib().msa_qk_norm_rope_fp8(q.data_ptr(), q_stride, k_ptr, k_stride, float(q_scale), float(k_scale), seqs.ref(), H_q,
                                        H_kv, d, qw, kw, float(eps), _rope(rope, dev), q_out.data_ptr(), k_out_ptr, _raw_stream(dev))
    _check(st, "msa_qk_norm_rope" if scales is None else "msa_qk_norm_rope_fp8")
    return q_out, k_out


def qk_norm_rope(q, k, seqs: Seqs, rope: Optional[Rope], q_weight=None, k_weight=None, eps: float = 1e-6,
                 q_out=None, k_out=None):
    """Norm of each head and rotation by position of the new rows' q [Tq, H_q, d] and k [Tq, H_kv, d] (bf16; rows
    may be columns of a wider tensor; ``k`` may be None): (q_out, k_out), contiguous bf16."""
    return _norm_rope(None, q, k, seqs, rope, q_weight, k_weight, eps, q_out, k_out)


def qk_norm_rope_fp8(q, k, scales, seqs: Seqs, rope: Optional[Rope], q_weight=None, k_weight=None, eps: float = 1e-6,
                     q_out=None, k_out=None):
    """The same into e4m3 codes (uint8) with per-tensor scales (q, k)."""
    return _norm_rope(scales, q, k, seqs, rope, q_weight, k_weight, eps, q_out, k_out)


def qk_norm_rope_backward_workspace_size(seqs: Seqs, num_q_heads: int, num_kv_heads: int, head_dim: int) -> int:
    return int(lib().msa_qk_norm_rope_backward_workspace_size(seqs.ref(), num_q_heads, num_kv_heads, head_dim))


def _grad_side(name, seqs: Seqs, x, g, w, d, dw):
    """(input, its row stride, heads, gradient, its row stride, weight, its gradient) of q or k; no heads where the
    tensor's upstream gradient is None."""
    if g is None:
        if d is not None or dw is not None:
            raise ValueError(f"d_{name} or d_{name}_weight: given without d_{name}_out")
        return None, 0, 0, None, 0, None, None
    T, dev = seqs.total_q_rows, seqs.device
    h, dim, stride = _heads(g, f"d_{name}_out", T, dev)
    if stride != h * dim:
        raise ValueError(f"d_{name}_out: must be contiguous")
    x_ptr, x_stride, w_ptr = None, 0, None
    if w is not None:
        if x is None:
            raise ValueError(f"{name}: needed for the norm's gradient")
        hx, dim_x, x_stride = _heads(x, name, T, dev)
        if hx != h or dim_x != dim:
            raise ValueError(f"{name}: expected shape {tuple(g.shape)}, got {tuple(x.shape)}")
        x_ptr, w_ptr = x.data_ptr(), _weight(w, f"{name}_weight", dim, dev)
        if dw is None:
            dw = torch.empty(dim, dtype=torch.float32, device=dev)
        else:
            _need(dw, f"d_{name}_weight", torch.float32, (dim,), dev)
    elif dw is not None:
        raise ValueError(f"d_{name}_weight: given without {name}_weight")
    if d is None:
        return x_ptr, x_stride, h, torch.empty(T, h, dim, dtype=torch.bfloat16, device=dev), h * dim, w_ptr, dw
    hd, dim_d, d_stride = _heads(d, f"d_{name}", T, dev)
    if hd != h or dim_d != dim:
        raise ValueError(f"d_{name}: expected shape {tuple(g.shape)}, got {tuple(d.shape)}")
    return x_ptr, x_stride, h, d, d_stride, w_ptr, dw


def qk_norm_rope_backward(q, k, d_q_out, d_k_out, seqs: Seqs, rope: Optional[Rope], q_weight=None, k_weight=None,
                          eps: float = 1e-6, d_q=None, d_k=None, d_q_weight=None, d_k_weight=None, workspace=None):
    """Gradients of qk_norm_rope: (d_q, d_k, d_q_weight, d_k_weight); a weight's is None where it is None, both of a
    tensor's where its upstream gradient is.  ``q`` and ``k`` are the forward's inputs (not read, and may be None,
    without weight); d_q and d_k may be columns of a wider tensor."""
    if d_q_out is None and d_k_out is None:
        raise ValueError("d_q_out or d_k_out is needed")
    dev = seqs.device
    q_in, q_stride, H_q, d_q, dq_stride, qw, d_q_weight = _grad_side("q", seqs, q, d_q_out, q_weight, d_q, d_q_weight)
    k_in, k_stride, H_kv, d_k, dk_stride, kw, d_k_weight = _grad_side("k", seqs, k, d_k_out, k_weight, d_k, d_k_weight)
    dim = (d_k_out if d_q_out is None else d_q_out).shape[2]
    if d_k_out is not None and d_k_out.shape[2] != dim:
        raise ValueError(f"d_k_out: expected head size {dim}, got {d_k_out.shape[2]}")
    _need_workspace(workspace, dev)
    if not _current(dev):
        with torch.cuda.device(dev):
            return qk_norm_rope_backward(q, k, d_q_out, d_k_out, seqs, rope, q_weight, k_weight, eps, d_q, d_k, d_q_weight,
                                         d_k_weight, workspace)
    ref = seqs.ref()
    if workspace is None and (qw is not None or kw is not None):
        workspace = _workspace(lib().msa_qk_norm_rope_backward_workspace_size(ref, H_q, H_kv, dim), dev, None)
    ws, ws_bytes = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    st = lib().msa_qk_norm_rope_backward(
        q_in, q_stride, k_in, k_stride, _ptr(d_q_out), _ptr(d_k_out), ref, H_q, H_kv, dim, qw, kw, float(eps),
        _rope(rope, dev), _ptr(d_q), dq_stride, _ptr(d_k), dk_stride, _ptr(d_q_weight), _ptr(d_k_weight), ws, ws_bytes, _raw_stream(dev))
    _check(st, "msa_qk_norm_rope_backward")
    return d_q, d_k, d_q_weight, d_k_weight


def _append(scales, k, v, seqs: Seqs, rope, k_cache, v_cache, k_weight, eps, index_k, index_k_cache, index_k_weight,
            index_rope):
    dev, T = seqs.device, seqs.total_q_rows
    H_kv, d, k_stride = _heads(k, "k", T, dev)
    H_v, d_v, v_stride = _heads(v, "v", T, dev)
    if H_v != H_kv or d_v != d:
        raise ValueError(f"v: expected shape {tuple(k.shape)}, got {tuple(v.shape)}")
    dtype = torch.bfloat16 if scales is None else torch.uint8
    _need(k_cache, "k_cache", dtype, (seqs.total_kv_rows, H_kv, d), dev)
    _need(v_cache, "v_cache", dtype, (seqs.total_kv_rows, H_kv, d), dev)
    d_idx, i_stride, i_ptr, ic_ptr, iw, ir = 0, 0, None, None, None, None
    if (index_k is None) != (index_k_cache is None):
        raise ValueError("index_k and index_k_cache go together")
    if index_k is not None:
        if index_k.dtype is not torch.bfloat16:
            raise TypeError(f"index_k: expected torch.bfloat16, got {index_k.dtype}")
        if index_k.dim() != 2 or index_k.shape[0] != T or index_k.device != dev:
            raise ValueError(f"index_k: expected shape ({T}, d_idx) on {dev}, got {tuple(index_k.shape)} on {index_k.device}")
        d_idx = index_k.shape[1]
        i_stride, step = index_k.stride()
        if step != 1 and d_idx != 1:
            raise ValueError("index_k: a row must be contiguous")
        if T <= 1:
            i_stride = d_idx
        _need(index_k_cache, "index_k_cache", torch.bfloat16, (seqs.total_kv_rows, d_idx), dev)
        i_ptr, ic_ptr = index_k.data_ptr(), index_k_cache.data_ptr()
        iw, ir = _weight(index_k_weight, "index_k_weight", d_idx, dev), _rope(index_rope, dev)
    kw = _weight(k_weight, "k_weight", d, dev)
    if not _current(dev):
        with torch.cuda.device(dev):
            return _append(scales, k, v, seqs, rope, k_cache, v_cache, k_weight, eps, index_k, index_k_cache, index_k_weight,
                           index_rope)
    if scales is None:
        st = lib().msa_kv_append(k.data_ptr(), k_stride, v.data_ptr(), v_stride, i_ptr, i_stride, seqs.ref(), H_kv, d, d_idx,
                                 kw, iw, float(eps), _rope(rope, dev), ir, k_cache.data_ptr(), v_cache.data_ptr(), ic_ptr,
                                 _raw_stream(dev))
    else:
        k_scale, v_scale = scales
        st = lib().msa_kv_append_fp8(k.data_ptr(), k_stride, v.data_ptr(), v_stride, float(k_scale), float(v_scale), i_ptr,
                                     i_stride, seqs.ref(), H_kv, d, d_idx, kw, iw, float(eps), _rope(rope, dev), ir,
                                     k_cache.data_ptr(), v_cache.data_ptr(), ic_ptr, _raw_stream(dev))
    _check(st, "msa_kv_append" if scales is None else "msa_kv_append_fp8")


def kv_append(k, v, seqs: Seqs, rope: Optional[Rope], k_cache, v_cache, k_weight=None, eps: float = 1e-6, index_k=None,
              index_k_cache=None, index_k_weight=None, index_rope: Optional[Rope] = None) -> None:
    """The new rows' k (norm, rotation), v and index_k (norm, rotation) into their cache rows, in place."""
    _append(None, k, v, seqs, rope, k_cache, v_cache, k_weight, eps, index_k, index_k_cache, index_k_weight,
            index_rope)


def kv_append_fp8(k, v, scales, seqs: Seqs, rope: Optional[Rope], k_cache, v_cache, k_weight=None, eps: float = 1e-6,
                  index_k=None, index_k_cache=None, index_k_weight=None, index_rope: Optional[Rope] = None) -> None:
    """The same with e4m3 k and v caches (uint8) and per-tensor scales (k, v); index keys stay bf16."""
    _append(scales, k, v, seqs, rope, k_cache, v_cache, k_weight, eps, index_k, index_k_cache, index_k_weight,
            index_rope)


# ---------------------------------------------------------------- latent attention
LATENT_HEAD_DIM = 128             # a head's own key part, and its values (expanded form)
LATENT_ROPE_DIM = 64              # the key part that the heads share


def _latent_scale(softmax_scale) -> float:
    if softmax_scale is None:
        return 1.0 / math.sqrt(LATENT_HEAD_DIM + LATENT_ROPE_DIM)
    return float(softmax_scale)


def _strided(t: torch.Tensor, name: str, shape: Sequence[int], device):
    """(row stride, head stride) of a bf16 [rows, heads, dim] tensor whose rows and heads may lie anywhere."""
    if t.dtype is not torch.bfloat16:
        raise TypeError(f"{name}: expected torch.bfloat16, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name}: expected device {device}, got {t.device}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    rows, heads, dim = t.stride()
    if dim != 1:
        raise ValueError(f"{name}: a head must be contiguous")
    return (rows if shape[0] > 1 else 0), (heads if shape[1] > 1 else 0)


def _rows(t: torch.Tensor, name: str, rows: int, dim: Optional[int], device):
    """Row stride of a bf16 [rows, dim] tensor whose rows may be apart (columns of a wider one)."""
    if t.dtype is not torch.bfloat16:
        raise TypeError(f"{name}: expected torch.bfloat16, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name}: expected device {device}, got {t.device}")
    if t.dim() != 2 or t.shape[0] != rows or (dim is not None and t.shape[1] != dim):
        raise ValueError(f"{name}: expected shape ({rows}, {'latent' if dim is None else dim}), got {tuple(t.shape)}")
    stride, step = t.stride()
    if step != 1:
        raise ValueError(f"{name}: a row must be contiguous")
    return stride if rows > 1 else t.shape[1]


def _latent_append(scale, latent, k_rope, seqs: Seqs, rope, cache, weight, eps):
    dev, T = seqs.device, seqs.total_q_rows
    l_stride = _rows(latent, "latent", T, None, dev)
    k_stride = _rows(k_rope, "k_rope", T, LATENT_ROPE_DIM, dev)
    R = latent.shape[1]
    _need(cache, "cache", torch.bfloat16 if scale is None else torch.uint8, (seqs.total_kv_rows, R + LATENT_ROPE_DIM), dev)
    w = _weight(weight, "weight", R, dev)
    if not _current(dev):
        with torch.cuda.device(dev):
            return _latent_append(scale, latent, k_rope, seqs, rope, cache, weight, eps)
    if scale is None:
        st = lib().msa_latent_append(latent.data_ptr(), l_stride, k_rope.data_ptr(), k_stride, seqs.ref(), R, w, float(eps),
                                     _rope(rope, dev), cache.data_ptr(), _raw_stream(dev))
    else:
        st = lib().msa_latent_append_fp8(latent.data_ptr(), l_stride, k_rope.data_ptr(), k_stride, float(scale), seqs.ref(), R,
                                         w, float(eps), _rope(rope, dev), cache.data_ptr(), _raw_stream(dev))
    _check(st, "msa_latent_append" if scale is None else "msa_latent_append_fp8")


def latent_append(latent, k_rope, seqs: Seqs, rope: Optional[Rope], cache, weight=None, eps: float = 1e-6) -> None:
    """The new rows' latents [Tq, R] (norm, if ``weight``) and shared key parts [Tq, 64] (rotation) into their rows of
    ``cache`` [Tkv, R + 64], in place; rows may be columns of a wider tensor."""
    _latent_append(None, latent, k_rope, seqs, rope, cache, weight, eps)


def latent_append_fp8(latent, k_rope, scale, seqs: Seqs, rope: Optional[Rope], cache, weight=None, eps: float = 1e-6) -> None:
    """The same into a cache of e4m3 codes (uint8) with a per-tensor scale."""
    _latent_append(scale, latent, k_rope, seqs, rope, cache, weight, eps)


def latent_attn_paged_workspace_size(seqs: Seqs, num_heads: int, latent_dim: int) -> int:
    return int(lib().msa_latent_attn_paged_workspace_size(seqs.ref(), num_heads, latent_dim))


def _latent_paged(cache_scale, q, q_rope, cache, seqs: Seqs, softmax_scale, out, lse, workspace):
    dev, T = seqs.device, seqs.total_q_rows
    if q.dim() != 3:
        raise ValueError(f"q: expected shape ({T}, heads, latent), got {tuple(q.shape)}")
    H, R = q.shape[1], q.shape[2]
    qs, qh = _strided(q, "q", (T, H, R), dev)
    es, eh = _strided(q_rope, "q_rope", (T, H, LATENT_ROPE_DIM), dev)
    _need(cache, "cache", torch.bfloat16 if cache_scale is None else torch.uint8, (seqs.total_kv_rows, R + LATENT_ROPE_DIM), dev)
    _need_workspace(workspace, dev)
    if not _current(dev):
        with torch.cuda.device(dev):
            return _latent_paged(cache_scale, q, q_rope, cache, seqs, softmax_scale, out, lse, workspace)
    if out is None:
        out = torch.empty(T, H, R, dtype=torch.bfloat16, device=dev)
    else:
        _need(out, "o", torch.bfloat16, (T, H, R), dev)
    if lse is None:
        lse = torch.empty(T, H, dtype=torch.float32, device=dev)
    else:
        _need(lse, "lse", torch.float32, (T, H), dev)
    L, ref = lib(), seqs.ref()
    if workspace is None:
        workspace = _workspace(L.msa_latent_attn_paged_workspace_size(ref, H, R), dev, None)
    ws, ws_bytes = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    scale = _latent_scale(softmax_scale)
    if cache_scale is None:
        st = L.msa_latent_attn_paged(q.data_ptr(), qs, qh, q_rope.data_ptr(), es, eh, cache.data_ptr(), ref, H, R, scale,
                                     out.data_ptr(), lse.data_ptr(), ws, ws_bytes, _raw_stream(dev))
    else:
        st = L.msa_latent_attn_paged_fp8(q.data_ptr(), qs, qh, q_rope.data_ptr(), es, eh, cache.data_ptr(), float(cache_scale),
                                         ref, H, R, scale, out.data_ptr(), lse.data_ptr(), ws, ws_bytes, _raw_stream(dev))
    _check(st, "msa_latent_attn_paged" if cache_scale is None else "msa_latent_attn_paged_fp8")
    return out, lse


def latent_attn_paged(q, q_rope, cache, seqs: Seqs, softmax_scale=None, out=None, lse=None, workspace=None):
    """Latent attention, absorbed form, over a paged cache [Tkv, R + 64]: (O bf16 [Tq, H, R], the weighted latents, LSE fp32
    [Tq, H]) of q [Tq, H, R] (queries times the key up-projection) and q_rope [Tq, H, 64], both with any row and
    head strides.  ``softmax_scale`` defaults to that of the expanded head, 1 / sqrt(128 + 64)."""
    return _latent_paged(None, q, q_rope, cache, seqs, softmax_scale, out, lse, workspace)


def latent_attn_paged_fp8(q, q_rope, cache, scale, seqs: Seqs, softmax_scale=None, out=None, lse=None, workspace=None):
    """The same on a cache of e4m3 codes (uint8) with a per-tensor scale; queries stay bf16."""
    return _latent_paged(float(scale), q, q_rope, cache, seqs, softmax_scale, out, lse, workspace)


def latent_attn_workspace_size(seqs: Seqs, num_heads: int) -> int:
    return int(lib().msa_latent_attn_workspace_size(seqs.ref(), num_heads))


def latent_attn(q, q_rope, kv, k_rope, seqs: Seqs, softmax_scale=None, out=None, lse=None, workspace=None):
    """Latent attention, expanded form: (O bf16 [Tq, H, 128], LSE fp32 [Tq, H]) of q [Tq, H, 128] and q_rope [Tq, H, 64], both
    with any row and head strides, over kv [Tkv, H, 256] (a head's own key part, then its values) and the shared
    k_rope [Tkv, 64], whose rows may be columns of a wider tensor."""
    dev, T = seqs.device, seqs.total_q_rows
    if q.dim() != 3:
        raise ValueError(f"q: expected shape ({T}, heads, {LATENT_HEAD_DIM}), got {tuple(q.shape)}")
    H = q.shape[1]
    qs, qh = _strided(q, "q", (T, H, LATENT_HEAD_DIM), dev)
    es, eh = _strided(q_rope, "q_rope", (T, H, LATENT_ROPE_DIM), dev)
    _need(kv, "kv", torch.bfloat16, (seqs.total_kv_rows, H, 2 * LATENT_HEAD_DIM), dev)
    ks = _rows(k_rope, "k_rope", seqs.total_kv_rows, LATENT_ROPE_DIM, dev)
    _need_workspace(workspace, dev)
    if not _current(dev):
        with torch.cuda.device(dev):
            return latent_attn(q, q_rope, kv, k_rope, seqs, softmax_scale, out, lse, workspace)
    if out is None:
        out = torch.empty(T, H, LATENT_HEAD_DIM, dtype=torch.bfloat16, device=dev)
    else:
        _need(out, "o", torch.bfloat16, (T, H, LATENT_HEAD_DIM), dev)
    if lse is None:
        lse = torch.empty(T, H, dtype=torch.float32, device=dev)
    else:
        _need(lse, "lse", torch.float32, (T, H), dev)
    L, ref = lib(), seqs.ref()
    if workspace is None:
        workspace = _workspace(L.msa_latent_attn_workspace_size(ref, H), dev, None)
    ws, ws_bytes = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    st = L.msa_latent_attn(q.data_ptr(), qs, qh, q_rope.data_ptr(), es, eh, kv.data_ptr(), k_rope.data_ptr(), ks, ref, H,
                           _latent_scale(softmax_scale), out.data_ptr(), lse.data_ptr(), ws, ws_bytes, _raw_stream(dev))
    _check(st, "msa_latent_attn")
    return out, lse


def latent_attn_backward_workspace_size(seqs: Seqs, num_heads: int) -> int:
    return int(lib().msa_latent_attn_backward_workspace_size(seqs.ref(), num_heads))


def latent_attn_backward(q, q_rope, kv, k_rope, o, lse, d_o, seqs: Seqs, softmax_scale=None, d_q=None, d_q_rope=None, d_kv=None,
                         d_k_rope=None, workspace=None):
    """Gradients of latent_attn for the upstream gradient d_o, given its inputs and outputs: (d_q, d_q_rope, d_kv, d_k_rope), the
    last summed over the heads; d_q, d_q_rope and d_k_rope may be columns of wider tensors."""
    dev, T, N = seqs.device, seqs.total_q_rows, seqs.total_kv_rows
    if q.dim() != 3:
        raise ValueError(f"q: expected shape ({T}, heads, {LATENT_HEAD_DIM}), got {tuple(q.shape)}")
    H = q.shape[1]
    qs, qh = _strided(q, "q", (T, H, LATENT_HEAD_DIM), dev)
    es, eh = _strided(q_rope, "q_rope", (T, H, LATENT_ROPE_DIM), dev)
    _need(kv, "kv", torch.bfloat16, (N, H, 2 * LATENT_HEAD_DIM), dev)
    ks = _rows(k_rope, "k_rope", N, LATENT_ROPE_DIM, dev)
    _need(o, "o", torch.bfloat16, (T, H, LATENT_HEAD_DIM), dev)
    _need(lse, "lse", torch.float32, (T, H), dev)
    _need(d_o, "d_o", torch.bfloat16, (T, H, LATENT_HEAD_DIM), dev)
    _need_workspace(workspace, dev)
    if not _current(dev):
        with torch.cuda.device(dev):
            return latent_attn_backward(q, q_rope, kv, k_rope, o, lse, d_o, seqs, softmax_scale, d_q, d_q_rope, d_kv, d_k_rope,
                                        workspace)
    if d_q is None:
        d_q = torch.empty(T, H, LATENT_HEAD_DIM, dtype=torch.bfloat16, device=dev)
    dqs, dqh = _strided(d_q, "d_q", (T, H, LATENT_HEAD_DIM), dev)
    if d_q_rope is None:
        d_q_rope = torch.empty(T, H, LATENT_ROPE_DIM, dtype=torch.bfloat16, device=dev)
    des, deh = _strided(d_q_rope, "d_q_rope", (T, H, LATENT_ROPE_DIM), dev)
    if d_kv is None:
        d_kv = torch.empty(N, H, 2 * LATENT_HEAD_DIM, dtype=torch.bfloat16, device=dev)
    else:
        _need(d_kv, "d_kv", torch.bfloat16, (N, H, 2 * LATENT_HEAD_DIM), dev)
    if d_k_rope is None:
        d_k_rope = torch.empty(N, LATENT_ROPE_DIM, dtype=torch.bfloat16, device=dev)
    dks = _rows(d_k_rope, "d_k_rope", N, LATENT_ROPE_DIM, dev)
    L, ref = lib(), seqs.ref()
    if workspace is None:
        workspace = _workspace(L.msa_latent_attn_backward_workspace_size(ref, H), dev, None)
    ws, ws_bytes = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    st = L.msa_latent_attn_backward(
        q.data_ptr(), qs, qh, q_rope.data_ptr(), es, eh, kv.data_ptr(), k_rope.data_ptr(), ks, o.data_ptr(), lse.data_ptr(),
        d_o.data_ptr(), ref, H, _latent_scale(softmax_scale), d_q.data_ptr(), dqs, dqh, d_q_rope.data_ptr(), des, deh,
        d_kv.data_ptr(), d_k_rope.data_ptr(), dks, ws, ws_bytes, _raw_stream(dev))
    _check(st, "msa_latent_attn_backward")
    return d_q, d_q_rope, d_kv, d_k_rope


# ---------------------------------------------------------------- kernel timing
# ---------------------------------------------------------------- training backward
def sparse_attn_backward_workspace_size(seqs: Seqs, num_q_heads, num_kv_heads, head_dim, block_size, topk) -> int:
    return int(lib().msa_sparse_attn_backward_workspace_size(seqs.ref(), num_q_heads, num_kv_heads, head_dim,
                                                              block_size, topk))


def sparse_attn_backward(q, k, v, o, lse, d_o, block_ids, seqs: Seqs, block_size: int, softmax_scale=None,
                         d_q=None, d_k=None, d_v=None, workspace=None):
    """dQ [Tq, H_q, d_h], dK and dV [Tkv, H_kv, d_h] (bf16) of the Main Branch for
    the upstream gradient d_o, given the forward's O and LSE."""
    Tq, H_q, d_h = q.shape
    H_kv = k.shape[1]
    topk = block_ids.shape[2]
    dev = seqs.device
    _need(q, "q", torch.bfloat16, (seqs.total_q_rows, H_q, d_h), dev)
    _need(k, "k", torch.bfloat16, (seqs.total_kv_rows, H_kv, d_h), dev)
    _need(v, "v", torch.bfloat16, (seqs.total_kv_rows, H_kv, d_h), dev)
    _need(o, "o", torch.bfloat16, (Tq, H_q, d_h), dev)
    _need(lse, "lse", torch.float32, (Tq, H_q), dev)
    _need(d_o, "d_o", torch.bfloat16, (Tq, H_q, d_h), dev)
    _need(block_ids, "block_ids", torch.int32, (Tq, H_kv, topk), dev)
    if d_q is None:
        d_q = torch.empty_like(q)
    if d_k is None:
        d_k = torch.empty_like(k)
    if d_v is None:
        d_v = torch.empty_like(v)
    _need(d_q, "d_q", torch.bfloat16, tuple(q.shape), dev)
    _need(d_k, "d_k", torch.bfloat16, tuple(k.shape), dev)
    _need(d_v, "d_v", torch.bfloat16, tuple(v.shape), dev)
    scale = 1.0 / math.sqrt(d_h) if softmax_scale is None else float(softmax_scale)
    L = lib()
    nbytes = int(L.msa_sparse_attn_backward_workspace_size(seqs.ref(), H_q, H_kv, d_h, block_size, topk))
    ws = _workspace(nbytes, dev, workspace)
    st = L.msa_sparse_attn_backward(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(d_o), _ptr(block_ids),
                                    seqs.ref(), H_q, H_kv, d_h, block_size, topk, scale, _ptr(d_q), _ptr(d_k),
                                    _ptr(d_v), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                    _stream())
    _check(st, "msa_sparse_attn_backward")
    return d_q, d_k, d_v


def sparse_kl_backward_workspace_size(seqs: Seqs, num_q_heads, num_kv_heads, d_idx, head_dim, block_size,
                                      topk) -> int:
    return int(lib().msa_sparse_kl_backward_workspace_size(seqs.ref(), num_q_heads, num_kv_heads, d_idx, head_dim,
                                                            block_size, topk))


def sparse_kl_backward(index_q, index_k, q, k, lse, block_ids, seqs: Seqs, block_size: int, grad_scale: float = 1.0,
                       softmax_scale=None, with_kl: bool = True, d_index_q=None, d_index_k=None, kl=None,
                       workspace=None):
    """Sparse KL loss of the Index Branch: (d_index_q [Tq, H_kv, d_idx] bf16,
    d_index_k [Tkv, d_idx] bf16, kl [Tq, H_kv] fp32 or None); the gradients are
    grad_scale times those of sum(kl)."""
    Tq, H_kv, d_idx = index_q.shape
    H_q, d_h = q.shape[1], q.shape[2]
    topk = block_ids.shape[2]
    dev = seqs.device
    _need(index_q, "index_q", torch.bfloat16, (seqs.total_q_rows, H_kv, d_idx), dev)
    _need(index_k, "index_k", torch.bfloat16, (seqs.total_kv_rows, d_idx), dev)
    _need(q, "q", torch.bfloat16, (seqs.total_q_rows, H_q, d_h), dev)
    _need(k, "k", torch.bfloat16, (seqs.total_kv_rows, H_kv, d_h), dev)
    _need(lse, "lse", torch.float32, (Tq, H_q), dev)
    _need(block_ids, "block_ids", torch.int32, (Tq, H_kv, topk), dev)
    if d_index_q is None:
        d_index_q = torch.empty_like(index_q)
    if d_index_k is None:
        d_index_k = torch.empty_like(index_k)
    if with_kl and kl is None:
        kl = torch.empty((Tq, H_kv), dtype=torch.float32, device=dev)
    _need(d_index_q, "d_index_q", torch.bfloat16, tuple(index_q.shape), dev)
    _need(d_index_k, "d_index_k", torch.bfloat16, tuple(index_k.shape), dev)
    if kl is not None:
        _need(kl, "kl", torch.float32, (Tq, H_kv), dev)
    scale = 1.0 / math.sqrt(d_h) if softmax_scale is None else float(softmax_scale)
    L = lib()
    nbytes = int(L.msa_sparse_kl_backward_workspace_size(seqs.ref(), H_q, H_kv, d_idx, d_h, block_size, topk))
    ws = _workspace(nbytes, dev, workspace)
    st = L.msa_sparse_kl_backward(_ptr(index_q), _ptr(index_k), _ptr(q), _ptr(k), _ptr(lse), _ptr(block_ids),
                                  seqs.ref(), H_q, H_kv, d_idx, d_h, block_size, topk, scale, float(grad_scale),
                                  _ptr(d_index_q), _ptr(d_index_k), _ptr(kl), _ptr(ws),
                                  0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(st, "msa_sparse_kl_backward")
    return d_index_q, d_index_k, kl


def profile_enable(on: bool = True) -> None:
    """Bracket every kernel of later calls with HIP events on its stream."""
    _check(lib().msa_profile_enable(1 if on else 0), "msa_profile_enable")


def profile_reset() -> None:
    _check(lib().msa_profile_reset(), "msa_profile_reset")


def profile_read() -> dict:
    """{kernel name: (launches, summed ms)} since the last reset (waits for the events)."""
    L = lib()
    out = {}
    i = 0
    while True:
        name = L.msa_profile_kernel_name(i)
        if name is None:
            break
        n = ctypes.c_int64(0)
        ms = ctypes.c_double(0.0)
        _check(L.msa_profile_read(name, ctypes.byref(n), ctypes.byref(ms)), "msa_profile_read")
        if n.value > 0:
            out[name.decode()] = (int(n.value), float(ms.value))
        i += 1
    return out
