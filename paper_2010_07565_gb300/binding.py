"""Python binding of libbigcn.so (include/bigcn.h): argument marshalling only.

The ``bigcn_*`` functions mirror the C entry points one to one and take torch
CUDA tensors for every array; they read pointers, sizes and row strides off
the tensors, pass the current torch stream (or ``stream``), and raise
:class:`BigcnError` on a non-OK status. Every step of the computation runs in
the library's kernels; there is no Python or CPU fallback, and the library
must have been built (``__graft_entry__.build()``) before first use.

The lower-case helpers (``pack_rows``, ``layer_forward``, ...) only allocate
the outputs with torch and call the matching ``bigcn_*`` function.
"""
from __future__ import annotations

import ctypes
import os
import threading

import torch

from . import build as _build

_lib = None
_lock = threading.Lock()

BIGCN_OK = 0
STATUS_NAMES = {0: "BIGCN_OK", 1: "BIGCN_ERR_INVALID_ARG", 2: "BIGCN_ERR_MISALIGNED",
                3: "BIGCN_ERR_CUDA", 4: "BIGCN_ERR_UNSUPPORTED", 5: "BIGCN_ERR_SCRATCH_LIMIT"}
STATIC_SCRATCH_BYTES = (32 << 20) + 256   # BIGCN_STATIC_SCRATCH_BYTES

_p = ctypes.c_void_p
_i32 = ctypes.c_int32
_i64 = ctypes.c_int64
_sz = ctypes.c_size_t

SIGNATURES = {
    "bigcn_status_string": ([ctypes.c_int], ctypes.c_char_p),
    "bigcn_words": ([_i32], _i32),
    "bigcn_pack_rows": ([_p, _i64, _i32, _i64, _p, _p, _p, _i32, _p, _p], ctypes.c_int),
    "bigcn_pack_weights": ([_p, _i32, _i32, _i64, _p, _i32, _p, _p], ctypes.c_int),
    "bigcn_xnor_gemm": ([_p, _p, _i64, _p, _p, _i32, _i32, _i32, _p, _i64, _p, _p],
                        ctypes.c_int),
    "bigcn_xnor_gemm_degscaled": ([_p, _p, _i64, _p, _p, _i32, _i32, _i32, _p, _p, _i64, _p],
                                  ctypes.c_int),
    "bigcn_spmm_norm": ([_p, _p, _i64, _i64, _p, _i64, _i32, _p, _i64, _p], ctypes.c_int),
    "bigcn_spmm_prescaled": ([_p, _p, _i64, _i64, _p, _i64, _i32, _p, _i64, _p], ctypes.c_int),
    "bigcn_device_timeouts": ([], _i32),
    "bigcn_layer_workspace_bytes": ([_i64, _i32, _i32], _sz),
    "bigcn_layer_forward": ([_p, _i64, _i32, _i64, _p, _p, _p, _i32, _i64, _p, _p, _i64, _p,
                             _sz, _p, _i64, _p], ctypes.c_int),
    "bigcn_layer_forward_timed": ([_p, _i64, _i32, _i64, _p, _p, _p, _i32, _i64, _p, _p, _i64,
                                   _p, _sz, _p, _i64, _p, _i32, _p], ctypes.c_int),
    "bigcn_layer_backward_workspace_bytes": ([_i64, _i32, _i32], _sz),
    "bigcn_layer_backward": ([_p, _i64, _i32, _i64, _p, _p, _p, _i32, _i64, _p, _p, _i64, _p,
                              _i64, _p, _i64, _p, _i64, _p, _sz, _p], ctypes.c_int),
    "bigcn_forward_2layer_workspace_bytes": ([_i64, _i32, _i32, _i32], _sz),
    "bigcn_forward_2layer_launches": ([_i64, _i32, _i32, _i32], _i32),
    "bigcn_forward_2layer_aggregation": ([_i32, _i32, _i32], _i32),
    "bigcn_spmm_prescaled_rows": ([_p, _p, _i64, _i64, _i64, _p, _i64, _i32, _p, _i64, _p],
                                  ctypes.c_int),
    "bigcn_forward_2layer": ([_p, _i64, _i32, _i64, _p, _p, _p, _i32, _i64, _p, _i32, _i64, _p,
                              _p, _i64, _p, _sz, _p, _i64, _p, _i64, _p, _p, _i32, _p],
                             ctypes.c_int),
    "bigcn_real_binary_gemm": ([_p, _i64, _i32, _i64, _p, _p, _p, _p, _i32, _i32, _p, _i64,
                                _p], ctypes.c_int),
    "bigcn_binary_real_gemm_workspace_bytes": ([_i32, _i32], _sz),
    "bigcn_binary_real_gemm": ([_p, _p, _i64, _i32, _i32, _p, _i32, _i64, _p, _sz, _p, _i64,
                                _p], ctypes.c_int),
    "bigcn_layer_ablation_workspace_bytes": ([_i32, _i64, _i32, _i32], _sz),
    "bigcn_layer_forward_ablation": ([_i32, _p, _i64, _i32, _i64, _p, _p, _p, _i32, _i64, _p,
                                      _p, _i64, _p, _sz, _p, _i64, _p], ctypes.c_int),
    "bigcn_inductive_layer_workspace_bytes": ([_i32, _i64, _i32, _i32], _sz),
    "bigcn_inductive_layer_forward": ([_i32, _p, _i64, _i32, _i64, _p, _p, _p, _i32, _i64, _p,
                                       _i64, _p, _p, _i64, _p, _sz, _p, _i64, _p], ctypes.c_int),
    "bigcn_pack_rows_bucketed": ([_p, _i64, _i32, _i64, _p, _p, _i32, _p, _i32, _p, _p],
                                 ctypes.c_int),
    "bigcn_pack_weights_bucketed": ([_p, _i32, _i32, _i64, _i32, _p, _i32, _p, _p], ctypes.c_int),
    "bigcn_xnor_gemm_bucketed": ([_p, _p, _i64, _p, _p, _i32, _i32, _i32, _i32, _p, _i64, _p],
                                 ctypes.c_int),
    "bigcn_layer_bucketed_workspace_bytes": ([_i64, _i32, _i32, _i32], _sz),
    "bigcn_layer_forward_bucketed": ([_i32, _p, _i64, _i32, _i64, _p, _p, _p, _i32, _i64, _p,
                                      _p, _i64, _p, _sz, _p, _i64, _p], ctypes.c_int),
    "bigcn_layer_forward_static": ([_p, _i64, _i32, _i64, _p, _p, _p, _i32, _i64, _p, _p, _i64,
                                    _p, _i64, _p], ctypes.c_int),
    "bigcn_checkpoint_groups": ([_i32], _i32),
    "bigcn_checkpoint_pack": ([_i32, _p, _i64, _i32, _i64, _p, _i64, _p, _i64, _p], ctypes.c_int),
    "bigcn_checkpoint_unpack": ([_i32, _p, _i64, _p, _i64, _i64, _i32, _p, _p, _p, _i64, _p],
                                ctypes.c_int),
    "bigcn_layer_norm_forward": ([_i32, _p, _i64, _i32, _i64, _p, _p, ctypes.c_float, _p, _i64,
                                  _p, _p, _p, _i64, _p, _i64, _p], ctypes.c_int),
    "bigcn_layer_norm_backward_workspace_bytes": ([_i64, _i32], _sz),
    "bigcn_layer_norm_backward": ([_i32, _p, _i64, _i32, _i64, _p, _p, _i64, _p, _p, _i64, _p,
                                   _i64, _p, _p, _i64, _p, _p, _p, _sz, _p], ctypes.c_int),
    "bigcn_checkpoint_weight_grad_workspace_bytes": ([_i64, _i32, _i32], _sz),
    "bigcn_checkpoint_weight_grad": ([_i32, _p, _i64, _p, _i64, _i64, _i32, _p, _p, _p, _i32,
                                      _i64, _p, _i64, _p, _p, _sz, _p], ctypes.c_int),
    "bigcn_rms_norm_forward": ([_i32, _p, _i64, _i32, _i64, _p, _i64, _p, ctypes.c_float, _p, _i64,
                                _p, _i64, _p, _p, _i64, _p, _i64, _p], ctypes.c_int),
    "bigcn_rms_norm_backward_workspace_bytes": ([_i64, _i32], _sz),
    "bigcn_rms_norm_backward": ([_i32, _p, _i64, _i32, _i64, _p, _p, _i64, _p, _i64, _p, _i64, _p,
                                 _p, _i64, _p, _i64, _p, _p, _sz, _p], ctypes.c_int),
    "bigcn_fp4_pack": ([_i32, _p, _i64, _i32, _i64, _p, _i64, _p, _i64, _p], ctypes.c_int),
    "bigcn_fp4_pack_columns": ([_i32, _p, _i32, _i32, _i64, _p, _i64, _p, _i64, _p], ctypes.c_int),
    "bigcn_fp4_unpack": ([_i32, _p, _i64, _p, _i64, _i64, _i32, _p, _i64, _p], ctypes.c_int),
    "bigcn_fp4_gemm": ([_i32, _p, _i64, _p, _i64, _i64, _p, _i64, _p, _i64, _i32, _i32, _p, _p,
                        _i64, _p], ctypes.c_int),
    "bigcn_grad_norm_workspace_bytes": ([_i32], _sz),
    "bigcn_grad_norm": ([_i32, _p, _p, _p, _p, _p, _sz, _p], ctypes.c_int),
    "bigcn_clip_grad_norm": ([_i32, _p, _p, _p, _p, ctypes.c_float, _p, _p, _sz, _p], ctypes.c_int),
    "bigcn_weighted_dinv": ([_p, _p, _i64, _i64, _p, _p], ctypes.c_int),
    "bigcn_spmm_norm_weighted": ([_p, _p, _p, _p, _i64, _i64, _p, _i64, _i32, _p, _i64, _p],
                                 ctypes.c_int),
    "bigcn_weighted_layer_workspace_bytes": ([_i64, _i32, _i32], _sz),
    "bigcn_weighted_layer_forward": ([_p, _i64, _i32, _i64, _p, _p, _p, _i32, _i64, _p, _p, _p,
                                      _i64, _p, _sz, _p, _i64, _p], ctypes.c_int),
}


class BigcnError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} returned {STATUS_NAMES.get(status, status)}")
        self.status = status


def library_path() -> str:
    return _build.LIB


def lib() -> ctypes.CDLL:
    """The loaded libbigcn.so. Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            path = _build.LIB
            if not os.path.exists(path):
                raise RuntimeError(
                    f"{path} is missing: build the CUDA library first "
                    "(python -c 'import __graft_entry__ as g; g.build()')")
            h = ctypes.CDLL(path)
            for name, (args, res) in SIGNATURES.items():
                fn = getattr(h, name)
                fn.argtypes = args
                fn.restype = res
            _lib = h
    return _lib


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None:
        # The private calls give the same handle without the Stream object (1 us against 4). Where
        # CUDA is not up, or not in this torch, its public call brings it up or says why not.
        if torch.cuda.is_initialized():
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return ctypes.c_void_p(stream.cuda_stream)
    return ctypes.c_void_p(int(stream))


def _ld(t):
    """Row stride in elements of a 2-D tensor whose rows are contiguous."""
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError("expected a 2-D tensor with unit column stride")
    return t.stride(0)


def _check(fn: str, status: int):
    if status != BIGCN_OK:
        raise BigcnError(fn, status)


def status_string(status: int) -> str:
    return lib().bigcn_status_string(status).decode()


def device_timeouts() -> int:
    """Bounded device waits that ran out since the last call (synchronizes)."""
    return int(lib().bigcn_device_timeouts())


def words_for(K: int) -> int:
    return int(lib().bigcn_words(K))


# ------------------------------------------------------ one-to-one entries ---
def bigcn_pack_rows(X, scale, shift, bits, alpha, stream=None, K=None):
    """Steps 1+2 (Sec. 6.2, Eqs. 7-8): bits, alpha <- X (N x K fp32)."""
    N, Kx = X.shape
    K = Kx if K is None else K
    _check("bigcn_pack_rows", lib().bigcn_pack_rows(
        _ptr(X), N, K, _ld(X), _ptr(scale), _ptr(shift), _ptr(bits), _ld(bits),
        _ptr(alpha), _stream(stream)))


def bigcn_pack_weights(Wt, bits, beta, stream=None):
    """Step 3 (Eqs. 3-4): bits (F x words), beta <- Wt (K x F fp32)."""
    K, F = Wt.shape
    _check("bigcn_pack_weights", lib().bigcn_pack_weights(
        _ptr(Wt), K, F, _ld(Wt), _ptr(bits), _ld(bits), _ptr(beta), _stream(stream)))


def bigcn_xnor_gemm(a_bits, alpha, b_bits, beta, K, Z, dots=None, stream=None):
    """Step 4 (Eqs. 11-12): Z = alpha_i beta_j (K - 2 popc(a_i ^ b_j))."""
    N, words = a_bits.shape
    F = b_bits.shape[0]
    if b_bits.shape[1] != words:
        raise ValueError("a_bits and b_bits must have the same row width")
    _check("bigcn_xnor_gemm", lib().bigcn_xnor_gemm(
        _ptr(a_bits), _ptr(alpha), N, _ptr(b_bits), _ptr(beta), F, K, words, _ptr(Z), _ld(Z),
        _ptr(dots), _stream(stream)))


def bigcn_spmm_norm(rowptr, colidx, Z, H, stream=None):
    """Step 5 (Eqs. 1, 13): H = D^-1/2 (A + I) D^-1/2 Z."""
    N = rowptr.shape[0] - 1
    F = Z.shape[1]
    _check("bigcn_spmm_norm", lib().bigcn_spmm_norm(
        _ptr(rowptr), _ptr(colidx) if colidx.numel() else None, N, colidx.numel(), _ptr(Z),
        _ld(Z), F, _ptr(H), _ld(H), _stream(stream)))


def bigcn_xnor_gemm_degscaled(a_bits, alpha, b_bits, beta, K, rowptr, Z, stream=None):
    """Step 4 with row i also scaled by 1/sqrt(dhat_i) (the source-side factor
    of Eq. 1's normalisation)."""
    N, words = a_bits.shape
    F = b_bits.shape[0]
    if b_bits.shape[1] != words:
        raise ValueError("a_bits and b_bits must have the same row width")
    _check("bigcn_xnor_gemm_degscaled", lib().bigcn_xnor_gemm_degscaled(
        _ptr(a_bits), _ptr(alpha), N, _ptr(b_bits), _ptr(beta), F, K, words, _ptr(rowptr),
        _ptr(Z), _ld(Z), _stream(stream)))


def bigcn_spmm_prescaled(rowptr, colidx, Z, H, stream=None):
    """Step 5 over rows that already carry their 1/sqrt(dhat_j)."""
    N = rowptr.shape[0] - 1
    F = Z.shape[1]
    _check("bigcn_spmm_prescaled", lib().bigcn_spmm_prescaled(
        _ptr(rowptr), _ptr(colidx) if colidx.numel() else None, N, colidx.numel(), _ptr(Z),
        _ld(Z), F, _ptr(H), _ld(H), _stream(stream)))


def bigcn_spmm_prescaled_rows(rowptr, colidx, Z, H, stream=None):
    """A block of output rows (H: n_rows x F) aggregated over a table of
    pre-scaled rows (Z: n_cols x F, the block's own rows first)."""
    n_rows, n_cols = H.shape[0], Z.shape[0]
    _check("bigcn_spmm_prescaled_rows", lib().bigcn_spmm_prescaled_rows(
        _ptr(rowptr), _ptr(colidx) if colidx.numel() else None, n_rows, n_cols, colidx.numel(),
        _ptr(Z), _ld(Z), Z.shape[1], _ptr(H), _ld(H), _stream(stream)))


def bigcn_layer_workspace_bytes(N: int, K: int, F: int) -> int:
    return int(lib().bigcn_layer_workspace_bytes(N, K, F))


def bigcn_layer_forward(X, scale, shift, Wt, rowptr, colidx, workspace, H, stream=None):
    """One fused layer (Eq. 13 with zeta of Eqs. 11-12)."""
    N, K = X.shape
    F = Wt.shape[1]
    _check("bigcn_layer_forward", lib().bigcn_layer_forward(
        _ptr(X), N, K, _ld(X), _ptr(scale), _ptr(shift), _ptr(Wt), F, _ld(Wt), _ptr(rowptr),
        _ptr(colidx) if colidx.numel() else None, colidx.numel(), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(H), _ld(H), _stream(stream)))


def bigcn_layer_forward_timed(X, scale, shift, Wt, rowptr, colidx, workspace, H, events,
                              stream=None):
    """bigcn_layer_forward recording ``events`` (torch.cuda.Event objects
    created with enable_timing=True and recorded once, so that the CUDA event
    exists) before each of its four kernels and after the last."""
    N, K = X.shape
    F = Wt.shape[1]
    ev = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
    _check("bigcn_layer_forward_timed", lib().bigcn_layer_forward_timed(
        _ptr(X), N, K, _ld(X), _ptr(scale), _ptr(shift), _ptr(Wt), F, _ld(Wt), _ptr(rowptr),
        _ptr(colidx) if colidx.numel() else None, colidx.numel(), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(H), _ld(H), ev, len(events),
        _stream(stream)))


# Which operands of Eq. 11 are binarized (enum bigcn_binarize).
BINARIZE = {"both": 0, "weights": 1, "features": 2}


def bigcn_real_binary_gemm(X, scale, shift, b_bits, beta, Z, stream=None):
    """Weights binarized, features real: Z = Y W~ (Y = X centred by
    scale/shift)."""
    N, K = X.shape
    F = beta.shape[0]
    _check("bigcn_real_binary_gemm", lib().bigcn_real_binary_gemm(
        _ptr(X), N, K, _ld(X), _ptr(scale), _ptr(shift), _ptr(b_bits), _ptr(beta), F,
        _ld(b_bits), _ptr(Z), _ld(Z), _stream(stream)))


def bigcn_binary_real_gemm_workspace_bytes(K: int, F: int) -> int:
    return int(lib().bigcn_binary_real_gemm_workspace_bytes(K, F))


def bigcn_binary_real_gemm(a_bits, alpha, K, Wt, workspace, Z, stream=None):
    """Features binarized, weights real: Z = H~ W (H~ = diag(alpha) signs)."""
    N = alpha.shape[0]
    F = Wt.shape[1]
    _check("bigcn_binary_real_gemm", lib().bigcn_binary_real_gemm(
        _ptr(a_bits), _ptr(alpha), N, K, _ld(a_bits), _ptr(Wt), F, _ld(Wt), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(Z), _ld(Z), _stream(stream)))


def bigcn_layer_ablation_workspace_bytes(binarize, N: int, K: int, F: int) -> int:
    return int(lib().bigcn_layer_ablation_workspace_bytes(BINARIZE.get(binarize, binarize),
                                                          N, K, F))


def bigcn_layer_forward_ablation(binarize, X, scale, shift, Wt, rowptr, colidx, workspace, H,
                                 stream=None):
    """One layer with the operands of Eq. 11 binarized as ``binarize`` says
    ("both", "weights", "features" or the enum's value)."""
    N, K = X.shape
    F = Wt.shape[1]
    _check("bigcn_layer_forward_ablation", lib().bigcn_layer_forward_ablation(
        BINARIZE.get(binarize, binarize), _ptr(X), N, K, _ld(X), _ptr(scale), _ptr(shift),
        _ptr(Wt), F, _ld(Wt), _ptr(rowptr), _ptr(colidx) if colidx.numel() else None,
        colidx.numel(), _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(H),
        _ld(H), _stream(stream)))


def bigcn_pack_rows_bucketed(X, scale, shift, B, bits, alpha, stream=None):
    """Sub-row bucketing (Sec. 4.1): packed signs and alpha (N x nb) per
    bucket of B features (a multiple of 64)."""
    N, K = X.shape
    _check("bigcn_pack_rows_bucketed", lib().bigcn_pack_rows_bucketed(
        _ptr(X), N, K, _ld(X), _ptr(scale), _ptr(shift), B, _ptr(bits), _ld(bits), _ptr(alpha),
        _stream(stream)))


def bigcn_pack_weights_bucketed(Wt, B, bits, beta, stream=None):
    """Packed weight columns and beta (F x nb) per bucket of B entries."""
    K, F = Wt.shape
    _check("bigcn_pack_weights_bucketed", lib().bigcn_pack_weights_bucketed(
        _ptr(Wt), K, F, _ld(Wt), B, _ptr(bits), _ld(bits), _ptr(beta), _stream(stream)))


def bigcn_xnor_gemm_bucketed(a_bits, alpha, b_bits, beta, K, B, Z, stream=None):
    """Z = sum over buckets of alpha_ib beta_jb dot_b."""
    N = a_bits.shape[0]
    F = b_bits.shape[0]
    _check("bigcn_xnor_gemm_bucketed", lib().bigcn_xnor_gemm_bucketed(
        _ptr(a_bits), _ptr(alpha), N, _ptr(b_bits), _ptr(beta), F, K, _ld(a_bits), B, _ptr(Z),
        _ld(Z), _stream(stream)))


def bigcn_layer_bucketed_workspace_bytes(N: int, K: int, F: int, B: int) -> int:
    return int(lib().bigcn_layer_bucketed_workspace_bytes(N, K, F, B))


def bigcn_layer_forward_bucketed(B, X, scale, shift, Wt, rowptr, colidx, workspace, H,
                                 stream=None):
    """One layer with bucketed binarization (buckets of B features)."""
    N, K = X.shape
    F = Wt.shape[1]
    _check("bigcn_layer_forward_bucketed", lib().bigcn_layer_forward_bucketed(
        B, _ptr(X), N, K, _ld(X), _ptr(scale), _ptr(shift), _ptr(Wt), F, _ld(Wt), _ptr(rowptr),
        _ptr(colidx) if colidx.numel() else None, colidx.numel(), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(H), _ld(H), _stream(stream)))


# Aggregators of the inductive layers (enum bigcn_aggregator).
AGGREGATOR = {"gcn": 0, "mean": 1, "sage": 2}


def bigcn_inductive_layer_workspace_bytes(aggregator, N: int, K: int, F: int) -> int:
    return int(lib().bigcn_inductive_layer_workspace_bytes(
        AGGREGATOR.get(aggregator, aggregator), N, K, F))


def bigcn_inductive_layer_forward(aggregator, X, scale, shift, Wt, rowptr, colidx, workspace, H,
                                  W_neigh=None, stream=None):
    """One binarized inductive layer: the product, then the ``aggregator``
    ("gcn", "mean", "sage"; "sage" takes W_neigh)."""
    N, K = X.shape
    F = Wt.shape[1]
    _check("bigcn_inductive_layer_forward", lib().bigcn_inductive_layer_forward(
        AGGREGATOR.get(aggregator, aggregator), _ptr(X), N, K, _ld(X), _ptr(scale), _ptr(shift),
        _ptr(Wt), F, _ld(Wt), _ptr(W_neigh), _ld(W_neigh) if W_neigh is not None else 0,
        _ptr(rowptr), _ptr(colidx) if colidx.numel() else None, colidx.numel(), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(H), _ld(H), _stream(stream)))


def bigcn_layer_backward_workspace_bytes(N: int, K: int, F: int) -> int:
    return int(lib().bigcn_layer_backward_workspace_bytes(N, K, F))


def bigcn_layer_backward(X, scale, shift, Wt, rowptr, colidx, dH, workspace, dW, dX=None,
                         stream=None):
    """Algorithm 1 for one layer: dW (K x F, Eq. bp-W) and optionally dX
    (N x K, Eq. bp-H) from dH = dL/dH^(l+1) (N x F)."""
    N, K = X.shape
    F = Wt.shape[1]
    _check("bigcn_layer_backward", lib().bigcn_layer_backward(
        _ptr(X), N, K, _ld(X), _ptr(scale), _ptr(shift), _ptr(Wt), F, _ld(Wt), _ptr(rowptr),
        _ptr(colidx) if colidx.numel() else None, colidx.numel(), _ptr(dH), _ld(dH), _ptr(dX),
        _ld(dX) if dX is not None else 0, _ptr(dW), _ld(dW), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def bigcn_forward_2layer_workspace_bytes(N: int, K: int, Fh: int, Fo: int) -> int:
    return int(lib().bigcn_forward_2layer_workspace_bytes(N, K, Fh, Fo))


def bigcn_forward_2layer_launches(N: int, K: int, Fh: int, Fo: int) -> int:
    n = int(lib().bigcn_forward_2layer_launches(N, K, Fh, Fo))
    if n < 0:
        raise BigcnError("bigcn_forward_2layer_launches", 1)
    return n


def bigcn_forward_2layer_aggregation(K: int, Fh: int, Fo: int) -> int:
    """1 when bigcn_forward_2layer aggregates on the tensor cores (fp16 dots),
    0 on the CUDA cores."""
    n = int(lib().bigcn_forward_2layer_aggregation(K, Fh, Fo))
    if n < 0:
        raise BigcnError("bigcn_forward_2layer_aggregation", 1)
    return n


def bigcn_forward_2layer(X, scale, shift, W1, W2, rowptr, colidx, workspace, out, H1=None,
                         events=None, stream=None, pred=None):
    """The two-layer forward of Sec. 6.2 (hidden layer on centred X, output
    layer on H1 raw). ``events``: torch.cuda.Event objects (created with
    enable_timing=True, external=True and recorded once) to be recorded
    before each kernel and after the last. ``pred``: optional int32 tensor of
    N that receives each row's argmax of the logits."""
    N, K = X.shape
    Fh, Fo = W1.shape[1], W2.shape[1]
    if W2.shape[0] != Fh:
        raise ValueError("W2 must have as many rows as W1 has columns")
    if events:
        ev = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
        n_ev = len(events)
    else:
        ev, n_ev = None, 0
    _check("bigcn_forward_2layer", lib().bigcn_forward_2layer(
        _ptr(X), N, K, _ld(X), _ptr(scale), _ptr(shift), _ptr(W1), Fh, _ld(W1), _ptr(W2), Fo,
        _ld(W2), _ptr(rowptr), _ptr(colidx) if colidx.numel() else None, colidx.numel(),
        _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(H1),
        _ld(H1) if H1 is not None else 0, _ptr(out), _ld(out), _ptr(pred), ev, n_ev,
        _stream(stream)))


def bigcn_layer_forward_static(X, scale, shift, Wt, rowptr, colidx, H, stream=None):
    """The layer on the library's own static device scratch, for callers that
    cannot allocate device memory (no workspace argument; layers whose
    workspace exceeds STATIC_SCRATCH_BYTES are refused)."""
    N, K = X.shape
    F = Wt.shape[1]
    _check("bigcn_layer_forward_static", lib().bigcn_layer_forward_static(
        _ptr(X), N, K, _ld(X), _ptr(scale), _ptr(shift), _ptr(Wt), F, _ld(Wt), _ptr(rowptr),
        _ptr(colidx) if colidx.numel() else None, colidx.numel(), _ptr(H), _ld(H),
        _stream(stream)))


def bigcn_weighted_dinv(rowptr, values, dinv, stream=None):
    """dinv_i = 1/sqrt(1 + sum of row i's edge weights) (Sec. 3, weighted A)."""
    N = rowptr.numel() - 1
    _check("bigcn_weighted_dinv", lib().bigcn_weighted_dinv(
        _ptr(rowptr), _ptr(values) if values.numel() else None, N, values.numel(), _ptr(dinv),
        _stream(stream)))


def bigcn_spmm_norm_weighted(rowptr, colidx, values, dinv, Z, H, stream=None):
    N, F = Z.shape
    _check("bigcn_spmm_norm_weighted", lib().bigcn_spmm_norm_weighted(
        _ptr(rowptr), _ptr(colidx) if colidx.numel() else None,
        _ptr(values) if values.numel() else None, _ptr(dinv), N, colidx.numel(), _ptr(Z), _ld(Z),
        F, _ptr(H), _ld(H), _stream(stream)))


def bigcn_weighted_layer_workspace_bytes(N: int, K: int, F: int) -> int:
    return int(lib().bigcn_weighted_layer_workspace_bytes(N, K, F))


def bigcn_weighted_layer_forward(X, scale, shift, Wt, rowptr, colidx, values, workspace, H,
                                 stream=None):
    N, K = X.shape
    F = Wt.shape[1]
    _check("bigcn_weighted_layer_forward", lib().bigcn_weighted_layer_forward(
        _ptr(X), N, K, _ld(X), _ptr(scale), _ptr(shift), _ptr(Wt), F, _ld(Wt), _ptr(rowptr),
        _ptr(colidx) if colidx.numel() else None, _ptr(values) if values.numel() else None,
        colidx.numel(), _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(H),
        _ld(H), _stream(stream)))


# Element types of the row-wise operators (enum bigcn_dtype).
DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _dtype(t, like=None):
    """The bigcn_dtype of a tensor (which must be ``like``'s, where given)."""
    if t.dtype not in DTYPE or (like is not None and t.dtype != like.dtype):
        raise ValueError("expected float32, bfloat16 or float16 tensors, all of one type")
    return DTYPE[t.dtype]


def _vector(t, n, what):
    """Pointer of a contiguous fp32 vector of n entries (None: NULL)."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous float32 vector of {n} entries")
    return t.data_ptr()


def _kept(q, exps, N, K):
    """(q, ldq, exps, lde) of a checkpoint of N x K, or NULLs for none."""
    if q is None or exps is None:
        return _ptr(q), 0, _ptr(exps), 0
    if q.dtype != torch.int8 or exps.dtype != torch.uint8 or q.shape != (N, K) or \
            exps.shape != (N, (K + 31) // 32):
        raise ValueError("a checkpoint is q (N x K int8) and exps (N x ceil(K / 32) uint8)")
    return _ptr(q), _ld(q), _ptr(exps), _ld(exps)


def _matrix(t, N, K, what, like=None):
    """(pointer, row stride) of an N x K matrix (None: NULL)."""
    if t is None:
        return None, 0
    if t.shape != (N, K):
        raise ValueError(f"{what} must be {N} x {K}")
    if like is not None:
        _dtype(t, like)
    return _ptr(t), _ld(t)


def _bytes(workspace):
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


def bigcn_checkpoint_groups(K: int) -> int:
    return int(lib().bigcn_checkpoint_groups(K))


def bigcn_checkpoint_pack(X, q, exps, stream=None):
    """X (N x K, fp32, bf16 or fp16) to 8 bits: q (N x K int8) and exps
    (N x ceil(K/32) uint8), views of rows of the strides that the header asks for
    (:func:`checkpoint_buffers`)."""
    N, K = X.shape
    _check("bigcn_checkpoint_pack", lib().bigcn_checkpoint_pack(
        _dtype(X), _ptr(X), N, K, _ld(X), *_kept(q, exps, N, K), _stream(stream)))


def bigcn_checkpoint_unpack(q, exps, X, gamma=None, beta=None, stream=None):
    """X = gamma v + beta from the checkpoint v."""
    N, K = X.shape
    _check("bigcn_checkpoint_unpack", lib().bigcn_checkpoint_unpack(
        _dtype(X), *_kept(q, exps, N, K), N, K, _vector(gamma, K, "gamma"),
        _vector(beta, K, "beta"), _ptr(X), _ld(X), _stream(stream)))


def bigcn_layer_norm_forward(X, gamma, beta, eps, Y, mean=None, rstd=None, q=None, exps=None,
                             stream=None):
    """Y = gamma xhat + beta, xhat the rows of X normalised; mean and rstd (N fp32) and the
    checkpoint of xhat where given. gamma, beta: None for 1, 0."""
    N, K = X.shape
    _check("bigcn_layer_norm_forward", lib().bigcn_layer_norm_forward(
        _dtype(X), _ptr(X), N, K, _ld(X), _vector(gamma, K, "gamma"), _vector(beta, K, "beta"),
        eps, *_matrix(Y, N, K, "Y", X), _vector(mean, N, "mean"), _vector(rstd, N, "rstd"),
        *_kept(q, exps, N, K), _stream(stream)))


def bigcn_layer_norm_backward_workspace_bytes(N: int, K: int) -> int:
    return int(lib().bigcn_layer_norm_backward_workspace_bytes(N, K))


def bigcn_layer_norm_backward(dY, gamma, rstd, workspace, X=None, mean=None, q=None, exps=None,
                              dX=None, dgamma=None, dbeta=None, stream=None):
    """The gradients of the norm's input and parameters (those given) from dY, with xhat from
    X and mean or from the checkpoint q, exps. workspace: None where neither dgamma nor dbeta
    is given."""
    N, K = dY.shape
    x, ldx = _matrix(X, N, K, "X", dY)
    dx, lddx = _matrix(dX, N, K, "dX", dY)
    _check("bigcn_layer_norm_backward", lib().bigcn_layer_norm_backward(
        _dtype(dY), _ptr(dY), N, K, _ld(dY), _vector(gamma, K, "gamma"), x, ldx,
        _vector(mean, N, "mean"), *_kept(q, exps, N, K), _vector(rstd, N, "rstd"), dx, lddx,
        _vector(dgamma, K, "dgamma"), _vector(dbeta, K, "dbeta"), _ptr(workspace),
        _bytes(workspace), _stream(stream)))


def bigcn_checkpoint_weight_grad_workspace_bytes(N: int, K: int, F: int) -> int:
    return int(lib().bigcn_checkpoint_weight_grad_workspace_bytes(N, K, F))


def bigcn_checkpoint_weight_grad(q, exps, dZ, workspace, dW, gamma=None, beta=None, db=None,
                                 stream=None):
    """dW (K x F fp32) and db (F) of Z = (gamma v + beta) W + b from the checkpoint v and dZ."""
    N, F = dZ.shape
    K = dW.shape[0]
    if dW.dtype != torch.float32:
        raise ValueError("dW must be float32")
    dw, lddw = _matrix(dW, K, F, "dW")
    _check("bigcn_checkpoint_weight_grad", lib().bigcn_checkpoint_weight_grad(
        _dtype(dZ), *_kept(q, exps, N, K), N, K, _vector(gamma, K, "gamma"),
        _vector(beta, K, "beta"), _ptr(dZ), F, _ld(dZ), dw, lddw, _vector(db, F, "db"),
        _ptr(workspace), _bytes(workspace), _stream(stream)))


# The calls below check a tensor's device along with its type and shape, each in as few torch calls
# as do it: on one row a call's time is these checks' (9.5 us, of which the argument passing is 3).
def _current(stream):
    """(the current CUDA device, or None before CUDA is up; the stream's handle)."""
    if not torch.cuda.is_initialized():
        return None, stream
    device = torch._C._cuda_getDevice()
    if stream is None:
        return device, torch._C._cuda_getCurrentRawStream(device)
    return device, _stream(stream)


def _elsewhere(what):
    raise ValueError(f"{what} must be on the current CUDA device, whose stream the call takes")


def _rows(t, shape, dtype, device, what):
    """(pointer, row stride) of a matrix of ``shape`` and ``dtype`` (None: NULL)."""
    if t is None:
        return None, 0
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{what} must be {tuple(shape)} {dtype}")
    ld, unit = t.stride()
    if unit != 1:
        raise ValueError(f"{what} must have unit column stride")
    if t.get_device() != device:
        _elsewhere(what)
    return t.data_ptr(), ld


def _floats(t, n, device, what):
    """Pointer of a contiguous fp32 vector of n entries (None: NULL)."""
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous float32 vector of {n} entries")
    if t.get_device() != device:
        _elsewhere(what)
    return t.data_ptr()


def _room(workspace, device):
    """(pointer, bytes) of a workspace (None: NULL)."""
    if workspace is None:
        return None, 0
    if workspace.get_device() != device:
        _elsewhere("workspace")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _checkpoint(q, exps, N, K, device):
    if q is None or exps is None:
        return _ptr(q), 0, _ptr(exps), 0
    kept = _kept(q, exps, N, K)
    if q.get_device() != device or exps.get_device() != device:
        _elsewhere("a checkpoint")
    return kept


def bigcn_rms_norm_forward(X, gamma, eps, R=None, S=None, Y=None, rstd=None, q=None, exps=None,
                           stream=None):
    """S = X + R (X without R), Y = gamma shat with shat the rows of S over their root mean
    square; rstd (N fp32) and the checkpoint of shat where given. S may be R or X. gamma: None
    for 1."""
    device, stream = _current(stream)
    shape, t = X.shape, X.dtype
    N, K = shape
    dtype = _dtype(X)
    x, ldx = _rows(X, shape, t, device, "X")
    r, ldr = _rows(R, shape, t, device, "R")
    s, lds = _rows(S, shape, t, device, "S")
    y, ldy = _rows(Y, shape, t, device, "Y")
    g, out = _floats(gamma, K, device, "gamma"), _floats(rstd, N, device, "rstd")
    q, ldq, exps, lde = _checkpoint(q, exps, N, K, device)
    _check("bigcn_rms_norm_forward", lib().bigcn_rms_norm_forward(
        dtype, x, N, K, ldx, r, ldr, g, eps, s, lds, y, ldy, out, q, ldq, exps, lde, stream))


def bigcn_rms_norm_backward_workspace_bytes(N: int, K: int) -> int:
    return int(lib().bigcn_rms_norm_backward_workspace_bytes(N, K))


def bigcn_rms_norm_backward(dY, gamma, rstd, workspace, S=None, q=None, exps=None, dS=None, dX=None,
                            dgamma=None, stream=None):
    """dX (of the sum's addends alike) and dgamma (those given) from dY, with shat from the sum S or
    from the checkpoint q, exps; dS, which dX may be, is added to dX. workspace: None where dgamma is
    not given."""
    device, stream = _current(stream)
    shape, t = dY.shape, dY.dtype
    N, K = shape
    dtype = _dtype(dY)
    dy, lddy = _rows(dY, shape, t, device, "dY")
    s, lds = _rows(S, shape, t, device, "S")
    ds, ldds = _rows(dS, shape, t, device, "dS")
    dx, lddx = _rows(dX, shape, t, device, "dX")
    g, r = _floats(gamma, K, device, "gamma"), _floats(rstd, N, device, "rstd")
    out = _floats(dgamma, K, device, "dgamma")
    q, ldq, exps, lde = _checkpoint(q, exps, N, K, device)
    ws, ws_bytes = _room(workspace, device)
    _check("bigcn_rms_norm_backward", lib().bigcn_rms_norm_backward(
        dtype, dy, N, K, lddy, g, s, lds, q, ldq, exps, lde, r, ds, ldds, dx, lddx, out, ws,
        ws_bytes, stream))


def _fp4(q, exps, N, K, device, what):
    """(q, ldq, exps, lde) of N 4-bit rows of K columns."""
    if q.dtype is not torch.uint8 or exps.dtype is not torch.uint8 or \
            q.shape != (N, (K + 1) // 2) or exps.shape != (N, (K + 31) // 32):
        raise ValueError(f"{what}: 4-bit rows are q (N x ceil(K / 2)) and exps (N x ceil(K / 32)), "
                         "both uint8")
    ldq, unit = q.stride()
    lde, unit_e = exps.stride()
    if unit != 1 or unit_e != 1:
        raise ValueError(f"{what} must have unit column stride")
    if q.get_device() != device or exps.get_device() != device:
        _elsewhere(what)
    return q.data_ptr(), ldq, exps.data_ptr(), lde


def bigcn_fp4_pack(X, q, exps, stream=None):
    """X (N x K, fp32, bf16 or fp16) to 4 bits: q (N x ceil(K/2) uint8) and exps (N x ceil(K/32)
    uint8), views of rows of the strides that the header asks for (:func:`fp4_buffers`)."""
    device, stream = _current(stream)
    N, K = X.shape
    dtype, (x, ldx) = _dtype(X), _rows(X, X.shape, X.dtype, device, "X")
    _check("bigcn_fp4_pack", lib().bigcn_fp4_pack(
        dtype, x, N, K, ldx, *_fp4(q, exps, N, K, device, "X"), stream))


def bigcn_fp4_pack_columns(W, q, exps, stream=None):
    """The columns of W (K x F) to F 4-bit rows of K."""
    device, stream = _current(stream)
    K, F = W.shape
    dtype, (w, ldw) = _dtype(W), _rows(W, W.shape, W.dtype, device, "W")
    _check("bigcn_fp4_pack_columns", lib().bigcn_fp4_pack_columns(
        dtype, w, K, F, ldw, *_fp4(q, exps, F, K, device, "W"), stream))


def bigcn_fp4_unpack(q, exps, X, stream=None):
    """X (N x K) from its 4 bits."""
    device, stream = _current(stream)
    N, K = X.shape
    dtype, (x, ldx) = _dtype(X), _rows(X, X.shape, X.dtype, device, "X")
    _check("bigcn_fp4_unpack", lib().bigcn_fp4_unpack(
        dtype, *_fp4(q, exps, N, K, device, "X"), N, K, x, ldx, stream))


def bigcn_fp4_gemm(aq, a_exps, bq, b_exps, K, Z, bias=None, stream=None):
    """Z = A B^T + bias (N x F) of the 4-bit rows A (N x K) and B (F x K)."""
    device, stream = _current(stream)
    N, F = Z.shape
    dtype, (z, ldz) = _dtype(Z), _rows(Z, Z.shape, Z.dtype, device, "Z")
    a, lda, ae, ldae = _fp4(aq, a_exps, N, K, device, "A")
    b, ldb, be, ldbe = _fp4(bq, b_exps, F, K, device, "B")
    _check("bigcn_fp4_gemm", lib().bigcn_fp4_gemm(
        dtype, a, lda, ae, ldae, N, b, ldb, be, ldbe, F, K, _floats(bias, F, device, "bias"), z, ldz,
        stream))


class TensorList:
    """Contiguous fp32, bf16 or fp16 tensors of any shapes as the calls over many tensors take
    them: built once and kept by a program whose gradients stay where they are (it holds them)."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        n = len(self.tensors)
        for t in self.tensors:
            if not t.is_contiguous():
                raise ValueError("expected contiguous tensors")
        self.dtypes = (_i32 * n)(*[_dtype(t) for t in self.tensors])
        self.pointers = (_p * n)(*[t.data_ptr() for t in self.tensors])
        self.counts = (_i64 * n)(*[t.numel() for t in self.tensors])
        self.devices = {t.get_device() for t in self.tensors}

    def __len__(self):
        return len(self.tensors)


def _list(tensors):
    return tensors if isinstance(tensors, TensorList) else TensorList(tensors)


def bigcn_grad_norm_workspace_bytes(tensors) -> int:
    """For a list of tensors (or their number)."""
    n = tensors if isinstance(tensors, int) else len(tensors)
    return int(lib().bigcn_grad_norm_workspace_bytes(n))


def bigcn_grad_norm(tensors, norm, workspace, stream=None):
    """norm (one fp32) = the norm of all tensors together (a :class:`TensorList` or tensors)."""
    device, stream = _current(stream)
    t, out = _list(tensors), _floats(norm, 1, device, "norm")
    if t.devices and t.devices != {device}:
        _elsewhere("tensors")
    ws, ws_bytes = _room(workspace, device)
    _check("bigcn_grad_norm", lib().bigcn_grad_norm(
        len(t), t.dtypes, t.pointers, t.counts, out, ws, ws_bytes, stream))


def bigcn_clip_grad_norm(tensors, max_norm, norm, workspace, out=None, stream=None):
    """norm as above, and out (None: the tensors themselves) = tensors min(1, max_norm / norm)."""
    device, stream = _current(stream)
    t, n = _list(tensors), _floats(norm, 1, device, "norm")
    o = t if out is None else _list(out)
    if o is not t and (bytes(o.counts) != bytes(t.counts) or bytes(o.dtypes) != bytes(t.dtypes)):
        raise ValueError("out must be tensors of the same types and lengths")
    if t.devices and (t.devices != {device} or o.devices != {device}):
        _elsewhere("tensors")
    ws, ws_bytes = _room(workspace, device)
    _check("bigcn_clip_grad_norm", lib().bigcn_clip_grad_norm(
        len(t), t.dtypes, t.pointers, o.pointers, t.counts, max_norm, n, ws, ws_bytes, stream))


# ------------------------------------------------- allocating conveniences ---
def pack_rows(X, scale=None, shift=None, stream=None):
    N, K = X.shape
    bits = torch.empty((N, words_for(K)), dtype=torch.int64, device=X.device)
    alpha = torch.empty(N, dtype=torch.float32, device=X.device)
    bigcn_pack_rows(X, scale, shift, bits, alpha, stream)
    return bits, alpha


def pack_weights(Wt, stream=None):
    K, F = Wt.shape
    bits = torch.empty((F, words_for(K)), dtype=torch.int64, device=Wt.device)
    beta = torch.empty(F, dtype=torch.float32, device=Wt.device)
    bigcn_pack_weights(Wt, bits, beta, stream)
    return bits, beta


def xnor_gemm(a_bits, alpha, b_bits, beta, K, with_dots=False, stream=None):
    N, F = a_bits.shape[0], b_bits.shape[0]
    Z = torch.empty((N, F), dtype=torch.float32, device=a_bits.device)
    dots = torch.empty((N, F), dtype=torch.int32, device=a_bits.device) if with_dots else None
    bigcn_xnor_gemm(a_bits, alpha, b_bits, beta, K, Z, dots, stream)
    return (Z, dots) if with_dots else Z


def spmm_norm(rowptr, colidx, Z, stream=None):
    H = torch.empty_like(Z, memory_format=torch.contiguous_format)
    bigcn_spmm_norm(rowptr, colidx, Z, H, stream)
    return H


def layer_workspace(N, K, F, device):
    nbytes = bigcn_layer_workspace_bytes(N, K, F)
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)


def layer_forward(X, Wt, rowptr, colidx, scale=None, shift=None, workspace=None, stream=None):
    N, K = X.shape
    F = Wt.shape[1]
    if workspace is None:
        workspace = layer_workspace(N, K, F, X.device)
    H = torch.empty((N, F), dtype=torch.float32, device=X.device)
    bigcn_layer_forward(X, scale, shift, Wt, rowptr, colidx, workspace, H, stream)
    return H


def checkpoint_buffers(N, K, device):
    """(q, exps) for a checkpoint of N x K: views of rows padded as the header asks."""
    q = torch.empty((N, (K + 15) // 16 * 16), dtype=torch.int8, device=device)
    groups = (K + 31) // 32
    exps = torch.empty((N, (groups + 3) // 4 * 4), dtype=torch.uint8, device=device)
    return q[:, :K], exps[:, :groups]


def checkpoint_pack(X, stream=None):
    q, exps = checkpoint_buffers(*X.shape, X.device)
    bigcn_checkpoint_pack(X, q, exps, stream)
    return q, exps


def checkpoint_unpack(q, exps, dtype=torch.float32, gamma=None, beta=None, stream=None):
    X = torch.empty(q.shape, dtype=dtype, device=q.device)
    bigcn_checkpoint_unpack(q, exps, X, gamma, beta, stream)
    return X


def layer_norm_forward(X, gamma=None, beta=None, eps=1e-5, checkpoint=True, stream=None):
    """(Y, mean, rstd, q, exps); without ``checkpoint`` the last two are None."""
    N, K = X.shape
    Y = torch.empty((N, K), dtype=X.dtype, device=X.device)
    mean = torch.empty(N, dtype=torch.float32, device=X.device)
    rstd = torch.empty_like(mean)
    q, exps = checkpoint_buffers(N, K, X.device) if checkpoint else (None, None)
    bigcn_layer_norm_forward(X, gamma, beta, eps, Y, mean, rstd, q, exps, stream)
    return Y, mean, rstd, q, exps


def layer_norm_backward(dY, gamma, rstd, X=None, mean=None, q=None, exps=None, stream=None):
    """(dX, dgamma, dbeta) with xhat from X and mean or from q and exps."""
    N, K = dY.shape
    ws = torch.empty(bigcn_layer_norm_backward_workspace_bytes(N, K), dtype=torch.uint8,
                     device=dY.device)
    dX = torch.empty((N, K), dtype=dY.dtype, device=dY.device)
    dgamma = torch.empty(K, dtype=torch.float32, device=dY.device)
    dbeta = torch.empty_like(dgamma)
    bigcn_layer_norm_backward(dY, gamma, rstd, ws, X, mean, q, exps, dX, dgamma, dbeta, stream)
    return dX, dgamma, dbeta


def checkpoint_weight_grad(q, exps, dZ, gamma=None, beta=None, stream=None):
    """(dW, db)."""
    N, F = dZ.shape
    K = q.shape[1]
    ws = torch.empty(bigcn_checkpoint_weight_grad_workspace_bytes(N, K, F), dtype=torch.uint8,
                     device=dZ.device)
    dW = torch.empty((K, F), dtype=torch.float32, device=dZ.device)
    db = torch.empty(F, dtype=torch.float32, device=dZ.device)
    bigcn_checkpoint_weight_grad(q, exps, dZ, ws, dW, gamma, beta, db, stream)
    return dW, db


def rms_norm_forward(X, gamma=None, eps=1e-5, R=None, checkpoint=True, stream=None):
    """(Y, S, rstd, q, exps); S is X without R, q and exps None without ``checkpoint``."""
    N, K = X.shape
    Y = torch.empty((N, K), dtype=X.dtype, device=X.device)
    S = torch.empty_like(Y) if R is not None else None
    rstd = torch.empty(N, dtype=torch.float32, device=X.device)
    q, exps = checkpoint_buffers(N, K, X.device) if checkpoint else (None, None)
    bigcn_rms_norm_forward(X, gamma, eps, R, S, Y, rstd, q, exps, stream)
    return Y, X if S is None else S, rstd, q, exps


def rms_norm_backward(dY, gamma, rstd, S=None, q=None, exps=None, dS=None, stream=None):
    """(dX, dgamma) with shat from S or from q and exps."""
    N, K = dY.shape
    ws = torch.empty(bigcn_rms_norm_backward_workspace_bytes(N, K), dtype=torch.uint8,
                     device=dY.device)
    dX = torch.empty((N, K), dtype=dY.dtype, device=dY.device)
    dgamma = torch.empty(K, dtype=torch.float32, device=dY.device)
    bigcn_rms_norm_backward(dY, gamma, rstd, ws, S, q, exps, dS, dX, dgamma, stream)
    return dX, dgamma


def fp4_buffers(N, K, device):
    """(q, exps) for N 4-bit rows of K columns: views of rows padded as the header asks."""
    groups = (K + 31) // 32
    q = torch.empty((N, groups * 16), dtype=torch.uint8, device=device)
    exps = torch.empty((N, (groups + 3) // 4 * 4), dtype=torch.uint8, device=device)
    return q[:, :(K + 1) // 2], exps[:, :groups]


def fp4_pack(X, stream=None):
    q, exps = fp4_buffers(*X.shape, X.device)
    bigcn_fp4_pack(X, q, exps, stream)
    return q, exps


def fp4_pack_columns(W, stream=None):
    q, exps = fp4_buffers(W.shape[1], W.shape[0], W.device)
    bigcn_fp4_pack_columns(W, q, exps, stream)
    return q, exps


def fp4_unpack(q, exps, K, dtype=torch.float32, stream=None):
    X = torch.empty((q.shape[0], K), dtype=dtype, device=q.device)
    bigcn_fp4_unpack(q, exps, X, stream)
    return X


def fp4_gemm(aq, a_exps, bq, b_exps, K, bias=None, dtype=torch.float32, stream=None):
    Z = torch.empty((aq.shape[0], bq.shape[0]), dtype=dtype, device=aq.device)
    bigcn_fp4_gemm(aq, a_exps, bq, b_exps, K, Z, bias, stream)
    return Z


def _norm_buffers(tensors):
    tensors = _list(tensors)
    device = tensors.tensors[0].device if len(tensors) else torch.device("cuda")
    ws = torch.empty(bigcn_grad_norm_workspace_bytes(tensors), dtype=torch.uint8, device=device)
    return tensors, torch.empty(1, dtype=torch.float32, device=device), ws


def grad_norm(tensors, stream=None):
    """The norm of all tensors together (a tensor of one fp32)."""
    tensors, norm, ws = _norm_buffers(tensors)
    bigcn_grad_norm(tensors, norm, ws, stream)
    return norm


def clip_grad_norm(tensors, max_norm, stream=None):
    """Scales the tensors in place to at most ``max_norm`` together; their norm before."""
    tensors, norm, ws = _norm_buffers(tensors)
    bigcn_clip_grad_norm(tensors, max_norm, norm, ws, stream=stream)
    return norm
