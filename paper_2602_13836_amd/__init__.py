"""Python binding of libspecvocab.so (the C ABI declared in include/specvocab.h).

Argument marshalling only: every step of the draft-step path runs in the HIP kernels of the
library.  torch is used for device memory and the current stream, nothing else.  There is no
CPU fallback: if the library has not been built, or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import NamedTuple, Optional, Tuple, Union

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspecvocab.so")

SV_OK = 0
SV_F32, SV_BF16 = 0, 1
SV_IDX_PER_ROW, SV_IDX_PER_STEP = 0, 1
SV_OP_SELECT, SV_OP_SUBSET_LOGITS, SV_OP_DRAFT_TOPK, SV_OP_DENSE_LOGITS, SV_OP_DRAFT_STEP = 0, 1, 2, 3, 4
SV_OP_INDEXED_HEAD_NAIVE = 5
SV_OP_AUX_LOG_SOFTMAX = 6
SV_OP_QUANTIZED_DENSE_LOGITS, SV_OP_QUANTIZED_SUBSET_LOGITS, SV_OP_QUANTIZED_SAMPLE_STEP, SV_OP_SAMPLE = 7, 8, 9, 10
SV_OP_TOKEN_LOGPROBS, SV_OP_DISTILL = 11, 12
SV_E4M3 = 2              # rows in 8 bits, where a workspace size is asked for
SV_IDX_PADDED = 4        # OR into idx_mode: the list may hold padding slots (-1)
SV_IDX_SORTED = 8        # OR into idx_mode: every list is sorted by ascending id (what select emits)
MAX_KD = 64
MAX_TOP, MAX_GIVEN, MAX_TEACHER = 64, 64, 512
SELECT_SAMPLE = 8192     # sampled tokens of a batch's selection, d' > 512: ids floor(j * V / SELECT_SAMPLE)
SELECT_CODE_SAMPLE = 4096            # ... with one byte per score in memory: floor(j * V / SELECT_CODE_SAMPLE), every second one of those

EXPORTS = (
    "specvocab_version",
    "specvocab_init",
    "specvocab_status_string",
    "specvocab_workspace_bytes",
    "specvocab_select",
    "specvocab_select_static",
    "specvocab_select_threshold",
    "specvocab_subset_logits",
    "specvocab_draft_topk",
    "specvocab_draft_step",
    "specvocab_indexed_head_naive",
    "specvocab_pack_rows",
    "specvocab_aux_log_softmax",
    "specvocab_stream_read_probe",
    "specvocab_dense_logits",
    "specvocab_quantize_rows",
    "specvocab_rms_norm",
    "specvocab_quantized_dense_logits",
    "specvocab_quantized_subset_logits",
    "specvocab_sample",
    "specvocab_quantized_sample_step",
    "specvocab_token_logprobs",
    "specvocab_token_logprobs_grad",
    "specvocab_distill",
    "specvocab_distill_grad",
)


class SpecVocabError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({status_string(status)})")


_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load the built library (never builds it). Raises if it is missing."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise FileNotFoundError(
            f"{p} not found: build it first (python -m paper_2602_13836_amd.build, or "
            f"__graft_entry__.build()); there is no fallback path")
    lib = ctypes.CDLL(p)
    i64, vp, ci = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    lib.specvocab_version.restype = ci
    lib.specvocab_version.argtypes = []
    lib.specvocab_status_string.restype = ctypes.c_char_p
    lib.specvocab_status_string.argtypes = [ci]
    lib.specvocab_workspace_bytes.restype = ci
    lib.specvocab_workspace_bytes.argtypes = [ci, i64, i64, i64, i64, i64, i64, ci, ci,
                                              ctypes.POINTER(ctypes.c_size_t)]
    lib.specvocab_select.restype = ci
    lib.specvocab_select.argtypes = [vp, i64, i64, i64, vp, i64, vp, i64, ci, i64, vp, vp, vp,
                                     ctypes.c_size_t, vp]
    lib.specvocab_init.restype = ci
    lib.specvocab_init.argtypes = []
    lib.specvocab_select_static.restype = ci
    lib.specvocab_select_static.argtypes = [vp, i64, i64, i64, vp, i64, vp, i64, ci, i64, vp, vp, vp]
    lib.specvocab_select_threshold.restype = ci
    lib.specvocab_select_threshold.argtypes = [vp, i64, i64, i64, vp, i64, vp, i64, ci, i64, ctypes.c_float, vp, vp,
                                               vp, ctypes.c_size_t, vp]
    lib.specvocab_subset_logits.restype = ci
    lib.specvocab_subset_logits.argtypes = [vp, i64, i64, i64, vp, i64, i64, ci, vp, i64, ci, vp, vp,
                                            ctypes.c_size_t, vp]
    lib.specvocab_indexed_head_naive.restype = ci
    lib.specvocab_indexed_head_naive.argtypes = lib.specvocab_subset_logits.argtypes
    lib.specvocab_aux_log_softmax.restype = ci
    lib.specvocab_aux_log_softmax.argtypes = [vp, i64, i64, i64, vp, i64, vp, i64, ci, vp, vp, ctypes.c_size_t, vp]
    lib.specvocab_pack_rows.restype = ci
    lib.specvocab_pack_rows.argtypes = [vp, i64, i64, i64, ci, vp, i64, vp, vp]
    lib.specvocab_draft_topk.restype = ci
    lib.specvocab_draft_topk.argtypes = [vp, vp, ci, i64, i64, i64, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.specvocab_draft_step.restype = ci
    lib.specvocab_draft_step.argtypes = [vp, i64, i64, i64, vp, i64, i64, ci, vp, i64, ci, i64, vp, vp, vp, vp, vp,
                                         ctypes.c_size_t, vp]
    lib.specvocab_stream_read_probe.restype = ci
    lib.specvocab_stream_read_probe.argtypes = [vp, ctypes.c_size_t, vp, ctypes.c_size_t, vp]
    lib.specvocab_dense_logits.restype = ci
    lib.specvocab_dense_logits.argtypes = [vp, i64, i64, i64, vp, i64, i64, ci, vp, vp, ctypes.c_size_t, vp]
    sz, cf = ctypes.c_size_t, ctypes.c_float
    lib.specvocab_quantize_rows.restype = ci
    lib.specvocab_quantize_rows.argtypes = [vp, i64, i64, i64, ci, vp, i64, vp, i64, vp]
    lib.specvocab_rms_norm.restype = ci
    lib.specvocab_rms_norm.argtypes = [vp, i64, i64, i64, vp, i64, vp, cf, cf, ci, vp, i64, vp, i64, vp, i64, vp, i64, vp]
    head = [vp, vp, i64, i64, i64, i64, vp, vp, i64, i64, i64]
    lib.specvocab_quantized_dense_logits.restype = ci
    lib.specvocab_quantized_dense_logits.argtypes = head + [vp, vp, sz, vp]
    lib.specvocab_quantized_subset_logits.restype = ci
    lib.specvocab_quantized_subset_logits.argtypes = head + [vp, i64, ci, vp, vp, sz, vp]
    lib.specvocab_sample.restype = ci
    lib.specvocab_sample.argtypes = [vp, i64, i64, i64, vp, ci, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.specvocab_quantized_sample_step.restype = ci
    lib.specvocab_quantized_sample_step.argtypes = head + [vp, i64, ci, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.specvocab_token_logprobs.restype = ci
    lib.specvocab_token_logprobs.argtypes = [vp, i64, i64, i64, ci, vp, ci, vp, vp, i64, i64, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.specvocab_token_logprobs_grad.restype = ci
    lib.specvocab_token_logprobs_grad.argtypes = [vp, i64, i64, i64, ci, vp, vp, i64, vp, vp, vp, vp, i64, ci, vp]
    lib.specvocab_distill.restype = ci
    lib.specvocab_distill.argtypes = [vp, i64, i64, i64, ci, vp, vp, i64, ci, cf, vp, vp, vp, vp, i64, ci, vp, sz, vp]
    lib.specvocab_distill_grad.restype = ci
    lib.specvocab_distill_grad.argtypes = [vp, i64, i64, i64, ci, vp, vp, i64, ci, cf, vp, vp, vp, i64, ci, vp]
    if path is None:
        _lib = lib
    return lib


STATIC_SCRATCH_BYTES = 8 << 20       # SPECVOCAB_STATIC_SCRATCH_BYTES


def init() -> None:
    """specvocab_init: one-time set-up of the current device (needed explicitly only before a first call that
    would fall inside a stream capture)."""
    _check(load_library().specvocab_init(), "specvocab_init")


def version() -> int:
    return int(load_library().specvocab_version())


def status_string(status: int) -> str:
    return load_library().specvocab_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != SV_OK:
        raise SpecVocabError(status, where)


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return SV_F32
    if t.dtype == torch.bfloat16:
        return SV_BF16
    raise TypeError(f"storage dtype must be float32 or bfloat16, got {t.dtype}")


def _mat(t: torch.Tensor, name: str) -> Tuple[int, int, int]:
    """(rows, cols, row stride in elements) of a device matrix with contiguous rows."""
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError(f"{name} must be a 2-D tensor with contiguous rows")
    rows, cols = t.shape
    ld = t.stride(0)
    return rows, cols, ld if rows > 1 or ld > cols else cols


# Marshalling is on the path of every call, and a small draft step is over in the time that a few Python objects take:
# pointers and streams travel as plain integers (the declared argument types convert them), the current stream is asked
# for its raw handle (0.3 against 1.6 us through a Stream object), and a workspace size, which depends on nothing but the
# arguments, is asked for once per set of arguments.
def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# (the raw handle comes from a private function; a torch without it goes through the Stream object)
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is not None:
        return stream.cuda_stream
    return _current_raw_stream(torch.cuda.current_device())


def _idx(idx: torch.Tensor, rows: int) -> Tuple[int, int]:
    if not idx.is_cuda or idx.dtype != torch.int32 or not idx.is_contiguous():
        raise ValueError("idx must be a contiguous int32 GPU tensor")
    if idx.dim() == 1:
        return SV_IDX_PER_STEP, idx.shape[0]
    if idx.dim() == 2 and idx.shape[0] == rows:
        return SV_IDX_PER_ROW, idx.shape[1]
    raise ValueError("idx must be [k] (one set per step) or [rows x k]")


@functools.lru_cache(maxsize=512, typed=True)
def _workspace_bytes(lib: ctypes.CDLL, op: int, rows: int, d: int, V: int, k: int, d_prime: int, kd: int, dt: int,
                     idx_mode: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib.specvocab_workspace_bytes(op, rows, d, V, k, d_prime, kd, dt, idx_mode, ctypes.byref(out)),
           "specvocab_workspace_bytes")
    return int(out.value)


def workspace_bytes(op: int, rows: int = 0, d: int = 0, V: int = 0, k: int = 0, d_prime: int = 0,
                    kd: int = 0, dt: int = SV_BF16, idx_mode: int = SV_IDX_PER_ROW) -> int:
    return _workspace_bytes(load_library(), op, rows, d, V, k, d_prime, kd, dt, idx_mode)


def _workspace(nbytes: int, device, ws: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    if ws is not None:
        if ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.numel() < nbytes:
            raise ValueError(f"workspace must be a contiguous uint8 tensor of >= {nbytes} bytes")
        return ws
    if nbytes == 0:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def select(h: torch.Tensor, W_down: torch.Tensor, W_vocab: torch.Tensor, k: int,
           idx_out: Optional[torch.Tensor] = None, scores_out: Optional[torch.Tensor] = None,
           want_scores: bool = False, ws: Optional[torch.Tensor] = None,
           stream: Optional[torch.cuda.Stream] = None, tau: Optional[float] = None):
    """specvocab_select: ids of the k largest approximate logits per row, ascending.
    Returns (idx [rows x k] int32, scores [rows x k] float32 or None).
    tau: specvocab_select_threshold -- selected tokens scoring below tau become padding slots (-1)."""
    rows, d, ldh = _mat(h, "h")
    dp, d2, ldd = _mat(W_down, "W_down")
    V, dp2, ldv = _mat(W_vocab, "W_vocab")
    if d2 != d or dp2 != dp or ldd != d or ldv != dp:
        raise ValueError("W_down must be a dense [d' x d] and W_vocab a dense [V x d']")
    dt = _dt(h)
    if _dt(W_down) != dt or _dt(W_vocab) != dt:
        raise TypeError("h, W_down and W_vocab must share a dtype")
    if idx_out is None:
        idx_out = torch.empty((rows, k), dtype=torch.int32, device=h.device)
    if scores_out is None and want_scores:
        scores_out = torch.empty((rows, k), dtype=torch.float32, device=h.device)
    nbytes = workspace_bytes(SV_OP_SELECT, rows, d, V, k, dp, 0, dt)
    ws = _workspace(nbytes, h.device, ws)
    if tau is None:
        _check(load_library().specvocab_select(_ptr(h), rows, d, ldh, _ptr(W_down), dp, _ptr(W_vocab), V, dt, k,
                                               _ptr(idx_out), _ptr(scores_out), _ptr(ws),
                                               0 if ws is None else ws.numel(), _stream(stream)),
               "specvocab_select")
    else:
        _check(load_library().specvocab_select_threshold(_ptr(h), rows, d, ldh, _ptr(W_down), dp, _ptr(W_vocab), V,
                                                         dt, k, tau, _ptr(idx_out),
                                                         _ptr(scores_out), _ptr(ws),
                                                         0 if ws is None else ws.numel(), _stream(stream)),
               "specvocab_select_threshold")
    return idx_out, scores_out


def select_static(h: torch.Tensor, W_down: torch.Tensor, W_vocab: torch.Tensor, k: int,
                  idx_out: torch.Tensor, scores_out: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None):
    """specvocab_select_static: specvocab_select on the library's static device scratch.  Allocates nothing:
    the caller passes the outputs."""
    rows, d, ldh = _mat(h, "h")
    dp, d2, ldd = _mat(W_down, "W_down")
    V, dp2, ldv = _mat(W_vocab, "W_vocab")
    if d2 != d or dp2 != dp or ldd != d or ldv != dp:
        raise ValueError("W_down must be a dense [d' x d] and W_vocab a dense [V x d']")
    dt = _dt(h)
    if _dt(W_down) != dt or _dt(W_vocab) != dt:
        raise TypeError("h, W_down and W_vocab must share a dtype")
    if idx_out.shape != (rows, k) or idx_out.dtype != torch.int32 or not idx_out.is_contiguous():
        raise ValueError("idx_out must be a contiguous [rows x k] int32 GPU tensor")
    _check(load_library().specvocab_select_static(_ptr(h), rows, d, ldh, _ptr(W_down), dp, _ptr(W_vocab), V, dt, k,
                                                  _ptr(idx_out), _ptr(scores_out), _stream(stream)),
           "specvocab_select_static")
    return idx_out, scores_out


def subset_logits(h: torch.Tensor, U: torch.Tensor, idx: torch.Tensor,
                  out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None, padded: bool = False,
                  sorted_lists: bool = False) -> torch.Tensor:
    """specvocab_subset_logits: out[r, j] = <U[idx(r, j)], h_r>, [rows x k] float32.
    padded=True: idx may hold padding slots (-1), whose logit is -inf.
    sorted_lists=True: the caller declares every list sorted by ascending id (SV_IDX_SORTED)."""
    rows, d, ldh = _mat(h, "h")
    V, d2, ldu = _mat(U, "U")
    if d2 != d:
        raise ValueError("U and h disagree on d")
    dt = _dt(h)
    if _dt(U) != dt:
        raise TypeError("h and U must share a dtype")
    mode, k = _idx(idx, rows)
    if padded:
        mode |= SV_IDX_PADDED
    if sorted_lists:
        mode |= SV_IDX_SORTED
    if out is None:
        out = torch.empty((rows, k), dtype=torch.float32, device=h.device)
    nbytes = workspace_bytes(SV_OP_SUBSET_LOGITS, rows, d, V, k, 0, 0, dt, mode)
    ws = _workspace(nbytes, h.device, ws)
    _check(load_library().specvocab_subset_logits(_ptr(h), rows, d, ldh, _ptr(U), V, ldu, dt, _ptr(idx), k,
                                                  mode, _ptr(out), _ptr(ws),
                                                  0 if ws is None else ws.numel(), _stream(stream)),
           "specvocab_subset_logits")
    return out


def indexed_head_naive(h: torch.Tensor, U: torch.Tensor, idx: torch.Tensor,
                       out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """specvocab_indexed_head_naive: the comparator that materialises U[idx] and multiplies the copy."""
    rows, d, ldh = _mat(h, "h")
    V, d2, ldu = _mat(U, "U")
    if d2 != d:
        raise ValueError("U and h disagree on d")
    dt = _dt(h)
    if _dt(U) != dt:
        raise TypeError("h and U must share a dtype")
    mode, k = _idx(idx, rows)
    if out is None:
        out = torch.empty((rows, k), dtype=torch.float32, device=h.device)
    nbytes = workspace_bytes(SV_OP_INDEXED_HEAD_NAIVE, rows, d, V, k, 0, 0, dt, mode)
    ws = _workspace(nbytes, h.device, ws)
    _check(load_library().specvocab_indexed_head_naive(_ptr(h), rows, d, ldh, _ptr(U), V, ldu, dt, _ptr(idx), k,
                                                       mode, _ptr(out), _ptr(ws),
                                                       0 if ws is None else ws.numel(), _stream(stream)),
           "specvocab_indexed_head_naive")
    return out


def aux_log_softmax(h: torch.Tensor, W_down: torch.Tensor, W_vocab: torch.Tensor,
                    out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """specvocab_aux_log_softmax: log q_aux = log softmax(W_vocab (W_down h)) over the whole vocabulary,
    [rows x V] float32."""
    rows, d, ldh = _mat(h, "h")
    dp, d2, ldd = _mat(W_down, "W_down")
    V, dp2, ldv = _mat(W_vocab, "W_vocab")
    if d2 != d or dp2 != dp or ldd != d or ldv != dp:
        raise ValueError("W_down must be a dense [d' x d] and W_vocab a dense [V x d']")
    dt = _dt(h)
    if _dt(W_down) != dt or _dt(W_vocab) != dt:
        raise TypeError("h, W_down and W_vocab must share a dtype")
    if out is None:
        out = torch.empty((rows, V), dtype=torch.float32, device=h.device)
    elif out.shape != (rows, V) or out.dtype != torch.float32 or not out.is_contiguous() or not out.is_cuda:
        raise ValueError("out must be a contiguous [rows x V] float32 GPU tensor")
    nbytes = workspace_bytes(SV_OP_AUX_LOG_SOFTMAX, rows, d, V, 0, dp, 0, dt)
    ws = _workspace(nbytes, h.device, ws)
    _check(load_library().specvocab_aux_log_softmax(_ptr(h), rows, d, ldh, _ptr(W_down), dp, _ptr(W_vocab), V, dt,
                                                    _ptr(out), _ptr(ws), 0 if ws is None else ws.numel(),
                                                    _stream(stream)),
           "specvocab_aux_log_softmax")
    return out


def pack_rows(U: torch.Tensor, idx: torch.Tensor, out: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """specvocab_pack_rows: U' = U[idx, :] as a dense [k x d] matrix (static-vocabulary mode)."""
    V, d, ldu = _mat(U, "U")
    dt = _dt(U)
    if not idx.is_cuda or idx.dtype != torch.int32 or idx.dim() != 1 or not idx.is_contiguous():
        raise ValueError("idx must be a contiguous [k] int32 GPU tensor")
    k = idx.shape[0]
    if out is None:
        out = torch.empty((k, d), dtype=U.dtype, device=U.device)
    elif out.shape != (k, d) or out.dtype != U.dtype or not out.is_contiguous() or not out.is_cuda:
        raise ValueError("out must be a contiguous [k x d] GPU tensor of U's dtype")
    _check(load_library().specvocab_pack_rows(_ptr(U), V, d, ldu, dt, _ptr(idx), k, _ptr(out), _stream(stream)),
           "specvocab_pack_rows")
    return out


def draft_topk(logits: torch.Tensor, idx: torch.Tensor, kd: int,
               tok_out: Optional[torch.Tensor] = None, prob_out: Optional[torch.Tensor] = None,
               probs_full_out: Optional[torch.Tensor] = None, want_probs: bool = False,
               ws: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """specvocab_draft_topk: subset softmax + top-kd tokens per row.
    Returns (tok [rows x kd] int32, prob [rows x kd] float32, q_K [rows x k] float32 or None)."""
    if not logits.is_cuda or logits.dtype != torch.float32 or logits.dim() != 2 or not logits.is_contiguous():
        raise ValueError("logits must be a contiguous [rows x k] float32 GPU tensor")
    rows, k = logits.shape
    mode, k2 = _idx(idx, rows)
    if k2 != k:
        raise ValueError("idx and logits disagree on k")
    if tok_out is None:
        tok_out = torch.empty((rows, kd), dtype=torch.int32, device=logits.device)
    if prob_out is None:
        prob_out = torch.empty((rows, kd), dtype=torch.float32, device=logits.device)
    if probs_full_out is None and want_probs:
        probs_full_out = torch.empty((rows, k), dtype=torch.float32, device=logits.device)
    nbytes = workspace_bytes(SV_OP_DRAFT_TOPK, rows, 0, 0, k, 0, kd, SV_F32, mode)
    ws = _workspace(nbytes, logits.device, ws)
    _check(load_library().specvocab_draft_topk(_ptr(logits), _ptr(idx), mode, rows, k, kd, _ptr(tok_out),
                                               _ptr(prob_out), _ptr(probs_full_out), _ptr(ws),
                                               0 if ws is None else ws.numel(), _stream(stream)),
           "specvocab_draft_topk")
    return tok_out, prob_out, probs_full_out


def draft_step(h: torch.Tensor, U: torch.Tensor, idx: torch.Tensor, kd: int,
               logits_out: Optional[torch.Tensor] = None, tok_out: Optional[torch.Tensor] = None,
               prob_out: Optional[torch.Tensor] = None, probs_full_out: Optional[torch.Tensor] = None,
               want_probs: bool = False, ws: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None, padded: bool = False, sorted_lists: bool = False):
    """specvocab_draft_step: subset logits, then subset softmax and top-kd tokens of every row,
    enqueued back to back. Returns (logits [rows x k], tok [rows x kd], prob [rows x kd],
    q_K [rows x k] or None)."""
    rows, d, ldh = _mat(h, "h")
    V, d2, ldu = _mat(U, "U")
    if d2 != d:
        raise ValueError("U and h disagree on d")
    dt = _dt(h)
    if _dt(U) != dt:
        raise TypeError("h and U must share a dtype")
    mode, k = _idx(idx, rows)
    if padded:
        mode |= SV_IDX_PADDED
    if sorted_lists:
        mode |= SV_IDX_SORTED
    dev = h.device
    if logits_out is None:
        logits_out = torch.empty((rows, k), dtype=torch.float32, device=dev)
    if tok_out is None:
        tok_out = torch.empty((rows, kd), dtype=torch.int32, device=dev)
    if prob_out is None:
        prob_out = torch.empty((rows, kd), dtype=torch.float32, device=dev)
    if probs_full_out is None and want_probs:
        probs_full_out = torch.empty((rows, k), dtype=torch.float32, device=dev)
    nbytes = workspace_bytes(SV_OP_DRAFT_STEP, rows, d, V, k, 0, kd, dt, mode)
    ws = _workspace(nbytes, dev, ws)
    _check(load_library().specvocab_draft_step(_ptr(h), rows, d, ldh, _ptr(U), V, ldu, dt, _ptr(idx), k, mode, kd,
                                               _ptr(logits_out), _ptr(tok_out), _ptr(prob_out),
                                               _ptr(probs_full_out), _ptr(ws), 0 if ws is None else ws.numel(),
                                               _stream(stream)),
           "specvocab_draft_step")
    return logits_out, tok_out, prob_out, probs_full_out


def stream_read_probe(buf: torch.Tensor, ws: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """specvocab_stream_read_probe: one plain streaming read of buf (measurement aid)."""
    if not buf.is_cuda or not buf.is_contiguous() or not ws.is_cuda or ws.dtype != torch.uint8:
        raise ValueError("buf and ws must be contiguous GPU tensors (ws uint8)")
    nbytes = buf.numel() * buf.element_size()
    _check(load_library().specvocab_stream_read_probe(_ptr(buf), nbytes - nbytes % 16, _ptr(ws), ws.numel(),
                                                      _stream(stream)), "specvocab_stream_read_probe")


def dense_logits(h: torch.Tensor, U: torch.Tensor, out: Optional[torch.Tensor] = None,
                 ws: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """specvocab_dense_logits: the full-vocabulary baseline, out[r, v] = <U[v], h_r>."""
    rows, d, ldh = _mat(h, "h")
    V, d2, ldu = _mat(U, "U")
    if d2 != d:
        raise ValueError("U and h disagree on d")
    dt = _dt(h)
    if _dt(U) != dt:
        raise TypeError("h and U must share a dtype")
    if out is None:
        out = torch.empty((rows, V), dtype=torch.float32, device=h.device)
    nbytes = workspace_bytes(SV_OP_DENSE_LOGITS, rows, d, V, 0, 0, 0, dt)
    ws = _workspace(nbytes, h.device, ws)
    _check(load_library().specvocab_dense_logits(_ptr(h), rows, d, ldh, _ptr(U), V, ldu, dt, _ptr(out),
                                                 _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)),
           "specvocab_dense_logits")
    return out


# ---- from a layer's output to a token, with the output embedding in 8 bits

class QuantizedRows(NamedTuple):
    """Rows in 8 bits: q [rows x d] float8_e4m3fn and scales [rows x scale_columns(d)] float8_e8m0fnu, one per block of 128."""
    q: torch.Tensor
    scales: torch.Tensor


def scale_columns(d: int) -> int:
    """Scale bytes of a row of d values: one per block of 128, in whole words."""
    return 4 * ((d + 511) // 512)


# These calls check that what they are given lives on the current device, whose stream they go to, and spend as little
# as they can on it: a norm of one row is over in less time than ten Python calls take.  Tensors that they make are not checked.
# With a stream given they run with it as the current one: outputs and workspaces that a call makes are that stream's, so nobody else is
# handed their memory while it works on them.
def _tensor(t, name: str) -> None:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor, got {type(t).__name__}")


def _rows(t: torch.Tensor, name: str, here: int) -> Tuple[int, int, int]:
    """_mat of a tensor on the current device."""
    _tensor(t, name)
    if t.get_device() != here:
        raise ValueError(f"{name} must live on the current GPU (cuda:{here}), not on {t.device}")
    if t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor with contiguous rows")
    ld, step = t.stride()
    rows, cols = t.shape
    if step != 1 and cols > 1:
        raise ValueError(f"{name} must be a 2-D tensor with contiguous rows")
    return rows, cols, ld if rows > 1 or ld > cols else cols


def _flat(t: Optional[torch.Tensor], shape: tuple, dtype: torch.dtype, name: str, here: int) -> Optional[int]:
    """Pointer of a contiguous tensor of this shape and type on the current device, or None."""
    if t is None:
        return None
    _tensor(t, name)
    if t.get_device() != here or t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {list(shape)} {dtype} tensor on the current GPU (cuda:{here})")
    return t.data_ptr()


def _scratch(nbytes: int, like: torch.Tensor, ws: Optional[torch.Tensor], here: int) -> Tuple[Optional[torch.Tensor], Optional[int], int]:
    """(workspace, its pointer, its size)."""
    if ws is None:
        if nbytes == 0:
            return None, None, 0
        ws = torch.empty(nbytes, dtype=torch.uint8, device=like.device)
        return ws, ws.data_ptr(), nbytes
    _tensor(ws, "workspace")
    if ws.get_device() != here or ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.numel() < nbytes:
        raise ValueError(f"workspace must be a contiguous uint8 tensor of >= {nbytes} bytes on the current GPU (cuda:{here})")
    return ws, ws.data_ptr(), ws.numel()


def _quantized(t: QuantizedRows, name: str, here: int) -> Tuple[int, int, int, int]:
    """(rows, d, row stride of the codes, row stride of the scales)."""
    if not isinstance(t, QuantizedRows):
        raise TypeError(f"{name} must be QuantizedRows, got {type(t).__name__}")
    q, scales = t
    rows, d, ld = _rows(q, name, here)
    if q.dtype != torch.float8_e4m3fn or scales.dtype != torch.float8_e8m0fnu:
        raise TypeError(f"{name} must be float8_e4m3fn codes with float8_e8m0fnu scales")
    srows, cols, lds = _rows(scales, f"{name}.scales", here)
    if srows != rows or cols != scale_columns(d):
        raise ValueError(f"{name}.scales must be [{rows} x {scale_columns(d)}]")
    return rows, d, ld, lds


def _quantized_out(rows: int, d: int, like: torch.Tensor, out: Optional[QuantizedRows], here: int) -> Tuple[QuantizedRows, int, int]:
    """(where rows in 8 bits go, row stride of the codes, of the scales)."""
    if out is None:
        cols = scale_columns(d)
        return QuantizedRows(torch.empty((rows, d), dtype=torch.float8_e4m3fn, device=like.device),
                             torch.empty((rows, cols), dtype=torch.float8_e8m0fnu, device=like.device)), d, cols
    r, c, ldq, lds = _quantized(out, "the quantized output", here)
    if r != rows or c != d:
        raise ValueError(f"the quantized output must be [{rows} x {d}]")
    return out, ldq, lds


def quantize_rows(x: torch.Tensor, out: Optional[QuantizedRows] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> QuantizedRows:
    """specvocab_quantize_rows: the rows of x in 8 bits, a power-of-two scale per block of 128."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return quantize_rows(x, out)
    here = torch.cuda.current_device()
    rows, d, ldx = _rows(x, "x", here)
    out, ldq, lds = _quantized_out(rows, d, x, out, here)
    _check(load_library().specvocab_quantize_rows(x.data_ptr(), rows, d, ldx, _dt(x), out.q.data_ptr(), ldq, out.scales.data_ptr(),
                                                  lds, _current_raw_stream(here)), "specvocab_quantize_rows")
    return out


def _like(t: torch.Tensor, x: torch.Tensor, name: str, here: int) -> int:
    """Row stride of a matrix of x's shape and type."""
    ld = _rows(t, name, here)[2]
    if t.shape != x.shape or t.dtype != x.dtype:
        raise ValueError(f"{name} must have x's shape and dtype")
    return ld


def rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
             weight_offset: float = 0.0, want_y: bool = True, want_quantized: bool = False,
             sum_out: Optional[torch.Tensor] = None, y_out: Optional[torch.Tensor] = None,
             quantized_out: Optional[QuantizedRows] = None, stream: Optional[torch.cuda.Stream] = None):
    """specvocab_rms_norm: root-mean-square norm of x + residual.
    Returns (y or None, the sum (x itself without a residual), QuantizedRows of y or None)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return rms_norm(x, weight, eps, residual, weight_offset, want_y, want_quantized, sum_out, y_out, quantized_out)
    here = torch.cuda.current_device()
    rows, d, ldx = _rows(x, "x", here)
    w = _flat(weight, (d,), x.dtype, "weight", here)
    if w is None:
        raise ValueError("weight must be given")
    r = t = y = q = s = None
    ldr = ld_sum = ldy = ldq = lds = 0
    if residual is not None:
        ldr, r = _like(residual, x, "residual", here), residual.data_ptr()
        if sum_out is None:
            sum_out, ld_sum = torch.empty((rows, d), dtype=x.dtype, device=x.device), d
        else:
            ld_sum = _like(sum_out, x, "sum_out", here)
        t = sum_out.data_ptr()
    elif sum_out is not None:
        raise ValueError("sum_out needs a residual")
    if y_out is not None:
        ldy, y = _like(y_out, x, "y_out", here), y_out.data_ptr()
    elif want_y:
        y_out, ldy = torch.empty((rows, d), dtype=x.dtype, device=x.device), d
        y = y_out.data_ptr()
    if quantized_out is not None or want_quantized:
        quantized_out, ldq, lds = _quantized_out(rows, d, x, quantized_out, here)
        q, s = quantized_out.q.data_ptr(), quantized_out.scales.data_ptr()
    _check(load_library().specvocab_rms_norm(x.data_ptr(), rows, d, ldx, r, ldr, w, weight_offset, eps, _dt(x), t, ld_sum, y, ldy,
                                             q, ldq, s, lds, _current_raw_stream(here)), "specvocab_rms_norm")
    return y_out, x if residual is None else sum_out, quantized_out


def _head_operands(h: Union[torch.Tensor, QuantizedRows], U: QuantizedRows, here: int):
    """(leading arguments of the products with an 8-bit embedding, rows, d, V, dtype of h)."""
    V, d2, ldu, ldus = _quantized(U, "U", here)
    if isinstance(h, QuantizedRows):
        rows, d, ldh, ldhs = _quantized(h, "h", here)
        hp, hs, dt = h.q.data_ptr(), h.scales.data_ptr(), SV_E4M3
    else:
        rows, d, ldh = _rows(h, "h", here)
        if h.dtype != torch.bfloat16:
            raise TypeError(f"h must be bfloat16 or QuantizedRows, got {h.dtype}")
        hp, hs, ldhs, dt = h.data_ptr(), None, 0, SV_BF16
    if d2 != d:
        raise ValueError("U and h disagree on d")
    return (hp, hs, rows, d, ldh, ldhs, U.q.data_ptr(), U.scales.data_ptr(), V, ldu, ldus), rows, d, V, dt


def _logits_out(out: Optional[torch.Tensor], rows: int, n: int, U: QuantizedRows, here: int) -> Tuple[torch.Tensor, int]:
    if out is None:
        out = torch.empty((rows, n), dtype=torch.float32, device=U.q.device)
        return out, out.data_ptr()
    return out, _flat(out, (rows, n), torch.float32, "the logits' tensor", here)


def _list(idx: torch.Tensor, rows: int, padded: bool, here: int) -> Tuple[int, int, int]:
    """(pointer, idx_mode, length) of an index list."""
    _tensor(idx, "idx")
    if idx.get_device() != here or idx.dtype != torch.int32 or not idx.is_contiguous():
        raise ValueError(f"idx must be a contiguous int32 tensor on the current GPU (cuda:{here})")
    flag = SV_IDX_PADDED if padded else 0
    if idx.dim() == 1:
        return idx.data_ptr(), SV_IDX_PER_STEP | flag, idx.shape[0]
    if idx.dim() == 2 and idx.shape[0] == rows:
        return idx.data_ptr(), SV_IDX_PER_ROW | flag, idx.shape[1]
    raise ValueError("idx must be [k] (one set per step) or [rows x k]")


def quantized_dense_logits(h: Union[torch.Tensor, QuantizedRows], U: QuantizedRows, out: Optional[torch.Tensor] = None,
                           ws: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """specvocab_quantized_dense_logits: out[r, v] = <U[v], h_r> with U in 8 bits, h in 8 bits or bfloat16."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return quantized_dense_logits(h, U, out, ws)
    here = torch.cuda.current_device()
    args, rows, d, V, dt = _head_operands(h, U, here)
    out, op = _logits_out(out, rows, V, U, here)
    ws, wp, wn = _scratch(workspace_bytes(SV_OP_QUANTIZED_DENSE_LOGITS, rows, d, V, 0, 0, 0, dt), U.q, ws, here)
    _check(load_library().specvocab_quantized_dense_logits(*args, op, wp, wn, _current_raw_stream(here)),
           "specvocab_quantized_dense_logits")
    return out


def quantized_subset_logits(h: Union[torch.Tensor, QuantizedRows], U: QuantizedRows, idx: torch.Tensor,
                            out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                            stream: Optional[torch.cuda.Stream] = None, padded: bool = False) -> torch.Tensor:
    """specvocab_quantized_subset_logits: out[r, j] = <U[idx(r, j)], h_r>.  padded: idx may hold padding slots (-1)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return quantized_subset_logits(h, U, idx, out, ws, padded=padded)
    here = torch.cuda.current_device()
    args, rows, d, V, dt = _head_operands(h, U, here)
    ip, mode, k = _list(idx, rows, padded, here)
    out, op = _logits_out(out, rows, k, U, here)
    ws, wp, wn = _scratch(workspace_bytes(SV_OP_QUANTIZED_SUBSET_LOGITS, rows, d, V, k, 0, 0, dt, mode), U.q, ws, here)
    _check(load_library().specvocab_quantized_subset_logits(*args, ip, k, mode, op, wp, wn, _current_raw_stream(here)),
           "specvocab_quantized_subset_logits")
    return out


def _sampling(rows: int, u, temperature, top_k, top_p, min_p, here: int):
    f32, shape = torch.float32, (rows,)
    if u is None:
        raise ValueError("u must be given")
    return (_flat(temperature, shape, f32, "temperature", here), _flat(top_k, shape, torch.int32, "top_k", here),
            _flat(top_p, shape, f32, "top_p", here), _flat(min_p, shape, f32, "min_p", here), _flat(u, shape, f32, "u", here))


def _drawn(rows: int, like: torch.Tensor, tok_out: Optional[torch.Tensor], prob_out: Optional[torch.Tensor], here: int):
    if tok_out is None:
        tok_out = torch.empty(rows, dtype=torch.int32, device=like.device)
    else:
        _flat(tok_out, (rows,), torch.int32, "tok_out", here)
    if prob_out is None:
        prob_out = torch.empty(rows, dtype=torch.float32, device=like.device)
    else:
        _flat(prob_out, (rows,), torch.float32, "prob_out", here)
    return tok_out, prob_out


def sample(logits: torch.Tensor, u: torch.Tensor, temperature: Optional[torch.Tensor] = None,
           top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None,
           idx: Optional[torch.Tensor] = None, tok_out: Optional[torch.Tensor] = None, prob_out: Optional[torch.Tensor] = None,
           ws: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """specvocab_sample: one token per row from the random numbers u [rows]; temperature, top_p, min_p float32 [rows], top_k int32
    [rows], each or None.  idx: the token ids of the places, [n] or [rows x n].
    Returns (tok [rows] int32, prob [rows] float32)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return sample(logits, u, temperature, top_k, top_p, min_p, idx, tok_out, prob_out, ws)
    here = torch.cuda.current_device()
    rows, n, ld = _rows(logits, "logits", here)
    if logits.dtype != torch.float32:
        raise TypeError(f"logits must be float32, got {logits.dtype}")
    settings = _sampling(rows, u, temperature, top_k, top_p, min_p, here)
    ip, mode = None, SV_IDX_PER_ROW
    if idx is not None:
        ip, mode, k = _list(idx, rows, False, here)
        if k != n:
            raise ValueError("idx and logits disagree on n")
    tok_out, prob_out = _drawn(rows, logits, tok_out, prob_out, here)
    ws, wp, wn = _scratch(workspace_bytes(SV_OP_SAMPLE, rows, 0, 0, n, 0, 0, SV_F32), logits, ws, here)
    _check(load_library().specvocab_sample(logits.data_ptr(), ld, rows, n, ip, mode, *settings, tok_out.data_ptr(),
                                           prob_out.data_ptr(), wp, wn, _current_raw_stream(here)), "specvocab_sample")
    return tok_out, prob_out


def quantized_sample_step(h: Union[torch.Tensor, QuantizedRows], U: QuantizedRows, u: torch.Tensor,
                          idx: Optional[torch.Tensor] = None, temperature: Optional[torch.Tensor] = None,
                          top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None,
                          min_p: Optional[torch.Tensor] = None, logits_out: Optional[torch.Tensor] = None,
                          tok_out: Optional[torch.Tensor] = None, prob_out: Optional[torch.Tensor] = None,
                          ws: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None, padded: bool = False):
    """specvocab_quantized_sample_step: logits over idx (None: the whole vocabulary) with U in 8 bits, then a token per row.
    Returns (logits, tok, prob)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return quantized_sample_step(h, U, u, idx, temperature, top_k, top_p, min_p, logits_out, tok_out, prob_out, ws, padded=padded)
    here = torch.cuda.current_device()
    args, rows, d, V, dt = _head_operands(h, U, here)
    ip, mode, k = (None, SV_IDX_PER_ROW, 0) if idx is None else _list(idx, rows, padded, here)
    settings = _sampling(rows, u, temperature, top_k, top_p, min_p, here)
    logits_out, op = _logits_out(logits_out, rows, V if idx is None else k, U, here)
    tok_out, prob_out = _drawn(rows, U.q, tok_out, prob_out, here)
    ws, wp, wn = _scratch(workspace_bytes(SV_OP_QUANTIZED_SAMPLE_STEP, rows, d, V, k, 0, 0, dt, mode), U.q, ws, here)
    _check(load_library().specvocab_quantized_sample_step(*args, ip, k, mode, *settings, op, tok_out.data_ptr(), prob_out.data_ptr(),
                                                          wp, wn, _current_raw_stream(here)), "specvocab_quantized_sample_step")
    return logits_out, tok_out, prob_out


# ---- over finished rows of logits: log probabilities of given tokens, distillation from a teacher's largest logits

class TokenLogprobs(NamedTuple):
    """logprob [rows] or [rows x given] (None without tokens), entropy [rows], top_tok int32 and top_logprob [rows x top] (None for top
    0), state [rows x 4] (None unless asked for); float32 where nothing else is said."""
    logprob: Optional[torch.Tensor]
    entropy: torch.Tensor
    top_tok: Optional[torch.Tensor]
    top_logprob: Optional[torch.Tensor]
    state: Optional[torch.Tensor]


class Distilled(NamedTuple):
    """loss [rows] float32, grad [rows x n] (None unless asked for), state [rows x 4] float32 (None unless asked for)."""
    loss: torch.Tensor
    grad: Optional[torch.Tensor]
    state: Optional[torch.Tensor]


_TEACHER_KINDS = {"logits": 0, "logprobs": 1, "rest": 2}


def _out(t: Optional[torch.Tensor], shape: tuple, dtype: torch.dtype, name: str, like: torch.Tensor, here: int) -> Tuple[torch.Tensor, int]:
    """(the caller's output or a new one, its pointer)."""
    if t is None:
        # (a tensor by its strides is made in 1.3 us, by its shape alone in 1.7, and a call makes up to five)
        t = torch.empty_strided(shape, (1,) if len(shape) == 1 else (shape[1], 1), dtype=dtype, device=like.device)
        return t, t.data_ptr()
    return t, _flat(t, shape, dtype, name, here)


def _gradient(out: Optional[torch.Tensor], dtype: Optional[torch.dtype], logits: torch.Tensor, here: int) -> Tuple[torch.Tensor, int, int]:
    """(where a gradient goes, its row stride, its type)."""
    if out is None:
        out = torch.empty(logits.shape, dtype=dtype or logits.dtype, device=logits.device)
        return out, out.shape[1], _dt(out)
    ld = _rows(out, "grad_out", here)[2]
    if out.shape != logits.shape:
        raise ValueError("grad_out must have the logits' shape")
    if dtype is not None and out.dtype != dtype:
        raise ValueError(f"grad_out is {out.dtype}, not {dtype}")
    return out, ld, _dt(out)


def _given(tokens: torch.Tensor, rows: int, here: int) -> Tuple[int, int]:
    """(pointer, tokens of a row)."""
    _tensor(tokens, "tokens")
    if tokens.dim() not in (1, 2):
        raise ValueError("tokens must be [rows] or [rows x given]")
    shape = (rows,) if tokens.dim() == 1 else (rows, tokens.shape[1])
    return _flat(tokens, shape, torch.int32, "tokens", here), 1 if tokens.dim() == 1 else tokens.shape[1]


def token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, top: int = 0,
                   temperature: Optional[torch.Tensor] = None, idx: Optional[torch.Tensor] = None, want_state: bool = False,
                   logprob_out: Optional[torch.Tensor] = None, entropy_out: Optional[torch.Tensor] = None,
                   top_tok_out: Optional[torch.Tensor] = None, top_logprob_out: Optional[torch.Tensor] = None,
                   state_out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> TokenLogprobs:
    """specvocab_token_logprobs: log probabilities of the given tokens (int32 [rows] or [rows x given]), the entropy and the `top` largest
    alternatives of every row of logits (float32 or bfloat16), at temperature [rows] float32 (None: 1).  idx: the token ids of the places,
    [n] or [rows x n].  state: what token_logprobs_grad needs."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return token_logprobs(logits, tokens, top, temperature, idx, want_state, logprob_out, entropy_out, top_tok_out, top_logprob_out,
                                  state_out, ws)
    here = torch.cuda.current_device()
    rows, n, ld = _rows(logits, "logits", here)
    dt, f32 = _dt(logits), torch.float32
    tp, given = (None, 0) if tokens is None else _given(tokens, rows, here)
    t = _flat(temperature, (rows,), f32, "temperature", here)
    ip, mode = None, SV_IDX_PER_ROW
    if idx is not None:
        ip, mode, k = _list(idx, rows, False, here)
        if k != n:
            raise ValueError("idx and logits disagree on n")
    lp = kp = vp = sp = None
    if tokens is not None:
        logprob_out, lp = _out(logprob_out, tuple(tokens.shape), f32, "logprob_out", logits, here)
    elif logprob_out is not None:
        raise ValueError("logprob_out needs tokens")
    entropy_out, ep = _out(entropy_out, (rows,), f32, "entropy_out", logits, here)
    if top > 0:
        top_tok_out, kp = _out(top_tok_out, (rows, top), torch.int32, "top_tok_out", logits, here)
        top_logprob_out, vp = _out(top_logprob_out, (rows, top), f32, "top_logprob_out", logits, here)
    elif top_tok_out is not None or top_logprob_out is not None:
        raise ValueError("top_tok_out and top_logprob_out need top > 0")
    if want_state or state_out is not None:
        state_out, sp = _out(state_out, (rows, 4), f32, "state_out", logits, here)
    ws, wp, wn = _scratch(workspace_bytes(SV_OP_TOKEN_LOGPROBS, rows, 0, 0, n, 0, top, dt), logits, ws, here)
    _check(load_library().specvocab_token_logprobs(logits.data_ptr(), ld, rows, n, dt, ip, mode, t, tp, given, top, lp, ep, kp, vp, sp,
                                                   wp, wn, _current_raw_stream(here)), "specvocab_token_logprobs")
    return TokenLogprobs(logprob_out, entropy_out, top_tok_out, top_logprob_out, state_out)


def token_logprobs_grad(logits: torch.Tensor, tokens: Optional[torch.Tensor], state: torch.Tensor,
                        grad_logprob: Optional[torch.Tensor] = None, grad_entropy: Optional[torch.Tensor] = None,
                        temperature: Optional[torch.Tensor] = None, grad_dtype: Optional[torch.dtype] = None,
                        grad_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """specvocab_token_logprobs_grad: the logits' gradient [rows x n] from those of token_logprobs' log probabilities (the tokens' shape)
    and entropy [rows].  grad_dtype: float32 or bfloat16 (None: the logits' type); grad_out may be the logits themselves."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return token_logprobs_grad(logits, tokens, state, grad_logprob, grad_entropy, temperature, grad_dtype, grad_out)
    here = torch.cuda.current_device()
    rows, n, ld = _rows(logits, "logits", here)
    dt, f32 = _dt(logits), torch.float32
    tp, given = (None, 0) if tokens is None else _given(tokens, rows, here)
    t = _flat(temperature, (rows,), f32, "temperature", here)
    if state is None:
        raise ValueError("state must be given")
    sp = _flat(state, (rows, 4), f32, "state", here)
    if grad_logprob is not None and tokens is None:
        raise ValueError("grad_logprob needs tokens")
    gp = None if grad_logprob is None else _flat(grad_logprob, tuple(tokens.shape), f32, "grad_logprob", here)
    ge = _flat(grad_entropy, (rows,), f32, "grad_entropy", here)
    grad_out, ldg, gdt = _gradient(grad_out, grad_dtype, logits, here)
    _check(load_library().specvocab_token_logprobs_grad(logits.data_ptr(), ld, rows, n, dt, t, tp, given, sp, gp, ge, grad_out.data_ptr(),
                                                        ldg, gdt, _current_raw_stream(here)), "specvocab_token_logprobs_grad")
    return grad_out


def _teacher(logits: torch.Tensor, tok: torch.Tensor, teacher: torch.Tensor, kind: str, weight: Optional[torch.Tensor], here: int):
    """(leading arguments of a distillation but for the temperature and the weight, the weight's pointer, rows, n, dtype)."""
    rows, n, ld = _rows(logits, "logits", here)
    dt = _dt(logits)
    _tensor(tok, "tok")
    _tensor(teacher, "teacher")
    if tok.dim() != 2:
        raise ValueError("tok must be [rows x known]")
    known = tok.shape[1]
    tp = _flat(tok, (rows, known), torch.int32, "tok", here)
    vp = _flat(teacher, (rows, known), torch.float32, "teacher", here)
    if kind not in _TEACHER_KINDS:
        raise ValueError(f"kind must be one of {sorted(_TEACHER_KINDS)}, got {kind!r}")
    w = _flat(weight, (rows,), torch.float32, "weight", here)
    return (logits.data_ptr(), ld, rows, n, dt, tp, vp, known, _TEACHER_KINDS[kind]), w, rows, n, dt


def distill(logits: torch.Tensor, tok: torch.Tensor, teacher: torch.Tensor, kind: str = "logits", temperature: float = 1.0,
            weight: Optional[torch.Tensor] = None, want_grad: bool = False, grad_dtype: Optional[torch.dtype] = None,
            want_state: bool = False, loss_out: Optional[torch.Tensor] = None, grad_out: Optional[torch.Tensor] = None,
            state_out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
            stream: Optional[torch.cuda.Stream] = None) -> Distilled:
    """specvocab_distill: every row's divergence from a teacher that lists tokens tok [rows x known] int32 (-1: padding) with values teacher
    [rows x known] float32 -- kind "logits", "logprobs" (what the list leaves counts nothing) or "rest" (it counts as one more token) --
    times weight [rows].  want_grad, grad_dtype or grad_out: the logits' gradient of the sum of the losses too, in float32 or bfloat16 (the
    logits' type unless said); grad_out may be the logits themselves.  state: what distill_grad needs."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return distill(logits, tok, teacher, kind, temperature, weight, want_grad, grad_dtype, want_state, loss_out, grad_out, state_out, ws)
    here = torch.cuda.current_device()
    args, w, rows, n, dt = _teacher(logits, tok, teacher, kind, weight, here)
    loss_out, lp = _out(loss_out, (rows,), torch.float32, "loss_out", logits, here)
    sp = gp = None
    ldg, gdt = 0, SV_F32
    if want_state or state_out is not None:
        state_out, sp = _out(state_out, (rows, 4), torch.float32, "state_out", logits, here)
    if want_grad or grad_dtype is not None or grad_out is not None:
        grad_out, ldg, gdt = _gradient(grad_out, grad_dtype, logits, here)
        gp = grad_out.data_ptr()
    ws, wp, wn = _scratch(workspace_bytes(SV_OP_DISTILL, rows, 0, 0, n, 0, 0, dt), logits, ws, here)
    _check(load_library().specvocab_distill(*args, temperature, w, lp, sp, gp, ldg, gdt, wp, wn, _current_raw_stream(here)),
           "specvocab_distill")
    return Distilled(loss_out, grad_out, state_out)


def distill_grad(logits: torch.Tensor, tok: torch.Tensor, teacher: torch.Tensor, state: torch.Tensor, kind: str = "logits",
                 temperature: float = 1.0, weight: Optional[torch.Tensor] = None, grad_dtype: Optional[torch.dtype] = None,
                 grad_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """specvocab_distill_grad: the logits' gradient of distill's losses from the state that it left; weight: whatever factor each row's
    divergence has by now, but a row that distill was given with weight 0 has no gradient."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return distill_grad(logits, tok, teacher, state, kind, temperature, weight, grad_dtype, grad_out)
    here = torch.cuda.current_device()
    args, w, rows, _, _ = _teacher(logits, tok, teacher, kind, weight, here)
    if state is None:
        raise ValueError("state must be given")
    sp = _flat(state, (rows, 4), torch.float32, "state", here)
    grad_out, ldg, gdt = _gradient(grad_out, grad_dtype, logits, here)
    _check(load_library().specvocab_distill_grad(*args, temperature, w, sp, grad_out.data_ptr(), ldg, gdt, _current_raw_stream(here)),
           "specvocab_distill_grad")
    return grad_out
