"""Thin Python binding of libmosaic.so (the C ABI declared in include/mosaic.h).

Argument marshalling only: every function takes torch tensors that already
live on the CUDA device (torch is used for device memory and streams), passes
their raw pointers and sizes through ctypes, and raises `MosaicError` on a
non-zero status.  All arithmetic of the method runs inside the library's CUDA
kernels; there is no CPU fallback - if the library cannot be loaded the import
of a function here fails loudly.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from threading import get_ident as _thread

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmosaic.so")

F32, BF16 = 0, 1
RESET_ACCUM = 1
GLOBAL_NORM, PER_CATEGORY_NORM = 0, 1
WEIGHTED_MEAN = 2        # flag, or-ed into the mode
REDISTRIBUTE = 4         # flag, or-ed into the mode: clamp and redistribute
ROWS_GIVEN, COLS_GIVEN, RANK_ONLY, SCORES_ONLY, SCORES_ACCUM = 1, 2, 4, 8, 16
OK, ERR_INFEASIBLE, ERR_TIMEOUT = 0, -9, -10
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3
_ACTS = {"none": ACT_NONE, "relu": ACT_RELU, "gelu": ACT_GELU, "silu": ACT_SILU}

# every symbol include/mosaic.h declares
SYMBOLS = (
    "mosaic_version", "mosaic_status_string",
    "mosaic_act_norms_workspace_bytes", "mosaic_act_norms",
    "mosaic_score",
    "mosaic_outlier_ratio_workspace_bytes", "mosaic_outlier_ratio", "mosaic_ratio_from_count",
    "mosaic_outlier_ratio_static_max_workspace_bytes", "mosaic_outlier_ratio_static",
    "mosaic_outlier_ratio_batch_workspace_bytes", "mosaic_outlier_ratio_batch", "mosaic_outlier_ratio_grouped",
    "mosaic_allocate_sparsity",
    "mosaic_prune_unstructured_workspace_bytes", "mosaic_prune_unstructured",
    "mosaic_prune_unstructured_batch_workspace_bytes", "mosaic_prune_unstructured_batch",
    "mosaic_prune_structured_compact_workspace_bytes", "mosaic_prune_structured_compact",
    "mosaic_rank_units", "mosaic_sum_unit_scores",
    "mosaic_unit_scores_batch_workspace_bytes", "mosaic_unit_scores_batch", "mosaic_add_unit_scores_batch",
    "mosaic_rank_units_batch", "mosaic_compact_batch",
    "mosaic_gram_accumulate",
    "mosaic_linear_workspace_bytes", "mosaic_linear",
    "mosaic_linear_backward_workspace_bytes", "mosaic_linear_backward",
    "mosaic_checkpoint_store", "mosaic_checkpoint_load",
    "mosaic_gated_linear_workspace_bytes", "mosaic_gated_linear",
    "mosaic_gated_linear_backward_workspace_bytes", "mosaic_gated_linear_backward",
    "mosaic_quantize4", "mosaic_dequantize4",
    "mosaic_linear4_workspace_bytes", "mosaic_linear4", "mosaic_gated_linear4_workspace_bytes", "mosaic_gated_linear4",
    "mosaic_top_logits_workspace_bytes", "mosaic_top_logits",
    "mosaic_distill_workspace_bytes", "mosaic_distill_loss", "mosaic_distill_grad", "mosaic_distill_loss_grad",
    "mosaic_bounded_wait_selftest",
)


class MosaicError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} ({status})")


_lib = None


def lib() -> C.CDLL:
    """Load libmosaic.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2504_06323_b200.build` "
                "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        i64, vp, sz, ci, dbl, flt = C.c_int64, C.c_void_p, C.c_size_t, C.c_int, C.c_double, C.c_float
        L.mosaic_version.restype = ci
        L.mosaic_status_string.restype = C.c_char_p
        L.mosaic_status_string.argtypes = [ci]
        L.mosaic_bounded_wait_selftest.restype = ci
        L.mosaic_bounded_wait_selftest.argtypes = [i64, vp, vp]
        L.mosaic_gram_accumulate.restype = ci
        L.mosaic_gram_accumulate.argtypes = [vp, i64, i64, i64, ci, vp, i64, ci, vp, vp]
        L.mosaic_act_norms_workspace_bytes.restype = sz
        L.mosaic_act_norms_workspace_bytes.argtypes = [i64, i64]
        L.mosaic_act_norms.restype = ci
        L.mosaic_act_norms.argtypes = [vp, i64, i64, i64, ci, vp, vp, ci, vp, sz, vp]
        L.mosaic_score.restype = ci
        L.mosaic_score.argtypes = [vp, i64, i64, i64, ci, vp, vp, vp]
        L.mosaic_outlier_ratio_workspace_bytes.restype = sz
        L.mosaic_outlier_ratio_workspace_bytes.argtypes = [i64, i64]
        L.mosaic_outlier_ratio.restype = ci
        L.mosaic_outlier_ratio.argtypes = [vp, i64, i64, i64, ci, vp, flt, vp, vp, vp, sz, vp]
        L.mosaic_outlier_ratio_static_max_workspace_bytes.restype = sz
        L.mosaic_outlier_ratio_static_max_workspace_bytes.argtypes = []
        L.mosaic_outlier_ratio_static.restype = ci
        L.mosaic_outlier_ratio_static.argtypes = [vp, i64, i64, i64, ci, vp, flt, vp, vp, vp]
        L.mosaic_outlier_ratio_batch_workspace_bytes.restype = sz
        L.mosaic_outlier_ratio_batch_workspace_bytes.argtypes = [vp, i64]
        L.mosaic_outlier_ratio_batch.restype = ci
        L.mosaic_outlier_ratio_batch.argtypes = [vp, i64, ci, flt, vp, sz, vp]
        L.mosaic_outlier_ratio_grouped.restype = ci
        L.mosaic_outlier_ratio_grouped.argtypes = [vp, vp, i64, ci, flt, vp, sz, vp]
        L.mosaic_ratio_from_count.restype = dbl
        L.mosaic_ratio_from_count.argtypes = [i64, i64]
        L.mosaic_allocate_sparsity.restype = ci
        L.mosaic_allocate_sparsity.argtypes = [vp, vp, vp, ci, ci, dbl, dbl, ci, vp, vp]
        L.mosaic_prune_unstructured_workspace_bytes.restype = sz
        L.mosaic_prune_unstructured_workspace_bytes.argtypes = [i64, i64]
        L.mosaic_prune_unstructured.restype = ci
        L.mosaic_prune_unstructured.argtypes = [vp, vp, i64, i64, i64, ci, vp, i64, vp, vp, sz, vp]
        L.mosaic_prune_unstructured_batch_workspace_bytes.restype = sz
        L.mosaic_prune_unstructured_batch_workspace_bytes.argtypes = [vp, i64, ci]
        L.mosaic_prune_unstructured_batch.restype = ci
        L.mosaic_prune_unstructured_batch.argtypes = [vp, i64, ci, vp, sz, vp]
        L.mosaic_prune_structured_compact_workspace_bytes.restype = sz
        L.mosaic_prune_structured_compact_workspace_bytes.argtypes = [i64, i64]
        L.mosaic_prune_structured_compact.restype = ci
        L.mosaic_prune_structured_compact.argtypes = [vp, i64, i64, i64, ci, vp, i64, i64, i64, i64, vp, vp, ci, vp,
                                                      vp, vp, sz, vp]
        L.mosaic_rank_units.restype = ci
        L.mosaic_rank_units.argtypes = [vp, i64, i64, vp, vp]
        L.mosaic_sum_unit_scores.restype = ci
        L.mosaic_sum_unit_scores.argtypes = [vp, vp, i64, vp]
        L.mosaic_unit_scores_batch_workspace_bytes.restype = sz
        L.mosaic_unit_scores_batch_workspace_bytes.argtypes = [vp, i64]
        L.mosaic_unit_scores_batch.restype = ci
        L.mosaic_unit_scores_batch.argtypes = [vp, i64, ci, vp, sz, vp]
        L.mosaic_add_unit_scores_batch.restype = ci
        L.mosaic_add_unit_scores_batch.argtypes = [vp, i64, vp]
        L.mosaic_rank_units_batch.restype = ci
        L.mosaic_rank_units_batch.argtypes = [vp, i64, vp]
        L.mosaic_compact_batch.restype = ci
        L.mosaic_compact_batch.argtypes = [vp, i64, ci, vp]
        L.mosaic_linear_workspace_bytes.restype = sz
        L.mosaic_linear_workspace_bytes.argtypes = [vp, i64, vp, i64, i64, i64, i64]
        L.mosaic_linear.restype = ci
        L.mosaic_linear.argtypes = [vp, i64, vp, i64, i64, i64, i64, ci, vp, vp, i64, ci, vp, i64, vp, i64, vp, vp, sz, vp]
        L.mosaic_linear_backward_workspace_bytes.restype = sz
        L.mosaic_linear_backward_workspace_bytes.argtypes = [vp, i64, vp, i64, vp, i64, i64, i64, i64, ci, ci, ci, ci]
        L.mosaic_linear_backward.restype = ci
        L.mosaic_linear_backward.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, i64, i64, i64, ci, ci, vp, i64, vp, i64, vp,
                                             vp, vp, sz, vp]
        L.mosaic_top_logits.restype = ci
        L.mosaic_top_logits.argtypes = [vp, i64, i64, i64, ci, i64, flt, vp, vp, vp, vp, sz, vp]
        L.mosaic_checkpoint_store.restype = ci
        L.mosaic_checkpoint_store.argtypes = [vp, i64, i64, i64, ci, vp, vp]
        L.mosaic_checkpoint_load.restype = ci
        L.mosaic_checkpoint_load.argtypes = [vp, i64, i64, vp, i64, ci, vp]
        L.mosaic_gated_linear_workspace_bytes.restype = sz
        L.mosaic_gated_linear_workspace_bytes.argtypes = [vp, i64, vp, i64, vp, i64, i64, i64, i64, ci]
        L.mosaic_gated_linear.restype = ci
        L.mosaic_gated_linear.argtypes = [vp, i64, vp, i64, vp, i64, i64, i64, i64, ci, vp, vp, ci, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, sz, vp]
        L.mosaic_gated_linear_backward_workspace_bytes.restype = sz
        L.mosaic_gated_linear_backward_workspace_bytes.argtypes = [vp, i64, ci, vp, i64, vp, i64, i64, i64, i64, ci, ci, ci]
        L.mosaic_gated_linear_backward.restype = ci
        L.mosaic_gated_linear_backward.argtypes = [vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, i64, i64, i64, ci, ci, vp, i64,
                                                   vp, i64, vp, i64, vp, vp, vp, i64, vp, vp, sz, vp]
        L.mosaic_quantize4.restype = ci
        L.mosaic_quantize4.argtypes = [vp, i64, i64, i64, ci, vp, vp]
        L.mosaic_dequantize4.restype = ci
        L.mosaic_dequantize4.argtypes = [vp, i64, i64, vp, i64, ci, vp]
        L.mosaic_linear4_workspace_bytes.restype = sz
        L.mosaic_linear4_workspace_bytes.argtypes = [vp, i64, i64, i64, i64]
        L.mosaic_linear4.restype = ci
        L.mosaic_linear4.argtypes = [vp, i64, vp, i64, i64, i64, ci, vp, vp, i64, ci, vp, i64, vp, vp, sz, vp]
        L.mosaic_gated_linear4_workspace_bytes.restype = sz
        L.mosaic_gated_linear4_workspace_bytes.argtypes = [vp, i64, i64, i64, i64]
        L.mosaic_gated_linear4.restype = ci
        L.mosaic_gated_linear4.argtypes = [vp, i64, vp, vp, i64, i64, i64, ci, vp, vp, ci, vp, i64, vp, vp, sz, vp]
        L.mosaic_top_logits_workspace_bytes.restype = sz
        L.mosaic_top_logits_workspace_bytes.argtypes = [i64, i64, ci, i64]
        teacher = [vp, i64, i64, i64, ci, vp, vp, i64, vp, vp, flt]
        L.mosaic_distill_workspace_bytes.restype = sz
        L.mosaic_distill_workspace_bytes.argtypes = [i64, i64]
        L.mosaic_distill_loss.restype = ci
        L.mosaic_distill_loss.argtypes = teacher + [vp, vp, vp, sz, vp]
        L.mosaic_distill_grad.restype = ci
        L.mosaic_distill_grad.argtypes = teacher + [vp, vp, flt, vp, i64, vp, sz, vp]
        L.mosaic_distill_loss_grad.restype = ci
        L.mosaic_distill_loss_grad.argtypes = teacher + [vp, vp, vp, flt, vp, i64, vp, sz, vp]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().mosaic_status_string(int(status)).decode()


def _check(status: int, what: str, allow=()):
    if status != OK and status not in allow:
        raise MosaicError(status, what)
    return status


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"unsupported dtype {t.dtype}: the library takes float32 or bfloat16")


def _dev(t: torch.Tensor, name: str, dtype=None, ndim=None) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor (no CPU path exists)")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims")
    return t


def _mat(t: torch.Tensor, name: str):
    _dev(t, name, ndim=2)
    if t.stride(1) != 1:
        raise ValueError(f"{name} must be row-major (unit stride along columns)")
    return t.data_ptr(), t.shape[0], t.shape[1], (t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1]))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream) -> int | None:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream or None


class Workspace:
    """Growable scratch (the library itself allocates nothing): a buffer of its own for every stream that calls are issued
    to and every host thread that issues them.  What two streams run at once, or two threads interleave on one, must not
    meet in one buffer; within a thread a stream's calls run one after another, and their scratch may be the same.
    A buffer belongs to its stream in the allocator's books as well: when the Workspace goes, it is handed on only behind
    the work that still uses it.  One that was outgrown is kept as long as the Workspace, for a captured graph may go on
    using it; each is at least twice the one before, so all that were outgrown are together smaller than the last.
    Graphs captured on one stream share its buffer: to replay two of them at once, give each a Workspace.  A graph uses the
    buffers of the Workspace that it was captured with, as it uses the tensors of its calls: all must live as long as it is
    replayed (the default one, used where none is given, always does)."""

    def __init__(self, device="cuda"):
        self.device = torch.device(device)
        self._bufs: dict[tuple, torch.Tensor] = {}     # (raw stream, thread) -> buffer
        self._outgrown: list[torch.Tensor] = []

    def get(self, nbytes: int, stream: int | None = None) -> tuple[int, int]:
        """(pointer, size) of at least `nbytes` for calls on `stream`: a raw handle (0: the default stream), None the current one."""
        if stream is None:
            stream = torch.cuda.current_stream(self.device).cuda_stream
        key = (stream, _thread())
        buf = self._bufs.get(key)
        if buf is None or buf.numel() < nbytes:
            least = 256
            if buf is not None:
                self._outgrown.append(buf)
                least = 2 * buf.numel()
            buf = self._bufs[key] = self._new(max(int(nbytes), least), stream)
            assert buf.data_ptr() % 256 == 0 or not buf.is_cuda
        return buf.data_ptr(), buf.numel()

    def _new(self, nbytes: int, stream: int) -> torch.Tensor:
        if self.device.type != "cuda":
            return torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        on = torch.cuda.ExternalStream(stream, self.device) if stream else torch.cuda.default_stream(self.device)
        with torch.cuda.stream(on):
            return torch.empty(nbytes, dtype=torch.uint8, device=self.device)


_default_ws: dict[int, Workspace] = {}


def _ws(ws: Workspace | None, device) -> Workspace:
    if ws is not None:
        return ws
    idx = device if isinstance(device, int) else torch.device(device).index
    idx = torch.cuda.current_device() if idx is None else idx
    found = _default_ws.get(idx)
    return found if found is not None else _default_ws.setdefault(idx, Workspace(torch.device("cuda", idx)))


# --------------------------------------------------------------------------- calls
def mosaic_version() -> int:
    return int(lib().mosaic_version())


def mosaic_act_norms(X: torch.Tensor, sumsq_accum: torch.Tensor, norms_out: torch.Tensor | None = None,
                     flags: int = 0, ws: Workspace | None = None, stream=None) -> None:
    """sumsq_accum[j] += sum_t X[t,j]^2 (fp64); optionally norms_out = sqrt (Eq. 5's norm term)."""
    xp, tokens, cols, ldx = _mat(X, "X")
    _dev(sumsq_accum, "sumsq_accum", torch.float64)
    if sumsq_accum.numel() != cols or (norms_out is not None and norms_out.numel() != cols):
        raise ValueError("sumsq_accum / norms_out must have one entry per column of X")
    if norms_out is not None:
        _dev(norms_out, "norms_out", torch.float32)
    L = lib()
    st = _stream(stream)
    wp, wn = _ws(ws, X.device).get(L.mosaic_act_norms_workspace_bytes(tokens, cols), st or 0)
    _check(L.mosaic_act_norms(xp, tokens, cols, ldx, _dtype_code(X), sumsq_accum.data_ptr(), _ptr(norms_out),
                              int(flags), wp, wn, st), "mosaic_act_norms")


def mosaic_gram_accumulate(X: torch.Tensor, G: torch.Tensor, flags: int = 0, status: torch.Tensor | None = None,
                           stream=None) -> None:
    """G[j,l] += sum_t X[t,j] X[t,l] (fp32, both triangles): the second moments of a projection's
    input, from which the inverse-Hessian back-end forms H = (2/T) G.  `status` (one int32 on the
    device) reads 1 after synchronisation if a bounded wait of the kernel ran out."""
    xp, tokens, cols, ldx = _mat(X, "X")
    _dev(G, "G", torch.float32)
    if G.dim() != 2 or tuple(G.shape) != (cols, cols) or G.stride(1) != 1:
        raise ValueError("G must be a [cols, cols] fp32 matrix with unit column stride")
    if status is not None:
        _dev(status, "status", torch.int32)
    _check(lib().mosaic_gram_accumulate(xp, tokens, cols, ldx, _dtype_code(X), G.data_ptr(), G.stride(0), int(flags),
                                        _ptr(status), _stream(stream)), "mosaic_gram_accumulate")


def mosaic_bounded_wait_selftest(budget_cycles: int, status: torch.Tensor, stream=None) -> None:
    """Diagnostic: the bounded mbarrier wait of the tensor-core kernel on its own, on a barrier that
    nothing completes.  `status` (one int32 on the device) reads 1 after synchronisation if the wait
    gave up after `budget_cycles` and raised the error word, as it must."""
    _dev(status, "status", torch.int32)
    _check(lib().mosaic_bounded_wait_selftest(int(budget_cycles), status.data_ptr(), _stream(stream)),
           "mosaic_bounded_wait_selftest")


def mosaic_score(W: torch.Tensor, norms: torch.Tensor, score_out: torch.Tensor, stream=None) -> None:
    """score_out[i,j] = norms[j] * |W[i,j]| in fp32 (Eq. 5, materialised)."""
    p, rows, cols, ldw = _mat(W, "W")
    _dev(norms, "norms", torch.float32)
    _dev(score_out, "score_out", torch.float32)
    if norms.numel() != cols or tuple(score_out.shape) != (rows, cols) or not score_out.is_contiguous():
        raise ValueError("norms must be [cols] and score_out a contiguous [rows, cols]")
    _check(lib().mosaic_score(p, rows, cols, ldw, _dtype_code(W), norms.data_ptr(), score_out.data_ptr(),
                              _stream(stream)), "mosaic_score")


def mosaic_outlier_ratio(W: torch.Tensor, norms: torch.Tensor, alpha: float, outlier_count_out: torch.Tensor,
                         score_sum_out: torch.Tensor | None = None, ws: Workspace | None = None, stream=None) -> None:
    """Eq. 6: outlier_count_out[0] = #{score > alpha*mean(score)}; score_sum_out[0] = fp64 sum of scores."""
    p, rows, cols, ldw = _mat(W, "W")
    _dev(norms, "norms", torch.float32)
    _dev(outlier_count_out, "outlier_count_out", torch.int64)
    if score_sum_out is not None:
        _dev(score_sum_out, "score_sum_out", torch.float64)
    if norms.numel() != cols:
        raise ValueError("norms must be [cols]")
    L = lib()
    st = _stream(stream)
    wp, wn = _ws(ws, W.device).get(L.mosaic_outlier_ratio_workspace_bytes(rows, cols), st or 0)
    _check(L.mosaic_outlier_ratio(p, rows, cols, ldw, _dtype_code(W), norms.data_ptr(), float(alpha),
                                  outlier_count_out.data_ptr(), _ptr(score_sum_out), wp, wn, st),
           "mosaic_outlier_ratio")


def mosaic_outlier_ratio_static(W: torch.Tensor, norms: torch.Tensor, alpha: float, outlier_count_out: torch.Tensor,
                                score_sum_out: torch.Tensor | None = None, stream=None) -> None:
    """mosaic_outlier_ratio for callers that cannot allocate device memory: no workspace is
    passed, the library uses the fixed scratch array it carries on the device.  Calls on one
    device share that array, so do not let two of them overlap on the GPU."""
    p, rows, cols, ldw = _mat(W, "W")
    _dev(norms, "norms", torch.float32)
    _dev(outlier_count_out, "outlier_count_out", torch.int64)
    if score_sum_out is not None:
        _dev(score_sum_out, "score_sum_out", torch.float64)
    if norms.numel() != cols:
        raise ValueError("norms must be [cols]")
    _check(lib().mosaic_outlier_ratio_static(p, rows, cols, ldw, _dtype_code(W), norms.data_ptr(), float(alpha),
                                             outlier_count_out.data_ptr(), _ptr(score_sum_out), _stream(stream)),
           "mosaic_outlier_ratio_static")


class OutlierJob(C.Structure):
    """mosaic_outlier_job of include/mosaic.h."""
    _fields_ = [("W", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ldw", C.c_int64),
                ("norms", C.c_void_p), ("outlier_count_out", C.c_void_p), ("score_sum_out", C.c_void_p)]


class OutlierBatch:
    """The marshalled job list of mosaic_outlier_ratio_batch for a list of
    (W, norms, outlier_count_out[1], score_sum_out[1] or None); the count tensors may be
    one-element views of a larger int64 tensor.  Checked and laid out once; run() only makes
    the call, so a caller that repeats the sweep over matrices that stay where they are pays
    the per-job Python work once.  The tensors are kept alive by the object."""

    def __init__(self, jobs):
        self.jobs = list(jobs)
        if not self.jobs:
            raise ValueError("empty batch")
        self.arr = (OutlierJob * len(self.jobs))()
        dtype = self.jobs[0][0].dtype
        for i, (W, norms, cnt, ssum) in enumerate(self.jobs):
            p, rows, cols, ldw = _mat(W, "W")
            if W.dtype != dtype:
                raise TypeError("one dtype per batch")
            _dev(norms, "norms", torch.float32)
            _dev(cnt, "outlier_count_out", torch.int64)
            if ssum is not None:
                _dev(ssum, "score_sum_out", torch.float64)
            if norms.numel() != cols:
                raise ValueError("norms must be [cols]")
            self.arr[i] = OutlierJob(p, rows, cols, ldw, norms.data_ptr(), cnt.data_ptr(), _ptr(ssum))
        self.code = _dtype_code(self.jobs[0][0])
        self.device = self.jobs[0][0].device
        self.ws_bytes = lib().mosaic_outlier_ratio_batch_workspace_bytes(C.addressof(self.arr), len(self.jobs))

    def run(self, alpha: float, ws: Workspace | None = None, stream=None, group_of=None) -> None:
        """group_of: None (every matrix against its own mean, Eq. 6) or one group id per job - adjacent jobs
        with equal ids are counted against the mean over the whole group (Eq. 3-4, layer outlier distribution)."""
        st = _stream(stream)
        wp, wn = _ws(ws, self.device).get(self.ws_bytes, st or 0)
        if group_of is None:
            _check(lib().mosaic_outlier_ratio_batch(C.addressof(self.arr), len(self.jobs), self.code, float(alpha), wp, wn,
                                                    st), "mosaic_outlier_ratio_batch")
            return
        if len(group_of) != len(self.jobs):
            raise ValueError("one group id per job")
        g = (C.c_int32 * len(self.jobs))(*[int(v) for v in group_of])
        _check(lib().mosaic_outlier_ratio_grouped(C.addressof(self.arr), C.addressof(g), len(self.jobs), self.code, float(alpha),
                                                  wp, wn, st), "mosaic_outlier_ratio_grouped")


def mosaic_outlier_ratio_batch(jobs, alpha: float, ws: Workspace | None = None, stream=None) -> None:
    """mosaic_outlier_ratio over a list of (W, norms, outlier_count_out[1], score_sum_out[1] or None)
    in a handful of launches (bf16: one sweep over the weights); the count tensors may be one-element
    views of a larger int64 tensor."""
    if jobs:
        OutlierBatch(jobs).run(alpha, ws, stream)


def mosaic_outlier_ratio_grouped(jobs, group_of, alpha: float, ws: Workspace | None = None, stream=None) -> None:
    """Eq. 3-4: as mosaic_outlier_ratio_batch, with adjacent jobs of equal group id sharing one threshold."""
    if jobs:
        OutlierBatch(jobs).run(alpha, ws, stream, group_of=group_of)


def mosaic_ratio_from_count(outlier_count: int, numel: int) -> float:
    return float(lib().mosaic_ratio_from_count(int(outlier_count), int(numel)))


def mosaic_allocate_sparsity(outlier_counts, numels, cols, n_layers: int, n_proj: int, p: float,
                             lam: float = 0.08, mode: int = GLOBAL_NORM):
    """Host call: (sparsity[N*M] fp64, k[N*M] int64, infeasible flag) from the outlier counts."""
    n = n_layers * n_proj
    oc, ne, cl = (np.ascontiguousarray(v, dtype=np.int64) for v in (outlier_counts, numels, cols))
    if not (oc.shape == ne.shape == cl.shape == (n,)):
        raise ValueError("outlier_counts, numels and cols need one entry per projection")
    s, k = np.empty(n, dtype=np.float64), np.empty(n, dtype=np.int64)
    st = _check(lib().mosaic_allocate_sparsity(oc.ctypes.data, ne.ctypes.data, cl.ctypes.data, n_layers, n_proj,
                                               float(p), float(lam), int(mode), s.ctypes.data, k.ctypes.data),
                "mosaic_allocate_sparsity", allow=(ERR_INFEASIBLE,))
    return s.tolist(), k.tolist(), st == ERR_INFEASIBLE


def _out_ptr(W_in: torch.Tensor, W_out: torch.Tensor | None, rows: int, cols: int, ldw: int):
    """Pointer of the pruned-weights output, or None for mask-only mode."""
    if W_out is None:
        return None
    po, r2, c2, ld2 = _mat(W_out, "W_out")
    if (r2, c2) != (rows, cols) or W_out.dtype != W_in.dtype or (rows > 1 and ld2 != ldw):
        raise ValueError("W_out must match W_in in shape, dtype and leading dimension")
    return po


def mosaic_prune_unstructured(W_in: torch.Tensor, W_out: torch.Tensor | None, norms: torch.Tensor, k: int,
                              mask_out: torch.Tensor | None = None, ws: Workspace | None = None, stream=None) -> None:
    """Per row, zero the k entries first under (score asc, column asc); optional keep bitmask.
    W_out None: mask-only mode (mask_out is then the only output)."""
    p, rows, cols, ldw = _mat(W_in, "W_in")
    po = _out_ptr(W_in, W_out, rows, cols, ldw)
    if W_out is None and mask_out is None:
        raise ValueError("mask-only mode needs mask_out")
    _dev(norms, "norms", torch.float32)
    if norms.numel() != cols:
        raise ValueError("norms must be [cols]")
    if mask_out is not None:
        _dev(mask_out, "mask_out", torch.int32)
        if tuple(mask_out.shape) != (rows, (cols + 31) // 32) or not mask_out.is_contiguous():
            raise ValueError("mask_out must be a contiguous int32 [rows, ceil(cols/32)]")
    _check(lib().mosaic_prune_unstructured(p, po, rows, cols, ldw, _dtype_code(W_in), norms.data_ptr(), int(k),
                                           _ptr(mask_out), None, 0, _stream(stream)), "mosaic_prune_unstructured")


class PruneJob(C.Structure):
    """mosaic_prune_job of include/mosaic.h."""
    _fields_ = [("W_in", C.c_void_p), ("W_out", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64),
                ("ldw", C.c_int64), ("norms", C.c_void_p), ("k", C.c_int64), ("mask_out", C.c_void_p)]


class PruneBatch:
    """The marshalled job list of mosaic_prune_unstructured_batch for a list of
    (W_in, W_out or None, norms, k, mask_out or None).  Checked and laid out once; run() may replace
    the per-row prune counts and then only makes the call.  The tensors are kept alive by the object."""

    def __init__(self, jobs):
        self.jobs = list(jobs)
        if not self.jobs:
            raise ValueError("empty batch")
        self.arr = (PruneJob * len(self.jobs))()
        dtype = self.jobs[0][0].dtype
        for i, (W_in, W_out, norms, k, mask_out) in enumerate(self.jobs):
            p, rows, cols, ldw = _mat(W_in, "W_in")
            po = _out_ptr(W_in, W_out, rows, cols, ldw)
            if W_in.dtype != dtype:
                raise TypeError("one dtype per batch")
            if W_out is None and mask_out is None:
                raise ValueError("mask-only mode needs mask_out")
            _dev(norms, "norms", torch.float32)
            if norms.numel() != cols:
                raise ValueError("norms must be [cols]")
            if mask_out is not None:
                _dev(mask_out, "mask_out", torch.int32)
                if tuple(mask_out.shape) != (rows, (cols + 31) // 32) or not mask_out.is_contiguous():
                    raise ValueError("mask_out must be a contiguous int32 [rows, ceil(cols/32)]")
            self.arr[i] = PruneJob(p, po, rows, cols, ldw, norms.data_ptr(), int(k), _ptr(mask_out))
        self.code = _dtype_code(self.jobs[0][0])
        self.device = self.jobs[0][0].device
        self.ws_bytes = lib().mosaic_prune_unstructured_batch_workspace_bytes(C.addressof(self.arr), len(self.jobs), self.code)

    def run(self, k=None, ws: Workspace | None = None, stream=None) -> None:
        """k: None (the counts given at construction) or one prune count per job."""
        if k is not None:
            if len(k) != len(self.jobs):
                raise ValueError("one k per job")
            # (the k fields of all jobs in one strided write: a job is 8 words, k the seventh)
            np.frombuffer(self.arr, dtype=np.int64).reshape(len(self.jobs), 8)[:, 6] = np.asarray(k, dtype=np.int64)
            self.ws_bytes = lib().mosaic_prune_unstructured_batch_workspace_bytes(C.addressof(self.arr), len(self.jobs), self.code)
        st = _stream(stream)
        wp, wn = _ws(ws, self.device).get(self.ws_bytes, st or 0)
        _check(lib().mosaic_prune_unstructured_batch(C.addressof(self.arr), len(self.jobs), self.code, wp, wn, st),
               "mosaic_prune_unstructured_batch")


def mosaic_prune_unstructured_batch(jobs, ws: Workspace | None = None, stream=None) -> None:
    """mosaic_prune_unstructured over a list of (W_in, W_out, norms, k, mask_out or None) in few launches."""
    if jobs:
        PruneBatch(jobs).run(None, ws, stream)


def mosaic_prune_structured_compact(W_in: torch.Tensor, norms: torch.Tensor | None, row_group: int, col_group: int,
                                    row_units_keep: int, col_units_keep: int, row_keep_units: torch.Tensor | None,
                                    col_keep_units: torch.Tensor | None, flags: int = 0,
                                    W_out: torch.Tensor | None = None, unit_scores_out: torch.Tensor | None = None,
                                    ws: Workspace | None = None, stream=None) -> None:
    """Unit scores -> ranked keep lists -> dense compacted W_out (see include/mosaic.h)."""
    p, rows, cols, ldw = _mat(W_in, "W_in")
    if norms is not None:
        _dev(norms, "norms", torch.float32)
    for t, nm, n in ((row_keep_units, "row_keep_units", row_units_keep), (col_keep_units, "col_keep_units", col_units_keep)):
        if t is not None:
            _dev(t, nm, torch.int32)
            if t.numel() < n:
                raise ValueError(f"{nm} is shorter than the number of kept units")
    if W_out is not None:
        _dev(W_out, "W_out", W_in.dtype)
        if not W_out.is_contiguous() or W_out.numel() < row_units_keep * row_group * col_units_keep * col_group:
            raise ValueError("W_out must be contiguous and hold the compacted matrix")
    if unit_scores_out is not None:
        _dev(unit_scores_out, "unit_scores_out", torch.float32)
        if unit_scores_out.numel() < rows // row_group + cols // col_group:
            raise ValueError("unit_scores_out too short")
    L = lib()
    st = _stream(stream)
    wp, wn = _ws(ws, W_in.device).get(L.mosaic_prune_structured_compact_workspace_bytes(rows, cols), st or 0)
    _check(L.mosaic_prune_structured_compact(p, rows, cols, ldw, _dtype_code(W_in), _ptr(norms), int(row_group),
                                             int(col_group), int(row_units_keep), int(col_units_keep),
                                             _ptr(row_keep_units), _ptr(col_keep_units), int(flags), _ptr(W_out),
                                             _ptr(unit_scores_out), wp, wn, st),
           "mosaic_prune_structured_compact")


def mosaic_rank_units(scores: torch.Tensor, keep: int, keep_out: torch.Tensor, stream=None) -> None:
    """Ascending indices of the `keep` units that survive removal of the lowest-scored ones."""
    _dev(scores, "scores", torch.float32)
    _dev(keep_out, "keep_out", torch.int32)
    if keep_out.numel() < keep:
        raise ValueError("keep_out too short")
    _check(lib().mosaic_rank_units(scores.data_ptr(), scores.numel(), int(keep), keep_out.data_ptr(), _stream(stream)),
           "mosaic_rank_units")


def mosaic_sum_unit_scores(dst: torch.Tensor, src: torch.Tensor, stream=None) -> None:
    """dst[u] += src[u] in fp32: running total of the unit scores of coupled projections."""
    _dev(dst, "dst", torch.float32)
    _dev(src, "src", torch.float32)
    if dst.numel() != src.numel() or not dst.is_contiguous() or not src.is_contiguous():
        raise ValueError("dst and src must be contiguous and of equal length")
    _check(lib().mosaic_sum_unit_scores(dst.data_ptr(), src.data_ptr(), dst.numel(), _stream(stream)),
           "mosaic_sum_unit_scores")


# --------------------------------------------------------------------------- batched structured steps
class UnitScoreJob(C.Structure):
    """mosaic_unit_score_job of include/mosaic.h."""
    _fields_ = [("W", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ldw", C.c_int64), ("norms", C.c_void_p),
                ("row_group", C.c_int64), ("col_group", C.c_int64), ("row_scores_out", C.c_void_p),
                ("col_scores_out", C.c_void_p)]


class AddJob(C.Structure):
    """mosaic_add_job of include/mosaic.h."""
    _fields_ = [("dst", C.c_void_p), ("a", C.c_void_p), ("b", C.c_void_p), ("n", C.c_int64)]


class RankJob(C.Structure):
    """mosaic_rank_job of include/mosaic.h."""
    _fields_ = [("scores", C.c_void_p), ("n_units", C.c_int64), ("keep", C.c_int64), ("keep_out", C.c_void_p)]


class CompactJob(C.Structure):
    """mosaic_compact_job of include/mosaic.h."""
    _fields_ = [("W_in", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ldw", C.c_int64),
                ("row_keep_units", C.c_void_p), ("row_units_keep", C.c_int64), ("row_group", C.c_int64),
                ("col_keep_units", C.c_void_p), ("col_units_keep", C.c_int64), ("col_group", C.c_int64),
                ("W_out", C.c_void_p)]


class UnitScoreBatch:
    """The marshalled job list of mosaic_unit_scores_batch for a list of (W, norms or None, row_group,
    col_group, row_scores_out or None, col_scores_out or None).  Checked and laid out once; run() only
    makes the call.  The tensors are kept alive by the object."""

    def __init__(self, jobs):
        self.jobs = list(jobs)
        if not self.jobs:
            raise ValueError("empty batch")
        self.arr = (UnitScoreJob * len(self.jobs))()
        dtype = self.jobs[0][0].dtype
        for i, (W, norms, rg, cg, rs, cs) in enumerate(self.jobs):
            p, rows, cols, ldw = _mat(W, "W")
            if W.dtype != dtype:
                raise TypeError("one dtype per batch")
            if norms is not None:
                _dev(norms, "norms", torch.float32)
            for t, nm, n in ((rs, "row_scores_out", rows // rg), (cs, "col_scores_out", cols // cg)):
                if t is not None:
                    _dev(t, nm, torch.float32)
                    if t.numel() < n or not t.is_contiguous():
                        raise ValueError(f"{nm} must be contiguous with one entry per unit")
            self.arr[i] = UnitScoreJob(p, rows, cols, ldw, _ptr(norms), int(rg), int(cg), _ptr(rs), _ptr(cs))
        self.code = _dtype_code(self.jobs[0][0])
        self.device = self.jobs[0][0].device
        self.ws_bytes = lib().mosaic_unit_scores_batch_workspace_bytes(C.addressof(self.arr), len(self.jobs))

    def run(self, ws: Workspace | None = None, stream=None) -> None:
        st = _stream(stream)
        wp, wn = _ws(ws, self.device).get(self.ws_bytes, st or 0)
        _check(lib().mosaic_unit_scores_batch(C.addressof(self.arr), len(self.jobs), self.code, wp, wn, st),
               "mosaic_unit_scores_batch")


class AddBatch:
    """The marshalled list of mosaic_add_unit_scores_batch for (dst, a, b) fp32 vectors of equal length."""

    def __init__(self, jobs):
        self.jobs = list(jobs)
        if not self.jobs:
            raise ValueError("empty batch")
        self.arr = (AddJob * len(self.jobs))()
        for i, (dst, a, b) in enumerate(self.jobs):
            for t, nm in ((dst, "dst"), (a, "a"), (b, "b")):
                _dev(t, nm, torch.float32)
                if not t.is_contiguous() or t.numel() != dst.numel():
                    raise ValueError("dst, a and b must be contiguous and of equal length")
            self.arr[i] = AddJob(dst.data_ptr(), a.data_ptr(), b.data_ptr(), dst.numel())

    def run(self, stream=None) -> None:
        _check(lib().mosaic_add_unit_scores_batch(C.addressof(self.arr), len(self.jobs), _stream(stream)),
               "mosaic_add_unit_scores_batch")


class RankBatch:
    """The marshalled list of mosaic_rank_units_batch for (scores, keep, keep_out)."""

    def __init__(self, jobs):
        self.jobs = list(jobs)
        if not self.jobs:
            raise ValueError("empty batch")
        self.arr = (RankJob * len(self.jobs))()
        for i, (scores, keep, keep_out) in enumerate(self.jobs):
            _dev(scores, "scores", torch.float32)
            _dev(keep_out, "keep_out", torch.int32)
            if keep_out.numel() < keep or not scores.is_contiguous():
                raise ValueError("keep_out too short or scores not contiguous")
            self.arr[i] = RankJob(scores.data_ptr(), scores.numel(), int(keep), keep_out.data_ptr())

    def run(self, stream=None) -> None:
        _check(lib().mosaic_rank_units_batch(C.addressof(self.arr), len(self.jobs), _stream(stream)), "mosaic_rank_units_batch")


class CompactBatch:
    """The marshalled list of mosaic_compact_batch for (W_in, row_keep_units, row_units_keep, row_group,
    col_keep_units, col_units_keep, col_group, W_out)."""

    def __init__(self, jobs):
        self.jobs = list(jobs)
        if not self.jobs:
            raise ValueError("empty batch")
        self.arr = (CompactJob * len(self.jobs))()
        dtype = self.jobs[0][0].dtype
        for i, (W_in, rk, n_rk, rg, ck, n_ck, cg, W_out) in enumerate(self.jobs):
            p, rows, cols, ldw = _mat(W_in, "W_in")
            if W_in.dtype != dtype:
                raise TypeError("one dtype per batch")
            _dev(rk, "row_keep_units", torch.int32)
            _dev(ck, "col_keep_units", torch.int32)
            _dev(W_out, "W_out", W_in.dtype)
            if rk.numel() < n_rk or ck.numel() < n_ck:
                raise ValueError("keep list shorter than the number of kept units")
            if not W_out.is_contiguous() or W_out.numel() < n_rk * rg * n_ck * cg:
                raise ValueError("W_out must be contiguous and hold the compacted matrix")
            self.arr[i] = CompactJob(p, rows, cols, ldw, rk.data_ptr(), int(n_rk), int(rg), ck.data_ptr(), int(n_ck), int(cg),
                                     W_out.data_ptr())
        self.code = _dtype_code(self.jobs[0][0])

    def run(self, stream=None) -> None:
        _check(lib().mosaic_compact_batch(C.addressof(self.arr), len(self.jobs), self.code, _stream(stream)),
               "mosaic_compact_batch")


def mosaic_unit_scores_batch(jobs, ws: Workspace | None = None, stream=None) -> None:
    """Unit scores of a list of (W, norms or None, row_group, col_group, row_scores_out or None,
    col_scores_out or None) in two launches."""
    if jobs:
        UnitScoreBatch(jobs).run(ws, stream)


def mosaic_add_unit_scores_batch(jobs, stream=None) -> None:
    """dst[u] = fl32(a[u] + b[u]) for a list of (dst, a, b): fp32 vectors of equal length."""
    if jobs:
        AddBatch(jobs).run(stream)


def mosaic_rank_units_batch(jobs, stream=None) -> None:
    """mosaic_rank_units for a list of (scores, keep, keep_out) in one launch."""
    if jobs:
        RankBatch(jobs).run(stream)


def mosaic_compact_batch(jobs, stream=None) -> None:
    """Dense compaction of a list of (W_in, row_keep_units, row_units_keep, row_group, col_keep_units,
    col_units_keep, col_group, W_out) in one launch."""
    if jobs:
        CompactBatch(jobs).run(stream)


# ------------------------------------------------------------------ recovery of a pruned model
_Tensor, _device, _raw_stream = torch.Tensor, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


# These calls are made many times per token or training step, so their marshalling is kept short: one helper per
# kind of argument, the raw stream handle, the workspace query only where the answer is not zero by inspection.
def _act_code(act) -> int:
    """An activation by its name or its code."""
    if isinstance(act, str):
        if act not in _ACTS:
            raise ValueError(f"unknown activation {act!r}: one of {sorted(_ACTS)}")
        return _ACTS[act]
    return int(act)


def _refuse(t, name: str, dtype, device: int, ndim: int | None):
    """The error of an argument that is no tensor of this type, number of dimensions (None: any) and device (-1: any)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor (no CPU path exists)")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims")
    if device >= 0 and t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}: the tensors of one call live on one device")


def _matrix(t, name: str, dtype, device: int = -1):
    """(pointer, rows, columns, leading dimension) of a row-major matrix; on `device`, if one is given."""
    if not isinstance(t, _Tensor) or t.dtype is not dtype or t.dim() != 2 or (t.get_device() != device if device >= 0 else not t.is_cuda):
        _refuse(t, name, dtype, device, 2)
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name} must be row-major (unit stride along columns)")
    return t.data_ptr(), rows, cols, (ld if rows > 1 else max(ld, cols))


def _like(t, name: str, dtype, device: int, rows: int, cols: int):
    """(pointer, leading dimension) of an optional [rows, cols] matrix."""
    if t is None:
        return None, cols
    if isinstance(t, _Tensor) and t.shape == (rows, cols) and t.dtype is dtype and t.get_device() == device:   # as it should be
        ld, step = t.stride()
        if step == 1 or cols <= 1:
            return t.data_ptr(), (ld if rows > 1 else max(ld, cols))
    p, r, c, ld = _matrix(t, name, dtype, device)
    if r != rows or c != cols:
        raise ValueError(f"{name} must be [{rows}, {cols}], got [{r}, {c}]")
    return p, ld


def _dense(t, name: str, dtype, device: int, *shape):
    """Pointer of a contiguous tensor of this shape."""
    if not isinstance(t, _Tensor) or t.dtype is not dtype or t.get_device() != device:
        _refuse(t, name, dtype, device, None)
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous {list(shape)}, got {list(t.shape)}")
    return t.data_ptr()


def _dense_or_none(t, name: str, dtype, device: int, *shape):
    return None if t is None else _dense(t, name, dtype, device, *shape)


def _run_on(t: torch.Tensor, stream):
    """(device index, raw stream) of a call: its tensors' device must be the current one, where it launches."""
    device = t.get_device()
    if device != _device():
        raise ValueError(f"the call's tensors are on cuda:{device}, the current device is cuda:{_device()}")
    return device, (_raw_stream(device) if stream is None else stream.cuda_stream) or None


@functools.lru_cache(maxsize=1024)
def _scratch(query: str, device: int, *sizes) -> int:
    """A workspace query whose answer depends on sizes (and the device) alone."""
    return getattr(lib(), query)(*sizes)


def _logits_code(t, name: str) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor (no CPU path exists)")
    return _dtype_code(t)


def mosaic_linear(X, W, Y, bias=None, residual=None, act=ACT_NONE, Z=None, status: torch.Tensor | None = None,
                  ws: Workspace | None = None, stream=None) -> None:
    """Y = act(X W^T + bias) + residual for bf16 X [tokens, in], W [out, in], Y / residual / Z [tokens, out]
    and bias [out]; Z, if given, receives the value before the activation.  `act` is one of the ACT_*
    codes or "none" / "relu" / "gelu" / "silu"; `residual` may be Y (added in place).  `status` (int32, one
    word) as in mosaic_gram_accumulate."""
    bf16 = torch.bfloat16
    xp, tokens, n_in, ldx = _matrix(X, "X", bf16)
    dev, st = _run_on(X, stream)
    wp, n_out, w_in, ldw = _matrix(W, "W", bf16, dev)
    if w_in != n_in:
        raise ValueError(f"W must be [out, {n_in}], got [{n_out}, {w_in}]")
    if Y is None:
        raise TypeError("Y must be a CUDA tensor")
    yp, ldy = _like(Y, "Y", bf16, dev, tokens, n_out)
    rp, ldr = _like(residual, "residual", bf16, dev, tokens, n_out)
    zp, ldz = _like(Z, "Z", bf16, dev, tokens, n_out)
    bp = _dense_or_none(bias, "bias", bf16, dev, n_out)
    sp = _dense_or_none(status, "status", torch.int32, dev, 1)
    L, sc, sn = lib(), None, 0
    if (xp | wp) & 15 or (ldx | ldw) & 7:      # an operand that is not 16-byte aligned is copied first
        need = L.mosaic_linear_workspace_bytes(xp, ldx, wp, ldw, tokens, n_out, n_in)
        if need:
            sc, sn = _ws(ws, dev).get(need, st or 0)
    _check(L.mosaic_linear(xp, ldx, wp, ldw, tokens, n_out, n_in, BF16, bp, rp, ldr, _act_code(act), yp, ldy, zp, ldz, sp, sc, sn, st),
           "mosaic_linear")


def mosaic_linear_backward(dY, X, W, Z=None, act=ACT_NONE, dX=None, dW=None, dbias=None, status: torch.Tensor | None = None,
                           ws: Workspace | None = None, stream=None) -> None:
    """Gradients of mosaic_linear: dX [tokens, in], dW [out, in], dbias [out] (each optional, all bf16) from dY
    [tokens, out], the inputs X and W, and - unless the activation is none - the stored Z."""
    bf16 = torch.bfloat16
    dyp, tokens, n_out, lddy = _matrix(dY, "dY", bf16)
    dev, st = _run_on(dY, stream)
    if X is None and W is None:
        raise TypeError("X or W must be given")
    if (dW is not None and X is None) or (dX is not None and W is None):
        raise ValueError("dW needs X and dX needs W")
    n_in = _matrix(X, "X", bf16, dev)[2] if X is not None else _matrix(W, "W", bf16, dev)[2]
    act = _act_code(act)
    if act != ACT_NONE and Z is None:
        raise ValueError("the backward pass of an activation needs the stored Z")
    xp, ldx = _like(X, "X", bf16, dev, tokens, n_in)
    wp, ldw = _like(W, "W", bf16, dev, n_out, n_in)
    zp, ldz = _like(Z, "Z", bf16, dev, tokens, n_out)
    dxp, lddx = _like(dX, "dX", bf16, dev, tokens, n_in)
    dwp, lddw = _like(dW, "dW", bf16, dev, n_out, n_in)
    dbp = _dense_or_none(dbias, "dbias", bf16, dev, n_out)
    sp = _dense_or_none(status, "status", torch.int32, dev, 1)
    L = lib()
    need = L.mosaic_linear_backward_workspace_bytes(dyp, lddy, xp, ldx, wp, ldw, tokens, n_out, n_in, act, dxp is not None, dwp is not None,
                                                    dbp is not None)
    sc, sn = _ws(ws, dev).get(need, st or 0) if need else (None, 0)
    _check(L.mosaic_linear_backward(dyp, lddy, xp, ldx, wp, ldw, zp, ldz, tokens, n_out, n_in, BF16, act, dxp, lddx, dwp, lddw, dbp, sp, sc, sn, st),
           "mosaic_linear_backward")


class _CheckpointStruct(C.Structure):
    """mosaic_checkpoint of include/mosaic.h."""
    _fields_ = [("codes", C.c_void_p), ("ldc", C.c_int64), ("exponents", C.c_void_p), ("lde", C.c_int64)]


class Checkpoint:
    """A matrix of activations in 8 bits: `codes` int8 [rows, cols rounded up to 16 or more] and `exponents` uint8
    [rows, ceil(cols / 16)], both with unit column stride.  The tensors are checked here and kept alive by the object; where one
    has been put in another place since, a call checks and reads what is there now."""

    def __init__(self, codes: torch.Tensor, exponents: torch.Tensor, cols: int):
        self.codes, self.exponents, self.cols = codes, exponents, int(cols)
        self._lay_out()

    def _lay_out(self) -> None:
        codes, exponents, cols = self.codes, self.exponents, self.cols
        groups = -(-cols // 16)
        for t, name, dtype, least in ((codes, "codes", torch.int8, 16 * groups), (exponents, "exponents", torch.uint8, groups)):
            _, rows, width, _ = _matrix(t, name, dtype)
            if cols <= 0 or width < least or rows != codes.shape[0]:
                raise ValueError(f"{name} must be [{codes.shape[0]}, {least}] or wider for {cols} columns, got {list(t.shape)}")
        if codes.device != exponents.device:
            raise ValueError("codes and exponents must be on one device")
        self.rows, self.device, self.at_codes, self.at_exponents = codes.shape[0], codes.get_device(), codes.data_ptr(), exponents.data_ptr()
        ldc = _matrix(codes, "codes", torch.int8)[3]
        self._struct = _CheckpointStruct(self.at_codes, -(-ldc // 16) * 16 if self.rows <= 1 else ldc, self.at_exponents,
                                         _matrix(exponents, "exponents", torch.uint8)[3])
        self.ptr = C.addressof(self._struct)

    @classmethod
    def empty(cls, rows: int, cols: int, device="cuda") -> "Checkpoint":
        groups = -(-int(cols) // 16)
        return cls(torch.empty(rows, 16 * groups, dtype=torch.int8, device=device), torch.empty(rows, groups, dtype=torch.uint8, device=device), cols)


def _saved(c, name: str, device: int, rows: int, cols: int):
    """Pointer of a checkpoint of a [rows, cols] matrix."""
    if not isinstance(c, Checkpoint):
        raise TypeError(f"{name} must be a Checkpoint")
    if c.codes.data_ptr() != c.at_codes or c.exponents.data_ptr() != c.at_exponents:
        c._lay_out()
    if c.rows != rows or c.cols != cols:
        raise ValueError(f"{name} must keep [{rows}, {cols}], keeps [{c.rows}, {c.cols}]")
    if c.device != device:
        raise ValueError(f"{name} is on cuda:{c.device}: the tensors of one call live on one device")
    return c.ptr


def _either(t, name: str, device: int, rows: int, cols: int):
    """(pointer, leading dimension, checkpoint pointer) of a bf16 matrix or its Checkpoint (None: neither)."""
    if isinstance(t, Checkpoint):
        return None, cols, _saved(t, name, device, rows, cols)
    return *_like(t, name, torch.bfloat16, device, rows, cols), None


def mosaic_checkpoint_store(X, out: Checkpoint, stream=None) -> None:
    """Keeps X (bf16 [rows, cols]) in 8 bits."""
    xp, rows, cols, ldx = _matrix(X, "X", torch.bfloat16)
    dev, st = _run_on(X, stream)
    _check(lib().mosaic_checkpoint_store(xp, rows, cols, ldx, BF16, _saved(out, "out", dev, rows, cols), st), "mosaic_checkpoint_store")


def mosaic_checkpoint_load(saved: Checkpoint, X, stream=None) -> None:
    """Writes the values that a checkpoint keeps to X (bf16 [rows, cols])."""
    xp, rows, cols, ldx = _matrix(X, "X", torch.bfloat16)
    dev, st = _run_on(X, stream)
    _check(lib().mosaic_checkpoint_load(_saved(saved, "saved", dev, rows, cols), rows, cols, xp, ldx, BF16, st), "mosaic_checkpoint_load")


def mosaic_gated_linear(X, W_gate, W_up, H, bias_gate=None, bias_up=None, act="silu", Z=None, U=None, status: torch.Tensor | None = None,
                        ws: Workspace | None = None, stream=None) -> None:
    """H = act(X W_gate^T + bias_gate) * (X W_up^T + bias_up) for bf16 X [tokens, in], W [channels, in], H [tokens,
    channels] and biases [channels].  Z and U, if given, receive the two before the activation and the product: bf16
    [tokens, channels], or both a Checkpoint."""
    bf16 = torch.bfloat16
    xp, tokens, n_in, ldx = _matrix(X, "X", bf16)
    dev, st = _run_on(X, stream)
    gp, n, g_in, ldg = _matrix(W_gate, "W_gate", bf16, dev)
    if g_in != n_in:
        raise ValueError(f"W_gate must be [channels, {n_in}], got [{n}, {g_in}]")
    if W_up is None or H is None:
        raise TypeError("W_up and H must be CUDA tensors")
    up, ldu = _like(W_up, "W_up", bf16, dev, n, n_in)
    hp, ldh = _like(H, "H", bf16, dev, tokens, n)
    zp, ldz, z8 = _either(Z, "Z", dev, tokens, n)
    vp, ldv, u8 = _either(U, "U", dev, tokens, n)
    if (z8 is None) != (u8 is None):
        raise ValueError("Z and U must both be checkpoints, or neither")
    bg = _dense_or_none(bias_gate, "bias_gate", bf16, dev, n)
    bu = _dense_or_none(bias_up, "bias_up", bf16, dev, n)
    sp = _dense_or_none(status, "status", torch.int32, dev, 1)
    L, sc, sn = lib(), None, 0
    if (xp | gp | up) & 15 or (ldx | ldg | ldu) & 7 or z8:
        need = L.mosaic_gated_linear_workspace_bytes(xp, ldx, gp, ldg, up, ldu, tokens, n, n_in, z8 is not None)
        if need:
            sc, sn = _ws(ws, dev).get(need, st or 0)
    _check(L.mosaic_gated_linear(xp, ldx, gp, ldg, up, ldu, tokens, n, n_in, BF16, bg, bu, _act_code(act), hp, ldh, zp, ldz, vp, ldv, z8, u8, sp,
                                 sc, sn, st), "mosaic_gated_linear")


def mosaic_gated_linear_backward(dH, X, W_gate, W_up, Z, U, act="silu", dX=None, dW_gate=None, dW_up=None, dbias_gate=None, dbias_up=None,
                                 H=None, status: torch.Tensor | None = None, ws: Workspace | None = None, stream=None) -> None:
    """Gradients of mosaic_gated_linear from dH [tokens, channels], its inputs and the Z and U that it kept: dX [tokens, in],
    dW_gate and dW_up [channels, in], dbias_gate and dbias_up [channels] (each optional, all bf16); H, if given, receives
    act(Z) * U once more.  X, and Z with U, may be a Checkpoint."""
    bf16 = torch.bfloat16
    dhp, tokens, n, lddh = _matrix(dH, "dH", bf16)
    dev, st = _run_on(dH, stream)
    want_dw = dW_gate is not None or dW_up is not None
    if Z is None or U is None:
        raise ValueError("the backward pass needs the Z and U that the forward pass kept")
    if (want_dw and X is None) or (dX is not None and (W_gate is None or W_up is None)):
        raise ValueError("dW_gate and dW_up need X, dX needs W_gate and W_up")
    sized = next((t for t in (X, W_gate, W_up) if t is not None), None)
    if sized is None:
        raise TypeError("X or a weight matrix must be given")
    n_in = sized.cols if isinstance(sized, Checkpoint) else _matrix(sized, "X" if sized is X else "W", bf16, dev)[2]
    xp, ldx, x8 = _either(X, "X", dev, tokens, n_in)
    gp, ldg = _like(W_gate, "W_gate", bf16, dev, n, n_in)
    up, ldu = _like(W_up, "W_up", bf16, dev, n, n_in)
    zp, ldz, z8 = _either(Z, "Z", dev, tokens, n)
    vp, ldv, u8 = _either(U, "U", dev, tokens, n)
    if (z8 is None) != (u8 is None):
        raise ValueError("Z and U must both be checkpoints, or neither")
    dxp, lddx = _like(dX, "dX", bf16, dev, tokens, n_in)
    dgp, lddg = _like(dW_gate, "dW_gate", bf16, dev, n, n_in)
    dup, lddu = _like(dW_up, "dW_up", bf16, dev, n, n_in)
    hp, ldh = _like(H, "H", bf16, dev, tokens, n)
    dbg = _dense_or_none(dbias_gate, "dbias_gate", bf16, dev, n)
    dbu = _dense_or_none(dbias_up, "dbias_up", bf16, dev, n)
    sp = _dense_or_none(status, "status", torch.int32, dev, 1)
    L = lib()
    # of the pointers the query looks at the alignment alone
    need = _scratch("mosaic_gated_linear_backward_workspace_bytes", dev, (xp or 0) & 15, ldx, x8 is not None, (gp or 0) & 15, ldg, (up or 0) & 15, ldu,
                    tokens, n, n_in, dX is not None, want_dw, dbg is not None or dbu is not None)
    sc, sn = _ws(ws, dev).get(need, st or 0) if need else (None, 0)
    _check(L.mosaic_gated_linear_backward(dhp, lddh, xp, ldx, x8, gp, ldg, up, ldu, zp, ldz, vp, ldv, z8, u8, tokens, n, n_in, BF16, _act_code(act),
                                          dxp, lddx, dgp, lddg, dup, lddu, dbg, dbu, hp, ldh, sp, sc, sn, st), "mosaic_gated_linear_backward")


class _Weight4Struct(C.Structure):
    """mosaic_weight4 of include/mosaic.h."""
    _fields_ = [("codes", C.c_void_p), ("ldc", C.c_int64), ("scales", C.c_void_p), ("lds", C.c_int64), ("group", C.c_int64)]


class Weight4:
    """A weight matrix in 4 bits: `codes` uint8 [rows, 16 for every 32 columns, or more] and `scales` bf16 [rows, ceil(cols /
    group)], both with unit column stride; `group` is 32, 64 or 128.  The tensors are checked here and kept alive by the
    object; where one has been put in another place since, a call checks and reads what is there now."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, cols: int, group: int):
        self.codes, self.scales, self.cols, self.group = codes, scales, int(cols), int(group)
        if self.group not in (32, 64, 128):
            raise ValueError(f"group must be 32, 64 or 128, got {group}")
        self._lay_out()

    def _lay_out(self) -> None:
        codes, scales, cols, group = self.codes, self.scales, self.cols, self.group
        for t, name, dtype, least in ((codes, "codes", torch.uint8, -(-cols // 32) * 16), (scales, "scales", torch.bfloat16, -(-cols // group))):
            _, rows, width, _ = _matrix(t, name, dtype)
            if cols <= 0 or width < least or rows != codes.shape[0]:
                raise ValueError(f"{name} must be [{codes.shape[0]}, {least}] or wider for {cols} columns, got {list(t.shape)}")
        if codes.device != scales.device:
            raise ValueError("codes and scales must be on one device")
        self.rows, self.device, self.at_codes, self.at_scales = codes.shape[0], codes.get_device(), codes.data_ptr(), scales.data_ptr()
        ldc = _matrix(codes, "codes", torch.uint8)[3]
        self._struct = _Weight4Struct(self.at_codes, -(-ldc // 16) * 16 if self.rows <= 1 else ldc, self.at_scales,
                                      _matrix(scales, "scales", torch.bfloat16)[3], group)
        self.ptr = C.addressof(self._struct)

    @classmethod
    def empty(cls, rows: int, cols: int, group: int = 128, device="cuda") -> "Weight4":
        return cls(torch.empty(rows, -(-int(cols) // 32) * 16, dtype=torch.uint8, device=device),
                   torch.empty(rows, -(-int(cols) // max(int(group), 1)), dtype=torch.bfloat16, device=device), cols, group)

    @classmethod
    def of(cls, W: torch.Tensor, group: int = 128) -> "Weight4":
        """W (bf16 [rows, cols]) in 4 bits."""
        out = cls.empty(*W.shape, group, W.device)
        mosaic_quantize4(W, out)
        return out


def _weight4(w, name: str, device: int, rows: int | None, cols: int):
    """Pointer of a 4-bit [rows, cols] matrix (rows None: any number)."""
    if not isinstance(w, Weight4):
        raise TypeError(f"{name} must be a Weight4")
    if w.codes.data_ptr() != w.at_codes or w.scales.data_ptr() != w.at_scales:
        w._lay_out()
    if (rows is not None and w.rows != rows) or w.cols != cols:
        raise ValueError(f"{name} must be [{'rows' if rows is None else rows}, {cols}], is [{w.rows}, {w.cols}]")
    if w.device != device:
        raise ValueError(f"{name} is on cuda:{w.device}: the tensors of one call live on one device")
    return w.ptr


def mosaic_quantize4(W, out: Weight4, stream=None) -> None:
    """Packs W (bf16 [rows, cols]) into 4 bits."""
    wp, rows, cols, ldw = _matrix(W, "W", torch.bfloat16)
    dev, st = _run_on(W, stream)
    _check(lib().mosaic_quantize4(wp, rows, cols, ldw, BF16, _weight4(out, "out", dev, rows, cols), st), "mosaic_quantize4")


def mosaic_dequantize4(W4: Weight4, W, stream=None) -> None:
    """Writes the values of a 4-bit matrix to W (bf16 [rows, cols]); they are bf16 numbers, exactly."""
    wp, rows, cols, ldw = _matrix(W, "W", torch.bfloat16)
    dev, st = _run_on(W, stream)
    _check(lib().mosaic_dequantize4(_weight4(W4, "W4", dev, rows, cols), rows, cols, wp, ldw, BF16, st), "mosaic_dequantize4")


FEW4_TOKENS = 256   # beyond, the products need scratch for a bf16 copy of the weights


def mosaic_linear4(X, W: Weight4, Y, bias=None, residual=None, act=ACT_NONE, status: torch.Tensor | None = None, ws: Workspace | None = None,
                   stream=None) -> None:
    """mosaic_linear with 4-bit weights: Y = act(X W^T + bias) + residual.  `residual` may be Y (added in place)."""
    bf16 = torch.bfloat16
    xp, tokens, n_in, ldx = _matrix(X, "X", bf16)
    dev, st = _run_on(X, stream)
    wp = _weight4(W, "W", dev, None, n_in)
    n_out = W.rows
    if Y is None:
        raise TypeError("Y must be a CUDA tensor")
    yp, ldy = _like(Y, "Y", bf16, dev, tokens, n_out)
    rp, ldr = _like(residual, "residual", bf16, dev, tokens, n_out)
    bp = _dense_or_none(bias, "bias", bf16, dev, n_out)
    sp = _dense_or_none(status, "status", torch.int32, dev, 1)
    L, sc, sn = lib(), None, 0
    if xp & 15 or ldx & 7 or tokens > FEW4_TOKENS:
        need = L.mosaic_linear4_workspace_bytes(xp, ldx, tokens, n_out, n_in)
        if need:
            sc, sn = _ws(ws, dev).get(need, st or 0)
    _check(L.mosaic_linear4(xp, ldx, wp, tokens, n_out, n_in, BF16, bp, rp, ldr, _act_code(act), yp, ldy, sp, sc, sn, st), "mosaic_linear4")


def mosaic_gated_linear4(X, W_gate: Weight4, W_up: Weight4, H, bias_gate=None, bias_up=None, act="silu", status: torch.Tensor | None = None,
                         ws: Workspace | None = None, stream=None) -> None:
    """mosaic_gated_linear with 4-bit weights: H = act(X W_gate^T + bias_gate) * (X W_up^T + bias_up)."""
    bf16 = torch.bfloat16
    xp, tokens, n_in, ldx = _matrix(X, "X", bf16)
    dev, st = _run_on(X, stream)
    gp = _weight4(W_gate, "W_gate", dev, None, n_in)
    n = W_gate.rows
    up = _weight4(W_up, "W_up", dev, n, n_in)
    if H is None:
        raise TypeError("H must be a CUDA tensor")
    hp, ldh = _like(H, "H", bf16, dev, tokens, n)
    bg = _dense_or_none(bias_gate, "bias_gate", bf16, dev, n)
    bu = _dense_or_none(bias_up, "bias_up", bf16, dev, n)
    sp = _dense_or_none(status, "status", torch.int32, dev, 1)
    L, sc, sn = lib(), None, 0
    if xp & 15 or ldx & 7 or tokens > FEW4_TOKENS:
        need = L.mosaic_gated_linear4_workspace_bytes(xp, ldx, tokens, n, n_in)
        if need:
            sc, sn = _ws(ws, dev).get(need, st or 0)
    _check(L.mosaic_gated_linear4(xp, ldx, gp, up, tokens, n, n_in, BF16, bg, bu, _act_code(act), hp, ldh, sp, sc, sn, st), "mosaic_gated_linear4")


def mosaic_top_logits(L, values, indices, lse=None, temperature: float = 1.0, ws: Workspace | None = None, stream=None) -> None:
    """The values.shape[1] largest logits of every row of L [rows, vocab] (fp32 or bf16), in order (value
    descending, ties by index): `values` fp32 and `indices` int32 [rows, top]; `lse`, fp32 [rows], receives
    log sum exp(L / temperature) over the whole row."""
    code = _logits_code(L, "L")
    lp, rows, vocab, ldl = _matrix(L, "L", L.dtype)
    dev, st = _run_on(L, stream)
    top = values.shape[-1] if isinstance(values, torch.Tensor) and values.dim() == 2 else 0
    vp = _dense(values, "values", torch.float32, dev, rows, top)
    ip = _dense(indices, "indices", torch.int32, dev, rows, top)
    sp = _dense_or_none(lse, "lse", torch.float32, dev, rows)
    wp, wn = _ws(ws, dev).get(_scratch("mosaic_top_logits_workspace_bytes", dev, rows, vocab, code, top), st or 0)
    _check(lib().mosaic_top_logits(lp, rows, vocab, ldl, code, top, temperature, vp, ip, sp, wp, wn, st), "mosaic_top_logits")


def _distill_args(S, t_values, t_indices, t_lse, row_weight, temperature, stream, ws):
    """What the three distillation calls share: (leading arguments, (rows, vocab, device), workspace, its size, stream)."""
    code = _logits_code(S, "S")
    sp, rows, vocab, lds = _matrix(S, "S", S.dtype)
    dev, st = _run_on(S, stream)
    top = t_values.shape[-1] if isinstance(t_values, torch.Tensor) and t_values.dim() == 2 else 0
    tv = _dense(t_values, "t_values", torch.float32, dev, rows, top)
    ti = _dense(t_indices, "t_indices", torch.int32, dev, rows, top)
    tl = _dense_or_none(t_lse, "t_lse", torch.float32, dev, rows)
    rw = _dense_or_none(row_weight, "row_weight", torch.float32, dev, rows)
    wp, wn = _ws(ws, dev).get(_scratch("mosaic_distill_workspace_bytes", dev, rows, top), st or 0)
    return (sp, rows, vocab, lds, code, tv, ti, top, tl, rw, temperature), (rows, vocab, dev), wp, wn, st


def mosaic_distill_loss(S, t_values, t_indices, loss, lse=None, t_lse=None, row_weight=None, temperature: float = 1.0,
                        ws: Workspace | None = None, stream=None) -> None:
    """Distillation loss of every row of the student's logits S [rows, vocab] (fp32 or bf16) against a teacher's
    kept logits (t_values fp32, t_indices int32 [rows, top]); `loss` and `lse` (optional) are fp32 [rows]."""
    args, (rows, _, dev), wp, wn, st = _distill_args(S, t_values, t_indices, t_lse, row_weight, temperature, stream, ws)
    lo, ls = _dense(loss, "loss", torch.float32, dev, rows), _dense_or_none(lse, "lse", torch.float32, dev, rows)
    _check(lib().mosaic_distill_loss(*args, lo, ls, wp, wn, st), "mosaic_distill_loss")


def mosaic_distill_grad(S, t_values, t_indices, lse, dS, t_lse=None, row_weight=None, grad_rows=None, grad_scale: float = 1.0,
                        temperature: float = 1.0, ws: Workspace | None = None, stream=None) -> None:
    """Gradient of mosaic_distill_loss with respect to S, from the lse that call stored; `grad_rows` (fp32 [rows]) times
    `grad_scale` is the gradient of each row's loss.  dS may be S."""
    args, (rows, vocab, dev), wp, wn, st = _distill_args(S, t_values, t_indices, t_lse, row_weight, temperature, stream, ws)
    ls = _dense(lse, "lse", torch.float32, dev, rows)
    gr = _dense_or_none(grad_rows, "grad_rows", torch.float32, dev, rows)
    if dS is None:
        raise TypeError("dS must be a CUDA tensor")
    dp, ldd = _like(dS, "dS", S.dtype, dev, rows, vocab)
    _check(lib().mosaic_distill_grad(*args, ls, gr, grad_scale, dp, ldd, wp, wn, st), "mosaic_distill_grad")


def mosaic_distill_loss_grad(S, t_values, t_indices, loss, lse, dS, t_lse=None, row_weight=None, grad_rows=None, grad_scale: float = 1.0,
                             temperature: float = 1.0, ws: Workspace | None = None, stream=None) -> None:
    """mosaic_distill_loss and mosaic_distill_grad in one pass over S (the training step, where the gradient of each row's
    loss is known beforehand).  `lse` may be None; dS may be S."""
    args, (rows, vocab, dev), wp, wn, st = _distill_args(S, t_values, t_indices, t_lse, row_weight, temperature, stream, ws)
    lo, ls = _dense(loss, "loss", torch.float32, dev, rows), _dense_or_none(lse, "lse", torch.float32, dev, rows)
    gr = _dense_or_none(grad_rows, "grad_rows", torch.float32, dev, rows)
    if dS is None:
        raise TypeError("dS must be a CUDA tensor")
    dp, ldd = _like(dS, "dS", S.dtype, dev, rows, vocab)
    _check(lib().mosaic_distill_loss_grad(*args, lo, ls, gr, grad_scale, dp, ldd, wp, wn, st), "mosaic_distill_loss_grad")
