"""l1csr: the training hot path of l1-regularised compressed learning on MI355X.

A thin ctypes binding over ``libl1csr.so`` (built by
``python -m paper_1905_07931_amd.build``).  The functions keep the names of
the C ABI in ``include/l1csr.h``; they only check and marshal arguments
(torch tensors on the GPU -> device pointers, torch's current HIP stream) and
raise :class:`L1CSRError` on a non-zero status.  Every computation runs in the
library's HIP kernels; there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import os
from array import array
from dataclasses import dataclass, field

__all__ = [
    "CSR", "CSC", "L1CSRError", "lib", "status_str", "workspace_bytes",
    "csr_spmm_fwd", "csc_build", "csc_update_vals", "csr_spmm_bwd_t", "dense_wgrad", "sddmm_masked_wgrad",
    "prox_l1_step", "csr_recompress", "prox_l1_recompress", "csr_compact", "csr_validate", "relu_fwd", "relu_bwd",
    "softmax_xent", "PROX_DENSE", "PROX_CSR", "F32", "BF16", "BF16X3",
    "prox_adaptive_step", "prox_adaptive_recompress", "SOLVER_RMSPROP", "SOLVER_ADAM", "AdaptiveState",
    "ConvGeom", "csr_conv_fwd", "csr_conv_bwd_data", "conv_im2col", "maxpool_fwd",
    "l1_step", "side_stream", "prox_l1_recompress_noalloc", "dense_wgrad_prox", "csr_recompress_counted",
    "dense_wgrad_prox_recompress", "csr_bitmap_build", "Bitmap", "SpmmPlan", "csr_spmm_plan", "csr_spmm_planned",
    "csr_spmm_bwd_t_plan", "csr_spmm_bwd_t_planned",
    "token_logp", "policy_loss", "preference_loss", "F16", "MuonState", "orthogonalize", "prox_muon_step",
    "prox_muon_recompress",
    "embedding_fwd", "EmbeddingPlan", "embedding_plan", "embedding_bwd", "embedding_masked_bwd",
    "residual_norm_fwd", "residual_norm_bwd", "ResidualNormGrads", "grad_norm", "clip_grad_norm",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libl1csr.so")

OK, EINVAL, ECAPACITY, EBADCSR, EHIP, EUNSUPPORTED, ESCRATCH = 0, -1, -2, -3, -4, -5, -6
NOALLOC_SCRATCH_BYTES = 16 << 20  # L1CSR_NOALLOC_SCRATCH_BYTES
PROX_DENSE, PROX_CSR = 0, 1
F32, BF16, BF16X3, F16 = 0, 1, 2, 3
SOLVER_RMSPROP, SOLVER_ADAM = 1, 2
OP_CSC_BUILD, OP_RECOMPRESS, OP_SDDMM, OP_SPMM, OP_COMPACT, OP_SOFTMAX_XENT = 1, 2, 3, 4, 5, 6
OP_PROX_RECOMPRESS = 7
OP_DENSE_WGRAD = 8
OP_WGRAD_PROX = 9
OP_WGRAD_PACKED = 10
OP_SDDMM_PACKED = 11
OP_SPMM_PACKED = 12
OP_PROX_DENSE = 13
OP_MUON = 14
OP_MUON_F16 = 15
OP_TOKEN_LOSS = 16
OP_EMBEDDING_PLAN = 17
OP_EMBEDDING_BWD = 18
OP_RESIDUAL_NORM = 19
OP_GRAD_NORM = 20
GATE_NONE, GATE_ROW, GATE_FULL = 0, 1, 2
MUON_MAX_STEPS = 32  # L1CSR_MUON_MAX_STEPS


class L1CSRError(RuntimeError):
    def __init__(self, name, status):
        self.status = status
        super().__init__(f"{name} failed: {status_str(status)} ({status})")


_lib = None


def lib():
    """Load the HIP library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_1905_07931_amd.build`")
        # torch ships its own libamdhip64.so.7; loaded first, it is the copy the
        # dynamic linker hands the library, so the process holds one HIP
        # runtime and torch's streams and memory are valid in the library's
        # launches (loaded the other way round, the library would bind the
        # system runtime and torch a second one)
        import torch  # noqa: F401
        L = C.CDLL(LIB_PATH)
        i32, i64, f32, vp, sz = C.c_int32, C.c_int64, C.c_float, C.c_void_p, C.c_size_t
        L.l1csr_status_str.argtypes = [C.c_int]
        L.l1csr_status_str.restype = C.c_char_p
        L.l1csr_workspace_bytes.argtypes = [C.c_int, i32, i32, i64, i32]
        L.l1csr_workspace_bytes.restype = sz
        L.l1csr_host_alloc_mapped.argtypes = [sz, C.POINTER(vp), C.POINTER(vp)]
        L.l1csr_host_free_mapped.argtypes = [vp]
        L.csr_spmm_fwd.argtypes = [i32, i32, i64, vp, vp, vp, vp, i64, i32, vp, i64, vp, sz, vp]
        L.csr_spmm_plan.argtypes = [i32, i32, i64, vp, vp, vp, i32, vp, sz, vp]
        L.csr_spmm_planned.argtypes = [i32, i32, i64, vp, vp, vp, vp, i64, i32, vp, i64, vp, sz, vp]
        L.csc_build.argtypes = [i32, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.csc_update_vals.argtypes = [i32, i64, vp, vp, vp, vp, vp]
        L.csr_spmm_bwd_t.argtypes = [i32, i32, i64, vp, vp, vp, vp, vp, vp, vp, i64, i32, vp, i64,
                                     vp, sz, vp]
        L.dense_wgrad.argtypes = [i32, i32, i32, vp, i64, vp, i64, vp, i64, C.c_int, vp, sz, vp]
        L.sddmm_masked_wgrad.argtypes = [i32, i32, i64, vp, vp, vp, i64, vp, i64, i32, vp, vp, sz, vp]
        L.prox_l1_step.argtypes = [C.c_int, i32, i32, i64, vp, vp, vp, vp, i64, f32, f32, vp, i64,
                                   vp, vp]
        L.csr_recompress.argtypes = [i32, i32, vp, i64, f32, vp, vp, vp, vp, i64, vp,
                                     C.POINTER(C.c_int64), vp, sz, vp]
        L.prox_l1_recompress.argtypes = [i32, i32, i64, vp, vp, vp, vp, i64, f32, f32, vp, vp, vp,
                                         i64, vp, C.POINTER(C.c_int64), vp, sz, vp]
        L.prox_l1_recompress_noalloc.argtypes = [i32, i32, i64, vp, vp, vp, vp, i64, f32, f32, vp, vp,
                                                 vp, i64, vp, C.POINTER(C.c_int64), vp]
        L.dense_wgrad_prox.argtypes = [i32, i32, i32, vp, i64, vp, i64, C.c_int, i64, vp, vp, vp, vp, vp, f32, f32,
                                       vp, i64, vp, vp, sz, vp]
        L.csr_recompress_counted.argtypes = [i32, i32, vp, i64, vp, vp, vp, vp, i64, vp, C.POINTER(C.c_int64),
                                             vp, sz, vp]
        L.csr_bitmap_build.argtypes = [i32, i32, i64, vp, vp, vp, vp, vp]
        L.prox_adaptive_step.argtypes = [C.c_int, C.c_int, i32, i32, i64, vp, vp, vp, vp, i64, vp, vp,
                                         i64, f32, f32, f32, f32, f32, i64, vp, i64, vp, vp, sz, vp]
        L.prox_adaptive_recompress.argtypes = [C.c_int, i32, i32, i64, vp, vp, vp, vp, i64, vp, vp, i64,
                                               f32, f32, f32, f32, f32, i64, vp, vp, vp, i64, vp,
                                               C.POINTER(C.c_int64), vp, sz, vp]
        L.csr_compact.argtypes = [i32, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.csr_conv_fwd.argtypes = [vp, i32, i64, vp, vp, vp, vp, i64, i32, vp, i64, vp]
        L.csr_conv_bwd_data.argtypes = [vp, i32, i64, vp, vp, vp, vp, i64, i32, vp, i64, vp]
        L.conv_im2col.argtypes = [vp, vp, i64, i32, vp, i64, vp]
        L.l1csr_maxpool_fwd.argtypes = [vp, vp, i64, i32, vp, i64, vp]
        L.csr_validate.argtypes = [i32, i32, i64, vp, vp, vp, vp]
        L.l1csr_relu_fwd.argtypes = [i64, vp, vp, vp]
        L.l1csr_relu_bwd.argtypes = [i64, vp, vp, vp, vp]
        L.l1csr_softmax_xent.argtypes = [i32, i32, vp, i64, vp, vp, vp, vp, sz, vp]
        L.l1csr_token_logp.argtypes = [i32, i32, C.c_int, vp, i64, vp, vp, vp, sz, vp]
        L.l1csr_policy_loss.argtypes = [i32, i32, C.c_int, vp, i64, vp, vp, vp, vp, vp, f32, f32, f32, vp, i64, vp, vp,
                                        vp, sz, vp]
        L.l1csr_preference_loss.argtypes = [i32, i32, C.c_int, vp, i64, vp, i32, vp, vp, vp, f32, f32, vp, i64, vp, vp,
                                            vp, sz, vp]
        for name, at in (("l1csr_policy_loss", 13), ("l1csr_preference_loss", 12)):  # (grad_scale in front of dlogits)
            plain = getattr(L, name).argtypes
            getattr(L, name + "_scaled").argtypes = [*plain[:at], f32, *plain[at:]]
        L.muon_update.argtypes = [i32, i32, C.c_int, vp, i64, vp, i64, vp, i64, f32, C.c_int, C.c_int, f32, f32, C.c_int,
                                  vp, i64, vp, sz, vp]
        L.l1csr_embedding_fwd.argtypes = [i32, i32, i32, C.c_int, vp, i64, vp, f32, C.c_int, vp, i64, vp]
        L.l1csr_embedding_csr_fwd.argtypes = [i32, i32, i64, vp, vp, vp, i32, vp, f32, vp, i64, vp]
        L.l1csr_embedding_plan.argtypes = [i32, i32, vp, vp, sz, vp]
        L.l1csr_embedding_bwd.argtypes = [i32, i32, i32, C.c_int, vp, i64, vp, sz, f32, C.c_int, vp, i64, vp, i64, vp, sz, vp]
        L.l1csr_embedding_masked_bwd.argtypes = [i32, i32, i64, vp, vp, i32, vp, i64, vp, sz, f32, vp, vp, sz, vp]
        L.l1csr_residual_norm_fwd.argtypes = [i32, i32, C.c_int, vp, i64, vp, i64, C.c_int, C.c_int, vp, i64, vp, vp, f32, f32,
                                              vp, i64, vp, i64, vp, sz, vp]
        L.l1csr_residual_norm_bwd.argtypes = [i32, i32, C.c_int, vp, i64, vp, i64, vp, i64, vp, i64, C.c_int, C.c_int, vp, i64,
                                              vp, vp, f32, f32, vp, i64, vp, i64, vp, i64, vp, vp, vp, sz, vp]
        L.l1csr_grad_norm.argtypes = [i32, vp, vp, vp, vp, vp, f32, vp, vp, sz, vp]
        L.l1csr_clip_grad_norm.argtypes = [i32, vp, vp, vp, vp, vp, vp, vp, vp, f32, f32, f32, C.c_int, vp, vp, sz, vp]
        for name in ("l1csr_embedding_fwd", "l1csr_embedding_csr_fwd", "l1csr_embedding_plan", "l1csr_embedding_bwd",
                     "l1csr_embedding_masked_bwd", "l1csr_residual_norm_fwd", "l1csr_residual_norm_bwd", "l1csr_grad_norm",
                     "l1csr_clip_grad_norm",
                     "l1csr_token_logp", "l1csr_policy_loss", "l1csr_preference_loss", "l1csr_policy_loss_scaled",
                     "l1csr_preference_loss_scaled", "muon_update", "csr_spmm_fwd", "csr_spmm_plan", "csr_spmm_planned", "csc_build", "csc_update_vals", "csr_spmm_bwd_t", "dense_wgrad",
                     "sddmm_masked_wgrad", "prox_l1_step", "csr_recompress", "prox_l1_recompress",
                     "prox_l1_recompress_noalloc", "dense_wgrad_prox", "csr_recompress_counted", "csr_bitmap_build",
                     "csr_compact", "csr_validate", "l1csr_relu_fwd", "l1csr_relu_bwd", "l1csr_softmax_xent",
                     "prox_adaptive_step", "prox_adaptive_recompress", "csr_conv_fwd",
                     "csr_conv_bwd_data", "conv_im2col", "l1csr_maxpool_fwd"):
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def status_str(status: int) -> str:
    return lib().l1csr_status_str(int(status)).decode()


@functools.lru_cache(maxsize=4096)  # a pure function of the sizes
def workspace_bytes(op: int, n_rows: int, n_cols: int, nnz: int, B: int) -> int:
    return int(lib().l1csr_workspace_bytes(op, n_rows, n_cols, nnz, B))


def _two_sizes(plain_op, packed_op, n_rows, n_cols, nnz, B):
    """The workspace of a call's packed route (its plain one where there is none) and the plain one."""
    plain = workspace_bytes(plain_op, n_rows, n_cols, nnz, B)
    return max(plain, workspace_bytes(packed_op, n_rows, n_cols, nnz, B)), plain


# ---------------------------------------------------------------------------
# marshalling helpers
# ---------------------------------------------------------------------------

_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _check(rc, name):
    if rc != OK:
        raise L1CSRError(name, rc)


def _p(t):
    return None if t is None else t.data_ptr()


class _HostWord:
    """One int32 of pinned host memory that kernels write directly
    (l1csr_host_alloc_mapped), as a call's d_nnz_out: the count reaches the
    host with the call's own kernels, and no copy is queued behind it."""

    def __init__(self, host: int, dev: int):
        self.host, self.dev, self.event = host, dev, None

    def value(self) -> int:
        return C.c_int32.from_address(self.host).value


class _HostWords:
    """A CSR holds one word for its lifetime; when it goes, the word returns
    here and is handed out again only after the event recorded behind its
    last write has completed.  Pages are never freed (queued work may still
    write them)."""
    PAGE = 1024  # words per page

    def __init__(self):
        self.free: list = []
        self.disabled = False

    def acquire(self):
        for i, w in enumerate(self.free):
            if w.event is None or w.event.query():
                return self.free.pop(i)
        if self.disabled:
            return None
        h, d = C.c_void_p(), C.c_void_p()
        if lib().l1csr_host_alloc_mapped(4 * self.PAGE, C.byref(h), C.byref(d)) != 0:
            self.disabled = True  # the runtime refused: the calls fall back to a queued copy
            return None
        words = [_HostWord(h.value + 4 * i, d.value + 4 * i) for i in range(self.PAGE)]
        self.free.extend(words[1:])
        return words[0]

    def release(self, w):
        self.free.append(w)


_words = _HostWords()


def _nnz_word(out):
    """The word `out` has kernels write its nnz into (acquired on first use),
    or None under graph capture or where no mapped memory is available."""
    import weakref
    torch = _torch()
    if torch.cuda.is_current_stream_capturing():
        return None
    w = getattr(out, "_word", None)
    if w is None:
        w = _words.acquire()
        if w is not None:
            out._word = w
            weakref.finalize(out, _words.release, w)
    return w


def _nnz_dev(out):
    w = _nnz_word(out)
    return None if w is None else w.dev


def _set_nnz(out, need, stream):
    """The host count a call returned (>= 0), else the count its kernels
    wrote into out's host word (an event behind them), else a queued copy.
    Whenever the call was given the word, the event goes behind it even if
    the host count is known: its kernels write the word all the same, and the
    pool hands the word to another CSR only once that write is done."""
    torch = _torch()
    w = getattr(out, "_word", None)
    capturing = torch.cuda.is_current_stream_capturing()
    ev = None
    if w is not None and not capturing:
        s = torch.cuda.current_stream(out.row_ptr.device) if stream is None else stream
        ev = torch.cuda.Event()
        ev.record(s)
        w.event = ev
    if need >= 0:
        out.nnz = int(need)
        out._pending = None
        return
    if ev is None:
        out.track_nnz(stream)
        return
    out.nnz = None
    out._pending = (w, ev)


def _raw_stream(device_index):
    """The handle of a device's current stream, without a Stream object around it."""
    return _torch()._C._cuda_getCurrentRawStream(device_index)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(_torch().cuda.current_device())


def _dev(t, dtype, name):
    torch = _torch_module or _torch()
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype:
        return t
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must live on the GPU (got {t.device})")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    return t


def _vec(t, dtype, name):
    _dev(t, dtype, name)
    if t.dim() != 1 or (t.stride()[0] != 1 and t.numel() > 1):
        raise ValueError(f"{name} must be a contiguous 1-D tensor")
    return t


def _mat(t, name):
    """A [rows][ld] float32 matrix with unit column stride; returns (rows, cols, ld)."""
    _dev(t, (_torch_module or _torch()).float32, name)
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{name} must be 2-D")
    rows, cols = shape
    ld, unit = t.stride()
    if unit != 1 and cols > 1:
        raise ValueError(f"{name} must have a contiguous last dimension")
    return rows, cols, ld if rows > 1 else max(cols, 1)


_DTYPES: dict = {}  # torch dtype -> l1csr_dtype


def _kinds():
    """The element types of the calls that take more than float32: torch dtype -> l1csr_dtype."""
    if not _DTYPES:
        torch = _torch()
        _DTYPES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    return _DTYPES


def _dtype_code(t, name):
    """l1csr_dtype of a GPU tensor."""
    torch = _torch_module or _torch()
    _kinds()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU (got {t.device})")
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16 (got {t.dtype})")
    return code


def _typed_mat(t, name):
    """A [rows][ld] matrix of one of the element types; returns (rows, cols, ld, l1csr_dtype)."""
    code = _dtype_code(t, name)
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{name} must be 2-D")
    rows, cols = shape
    ld, unit = t.stride()
    if (unit != 1 and cols > 1) or (rows > 1 and ld < cols):
        raise ValueError(f"{name} must have a contiguous last dimension and rows that do not overlap")
    return rows, cols, ld if rows > 1 else max(cols, 1), code


def _device_of(first):
    """The device index of a call's first tensor, which has to be the current one: a call launches on the
    current device's stream."""
    index = first.get_device()
    if index != _torch_module.cuda.current_device():
        raise ValueError(f"the tensors live on {first.device}: make it the current device "
                         "(torch.cuda.device) for the call")
    return index


def _same_device(index, t, name):
    if t.get_device() != index:
        raise ValueError(f"{name} lives on {t.device}, another tensor on device {index}")
    return t


def _vec_of(t, dtype, n, index, name, what):
    """A contiguous vector of n values on device `index`."""
    if isinstance(t, _torch_module.Tensor) and t.dtype is dtype and t.shape == (n,) and t.get_device() == index and \
            t.is_contiguous():
        return t
    _vec(t, dtype, name)
    if t.numel() != n:
        raise ValueError(f"{name} must hold one value per {what}")
    return _same_device(index, t, name)


def _new(shape, dtype, device, stream):
    """An output of a call, allocated in the order of the stream that the call runs on."""
    torch = _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


_ws_cache: dict = {}
_WS_KEEP = 512 << 20  # the largest buffer kept for a stream


def _empty_bytes(nbytes, device, stream):
    """A buffer allocated with its stream current: the caching allocator reuses
    it only in that stream's order once it is dropped."""
    torch = _torch()
    with torch.cuda.stream(torch.cuda.current_stream(device) if stream is None else stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _workspace(nbytes, device, stream=None, least=None, keep=True):
    """Scratch for one call, cached per (device, stream the call runs on): calls
    on one stream run in order and may share it, calls on two streams never do.
    Beyond _WS_KEEP bytes, without `keep` or while the current stream is being
    captured, the buffer is the call's own and goes back to the caching allocator
    behind it (to the graph's memory pool under capture: a graph shares its scratch
    neither with eager calls nor with another graph that is replayed beside it, and
    keeps it when a later call needs a larger buffer).  A call that can do with
    `least` bytes (its route without the packed operands) gets those where
    memory for `nbytes` is short.  Returns (buffer or None, its bytes)."""
    if nbytes == 0:
        return None, 0
    if keep and _torch().cuda.is_current_stream_capturing():
        keep = False
    index = device.index
    key = (index, _raw_stream(index) if stream is None else stream.cuda_stream)
    buf = _ws_cache.get(key) if keep else None
    if buf is None or buf.numel() < nbytes:
        try:
            buf = _empty_bytes(nbytes, device, stream)
        except _torch().OutOfMemoryError:
            if least is None or least >= nbytes:
                raise
            return _workspace(least, device, stream, keep=keep)
        if keep and nbytes <= _WS_KEEP:
            _ws_cache[key] = buf
    return buf, nbytes


@dataclass
class CSR:
    """An N x K CSR matrix in device memory (int32 indices, float32 values).

    ``nnz`` is the host-side count when known.  A call that writes a CSR
    without waiting (:func:`csr_recompress`, :func:`prox_l1_recompress`, ...
    at full capacity) leaves it ``None``: ``row_ptr[-1]`` holds it on the
    device, and the call's own kernels have also written it into a word of
    mapped pinned host memory that the CSR keeps (or, where the runtime gives
    no such memory, the call has queued a copy behind its last kernel).  The
    first use of the matrix then waits for that call only (an event), not for
    the whole device; set ``nnz`` beforehand (e.g. under graph capture) to
    avoid the wait.
    ``col_idx``/``vals`` may be longer than nnz (capacity).
    """
    n_rows: int
    n_cols: int
    row_ptr: "object"
    col_idx: "object"
    vals: "object"
    nnz: int | None = None
    _pending: "object" = None  # (pinned int32 holding nnz (a copy or a word kernels write), its event)

    def host_nnz(self) -> int:
        if self.nnz is None:
            if self._pending is not None:
                host, ev = self._pending
                ev.synchronize()
                self.nnz = host.value() if isinstance(host, _HostWord) else int(host[0])
            else:
                self.nnz = int(self.row_ptr[-1].item())
        self._pending = None
        return self.nnz

    def track_nnz(self, stream=None):
        """Queue the copy of row_ptr[-1] to pinned host memory on `stream`
        (after the kernels that wrote it) and forget the host count."""
        torch = _torch()
        s = torch.cuda.current_stream(self.row_ptr.device) if stream is None else stream
        self.nnz = None
        self._pending = None
        if torch.cuda.is_current_stream_capturing():
            return  # a captured graph has no host copy to wait for: the caller sets nnz
        host = torch.empty(1, dtype=torch.int32, pin_memory=True)
        with torch.cuda.stream(s):
            host.copy_(self.row_ptr[-1:], non_blocking=True)
            ev = torch.cuda.Event()
            ev.record(s)
        self._pending = (host, ev)

    def validate_shapes(self):
        torch = _torch()
        _vec(self.row_ptr, torch.int32, "row_ptr")
        _vec(self.col_idx, torch.int32, "col_idx")
        _vec(self.vals, torch.float32, "vals")
        if self.row_ptr.numel() != self.n_rows + 1:
            raise ValueError("row_ptr must have n_rows + 1 entries")
        # the stored count sizes plans and workspaces: never guess it from the capacity
        nnz = self.host_nnz()
        if self.col_idx.numel() < nnz or self.vals.numel() < nnz:
            raise ValueError("col_idx/vals shorter than nnz")
        return nnz

    @staticmethod
    def from_host(row_ptr, col_idx, vals, n_cols, device="cuda", capacity=None):
        torch = _torch()
        import numpy as np
        rp = torch.as_tensor(np.ascontiguousarray(row_ptr, dtype=np.int32), device=device)
        nnz = int(rp[-1].item()) if rp.numel() else 0
        cap = max(nnz if capacity is None else capacity, 1)
        ci = torch.zeros(cap, dtype=torch.int32, device=device)
        v = torch.zeros(cap, dtype=torch.float32, device=device)
        if nnz:
            ci[:nnz] = torch.as_tensor(np.ascontiguousarray(col_idx[:nnz], dtype=np.int32), device=device)
            v[:nnz] = torch.as_tensor(np.ascontiguousarray(vals[:nnz], dtype=np.float32), device=device)
        return CSR(rp.numel() - 1, n_cols, rp, ci, v, nnz)

    def to_host(self):
        nnz = self.host_nnz()
        return (self.row_ptr.cpu().numpy(), self.col_idx[:nnz].cpu().numpy(),
                self.vals[:nnz].cpu().numpy())


@dataclass
class CSC:
    """Column-major copy of a CSR matrix: col_ptr, row_idx, perm (CSR position of
    each entry) and vals_t (its value)."""
    col_ptr: "object"
    row_idx: "object"
    perm: "object"
    vals_t: "object"

    @staticmethod
    def empty(n_cols, capacity, device):
        torch = _torch()
        cap = max(int(capacity), 1)
        return CSC(torch.empty(n_cols + 1, dtype=torch.int32, device=device),
                   torch.empty(cap, dtype=torch.int32, device=device),
                   torch.empty(cap, dtype=torch.int32, device=device),
                   torch.empty(cap, dtype=torch.float32, device=device))


# ---------------------------------------------------------------------------
# the ABI, one function per entry point
# ---------------------------------------------------------------------------

def csr_spmm_fwd(W: CSR, X, Y=None, stream=None):
    """Y = W . X  (X [K][B], Y [N][B], batch contiguous)."""
    torch = _torch()
    nnz = W.validate_shapes()
    K, B, ldx = _mat(X, "X")
    if K != W.n_cols:
        raise ValueError(f"X has {K} rows, W has {W.n_cols} columns")
    if Y is None:
        Y = torch.empty((W.n_rows, B), dtype=torch.float32, device=X.device)
    N, By, ldy = _mat(Y, "Y")
    if N != W.n_rows or By != B:
        raise ValueError("Y must be [n_rows][B]")
    need, least = _two_sizes(OP_SPMM, OP_SPMM_PACKED, W.n_rows, W.n_cols, nnz, B)
    ws, wsb = _workspace(need, X.device, stream, least)
    _check(lib().csr_spmm_fwd(W.n_rows, W.n_cols, nnz, _p(W.row_ptr), _p(W.col_idx), _p(W.vals),
                              _p(X), ldx, B, _p(Y), ldy, _p(ws), wsb, _stream(stream)),
           "csr_spmm_fwd")
    return Y


class SpmmPlan:
    """A caller-owned plan of a tiled product (csr_spmm_plan): its device
    buffer and the (n_rows, n_cols, nnz, B) it was made for.  Where the product
    packs its operands instead (OP_SPMM_PACKED) there is nothing to plan: the
    plan is empty and the planned call is the whole product."""

    def __init__(self, n_rows, n_cols, nnz, B, device):
        self.buf = None
        self.device = device
        self.reshape(n_rows, n_cols, nnz, B)

    def reshape(self, n_rows, n_cols, nnz, B):
        """Take this buffer for another shape, growing it if it is too small
        (the caller orders the reuse after the last use of the old plan)."""
        torch = _torch()
        self.key = (n_rows, n_cols, nnz, B)
        self.packed = workspace_bytes(OP_SPMM_PACKED, n_rows, n_cols, nnz, B) > 0
        self.nbytes = 0 if self.packed else workspace_bytes(OP_SPMM, n_rows, n_cols, nnz, B)
        if self.nbytes and (self.buf is None or self.buf.numel() < self.nbytes):
            self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=self.device)
        return self


def _plan_args(plan, key):
    if plan.key != key:
        raise ValueError(f"plan made for (n_rows, n_cols, nnz, B) = {plan.key}, used for {key}")
    return _p(plan.buf), plan.nbytes


def csr_spmm_plan(W: CSR, B: int, plan: SpmmPlan | None = None, stream=None) -> SpmmPlan:
    """The planning launches of Y = W . X for a batch of B columns (no X needed)."""
    nnz = W.validate_shapes()
    key = (W.n_rows, W.n_cols, nnz, int(B))
    if plan is None:
        plan = SpmmPlan(*key, W.row_ptr.device)
    pp, pb = _plan_args(plan, key)
    if plan.packed:
        return plan
    _check(lib().csr_spmm_plan(W.n_rows, W.n_cols, nnz, _p(W.row_ptr), _p(W.col_idx), _p(W.vals), int(B), pp, pb,
                               _stream(stream)), "csr_spmm_plan")
    return plan


def csr_spmm_planned(W: CSR, X, plan: SpmmPlan, Y=None, stream=None):
    """Y = W . X from a plan made by csr_spmm_plan(W, B)."""
    torch = _torch()
    nnz = W.validate_shapes()
    K, B, ldx = _mat(X, "X")
    if K != W.n_cols:
        raise ValueError(f"X has {K} rows, W has {W.n_cols} columns")
    if Y is None:
        Y = torch.empty((W.n_rows, B), dtype=torch.float32, device=X.device)
    N, By, ldy = _mat(Y, "Y")
    if N != W.n_rows or By != B:
        raise ValueError("Y must be [n_rows][B]")
    pp, pb = _plan_args(plan, (W.n_rows, W.n_cols, nnz, B))
    if plan.packed:
        # the packed operands in a buffer of the call's own: like a plan it is shared with no
        # other call, so a captured graph keeps it and another thread does not reach it
        need, least = _two_sizes(OP_SPMM, OP_SPMM_PACKED, W.n_rows, W.n_cols, nnz, B)
        ws, wsb = _workspace(need, X.device, stream, least, keep=False)
        _check(lib().csr_spmm_fwd(W.n_rows, W.n_cols, nnz, _p(W.row_ptr), _p(W.col_idx), _p(W.vals), _p(X), ldx, B,
                                  _p(Y), ldy, _p(ws), wsb, _stream(stream)), "csr_spmm_planned")
        return Y
    _check(lib().csr_spmm_planned(W.n_rows, W.n_cols, nnz, _p(W.row_ptr), _p(W.col_idx), _p(W.vals), _p(X), ldx, B,
                                  _p(Y), ldy, pp, pb, _stream(stream)), "csr_spmm_planned")
    return Y


def _csc_as_csr(W: CSR, csc: CSC) -> CSR:
    """W^T in CSR form: the CSC copy's arrays (for the planned backward product)."""
    return CSR(W.n_cols, W.n_rows, csc.col_ptr, csc.row_idx, csc.vals_t, W.host_nnz())


def csr_spmm_bwd_t_plan(W: CSR, csc: CSC, B: int, plan: SpmmPlan | None = None, stream=None) -> SpmmPlan:
    """The planning launches of dX = W^T . dY over the CSC copy (needs W's pattern and values only)."""
    return csr_spmm_plan(_csc_as_csr(W, csc), B, plan, stream)


def csr_spmm_bwd_t_planned(W: CSR, dY, csc: CSC, plan: SpmmPlan, dX=None, stream=None):
    """dX = W^T . dY from a plan made by csr_spmm_bwd_t_plan (the same bits as csr_spmm_bwd_t)."""
    return csr_spmm_planned(_csc_as_csr(W, csc), dY, plan, dX, stream)


def csc_build(W: CSR, out: CSC | None = None, bitmap: "Bitmap | None" = None, stream=None) -> CSC:
    """Deterministic CSC copy of W (col_ptr, row_idx, perm, vals_t), built from
    W's bitmap index (given, or built by the call)."""
    nnz = W.validate_shapes()
    dev = W.row_ptr.device
    if out is None:
        out = CSC.empty(W.n_cols, max(nnz, 1), dev)
    ws, wsb = _workspace(workspace_bytes(OP_CSC_BUILD, W.n_rows, W.n_cols, nnz, 0), dev, stream)
    mask = None if bitmap is None else _p(bitmap.mask)
    pos = None if bitmap is None else _p(bitmap.pos)
    _check(lib().csc_build(W.n_rows, W.n_cols, nnz, _p(W.row_ptr), _p(W.col_idx), _p(W.vals), mask, pos,
                           _p(out.col_ptr), _p(out.row_idx), _p(out.perm), _p(out.vals_t), _p(ws),
                           wsb, _stream(stream)), "csc_build")
    return out


def csc_update_vals(W: CSR, csc: CSC, stream=None) -> CSC:
    """vals_t <- vals[perm] after a values-only update of W."""
    nnz = W.validate_shapes()
    _check(lib().csc_update_vals(W.n_cols, nnz, _p(csc.col_ptr), _p(csc.perm), _p(W.vals),
                                 _p(csc.vals_t), _stream(stream)), "csc_update_vals")
    return csc


def csr_spmm_bwd_t(W: CSR, dY, csc: CSC | None = None, dX=None, stream=None):
    """dX = W^T . dY through the CSC copy (deterministic) or, with csc=None, float atomics."""
    torch = _torch()
    nnz = W.validate_shapes()
    N, B, ldy = _mat(dY, "dY")
    if N != W.n_rows:
        raise ValueError("dY must be [n_rows][B]")
    if dX is None:
        dX = torch.empty((W.n_cols, B), dtype=torch.float32, device=dY.device)
    K, Bx, ldx = _mat(dX, "dX")
    if K != W.n_cols or Bx != B:
        raise ValueError("dX must be [n_cols][B]")
    cp = ri = vt = ws = None
    wsb = 0
    if csc is not None:
        cp, ri, vt = csc.col_ptr, csc.row_idx, csc.vals_t
        need, least = _two_sizes(OP_SPMM, OP_SPMM_PACKED, W.n_cols, W.n_rows, nnz, B)
        ws, wsb = _workspace(need, dY.device, stream, least)
    _check(lib().csr_spmm_bwd_t(W.n_rows, W.n_cols, nnz, _p(W.row_ptr), _p(W.col_idx), _p(W.vals),
                                _p(cp), _p(ri), _p(vt), _p(dY), ldy, B, _p(dX), ldx, _p(ws), wsb,
                                _stream(stream)), "csr_spmm_bwd_t")
    return dX


def dense_wgrad(dY, X, dW=None, precision=F32, stream=None):
    """dW = dY . X^T on the matrix cores: fp32 operands (F32); operands
    rounded to bf16 with exact products and fp32 sums (BF16); or operands split
    into bf16 hi + lo with three exact products per pair and fp32 sums (BF16X3,
    inside the fp32 contract)."""
    torch = _torch()
    N, B, ldy = _mat(dY, "dY")
    K, Bx, ldx = _mat(X, "X")
    if Bx != B:
        raise ValueError("dY and X must share the batch dimension")
    if dW is None:
        dW = torch.empty((N, K), dtype=torch.float32, device=dY.device)
    Nw, Kw, ldw = _mat(dW, "dW")
    if (Nw, Kw) != (N, K):
        raise ValueError("dW must be [N][K]")
    need, least = _two_sizes(OP_DENSE_WGRAD, OP_WGRAD_PACKED, N, K, 0, B)
    ws, wsb = _workspace(least if precision == BF16 else need, dY.device, stream, least)
    _check(lib().dense_wgrad(N, K, B, _p(dY), ldy, _p(X), ldx, _p(dW), ldw, int(precision), _p(ws), wsb,
                             _stream(stream)), "dense_wgrad")
    return dW


def sddmm_masked_wgrad(W: CSR, dY, X, gv=None, stream=None):
    """gv[p] = (dY . X^T)[row(p), col(p)] on W's pattern."""
    torch = _torch()
    nnz = W.validate_shapes()
    N, B, ldy = _mat(dY, "dY")
    K, Bx, ldx = _mat(X, "X")
    if N != W.n_rows or K != W.n_cols or Bx != B:
        raise ValueError("shape mismatch")
    if gv is None:
        gv = torch.empty(max(nnz, 1), dtype=torch.float32, device=dY.device)
    need, least = _two_sizes(OP_SDDMM, OP_SDDMM_PACKED, W.n_rows, W.n_cols, nnz, B)
    ws, wsb = _workspace(need, dY.device, stream, least)
    _check(lib().sddmm_masked_wgrad(W.n_rows, W.n_cols, nnz, _p(W.row_ptr), _p(W.col_idx), _p(dY),
                                    ldy, _p(X), ldx, B, _p(gv), _p(ws), wsb, _stream(stream)),
           "sddmm_masked_wgrad")
    return gv


def prox_l1_step(mode, W: CSR, G, eta, lam, Z=None, row_counts=None, stream=None):
    """Eq. (prox).  Dense mode returns Z (may be G itself); CSR mode updates W.vals in place."""
    torch = _torch()
    nnz = W.validate_shapes()
    if mode == PROX_CSR:
        _vec(G, torch.float32, "G")
        if G.numel() < nnz:
            raise ValueError("G must hold one gradient per stored entry")
        _check(lib().prox_l1_step(PROX_CSR, W.n_rows, W.n_cols, nnz, _p(W.row_ptr), _p(W.col_idx),
                                  _p(W.vals), _p(G), 0, float(eta), float(lam), None, 0, None,
                                  _stream(stream)), "prox_l1_step")
        return W
    N, K, ldg = _mat(G, "G")
    if (N, K) != (W.n_rows, W.n_cols):
        raise ValueError("G must be [n_rows][n_cols]")
    if Z is None:
        Z = torch.empty((N, K), dtype=torch.float32, device=G.device)
    Nz, Kz, ldz = _mat(Z, "Z")
    if (Nz, Kz) != (N, K):
        raise ValueError("Z must be [n_rows][n_cols]")
    if row_counts is not None:
        _vec(row_counts, torch.int32, "row_counts")
    _check(lib().prox_l1_step(PROX_DENSE, W.n_rows, W.n_cols, nnz, _p(W.row_ptr), _p(W.col_idx),
                              _p(W.vals), _p(G), ldg, float(eta), float(lam), _p(Z), ldz,
                              _p(row_counts), _stream(stream)), "prox_l1_step")
    return Z


def csr_recompress(Z, t=0.0, row_counts=None, capacity=None, out: CSR | None = None, stream=None):
    """Dense Z -> canonical CSR keeping |Z| > t.

    With the default capacity (N*K) the call never waits and the result's
    ``nnz`` is None (read ``row_ptr[-1]``).  With a smaller capacity it waits
    and raises L1CSRError(ECAPACITY) if the result does not fit.
    """
    torch = _torch()
    N, K, ldz = _mat(Z, "Z")
    dev = Z.device
    if out is None:
        cap = N * K if capacity is None else int(capacity)
        out = CSR(N, K, torch.empty(N + 1, dtype=torch.int32, device=dev),
                  torch.empty(max(cap, 1), dtype=torch.int32, device=dev),
                  torch.empty(max(cap, 1), dtype=torch.float32, device=dev), None)
    cap = min(out.col_idx.numel(), out.vals.numel()) if capacity is None else int(capacity)
    ws, wsb = _workspace(workspace_bytes(OP_RECOMPRESS, N, K, 0, 0), dev, stream)
    need = C.c_int64(-1)
    _check(lib().csr_recompress(N, K, _p(Z), ldz, float(t), _p(row_counts), _p(out.row_ptr),
                                _p(out.col_idx), _p(out.vals), cap, _nnz_dev(out), C.byref(need), _p(ws), wsb,
                                _stream(stream)), "csr_recompress")
    _set_nnz(out, need.value, stream)
    return out


@dataclass
class Bitmap:
    """Bitmap index of a CSR pattern, word-major: mask / pos
    [ceil(n_cols / 32)][n_rows] (csr_bitmap_build)."""
    mask: "object"
    pos: "object"

    @staticmethod
    def empty(n_rows, n_cols, device):
        torch = _torch()
        kw = max((n_cols + 31) // 32, 1)  # word-major: [kw][n_rows]
        return Bitmap(torch.empty((kw, max(n_rows, 1)), dtype=torch.int32, device=device),
                      torch.empty((kw, max(n_rows, 1)), dtype=torch.int32, device=device))


def csr_bitmap_build(W: CSR, bm: Bitmap | None = None, stream=None) -> Bitmap:
    """W's bitmap index for dense_wgrad_prox_recompress (depends on the pattern only)."""
    nnz = W.validate_shapes()
    if bm is None:
        bm = Bitmap.empty(W.n_rows, W.n_cols, W.row_ptr.device)
    kw = (W.n_cols + 31) // 32
    for t_ in (bm.mask, bm.pos):
        if not t_.is_contiguous() or t_.numel() < W.n_rows * kw:
            raise ValueError("bitmap arrays must be contiguous with n_rows * ceil(n_cols / 32) entries")
    _check(lib().csr_bitmap_build(W.n_rows, W.n_cols, nnz, _p(W.row_ptr), _p(W.col_idx), _p(bm.mask),
                                  _p(bm.pos), _stream(stream)), "csr_bitmap_build")
    return bm


def dense_wgrad_prox(W: CSR, dY, X, eta, lam, bitmap: Bitmap, Z=None, word_counts=None, precision=F32,
                     stream=None):
    """Z = S_{eta*lam}(W - eta * dY.X^T) ([N][K], dW never stored) and the
    nonzero count of every 32-column word of Z's rows ([N][ceil(K/32)]), one
    GEMM launch; W read through its bitmap index.  Returns (Z, word_counts)."""
    torch = _torch()
    nnz = W.validate_shapes()
    N, B, ldy = _mat(dY, "dY")
    K, Bx, ldx = _mat(X, "X")
    if (N, K) != (W.n_rows, W.n_cols) or Bx != B:
        raise ValueError("dY must be [N][B] and X [K][B] for an N x K layer")
    dev = dY.device
    if Z is None:
        Z = torch.empty((N, K), dtype=torch.float32, device=dev)
    rz, cz, ldz = _mat(Z, "Z")
    if (rz, cz) != (N, K):
        raise ValueError("Z must be [N][K]")
    kw = (K + 31) // 32
    if word_counts is None:
        word_counts = torch.empty((max(N, 1), max(kw, 1)), dtype=torch.int32, device=dev)
    if not word_counts.is_contiguous() or word_counts.numel() < N * kw:
        raise ValueError("word_counts must be contiguous with N * ceil(K/32) entries")
    ws, wsb = (None, 0)
    if precision != BF16:
        least = workspace_bytes(OP_WGRAD_PROX, N, K, nnz, B)
        ws, wsb = _workspace(max(least, workspace_bytes(OP_WGRAD_PACKED, N, K, 0, B)), dev, stream, least)
    _check(lib().dense_wgrad_prox(N, K, B, _p(dY), ldy, _p(X), ldx, int(precision), nnz, _p(W.row_ptr),
                                  _p(W.col_idx), _p(W.vals), _p(bitmap.mask), _p(bitmap.pos), float(eta), float(lam),
                                  _p(Z), ldz, _p(word_counts), _p(ws), wsb, _stream(stream)), "dense_wgrad_prox")
    return Z, word_counts


def csr_recompress_counted(Z, word_counts, out: CSR | None = None, capacity=None, stream=None) -> CSR:
    """Z -> CSR of its nonzeros using dense_wgrad_prox's word counts (Z read once)."""
    torch = _torch()
    N, K, ldz = _mat(Z, "Z")
    dev = Z.device
    if out is None:
        cap = N * K if capacity is None else int(capacity)
        out = CSR(N, K, torch.empty(N + 1, dtype=torch.int32, device=dev),
                  torch.empty(max(cap, 1), dtype=torch.int32, device=dev),
                  torch.empty(max(cap, 1), dtype=torch.float32, device=dev), None)
    cap = min(out.col_idx.numel(), out.vals.numel()) if capacity is None else int(capacity)
    ws, wsb = _workspace(workspace_bytes(OP_RECOMPRESS, N, K, 0, 0), dev, stream)
    need = C.c_int64(-1)
    _check(lib().csr_recompress_counted(N, K, _p(Z), ldz, _p(word_counts), _p(out.row_ptr), _p(out.col_idx),
                                        _p(out.vals), cap, _nnz_dev(out), C.byref(need), _p(ws), wsb, _stream(stream)),
           "csr_recompress_counted")
    _set_nnz(out, need.value, stream)
    return out


def dense_wgrad_prox_recompress(W: CSR, dY, X, eta, lam, Z=None, out: CSR | None = None,
                                precision=F32, capacity=None, bitmap: Bitmap | None = None, stream=None):
    """The whole l1 update: csr_bitmap_build (unless `bitmap` is given),
    dense_wgrad_prox and csr_recompress_counted, in that order on `stream`.
    Z = S_{eta*lam}(W - eta * dY.X^T) and W' = CSR(Z), bit for bit as
    dense_wgrad + prox_l1_step + csr_recompress.  Returns (Z, out)."""
    if bitmap is None:
        bitmap = csr_bitmap_build(W, stream=stream)
    Z, wc = dense_wgrad_prox(W, dY, X, eta, lam, bitmap, Z=Z, precision=precision, stream=stream)
    out = csr_recompress_counted(Z, wc, out=out, capacity=capacity, stream=stream)
    return Z, out


def prox_l1_recompress_noalloc(W: CSR, G, eta, lam, out: CSR, capacity=None, stream=None):
    """prox_l1_recompress without a workspace: the library's static per-device
    scratch (L1CSR_NOALLOC_SCRATCH_BYTES) serves the call, which allocates
    nothing; `out` must be given.  Calls of it that overlap on one GPU race."""
    nnz = W.validate_shapes()
    N, K, ldg = _mat(G, "G")
    if (N, K) != (W.n_rows, W.n_cols):
        raise ValueError("G must be [n_rows][n_cols]")
    cap = min(out.col_idx.numel(), out.vals.numel()) if capacity is None else int(capacity)
    need = C.c_int64(-1)
    _check(lib().prox_l1_recompress_noalloc(N, K, nnz, _p(W.row_ptr), _p(W.col_idx), _p(W.vals), _p(G),
                                            ldg, float(eta), float(lam), _p(out.row_ptr), _p(out.col_idx),
                                            _p(out.vals), cap, _nnz_dev(out), C.byref(need), _stream(stream)),
           "prox_l1_recompress_noalloc")
    _set_nnz(out, need.value, stream)
    return out


def prox_l1_recompress(W: CSR, G, eta, lam, capacity=None, out: CSR | None = None, stream=None):
    """W' = CSR(S_{eta*lam}(W - eta*G)) in one call (same bits as prox + recompress)."""
    torch = _torch()
    nnz = W.validate_shapes()
    N, K, ldg = _mat(G, "G")
    if (N, K) != (W.n_rows, W.n_cols):
        raise ValueError("G must be [n_rows][n_cols]")
    dev = G.device
    if out is None:
        cap = N * K if capacity is None else int(capacity)
        out = CSR(N, K, torch.empty(N + 1, dtype=torch.int32, device=dev),
                  torch.empty(max(cap, 1), dtype=torch.int32, device=dev),
                  torch.empty(max(cap, 1), dtype=torch.float32, device=dev), None)
    cap = min(out.col_idx.numel(), out.vals.numel()) if capacity is None else int(capacity)
    ws, wsb = _workspace(workspace_bytes(OP_PROX_RECOMPRESS, N, K, nnz, 0), dev, stream)
    return _prox_l1_recompress(W, nnz, G, ldg, eta, lam, cap, out, ws, wsb, stream)


def _prox_l1_recompress(W, nnz, G, ldg, eta, lam, cap, out, ws, wsb, stream):
    """The call itself, on checked arguments and memory that is there."""
    need = C.c_int64(-1)
    _check(lib().prox_l1_recompress(W.n_rows, W.n_cols, nnz, _p(W.row_ptr), _p(W.col_idx), _p(W.vals), _p(G), ldg,
                                    float(eta), float(lam), _p(out.row_ptr), _p(out.col_idx),
                                    _p(out.vals), cap, _nnz_dev(out), C.byref(need), _p(ws), wsb,
                                    _stream(stream)), "prox_l1_recompress")
    _set_nnz(out, need.value, stream)
    return out


@dataclass
class AdaptiveState:
    """Hyper-parameters and per-weight state of Prox-RMSProp / Prox-ADAM
    (Algorithms 1-2).  m (ADAM only) and v are float32 device tensors: [N][K]
    (a leading dimension >= K is allowed) for the dense form, [nnz] for the
    stored-entry form; both start at zero.  t is the step number of the next
    call (from 1); the binding increments it after each call."""
    solver: int
    v: object
    m: object = None
    eps: float = 1e-8
    beta1: float = 0.9
    beta2: float = 0.999
    t: int = 1

    @staticmethod
    def zeros(solver, shape, device, **kw):
        torch = _torch()
        v = torch.zeros(shape, dtype=torch.float32, device=device)
        m = torch.zeros(shape, dtype=torch.float32, device=device) if solver == SOLVER_ADAM else None
        return AdaptiveState(solver, v, m, **kw)


def _state_mat(st: AdaptiveState, N, K):
    n, k, lds = _mat(st.v, "v")
    if (n, k) != (N, K):
        raise ValueError("state v must be [n_rows][n_cols]")
    if st.solver == SOLVER_ADAM:
        if st.m is None:
            raise ValueError("Prox-ADAM needs the first-moment state m")
        nm, km, ldm = _mat(st.m, "m")
        if (nm, km, ldm) != (N, K, lds):
            raise ValueError("m and v must have the same shape and leading dimension")
    return lds


def prox_adaptive_step(mode, W: CSR, G, st: AdaptiveState, eta, lam, Z=None, row_counts=None,
                       stream=None):
    """One Prox-RMSProp / Prox-ADAM step (Algorithms 1-2).  Dense mode returns Z
    (may be G itself) and updates st.m, st.v in place; CSR mode updates W.vals
    and the per-entry state in place.  st.t advances by one."""
    torch = _torch()
    nnz = W.validate_shapes()
    m = st.m if st.solver == SOLVER_ADAM else None
    if mode == PROX_CSR:
        _vec(G, torch.float32, "G")
        _vec(st.v, torch.float32, "v")
        if m is not None:
            _vec(m, torch.float32, "m")
        if G.numel() < nnz or st.v.numel() < nnz or (m is not None and m.numel() < nnz):
            raise ValueError("G and the state must hold one entry per stored weight")
        _check(lib().prox_adaptive_step(PROX_CSR, st.solver, W.n_rows, W.n_cols, nnz, _p(W.row_ptr),
                                        _p(W.col_idx), _p(W.vals), _p(G), 0, _p(m), _p(st.v), 0,
                                        float(eta), float(lam), float(st.eps), float(st.beta1),
                                        float(st.beta2), int(st.t), None, 0, None, None, 0,
                                        _stream(stream)), "prox_adaptive_step")
        st.t += 1
        return W
    N, K, ldg = _mat(G, "G")
    if (N, K) != (W.n_rows, W.n_cols):
        raise ValueError("G must be [n_rows][n_cols]")
    lds = _state_mat(st, N, K)
    if Z is None:
        Z = torch.empty((N, K), dtype=torch.float32, device=G.device)
    Nz, Kz, ldz = _mat(Z, "Z")
    if (Nz, Kz) != (N, K):
        raise ValueError("Z must be [n_rows][n_cols]")
    if row_counts is not None:
        _vec(row_counts, torch.int32, "row_counts")
    ws, wsb = _workspace(workspace_bytes(OP_PROX_RECOMPRESS, N, K, nnz, 0), G.device, stream)
    _check(lib().prox_adaptive_step(PROX_DENSE, st.solver, N, K, nnz, _p(W.row_ptr), _p(W.col_idx),
                                    _p(W.vals), _p(G), ldg, _p(m), _p(st.v), lds, float(eta),
                                    float(lam), float(st.eps), float(st.beta1), float(st.beta2),
                                    int(st.t), _p(Z), ldz, _p(row_counts), _p(ws), wsb,
                                    _stream(stream)), "prox_adaptive_step")
    st.t += 1
    return Z


def prox_adaptive_recompress(W: CSR, G, st: AdaptiveState, eta, lam, capacity=None,
                             out: CSR | None = None, stream=None):
    """W' = CSR of the Prox-RMSProp / Prox-ADAM step over all N*K weights, in
    one call (same bits as prox_adaptive_step + csr_recompress); st.m, st.v are
    updated in place and st.t advances by one (not on a capacity error)."""
    torch = _torch()
    nnz = W.validate_shapes()
    N, K, ldg = _mat(G, "G")
    if (N, K) != (W.n_rows, W.n_cols):
        raise ValueError("G must be [n_rows][n_cols]")
    lds = _state_mat(st, N, K)
    m = st.m if st.solver == SOLVER_ADAM else None
    dev = G.device
    if out is None:
        cap = N * K if capacity is None else int(capacity)
        out = CSR(N, K, torch.empty(N + 1, dtype=torch.int32, device=dev),
                  torch.empty(max(cap, 1), dtype=torch.int32, device=dev),
                  torch.empty(max(cap, 1), dtype=torch.float32, device=dev), None)
    cap = min(out.col_idx.numel(), out.vals.numel()) if capacity is None else int(capacity)
    need_ws = least = workspace_bytes(OP_PROX_RECOMPRESS, N, K, nnz, 0)
    if cap >= N * K:
        need_ws = max(need_ws, workspace_bytes(OP_PROX_DENSE, N, K, 0, 0))
    ws, wsb = _workspace(need_ws, dev, stream, least)
    need = C.c_int64(-1)
    _check(lib().prox_adaptive_recompress(st.solver, N, K, nnz, _p(W.row_ptr), _p(W.col_idx),
                                          _p(W.vals), _p(G), ldg, _p(m), _p(st.v), lds, float(eta),
                                          float(lam), float(st.eps), float(st.beta1),
                                          float(st.beta2), int(st.t), _p(out.row_ptr),
                                          _p(out.col_idx), _p(out.vals), cap, _nnz_dev(out), C.byref(need),
                                          _p(ws), wsb, _stream(stream)), "prox_adaptive_recompress")
    st.t += 1
    _set_nnz(out, need.value, stream)
    return out


@dataclass
class ConvGeom:
    """Convolution geometry: input channels C, maps H x W, filters KH x KW,
    stride SH x SW, zero padding PH x PW."""
    C: int
    H: int
    W: int
    KH: int
    KW: int
    SH: int = 1
    SW: int = 1
    PH: int = 0
    PW: int = 0

    @property
    def out_hw(self):
        return ((self.H + 2 * self.PH - self.KH) // self.SH + 1,
                (self.W + 2 * self.PW - self.KW) // self.SW + 1)

    @property
    def in_rows(self):
        return self.C * self.H * self.W

    @property
    def filter_cols(self):
        return self.C * self.KH * self.KW

    def _arr(self):
        return _geom_array(self.C, self.H, self.W, self.KH, self.KW, self.SH, self.SW, self.PH, self.PW)


@functools.lru_cache(maxsize=256)
def _geom_array(*sizes):
    """The calls' geometry argument (only ever read) for these sizes."""
    return (C.c_int32 * 9)(*sizes)


def csr_conv_fwd(g: ConvGeom, W: CSR, X, Y=None, stream=None):
    """Output maps [n_out*OH*OW][B] of the CSR filter bank W on maps X [C*H*W][B]."""
    torch = _torch()
    nnz = W.validate_shapes()
    rows, B, ldx = _mat(X, "X")
    if rows != g.in_rows or W.n_cols != g.filter_cols:
        raise ValueError("X must be [C*H*W][B] and W must have C*KH*KW columns")
    OH, OW = g.out_hw
    if Y is None:
        Y = torch.empty((W.n_rows * OH * OW, B), dtype=torch.float32, device=X.device)
    ry, by, ldy = _mat(Y, "Y")
    if (ry, by) != (W.n_rows * OH * OW, B):
        raise ValueError("Y must be [n_out*OH*OW][B]")
    _check(lib().csr_conv_fwd(g._arr(), W.n_rows, nnz, _p(W.row_ptr), _p(W.col_idx), _p(W.vals), _p(X), ldx,
                              B, _p(Y), ldy, _stream(stream)), "csr_conv_fwd")
    return Y


def csr_conv_bwd_data(g: ConvGeom, n_out: int, csc: CSC, dY, dX=None, nnz=None, stream=None):
    """Input-map gradient [C*H*W][B] from dY [n_out*OH*OW][B] and the CSC copy
    of the filter bank (csc_build of the n_out x C*KH*KW CSR)."""
    torch = _torch()
    rows, B, ldy = _mat(dY, "dY")
    OH, OW = g.out_hw
    if rows != n_out * OH * OW:
        raise ValueError("dY must be [n_out*OH*OW][B]")
    if csc.col_ptr.numel() != g.filter_cols + 1:
        raise ValueError("the CSC must have C*KH*KW columns")
    n = csc.row_idx.numel() if nnz is None else int(nnz)
    if dX is None:
        dX = torch.empty((g.in_rows, B), dtype=torch.float32, device=dY.device)
    rx, bx, ldx = _mat(dX, "dX")
    if (rx, bx) != (g.in_rows, B):
        raise ValueError("dX must be [C*H*W][B]")
    _check(lib().csr_conv_bwd_data(g._arr(), n_out, n, _p(csc.col_ptr), _p(csc.row_idx), _p(csc.vals_t),
                                   _p(dY), ldy, B, _p(dX), ldx, _stream(stream)), "csr_conv_bwd_data")
    return dX


def conv_im2col(g: ConvGeom, X, Xcol=None, stream=None):
    """The lowered operand [C*KH*KW][OH*OW*B] of maps X [C*H*W][B]."""
    torch = _torch()
    rows, B, ldx = _mat(X, "X")
    if rows != g.in_rows:
        raise ValueError("X must be [C*H*W][B]")
    OH, OW = g.out_hw
    if Xcol is None:
        Xcol = torch.empty((g.filter_cols, OH * OW * B), dtype=torch.float32, device=X.device)
    rc, cc, ldc = _mat(Xcol, "Xcol")
    if (rc, cc) != (g.filter_cols, OH * OW * B):
        raise ValueError("Xcol must be [C*KH*KW][OH*OW*B]")
    _check(lib().conv_im2col(g._arr(), _p(X), ldx, B, _p(Xcol), ldc, _stream(stream)), "conv_im2col")
    return Xcol


def maxpool_fwd(g: ConvGeom, X, Y=None, stream=None):
    """Max pooling (KH x KW windows, stride SH x SW, no padding) of [C*H*W][B] maps."""
    torch = _torch()
    rows, B, ldx = _mat(X, "X")
    if rows != g.in_rows:
        raise ValueError("X must be [C*H*W][B]")
    OH, OW = g.out_hw
    if Y is None:
        Y = torch.empty((g.C * OH * OW, B), dtype=torch.float32, device=X.device)
    ry, by, ldy = _mat(Y, "Y")
    if (ry, by) != (g.C * OH * OW, B):
        raise ValueError("Y must be [C*OH*OW][B]")
    _check(lib().l1csr_maxpool_fwd(g._arr(), _p(X), ldx, B, _p(Y), ldy, _stream(stream)), "l1csr_maxpool_fwd")
    return Y


def csr_compact(W: CSR, out: CSR | None = None, stream=None) -> CSR:
    """Copy of W without its stored zeros (out of place)."""
    torch = _torch()
    nnz = W.validate_shapes()
    dev = W.row_ptr.device
    if out is None:
        cap = max(nnz, 1)
        out = CSR(W.n_rows, W.n_cols, torch.empty(W.n_rows + 1, dtype=torch.int32, device=dev),
                  torch.empty(cap, dtype=torch.int32, device=dev),
                  torch.empty(cap, dtype=torch.float32, device=dev), None)
    ws, wsb = _workspace(workspace_bytes(OP_COMPACT, W.n_rows, 0, nnz, 0), dev, stream)
    _check(lib().csr_compact(W.n_rows, nnz, _p(W.row_ptr), _p(W.col_idx), _p(W.vals), _p(out.row_ptr),
                             _p(out.col_idx), _p(out.vals), _nnz_dev(out), _p(ws), wsb, _stream(stream)),
           "csr_compact")
    _set_nnz(out, -1, stream)
    return out


def csr_validate(W: CSR, nnz: int | None = None, stream=None) -> bool:
    """Check on the device that W is a canonical CSR (row_ptr[0] = 0,
    non-decreasing, row_ptr[N] = nnz, columns in range and strictly increasing
    in each row).  Waits for the device status and returns True if well formed."""
    torch = _torch()
    _vec(W.row_ptr, torch.int32, "row_ptr")
    _vec(W.col_idx, torch.int32, "col_idx")
    if W.row_ptr.numel() != W.n_rows + 1:
        raise ValueError("row_ptr must hold n_rows + 1 entries")
    n = W.nnz if nnz is None else int(nnz)
    if n is None:
        n = W.host_nnz()
    if n < 0 or n > W.col_idx.numel():
        raise ValueError("nnz must lie within col_idx")
    status = torch.empty(1, dtype=torch.int32, device=W.row_ptr.device)
    _check(lib().csr_validate(W.n_rows, W.n_cols, n, _p(W.row_ptr), _p(W.col_idx), _p(status),
                              _stream(stream)), "csr_validate")
    return int(status.item()) == OK


def relu_fwd(x, y=None, stream=None):
    torch = _torch()
    _dev(x, torch.float32, "x")
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    y = torch.empty_like(x) if y is None else y
    _check(lib().l1csr_relu_fwd(x.numel(), _p(x), _p(y), _stream(stream)), "l1csr_relu_fwd")
    return y


def relu_bwd(x, dy, dx=None, stream=None):
    torch = _torch()
    _dev(x, torch.float32, "x")
    _dev(dy, torch.float32, "dy")
    if not (x.is_contiguous() and dy.is_contiguous()) or x.shape != dy.shape:
        raise ValueError("x and dy must be contiguous and of the same shape")
    dx = torch.empty_like(x) if dx is None else dx
    _check(lib().l1csr_relu_bwd(x.numel(), _p(x), _p(dy), _p(dx), _stream(stream)), "l1csr_relu_bwd")
    return dx


def softmax_xent(logits, labels, dlogits=None, loss=None, stream=None):
    """Mean softmax cross-entropy over batch columns; returns (loss[1], dlogits)."""
    torch = _torch()
    Cn, B, ld = _mat(logits, "logits")
    _vec(labels, torch.int32, "labels")
    if dlogits is None:
        dlogits = torch.empty_like(logits)
    _, _, ldd = _mat(dlogits, "dlogits")
    if ldd != ld:
        raise ValueError("dlogits must share the leading dimension of logits")
    if loss is None:
        loss = torch.empty(1, dtype=torch.float32, device=logits.device)
    ws, wsb = _workspace(workspace_bytes(OP_SOFTMAX_XENT, Cn, 0, 0, B), logits.device, stream)
    _check(lib().l1csr_softmax_xent(Cn, B, _p(logits), ld, _p(labels), _p(dlogits), _p(loss),
                                    _p(ws), wsb, _stream(stream)), "l1csr_softmax_xent")
    return loss, dlogits


def _token_args(logits, labels, weights, dlogits, grad, stream):
    """What the calls over logits[C][B] check alike; returns (C, B, dtype, ld, dlogits, its ld, device index)."""
    Cn, B, ld, code = _typed_mat(logits, "logits")
    torch = _torch_module
    index = _device_of(logits)
    _vec_of(labels, torch.int32, B, index, "labels", "token (B)")
    if weights is not None:
        _vec_of(weights, torch.float32, B, index, "weights", "token (B)")
    ldd = 0
    if grad:
        if dlogits is None:
            dlogits = _new((Cn, B), logits.dtype, logits.device, stream)
        rows, cols, ldd, dcode = _typed_mat(dlogits, "dlogits")
        if rows != Cn or cols != B or dcode != code:
            raise ValueError("dlogits must have the shape and type of logits")
        _same_device(index, dlogits, "dlogits")
        if rows == 1 and dlogits.data_ptr() == logits.data_ptr():
            ldd = ld
    elif dlogits is not None:
        raise ValueError("dlogits given to a call without gradient")
    return Cn, B, code, ld, dlogits, ldd, index


def _result(t, n, logits, index, name, what, stream):
    """A call's float32 output of n values: the caller's, or a new one."""
    if t is None:
        return _new((n,), _torch_module.float32, logits.device, stream)
    return _vec_of(t, _torch_module.float32, n, index, name, what)


def token_logp(logits, labels, logp=None, stream=None):
    """Log-probabilities of the taken tokens: logp[b] = logits[labels[b]][b] - log sum_c exp logits[c][b].

    logits [C][B] float32, bfloat16 or float16 (class-major, tokens contiguous, as softmax_xent's), labels [B] int32;
    a label outside [0, C) gives 0.  Returns logp (float32 [B])."""
    Cn, B, code, ld, _, _, index = _token_args(logits, labels, None, None, False, stream)
    logp = _result(logp, B, logits, index, "logp", "token (B)", stream)
    ws, wsb = _workspace(workspace_bytes(OP_TOKEN_LOSS, Cn, 0, 0, B), logits.device, stream)
    _check(lib().l1csr_token_logp(Cn, B, code, logits.data_ptr(), ld, labels.data_ptr(), logp.data_ptr(), _p(ws), wsb,
                                  _stream(stream)), "l1csr_token_logp")
    return logp


def policy_loss(logits, labels, old_logp, advantages, ref_logp=None, weights=None, clip_low=0.2, clip_high=0.2,
                kl_coef=0.0, dlogits=None, logp=None, stats=None, grad=True, stream=None, *, grad_scale=1.0):
    """Clipped policy loss with a penalty on the distance from a reference, and its gradient.

    With lp the token_logp of logits [C][B], r = exp(lp - old_logp) and the KL estimate
    k = exp(ref_logp - lp) - (ref_logp - lp) - 1 (0 without ref_logp), the loss is the weighted mean over the tokens of
    -min(r adv, clip(r, 1 - clip_low, 1 + clip_high) adv) + kl_coef k.  A token counts if its label lies in [0, C) and its
    weight (weights float32 [B], default 1) is not 0; the logits of the others are not used and their columns of
    dlogits are 0.  dlogits (the type and shape of logits) may be logits itself; grad=False leaves it out.  It receives
    grad_scale times the gradient, scaled ahead of its rounding (an fp16 gradient of a large vocabulary needs that:
    entries under 2^-24 are lost; nothing else is scaled).  No other output may share memory with an input (logp with
    old_logp, say).
    Returns (stats, dlogits, logp): stats[4] = loss, mean policy term, mean k, share of clipped tokens."""
    Cn, B, code, ld, dlogits, ldd, index = _token_args(logits, labels, weights, dlogits, grad, stream)
    f32 = _torch_module.float32
    _vec_of(old_logp, f32, B, index, "old_logp", "token (B)")
    _vec_of(advantages, f32, B, index, "advantages", "token (B)")
    if ref_logp is not None:
        _vec_of(ref_logp, f32, B, index, "ref_logp", "token (B)")
    logp = _result(logp, B, logits, index, "logp", "token (B)", stream)
    stats = _result(stats, 4, logits, index, "stats", "statistic (4)", stream)
    ws, wsb = _workspace(workspace_bytes(OP_TOKEN_LOSS, Cn, 0, 0, B), logits.device, stream)
    _check(lib().l1csr_policy_loss_scaled(Cn, B, code, logits.data_ptr(), ld, labels.data_ptr(), old_logp.data_ptr(),
                                          advantages.data_ptr(), _p(ref_logp), _p(weights), clip_low, clip_high, kl_coef,
                                          grad_scale, _p(dlogits), ldd, logp.data_ptr(), stats.data_ptr(), _p(ws), wsb,
                                          _stream(stream)), "l1csr_policy_loss")
    return stats, dlogits, logp


def preference_loss(logits, labels, seq_ptr, ref_logp=None, weights=None, beta=0.1, label_smoothing=0.0, dlogits=None,
                    rewards=None, loss=None, grad=True, stream=None, *, grad_scale=1.0):
    """Preference loss over pairs of sequences packed along the tokens, and its gradient.

    seq_ptr (int32 [2 pairs + 1], not decreasing, within [0, B]): sequence 2p is the preferred one of pair p, 2p + 1 the
    rejected one.  rewards[s] = beta (sum of weights * token_logp over s - ref_logp[s]) (ref_logp float32 [2 pairs],
    default 0), D = rewards[2p] - rewards[2p + 1], loss = the mean over the pairs of
    -(1 - ls) log sigmoid(D) - ls log sigmoid(-D) with ls = label_smoothing.  Tokens that do not count, dlogits and
    grad_scale as in policy_loss; columns in no sequence get 0.  Returns (loss[1], dlogits, rewards)."""
    Cn, B, code, ld, dlogits, ldd, index = _token_args(logits, labels, weights, dlogits, grad, stream)
    torch = _torch_module
    _vec(seq_ptr, torch.int32, "seq_ptr")
    pairs = seq_ptr.numel() // 2
    if seq_ptr.numel() != 2 * pairs + 1:
        raise ValueError("seq_ptr must hold 2 * pairs + 1 offsets")
    _same_device(index, seq_ptr, "seq_ptr")
    if ref_logp is not None:
        _vec_of(ref_logp, torch.float32, 2 * pairs, index, "ref_logp", "sequence (2 * pairs)")
    rewards = _result(rewards, 2 * pairs, logits, index, "rewards", "sequence (2 * pairs)", stream)
    loss = _result(loss, 1, logits, index, "loss", "call (1)", stream)
    ws, wsb = _workspace(workspace_bytes(OP_TOKEN_LOSS, Cn, pairs, 0, B), logits.device, stream)
    _check(lib().l1csr_preference_loss_scaled(Cn, B, code, logits.data_ptr(), ld, labels.data_ptr(), pairs,
                                              seq_ptr.data_ptr(), _p(ref_logp), _p(weights), beta, label_smoothing,
                                              grad_scale, _p(dlogits), ldd, rewards.data_ptr(), loss.data_ptr(), _p(ws),
                                              wsb, _stream(stream)), "l1csr_preference_loss")
    return loss, dlogits, rewards


@dataclass
class MuonState:
    """Hyper-parameters and momentum of Prox-Muon.  m is a float32 device tensor [N][K] (a leading dimension >= K is
    allowed) that starts at zero; scale multiplies the orthogonalised update (None: sqrt(max(1, N / K))); precision (F32 or
    F16, as in orthogonalize) is that of the update's products where a call does not name its own."""
    m: object
    mu: float = 0.95
    nesterov: bool = True
    steps: int = 5
    eps: float = 1e-7
    scale: float | None = None
    precision: int = F32

    @staticmethod
    def zeros(shape, device, **kw):
        torch = _torch()
        return MuonState(torch.zeros(shape, dtype=torch.float32, device=device), **kw)


def _muon_update(G, O, m, m_out, st, scale, precision, stream, room=0):
    """muon_update of G [N][K] into O; m None: no momentum.  Returns the workspace and its size, at least `room` bytes."""
    N, K, ldg, code = _typed_mat(G, "G")
    index = _device_of(G)
    if O is G:
        ldo = ldg
    else:
        ro, co, ldo, ocode = _typed_mat(O, "the update")
        if ro != N or co != K or ocode != code:
            raise ValueError("the update must have the shape and type of G")
        _same_device(index, O, "the update")
        if N == 1 and O.data_ptr() == G.data_ptr():
            ldo = ldg
    ldm = ldmo = 0
    if m is not None:
        rows, cols, ldm = _mat(_same_device(index, m, "m"), "m")
        if rows != N or cols != K:
            raise ValueError("m must be [n_rows][n_cols]")
        ldmo = ldm
        if m_out is not m:
            rows, cols, ldmo = _mat(_same_device(index, m_out, "m_out"), "m_out")
            if rows != N or cols != K:
                raise ValueError("m_out must be [n_rows][n_cols]")
    if precision is None:
        precision = st.precision
    if precision != F32 and precision != F16:
        raise ValueError("precision must be F32 or F16")
    need = workspace_bytes(OP_MUON if precision == F32 else OP_MUON_F16, N, K, 0, 0)
    ws, wsb = _workspace(max(need, room), G.device, stream)
    _check(lib().muon_update(N, K, code, G.data_ptr(), ldg, _p(m), ldm, _p(m_out), ldmo, st.mu, 1 if st.nesterov else 0,
                             st.steps, st.eps, scale, precision, O.data_ptr(), ldo, _p(ws), wsb, _stream(stream)),
           "muon_update")
    return ws, wsb


def orthogonalize(G, out=None, steps=5, eps=1e-7, scale=1.0, precision=F32, stream=None):
    """scale * NS(G / (|G|_F + eps)): `steps` quintic Newton-Schulz steps (muon_update without momentum).

    G [N][K] float32, bfloat16 or float16; out, of the same shape and type, may be G itself.  precision: F32 (fp32
    accuracy, whatever the type) or, where the caller asks for it, F16: operands rounded to fp16, about 1.5e-3 of the
    norm off, in 2/5 of the time for large matrices (as F32 where min(N, K) <= 128).  A bfloat16 result's own rounding is
    1.7e-3.  Returns out."""
    if out is None:
        N, K, _, _ = _typed_mat(G, "G")
        out = _new((N, K), G.dtype, G.device, stream)
    _muon_update(G, out, None, None, MuonState(None, 0.0, False, steps, eps), scale, precision, stream)
    return out


def _muon_args(W, G, st, eta, lam):
    """What the Prox-Muon calls check before the momentum is stored; returns (N, K, scale)."""
    N, K, _ = _mat(G, "G")
    if not (0 < C.c_float(eta).value < math.inf and 0 <= C.c_float(lam).value < math.inf):
        raise ValueError("eta must be positive, lam not negative, and both finite")
    if N != W.n_rows or K != W.n_cols:
        raise ValueError("G must be [n_rows][n_cols]")
    if st.m is None:
        raise ValueError("Prox-Muon needs the momentum m")
    index = G.get_device()
    for t_, name in ((W.row_ptr, "row_ptr"), (W.col_idx, "col_idx"), (W.vals, "vals")):
        _same_device(index, t_, name)
    scale = st.scale
    if scale is None:
        scale = math.sqrt(N / K) if N > K > 0 else 1.0
    return N, K, scale


def _span(t):
    """Bytes [first, past the last) that a tensor's elements lie in."""
    if not isinstance(t, _torch().Tensor):
        raise TypeError(f"a torch.Tensor is needed (got {type(t).__name__})")
    n = t.numel()
    if n == 0:
        return 0, 0
    p = t.data_ptr()
    if t.is_contiguous():
        return p, p + t.element_size() * n
    return p, p + t.element_size() * (1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride())))


def _apart(written, others, what):
    """Refuses tensors that a call writes (spans) and that share memory with others of the call."""
    for a0, a1 in written:
        for b0, b1 in others:
            if a0 < b1 and b0 < a1:
                raise ValueError(what)


def _muon_writes(W, O, st, m_out=None, row_counts=None):
    """What the Prox-Muon calls check before the momentum is stored: the prox reads W after the update and the momentum are
    written, so neither lies in W's arrays; row_counts lies in none of them."""
    layer = [_span(t) for t in (W.row_ptr, W.col_idx, W.vals)]
    dense = [_span(t) for t in ((O, st.m) if m_out is None else (O, st.m, m_out))]
    _apart(dense, layer, "the update or the momentum shares memory with W")
    if row_counts is not None:
        _apart([_span(row_counts)], layer + dense, "row_counts shares memory with W, the update or the momentum")


def _muon_out(W, out, capacity, index, dense):
    """What prox_muon_recompress checks of its output CSR before the momentum is stored: large enough, and apart from
    W's arrays and the `dense` tensors."""
    torch = _torch_module
    if out.n_rows != W.n_rows or out.n_cols != W.n_cols or out.row_ptr.numel() < W.n_rows + 1:
        raise ValueError("out must have the shape of W")
    if capacity is not None and capacity > min(out.col_idx.numel(), out.vals.numel()):
        raise ValueError("capacity exceeds out's arrays")
    outs = []
    for t, dtype, name in ((out.row_ptr, torch.int32, "out.row_ptr"), (out.col_idx, torch.int32, "out.col_idx"),
                           (out.vals, torch.float32, "out.vals")):
        _vec(_same_device(index, t, name), dtype, name)
        outs.append(_span(t))
    ins = [_span(t) for t in (W.row_ptr, W.col_idx, W.vals, *dense)]
    for i, a in enumerate(outs):
        _apart([a], outs[i + 1:] + ins, "out shares memory with W, the update, the momentum or itself")


def prox_muon_step(W: CSR, G, st: MuonState, eta, lam, Z=None, m_out=None, row_counts=None, precision=None,
                   stream=None):
    """One Prox-Muon step of the l1 phase over all N*K weights: m' = mu m + G, O = scale * NS(G + mu m') (muon_update;
    without nesterov NS(m')), Z = S_{eta*lam}(W - eta O).  Z may be G itself; st.m is updated in place, or m_out receives
    m' and st.m is kept.  Returns Z."""
    N, K, scale = _muon_args(W, G, st, eta, lam)
    W.validate_shapes()
    if row_counts is not None:
        _vec_of(row_counts, _torch_module.int32, N, G.get_device(), "row_counts", "row (n_rows)")
    if Z is None:
        Z = _new((N, K), _torch().float32, G.device, stream)
    _muon_writes(W, Z, st, m_out, row_counts)
    _muon_update(G, Z, st.m, st.m if m_out is None else m_out, st, scale, precision, stream)
    return prox_l1_step(PROX_DENSE, W, Z, eta, lam, Z=Z, row_counts=row_counts, stream=stream)


def prox_muon_recompress(W: CSR, G, st: MuonState, eta, lam, O=None, capacity=None, out: CSR | None = None,
                         precision=None, stream=None):
    """W' = CSR of the Prox-Muon step (the bits of prox_muon_step and csr_recompress), the recompression fused with the
    threshold (prox_l1_recompress).  O (float32 [N][K], may be G itself) receives the update; st.m is updated in
    place, but not by a call that fails, for its capacity, its arguments or want of memory."""
    torch = _torch()
    N, K, scale = _muon_args(W, G, st, eta, lam)
    nnz = W.validate_shapes()
    _muon_writes(W, G if O is None else O, st)
    if out is not None:
        _muon_out(W, out, capacity, G.get_device(), (st.m, G if O is None else O))
    # everything that the call needs is allocated before the update is launched, in the order of the call's stream
    if O is None:
        O = _new((N, K), torch.float32, G.device, stream)
    if out is None:
        cap = N * K if capacity is None else int(capacity)
        out = CSR(N, K, *(_new((n,), dtype, G.device, stream) for n, dtype in
                          ((N + 1, torch.int32), (max(cap, 1), torch.int32), (max(cap, 1), torch.float32))))
    cap = min(out.col_idx.numel(), out.vals.numel()) if capacity is None else int(capacity)
    short = cap < N * K  # the count may not fit: the momentum is stored behind the recompression
    m_new = _new((N, K), torch.float32, G.device, stream) if short else st.m
    ws, wsb = _muon_update(G, O, st.m, m_new, st, scale, precision, stream,
                           room=workspace_bytes(OP_PROX_RECOMPRESS, N, K, nnz, 0))
    _prox_l1_recompress(W, nnz, O, _mat(O, "O")[2], eta, lam, cap, out, ws, wsb, stream)
    if short:
        with torch.cuda.stream(torch.cuda.current_stream(G.device) if stream is None else stream):
            st.m.copy_(m_new)
    return out


# ---------------------------------------------------------------------------
# around the layers of a network on tokens
# ---------------------------------------------------------------------------

def _ld_of(t, rows, cols, dtype, index):
    """The leading dimension of a sound [rows][cols] matrix of `dtype` on device `index`, -1 for any other."""
    if not isinstance(t, _torch_module.Tensor) or t.dtype is not dtype or t.shape != (rows, cols) or t.get_device() != index:
        return -1
    ld, unit = t.stride()
    if rows <= 1:
        ld = max(cols, 1)
    return ld if (unit == 1 or cols <= 1) and ld >= cols else -1


def _out_mat(t, shape, dtypes, index, name, what, device, stream):
    """A call's output matrix, the caller's or a new one of the first type; returns (tensor, ld, l1csr_dtype)."""
    if t is None:
        t = _new(shape, dtypes[0], device, stream)
    for dtype in dtypes:
        ld = _ld_of(t, *shape, dtype, index)
        if ld >= 0:
            return t, ld, _kinds()[dtype]
    rows, cols, ld, code = _typed_mat(t, name)
    if (rows, cols) != tuple(shape) or t.dtype not in dtypes:
        raise ValueError(f"{name} must be {what}")
    _same_device(index, t, name)
    return t, ld, code


def _csr_on(W, index):
    for t_, name in ((W.row_ptr, "row_ptr"), (W.col_idx, "col_idx"), (W.vals, "vals")):
        _same_device(index, t_, name)


def embedding_fwd(E, tokens, X=None, scale=1.0, dtype=None, stream=None):
    """Rows of a table as columns of the activations: X[d][b] = scale * E[tokens[b]][d], 0 where tokens[b] lies outside
    [0, V) (padding).

    E is a table [V][D] (float32, bfloat16 or float16, features contiguous, as a layer's weights) or a CSR (V x D);
    tokens int32 [B]; X [D][B] of the table's type or float32 (dtype: which a new one has; default the table's).  Returns X."""
    torch = _torch()
    _vec(tokens, torch.int32, "tokens")
    index = _device_of(tokens)
    B = tokens.numel()
    if isinstance(E, CSR):
        nnz = E.validate_shapes()
        _csr_on(E, index)
        if dtype is not None and dtype is not torch.float32:
            raise ValueError("a CSR table gives float32")
        X, ldx, _ = _out_mat(X, (E.n_cols, B), (torch.float32,), index, "X", "[D][B] float32", tokens.device, stream)
        _check(lib().l1csr_embedding_csr_fwd(E.n_rows, E.n_cols, nnz, _p(E.row_ptr), _p(E.col_idx), _p(E.vals), B, _p(tokens),
                                             scale, _p(X), ldx, _stream(stream)), "l1csr_embedding_csr_fwd")
        return X
    V, D, lde, code = _typed_mat(E, "E")
    _same_device(index, E, "E")
    dtypes = (E.dtype, torch.float32)
    if dtype is not None:
        if dtype not in dtypes:
            raise ValueError("dtype must be the table's or float32")
        dtypes = (dtype,)
    X, ldx, xcode = _out_mat(X, (D, B), dtypes, index, "X", "[D][B] of the table's type or float32", E.device, stream)
    _check(lib().l1csr_embedding_fwd(V, D, B, code, E.data_ptr(), lde, tokens.data_ptr(), scale, xcode, X.data_ptr(), ldx,
                                     _stream(stream)), "l1csr_embedding_fwd")
    return X


@dataclass
class EmbeddingPlan:
    """The order that an embedding's gradients add up in (embedding_plan): of B tokens of a table of n_rows rows."""
    n_rows: int
    B: int
    buf: object  # device buffer, None for B = 0
    outgrown: list = field(default_factory=list)  # earlier buffers, which graphs may read


def embedding_plan(tokens, n_rows, plan: EmbeddingPlan | None = None, stream=None) -> EmbeddingPlan:
    """The order of the tokens (int32 [B]) of a table of n_rows rows, for embedding_bwd and embedding_masked_bwd.  It depends
    on the tokens alone, so it can be made beside the forward pass and serves every gradient of the batch.  A plan given
    is filled again, in its buffer where that is large enough (graphs captured with that buffer then read the new order:
    one that is to keep its own needs a plan of its own), else in one of at least twice the size; one that it outgrows lives
    as long as the plan, so a graph keeps the one it was captured with."""
    torch = _torch()
    _vec(tokens, torch.int32, "tokens")
    index = _device_of(tokens)
    B, n_rows = tokens.numel(), int(n_rows)
    need = workspace_bytes(OP_EMBEDDING_PLAN, n_rows, 0, 0, B)
    if plan is None:
        plan = EmbeddingPlan(n_rows, B, None)
    buf = old = plan.buf
    if need > 0 and (buf is None or buf.numel() < need or buf.get_device() != index):
        # (twice the size that was too small: what a plan outgrew on a device is together no larger than what it has)
        grown = 0 if old is None or old.get_device() != index else 2 * old.numel()
        buf = _empty_bytes(max(need, grown), tokens.device, stream)
    _check(lib().l1csr_embedding_plan(n_rows, B, tokens.data_ptr(), _p(buf), 0 if buf is None else buf.numel(),
                                      _stream(stream)), "l1csr_embedding_plan")
    if old is not None and buf is not old:
        plan.outgrown.append(old)
    plan.n_rows, plan.B, plan.buf = n_rows, B, buf
    return plan


def _embedding_scratch(tokens, n_rows, D, B, plan, device, index, stream):
    """The plan and the workspace of a gradient's call, (address, bytes) each; a plan that the caller has not is made behind
    the workspace."""
    need = workspace_bytes(OP_EMBEDDING_BWD, n_rows, D, 0, B)
    if plan is not None:
        if plan.n_rows != n_rows or plan.B != B:
            raise ValueError("the plan is of another table or batch")
        if plan.buf is not None:
            _same_device(index, plan.buf, "the plan")
        ws, _ = _workspace(need, device, stream)
        return (None, 0) if plan.buf is None else (plan.buf.data_ptr(), plan.buf.numel()), _p(ws), need, plan.buf, ws
    _vec_of(tokens, _torch_module.int32, B, index, "tokens", "token (B)")
    room = workspace_bytes(OP_EMBEDDING_PLAN, n_rows, 0, 0, B)
    ws, _ = _workspace(need + room, device, stream)
    at = None if ws is None else ws.data_ptr()
    order = (None, 0) if room == 0 else (at + need, room)
    _check(lib().l1csr_embedding_plan(n_rows, B, tokens.data_ptr(), *order, _stream(stream)), "l1csr_embedding_plan")
    return order, at, need, None, ws


def embedding_bwd(dX, tokens, n_rows, dE=None, scale=1.0, add=None, plan: EmbeddingPlan | None = None, stream=None):
    """The table's dense gradient, every row of it: dE[v][d] = add[v][d] + scale * sum of dX[d][b] over tokens[b] = v.

    dX [D][B] float32, bfloat16 or float16; dE [n_rows][D] float32 (a new one is) or of dX's type; add (of dE's shape and
    type, default 0) may be dE itself: then rows without tokens are not touched (a table tied to the output layer:
    add=dE=dense_wgrad(...)).  tokens int32 [B] (not looked at with a plan, and may be None then).  Sums are fp32 in an
    order that the tokens fix.  The dense gradient is what prox_l1_recompress and the other l1 updates take.  Returns dE."""
    torch = _torch()
    D, B, lddx, code = _typed_mat(dX, "dX")
    index, n_rows = _device_of(dX), int(n_rows)
    dE, ldde, ecode = _out_mat(dE, (n_rows, D), (torch.float32, dX.dtype), index, "dE", "[n_rows][D] float32 or of dX's type",
                               dX.device, stream)
    ldadd = 0
    if add is dE:
        ldadd = ldde
    elif add is not None:
        _, ldadd, acode = _out_mat(add, (n_rows, D), (dE.dtype,), index, "add", "of dE's shape and type", dX.device, stream)
        if n_rows == 1 and add.data_ptr() == dE.data_ptr():
            ldadd = ldde
    order, ws, wsb, *_ = held = _embedding_scratch(tokens, n_rows, D, B, plan, dX.device, index, stream)
    _check(lib().l1csr_embedding_bwd(n_rows, D, B, code, dX.data_ptr(), lddx, *order, scale, ecode, _p(add), ldadd,
                                     dE.data_ptr(), ldde, ws, wsb, _stream(stream)), "l1csr_embedding_bwd")
    del held  # (the buffers live until the call has been made)
    return dE


def embedding_masked_bwd(W: CSR, dX, tokens, gv=None, scale=1.0, plan: EmbeddingPlan | None = None, stream=None):
    """The gradient of a table kept in CSR, sampled on its pattern (debiasing, as sddmm_masked_wgrad):
    gv[p] = scale * sum of dX[col p][b] over tokens[b] = row of p.  dX [D][B] float32; tokens, plan as in embedding_bwd.
    Returns gv (float32 [nnz])."""
    torch = _torch()
    D, B, lddx = _mat(dX, "dX")
    index = _device_of(dX)
    nnz = W.validate_shapes()
    _csr_on(W, index)
    if D != W.n_cols:
        raise ValueError("dX must have as many rows as W has columns")
    if gv is None:
        gv = _new((nnz,), torch.float32, dX.device, stream)
    _vec(gv, torch.float32, "gv")
    _same_device(index, gv, "gv")
    if gv.numel() < nnz:
        raise ValueError("gv must hold nnz values")
    order, ws, wsb, *_ = held = _embedding_scratch(tokens, W.n_rows, D, B, plan, dX.device, index, stream)
    _check(lib().l1csr_embedding_masked_bwd(W.n_rows, D, nnz, _p(W.row_ptr), _p(W.col_idx), B, dX.data_ptr(), lddx, *order,
                                            scale, _p(gv), ws, wsb, _stream(stream)), "l1csr_embedding_masked_bwd")
    del held
    return gv


def _norm_like(t, K, B, dtype, index, name):
    """A matrix of a norm call; returns its leading dimension."""
    ld = _ld_of(t, K, B, dtype, index)
    if ld >= 0:
        return ld
    rows, cols, ld, _ = _typed_mat(t, name)
    if rows != K or cols != B or t.dtype is not dtype:
        raise ValueError(f"{name} must have the shape and type of the residual")
    _same_device(index, t, name)
    return ld


def _same_ld(out, ldo, t, ld, K):
    """A single row's leading dimension is its own: that of the matrix it is given over."""
    return ld if t is not None and K == 1 and out.data_ptr() == t.data_ptr() else ldo


def _gate_args(gate, y, K, B, dtype, index):
    """(gate kind, its leading dimension)"""
    if gate is None:
        return GATE_NONE, 0
    if y is None:
        raise ValueError("a gate needs the block's output y")
    if gate.dim() == 1:
        _vec_of(gate, _torch_module.float32, K, index, "gate", "feature (K)")
        return GATE_ROW, 0
    return GATE_FULL, _norm_like(gate, K, B, dtype, index, "gate")


def _gain(t, K, index, name):
    return None if t is None else _vec_of(t, _torch_module.float32, K, index, name, "feature (K)")


def residual_norm_fwd(r, y=None, gate=None, post_gain=None, pre_gain=None, alpha=1.0, eps=1e-6, sigmoid=False, r_out=None,
                      h=None, stream=None):
    """The norms before and after a block with its gate and its residual, per token (column) of activations [K][B]:

        n  = y / sqrt(mean_k y^2 + eps) * post_gain        (y itself without post_gain)
        r' = r + alpha * a(gate) * n
        h  = r' / sqrt(mean_k r'^2 + eps) * pre_gain       (left out without pre_gain)

    r is the residual, y the block's output (None: r' is r, the norm alone), h the next block's input; all [K][B] of one
    type (float32, bfloat16, float16), the gains float32 [K].  gate: None (a = 1), float32 [K] (a gain of the features)
    or [K][B] of r's type; a(g) = g, or with sigmoid the logistic function.  h comes from the unrounded r'.
    r_out and h may each be r or y themselves, but not each other.  Returns (r', h); h is None without pre_gain."""
    K, B, ldr, code = _typed_mat(r, "r")
    index, dtype, torch = _device_of(r), r.dtype, _torch_module
    if y is None and (pre_gain is None or post_gain is not None):
        raise ValueError("without y there is a norm of r alone: pre_gain is needed and post_gain has no meaning")
    ldy = 0 if y is None else _norm_like(y, K, B, dtype, index, "y")
    kind, ldg = _gate_args(gate, y, K, B, dtype, index)
    post_gain, pre_gain = _gain(post_gain, K, index, "post_gain"), _gain(pre_gain, K, index, "pre_gain")
    if (y is None and r_out is not None) or (pre_gain is None and h is not None):
        raise ValueError("r_out needs y, h needs pre_gain")
    ldro = ldh = 0
    if y is not None:
        if r_out is None:
            r_out, ldro = _new((K, B), dtype, r.device, stream), max(B, 1)
        else:
            ldro = _norm_like(r_out, K, B, dtype, index, "r_out")
            ldro = _same_ld(r_out, _same_ld(r_out, ldro, y, ldy, K), r, ldr, K)
    if pre_gain is not None:
        if h is None:
            h, ldh = _new((K, B), dtype, r.device, stream), max(B, 1)
        else:
            ldh = _norm_like(h, K, B, dtype, index, "h")
            ldh = _same_ld(h, _same_ld(h, ldh, y, ldy, K), r, ldr, K)
    ws, wsb = _workspace(workspace_bytes(OP_RESIDUAL_NORM, K, 0, 0, B), r.device, stream)
    _check(lib().l1csr_residual_norm_fwd(K, B, code, r.data_ptr(), ldr, _p(y), ldy, kind, 1 if sigmoid else 0, _p(gate), ldg,
                                         _p(post_gain), _p(pre_gain), alpha, eps, _p(r_out), ldro, _p(h), ldh, _p(ws), wsb,
                                         _stream(stream)), "l1csr_residual_norm_fwd")
    return (r if y is None else r_out), h


@dataclass
class ResidualNormGrads:
    """Gradients of residual_norm_fwd's arguments; None for what was not given."""
    r: object
    y: object
    gate: object
    post_gain: object
    pre_gain: object


def residual_norm_bwd(r_out, dr_out=None, dh=None, y=None, gate=None, post_gain=None, pre_gain=None, alpha=1.0, eps=1e-6,
                      sigmoid=False, dr=None, dy=None, dgate=None, stream=None) -> ResidualNormGrads:
    """The gradients of residual_norm_fwd: r_out is the r' it gave (the residual r itself where it had no y), dr_out the
    gradient of the loss with respect to r' from its further uses (None: none), dh that with respect to h (with
    pre_gain; one of both is needed); y, gate, post_gain, pre_gain, alpha, eps, sigmoid as there.

    The gate's gradient has its shape; it and the gains' are sums over the tokens where one serves all.  dr may be dr_out
    or dh itself, dy y itself and dgate a [K][B] gate itself; without pre_gain the gradient of r is dr_out, and
    none is stored.  Returns ResidualNormGrads."""
    K, B, ldr, code = _typed_mat(r_out, "r_out")
    index, dtype, torch = _device_of(r_out), r_out.dtype, _torch_module
    if y is None and (pre_gain is None or post_gain is not None):
        raise ValueError("without y there is a norm of r alone: pre_gain is needed and post_gain has no meaning")
    if (pre_gain is None) != (dh is None):
        raise ValueError("dh goes with pre_gain")
    if pre_gain is None and dr_out is None:
        raise ValueError("dr_out is needed without pre_gain")
    if (pre_gain is None and dr is not None) or (y is None and dy is not None) or (gate is None and dgate is not None):
        raise ValueError("an output is given for a gradient that this call has not")
    lddro = 0 if dr_out is None else _norm_like(dr_out, K, B, dtype, index, "dr_out")
    lddh = 0 if dh is None else _norm_like(dh, K, B, dtype, index, "dh")
    ldy = 0 if y is None else _norm_like(y, K, B, dtype, index, "y")
    kind, ldg = _gate_args(gate, y, K, B, dtype, index)
    post_gain, pre_gain = _gain(post_gain, K, index, "post_gain"), _gain(pre_gain, K, index, "pre_gain")
    lddr = lddy = lddg = max(B, 1)  # of new ones
    device = r_out.device
    if pre_gain is None:
        dpre = None
    else:
        dpre = _new((K,), torch.float32, device, stream)
        if dr is None:
            dr = _new((K, B), dtype, device, stream)
        else:
            lddr = _same_ld(dr, _same_ld(dr, _norm_like(dr, K, B, dtype, index, "dr"), dr_out, lddro, K), dh, lddh, K)
    if y is not None:
        if dy is None:
            dy = _new((K, B), dtype, device, stream)
        else:
            lddy = _same_ld(dy, _norm_like(dy, K, B, dtype, index, "dy"), y, ldy, K)
    if kind == GATE_ROW:
        if dgate is None:
            dgate = _new((K,), torch.float32, device, stream)
        else:
            _vec_of(dgate, torch.float32, K, index, "dgate", "feature (K)")
    elif kind == GATE_FULL:
        if dgate is None:
            dgate = _new((K, B), dtype, device, stream)
        else:
            lddg = _same_ld(dgate, _norm_like(dgate, K, B, dtype, index, "dgate"), gate, ldg, K)
    dpost = None if post_gain is None else _new((K,), torch.float32, device, stream)
    ws, wsb = _workspace(workspace_bytes(OP_RESIDUAL_NORM, K, 0, 0, B), r_out.device, stream)
    _check(lib().l1csr_residual_norm_bwd(K, B, code, r_out.data_ptr(), ldr, _p(dr_out), lddro, _p(dh), lddh, _p(y), ldy, kind,
                                         1 if sigmoid else 0, _p(gate), ldg, _p(post_gain), _p(pre_gain), alpha, eps, _p(dr),
                                         lddr, _p(dy), lddy, _p(dgate), lddg, _p(dpost), _p(dpre), _p(ws), wsb,
                                         _stream(stream)), "l1csr_residual_norm_bwd")
    return ResidualNormGrads(dr_out if pre_gain is None else dr, dy, dgate, dpost, dpre)


def _flat(t, index, name):
    """(address, rows, columns, leading dimension, l1csr_dtype) of a gradient: a whole buffer is one row."""
    code = _dtype_code(t, name)
    _same_device(index, t, name)
    if t.is_contiguous():
        n = t.numel()
        return t.data_ptr(), 1, n, n, code
    if t.dim() != 2:
        raise ValueError(f"{name} must be contiguous, or 2-D with a contiguous last dimension")
    rows, cols, ld, code = _typed_mat(t, name)
    return t.data_ptr(), rows, cols, ld, code


def _flat_all(tensors, index, name):
    """_flat of every tensor (several hundred of them: the common case without calls)."""
    kinds, tensor = _kinds(), _torch_module.Tensor
    out = []
    for i, t in enumerate(tensors):
        if isinstance(t, tensor) and t.dtype in kinds and t.get_device() == index and t.is_contiguous():
            n = t.numel()
            out.append((t.data_ptr(), 1, n, n, kinds[t.dtype]))
        else:
            out.append(_flat(t, index, f"{name}[{i}]"))
    return out


def _grad_args(grads):
    """The tensors of a norm call, flat; returns (n, flat, first tensor's device index)."""
    if not grads:
        raise ValueError("no gradients are given")
    _dtype_code(grads[0], "grads[0]")
    index = _device_of(grads[0])
    return len(grads), _flat_all(grads, index, "grads"), index


class _Columns:
    """Flat tensors as the C arrays of their addresses, rows, columns, leading dimensions and types."""

    def __init__(self, flat):
        p, rows, cols, ld, code = zip(*flat)
        n = len(p)
        self.words, self.codes = array("q", (*p, *rows, *cols, *ld)), array("i", code)
        at = self.words.buffer_info()[0]
        self.p, self.rows, self.cols, self.ld, self.code = at, at + 8 * n, at + 16 * n, at + 24 * n, self.codes.buffer_info()[0]


def grad_norm(grads, grad_scale=1.0, stats=None, stream=None):
    """The norm of many gradients together, sqrt(sum of all squares) / grad_scale (grad_scale: a factor that they hold, as
    the losses' grad_scale).  grads: a sequence of tensors (float32, bfloat16, float16; contiguous of any shape, or
    [N][K] with a leading dimension).  Returns stats (float32 [2], on the device): the norm and 1 / grad_scale."""
    grads = list(grads)
    n, flat, index = _grad_args(grads)
    torch = _torch_module
    stats = _result(stats, 2, grads[0], index, "stats", "statistic (2)", stream)
    ws, wsb = _workspace(workspace_bytes(OP_GRAD_NORM, n, 0, 0, 0), grads[0].device, stream)
    g = _Columns(flat)
    _check(lib().l1csr_grad_norm(n, g.p, g.rows, g.cols, g.ld, g.code, grad_scale, stats.data_ptr(), _p(ws), wsb,
                                 _stream(stream)), "l1csr_grad_norm")
    return stats


def clip_grad_norm(grads, max_norm, grad_scale=1.0, eps=1e-6, out=None, zero_nonfinite=False, stats=None, stream=None):
    """Clips many gradients to a norm that they have together, in place or into `out`:

        norm = sqrt(sum of all squares) / grad_scale,  f = min(1, max_norm / (norm + eps)) / grad_scale,  out = f * g

    grads and grad_scale as in grad_norm: a factor that they hold is taken out.  out: a sequence of tensors of the same
    shapes, each of its gradient's type or float32 (what the solvers take).  A norm that is not finite gives what the
    formula gives; with zero_nonfinite f = 0 and every result 0, so that nothing of the step reaches a
    momentum.  No tensor may be given twice.  Nothing waits: stats (float32 [2], on the device) = the norm and f."""
    grads = list(grads)
    n, flat, index = _grad_args(grads)
    torch = _torch_module
    targets, o = (None, None, None), None
    if out is not None:
        out = list(out)
        if len(out) != n:
            raise ValueError("out must hold one tensor per gradient")
        flat_out = _flat_all(out, index, "out")
        for i, (g, o, f) in enumerate(zip(grads, out, flat_out)):
            if o.shape != g.shape or (o.dtype is not g.dtype and o.dtype is not torch.float32):
                raise ValueError(f"out[{i}] must have the shape of grads[{i}] and its type or float32")
            if f[1] != flat[i][1]:  # one of both is whole, the other has rows: both by rows
                rows, cols = g.shape
                flat[i] = (flat[i][0], rows, cols, flat[i][3] if flat[i][1] == rows else cols, flat[i][4])
                flat_out[i] = (f[0], rows, cols, f[3] if f[1] == rows else cols, f[4])
        o = _Columns(flat_out)
        targets = (o.p, o.ld, o.code)
    g = _Columns(flat)
    stats = _result(stats, 2, grads[0], index, "stats", "statistic (2)", stream)
    ws, wsb = _workspace(workspace_bytes(OP_GRAD_NORM, n, 0, 0, 0), grads[0].device, stream)
    _check(lib().l1csr_clip_grad_norm(n, g.p, g.rows, g.cols, g.ld, g.code, *targets, max_norm, grad_scale, eps, 1 if zero_nonfinite else 0,
                                      stats.data_ptr(), _p(ws), wsb, _stream(stream)), "l1csr_clip_grad_norm")
    return stats


# the two-stream l1 step over the entry points above
from .step import l1_step, side_stream  # noqa: E402
