"""ctypes binding of libw2v (include/w2v.h): argument marshalling only.

Every function takes torch tensors that already live where the C ABI expects
them (device tensors on the current HIP device for GPU entry points), checks
dtypes and shapes, and passes raw pointers plus the current torch stream.
No arithmetic of the method happens here. If libw2v.so has not been built the
first call raises: there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libw2v.so")

_vp = ctypes.c_void_p
_i32 = ctypes.c_int32
_i64 = ctypes.c_int64
_f32 = ctypes.c_float
_f64 = ctypes.c_double
_u64 = ctypes.c_uint64

_lib = None

OK = 0
EINVAL = -1
EHIP = -2
ENOMEM = -3
EUNSUPPORTED = -4
EDEVICE_FLAG = -5
ENONFINITE = -6


class _BeamState(ctypes.Structure):
    """w2v_beam_state."""
    _fields_ = [("src", _vp), ("src_stride", _i64), ("dst", _vp), ("dst_stride", _i64),
                ("row_bytes", _i64)]


class W2VError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libw2v error {code}: {msg}")
        self.code = code


def lib():
    """The loaded libw2v.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
            "(hipcc, gfx950) before using the GPU path")
    L = ctypes.CDLL(LIB_PATH)
    L.w2v_version.restype = ctypes.c_int
    L.w2v_last_error.restype = ctypes.c_char_p
    L.w2v_init.argtypes = []
    L.w2v_init.restype = ctypes.c_int
    L.w2v_device_status.argtypes = [_vp]
    L.w2v_device_status.restype = ctypes.c_int
    L.w2v_check_loss.argtypes = [_vp, _i32, _vp]
    L.w2v_check_loss.restype = ctypes.c_int
    L.w2v_build_tables.argtypes = [_vp, _i32, _f64, _f64, _vp, _i64, _vp]
    L.w2v_build_tables.restype = ctypes.c_int
    L.w2v_train_epoch.argtypes = [
        _vp, _i64, _i64, _i64, _i32, _vp, _vp, _i32, _i32, _i32, _i32, _i32,
        _vp, _i64, _vp, _f32, _f32, _i32, _i32, _u64, _vp, _i32, _vp, _i32, _i32,
        _i32, _vp, ctypes.c_size_t, _i32, _i32, _vp]
    L.w2v_train_epoch.restype = ctypes.c_int
    L.w2v_train_epoch_noalloc.argtypes = (L.w2v_train_epoch.argtypes[:26] +
                                          L.w2v_train_epoch.argtypes[28:])
    L.w2v_train_epoch_noalloc.restype = ctypes.c_int
    L.w2v_build_vocab_workspace_bytes.argtypes = [_i32, _i64]
    L.w2v_build_vocab_workspace_bytes.restype = ctypes.c_size_t
    L.w2v_build_vocab.argtypes = [_vp, _i64, _i32, _i64, _vp, _vp, _vp, _vp, _vp,
                                  ctypes.c_size_t, _vp]
    L.w2v_build_vocab.restype = ctypes.c_int
    L.w2v_train_epoch_workspace_bytes.argtypes = [_i32, _i32]
    L.w2v_train_epoch_workspace_bytes.restype = ctypes.c_size_t
    L.w2v_debug_minibatches.argtypes = [
        _vp, _i64, _i64, _i64, _i32, _i32, _i32, _i32, _vp, _i64, _vp, _f32,
        _f32, _i32, _i32, _u64, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
    L.w2v_debug_minibatches.restype = ctypes.c_int
    L.w2v_hot_rows.argtypes = [_vp, _i32, _f64, _f64, _i32, _i32, _i64, _f64]
    L.w2v_hot_rows.restype = ctypes.c_int32
    L.w2v_default_inflight.argtypes = [_i32, _i32, _i32, _i32, _i32]
    L.w2v_default_inflight.restype = ctypes.c_int64
    L.w2v_pending_slots.argtypes = [_i32, _i32, _i32]
    L.w2v_pending_slots.restype = ctypes.c_int32
    L.w2v_step_batch_workspace_bytes.argtypes = [_i32, _i32]
    L.w2v_step_batch_workspace_bytes.restype = ctypes.c_size_t
    L.w2v_step_batch.argtypes = [
        _i32, _i32, _i32, _vp, _vp, _vp, _vp, _f32, _vp, _vp, _i32, _i32, _i32,
        _vp, ctypes.c_size_t, _vp, _vp]
    L.w2v_step_batch.restype = ctypes.c_int
    L.w2v_debug_step_route.argtypes = [_i32, _i32, _i32, _vp, _vp, _i32, _i32, _i32]
    L.w2v_debug_step_route.restype = ctypes.c_int32
    L.w2v_step_batch_sorted_workspace_bytes.argtypes = [_i32, _i32, _i32, _i32, _i32]
    L.w2v_step_batch_sorted_workspace_bytes.restype = ctypes.c_size_t
    L.w2v_step_batch_sorted.argtypes = L.w2v_step_batch.argtypes
    L.w2v_step_batch_sorted.restype = ctypes.c_int
    L.w2v_linear_workspace_bytes.argtypes = [_i32, _i32, _i32, _i32]
    L.w2v_linear_workspace_bytes.restype = ctypes.c_size_t
    L.w2v_linear.argtypes = [
        _vp, _i64, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _i64, _i32, _i32, _i32,
        _i32, _i32, _i32, _vp, ctypes.c_size_t, _vp]
    L.w2v_linear.restype = ctypes.c_int
    L.w2v_linear_backward_workspace_bytes.argtypes = [_i32, _i32, _i32, _i32, _i32]
    L.w2v_linear_backward_workspace_bytes.restype = ctypes.c_size_t
    L.w2v_linear_backward.argtypes = [
        _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i32, _i32,
        _i32, _i32, _i32, _vp, ctypes.c_size_t, _vp]
    L.w2v_linear_backward.restype = ctypes.c_int
    L.w2v_distill_workspace_bytes.argtypes = [_i32, _i32, _i32]
    L.w2v_distill_workspace_bytes.restype = ctypes.c_size_t
    L.w2v_distill_loss.argtypes = [
        _vp, _i64, _i32, _i32, _i32, _vp, _vp, _i32, _i32, _vp, _f32, _f32, _f32, _vp, _vp,
        _vp, _vp, _i64, _vp, ctypes.c_size_t, _vp]
    L.w2v_distill_loss.restype = ctypes.c_int
    L.w2v_distill_backward.argtypes = [
        _vp, _vp, _i64, _i32, _i32, _i32, _vp, _vp, _i32, _i32, _vp, _f32, _f32, _f32, _vp,
        _vp, _i64, _vp]
    L.w2v_distill_backward.restype = ctypes.c_int
    L.w2v_sample_workspace_bytes.argtypes = [_i32, _i32]
    L.w2v_sample_workspace_bytes.restype = ctypes.c_size_t
    L.w2v_sample_words.argtypes = [
        _vp, _i64, _vp, _i64, _i32, _i32, _i32, _vp, _f32, _vp, _i32, _vp, _f32, _vp, _f32,
        _vp, _vp, _vp, ctypes.c_size_t, _vp]
    L.w2v_sample_words.restype = ctypes.c_int
    L.w2v_embed.argtypes = [_vp, _i32, _vp, _i64, _i32, _i32, _i32, _f32, _vp, _i64, _i32, _vp]
    L.w2v_embed.restype = ctypes.c_int
    L.w2v_embed_backward_workspace_bytes.argtypes = [_i32, _i32, _i32]
    L.w2v_embed_backward_workspace_bytes.restype = ctypes.c_size_t
    L.w2v_embed_backward.argtypes = [
        _vp, _i64, _vp, _i32, _i32, _f32, _vp, _i64, _i32, _i32, _i32, _i32, _vp,
        ctypes.c_size_t, _vp]
    L.w2v_embed_backward.restype = ctypes.c_int
    L.w2v_dropout.argtypes = [
        _vp, _i64, _vp, _i64, _vp, _i64, _i32, _i32, _i32, _f64, _u64, _u64, _vp, _vp]
    L.w2v_dropout.restype = ctypes.c_int
    L.w2v_q4_packed_bytes.argtypes = [_i32, _i32, _i32]
    L.w2v_q4_packed_bytes.restype = ctypes.c_size_t
    L.w2v_q4_scale_count.argtypes = [_i32, _i32, _i32]
    L.w2v_q4_scale_count.restype = ctypes.c_size_t
    L.w2v_quantize_q4.argtypes = [_vp, _i64, _i32, _i32, _i32, _i32, _vp, _vp, _vp]
    L.w2v_quantize_q4.restype = ctypes.c_int
    L.w2v_linear_q4.argtypes = [
        _vp, _i64, _vp, _vp, _vp, _vp, _i64, _i32, _i32, _i32, _i32, _i32, _i32, _vp]
    L.w2v_linear_q4.restype = ctypes.c_int
    L.w2v_beam_step_workspace_bytes.argtypes = [_i32, _i32, _i32, _i32, _i32]
    L.w2v_beam_step_workspace_bytes.restype = ctypes.c_size_t
    L.w2v_beam_step.argtypes = [
        _vp, _i64, _i32, _i32, _i32, _i32, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp,
        ctypes.c_size_t, _vp]
    L.w2v_beam_step.restype = ctypes.c_int
    L.w2v_beam_reorder.argtypes = [ctypes.POINTER(_BeamState), _i32, _vp, _i32, _i32, _i32, _vp]
    L.w2v_beam_reorder.restype = ctypes.c_int
    _lib = L
    return L


def _check(rc: int):
    if rc != OK:
        raise W2VError(rc, lib().w2v_last_error().decode())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    return t.data_ptr()


def _stream(stream=None) -> int:
    import torch
    if stream is not None:
        return stream.cuda_stream
    # the current stream's handle without the Stream object around it, which
    # takes 2.5 us to make
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _dev(t, dtype, name, ndim=None):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if isinstance(dtype, tuple):
        if t.dtype not in dtype:
            raise TypeError(f"{name} must have dtype in {dtype}, got {t.dtype}")
    elif t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must be {ndim}-D")
    # The kernels index every argument but the two matrices as packed arrays
    # (contexts[b N + i], loss[2 b], ...): a strided view would be read at
    # the wrong places, so only contiguous tensors pass.
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _matrix(M, name):
    """Checks a V x D fp32 device matrix; rows may be padded (the row stride
    is passed to the library as ld), columns must be adjacent."""
    import torch
    if not isinstance(M, torch.Tensor) or not M.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if M.dtype != torch.float32:
        raise TypeError(f"{name} must have dtype torch.float32, got {M.dtype}")
    if M.dim() != 2:
        raise ValueError(f"{name} must be 2-D")
    if M.stride(1) != 1 or M.stride(0) < M.shape[1]:
        raise ValueError(f"{name} must have unit column stride and a row stride >= D")
    return M.shape[0], M.stride(0)


def version() -> int:
    return int(lib().w2v_version())


def build_tables(counts, neg_power: float = 0.75, sample_t: float = 1e-4,
                 table_size: int = 10**8, want_table: bool = True,
                 want_thresh: bool = True):
    """Host tables: (neg_table int32[table_size], keep_thresh uint32[V])."""
    counts = np.ascontiguousarray(counts, dtype=np.int64)
    V = counts.shape[0]
    table = np.empty(table_size, dtype=np.int32) if want_table else None
    thr = np.empty(V, dtype=np.uint32) if want_thresh else None
    _check(lib().w2v_build_tables(
        counts.ctypes.data, V, float(neg_power), float(sample_t),
        None if table is None else table.ctypes.data, int(table_size),
        None if thr is None else thr.ctypes.data))
    return table, thr


def hot_rows(counts, *, neg_power: float = 0.75, sample_t: float = 1e-4,
             window: int = 5, K: int = 5, inflight: int, tol: float = 0.05) -> int:
    """Leading ids to update atomically (see w2v_hot_rows). The default
    tolerance keeps the expected share of overwritten updates of a plain row
    near 5% (1 - exp(-tol))."""
    counts = np.ascontiguousarray(counts, dtype=np.int64)
    h = int(lib().w2v_hot_rows(counts.ctypes.data, counts.shape[0],
                                float(neg_power), float(sample_t), window, K,
                                int(inflight), float(tol)))
    if h < 0:
        _check(h)
    return h


def init():
    """Sets up the library's state on the current device (w2v_init)."""
    _check(lib().w2v_init())


def device_status(stream=None):
    """Waits for the stream, then raises W2VError (code EDEVICE_FLAG) if a
    kernel of the library skipped work for an id outside [0, V), a row of
    scores for an id, a label or a setting out of range, or a row for a word or
    a parent out of range, since this was last reported (w2v_device_status)."""
    _check(lib().w2v_device_status(_stream(stream)))


def check_loss(loss_buckets, stream=None):
    """Waits for the stream, then raises W2VError (code ENONFINITE) naming the
    first loss bucket whose sum or count is NaN or Inf (w2v_check_loss)."""
    import torch
    _dev(loss_buckets, torch.float64, "loss_buckets", 2)
    _check(lib().w2v_check_loss(_ptr(loss_buckets), loss_buckets.shape[0],
                                _stream(stream)))


def default_inflight(D: int, window: int = 5, K: int = 5, *, V: int,
                     group: int = 1) -> int:
    """Concurrent sentences of train_epoch with max_inflight = 0 over a
    vocabulary of V words (w2v_default_inflight)."""
    n = int(lib().w2v_default_inflight(V, D, window, K, group))
    if n < 0:
        _check(n)
    return n


def pending_slots(D: int, window: int = 5, K: int = 5) -> int:
    """LDS slots per wavefront in which HogBatch training collects pending
    updates of cold input rows (0: none)."""
    n = int(lib().w2v_pending_slots(D, window, K))
    if n < 0:
        _check(n)
    return n


ALGORITHMS = {"hogbatch": 0, "pairwise": 1, "hogbatch_immediate": 2}


def train_epoch(corpus, M_in, M_out, neg_table, keep_thresh=None, *,
                window: int = 5, K: int = 5, D: Optional[int] = None,
                alpha0: float = 0.025, min_alpha_frac: float = 1e-4,
                epoch: int = 0, n_epochs: int = 1, seed: int = 0,
                pos_begin: int = 0, pos_end: Optional[int] = None,
                sentence_len: int = 1000, loss_buckets=None, stats=None,
                max_inflight: int = 0, hot_rows: Optional[int] = None,
                split_rows: int = 0, workspace=None, algorithm: str = "hogbatch",
                group: int = 1, stream=None):
    """Hogwild HogBatch epoch over corpus[pos_begin:pos_end], in place.

    hot_rows: ids below it are updated with atomic adds, the others with
    plain read-modify-write stores; None makes every update atomic.
    split_rows: ids below it are updated through per-XCD partial rows that
    every read sums (see w2v_train_epoch); workspace (a device byte tensor of
    train_epoch_workspace_bytes(split_rows, ld)) is allocated when None.
    algorithm: "hogbatch" (Sec. 1.1; cold input rows collect their updates
        in LDS while their word is in the window, see w2v_train_epoch),
        "hogbatch_immediate" (every update applied at the end of its
        minibatch) or "pairwise" (Alg. 1, the baseline).
    group: consecutive targets sharing one draw of negatives (1: HogBatch as
    in the paper; 2, 4, 8: the sharing widened across targets)."""
    import torch
    _dev(corpus, torch.int32, "corpus", 1)
    V, ld = _matrix(M_in, "M_in")
    V2, ld2 = _matrix(M_out, "M_out")
    if (V, ld) != (V2, ld2):
        raise ValueError("M_in and M_out must have the same shape and stride")
    D = M_in.shape[1] if D is None else D
    _dev(neg_table, torch.int32, "neg_table", 1)
    if keep_thresh is not None:
        _dev(keep_thresh, (torch.int32, torch.uint32), "keep_thresh", 1)
        if keep_thresh.numel() != V:
            raise ValueError("keep_thresh must have V entries")
    n_b = 0
    if loss_buckets is not None:
        _dev(loss_buckets, torch.float64, "loss_buckets", 2)
        n_b = loss_buckets.shape[0]
    if stats is not None:
        _dev(stats, torch.int64, "stats", 1)
        if stats.numel() < 5:
            raise ValueError("stats must have 5 entries (see w2v_train_epoch)")
    T = corpus.numel()
    end = T if pos_end is None else pos_end
    need = train_epoch_workspace_bytes(split_rows, ld)
    if need and workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=M_in.device)
    ws_bytes = 0
    if workspace is not None:
        _dev(workspace, torch.uint8, "workspace", 1)
        ws_bytes = workspace.numel()
    _check(lib().w2v_train_epoch(
        _ptr(corpus), T, pos_begin, end, sentence_len, _ptr(M_in), _ptr(M_out),
        V, D, ld, window, K, _ptr(neg_table), neg_table.numel(),
        _ptr(keep_thresh), alpha0, min_alpha_frac, epoch, n_epochs, seed,
        _ptr(loss_buckets), n_b, _ptr(stats), max_inflight,
        V if hot_rows is None else int(hot_rows), int(split_rows),
        _ptr(workspace), ws_bytes, ALGORITHMS[algorithm], int(group),
        _stream(stream)))


NOALLOC_SCRATCH_BYTES = 4194304


def train_epoch_noalloc(corpus, M_in, M_out, neg_table, keep_thresh=None, *,
                        window: int = 5, K: int = 5, D: Optional[int] = None,
                        alpha0: float = 0.025, min_alpha_frac: float = 1e-4,
                        epoch: int = 0, n_epochs: int = 1, seed: int = 0,
                        pos_begin: int = 0, pos_end: Optional[int] = None,
                        sentence_len: int = 1000, loss_buckets=None, stats=None,
                        max_inflight: int = 0, hot_rows: Optional[int] = None,
                        split_rows: int = 0, algorithm: str = "hogbatch",
                        group: int = 1, stream=None):
    """train_epoch through w2v_train_epoch_noalloc: the split rows' partial
    rows live in the library's static device scratch array, so nothing is
    allocated here or in the library. init() must have run on the device."""
    import torch
    _dev(corpus, torch.int32, "corpus", 1)
    V, ld = _matrix(M_in, "M_in")
    if _matrix(M_out, "M_out") != (V, ld):
        raise ValueError("M_in and M_out must have the same shape and stride")
    D = M_in.shape[1] if D is None else D
    _dev(neg_table, torch.int32, "neg_table", 1)
    if keep_thresh is not None:
        _dev(keep_thresh, (torch.int32, torch.uint32), "keep_thresh", 1)
        if keep_thresh.numel() != V:
            raise ValueError("keep_thresh must have V entries")
    n_b = 0
    if loss_buckets is not None:
        _dev(loss_buckets, torch.float64, "loss_buckets", 2)
        n_b = loss_buckets.shape[0]
    if stats is not None:
        _dev(stats, torch.int64, "stats", 1)
        if stats.numel() < 5:
            raise ValueError("stats must have 5 entries (see w2v_train_epoch)")
    T = corpus.numel()
    end = T if pos_end is None else pos_end
    _check(lib().w2v_train_epoch_noalloc(
        _ptr(corpus), T, pos_begin, end, sentence_len, _ptr(M_in), _ptr(M_out),
        V, D, ld, window, K, _ptr(neg_table), neg_table.numel(),
        _ptr(keep_thresh), alpha0, min_alpha_frac, epoch, n_epochs, seed,
        _ptr(loss_buckets), n_b, _ptr(stats), max_inflight,
        V if hot_rows is None else int(hot_rows), int(split_rows),
        ALGORITHMS[algorithm], int(group), _stream(stream)))


def padded_ld(D: int) -> int:
    """Row stride (floats) that starts every row on a 128-byte line: D
    rounded up to a multiple of 32."""
    return (D + 31) // 32 * 32


def alloc_matrix(V: int, D: int, device="cuda", init=None):
    """A (V, D) fp32 view of a zeroed (V, padded_ld(D)) device buffer,
    optionally filled from `init` (array-like of shape (V, D)). Line-aligned
    rows cost fewer partial-line reads and writes than a packed (V, D)
    matrix when rows are gathered and scattered at random."""
    import torch
    buf = torch.zeros((V, padded_ld(D)), dtype=torch.float32, device=device)
    M = buf[:, :D]
    if init is not None:
        M.copy_(torch.as_tensor(init))
    return M


def train_epoch_workspace_bytes(split_rows: int, ld: int) -> int:
    return int(lib().w2v_train_epoch_workspace_bytes(split_rows, ld))


def debug_minibatches(corpus, neg_table, keep_thresh=None, *, V: int,
                      window: int = 5, K: int = 5, alpha0: float = 0.025,
                      min_alpha_frac: float = 1e-4, epoch: int = 0,
                      n_epochs: int = 1, seed: int = 0, pos_begin: int = 0,
                      pos_end: Optional[int] = None, sentence_len: int = 1000,
                      stats=None, stream=None):
    """Minibatches the epoch would form, indexed by raw position (GPU)."""
    import torch
    _dev(corpus, torch.int32, "corpus", 1)
    _dev(neg_table, torch.int32, "neg_table", 1)
    if keep_thresh is not None:
        _dev(keep_thresh, (torch.int32, torch.uint32), "keep_thresh", 1)
    if stats is not None:
        _dev(stats, torch.int64, "stats", 1)
        if stats.numel() < 5:
            raise ValueError("stats must have 5 entries (see w2v_train_epoch)")
    T = corpus.numel()
    end = T if pos_end is None else pos_end
    P = end - pos_begin
    dev = corpus.device
    out = dict(
        targets=torch.empty(P, dtype=torch.int32, device=dev),
        ctx=torch.empty((P, 2 * window), dtype=torch.int32, device=dev),
        negs=torch.empty((P, K), dtype=torch.int32, device=dev),
        mask=torch.empty((P, K), dtype=torch.uint8, device=dev),
        alpha=torch.empty(P, dtype=torch.float32, device=dev))
    _check(lib().w2v_debug_minibatches(
        _ptr(corpus), T, pos_begin, end, sentence_len, V, window, K,
        _ptr(neg_table), neg_table.numel(), _ptr(keep_thresh), alpha0,
        min_alpha_frac, epoch, n_epochs, seed, _ptr(out["targets"]),
        _ptr(out["ctx"]), _ptr(out["negs"]), _ptr(out["mask"]),
        _ptr(out["alpha"]), _ptr(stats), _stream(stream)))
    return out


def step_batch_workspace_bytes(V: int, ld: int) -> int:
    return int(lib().w2v_step_batch_workspace_bytes(V, ld))


def alloc_workspace(V: int, ld: int, device="cuda"):
    """A torch-owned byte buffer large enough for step_batch."""
    import torch
    n = step_batch_workspace_bytes(V, ld)
    return torch.empty(n, dtype=torch.uint8, device=device)


STEP_ROUTES = {0: "atomic", 1: "staged", 2: "pulled"}


def debug_step_route(B: int, N: int, K: int, V: int, D: int, ld: int, *,
                     in_ptr: int = 1 << 30, out_ptr: int = 1 << 45) -> str:
    """Route of step_batch (not sorted) for these sizes and the matrices'
    addresses, which are compared and not read (w2v_debug_step_route)."""
    r = int(lib().w2v_debug_step_route(B, N, K, in_ptr, out_ptr, V, D, ld))
    if r < 0:
        _check(r)
    return STEP_ROUTES[r]


def step_batch_sorted_workspace_bytes(B: int, N: int, K: int, V: int, ld: int) -> int:
    return int(lib().w2v_step_batch_sorted_workspace_bytes(B, N, K, V, ld))


def step_batch(targets, contexts, negatives, M_in, M_out, alpha=0.025, *,
               D: Optional[int] = None, workspace=None, stats=None,
               stream=None, sorted: bool = False):
    """One snapshot batch of B minibatches; updates M_in, M_out in place.
    sorted: sum each row's updates in a fixed order (w2v_step_batch_sorted:
    the same bits on every run) instead of by the way that is the fastest for
    the sizes, which may be fp64 atomics in arrival order."""
    import torch
    _dev(targets, torch.int32, "targets", 1)
    _dev(contexts, torch.int32, "contexts", 2)
    _dev(negatives, torch.int32, "negatives", 2)
    B = targets.shape[0]
    N = contexts.shape[1]
    K = negatives.shape[1]
    if contexts.shape[0] != B or negatives.shape[0] != B:
        raise ValueError("targets, contexts and negatives disagree on B")
    V, ld = _matrix(M_in, "M_in")
    if _matrix(M_out, "M_out") != (V, ld):
        raise ValueError("M_in and M_out must have the same shape and stride")
    D = M_in.shape[1] if D is None else D
    if isinstance(alpha, torch.Tensor):
        _dev(alpha, torch.float32, "alpha", 1)
        a_ptr, a_s = _ptr(alpha), 0.0
    else:
        a_ptr, a_s = None, float(alpha)
    if workspace is None:
        if sorted:
            n = step_batch_sorted_workspace_bytes(B, N, K, V, ld)
            if n == 0:
                raise W2VError(EINVAL if min(B, N, K) < 0 else EHIP,
                               "no workspace size for this batch (invalid shape "
                               "or failed sort size query)")
            workspace = torch.empty(n, dtype=torch.uint8, device=M_in.device)
        else:
            workspace = alloc_workspace(V, ld, M_in.device)
    if stats is not None:
        _dev(stats, torch.int64, "stats", 1)
        if stats.numel() < 5:
            raise ValueError("stats must have 5 entries (see w2v_train_epoch)")
    entry = lib().w2v_step_batch_sorted if sorted else lib().w2v_step_batch
    _check(entry(
        B, N, K, _ptr(targets), _ptr(contexts), _ptr(negatives), a_ptr, a_s,
        _ptr(M_in), _ptr(M_out), V, D, ld, _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(stats),
        _stream(stream)))
    return workspace


def build_vocab(raw, V_raw: int, min_count: int = 0, remap: bool = True,
                stream=None):
    """Counts, frequency ranks and min-count cut of a raw id stream on the GPU
    (w2v_build_vocab). Returns a dict of device tensors: ranked_counts
    int64[V_raw], rank_of int32[V_raw], corpus int32[T] (or None) and V (an
    int: this reads one value back from the device)."""
    import torch
    _dev(raw, torch.int32, "raw", 1)
    dev = raw.device
    T = raw.numel()
    ranked = torch.empty(V_raw, dtype=torch.int64, device=dev)
    rank_of = torch.empty(V_raw, dtype=torch.int32, device=dev)
    v_kept = torch.empty(1, dtype=torch.int32, device=dev)
    corpus = torch.empty(T, dtype=torch.int32, device=dev) if remap else None
    ws = torch.empty(int(lib().w2v_build_vocab_workspace_bytes(V_raw, T)),
                     dtype=torch.uint8, device=dev)
    _check(lib().w2v_build_vocab(_ptr(raw), T, V_raw, int(min_count), _ptr(ranked),
                                 _ptr(rank_of), _ptr(v_kept), _ptr(corpus), _ptr(ws),
                                 ws.numel(), _stream(stream)))
    return dict(ranked_counts=ranked, rank_of=rank_of, corpus=corpus,
                V=int(v_kept.item()))


# ------------------------------------------------------ the vocabulary head --

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3, "tanh": 4, "sigmoid": 5}


_DTYPES = None


def _dtypes():
    global _DTYPES
    if _DTYPES is None:
        import torch
        _DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    return _DTYPES


def _head_dtype(t, name):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    code = _dtypes().get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must have dtype float32, bfloat16 or float16, got {t.dtype}")
    return code


# Sizes are 32-bit numbers of the library's; ctypes would pass on the lower bits of others.
_MOST = 0x7FFFFFFF


def _operand(t, name, shape=None, dtype=None):
    """Row stride of a 2-D GPU matrix whose columns are adjacent."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    size = t.shape
    if len(size) != 2:
        raise ValueError(f"{name} must be 2-D")
    if shape is not None and size != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(size)}")
    _here(t, name)
    rows, cols = size
    if rows > _MOST or cols > _MOST:
        raise ValueError(f"{name} must have less than 2^31 rows and columns")
    ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError(f"{name} must have unit column stride")
    if rows <= 1:
        return max(cols, 1)
    if ld < cols:
        raise ValueError(f"{name} must have a row stride >= its columns")
    return ld


def _here(t, name):
    import torch
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{name} must be on the current device")


def _vector(t, dtype, name, n):
    _dev(t, dtype, name, 1)
    _here(t, name)
    if t.numel() != n:
        raise ValueError(f"{name} must have {n} entries")
    return t


def _allocations(stream):
    """Makes the call's stream current, so that what the binding allocates
    belongs to it and is not handed out again before its work is done."""
    import contextlib

    import torch
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _head_workspace(need, workspace, device):
    """The caller's workspace (the library checks its size), or one of `need`
    bytes."""
    import torch
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _dev(workspace, torch.uint8, "workspace", 1)
    _here(workspace, "workspace")
    return workspace


def _activation(name):
    if name not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}, got {name!r}")
    return ACTIVATIONS[name]


def linear_workspace_bytes(M: int, N: int, K: int, dtype) -> int:
    return int(lib().w2v_linear_workspace_bytes(M, N, K, _dtypes()[dtype]))


def linear_backward_workspace_bytes(M: int, N: int, K: int, dtype,
                                    activation: str = "none") -> int:
    return int(lib().w2v_linear_backward_workspace_bytes(M, N, K, _dtypes()[dtype],
                                                         _activation(activation)))


def linear(x, weight, bias=None, *, activation: str = "none", residual=None,
           out_dtype=None, out=None, pre=None, workspace=None, stream=None):
    """act(x weight^T + bias) + residual (w2v_linear).

    x (M, K) and weight (N, K) are float32, bfloat16 or float16, rows may be
    padded (a trained M_out of alloc_matrix is a weight); bias float32 (N,);
    residual (M, N) in the output's type. out_dtype: x's type (the default)
    or float32. out: receives the result (may be the residual itself). pre:
    an (M, N) tensor of x's type that receives the sum before the
    activation, for linear_backward."""
    import torch
    code = _head_dtype(x, "x")
    ldx = _operand(x, "x")
    M, K = x.shape
    ldw = _operand(weight, "weight", dtype=x.dtype)
    N = weight.shape[0]
    if weight.shape[1] != K:
        raise ValueError("x and weight must have the same number of columns")
    if bias is not None:
        _vector(bias, torch.float32, "bias", N)
    if out is not None:
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError("out and out_dtype disagree")
        out_dtype = out.dtype
    out_dtype = x.dtype if out_dtype is None else out_dtype
    if out_dtype not in (x.dtype, torch.float32):
        raise TypeError("out_dtype must be x's dtype or float32")
    act = _activation(activation)
    ldr = N if residual is None else _operand(residual, "residual", (M, N), out_dtype)
    ldp = N if pre is None else _operand(pre, "pre", (M, N), x.dtype)
    with _allocations(stream):
        if out is None:
            out = torch.empty((M, N), dtype=out_dtype, device=x.device)
        ldy = _operand(out, "out", (M, N), out_dtype)
        ws = _head_workspace(linear_workspace_bytes(M, N, K, x.dtype), workspace, x.device)
        _check(lib().w2v_linear(
            _ptr(x), ldx, _ptr(weight), ldw, _ptr(bias), _ptr(residual), ldr, _ptr(out), ldy,
            _ptr(pre), ldp, M, N, K, code, _dtypes()[out_dtype], act, _ptr(ws),
            0 if ws is None else ws.numel(), _stream(stream)))
    return out


def linear_backward(dy, x, weight, *, activation: str = "none", pre=None,
                    want_dx: bool = True, want_dw: bool = True, want_db: bool = True,
                    workspace=None, stream=None):
    """Gradients of linear() from dy (M, N): a dict of dx (M, K) and dw (N, K)
    in x's type and db float32 (N,), None where not wanted
    (w2v_linear_backward). pre: what linear() wrote, needed with an
    activation; dy act'(pre) is then rounded to x's type for dx and dw, and
    summed before that for db. The residual's gradient is dy."""
    import torch
    code = _head_dtype(x, "x")
    ldx = _operand(x, "x")
    M, K = x.shape
    ldw = _operand(weight, "weight", dtype=x.dtype)
    N = weight.shape[0]
    if weight.shape[1] != K:
        raise ValueError("x and weight must have the same number of columns")
    lddy = _operand(dy, "dy", (M, N), x.dtype)
    act = _activation(activation)
    if act != 0 and pre is None:
        raise ValueError("pre is needed with an activation")
    ldp = N if pre is None else _operand(pre, "pre", (M, N), x.dtype)
    with _allocations(stream):
        out = dict(
            dx=torch.empty((M, K), dtype=x.dtype, device=x.device) if want_dx else None,
            dw=torch.empty((N, K), dtype=x.dtype, device=x.device) if want_dw else None,
            db=torch.empty(N, dtype=torch.float32, device=x.device) if want_db else None)
        ws = _head_workspace(linear_backward_workspace_bytes(M, N, K, x.dtype, activation),
                             workspace, x.device)
        _check(lib().w2v_linear_backward(
            _ptr(dy), lddy, _ptr(x), ldx, _ptr(weight), ldw, _ptr(pre), ldp, _ptr(out["dx"]),
            K, _ptr(out["dw"]), K, _ptr(out["db"]), M, N, K, code, act, _ptr(ws),
            0 if ws is None else ws.numel(), _stream(stream)))
    return out


def _teacher_list(logits, teacher_ids, teacher_logits, labels):
    """Checked arguments that both distillation calls share, in the library's
    order."""
    import torch
    code = _head_dtype(logits, "logits")
    ld = _operand(logits, "logits")
    rows, V = logits.shape
    _dev(teacher_ids, torch.int32, "teacher_ids", 2)
    _here(teacher_ids, "teacher_ids")
    _head_dtype(teacher_logits, "teacher_logits")
    _dev(teacher_logits, teacher_logits.dtype, "teacher_logits", 2)
    _here(teacher_logits, "teacher_logits")
    if teacher_ids.shape[0] != rows or teacher_logits.shape != teacher_ids.shape:
        raise ValueError("teacher_ids and teacher_logits must have a row per row of logits")
    if labels is not None:
        _vector(labels, torch.int32, "labels", rows)
    return (_ptr(logits), ld, rows, V, code, _ptr(teacher_ids), _ptr(teacher_logits),
            teacher_ids.shape[1], _dtypes()[teacher_logits.dtype], _ptr(labels))


def distill_workspace_bytes(rows: int, V: int, dtype) -> int:
    return int(lib().w2v_distill_workspace_bytes(rows, V, _dtypes()[dtype]))


def distill_loss(logits, teacher_ids, teacher_logits, *, temperature: float = 1.0,
                 labels=None, soft: float = 1.0, hard: float = 0.0, row_weight=None,
                 want_grad: bool = False, grad=None, workspace=None, stream=None):
    """Distillation from a teacher's top logits (w2v_distill_loss): a dict of
    loss float32 (rows,), stats float32 (rows, 3) for distill_backward, and
    grad (logits' shape and type) or None.

    logits (rows, V) float32, bfloat16 or float16, rows may be padded;
    teacher_ids int32 (rows, K), -1 absent; teacher_logits (rows, K) of any of
    the three types; labels int32 (rows,), -1 none. The loss of a row is soft
    T^2 KL(teacher || student at T) + hard (-log p(label)). want_grad: the
    gradient of the losses' sum, each row's scaled by row_weight (float32
    (rows,), 1 if None). grad: receives it (logits itself: in place)."""
    import torch
    head = _teacher_list(logits, teacher_ids, teacher_logits, labels)
    rows = logits.shape[0]
    if row_weight is not None:
        _vector(row_weight, torch.float32, "row_weight", rows)
    with _allocations(stream):
        if want_grad and grad is None:
            grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        ldg = 0 if grad is None else _operand(grad, "grad", logits.shape, logits.dtype)
        loss = torch.empty(rows, dtype=torch.float32, device=logits.device)
        stats = torch.empty((rows, 3), dtype=torch.float32, device=logits.device)
        ws = _head_workspace(distill_workspace_bytes(rows, logits.shape[1], logits.dtype),
                             workspace, logits.device)
        _check(lib().w2v_distill_loss(
            *head, float(temperature), float(soft), float(hard), _ptr(row_weight), _ptr(loss),
            _ptr(stats), _ptr(grad), ldg, _ptr(ws), 0 if ws is None else ws.numel(),
            _stream(stream)))
    return dict(loss=loss, stats=stats, grad=grad)


def distill_backward(dloss, logits, teacher_ids, teacher_logits, stats, *,
                     temperature: float = 1.0, labels=None, soft: float = 1.0,
                     hard: float = 0.0, grad=None, stream=None):
    """Gradient of distill_loss() for the losses' gradients dloss float32
    (rows,), from its stats (w2v_distill_backward); the other arguments as
    they were there. grad: receives it (logits itself: in place)."""
    import torch
    head = _teacher_list(logits, teacher_ids, teacher_logits, labels)
    rows = logits.shape[0]
    _vector(dloss, torch.float32, "dloss", rows)
    _dev(stats, torch.float32, "stats", 2)
    _here(stats, "stats")
    if tuple(stats.shape) != (rows, 3):
        raise ValueError("stats must have shape (rows, 3)")
    with _allocations(stream):
        if grad is None:
            grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        ldg = _operand(grad, "grad", logits.shape, logits.dtype)
        _check(lib().w2v_distill_backward(
            _ptr(dloss), *head, float(temperature), float(soft), float(hard), _ptr(stats),
            _ptr(grad), ldg, _stream(stream)))
    return grad


MAX_TOP_K = 1024


def sample_workspace_bytes(rows: int, V: int) -> int:
    return int(lib().w2v_sample_workspace_bytes(rows, V))


def sample_words(logits, uniforms=None, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0,
                 want_logprob: bool = True, workspace=None, stream=None):
    """Draws a word from each row of scores (w2v_sample_words): a dict of ids
    int32 (rows,) and logprob float32 (rows,) or None.

    logits (rows, V) float32, bfloat16 or float16, -inf masks a word; uniforms
    float32 (rows, V), independent random numbers in (0, 1) (not needed at
    temperature 0). temperature, top_k, top_p and min_p are numbers, or
    tensors of one setting per row (float32; top_k int32). 0 for the
    temperature takes the best word; top_k 0, top_p 1 and min_p 0 are off. A
    row without a word gets id -1."""
    import torch
    code = _head_dtype(logits, "logits")
    ld = _operand(logits, "logits")
    rows, V = logits.shape
    ldu = V if uniforms is None else _operand(uniforms, "uniforms", (rows, V), torch.float32)

    def setting(v, name, dtype, kind):
        if isinstance(v, torch.Tensor):
            return _ptr(_vector(v, dtype, name, rows)), kind(0)
        return None, kind(v)

    t = setting(temperature, "temperature", torch.float32, float)
    k = setting(top_k, "top_k", torch.int32, int)
    p = setting(top_p, "top_p", torch.float32, float)
    least = setting(min_p, "min_p", torch.float32, float)
    with _allocations(stream):
        ids = torch.empty(rows, dtype=torch.int32, device=logits.device)
        logprob = torch.empty(rows, dtype=torch.float32, device=logits.device) \
            if want_logprob else None
        ws = _head_workspace(sample_workspace_bytes(rows, V), workspace, logits.device)
        _check(lib().w2v_sample_words(
            _ptr(logits), ld, _ptr(uniforms), ldu, rows, V, code, *t, *k, *p, *least,
            _ptr(ids), _ptr(logprob), _ptr(ws), 0 if ws is None else ws.numel(),
            _stream(stream)))
    return dict(ids=ids, logprob=logprob)


# ------------------------------------------------------- a word model's ends --

def embed(ids, weight, *, scale: float = 1.0, out_dtype=None, out=None, stream=None):
    """scale * weight[ids] (w2v_embed): (n, D) of out_dtype (weight's type by
    default).

    ids int32 (n,), -1 = absent, whose row is 0; weight (V, D) float32,
    bfloat16 or float16, rows may be padded (a trained M_in of alloc_matrix is
    one). out: receives the result."""
    import torch
    code = _head_dtype(weight, "weight")
    ldw = _operand(weight, "weight")
    V, D = weight.shape
    _dev(ids, torch.int32, "ids", 1)
    _here(ids, "ids")
    n = ids.numel()
    if out is not None:
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError("out and out_dtype disagree")
        out_dtype = out.dtype
    out_dtype = weight.dtype if out_dtype is None else out_dtype
    out_code = _dtypes().get(out_dtype)
    if out_code is None:
        raise TypeError(f"out_dtype must be float32, bfloat16 or float16, got {out_dtype}")
    with _allocations(stream):
        if out is None:
            out = torch.empty((n, D), dtype=out_dtype, device=weight.device)
        ldy = _operand(out, "out", (n, D), out_dtype)
        _check(lib().w2v_embed(_ptr(ids), n, _ptr(weight), ldw, V, D, code, float(scale),
                               _ptr(out), ldy, out_code, _stream(stream)))
    return out


def embed_backward_workspace_bytes(n: int, V: int, D: int) -> int:
    return int(lib().w2v_embed_backward_workspace_bytes(n, V, D))


def embed_backward(dy, ids, V: Optional[int] = None, *, scale: float = 1.0, grad=None,
                   accumulate: bool = False, dtype=None, workspace=None, stream=None):
    """Gradient of embed() for the weight from dy (n, D): rows of dy summed by
    word, times scale (w2v_embed_backward).

    A new (V, D) matrix of `dtype` (dy's by default), or `grad`, which is
    overwritten or, with accumulate, added to at the words that occur: with a
    negative scale that is a step of gradient descent on the weight itself."""
    import torch
    code = _head_dtype(dy, "dy")
    lddy = _operand(dy, "dy")
    n, D = dy.shape
    _vector(ids, torch.int32, "ids", n)
    if grad is not None:
        if dtype is not None and grad.dtype != dtype:
            raise TypeError("grad and dtype disagree")
        if V is not None and grad.shape[0] != V:
            raise ValueError("grad must have V rows")
    elif V is None:
        raise ValueError("V is needed without grad")
    elif accumulate:
        raise ValueError("accumulate needs grad")
    with _allocations(stream):
        if grad is None:
            grad = torch.empty((V, D), dtype=dy.dtype if dtype is None else dtype,
                               device=dy.device)
        grad_code = _head_dtype(grad, "grad")
        V = grad.shape[0]
        ldg = _operand(grad, "grad", (V, D))
        ws = _head_workspace(embed_backward_workspace_bytes(n, V, D), workspace, dy.device)
        _check(lib().w2v_embed_backward(
            _ptr(dy), lddy, _ptr(ids), n, code, float(scale), _ptr(grad), ldg, V, D, grad_code,
            1 if accumulate else 0, _ptr(ws), 0 if ws is None else ws.numel(),
            _stream(stream)))
    return grad


def dropout(x, p: float, *, seed: int, offset: int = 0, offset_dev=None, residual=None,
            out=None, stream=None):
    """x with each element dropped with probability p, the others over 1 - p,
    plus the residual (w2v_dropout).

    x (rows, cols) float32, bfloat16 or float16, rows may be padded. Which
    elements are dropped follows from seed, offset (a different one for every
    layer and step, both modulo 2^64) and an element's place alone: the
    gradient is dropout(dy, p, ...) with the same ones. offset_dev: an int64
    GPU tensor of one entry that the kernel adds to offset, for captured graphs.
    out: receives the result (may be x or the residual itself)."""
    import torch
    code = _head_dtype(x, "x")
    ldx = _operand(x, "x")
    rows, cols = x.shape
    ldr = cols if residual is None else _operand(residual, "residual", (rows, cols), x.dtype)
    if offset_dev is not None:
        _vector(offset_dev, torch.int64, "offset_dev", 1)
    with _allocations(stream):
        if out is None:
            out = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        ldy = _operand(out, "out", (rows, cols), x.dtype)
        _check(lib().w2v_dropout(
            _ptr(x), ldx, _ptr(residual), ldr, _ptr(out), ldy, rows, cols, code, float(p),
            seed & 0xFFFFFFFFFFFFFFFF, offset & 0xFFFFFFFFFFFFFFFF, _ptr(offset_dev),
            _stream(stream)))
    return out


def quantize_q4(weight, *, group: int = 32, stream=None):
    """weight (N, K) in 4 bits with a bfloat16 scale for each `group` (32, 64 or
    128) columns of a row (w2v_quantize_q4): a dict for linear_q4 of packed
    (uint8) and scales (bfloat16), laid out as w2v.h says, shape (N, K) and
    group."""
    import torch
    code = _head_dtype(weight, "weight")
    ldw = _operand(weight, "weight")
    N, K = weight.shape
    with _allocations(stream):
        packed = torch.empty(int(lib().w2v_q4_packed_bytes(N, K, group)), dtype=torch.uint8,
                             device=weight.device)
        scales = torch.empty(int(lib().w2v_q4_scale_count(N, K, group)), dtype=torch.bfloat16,
                             device=weight.device)
        _check(lib().w2v_quantize_q4(_ptr(weight), ldw, N, K, code, group, _ptr(packed),
                                     _ptr(scales), _stream(stream)))
    return dict(packed=packed, scales=scales, shape=(N, K), group=group)


def linear_q4(x, weight, bias=None, *, out_dtype=None, out=None, stream=None):
    """x W^T + bias for a W of quantize_q4() (w2v_linear_q4), which is read once
    for every 64 rows of x or fewer.

    x (M, K) float32, bfloat16 or float16, rows may be padded; bias float32
    (N,). out_dtype: x's type (the default) or float32. out: receives the
    result."""
    import torch
    code = _head_dtype(x, "x")
    ldx = _operand(x, "x")
    M, K = x.shape
    N, group = weight["shape"][0], weight["group"]
    if weight["shape"][1] != K:
        raise ValueError("x and weight must have the same number of columns")
    if group not in (32, 64, 128):
        raise ValueError("group must be 32, 64 or 128")
    # w2v_q4_packed_bytes and w2v_q4_scale_count, without the calls
    tiles, groups = (N + 15) // 16, (K + group - 1) // group
    _vector(weight["packed"], torch.uint8, "packed", tiles * groups * group * 8)
    _vector(weight["scales"], torch.bfloat16, "scales", tiles * groups * 16)
    if bias is not None:
        _vector(bias, torch.float32, "bias", N)
    if out is not None:
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError("out and out_dtype disagree")
        out_dtype = out.dtype
    out_dtype = x.dtype if out_dtype is None else out_dtype
    if out_dtype not in (x.dtype, torch.float32):
        raise TypeError("out_dtype must be x's dtype or float32")
    with _allocations(stream):
        if out is None:
            out = torch.empty((M, N), dtype=out_dtype, device=x.device)
        ldy = _operand(out, "out", (M, N), out_dtype)
        _check(lib().w2v_linear_q4(
            _ptr(x), ldx, _ptr(weight["packed"]), _ptr(weight["scales"]), _ptr(bias), _ptr(out),
            ldy, M, N, K, group, code, _dtypes()[out_dtype], _stream(stream)))
    return out


MAX_BEAMS = 64


def beam_step_workspace_bytes(batch: int, beams: int, width: int, V: int, dtype) -> int:
    return int(lib().w2v_beam_step_workspace_bytes(batch, beams, width, V, _dtypes()[dtype]))


def beam_step(logits, scores, *, width: Optional[int] = None, finished=None, end: int = -1,
              workspace=None, stream=None):
    """The best `width` (as many as beams by default) continuations of each
    entry's beams (w2v_beam_step): a dict of words and parents int32 (batch,
    width), scores float32 (batch, width), best first, and finished uint8
    (batch, width), or None without `end`.

    logits (batch * beams, V) float32, bfloat16 or float16, rows may be padded,
    -inf masks a word; scores float32 (batch, beams), a beam's log-probability
    so far, -inf where there is none (at first: 0 and then -inf); finished uint8
    (batch, beams): beams that have ended, which stay as they are; end: the word
    that ends a beam. Places without a continuation get -1, -1 and -inf."""
    import torch
    code = _head_dtype(logits, "logits")
    ld = _operand(logits, "logits")
    _dev(scores, torch.float32, "scores", 2)
    _here(scores, "scores")
    batch, beams = scores.shape
    rows, V = logits.shape
    if rows != batch * beams:
        raise ValueError("logits must have a row per score")
    width = beams if width is None else width
    if finished is not None:
        _dev(finished, torch.uint8, "finished", 2)
        _here(finished, "finished")
        if finished.shape != scores.shape:
            raise ValueError("finished must have the scores' shape")
    dev = logits.device
    with _allocations(stream):
        need = int(lib().w2v_beam_step_workspace_bytes(batch, beams, width, V, code))
        places = (batch, max(width, 0))
        words = torch.empty(places, dtype=torch.int32, device=dev)
        parents = torch.empty(places, dtype=torch.int32, device=dev)
        new_scores = torch.empty(places, dtype=torch.float32, device=dev)
        ended = torch.empty(places, dtype=torch.uint8, device=dev) if end != -1 else None
        ws = _head_workspace(need, workspace, dev)
        _check(lib().w2v_beam_step(
            _ptr(logits), ld, batch, beams, V, code, _ptr(scores), _ptr(finished), end, width,
            _ptr(words), _ptr(parents), _ptr(new_scores), _ptr(ended), _ptr(ws),
            0 if ws is None else ws.numel(), _stream(stream)))
    return dict(words=words, parents=parents, scores=new_scores, finished=ended)


MAX_BEAM_STATES = 16


def _state_rows(t, name):
    """Bytes of a row of a state, and from one row to the next."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    _here(t, name)
    size = t.shape
    if len(size) < 1:
        raise ValueError(f"{name} must have a first dimension")
    if t.is_conj() or t.is_neg():
        raise ValueError(f"{name} must hold its own values (resolve_conj, resolve_neg)")
    row = t.element_size()
    for n in size[1:]:
        row *= n
    if t.is_contiguous():
        return row, row
    if not t[0].is_contiguous():
        raise ValueError(f"{name} must have contiguous rows")
    step = t.stride(0) * t.element_size()
    if size[0] > 1 and step < row:
        raise ValueError(f"{name} must have rows that do not overlap")
    return row, max(step, row)


def beam_reorder(states, parents, *, out=None, stream=None):
    """The beams' states where beam_step() has their continuations
    (w2v_beam_reorder): row entry * width + j is row entry * beams +
    parents[entry, j], zeros where the parent is -1.

    states: a GPU tensor of batch * beams rows of any shape and type, or a list
    of up to 16; parents int32 (batch, width). out: receives the result, in
    states' form (not a state itself). Returns it in that form."""
    import torch
    one = isinstance(states, torch.Tensor)
    states = [states] if one else states
    _dev(parents, torch.int32, "parents", 2)
    _here(parents, "parents")
    batch, width = parents.shape
    if len(states) > MAX_BEAM_STATES:
        raise ValueError(f"at most {MAX_BEAM_STATES} states")
    new = None if out is None else [out] if one else list(out)
    if new is not None and len(new) != len(states):
        raise ValueError("out must have a tensor per state")
    beams = None
    table = (_BeamState * max(1, len(states)))()
    with _allocations(stream):
        made = []
        for i, t in enumerate(states):
            row, step = _state_rows(t, "states")
            size = t.shape
            of = size[0] // batch if batch else 1
            if of * batch != size[0] or of < 1 or (beams is not None and of != beams):
                raise ValueError("states must have batch * beams rows each")
            if of > _MOST:
                raise ValueError("states must have less than 2^31 rows of an entry")
            beams = of
            moved = (batch * width, *size[1:])
            if new is None:
                o, out_step = torch.empty(moved, dtype=t.dtype, device=t.device), row
                made.append(o)
            else:
                o = new[i]
                out_step = _state_rows(o, "out")[1]
                if o.dtype != t.dtype or o.shape != moved:
                    raise ValueError("out must have batch * width rows of the state's")
            entry = table[i]
            entry.src, entry.src_stride = t.data_ptr(), step
            entry.dst, entry.dst_stride, entry.row_bytes = o.data_ptr(), out_step, row
        _check(lib().w2v_beam_reorder(table, len(states), _ptr(parents), batch,
                                      1 if beams is None else beams, width, _stream(stream)))
    new = made if new is None else new
    return new[0] if one else new
