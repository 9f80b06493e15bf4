"""ctypes binding of the RS-DGC CUDA library (``include/rsdgc.h``).

Argument marshalling only: every step of the compression path runs in the library's
kernels.  PyTorch tensors supply device memory and the current CUDA stream.  There is no
CPU fallback: if the shared library is missing, :func:`lib` raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import List, Optional, Sequence, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
# RSDGC_LIBRARY selects another build of the same library (e.g. the bounds-checked one)
LIB_PATH = os.environ.get("RSDGC_LIBRARY") or os.path.join(_HERE, "librsdgc_b200.so")

RSDGC_F32, RSDGC_BF16, RSDGC_F16 = 0, 1, 2
KEEP_AT_LEAST_ONE = 1
NO_BULK_COPY = 2
MOMENTUM = 4
PAYLOAD_BF16 = 8
NO_FUSED_TAIL = 16
STATUS_NONFINITE, STATUS_PAYLOAD_OVERFLOW, STATUS_TIMEOUT, STATUS_BOUNDS = 1, 2, 4, 8
OK, ERR_INVALID, ERR_ALIGNMENT, ERR_CAPACITY, ERR_CUDA, ERR_NOMEM = 0, -1, -2, -3, -4, -5

EXPORTS = [
    "rsdgc_plan_create", "rsdgc_plan_destroy", "rsdgc_plan_info", "rsdgc_plan_layer_info",
    "rsdgc_plan_payload_bound", "rsdgc_plan_worklist", "rsdgc_update_ratios", "rsdgc_compress",
    "rsdgc_compress_host", "rsdgc_decompress_accumulate", "rsdgc_get_status", "rsdgc_launch_count",
    "rsdgc_strerror", "rsdgc_last_cuda_error", "rsdgc_profile_enable", "rsdgc_profile_read",
    "rsdgc_update_ratios_noalloc", "rsdgc_compress_momentum", "rsdgc_plan_reserve_workers",
    "rsdgc_compress_workers", "rsdgc_decompress_assign", "rsdgc_payload_to_coo", "rsdgc_compress_workers_host",
    "rsdgc_selftest_bounded_wait", "rsdgc_plan_tail_slices", "rsdgc_operator_status",
    "rsdgc_layer_norm_workspace_bytes", "rsdgc_layer_norm_forward", "rsdgc_layer_norm_backward",
    "rsdgc_head_workspace_bytes", "rsdgc_head_loss_forward", "rsdgc_head_loss_backward", "rsdgc_head_distill_forward",
    "rsdgc_head_distill_backward", "rsdgc_selftest_operator_polls",
    "rsdgc_selftest_operator_wait", "rsdgc_head_forward_workspace_bytes",
]
NOALLOC_MAX_LAYERS = 64
N_COMPRESS_KERNELS = 5
COMPRESS_KERNELS = ("accumulate_nsi", "refine2", "refine3_count", "mark", "gather")


class LayerDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("nh", C.c_int32), ("nw", C.c_int32)]


class Info(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("grad_dtype", C.c_int32), ("arena_elems", C.c_int64),
                ("total_elems", C.c_int64), ("total_tiles", C.c_int64), ("total_tiles_padded", C.c_int64),
                ("workspace_bytes", C.c_int64), ("max_slot", C.c_int32), ("reserved", C.c_int32)]


class LayerInfo(C.Structure):
    _fields_ = [("elem_offset", C.c_int64), ("tile_offset", C.c_int64), ("rows", C.c_int64),
                ("cols", C.c_int64), ("nh", C.c_int32), ("nw", C.c_int32), ("n_tiles", C.c_int64)]


class Status(C.Structure):
    _fields_ = [("flags", C.c_uint32), ("reserved", C.c_uint32), ("nonfinite", C.c_int64),
                ("idx_needed", C.c_int64), ("val_needed", C.c_int64)]


class RsdgcError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        msg = lib().rsdgc_strerror(code).decode()
        if code == ERR_CUDA:
            msg += " (cudaError %d)" % lib().rsdgc_last_cuda_error()
        super().__init__("%s: %s [%d]" % (what, msg, code))


_lib = None


def lib():
    """The loaded C library; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("CUDA library %s is missing: build it with "
                               "`python -m paper_2312_17530_b200.build`" % LIB_PATH)
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, f32, u32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_uint32
        L.rsdgc_plan_create.argtypes = [C.POINTER(LayerDesc), i32, i32, f32, u32, i32, C.POINTER(vp)]
        L.rsdgc_plan_destroy.argtypes = [vp]
        L.rsdgc_plan_info.argtypes = [vp, C.POINTER(Info)]
        L.rsdgc_plan_layer_info.argtypes = [vp, i32, C.POINTER(LayerInfo)]
        L.rsdgc_plan_payload_bound.argtypes = [vp, f32, C.POINTER(i64), C.POINTER(i64)]
        L.rsdgc_plan_worklist.argtypes = [vp, vp, i64, vp, vp]
        L.rsdgc_plan_worklist.restype = i64
        L.rsdgc_update_ratios.argtypes = [vp, vp, f32, vp, vp]
        L.rsdgc_compress.argtypes = [vp, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, vp]
        L.rsdgc_compress_momentum.argtypes = [vp, vp, vp, f32, vp, vp, vp, i64, vp, i64, vp, vp, vp, vp]
        L.rsdgc_plan_reserve_workers.argtypes = [vp, i32]
        L.rsdgc_compress_workers.argtypes = [vp, i32, C.POINTER(vp), C.POINTER(vp), vp, C.POINTER(vp), i64,
                                             C.POINTER(vp), i64, C.POINTER(vp), vp, vp]
        L.rsdgc_compress_host.argtypes = [vp, vp, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, vp, vp,
                                          C.POINTER(i64), C.POINTER(i64), vp]
        pp = C.POINTER(vp)
        L.rsdgc_compress_workers_host.argtypes = [vp, i32, pp, pp, pp, vp, pp, i64, pp, i64, pp, vp, pp, pp, pp,
                                                  C.POINTER(i64), C.POINTER(i64), vp]
        L.rsdgc_decompress_accumulate.argtypes = [vp, i32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), i64, i64, f32,
                                                  vp, vp]
        L.rsdgc_decompress_assign.argtypes = [vp, i32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), i64, i64, f32, vp,
                                              vp]
        L.rsdgc_payload_to_coo.argtypes = [vp, vp, vp, vp, i64, vp]
        L.rsdgc_get_status.argtypes = [vp, vp, C.POINTER(Status)]
        L.rsdgc_profile_enable.argtypes = [vp, i32]
        L.rsdgc_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(i64)]
        L.rsdgc_update_ratios_noalloc.argtypes = [vp, C.POINTER(i64), C.POINTER(i64), i32, f32, vp, vp]
        L.rsdgc_selftest_bounded_wait.argtypes = [vp, i32, vp]
        L.rsdgc_plan_tail_slices.argtypes = [vp, vp, i64, vp]
        L.rsdgc_plan_tail_slices.restype = i64
        L.rsdgc_operator_status.argtypes = [vp, C.POINTER(u32)]
        L.rsdgc_selftest_operator_polls.argtypes = [i32]
        L.rsdgc_selftest_operator_wait.argtypes = [i32, vp]
        L.rsdgc_layer_norm_workspace_bytes.argtypes = [i64, i64]
        L.rsdgc_layer_norm_workspace_bytes.restype = i64
        L.rsdgc_layer_norm_forward.argtypes = [vp, i64, vp, vp, vp, i64, vp, vp, i64, i64, i32, i32, f32, vp]
        L.rsdgc_layer_norm_backward.argtypes = [vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, vp, i32, i64, i64, i32, i32,
                                                vp, vp]
        L.rsdgc_head_workspace_bytes.argtypes = [i64, i64, i64, i64]
        L.rsdgc_head_workspace_bytes.restype = i64
        L.rsdgc_head_forward_workspace_bytes.argtypes = [i64, i64, i64, i64]
        L.rsdgc_head_forward_workspace_bytes.restype = i64
        L.rsdgc_head_loss_forward.argtypes = [vp, i64, vp, i64, vp, vp, vp, i64, i64, i64, i32, vp, vp]
        L.rsdgc_head_loss_backward.argtypes = [vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, i64, i32, i64, i64, i64, i32, vp,
                                               vp]
        L.rsdgc_head_distill_forward.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, i32, i64, f32, vp, vp, i64, i64, i64,
                                                 i32, vp, vp]
        L.rsdgc_head_distill_backward.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, i32, i64, f32, vp, vp, vp, i64, vp,
                                                  i64, i32, i64, i64, i64, i32, vp, vp]
        L.rsdgc_launch_count.argtypes = []
        L.rsdgc_launch_count.restype = i64
        L.rsdgc_strerror.argtypes = [C.c_int]
        L.rsdgc_strerror.restype = C.c_char_p
        L.rsdgc_last_cuda_error.argtypes = []
        for name in EXPORTS:
            fn = getattr(L, name)
            if fn.restype is C.c_int:  # default restype: all the int-returning entry points
                fn.restype = C.c_int
        _lib = L
    return _lib


def _check(code: int, what: str) -> None:
    if code != OK:
        raise RsdgcError(code, what)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


class _Torch:
    """What the calls need of torch, looked up once (importing this module does not import torch)."""

    def __init__(self):
        import torch

        self.f32, self.i64 = torch.float32, torch.int64
        self.codes = {torch.float32: RSDGC_F32, torch.bfloat16: RSDGC_BF16, torch.float16: RSDGC_F16}
        self.device = torch.cuda.current_device
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # the handle without a Stream object around it
        self.stream = raw or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


_torch = None


def _tt() -> _Torch:
    global _torch
    if _torch is None:
        _torch = _Torch()
    return _torch


def _stream() -> int:
    t = _torch or _tt()
    return t.stream(t.device())


class Plan:
    """Owns an ``rsdgc_plan``.  ``layers``: sequence of (rows, cols, nh, nw).  ``device`` < 0
    gives a host-only plan (sizes and offsets only; usable without a GPU)."""

    def __init__(self, layers: Sequence[Tuple[int, int, int, int]], grad_dtype: int = RSDGC_F32,
                 alpha: float = 0.5, flags: int = KEEP_AT_LEAST_ONE, device: int = 0):
        arr = (LayerDesc * max(1, len(layers)))()
        for i, (r, c, nh, nw) in enumerate(layers):
            arr[i] = LayerDesc(int(r), int(c), int(nh), int(nw))
        h = C.c_void_p()
        self._h = None
        _check(lib().rsdgc_plan_create(arr, len(layers), grad_dtype, alpha, flags, device, C.byref(h)),
               "rsdgc_plan_create")
        self._h = h
        self.device = device
        self.n_layers = len(layers)
        self.grad_dtype = grad_dtype
        self.flags = int(flags)
        info = Info()
        _check(lib().rsdgc_plan_info(self._h, C.byref(info)), "rsdgc_plan_info")
        self.info = info
        self.layers: List[LayerInfo] = []
        for l in range(self.n_layers):
            li = LayerInfo()
            _check(lib().rsdgc_plan_layer_info(self._h, l, C.byref(li)), "rsdgc_plan_layer_info")
            self.layers.append(li)

    def close(self) -> None:
        if self._h is not None:
            lib().rsdgc_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- sizes --------------------------------------------------------------------------
    def payload_bound(self, max_ratio: float) -> Tuple[int, int]:
        a, b = C.c_int64(), C.c_int64()
        _check(lib().rsdgc_plan_payload_bound(self._h, max_ratio, C.byref(a), C.byref(b)),
               "rsdgc_plan_payload_bound")
        return a.value, b.value

    def worklist(self):
        """(items [n,9] int32: layer, tr0, ntr, tc0, ntc, kernel, cta, shared-memory pitch, item
        flags (1 contiguous, 2 128-bit accesses, 4 bulk copies, 8 no clipped tile); grids [2];
        n_flush [L])."""
        import numpy as np

        n = lib().rsdgc_plan_worklist(self._h, None, 0, None, None)
        items = np.zeros((n, 9), dtype=np.int32)
        grids = np.zeros(2, dtype=np.int32)
        nf = np.zeros(self.n_layers, dtype=np.int32)
        lib().rsdgc_plan_worklist(self._h, items.ctypes.data, n, grids.ctypes.data, nf.ctypes.data)
        return items, grids, nf

    def tail_slices(self):
        """(slices [n,6] int32: layer, first tile, tiles, CTAs of the layer, rank, leader rank; info [3]:
        cluster-variant CTAs, one-CTA layers, clusters) of the single-kernel selection + pack; n = 0 when
        the plan takes the chained kernels."""
        import numpy as np

        n = lib().rsdgc_plan_tail_slices(self._h, None, 0, None)
        sl = np.zeros((max(n, 0), 6), dtype=np.int32)
        info = np.zeros(3, dtype=np.int32)
        lib().rsdgc_plan_tail_slices(self._h, sl.ctypes.data, n, info.ctypes.data)
        return sl, info

    # ---- device calls (torch tensors on the plan's device) -------------------------------
    def update_ratios(self, weights, global_keep: float, ratios) -> None:
        _check(lib().rsdgc_update_ratios(self._h, _ptr(weights), global_keep, _ptr(ratios), _stream()),
               "rsdgc_update_ratios")

    def compress(self, grads, residual, ratios, idx, val, counts, nsi=None, workspace=None) -> None:
        _check(lib().rsdgc_compress(self._h, _ptr(grads), _ptr(residual), _ptr(ratios), _ptr(idx), idx.numel(),
                                    _ptr(val), val.numel(), _ptr(counts), _ptr(nsi), _ptr(workspace), _stream()),
               "rsdgc_compress")

    def compress_momentum(self, grads, velocity, momentum: float, residual, ratios, idx, val, counts, nsi=None,
                          workspace=None) -> None:
        _check(lib().rsdgc_compress_momentum(self._h, _ptr(grads), _ptr(velocity), momentum, _ptr(residual),
                                             _ptr(ratios), _ptr(idx), idx.numel(), _ptr(val), val.numel(),
                                             _ptr(counts), _ptr(nsi), _ptr(workspace), _stream()),
               "rsdgc_compress_momentum")

    def reserve_workers(self, n_workers: int) -> None:
        _check(lib().rsdgc_plan_reserve_workers(self._h, int(n_workers)), "rsdgc_plan_reserve_workers")

    def compress_workers(self, grads, residuals, ratios, idx, val, counts, workspace) -> None:
        """One call for several workers: ``grads``, ``residuals``, ``idx``, ``val``, ``counts`` are
        sequences with one device tensor per worker; ``workspace`` holds n_workers * workspace_bytes."""
        n = len(grads)
        A = C.c_void_p * max(1, n)
        ga, ra, ia, va, ca = A(), A(), A(), A(), A()
        for w in range(n):
            ga[w], ra[w], ca[w] = grads[w].data_ptr(), residuals[w].data_ptr(), counts[w].data_ptr()
            ia[w], va[w] = idx[w].data_ptr(), val[w].data_ptr()
        _check(lib().rsdgc_compress_workers(self._h, n, ga, ra, _ptr(ratios), ia, min(t.numel() for t in idx), va,
                                            min(t.numel() for t in val), ca, _ptr(workspace), _stream()),
               "rsdgc_compress_workers")

    def compress_host(self, grads_host, grads_dev, residual, ratios, idx, val, counts, workspace,
                      idx_host, val_host, counts_host) -> Tuple[int, int]:
        ni, nv = C.c_int64(), C.c_int64()
        _check(lib().rsdgc_compress_host(self._h, _ptr(grads_host), _ptr(grads_dev), _ptr(residual), _ptr(ratios),
                                         _ptr(idx), idx.numel(), _ptr(val), val.numel(), _ptr(counts),
                                         _ptr(workspace), _ptr(idx_host), _ptr(val_host), _ptr(counts_host),
                                         C.byref(ni), C.byref(nv), _stream()), "rsdgc_compress_host")
        return ni.value, nv.value

    def compress_workers_host(self, grads_host, staging, residuals, ratios, idx, val, counts, workspace,
                              idx_host, val_host, counts_host):
        """rsdgc_compress_workers_host(): per-worker sequences of host gradients / host payload buffers and
        device residuals / payload buffers, ``staging`` = two device arenas.  Returns the per-worker
        (idx_used, val_used) lists."""
        n = len(grads_host)
        A = C.c_void_p * max(1, n)
        gh, rd, ia, va, ca, ih, vh, ch = A(), A(), A(), A(), A(), A(), A(), A()
        for w in range(n):
            gh[w], rd[w], ca[w] = grads_host[w].data_ptr(), residuals[w].data_ptr(), counts[w].data_ptr()
            ia[w], va[w] = idx[w].data_ptr(), val[w].data_ptr()
            ih[w], vh[w], ch[w] = idx_host[w].data_ptr(), val_host[w].data_ptr(), counts_host[w].data_ptr()
        st = (C.c_void_p * 2)(staging[0].data_ptr(), staging[1].data_ptr())
        ni, nv = (C.c_int64 * max(1, n))(), (C.c_int64 * max(1, n))()
        _check(lib().rsdgc_compress_workers_host(
            self._h, n, gh, st, rd, _ptr(ratios), ia, min(t.numel() for t in idx), va, min(t.numel() for t in val),
            ca, _ptr(workspace), ih, vh, ch, ni, nv, _stream()), "rsdgc_compress_workers_host")
        return list(ni)[:n], list(nv)[:n]

    def decompress_accumulate(self, payloads, dense, scale: float = 1.0, assign: bool = False) -> None:
        """``payloads``: sequence of (idx, val, counts) device tensors, one per worker.  ``assign``:
        rsdgc_decompress_assign() (the arena is zero-filled by the same launch)."""
        n = len(payloads)
        A = C.c_void_p * max(1, n)
        ia, va, ca = A(), A(), A()
        for w, (i, v, c) in enumerate(payloads):
            ia[w], va[w], ca[w] = i.data_ptr(), v.data_ptr(), c.data_ptr()
        fn = lib().rsdgc_decompress_assign if assign else lib().rsdgc_decompress_accumulate
        idx_cap = min((i.numel() for i, _, _ in payloads), default=0)
        val_cap = min((v.numel() for _, v, _ in payloads), default=0)
        _check(fn(self._h, n, ia, va, ca, idx_cap, val_cap, scale, _ptr(dense), _stream()),
               "rsdgc_decompress_assign" if assign else "rsdgc_decompress_accumulate")

    def decompress_assign(self, payloads, dense, scale: float = 1.0) -> None:
        self.decompress_accumulate(payloads, dense, scale, assign=True)

    def payload_to_coo(self, idx, counts, coo_index) -> None:
        """Arena position (int64) of every payload value, -1 for padding slots."""
        _check(lib().rsdgc_payload_to_coo(self._h, _ptr(idx), _ptr(counts), _ptr(coo_index), coo_index.numel(),
                                          _stream()), "rsdgc_payload_to_coo")

    def profile_enable(self, level: int) -> None:
        """0 off; 1 events around the first pass only; 2 events around every kernel."""
        _check(lib().rsdgc_profile_enable(self._h, int(level)), "rsdgc_profile_enable")

    def profile_read(self):
        """(milliseconds summed per compress kernel, number of compress calls recorded)."""
        ms = (C.c_double * N_COMPRESS_KERNELS)()
        n = C.c_int64()
        _check(lib().rsdgc_profile_read(self._h, ms, C.byref(n)), "rsdgc_profile_read")
        return list(ms), n.value

    def selftest_bounded_wait(self, polls: int = 256) -> None:
        """Diagnostic: a bounded on-chip wait that is certain to give up; sets STATUS_TIMEOUT."""
        _check(lib().rsdgc_selftest_bounded_wait(self._h, int(polls), _stream()), "rsdgc_selftest_bounded_wait")

    def status(self) -> Status:
        st = Status()
        _check(lib().rsdgc_get_status(self._h, _stream(), C.byref(st)), "rsdgc_get_status")
        return st


def update_ratios_noalloc(weights, layer_offsets: Sequence[int], layer_sizes: Sequence[int], global_keep: float,
                          ratios) -> None:
    """rsdgc_update_ratios_noalloc(): the ratio rule without a plan and without any allocation
    (scratch is a fixed array inside the library; at most NOALLOC_MAX_LAYERS layers)."""
    n = len(layer_offsets)
    offs = (C.c_int64 * max(1, n))(*[int(x) for x in layer_offsets])
    sizes = (C.c_int64 * max(1, n))(*[int(x) for x in layer_sizes])
    _check(lib().rsdgc_update_ratios_noalloc(_ptr(weights), offs, sizes, n, global_keep, _ptr(ratios), _stream()),
           "rsdgc_update_ratios_noalloc")


# ---- language-model operators (no plan; torch tensors on the current device) ---------------------
def _dtype_code(t) -> int:
    """rsdgc_dtype of a tensor; raises for a type the operators do not take."""
    code = (_torch or _tt()).codes.get(t.dtype)
    if code is None:
        raise ValueError("type %s is not taken: float32, bfloat16 or float16" % t.dtype)
    return code


def _on_device(*tensors) -> int:
    """The stream to work on.  The library sees plain pointers: every tensor given has to be on the current device."""
    t = _torch or _tt()
    dev = t.device()
    for x in tensors:
        if x is not None and x.get_device() != dev:
            raise ValueError("a tensor is not on the current CUDA device (%d)" % dev)
    return t.stream(dev)


def _rows(t, n: int, d: int, what: str) -> int:
    """Row stride of an n x d matrix whose rows are contiguous."""
    if t.shape != (n, d):
        raise ValueError("%s: a %d x %d matrix is wanted, got %s" % (what, n, d, tuple(t.shape)))
    row, col = t.stride()
    if col != 1 and d > 1:
        raise ValueError("%s: rows have to be contiguous" % what)
    return row if n > 1 else d


def _vector(t, n: int, dtype, what: str) -> Optional[int]:
    """Address of n contiguous values (of `dtype`, where one is given), or None."""
    if t is None:
        return None
    if t.numel() != n or t.dim() != 1 or not t.is_contiguous():
        raise ValueError("%s: %d contiguous values are wanted, got %s" % (what, n, tuple(t.shape)))
    if dtype is not None and t.dtype is not dtype:
        raise ValueError("%s: %s is wanted, got %s" % (what, dtype, t.dtype))
    return t.data_ptr()


def _holds(workspace, size: int) -> int:
    if workspace is None or workspace.nbytes < size:
        raise ValueError("workspace: %d bytes are wanted" % size)
    return workspace.data_ptr()


@functools.lru_cache(maxsize=4096)
def layer_norm_workspace_bytes(n_rows: int, width: int) -> int:
    """Bytes of workspace layer_norm_backward() needs for a weight's or bias's gradient."""
    return _size(lib().rsdgc_layer_norm_workspace_bytes(n_rows, width), "rsdgc_layer_norm_workspace_bytes")


def _size(n: int, what: str) -> int:
    if n < 0:
        _check(n, what)
    return n


def layer_norm_forward(x, weight, bias, y, mean=None, rstd=None, eps: float = 1e-5) -> None:
    """``y`` = layer norm of the rows of ``x`` (float32, bfloat16 or float16), times ``weight`` plus ``bias``
    (each may be None; ``x``'s type or float32).  ``mean``, ``rstd``: float32, one per row, for the backward pass."""
    n, d = x.shape
    stream = _on_device(x, weight, bias, y, mean, rstd)
    xs, ys = _rows(x, n, d, "x"), _rows(y, n, d, "y")
    if y.dtype != x.dtype:
        raise ValueError("y: %s is wanted, got %s" % (x.dtype, y.dtype))
    params = x if weight is None and bias is None else bias if weight is None else weight
    f32 = _torch.f32
    code = lib().rsdgc_layer_norm_forward(
        x.data_ptr(), xs, _vector(weight, d, params.dtype, "weight"), _vector(bias, d, params.dtype, "bias"), y.data_ptr(),
        ys, _vector(mean, n, f32, "mean"), _vector(rstd, n, f32, "rstd"), n, d, _dtype_code(x), _dtype_code(params), eps,
        stream)
    if code:
        _check(code, "rsdgc_layer_norm_forward")


def layer_norm_backward(dy, x, weight, mean, rstd, dx=None, dweight=None, dbias=None, workspace=None) -> None:
    """Gradients of layer_norm_forward() for ``dy``: ``dx`` like ``x``; ``dweight``, ``dbias`` (one value per column,
    any of the three types, e.g. a layer of a gradient arena).  Each may be None.  ``workspace``:
    layer_norm_workspace_bytes() bytes, needed for ``dweight`` or ``dbias``."""
    n, d = x.shape
    stream = _on_device(dy, x, weight, mean, rstd, dx, dweight, dbias, workspace)
    xs, gs = _rows(x, n, d, "x"), _rows(dy, n, d, "dy")
    ds = d if dx is None else _rows(dx, n, d, "dx")
    if dy.dtype != x.dtype or (dx is not None and dx.dtype != x.dtype):
        raise ValueError("dy and dx: %s is wanted" % x.dtype)
    grads = dbias if dweight is None else dweight
    f32 = _torch.f32
    code = lib().rsdgc_layer_norm_backward(
        dy.data_ptr(), gs, x.data_ptr(), xs, _vector(weight, d, None, "weight"), _vector(mean, n, f32, "mean"),
        _vector(rstd, n, f32, "rstd"), _ptr(dx), ds, _vector(dweight, d, None, "dweight"),
        _vector(dbias, d, None if grads is None else grads.dtype, "dbias"), RSDGC_F32 if grads is None else _dtype_code(grads),
        n, d, _dtype_code(x), _dtype_code(x if weight is None else weight),
        None if grads is None else _holds(workspace, layer_norm_workspace_bytes(n, d)), stream)
    if code:
        _check(code, "rsdgc_layer_norm_backward")


@functools.lru_cache(maxsize=4096)
def head_workspace_bytes(n_tokens: int, vocab: int, width: int, n_targets: int = 1) -> int:
    """Bytes of workspace (256-byte aligned) that the calls on a vocabulary head need; ``n_targets``: entries of the
    teacher per token (1 for labels)."""
    return _size(lib().rsdgc_head_workspace_bytes(n_tokens, vocab, width, n_targets), "rsdgc_head_workspace_bytes")


@functools.lru_cache(maxsize=4096)
def head_forward_workspace_bytes(n_tokens: int, vocab: int, width: int, n_targets: int = 1) -> int:
    """... that a forward call alone needs (scoring, evaluation)."""
    return _size(lib().rsdgc_head_forward_workspace_bytes(n_tokens, vocab, width, n_targets),
                 "rsdgc_head_forward_workspace_bytes")


def _head_args(hidden, weight, workspace, n_targets: int, size=head_workspace_bytes):
    """(n, v, d, hidden stride, weight stride, type, workspace's address) of a vocabulary head, after the checks that all
    its calls share."""
    n, d = hidden.shape
    v = weight.shape[0]
    if weight.dtype != hidden.dtype:
        raise ValueError("weight: %s is wanted, got %s" % (hidden.dtype, weight.dtype))
    hs, ws = _rows(hidden, n, d, "hidden"), _rows(weight, v, d, "weight")
    # the stride of a single row is free
    hs, ws = hs if n > 1 else (d + 7) // 8 * 8, ws if v > 1 else (d + 7) // 8 * 8
    return n, v, d, hs, ws, _dtype_code(hidden), _holds(workspace, size(n, v, d, n_targets))


def _head_grads(hidden, weight, dhidden, dweight):
    """(dhidden's stride, dweight's stride, dweight's type)"""
    if dhidden.dtype != hidden.dtype:
        raise ValueError("dhidden: %s is wanted, got %s" % (hidden.dtype, dhidden.dtype))
    n, d = hidden.shape
    return _rows(dhidden, n, d, "dhidden"), _rows(dweight, weight.shape[0], d, "dweight"), _dtype_code(dweight)


def _matrix(t, what: str) -> None:
    if t.dim() != 2:
        raise ValueError("%s: a matrix is wanted" % what)


def head_loss_forward(hidden, weight, labels, loss, lse, workspace) -> None:
    """``loss`` = cross entropy of the logits ``hidden`` @ ``weight``.T with ``labels`` (int64; negative: no loss), ``lse``
    = their log-sum-exp (None where no backward pass follows), both float32, without storing the logits.  bfloat16 or
    float16, rows 16-byte aligned."""
    _matrix(hidden, "hidden")
    stream = _on_device(hidden, weight, workspace, labels, loss, lse)
    n, v, d, hs, ws, code, space = _head_args(hidden, weight, workspace, 1, head_forward_workspace_bytes)
    f32 = _torch.f32
    if labels is None:
        raise ValueError("labels are wanted")
    code = lib().rsdgc_head_loss_forward(hidden.data_ptr(), hs, weight.data_ptr(), ws,
                                         _vector(labels, n, _torch.i64, "labels"), _vector(loss, n, f32, "loss"),
                                         _vector(lse, n, f32, "lse"), n, v, d, code, space, stream)
    if code:
        _check(code, "rsdgc_head_loss_forward")


def head_loss_backward(hidden, weight, labels, lse, grad_loss, dhidden, dweight, workspace) -> None:
    """Gradients of head_loss_forward() for ``grad_loss`` (float32, one per token): ``dhidden`` like ``hidden``, ``dweight``
    vocab x width in ``weight``'s type or float32, e.g. a layer of a gradient arena."""
    _matrix(hidden, "hidden")
    stream = _on_device(hidden, weight, workspace, labels, lse, grad_loss, dhidden, dweight)
    n, v, d, hs, ws, code, space = _head_args(hidden, weight, workspace, 1)
    dhs, dws, dwt = _head_grads(hidden, weight, dhidden, dweight)
    f32 = _torch.f32
    if labels is None:
        raise ValueError("labels are wanted")
    code = lib().rsdgc_head_loss_backward(hidden.data_ptr(), hs, weight.data_ptr(), ws,
                                          _vector(labels, n, _torch.i64, "labels"), _vector(lse, n, f32, "lse"),
                                          _vector(grad_loss, n, f32, "grad_loss"), dhidden.data_ptr(), dhs,
                                          dweight.data_ptr(), dws, dwt, n, v, d, code, space, stream)
    if code:
        _check(code, "rsdgc_head_loss_backward")


def _top_args(top_index, top_logit, n: int):
    """(entries per token, strides of the two, type of the logits)"""
    _matrix(top_index, "top_index")
    if top_index.dtype != _tt().i64:
        raise ValueError("top_index: int64 is wanted, got %s" % top_index.dtype)
    k = top_index.shape[1]
    return k, _rows(top_index, n, k, "top_index"), _rows(top_logit, n, k, "top_logit"), _dtype_code(top_logit)


def head_distill_forward(hidden, weight, top_index, top_logit, temperature: float, loss, lse, workspace) -> None:
    """``loss`` = T^2 KL(teacher || student) per token, the teacher being the softmax of its top logits ``top_logit`` at
    the vocabulary entries ``top_index`` (int64, negative: entry left out) and the student that of ``hidden`` @
    ``weight``.T, both at temperature T; ``lse`` = log-sum-exp of the student's logits / T."""
    _matrix(hidden, "hidden")
    stream = _on_device(hidden, weight, workspace, top_index, top_logit, loss, lse)
    k, istride, lstride, tcode = _top_args(top_index, top_logit, hidden.shape[0])
    n, v, d, hs, ws, code, space = _head_args(hidden, weight, workspace, k, head_forward_workspace_bytes)
    f32 = _torch.f32
    code = lib().rsdgc_head_distill_forward(hidden.data_ptr(), hs, weight.data_ptr(), ws, top_index.data_ptr(), istride,
                                            top_logit.data_ptr(), lstride, tcode, k, temperature,
                                            _vector(loss, n, f32, "loss"), _vector(lse, n, f32, "lse"), n, v, d, code, space,
                                            stream)
    if code:
        _check(code, "rsdgc_head_distill_forward")


def head_distill_backward(hidden, weight, top_index, top_logit, temperature: float, lse, grad_loss, dhidden, dweight,
                          workspace) -> None:
    """Gradients of head_distill_forward(), as head_loss_backward() gives them."""
    _matrix(hidden, "hidden")
    stream = _on_device(hidden, weight, workspace, top_index, top_logit, lse, grad_loss, dhidden, dweight)
    k, istride, lstride, tcode = _top_args(top_index, top_logit, hidden.shape[0])
    n, v, d, hs, ws, code, space = _head_args(hidden, weight, workspace, k)
    dhs, dws, dwt = _head_grads(hidden, weight, dhidden, dweight)
    f32 = _torch.f32
    code = lib().rsdgc_head_distill_backward(hidden.data_ptr(), hs, weight.data_ptr(), ws, top_index.data_ptr(), istride,
                                             top_logit.data_ptr(), lstride, tcode, k, temperature,
                                             _vector(lse, n, f32, "lse"), _vector(grad_loss, n, f32, "grad_loss"),
                                             dhidden.data_ptr(), dhs, dweight.data_ptr(), dws, dwt, n, v, d, code, space,
                                             stream)
    if code:
        _check(code, "rsdgc_head_distill_backward")


def operator_status() -> int:
    """Status bits raised by the operators since the last call (waits for the current stream, clears them)."""
    flags = C.c_uint32()
    _check(lib().rsdgc_operator_status(_stream(), C.byref(flags)), "rsdgc_operator_status")
    return flags.value


def selftest_operator_polls(polls: int = 0) -> None:
    """Operator calls made from now on give up a wait after ``polls`` polls (0: the library's own limit again)."""
    _check(lib().rsdgc_selftest_operator_polls(polls), "rsdgc_selftest_operator_polls")


def selftest_operator_wait(polls: int = 256) -> None:
    """A wait that runs out after ``polls`` polls on the current stream."""
    _check(lib().rsdgc_selftest_operator_wait(polls, _stream()), "rsdgc_selftest_operator_wait")


def launch_count() -> int:
    return int(lib().rsdgc_launch_count())
