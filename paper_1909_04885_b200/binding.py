"""ctypes binding over ``libchicle.so`` (the C ABI in ``include/chicle.h``), same names, argument marshalling only.

Every step of a round runs in the library's CUDA kernels. PyTorch is used for device memory (the library's
allocations are routed through torch's caching allocator) and for the stream. There is no host fallback: if the
shared library is missing, loading fails with an error.
"""
from __future__ import annotations

import array
import ctypes as C
import functools
import os
import threading
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("CHICLE_LIB_PATH") or os.path.join(_HERE, "libchicle.so")

OK, ERR_INVALID_ARG, ERR_BAD_STATE, ERR_OOM, ERR_CUDA, ERR_UNSUPPORTED, ERR_NUMERIC, ERR_TIMEOUT, ERR_INTERNAL = range(9)
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "BAD_STATE", 3: "OOM", 4: "CUDA", 5: "UNSUPPORTED", 6: "NUMERIC", 7: "TIMEOUT",
                8: "INTERNAL"}
LOSS = {"hinge": 0, "logistic": 1, "ridge": 2}
FMT = {"dense": 0, "csr": 1, "csc": 2}
MEM_HOST, MEM_DEVICE = 0, 1

EXPORTED = ["chicle_glm_create", "chicle_partition", "chicle_cocoa_round", "chicle_duality_gap", "chicle_get_alpha",
            "chicle_get_v", "chicle_get_partition", "chicle_get_permutation", "chicle_set_state", "chicle_get_info",
            "chicle_last_error", "chicle_glm_destroy", "chicle_partition_noalloc", "chicle_partition_sizes",
            "chicle_cocoa_round_steps", "chicle_chunks_cut", "chicle_chunks_assign", "chicle_chunks_scale_in",
            "chicle_chunks_scale_out", "chicle_chunks_rebalance_step", "chicle_partition_chunks", "chicle_cocoa_round_delta",
            "chicle_apply_deltas", "chicle_export_state_of", "chicle_import_state", "chicle_softmax_workspace",
            "chicle_softmax_loss", "chicle_softmax_loss_grad", "chicle_embedding", "chicle_embedding_grad_workspace",
            "chicle_embedding_grad", "chicle_clip_gradients"]


class ChicleError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("chicle: %s: %s" % (STATUS_NAMES.get(status, status), message))
        self.status = status


class Matrix(C.Structure):
    _fields_ = [("fmt", C.c_int), ("space", C.c_int), ("n_rows", C.c_int64), ("n_cols", C.c_int64), ("nnz", C.c_int64),
                ("ld", C.c_int64), ("indptr", C.c_void_p), ("indices", C.c_void_p), ("values", C.c_void_p)]


class Dense(C.Structure):
    _fields_ = [("type", C.c_int), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("data", C.c_void_p)]


ALLOC_FN = C.CFUNCTYPE(C.c_void_p, C.c_void_p, C.c_size_t)
FREE_FN = C.CFUNCTYPE(None, C.c_void_p, C.c_void_p)


class Allocator(C.Structure):
    _fields_ = [("alloc", ALLOC_FN), ("free", FREE_FN), ("ctx", C.c_void_p)]


class RoundStats(C.Structure):
    _fields_ = [("ms_permutation", C.c_float), ("ms_local", C.c_float), ("ms_reduce", C.c_float), ("ms_total", C.c_float),
                ("steps", C.c_int64), ("solver_variant", C.c_int32), ("ms_prepare", C.c_float),
                ("solver_slices", C.c_int32), ("cluster_ctas", C.c_int32), ("solver_launches", C.c_int32),
                ("order_launches", C.c_int32)]


_lib = None


def load():
    """Loads the shared library; raises if it has not been built (``python -m paper_1909_04885_b200.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libchicle.so is missing (%s): build it with `python -m paper_1909_04885_b200.build`; "
                           "there is no CPU path" % LIB_PATH)
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, u64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_float
    lib.chicle_glm_create.restype = C.c_int
    lib.chicle_glm_create.argtypes = [C.POINTER(Matrix), vp, f32, C.c_int, C.c_int, vp, C.POINTER(Allocator), C.POINTER(vp)]
    lib.chicle_partition.restype = C.c_int
    lib.chicle_partition.argtypes = [vp, i32, u64]
    lib.chicle_partition_sizes.restype = C.c_int
    lib.chicle_partition_sizes.argtypes = [vp, i32, u64, vp]
    lib.chicle_cocoa_round.restype = C.c_int
    lib.chicle_cocoa_round.argtypes = [vp, i64, f32, C.POINTER(RoundStats)]
    lib.chicle_cocoa_round_steps.restype = C.c_int
    lib.chicle_cocoa_round_steps.argtypes = [vp, vp, f32, C.POINTER(RoundStats)]
    lib.chicle_cocoa_round_delta.restype = C.c_int
    lib.chicle_cocoa_round_delta.argtypes = [vp, vp, f32, vp, i64, C.POINTER(RoundStats)]
    lib.chicle_apply_deltas.restype = C.c_int
    lib.chicle_apply_deltas.argtypes = [vp, vp, i32, i64]
    lib.chicle_export_state_of.restype = C.c_int
    lib.chicle_export_state_of.argtypes = [vp, vp, vp, i64]
    lib.chicle_import_state.restype = C.c_int
    lib.chicle_import_state.argtypes = [vp, vp, i64]
    lib.chicle_chunks_cut.restype = i64
    lib.chicle_chunks_cut.argtypes = [i64, vp, i64, i64, vp]
    lib.chicle_chunks_assign.restype = C.c_int
    lib.chicle_chunks_assign.argtypes = [i64, i32, C.c_uint64, vp]
    lib.chicle_chunks_scale_in.restype = C.c_int
    lib.chicle_chunks_scale_in.argtypes = [i64, i32, i32, vp]
    lib.chicle_chunks_scale_out.restype = C.c_int
    lib.chicle_chunks_scale_out.argtypes = [i64, i32, i32, C.c_uint64, vp]
    lib.chicle_chunks_rebalance_step.restype = C.c_int
    lib.chicle_chunks_rebalance_step.argtypes = [i64, vp, i32, vp, vp]
    lib.chicle_partition_chunks.restype = C.c_int
    lib.chicle_partition_chunks.argtypes = [vp, i32, C.c_uint64, i64, vp, vp]
    lib.chicle_duality_gap.restype = C.c_int
    lib.chicle_duality_gap.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(C.c_double)]
    for name in ("chicle_get_alpha", "chicle_get_v"):
        fn = getattr(lib, name)
        fn.restype = C.c_int
        fn.argtypes = [vp, vp, i64, C.c_int]
    lib.chicle_get_partition.restype = C.c_int
    lib.chicle_get_partition.argtypes = [vp, vp, i64]
    lib.chicle_get_permutation.restype = C.c_int
    lib.chicle_get_permutation.argtypes = [vp, i64, i32, vp, i64]
    lib.chicle_set_state.restype = C.c_int
    lib.chicle_set_state.argtypes = [vp, vp, vp, i64]
    lib.chicle_get_info.restype = C.c_int
    lib.chicle_get_info.argtypes = [vp, C.POINTER(i64), C.POINTER(i32), C.POINTER(i64), C.POINTER(i64)]
    lib.chicle_last_error.restype = C.c_char_p
    lib.chicle_last_error.argtypes = [vp]
    lib.chicle_glm_destroy.restype = None
    lib.chicle_glm_destroy.argtypes = [vp]
    lib.chicle_partition_noalloc.restype = C.c_int
    lib.chicle_partition_noalloc.argtypes = [C.c_int, vp, i64, i32, u64, vp, vp, C.c_char_p, C.c_size_t]
    dp, sz = C.POINTER(Dense), C.c_size_t
    tail = [vp, sz, vp, C.c_char_p, sz]  # workspace, its bytes, status word, error text, its bytes
    for name, args in (("chicle_softmax_workspace", [dp, dp, C.c_int, C.POINTER(sz)]),
                       ("chicle_softmax_loss", [C.c_int, vp, dp, dp, vp, vp, vp] + tail),
                       ("chicle_softmax_loss_grad", [C.c_int, vp, dp, dp, vp, vp, f32, vp, vp, dp, dp] + tail),
                       ("chicle_embedding", [C.c_int, vp, dp, vp, f32, dp, vp, C.c_char_p, sz]),
                       ("chicle_embedding_grad_workspace", [i64, i64, i64, C.POINTER(sz)]),
                       ("chicle_embedding_grad", [C.c_int, vp, vp, dp, f32, C.c_int, dp] + tail),
                       ("chicle_clip_gradients", [C.c_int, vp, i64, vp, f32, vp, vp, sz, C.c_char_p, sz])):
        fn = getattr(lib, name)
        fn.restype = C.c_int
        fn.argtypes = args
    _lib = lib
    return lib


def _stats_dict(rs) -> dict:
    return {"ms_permutation": rs.ms_permutation, "ms_local": rs.ms_local, "ms_reduce": rs.ms_reduce,
            "ms_total": rs.ms_total, "steps": rs.steps, "solver_variant": rs.solver_variant,
            "ms_prepare": rs.ms_prepare, "solver_slices": rs.solver_slices, "cluster_ctas": rs.cluster_ctas,
            "solver_launches": rs.solver_launches, "order_launches": rs.order_launches}


def _is_torch(x) -> bool:
    return x is not None and type(x).__module__.startswith("torch")


def _ptr(x):
    if x is None:
        return None
    if _is_torch(x):
        return C.c_void_p(x.data_ptr())
    return x.ctypes.data_as(C.c_void_p)


class _TorchAllocator:
    """Routes the library's device allocations through torch's caching allocator."""

    def __init__(self, device: int):
        import torch
        self._torch = torch
        self._device = torch.device("cuda", device)
        self._live = {}
        self.fail = False   # True: every request is refused (the callback returns NULL), to exercise the library's OOM paths
        self._alloc_cb = ALLOC_FN(self._alloc)
        self._free_cb = FREE_FN(self._free)
        self.struct = Allocator(self._alloc_cb, self._free_cb, None)

    def _alloc(self, _ctx, nbytes):
        if self.fail:
            return None
        try:
            t = self._torch.empty(int(nbytes), dtype=self._torch.uint8, device=self._device)
        except Exception:
            return None
        self._live[t.data_ptr()] = t
        return t.data_ptr()

    def _free(self, _ctx, ptr):
        self._live.pop(ptr, None)

    @property
    def bytes_live(self) -> int:
        return sum(t.numel() for t in self._live.values())


class Glm:
    """One training problem on one GPU. ``values``/``indptr``/``indices``/``labels`` are numpy arrays (host) or
    torch CUDA tensors (device), all in the same place. fp32 values and labels, int64 indptr, int32 indices."""

    def __init__(self, loss: str, fmt: str, n_rows: int, n_cols: int, values, labels, lam: float, indptr=None,
                 indices=None, device: int = 0, stream: Optional[int] = None, torch_allocator: bool = True,
                 ld: Optional[int] = None):
        self._lib = load()
        self._h = C.c_void_p(None)
        on_dev = _is_torch(values)
        if on_dev:
            import torch
            assert values.is_cuda and values.dtype == torch.float32 and values.is_contiguous()
            assert labels.is_cuda and labels.dtype == torch.float32
            if indptr is not None:
                assert indptr.dtype == torch.int64 and indices.dtype == torch.int32
            nvals = values.numel()
        else:
            values = np.ascontiguousarray(values, np.float32).reshape(-1)
            labels = np.ascontiguousarray(labels, np.float32)
            indptr = None if indptr is None else np.ascontiguousarray(indptr, np.int64)
            indices = None if indices is None else np.ascontiguousarray(indices, np.int32)
            nvals = values.size
        self._keep = (values, labels, indptr, indices)
        m = Matrix(FMT[fmt], MEM_DEVICE if on_dev else MEM_HOST, n_rows, n_cols, 0 if fmt == "dense" else nvals,
                   (ld or n_cols) if fmt == "dense" else 0, _ptr(indptr), _ptr(indices), _ptr(values))
        self._alloc = None
        alloc_ref = None
        if torch_allocator:
            self._alloc = _TorchAllocator(device)
            alloc_ref = C.byref(self._alloc.struct)
        if stream is None:
            import torch
            with torch.cuda.device(device):
                stream = torch.cuda.current_stream().cuda_stream
        self.stream = stream
        self.device = device
        self.loss, self.fmt = loss, fmt
        st = self._lib.chicle_glm_create(C.byref(m), _ptr(labels), C.c_float(lam), LOSS[loss], device,
                                         C.c_void_p(stream), alloc_ref, C.byref(self._h))
        if st != OK:
            raise ChicleError(st, self._lib.chicle_last_error(None).decode())
        self._keep = None
        self.n_coord = n_cols if loss == "ridge" else n_rows
        self.dim = n_rows if loss == "ridge" else n_cols
        self.K = 0

    # -- helpers
    def _check(self, st: int):
        if st != OK:
            raise ChicleError(st, self._lib.chicle_last_error(self._h).decode())

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.chicle_glm_destroy(self._h)
            self._h = C.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -- the ABI, one method per entry point
    def partition(self, K: int, seed: int, sizes=None):
        """``chicle_partition``, or ``chicle_partition_sizes`` when ``sizes`` (K positive integers summing to the number
        of coordinates) is given."""
        if sizes is None:
            self._check(self._lib.chicle_partition(self._h, K, C.c_uint64(seed & (2**64 - 1))))
        else:
            sz = np.ascontiguousarray(sizes, np.int64)
            if sz.size != K:
                raise ValueError("sizes must have K entries")
            self._check(self._lib.chicle_partition_sizes(self._h, K, C.c_uint64(seed & (2**64 - 1)), _ptr(sz)))
        self.K = K

    def partition_chunks(self, K: int, seed: int, chunk_off, chunk_task):
        """``chicle_partition_chunks``: the partition that a placement of data chunks on K tasks induces."""
        off = np.ascontiguousarray(chunk_off, np.int64)
        task = np.ascontiguousarray(chunk_task, np.int32)
        if off.size != task.size + 1:
            raise ValueError("chunk_off must have one entry more than chunk_task")
        self._check(self._lib.chicle_partition_chunks(self._h, K, C.c_uint64(seed & (2**64 - 1)), task.size, _ptr(off), _ptr(task)))
        self.K = K

    def cocoa_round(self, H: int = 0, sigma_prime: Optional[float] = None, stats: bool = False, steps=None):
        """One round; ``steps`` (K integers, 0 <= steps[k] <= size of partition k) gives each partition its own budget."""
        sp = float(self.K if sigma_prime is None else sigma_prime)
        rs = RoundStats() if stats else None
        ref = C.byref(rs) if stats else None
        if steps is not None:
            st = np.ascontiguousarray(steps, np.int64)
            if st.size != self.K:
                raise ValueError("steps must have K entries")
            self._check(self._lib.chicle_cocoa_round_steps(self._h, st.ctypes.data, C.c_float(sp), ref))
        else:
            self._check(self._lib.chicle_cocoa_round(self._h, H, C.c_float(sp), ref))
        return _stats_dict(rs) if stats else None

    def cocoa_round_delta(self, steps, sigma_prime: float, delta_out, stats: bool = False):
        """``chicle_cocoa_round_delta``: the round with budgets ``steps``; the summed update goes to ``delta_out`` (a
        CUDA tensor of ``dim`` floats on this handle's device) and v is left alone."""
        st = np.ascontiguousarray(steps, np.int64)
        if st.size != self.K:
            raise ValueError("steps must have K entries")
        rs = RoundStats() if stats else None
        self._check(self._lib.chicle_cocoa_round_delta(self._h, st.ctypes.data, C.c_float(float(sigma_prime)), _ptr(delta_out),
                                                       delta_out.numel(), C.byref(rs) if stats else None))
        return _stats_dict(rs) if stats else None

    def apply_deltas(self, deltas):
        """``chicle_apply_deltas``: ``deltas`` is a contiguous CUDA tensor of shape (count, dim)."""
        count = deltas.numel() // self.dim
        self._check(self._lib.chicle_apply_deltas(self._h, _ptr(deltas), count, self.dim))

    def export_state_of(self, keep, out):
        """``chicle_export_state_of``: ``keep`` holds K flags, ``out`` is a CUDA tensor of one float per coordinate."""
        kp = np.ascontiguousarray(keep, np.uint8)
        if kp.size != self.K:
            raise ValueError("keep must have K entries")
        self._check(self._lib.chicle_export_state_of(self._h, kp.ctypes.data, _ptr(out), out.numel()))

    def import_state(self, state):
        """``chicle_import_state``: ``state`` is a CUDA tensor of one float per coordinate."""
        self._check(self._lib.chicle_import_state(self._h, _ptr(state), state.numel()))

    def fail_allocations(self, on: bool):
        """Makes the allocator callback that the library was given refuse every request (return NULL) from now on, or
        serve them again: a way to see the library's out-of-memory behaviour without exhausting the device."""
        if self._alloc is None:
            raise RuntimeError("this handle allocates with cudaMalloc, not through a callback")
        self._alloc.fail = bool(on)

    def duality_gap(self):
        g, p, d = C.c_double(), C.c_double(), C.c_double()
        self._check(self._lib.chicle_duality_gap(self._h, C.byref(g), C.byref(p), C.byref(d)))
        return {"gap": g.value, "primal": p.value, "dual": d.value}

    def get_alpha(self, out=None) -> np.ndarray:
        return self._get(self._lib.chicle_get_alpha, self.n_coord, out)

    def get_v(self, out=None) -> np.ndarray:
        return self._get(self._lib.chicle_get_v, self.dim, out)

    def _get(self, fn, n, out):
        if out is None:
            out = np.empty(n, np.float32)
        space = MEM_DEVICE if _is_torch(out) else MEM_HOST
        self._check(fn(self._h, _ptr(out), n, space))
        return out

    def get_partition(self) -> np.ndarray:
        out = np.empty(self.n_coord, np.int32)
        self._check(self._lib.chicle_get_partition(self._h, _ptr(out), out.size))
        return out

    def get_permutation(self, rnd: int, k: int, n_k: int) -> np.ndarray:
        out = np.empty(n_k, np.int32)
        self._check(self._lib.chicle_get_permutation(self._h, rnd, k, _ptr(out), n_k))
        return out

    def set_state(self, alpha: np.ndarray, v: Optional[np.ndarray], rnd: int):
        alpha = np.ascontiguousarray(alpha, np.float32)
        v = None if v is None else np.ascontiguousarray(v, np.float32)
        assert alpha.size == self.n_coord and (v is None or v.size == self.dim)
        self._check(self._lib.chicle_set_state(self._h, _ptr(alpha), _ptr(v), rnd))

    def info(self):
        r, K, n, d = C.c_int64(), C.c_int32(), C.c_int64(), C.c_int64()
        self._check(self._lib.chicle_get_info(self._h, C.byref(r), C.byref(K), C.byref(n), C.byref(d)))
        return {"round": r.value, "K": K.value, "n_coord": n.value, "dim": d.value}


def from_workload(w, device: int = 0, on_device: bool = False, **kw) -> Glm:
    """Builds a ``Glm`` from a ``datagen.Workload`` (host arrays by default; ``on_device`` uploads them with torch
    first so that creation copies device to device)."""
    vals, labels, indptr, indices = w.values, w.labels, w.indptr, w.indices
    if on_device:
        import torch
        dev = torch.device("cuda", device)
        vals = torch.from_numpy(vals).to(dev)
        labels = torch.from_numpy(labels).to(dev)
        indptr = None if indptr is None else torch.from_numpy(indptr).to(dev)
        indices = None if indices is None else torch.from_numpy(indices).to(dev)
    return Glm(w.loss, w.fmt, w.n_rows, w.n_cols, vals, labels, w.lam, indptr, indices, device=device, **kw)


def partition_noalloc(n_coord: int, K: int, seed: int, owner_out, members_out, device: int = 0, stream: int = 0):
    """``chicle_partition_noalloc``: fills two caller-owned int32 CUDA tensors of ``n_coord`` entries with the partition
    map and the grouped member list, using the library's built-in workspace instead of allocating one. Meant for
    callers that may not touch a device allocator at this point (frozen memory pools, serving loops). Asynchronous on
    ``stream``; raises ``ChicleError`` with the library's message when the size is beyond the built-in limit."""
    lib = load()
    buf = C.create_string_buffer(256)
    st = lib.chicle_partition_noalloc(device, C.c_void_p(stream), n_coord, K, C.c_uint64(seed & (2**64 - 1)),
                                      C.c_void_p(owner_out.data_ptr()), C.c_void_p(members_out.data_ptr()), buf, 256)
    if st != OK:
        raise ChicleError(st, buf.value.decode())


# ---- mobile data chunks: host-side placement logic of the library (argument marshalling only) -------------------
def chunks_cut(n_coord: int, chunk_bytes: int, indptr=None, dense_dim: int = 0) -> np.ndarray:
    """``chicle_chunks_cut``: chunk offsets for chunks of at most ``chunk_bytes``."""
    off = np.empty(n_coord + 1, np.int64)
    ip = None if indptr is None else np.ascontiguousarray(indptr, np.int64)
    c = load().chicle_chunks_cut(n_coord, None if ip is None else _ptr(ip), dense_dim, chunk_bytes, _ptr(off))
    if c < 0:
        raise ValueError("chicle_chunks_cut: bad arguments")
    return off[:c + 1].copy()


def chunks_assign(n_chunks: int, K: int, seed: int) -> np.ndarray:
    task = np.empty(n_chunks, np.int32)
    st = load().chicle_chunks_assign(n_chunks, K, C.c_uint64(seed & (2**64 - 1)), _ptr(task))
    if st != OK:
        raise ChicleError(st, "chicle_chunks_assign: need 1 <= K <= number of chunks")
    return task


def chunks_scale_in(task, K_old: int, K_new: int) -> np.ndarray:
    out = np.array(task, np.int32, copy=True)
    st = load().chicle_chunks_scale_in(out.size, K_old, K_new, _ptr(out))
    if st != OK:
        raise ChicleError(st, "chicle_chunks_scale_in: need 1 <= K_new <= K_old")
    return out


def chunks_scale_out(task, K_old: int, K_new: int, seed: int) -> np.ndarray:
    out = np.array(task, np.int32, copy=True)
    st = load().chicle_chunks_scale_out(out.size, K_old, K_new, C.c_uint64(seed & (2**64 - 1)), _ptr(out))
    if st != OK:
        raise ChicleError(st, "chicle_chunks_scale_out: need 1 <= K_old <= K_new and tasks in [0, K_old)")
    return out


def chunks_rebalance_step(task, chunk_off, K: int, time_per_sample):
    """Returns (new placement, whether a chunk moved)."""
    out = np.array(task, np.int32, copy=True)
    off = np.ascontiguousarray(chunk_off, np.int64)
    t = np.ascontiguousarray(time_per_sample, np.float64)
    if off.size != out.size + 1 or t.size != K:
        raise ValueError("chunk_off needs one entry more than task, time_per_sample K entries")
    r = load().chicle_chunks_rebalance_step(out.size, _ptr(off), K, _ptr(t), _ptr(out))
    if r < 0:
        raise ValueError("chicle_chunks_rebalance_step: bad arguments")
    return out, bool(r)


# ---- operators of a softmax model with a vector per id ------------------------------------------------------------
# CUDA tensors in, CUDA tensors out; the work is enqueued on torch's current stream of the tensors' device, or on `stream`
# (a cudaStream_t), and outputs and workspaces come from torch's caching allocator for that stream. Nothing is kept between
# calls, no call synchronises, all can be captured into a CUDA graph. No autograd graph is recorded. `status`: an optional
# int32 CUDA tensor of one element whose bits the kernels set (STATUS_BAD_ID: a label or id beyond the last class or row,
# taken as none; STATUS_TIMEOUT: the results are not valid, and what is concerned of them is NaN with or without a status). What is
# written in place (out, the clipped tensors) is written behind autograd's back: version counters stay as they are. With `stream`, the
# inputs are the caller's to keep until the work is done: they are not recorded for that stream with the allocator.
STATUS_BAD_ID, STATUS_TIMEOUT = 4, 8
CLIP_WORKSPACE = 16384
_ERR_LEN = 256
_local = threading.local()  # the error text's buffer, one per thread
_dtypes = None


def _types():
    global _dtypes
    if _dtypes is None:
        import torch
        _dtypes = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    return _dtypes


def _errbuf():
    try:
        return _local.buf
    except AttributeError:
        _local.buf = C.create_string_buffer(_ERR_LEN)
        return _local.buf


def _dense(t, what: str) -> Dense:
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor of two dimensions" % what)
    ty = _types().get(t.dtype)
    if ty is None:
        raise ValueError("%s must be float32, bfloat16 or float16" % what)
    rows, cols = t.shape
    ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError("the rows of %s must be contiguous" % what)
    return Dense(ty, rows, cols, ld if rows > 1 else cols, t.data_ptr())


def _vector(t, n: int, dtype, device: int, what: str) -> int:
    if t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous() or t.get_device() != device:
        raise ValueError("%s must be a contiguous %s tensor of %d elements on the same device" % (what, str(dtype)[6:], n))
    return t.data_ptr()


def _status_ptr(status, device: int):
    if status is None:
        return None
    import torch
    if status.dtype != torch.int32 or status.numel() != 1 or status.get_device() != device:
        raise ValueError("status must be an int32 tensor of one element on the same device")
    return status.data_ptr()


def _operator(fn):
    """Adds the keyword ``stream`` to an operator: the caller's stream is torch's current one while outputs and workspaces
    are allocated and the work is enqueued."""
    name = fn.__code__.co_varnames[0]  # the first argument, which may be given by its name

    @functools.wraps(fn)
    def call(*args, stream: Optional[int] = None, **kw):
        if stream is None or (not args and name not in kw):
            return fn(*args, **kw)
        import torch
        first = args[0] if args else kw[name]
        if not isinstance(first, torch.Tensor):  # several: an iterator is used up here
            several = list(first)
            if args:
                args = (several,) + args[1:]
            else:
                kw[name] = several
            if not several:
                return fn(*args, **kw)
            first = several[0]
        with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=first.device)):
            return fn(*args, **kw)
    return call


def _raw_stream(device: int) -> int:
    import torch
    try:
        return torch._C._cuda_getCurrentRawStream(device)  # (the public form builds a Stream object: 1.4 us)
    except AttributeError:
        return torch.cuda.current_stream(device).cuda_stream


def _workspace(nbytes: int, like):
    import torch
    return torch.empty(nbytes, dtype=torch.uint8, device=like.device) if nbytes else None


def _raise(st: int, buf):
    if st != OK:
        raise ChicleError(st, buf.value.decode())


@functools.lru_cache(maxsize=1024)
def _softmax_bytes(x: tuple, w: tuple, grad: bool) -> int:
    """``chicle_softmax_workspace`` for two (type, rows, cols, ld, address mod 16): a function of these alone."""
    need = C.c_size_t()
    if load().chicle_softmax_workspace(C.byref(Dense(*x[:4], x[4] or 16)), C.byref(Dense(*w[:4], w[4] or 16)), int(grad), C.byref(need)) != OK:
        raise ChicleError(ERR_INVALID_ARG, "x and w must have one type and the same columns, w at least one row")
    return need.value


@functools.lru_cache(maxsize=1024)
def _embedding_grad_bytes(n: int, rows: int, cols: int) -> int:
    need = C.c_size_t()
    if load().chicle_embedding_grad_workspace(n, rows, cols, C.byref(need)) != OK:
        raise ChicleError(ERR_INVALID_ARG, "sizes out of range")
    return need.value


def _softmax(x, w, labels, grad: bool, weights=None, scale=1.0, status=None):
    import torch
    lib = load()
    dx, dw = _dense(x, "x"), _dense(w, "w")
    device = x.get_device()
    if w.get_device() != device:
        raise ValueError("x and w must be on one device")
    n = dx.rows
    lp = _vector(labels, n, torch.int32, device, "labels")
    wp = None if weights is None else _vector(weights, n, torch.float32, device, "weights")
    sp = _status_ptr(status, device)
    need = _softmax_bytes((dx.type, n, dx.cols, dx.ld, (dx.data or 0) % 16), (dw.type, dw.rows, dw.cols, dw.ld, (dw.data or 0) % 16), grad)
    ws = _workspace(need, x)
    loss, lse = torch.empty((2, n), dtype=torch.float32, device=x.device).unbind(0)
    buf = _errbuf()
    stream, wsp = _raw_stream(device), None if ws is None else ws.data_ptr()
    if not grad:
        _raise(lib.chicle_softmax_loss(device, stream, C.byref(dx), C.byref(dw), lp, loss.data_ptr(), lse.data_ptr(), wsp,
                                       need, sp, buf, _ERR_LEN), buf)
        return loss, lse
    gx, gw = x.new_empty(x.shape), w.new_empty(w.shape)
    _raise(lib.chicle_softmax_loss_grad(device, stream, C.byref(dx), C.byref(dw), lp, wp, scale, loss.data_ptr(), lse.data_ptr(),
                                        C.byref(Dense(dx.type, n, dx.cols, dx.cols, gx.data_ptr())),
                                        C.byref(Dense(dw.type, dw.rows, dw.cols, dw.cols, gw.data_ptr())), wsp, need, sp, buf,
                                        _ERR_LEN), buf)
    return loss, lse, gx, gw


@_operator
def softmax_loss(x, w, labels, status=None):
    """``chicle_softmax_loss``: softmax cross entropy of the linear map ``x @ w.T`` (x: n x d, w: classes x d, one type of
    float32, bfloat16, float16) against int32 ``labels`` (negative: none). Returns (loss, lse), n float32 each; both are 0
    for rows without a label. The logits are not kept."""
    return _softmax(x, w, labels, False, status=status)


@_operator
def softmax_loss_grad(x, w, labels, weights=None, scale: float = 1.0, status=None):
    """``chicle_softmax_loss_grad``: also the gradients of ``scale * sum(weights * loss)`` with respect to x and w, in their
    types. Returns (loss, lse, dx, dw). ``weights``: n float32, or None for 1."""
    return _softmax(x, w, labels, True, weights, scale, status)


@_operator
def embedding(table, ids, scale: float = 1.0, out=None, status=None):
    """``chicle_embedding``: ``scale * table[ids]`` for int32 ids (one dimension), rows of zeros for negative ids."""
    import torch
    lib = load()
    dt = _dense(table, "table")
    device = table.get_device()
    n = ids.shape[0]
    ip = _vector(ids, n, torch.int32, device, "ids")
    if out is None:
        out = torch.empty((n, dt.cols), dtype=table.dtype, device=table.device)
        do = Dense(dt.type, n, dt.cols, dt.cols, out.data_ptr())
    elif out.get_device() != device or out.shape[0] != n:
        raise ValueError("out must have a row per id and be on the table's device")
    else:
        do = _dense(out, "out")
    buf = _errbuf()
    _raise(lib.chicle_embedding(device, _raw_stream(device), C.byref(dt), ip, scale, C.byref(do), _status_ptr(status, device), buf, _ERR_LEN), buf)
    return out


@_operator
def embedding_grad(ids, grad, rows: int, scale: float = 1.0, out=None, accumulate: bool = False, status=None):
    """``chicle_embedding_grad``: ``scale *`` the sum of the rows of ``grad`` (n x d) by id, as a table of ``rows`` rows;
    negative ids are left out. ``accumulate``: added to ``out``, whose other rows are left as they are."""
    import torch
    lib = load()
    dg = _dense(grad, "grad")
    device = grad.get_device()
    ip = _vector(ids, dg.rows, torch.int32, device, "ids")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty((rows, dg.cols), dtype=grad.dtype, device=grad.device)
    elif out.get_device() != device or out.shape[0] != rows:
        raise ValueError("out must have `rows` rows and be on the gradient's device")
    dt = _dense(out, "out")
    need = _embedding_grad_bytes(dg.rows, rows, dg.cols)
    ws = _workspace(need, grad)
    buf = _errbuf()
    _raise(lib.chicle_embedding_grad(device, _raw_stream(device), ip, C.byref(dg), scale, int(bool(accumulate)), C.byref(dt),
                                     None if ws is None else ws.data_ptr(), need, _status_ptr(status, device), buf, _ERR_LEN), buf)
    return out


@_operator
def clip_gradients(tensors, max_norm: float, out=None):
    """``chicle_clip_gradients``: returns the 2-norm of all elements of all ``tensors`` (a float32 tensor without dimensions)
    and multiplies them by ``min(1, max_norm / (norm + 1e-6))``, in place or into the tensors of ``out`` (as many, of the same
    types and lengths). A norm that is not finite leaves the elements as they are. ``max_norm=inf``: the norm alone."""
    import torch
    lib = load()
    tensors = list(tensors)
    if not tensors:
        raise ValueError("no tensors")
    # (method by method over all tensors: a model has hundreds, and each look costs what a launch of a kernel does not)
    T = torch.Tensor
    device, count = tensors[0].get_device(), len(tensors)
    dtypes = [t.dtype for t in tensors]
    kinds = list(map(_types().get, dtypes))
    lens, ins = list(map(T.numel, tensors)), list(map(T.data_ptr, tensors))
    # (a tensor on the host has device -1)
    good = device >= 0 and None not in kinds and all(map(T.is_contiguous, tensors)) and set(map(T.get_device, tensors)) == {device}
    outs = ins
    if out is not None:
        out = list(out)
        outs = list(map(T.data_ptr, out))
        good = (good and lens == list(map(T.numel, out)) and dtypes == [t.dtype for t in out] and all(map(T.is_contiguous, out))
                and set(map(T.get_device, out)) == {device})
    if not good:
        raise ValueError("the tensors must be contiguous CUDA tensors of float32, bfloat16 or float16 on one device, and those of "
                         "out of the same number, types and lengths")
    table = array.array("q", bytes(32 * count))  # chicle_tensor_t: four words
    for k, column in enumerate((kinds, lens, ins, outs)):
        table[k::4] = array.array("q", column)
    ws = torch.empty(CLIP_WORKSPACE, dtype=torch.uint8, device=tensors[0].device)
    norm = torch.empty((), dtype=torch.float32, device=tensors[0].device)
    buf = _errbuf()
    _raise(lib.chicle_clip_gradients(device, _raw_stream(device), count, table.buffer_info()[0], max_norm, norm.data_ptr(),
                                     ws.data_ptr(), CLIP_WORKSPACE, buf, _ERR_LEN), buf)
    return norm
