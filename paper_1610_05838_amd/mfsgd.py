"""Thin ctypes binding of ``libmfsgd.so`` (C ABI in ``include/mfsgd.h``).

Argument marshalling only: every step of the computation runs in the HIP
kernels of the library.  Device arrays are torch tensors on the current GPU;
streams are torch streams (default: ``torch.cuda.current_stream()``).

Samples are int32 tensors of shape (nnz, 3) whose columns hold u, v and the
bit pattern of the float32 rating r -- exactly the packed 12-byte records the
library reads.  ``samples_to_device`` builds one from a numpy structured array.

The library is loaded on first use.  If it has not been built the binding
raises ``ImportError``: there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

import numpy as np
import torch  # loads the HIP runtime that the library then shares (same SONAME)

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmfsgd.so")

OK, EINVAL, ENOMEM, EHIP, ESTATE, ETIMEOUT, ENUMERIC = 0, -1, -2, -3, -4, -5, -6
BATCH_HOGWILD, WAVEFRONT, WAVEFRONT_DET, GLOBAL_TABLE = 0, 1, 2, 3
FP32, FP16, BF16 = 0, 1, 2  # BF16: the operators alone
P, Q = 0, 1
ACTS = {"none": 0, "relu": 1, "sigmoid": 2, "silu": 3, "gelu": 4}
DBG_VISITS, DBG_TRACE, DBG_PLAN_STARTS, DBG_PLAN_ORDER, DBG_TEAM_MAP, DBG_TEAM_SIZES = 1, 2, 3, 4, 5, 6
DBG_TABLE_STARTS, DBG_TABLE_ORDER, DBG_PRIORITY = 7, 8, 9

SCHEMES = {"hogwild": BATCH_HOGWILD, "wavefront": WAVEFRONT, "wavefront_det": WAVEFRONT_DET,
           "table": GLOBAL_TABLE}

SAMPLE_DTYPE = np.dtype([("u", "<i4"), ("v", "<i4"), ("r", "<f4")])


class MfsgdError(RuntimeError):
    def __init__(self, code: int, fn: str, msg: str):
        super().__init__(f"{fn} failed with status {code}: {msg}")
        self.code = code


_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                              "(hipcc for gfx950); there is no CPU fallback")
        L = C.CDLL(LIB_PATH)
        i32, i64, u64, f32, vp = C.c_int32, C.c_int64, C.c_uint64, C.c_float, C.c_void_p
        sig = {
            "mfsgd_set_option": ([C.c_char_p, i64], C.c_int),
            "mfsgd_get_option": ([C.c_char_p, C.POINTER(i64)], C.c_int),
            "mfsgd_reset_options": ([], C.c_int),
            "mfsgd_init": ([i64, i64, i32, u64], C.c_int),
            "mfsgd_plan": ([vp, i64, i32, vp], C.c_int),
            "mfsgd_epoch": ([vp, i64, f32, f32, f32, i32, vp], C.c_int),
            "mfsgd_epoch_staged": ([vp, i64, f32, f32, f32, vp], C.c_int),
            "mfsgd_rmse": ([vp, i64, C.POINTER(C.c_double), vp], C.c_int),
            "mfsgd_rmse_noalloc": ([vp, i64, vp, vp], C.c_int),
            "mfsgd_check_samples": ([vp, i64, vp], C.c_int),
            "mfsgd_sync": ([vp], C.c_int),
            "mfsgd_get_factors": ([vp, vp, vp], C.c_int),
            "mfsgd_set_factors": ([vp, vp, vp], C.c_int),
            "mfsgd_set_epoch": ([i64], C.c_int),
            "mfsgd_get_epoch": ([], i64),
            "mfsgd_debug_read": ([i32, vp, i64, vp], C.c_int),
            "mfsgd_finalize": ([], C.c_int),
            "mfsgd_last_error": ([], C.c_char_p),
            "mfsgd_version": ([], C.c_char_p),
        }
        sig.update({
            "mfsgd_embed": ([vp, i64, i64, i32, i32, vp, i64, i64, f32, vp, i64, vp], C.c_int),
            "mfsgd_embed_grad": ([vp, i64, vp, i64, i64, i32, i32, f32, vp, i64, i64, i32, vp, i64, vp], C.c_int),
            "mfsgd_embed_grad_workspace": ([i64, i32, C.POINTER(i64)], C.c_int),
            "mfsgd_embed_grad_workspace_rows": ([i64, i32, i64, C.POINTER(i64)], C.c_int),
            "mfsgd_rows": ([i32, vp, i64, i64, i32, i32, f32, vp, i64, vp], C.c_int),
            "mfsgd_add_rows": ([i32, vp, i64, vp, i64, i64, i32, i32, f32, vp, i64, vp], C.c_int),
            "mfsgd_linear": ([vp, i64, vp, i64, vp, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp],
                             C.c_int),
            "mfsgd_linear_workspace": ([i64, i64, i64, i32, C.POINTER(i64)], C.c_int),
            "mfsgd_linear_grad": ([vp, i64, vp, i64, vp, i64, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp, i64, vp,
                                   vp, i64, vp], C.c_int),
            "mfsgd_linear_grad_workspace": ([i64, i64, i64, i32, C.POINTER(i64)], C.c_int),
            "mfsgd_scores": ([vp, i64, i64, i64, i32, vp, i32, vp, i64, vp, i64, vp], C.c_int),
            "mfsgd_scores_workspace": ([i64, C.POINTER(i64)], C.c_int),
            "mfsgd_grad_norm": ([vp, i64, vp, vp, i64, vp], C.c_int),
            "mfsgd_clip_grads": ([vp, i64, C.c_double, vp, vp, i64, vp], C.c_int),
            "mfsgd_sgd_step": ([vp, vp, i64, f32, f32, C.c_double, vp, vp, i64, vp], C.c_int),
            "mfsgd_norm_workspace": ([i64, C.POINTER(i64)], C.c_int),
        })
        for name, (args, res) in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = res
        _lib = L
    return _lib


def _check(rc: int, fn: str) -> int:
    if rc != OK:
        raise MfsgdError(rc, fn, lib().mfsgd_last_error().decode())
    return rc


def _stream(stream) -> C.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _samples_ptr(t: torch.Tensor):
    if t.dtype != torch.int32 or t.dim() != 2 or t.shape[1] != 3 or not t.is_contiguous() or not t.is_cuda:
        raise TypeError("samples must be a contiguous int32 cuda tensor of shape (nnz, 3)")
    return C.c_void_p(t.data_ptr() if t.numel() else 0), t.shape[0]


def samples_to_device(a: np.ndarray, device="cuda") -> torch.Tensor:
    """numpy structured (u, v, r) records -> int32 (nnz, 3) device tensor."""
    a = np.ascontiguousarray(a)
    assert a.dtype == SAMPLE_DTYPE
    t = torch.from_numpy(a.view(np.int32).reshape(-1, 3).copy())
    return t.to(device)


def version() -> str:
    return lib().mfsgd_version().decode()


def set_option(key: str, value: int) -> None:
    _check(lib().mfsgd_set_option(key.encode(), int(value)), "mfsgd_set_option")


def get_option(key: str) -> int:
    v = C.c_int64()
    _check(lib().mfsgd_get_option(key.encode(), C.byref(v)), "mfsgd_get_option")
    return v.value


def reset_options() -> None:
    """Every option back to its default."""
    _check(lib().mfsgd_reset_options(), "mfsgd_reset_options")


def init(m: int, n: int, k: int, seed: int) -> None:
    _check(lib().mfsgd_init(m, n, k, seed), "mfsgd_init")


def plan(samples: torch.Tensor, s: int, stream=None) -> None:
    p, nnz = _samples_ptr(samples)
    _check(lib().mfsgd_plan(p, nnz, s, _stream(stream)), "mfsgd_plan")


def epoch(samples: torch.Tensor, lr: float, lambda_p: float, lambda_q: float, scheme="hogwild",
          stream=None) -> None:
    p, nnz = _samples_ptr(samples)
    sc = SCHEMES[scheme] if isinstance(scheme, str) else int(scheme)
    _check(lib().mfsgd_epoch(p, nnz, lr, lambda_p, lambda_q, sc, _stream(stream)), "mfsgd_epoch")


def epoch_staged(samples, lr: float, lambda_p: float, lambda_q: float, stream=None) -> None:
    """mfsgd_epoch_staged on host samples: a numpy (u, v, r) record array or
    an int32 (nnz, 3) CPU tensor (pinned or not).  A pinned array must stay
    alive and unchanged until the work on `stream` completes."""
    if isinstance(samples, np.ndarray):
        if samples.dtype != SAMPLE_DTYPE or not samples.flags["C_CONTIGUOUS"]:
            raise TypeError("samples must be a C-contiguous array of (u, v, r) records")
        p, nnz = C.c_void_p(samples.ctypes.data if samples.size else 0), samples.shape[0]
    else:
        t = samples
        if t.dtype != torch.int32 or t.dim() != 2 or t.shape[1] != 3 or not t.is_contiguous() or t.is_cuda:
            raise TypeError("samples must be a contiguous int32 CPU tensor of shape (nnz, 3)")
        p, nnz = C.c_void_p(t.data_ptr() if t.numel() else 0), t.shape[0]
    _check(lib().mfsgd_epoch_staged(p, nnz, lr, lambda_p, lambda_q, _stream(stream)), "mfsgd_epoch_staged")


def rmse(test: torch.Tensor, stream=None) -> float:
    p, n = _samples_ptr(test)
    out = C.c_double()
    _check(lib().mfsgd_rmse(p, n, C.byref(out), _stream(stream)), "mfsgd_rmse")
    return out.value


def rmse_noalloc(test: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    """Enqueue the test RMSE into out[0] (a float64 device tensor) without
    allocating or waiting (mfsgd_rmse_noalloc)."""
    if out.dtype != torch.float64 or not out.is_cuda or out.numel() < 1:
        raise ValueError("out must be a float64 device tensor with at least one element")
    p, n = _samples_ptr(test)
    _check(lib().mfsgd_rmse_noalloc(p, n, C.c_void_p(out.data_ptr()), _stream(stream)), "mfsgd_rmse_noalloc")


def check_samples(samples: torch.Tensor, stream=None) -> None:
    p, nnz = _samples_ptr(samples)
    _check(lib().mfsgd_check_samples(p, nnz, _stream(stream)), "mfsgd_check_samples")


def sync(stream=None) -> None:
    _check(lib().mfsgd_sync(_stream(stream)), "mfsgd_sync")


def _storage_dtype():
    return torch.float16 if get_option("dtype") == FP16 else torch.float32


def get_factors(m: int, n: int, k: int, dtype=None, device="cuda", stream=None):
    """(P, Q) copies, shapes (m, k) and (n, k), storage dtype of the model."""
    dtype = dtype or _storage_dtype()
    P = torch.empty((m, k), dtype=dtype, device=device)
    Q = torch.empty((n, k), dtype=dtype, device=device)
    _check(lib().mfsgd_get_factors(C.c_void_p(P.data_ptr()), C.c_void_p(Q.data_ptr()), _stream(stream)),
           "mfsgd_get_factors")
    return P, Q


def set_factors(P: torch.Tensor, Q: torch.Tensor, stream=None) -> None:
    P = P.contiguous()
    Q = Q.contiguous()
    _check(lib().mfsgd_set_factors(C.c_void_p(P.data_ptr()), C.c_void_p(Q.data_ptr()), _stream(stream)),
           "mfsgd_set_factors")


def set_epoch(t: int) -> None:
    _check(lib().mfsgd_set_epoch(t), "mfsgd_set_epoch")


def get_epoch() -> int:
    return lib().mfsgd_get_epoch()


def debug_visits(nnz: int, stream=None) -> torch.Tensor:
    out = torch.empty(nnz, dtype=torch.int32, device="cuda")
    _check(lib().mfsgd_debug_read(DBG_VISITS, C.c_void_p(out.data_ptr()), nnz, _stream(stream)), "mfsgd_debug_read")
    return out


def debug_trace(count: int, stream=None) -> torch.Tensor:
    out = torch.empty(count, dtype=torch.int32, device="cuda")
    _check(lib().mfsgd_debug_read(DBG_TRACE, C.c_void_p(out.data_ptr()), count, _stream(stream)),
           "mfsgd_debug_read")
    return out


def debug_plan_starts(s: int, stream=None) -> torch.Tensor:
    out = torch.empty(s * s + 1, dtype=torch.int64, device="cuda")
    _check(lib().mfsgd_debug_read(DBG_PLAN_STARTS, C.c_void_p(out.data_ptr()), s * s + 1, _stream(stream)),
           "mfsgd_debug_read")
    return out


def debug_plan_order(nnz: int, stream=None) -> torch.Tensor:
    out = torch.empty(max(nnz, 1), dtype=torch.int64, device="cuda")
    _check(lib().mfsgd_debug_read(DBG_PLAN_ORDER, C.c_void_p(out.data_ptr()), nnz, _stream(stream)),
           "mfsgd_debug_read")
    return out[:nnz]


def debug_table_starts(s: int, stream=None) -> torch.Tensor:
    out = torch.empty(s * s + 1, dtype=torch.int64, device="cuda")
    _check(lib().mfsgd_debug_read(DBG_TABLE_STARTS, C.c_void_p(out.data_ptr()), s * s + 1, _stream(stream)),
           "mfsgd_debug_read")
    return out


def debug_table_order(nnz: int, stream=None) -> torch.Tensor:
    out = torch.empty(max(nnz, 1), dtype=torch.int64, device="cuda")
    _check(lib().mfsgd_debug_read(DBG_TABLE_ORDER, C.c_void_p(out.data_ptr()), nnz, _stream(stream)),
           "mfsgd_debug_read")
    return out[:nnz]


def debug_team_layout(s: int, stream=None):
    """(map, sizes) of the last block-scheduled epoch: per (XCD x, arrival
    slot j) at x * (len(map) / xcds) + j -- or per workgroup for one-wavefront
    teams -- team << 16 | member (-1 idle), per team its workgroup count."""
    grid = get_option("teams_grid")
    tmap = torch.empty(max(grid, 1), dtype=torch.int32, device="cuda")
    sizes = torch.empty(s, dtype=torch.int32, device="cuda")
    _check(lib().mfsgd_debug_read(DBG_TEAM_MAP, C.c_void_p(tmap.data_ptr()), grid, _stream(stream)),
           "mfsgd_debug_read")
    _check(lib().mfsgd_debug_read(DBG_TEAM_SIZES, C.c_void_p(sizes.data_ptr()), s, _stream(stream)),
           "mfsgd_debug_read")
    return tmap[:grid], sizes


def debug_priority(s: int, stream=None):
    """Critical-path weight of every (team, wave) block of the last pooled
    block-scheduled epoch: uint32 tensor of s*s, entry t*s + w."""
    out = torch.empty(s * s, dtype=torch.int32, device="cuda")
    _check(lib().mfsgd_debug_read(DBG_PRIORITY, C.c_void_p(out.data_ptr()), s * s, _stream(stream)),
           "mfsgd_debug_read")
    return out


# --- operators on tables, gradients (see the header for what each computes) ---
#
# Outputs and workspaces not passed in are allocated on the stream the work runs
# on; tensors given to a call on another stream than the current one may be
# freed right after it (the order of work on the two is the caller's).  Row-major
# matrices may have any row pitch; a tensor on another device than the current
# one, of another dtype than its call's or with strided columns is refused
# before anything is enqueued, and so is an `out` that shares memory with what
# the call reads, unless it says that it may.
#
# Autograd does not see these calls: they take tensors that require gradients,
# their results require none, and the ..._grad calls are there to be called.  A
# tensor changed in place (an `out`, clipped gradients, updated parameters)
# counts as changed all the same, so that autograd refuses to go backward
# through a value it had saved of it.

_DTYPES = {torch.float32: FP32, torch.float16: FP16, torch.bfloat16: BF16}
_changed = torch.autograd.graph.increment_version  # of a tensor or several


class _On:
    """The stream of a call: its handle, and allocations that belong to it."""

    __slots__ = ("device", "stream", "handle")

    def __init__(self, stream):
        self.device = torch.cuda.current_device()
        self.stream = stream
        if stream is None:
            self.handle = _current_stream(self.device)
        else:
            if stream.device_index != self.device:
                raise ValueError("the stream is on another device than the current one")
            self.handle = stream.cuda_stream

    def uses(self, *tensors):
        """Keeps the memory of tensors freed after this call until the work on a stream of the caller's is done."""
        if self.stream is not None:
            for t in tensors:
                if t is not None:
                    t.record_stream(self.stream)

    def empty(self, shape, dtype):
        if self.stream is None:
            return torch.empty(shape, dtype=dtype, device=_cuda(self.device))
        with torch.cuda.stream(self.stream):
            return torch.empty(shape, dtype=dtype, device=_cuda(self.device))

    def workspace(self, nbytes):
        """(address, bytes, tensor) of a new workspace; the tensor must outlive the call."""
        if not nbytes:
            return None, 0, None
        t = self.empty((nbytes,), torch.uint8)
        return t.data_ptr(), nbytes, t


# the handle alone, where torch offers it: a Stream object costs as much as a small launch
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                          lambda device: torch.cuda.current_stream(device).cuda_stream)


@functools.lru_cache(maxsize=None)
def _cuda(index):
    return torch.device("cuda", index)


def _matrix(t, what, device, dtype=None, shape=None):
    """Row pitch of a matrix, after checking it."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or t.get_device() != device or t.dtype not in _DTYPES:
        raise TypeError(f"{what} must be a float32, float16 or bfloat16 matrix on the current GPU")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, not {t.dtype}")
    rows, width = t.shape
    if shape is not None and (rows, width) != shape:
        raise ValueError(f"{what} must have the shape {shape}, not {(rows, width)}")
    ld, col = t.stride()
    if width > 1 and col != 1 or rows > 1 and ld < width:
        raise ValueError(f"the rows of {what} must be contiguous and not overlap")
    return ld if rows > 1 and ld >= width else max(width, 1)


def _ids(t, device):
    """Address, stride and length of an id vector."""
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or t.dim() != 1 or t.get_device() != device:
        raise TypeError("ids must be an int32 vector on the current GPU")
    n = t.shape[0]
    stride = t.stride(0) if n > 1 else 1
    if stride < 1:
        raise ValueError("ids must have a positive stride")
    return t.data_ptr(), stride, n


@functools.lru_cache(maxsize=4096)
def _bytes(fn, *sizes):
    """What a ..._workspace call says of these sizes (it depends on nothing else)."""
    n = C.c_int64()
    _check(getattr(lib(), fn)(*sizes, C.byref(n)), fn)
    return n.value


def embed(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out=None, stream=None) -> torch.Tensor:
    """Rows of `table` by id, times `scale`; zeros where an id is outside the
    table (padding).  `ids` may be a column of a sample tensor."""
    on = _On(stream)
    ld = _matrix(table, "table", on.device)
    idp, stride, count = _ids(ids, on.device)
    rows, k = table.shape
    given = out is not None
    if not given:
        out = on.empty((count, k), table.dtype)
        ld_out = k
    else:
        ld_out = _matrix(out, "out", on.device, table.dtype, (count, k))
    on.uses(table, ids, out)
    _check(lib().mfsgd_embed(table.data_ptr(), rows, ld, k, _DTYPES[table.dtype], idp, stride, count, scale,
                             out.data_ptr(), ld_out, on.handle), "mfsgd_embed")
    if given:
        _changed(out)
    return out


def embed_grad(dout: torch.Tensor, ids: torch.Tensor, rows: int, scale: float = 1.0, out=None,
               accumulate: bool = False, stream=None) -> torch.Tensor:
    """The gradient of ``embed`` with respect to its table of `rows` rows: row r
    is `scale` times the sum of dout's rows whose id is r.  With `accumulate` it
    is added to `out`, of which only those rows are touched."""
    on = _On(stream)
    ld = _matrix(dout, "dout", on.device)
    idp, stride, count = _ids(ids, on.device)
    n, k = dout.shape
    if n != count:
        raise ValueError(f"dout has {n} rows for {count} ids")
    given = out is not None
    if not given:
        if accumulate:
            raise ValueError("accumulate needs an `out` to add to")
        out = on.empty((rows, k), dout.dtype)
        ld_out = k
    else:
        ld_out = _matrix(out, "out", on.device, dout.dtype, (rows, k))
    work, nbytes, keep = on.workspace(_bytes("mfsgd_embed_grad_workspace_rows", count, k, rows))
    on.uses(dout, ids, out)
    _check(lib().mfsgd_embed_grad(dout.data_ptr(), ld, idp, stride, count, k, _DTYPES[dout.dtype], scale,
                                  out.data_ptr(), rows, ld_out, accumulate, work, nbytes, on.handle),
           "mfsgd_embed_grad")
    if given:
        _changed(out)
    return out


def rows(side: int, ids: torch.Tensor, k: int, dtype=None, scale: float = 1.0, out=None,
         stream=None) -> torch.Tensor:
    """``embed`` on the model's own factors: `side` is P (users) or Q (items).
    k and dtype must be the model's (dtype by default: what option "dtype" says)."""
    on = _On(stream)
    idp, stride, count = _ids(ids, on.device)
    dtype = dtype or _storage_dtype()
    given = out is not None
    if not given:
        out = on.empty((count, k), dtype)
        ld_out = k
    else:
        ld_out = _matrix(out, "out", on.device, dtype, (count, k))
    on.uses(ids, out)
    _check(lib().mfsgd_rows(side, idp, stride, count, k, _DTYPES[dtype], scale, out.data_ptr(), ld_out, on.handle),
           "mfsgd_rows")
    if given:
        _changed(out)
    return out


def add_rows(side: int, dout: torch.Tensor, ids: torch.Tensor, scale: float, stream=None) -> None:
    """Adds `scale` times the sum of dout's rows of every id to that row of the
    model's factors, in place: the gradient step of those rows at scale = -lr.
    dout has the model's k and dtype."""
    on = _On(stream)
    ld = _matrix(dout, "dout", on.device)
    idp, stride, count = _ids(ids, on.device)
    n, k = dout.shape
    if n != count:
        raise ValueError(f"dout has {n} rows for {count} ids")
    work, nbytes, keep = on.workspace(_bytes("mfsgd_embed_grad_workspace", count, k))
    on.uses(dout, ids)
    _check(lib().mfsgd_add_rows(side, dout.data_ptr(), ld, idp, stride, count, k, _DTYPES[dout.dtype], scale, work,
                                nbytes, on.handle), "mfsgd_add_rows")


def _vector(t, what, n, device, dtype):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.get_device() != device:
        raise TypeError(f"{what} must be a {dtype} vector on the current GPU")
    if t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what} must be {n} contiguous values")
    return t.data_ptr()


def linear(x: torch.Tensor, w: torch.Tensor, bias=None, residual=None, act: str = "none", out=None,
           keep_z: bool = False, stream=None):
    """act(x w^T + bias) + residual for x (M, K) and w (N, K).  With `keep_z`
    also the pre-activation, which ``linear_grad`` takes: (y, z).  `residual`
    may be `out` itself."""
    on = _On(stream)
    dt = x.dtype if isinstance(x, torch.Tensor) else None
    ldx, ldw = _matrix(x, "x", on.device), _matrix(w, "w", on.device, dt)
    (M, K), (N, Kw) = x.shape, w.shape
    if K != Kw:
        raise ValueError(f"x has {K} columns, w {Kw}")
    bp = None if bias is None else _vector(bias, "bias", N, on.device, dt)
    ldr = 0 if residual is None else _matrix(residual, "residual", on.device, dt, (M, N))
    given = out is not None
    if not given:
        out = on.empty((M, N), dt)
        ldy = max(N, 1)
    else:
        ldy = _matrix(out, "out", on.device, dt, (M, N))
    z = on.empty((M, N), dt) if keep_z else None
    code = _DTYPES[dt]
    work, nbytes, keep = on.workspace(_bytes("mfsgd_linear_workspace", M, N, K, code))
    on.uses(x, w, bias, residual, out)
    _check(lib().mfsgd_linear(x.data_ptr(), ldx, w.data_ptr(), ldw, bp,
                              None if residual is None else residual.data_ptr(), ldr, M, N, K, code, ACTS[act],
                              out.data_ptr(), ldy, z.data_ptr() if keep_z else None, max(N, 1), work, nbytes,
                              on.handle), "mfsgd_linear")
    if given:
        _changed(out)
    return (out, z) if keep_z else out


def linear_grad(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, z=None, act: str = "none", dx: bool = True,
                dw: bool = True, dbias: bool = True, stream=None):
    """(dx, dw, dbias) of ``linear`` for dy, the gradient of its result, and the
    z it kept (not needed without an activation); None for those not asked for.
    The residual's gradient is dy."""
    on = _On(stream)
    dt = x.dtype if isinstance(x, torch.Tensor) else None
    ldx, ldw = _matrix(x, "x", on.device), _matrix(w, "w", on.device, dt)
    (M, K), (N, Kw) = x.shape, w.shape
    if K != Kw:
        raise ValueError(f"x has {K} columns, w {Kw}")
    lddy = _matrix(dy, "dy", on.device, dt, (M, N))
    if z is None and act != "none":
        raise ValueError("the gradient of an activation needs z")
    ldz = 0 if z is None else _matrix(z, "z", on.device, dt, (M, N))
    code = _DTYPES[dt]
    work, nbytes, keep = on.workspace(_bytes("mfsgd_linear_grad_workspace", M, N, K, code))
    gx = on.empty((M, K), dt) if dx else None
    gw = on.empty((N, K), dt) if dw else None
    gb = on.empty((N,), dt) if dbias else None
    on.uses(dy, x, w, z)
    _check(lib().mfsgd_linear_grad(dy.data_ptr(), lddy, None if z is None else z.data_ptr(), ldz, x.data_ptr(), ldx,
                                   w.data_ptr(), ldw, M, N, K, code, ACTS[act], gx.data_ptr() if dx else None,
                                   max(K, 1), gw.data_ptr() if dw else None, max(K, 1),
                                   gb.data_ptr() if dbias else None, work, nbytes, on.handle), "mfsgd_linear_grad")
    return gx, gw, gb


def scores(users: torch.Tensor, n: int, dtype=None, bias=None, act: str = "none", out=None,
           stream=None) -> torch.Tensor:
    """The model's scores of `users` against all its n items:
    act(p_user . q_item + bias of the item).  A user outside the model: act(bias)."""
    on = _On(stream)
    up, stride, count = _ids(users, on.device)
    dtype = dtype or _storage_dtype()
    bp = None if bias is None else _vector(bias, "bias", n, on.device, dtype)
    given = out is not None
    if not given:
        out = on.empty((count, n), dtype)
        ld = max(n, 1)
    else:
        ld = _matrix(out, "out", on.device, dtype, (count, n))
    need = C.c_int64()
    _check(lib().mfsgd_scores_workspace(count, C.byref(need)), "mfsgd_scores_workspace")
    work, nbytes, keep = on.workspace(need.value)
    on.uses(users, bias, out)
    _check(lib().mfsgd_scores(up, stride, count, n, _DTYPES[dtype], bp, ACTS[act], out.data_ptr(), ld, work, nbytes,
                              on.handle), "mfsgd_scores")
    if given:
        _changed(out)
    return out


class TensorList:
    """Tensors that ``grad_norm``, ``clip_grads`` and ``sgd_step`` take together,
    checked and laid out once.  It holds the tensors: they must keep the storage
    they had (not be moved, resized or set to another) while it is used."""

    class _Entry(C.Structure):
        _fields_ = [("data", C.c_void_p), ("n", C.c_int64), ("dtype", C.c_int32), ("unused", C.c_int32)]

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self.device = None
        self.entries = (TensorList._Entry * max(len(self.tensors), 1))()
        for i, t in enumerate(self.tensors):
            if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in _DTYPES or not t.is_contiguous():
                raise TypeError("the tensors must be contiguous float32, float16 or bfloat16 tensors on the GPU")
            if self.device is None:
                self.device = t.get_device()
            if t.get_device() != self.device:
                raise ValueError("the tensors must be on one device")
            self.entries[i].data, self.entries[i].n = t.data_ptr(), t.numel()
            self.entries[i].dtype = _DTYPES[t.dtype]
        self.workspace_bytes = _bytes("mfsgd_norm_workspace", len(self.tensors))

    def __len__(self):
        return len(self.tensors)


def _tensor_list(tensors, on):
    a = tensors if isinstance(tensors, TensorList) else TensorList(tensors)
    if a.device is not None and a.device != on.device:
        raise ValueError("the tensors are on another device than the current one")
    on.uses(*a.tensors)
    return a


def grad_norm(grads, stream=None) -> torch.Tensor:
    """The norm of all gradients together (a TensorList or an iterable of
    tensors): a float64 scalar on the GPU."""
    on = _On(stream)
    g = _tensor_list(grads, on)
    norm = on.empty((), torch.float64)
    work, nbytes, keep = on.workspace(g.workspace_bytes)
    _check(lib().mfsgd_grad_norm(g.entries, len(g), norm.data_ptr(), work, nbytes, on.handle), "mfsgd_grad_norm")
    return norm


def clip_grads(grads, max_norm: float, stream=None) -> torch.Tensor:
    """Scales all gradients in place so that their norm is at most `max_norm`;
    returns the norm they had."""
    on = _On(stream)
    g = _tensor_list(grads, on)
    norm = on.empty((), torch.float64)
    work, nbytes, keep = on.workspace(g.workspace_bytes)
    _check(lib().mfsgd_clip_grads(g.entries, len(g), max_norm, norm.data_ptr(), work, nbytes, on.handle),
           "mfsgd_clip_grads")
    _changed(g.tensors)
    return norm


def sgd_step(params, grads, lr: float, lam: float = 0.0, max_norm: float = float("inf"), stream=None) -> torch.Tensor:
    """p <- p - lr (c g + lam p) with c = min(1, max_norm / norm of all
    gradients), in place; the gradients stay.  Returns the norm."""
    on = _On(stream)
    p, g = _tensor_list(params, on), _tensor_list(grads, on)
    if len(p) != len(g):
        raise ValueError(f"{len(p)} parameters and {len(g)} gradients")
    norm = on.empty((), torch.float64)
    work, nbytes, keep = on.workspace(g.workspace_bytes)
    _check(lib().mfsgd_sgd_step(p.entries, g.entries, len(g), lr, lam, max_norm, norm.data_ptr(), work, nbytes,
                                on.handle), "mfsgd_sgd_step")
    _changed(p.tensors)
    return norm


def finalize() -> None:
    _check(lib().mfsgd_finalize(), "mfsgd_finalize")
