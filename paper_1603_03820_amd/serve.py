"""Answering with a trained factor model: ctypes binding of libals_serve.so (include/als_serve.h),
marshalling torch tensors, and the loop that a recommender runs on top of it.

``als_quantize`` holds factor rows in 8 bits, ``als_score`` scores users against items from such rows, and
``als_sample`` draws one item a row of scores; ``Recommender`` holds a model's items in 8 bits and answers
batches of users with the three in a row.  All arithmetic runs in the library's kernels; importing this
module fails loudly when libals_serve.so is not built: there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import os

import torch

from .als import ALS_OK, ALSError

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libals_serve.so")

ALS_SERVE_F_MAX = 131_071
ALS_SERVE_N_MAX = 4_194_304
EXPORTED = ("als_serve_workspace_bytes", "als_serve_init", "als_serve_destroy",
            "als_serve_last_hip_error", "als_quantize", "als_score", "als_sample")
_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


class _Limits(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
                ("min_p", ctypes.c_void_p), ("temperature_all", ctypes.c_float), ("top_k_all", ctypes.c_int32),
                ("top_p_all", ctypes.c_float), ("min_p_all", ctypes.c_float)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libals_serve.so is not built ({LIB_PATH}); run __graft_entry__.build() or "
                          "python paper_1603_03820_amd/build.py")
    lib = ctypes.CDLL(LIB_PATH)
    P, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    lib.als_serve_workspace_bytes.argtypes = [ctypes.c_int]
    lib.als_serve_workspace_bytes.restype = ctypes.c_size_t
    lib.als_serve_init.argtypes = [ctypes.POINTER(P), ctypes.c_int, P, ctypes.c_size_t]
    lib.als_serve_destroy.argtypes = [P]
    lib.als_serve_last_hip_error.argtypes = [P]
    lib.als_quantize.argtypes = [P, P, i32, i64, i64, P, i64, i32, P, i64, P, P]
    lib.als_score.argtypes = [P, P, i64, P, i64, P, i64, P, i64, i32, P, i32, i64, P]
    lib.als_sample.argtypes = [P, P, i32, i64, i64, i64, ctypes.POINTER(_Limits), P, P, P, P, i64, P, P, P]
    for fn in EXPORTED[1:]:
        getattr(lib, fn).restype = ctypes.c_int
    return lib


_lib = _load()


def _check(fn: str, rc: int, ctx=None):
    if rc != ALS_OK:
        raise ALSError(fn, rc, _lib.als_serve_last_hip_error(ctx) if ctx is not None else 0)


def als_serve_workspace_bytes(device: int = 0) -> int:
    return int(_lib.als_serve_workspace_bytes(device))


class Context:
    """An als_serve_ctx plus the workspace tensor it runs in (one per device)."""

    def __init__(self, device: int = 0):
        self.device = torch.device("cuda", device)
        nbytes = als_serve_workspace_bytes(device)
        if nbytes == 0:
            raise RuntimeError(f"als_serve_workspace_bytes failed for device {device} (not gfx950?)")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        h = ctypes.c_void_p()
        _check("als_serve_init", _lib.als_serve_init(ctypes.byref(h), device,
                                                     ctypes.c_void_p(self.workspace.data_ptr()), nbytes))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            _lib.als_serve_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _Call:
    """One call's stream and tensors.  A tensor that the call allocates is allocated on the call's stream, and
    one that is used on another stream than the current one is recorded there, so that its memory is not handed
    out again while the call may still run."""

    def __init__(self, ctx: Context, stream):
        if not ctx.handle:
            raise ValueError("the context is closed")
        self.device = ctx.device
        self.current = torch.cuda.current_stream(ctx.device)
        self.torch_stream = self.current if stream is None else stream
        self.other = self.torch_stream != self.current
        self.stream = ctypes.c_void_p(self.torch_stream.cuda_stream)

    def empty(self, shape, dtype):
        if not self.other:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self.torch_stream):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _use(self, t, name, dtypes):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise TypeError(f"{name} must be a device tensor")
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, the context on {self.device}")
        if t.dtype not in dtypes:
            raise TypeError(f"{name} must be {' or '.join(map(str, dtypes))}, got {t.dtype}")
        if self.other:
            t.record_stream(self.torch_stream)
        return ctypes.c_void_p(t.data_ptr()) if t.numel() else None

    def vector(self, t, name, dtype, length):
        p = self._use(t, name, (dtype,))
        if t.dim() != 1 or t.shape[0] != length:
            raise ValueError(f"{name} must have {length} elements, has shape {tuple(t.shape)}")
        if length > 1 and t.stride(0) != 1:
            raise ValueError(f"{name} must be contiguous")
        return p

    def matrix(self, t, name, dtypes, rows=None, cols=None):
        """(pointer, row stride) of a matrix whose rows are contiguous, at any distance."""
        p = self._use(t, name, dtypes)
        if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
            want = ("any" if rows is None else rows, "any" if cols is None else cols)
            raise ValueError(f"{name} must be a matrix of {want[0]} x {want[1]}, has shape {tuple(t.shape)}")
        if t.shape[1] > 1 and t.stride(1) != 1:
            raise ValueError(f"the rows of {name} must be contiguous")
        if t.shape[0] > 1 and t.stride(0) < t.shape[1]:
            raise ValueError(f"the rows of {name} overlap")
        return p, (t.stride(0) if t.shape[0] > 1 else max(t.shape[1], t.stride(0)))


def als_quantize(ctx: Context, x, users=None, q=None, scale=None, stream=None):
    """(q, scale): the rows of x (f32, f16 or bf16), or the rows `users` (int32) of it, as 8-bit integers
    with one scale each, x ~ scale q.  Without `q` the result is a view of rows whose stride is the next
    multiple of 16."""
    call = _Call(ctx, stream)
    px, ldx = call.matrix(x, "x", tuple(_DTYPES))
    of, f = x.shape
    rows = of if users is None else users.numel()
    pu = None if users is None else call.vector(users, "users", torch.int32, rows)
    if q is None:
        q = call.empty((rows, (f + 15) // 16 * 16), torch.int8)[:, :f]
    if scale is None:
        scale = call.empty((rows,), torch.float32)
    pq, ldq = call.matrix(q, "q", (torch.int8,), rows, f)
    ps = call.vector(scale, "scale", torch.float32, rows)
    rc = _lib.als_quantize(ctx.handle, px, _DTYPES[x.dtype], of, ldx, pu, rows, f, pq, ldq, ps, call.stream)
    _check("als_quantize", rc, ctx.handle)
    return q, scale


def als_score(ctx: Context, xq, xs, tq, ts, out=None, dtype=torch.float32, stream=None):
    """out[i, j] = xs_i ts_j sum_k xq_ik tq_jk for 8-bit rows with a scale each; out (f32, f16 or bf16, `dtype`
    where it is not given) may have any row stride."""
    call = _Call(ctx, stream)
    px, ldx = call.matrix(xq, "xq", (torch.int8,))
    m, f = xq.shape
    pt, ldt = call.matrix(tq, "tq", (torch.int8,), None, f)
    n = tq.shape[0]
    if out is None:
        if dtype not in _DTYPES:
            raise TypeError(f"dtype must be {' or '.join(map(str, _DTYPES))}, got {dtype}")
        out = call.empty((m, n), dtype)
    po, ldo = call.matrix(out, "out", tuple(_DTYPES), m, n)
    rc = _lib.als_score(ctx.handle, px, ldx, call.vector(xs, "xs", torch.float32, m), m, pt, ldt,
                        call.vector(ts, "ts", torch.float32, n), n, f, po, _DTYPES[out.dtype], ldo, call.stream)
    _check("als_score", rc, ctx.handle)
    return out


def als_sample(ctx: Context, scores, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, rated=None, users=None,
               index=None, log=None, stream=None):
    """(index, log): one column a row of `scores`, drawn by the uniform numbers `u` (float32, one a row), and the
    logarithm of its probability.  temperature, top_k, top_p and min_p are numbers, or tensors with one value
    a row (float32; top_k int32); `rated` = (rowptr, colidx) is a CSR of columns to leave out, row users[r] (int32)
    of it for row r, or row r.  See als_sample in include/als_serve.h for the definition."""
    call = _Call(ctx, stream)
    pz, ldz = call.matrix(scores, "scores", tuple(_DTYPES))
    rows, n = scores.shape
    lim = _Limits()
    for name, value, dtype in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32),
                               ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32)):
        if isinstance(value, torch.Tensor):
            setattr(lim, name, call.vector(value, name, dtype, rows))
        else:
            setattr(lim, name + "_all", value)
    pp = pi = pu = None
    of = 0
    if rated is not None:
        rowptr, colidx = rated
        of = rowptr.numel() - 1
        pp = call.vector(rowptr, "rated[0]", torch.int64, of + 1)
        pi = call.vector(colidx, "rated[1]", torch.int32, colidx.numel())
        if pi is None:
            pi = pp     # every row is empty: nothing is read
        if users is not None:
            pu = call.vector(users, "users", torch.int32, rows)
        elif of < rows:
            raise ValueError(f"rated has {of} rows, scores {rows}")
    elif users is not None:
        raise ValueError("users without rated")
    if index is None:
        index = call.empty((rows,), torch.int32)
    if log is None:
        log = call.empty((rows,), torch.float32)
    rc = _lib.als_sample(ctx.handle, pz, _DTYPES[scores.dtype], rows, n, ldz, ctypes.byref(lim),
                         call.vector(u, "u", torch.float32, rows), pp, pi, pu, of,
                         call.vector(index, "index", torch.int32, rows), call.vector(log, "log", torch.float32, rows),
                         call.stream)
    _check("als_sample", rc, ctx.handle)
    return index, log


class Recommender:
    """Draws items for batches of users of a trained model.  The items' factors are held in 8 bits; `rated`, the
    CSR of the training ratings, is what its users are not recommended again."""

    def __init__(self, ctx: Context, x, theta, rated=None):
        self.ctx, self.x, self.rated = ctx, x, rated
        self.items, self.item_scale = als_quantize(ctx, theta)

    def scores(self, users, dtype=torch.float32, stream=None):
        """The predicted ratings of `users` (int32 rows of X) for every item."""
        q, scale = als_quantize(self.ctx, self.x, users=users, stream=stream)
        return als_score(self.ctx, q, scale, self.items, self.item_scale, dtype=dtype, stream=stream)

    def recommend(self, users, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, stream=None):
        """(item, log probability) for each of `users`, by one uniform number each; item -1 where nothing is
        left to recommend."""
        z = self.scores(users, stream=stream)
        if self.rated is None:
            return als_sample(self.ctx, z, u, temperature, top_k, top_p, min_p, stream=stream)
        return als_sample(self.ctx, z, u, temperature, top_k, top_p, min_p, rated=self.rated, users=users,
                          stream=stream)
