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

ALS_ERR_ALIAS = -6
ALS_SERVE_F_MAX = 131_071
ALS_SERVE_N_MAX = 4_194_304
ALS_SERVE_HELD_MAX = 65_536
EXPORTED = ("als_serve_workspace_bytes", "als_serve_init", "als_serve_destroy",
            "als_serve_last_hip_error", "als_quantize", "als_quantize_into", "als_score", "als_sample")
_INT32_MAX = 2 ** 31 - 1
_FAR = 1 << 22               # row stride from which als_score does not read rows in place
_REFUSED = ALS_SERVE_F_MAX + 1       # what the library, which takes row lengths in 32 bits, is told of all longer ones
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
    lib.als_quantize_into.argtypes = [P, P, i32, i64, i64, P, i64, i32, P, i64, i32, P, P]
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


def _capturing(stream):
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


class Context:
    """An als_serve_ctx plus the workspace tensor it runs in (one per device).  Calls that work in the workspace (draws
    from rows of more than ALS_SERVE_HELD_MAX columns, scores of rows that are not read in place) follow one
    another also where they are on different streams: each waits for the last one's stream.  Not so calls that are
    captured into a graph: whoever launches it keeps its launches, and the eager calls beside them, apart, and keeps
    the context as long as the graph."""

    def __init__(self, device: int = 0):
        self.device = torch.device("cuda", device)
        self.index = device
        nbytes = als_serve_workspace_bytes(device)
        if nbytes == 0:
            raise RuntimeError(f"als_serve_workspace_bytes failed for device {device} (not gfx950?)")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        h = ctypes.c_void_p()
        _check("als_serve_init", _lib.als_serve_init(ctypes.byref(h), device,
                                                     ctypes.c_void_p(self.workspace.data_ptr()), nbytes))
        self.handle = h
        self._start(torch.cuda.current_stream(self.device))

    def _start(self, stream):
        self._limits = _Limits()
        self._limits_ref = ctypes.byref(self._limits)
        self._streams = {stream.cuda_stream}       # those that keep the workspace's memory
        self._last = stream                        # the one that used it last

    def _use_workspace(self, handle, other):
        """For a call on stream `handle` (`other`, or the current one where that is None) that works in the workspace:
        it follows the last such call, and the workspace's memory is not handed out again before it has run."""
        last = self._last
        if handle == last.cuda_stream:
            return
        stream = other or torch.cuda.current_stream(self.device)
        if handle not in self._streams:
            self.workspace.record_stream(stream)
            self._streams.add(handle)
        if not (_capturing(stream) or _capturing(last)):
            stream.wait_stream(last)
            self._last = stream

    def close(self):
        if getattr(self, "handle", None):
            _lib.als_serve_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# A call's checks take as long as its launch where the work is small, so they read each property of a tensor
# once and pass plain numbers on (an empty tensor's pointer is 0, which is NULL).  A tensor that is used on another
# stream than the current one is recorded there, so that its memory is not handed out again while the call may
# still run; the workspace on every stream but the one that it was allocated on.


def _stream(ctx: Context, stream):
    """(handle, stream or None): the stream of a call, and the stream itself where it is not the current one."""
    if not ctx.handle:
        raise ValueError("the context is closed")
    current = torch._C._cuda_getCurrentRawStream(ctx.index)
    if stream is None:
        return current, None
    handle = stream.cuda_stream
    return handle, stream if handle != current else None


def _use(ctx: Context, t, name, dtypes):
    """Says what is wrong with a tensor's place or type."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.get_device() != ctx.index:
        raise ValueError(f"{name} is on {t.device}, the context on {ctx.device}")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(map(str, dtypes))}, got {t.dtype}")


def _empty(ctx: Context, shape, dtype, other):
    """Allocated on the call's stream."""
    if other is None:
        return torch.empty(shape, dtype=dtype, device=ctx.device)
    with torch.cuda.stream(other):
        return torch.empty(shape, dtype=dtype, device=ctx.device)


def _vector(ctx: Context, t, name, dtypes, length, other):
    """Pointer of a contiguous vector of that length."""
    try:
        if (t.dtype in dtypes and t.get_device() == ctx.index and t.dim() == 1 and t.numel() == length
                and t.is_contiguous()):
            if other is not None:
                t.record_stream(other)
            return t.data_ptr()
    except AttributeError:
        pass
    _use(ctx, t, name, dtypes)
    if t.dim() != 1 or t.numel() != length:
        raise ValueError(f"{name} must have {length} elements, has shape {tuple(t.shape)}")
    raise ValueError(f"{name} must be contiguous")


def _matrix(ctx: Context, t, name, dtypes, rows, cols, other):
    """(pointer, row stride, rows, columns) of a matrix whose rows are contiguous, at any distance."""
    try:
        fits = t.dtype in dtypes and t.get_device() == ctx.index and t.dim() == 2
    except AttributeError:
        fits = False
    if not fits:
        _use(ctx, t, name, dtypes)
    shape = t.shape
    if not fits or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        want = ("any" if rows is None else rows, "any" if cols is None else cols)
        raise ValueError(f"{name} must be a matrix of {want[0]} x {want[1]}, has shape {tuple(shape)}")
    rows, cols = shape
    ld, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    if ld < cols:
        if rows > 1:
            raise ValueError(f"the rows of {name} overlap")
        ld = cols
    if other is not None:
        t.record_stream(other)
    return t.data_ptr(), ld, rows, cols


_I8, _I32, _I64, _F32, _FLOATS = (torch.int8,), (torch.int32,), (torch.int64,), (torch.float32,), tuple(_DTYPES)


def _own_columns(q, rows, f, ldq):
    """How many columns of each row of a given q may be written: those of the view, and its padding only where
    the rows start their memory's and leave no room for another such matrix.  (No operator needs the zeros.)"""
    start, width = q.storage_offset(), min(ldq, (f + 15) // 16 * 16)
    if ldq < 2 * f and start % ldq == 0 and start + (rows - 1) * ldq + width <= q.untyped_storage().nbytes():
        return width
    return f


def als_quantize(ctx: Context, x, users=None, q=None, scale=None, stream=None):
    """(q, scale): the rows of x (f32, f16 or bf16), or the rows `users` (int32) of it, as 8-bit integers
    with one scale each, x ~ scale q.  Without `q` the result is a view of rows whose stride is the next
    multiple of 16, with zeros up to it.  A given `q` may have any row stride; nothing but its elements is written,
    with one exception: where its rows start those of the memory that it is a view of, and are too short a distance
    apart for a second matrix like it (less than 2 f), zeros go up to the next multiple of 16 as far as the stride."""
    handle, other = _stream(ctx, stream)
    px, ldx, of, f = _matrix(ctx, x, "x", _FLOATS, None, None, other)
    rows, pu = of, None
    if users is not None:
        rows = users.numel()
        pu = _vector(ctx, users, "users", _I32, rows, other)
    if q is None:
        ldq = (f + 15) // 16 * 16
        q = _empty(ctx, (rows, ldq), torch.int8, other)
        pq, width = q.data_ptr(), ldq
        if ldq != f:
            q = q[:, :f]
    else:
        pq, ldq, _, _ = _matrix(ctx, q, "q", _I8, rows, f, other)
        width = f if ldq == f else _own_columns(q, rows, f, ldq)
    if scale is None:
        scale = _empty(ctx, (rows,), torch.float32, other)
        ps = scale.data_ptr()
    else:
        ps = _vector(ctx, scale, "scale", _F32, rows, other)
    if f > ALS_SERVE_F_MAX:
        f = width = _REFUSED
    rc = _lib.als_quantize_into(ctx.handle, px, _DTYPES[x.dtype], of, ldx, pu, rows, f, pq, ldq, width, ps, handle)
    if rc:
        _check("als_quantize", rc, ctx.handle)
    return q, scale


def als_score(ctx: Context, xq, xs, tq, ts, out=None, dtype=torch.float32, stream=None):
    """out[i, j] = xs_i ts_j sum_k xq_ik tq_jk for 8-bit rows with a scale each; out (f32, f16 or bf16, `dtype`
    where it is not given) may have any row stride."""
    handle, other = _stream(ctx, stream)
    px, ldx, m, f = _matrix(ctx, xq, "xq", _I8, None, None, other)
    pt, ldt, n, _ = _matrix(ctx, tq, "tq", _I8, None, f, other)
    if out is None:
        if dtype not in _DTYPES:
            raise TypeError(f"dtype must be {' or '.join(map(str, _DTYPES))}, got {dtype}")
        out = _empty(ctx, (m, n), dtype, other)
        po, ldo = out.data_ptr(), n
    else:
        dtype = out.dtype
        po, ldo, _, _ = _matrix(ctx, out, "out", _FLOATS, m, n, other)
    if (px | ldx | pt | ldt) & 15 or ldx >= _FAR or ldt >= _FAR:      # these rows are laid out anew
        ctx._use_workspace(handle, other)
    rc = _lib.als_score(ctx.handle, px, ldx, _vector(ctx, xs, "xs", _F32, m, other), m, pt, ldt,
                        _vector(ctx, ts, "ts", _F32, n, other), n, f if f <= ALS_SERVE_F_MAX else _REFUSED, po,
                        _DTYPES[dtype], ldo, handle)
    if rc:
        _check("als_score", rc, ctx.handle)
    return out


def _apart(p, rows, rated):
    """Refuses results on the left-out columns, of which the library does not know how many there are."""
    if rated is not None and p < rated[1].data_ptr() + 4 * rated[1].numel() and rated[1].data_ptr() < p + 4 * rows:
        raise ALSError("als_sample", ALS_ERR_ALIAS)


def als_sample(ctx: Context, scores, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, rated=None, users=None,
               index=None, log=None, stream=None):
    """(index, log): one column a row of `scores`, drawn by the uniform numbers `u` (float32, one a row), and the
    logarithm of its probability.  temperature, top_k, top_p and min_p are numbers, or tensors with one value
    a row (float32; top_k int32); `rated` = (rowptr, colidx) is a CSR of columns to leave out, row users[r] (int32)
    of it for row r, or row r.  See als_sample in include/als_serve.h for the definition."""
    handle, other = _stream(ctx, stream)
    pz, ldz, rows, n = _matrix(ctx, scores, "scores", _FLOATS, None, None, other)
    lim = ctx._limits
    lim.temperature = lim.top_k = lim.top_p = lim.min_p = None
    if isinstance(temperature, torch.Tensor):
        lim.temperature = _vector(ctx, temperature, "temperature", _F32, rows, other)
    else:
        lim.temperature_all = temperature
    if isinstance(top_k, torch.Tensor):
        lim.top_k = _vector(ctx, top_k, "top_k", _I32, rows, other)
    else:
        lim.top_k_all = min(max(int(top_k), 0), _INT32_MAX)
    if isinstance(top_p, torch.Tensor):
        lim.top_p = _vector(ctx, top_p, "top_p", _F32, rows, other)
    else:
        lim.top_p_all = top_p
    if isinstance(min_p, torch.Tensor):
        lim.min_p = _vector(ctx, min_p, "min_p", _F32, rows, other)
    else:
        lim.min_p_all = min_p
    pp = pi = pu = None
    of = 0
    if rated is not None:
        rowptr, colidx = rated
        of = rowptr.numel() - 1
        pp = _vector(ctx, rowptr, "rated[0]", _I64, of + 1, other)
        # (of a CSR without entries nothing is read)
        pi = _vector(ctx, colidx, "rated[1]", _I32, colidx.numel(), other) or pp
        if users is not None:
            pu = _vector(ctx, users, "users", _I32, rows, other)
        elif of < rows:
            raise ValueError(f"rated has {of} rows, scores {rows}")
    elif users is not None:
        raise ValueError("users without rated")
    if index is None:
        index = _empty(ctx, (rows,), torch.int32, other)
        p_index = index.data_ptr()
    else:
        p_index = _vector(ctx, index, "index", _I32, rows, other)
        _apart(p_index, rows, rated)
    if log is None:
        log = _empty(ctx, (rows,), torch.float32, other)
        p_log = log.data_ptr()
    else:
        p_log = _vector(ctx, log, "log", _F32, rows, other)
        _apart(p_log, rows, rated)
    if n > ALS_SERVE_HELD_MAX:
        ctx._use_workspace(handle, other)
    rc = _lib.als_sample(ctx.handle, pz, _DTYPES[scores.dtype], rows, n, ldz, ctx._limits_ref,
                         _vector(ctx, u, "u", _F32, rows, other), pp, pi, pu, of, p_index, p_log, handle)
    if rc:
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
