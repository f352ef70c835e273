"""How probable items are under a trained factor model: ctypes binding of libals_predict.so (include/als_predict.h),
marshalling torch tensors, and a model that evaluates and fits its offsets with it.

``als_predict`` gives predictions at the factors' own precision, with offsets, an activation and a residual;
``als_log_prob`` takes rows of scores as distributions and gives the log probabilities of items in them, their entropy
and best items; ``als_log_prob_grad`` is its gradient.  ``Predictor`` holds a model's factors and offsets.  All
arithmetic runs in the library's kernels; importing this module fails loudly when libals_predict.so is not built, or
libals_serve.so, with whose binding it shares the handling of tensors: there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import NamedTuple

import torch

from . import serve
from .als import ALS_OK, ALSError
from .serve import _empty, _matrix, _stream, _use, _vector

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libals_predict.so")

ALS_ERR_ALIAS = -6
ALS_PREDICT_F_MAX = 1_048_576
ALS_PREDICT_N_MAX = 4_194_304
ALS_PREDICT_TOP_MAX = 128
EXPORTED = ("als_predict_workspace_bytes", "als_predict_init", "als_predict_destroy", "als_predict_last_hip_error",
            "als_predict", "als_log_prob", "als_log_prob_grad")
ACTIVATIONS = {"none": 0, "clip": 1, "relu": 2, "gelu": 3, "silu": 4, "sigmoid": 5, "tanh": 6}
_INT32_MAX = 2 ** 31 - 1
_DTYPES = serve._DTYPES
_I32, _I64, _F32, _FLOATS = serve._I32, serve._I64, serve._F32, serve._FLOATS


class _Scores(ctypes.Structure):
    _fields_ = [("z", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("rows", ctypes.c_int64), ("n", ctypes.c_int64),
                ("ldz", ctypes.c_int64), ("temperature", ctypes.c_void_p), ("temperature_all", ctypes.c_float),
                ("rated_ptr", ctypes.c_void_p), ("rated_idx", ctypes.c_void_p), ("users", ctypes.c_void_p),
                ("of", ctypes.c_int64)]


class _Given(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("idx", ctypes.c_void_p), ("entries", ctypes.c_int64),
                ("each", ctypes.c_int64)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libals_predict.so is not built ({LIB_PATH}); run __graft_entry__.build() or "
                          "python paper_1603_03820_amd/build.py")
    lib = ctypes.CDLL(LIB_PATH)
    P, i64, i32, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float
    S, G = ctypes.POINTER(_Scores), ctypes.POINTER(_Given)
    lib.als_predict_workspace_bytes.argtypes = [ctypes.c_int]
    lib.als_predict_workspace_bytes.restype = ctypes.c_size_t
    lib.als_predict_init.argtypes = [ctypes.POINTER(P), ctypes.c_int, P, ctypes.c_size_t]
    lib.als_predict_destroy.argtypes = [P]
    lib.als_predict_last_hip_error.argtypes = [P]
    lib.als_predict.argtypes = [P, P, i64, i64, P, i64, P, i64, i64, i32, i32, P, P, i32, f32, f32, P, i64, P, i64,
                                i32, P]
    lib.als_log_prob.argtypes = [P, S, G, P, P, P, i32, P, P, P]
    lib.als_log_prob_grad.argtypes = [P, S, G, P, P, P, P, P, P, i64, P, P]
    for fn in EXPORTED[1:]:
        getattr(lib, fn).restype = ctypes.c_int
    return lib


_lib = _load()


def _check(fn: str, rc: int, ctx=None):
    if rc != ALS_OK:
        raise ALSError(fn, rc, _lib.als_predict_last_hip_error(ctx) if ctx is not None else 0)


def als_predict_workspace_bytes(device: int = 0) -> int:
    return int(_lib.als_predict_workspace_bytes(device))


class Context(serve.Context):
    """An als_predict_ctx plus the workspace tensor it runs in (one per device).  Its calls work in the workspace, and
    follow one another also where they are on different streams, as those of serve.Context do.  Calls that are captured
    into a graph do not: whoever launches it keeps its launches, and the eager calls beside them, apart, and keeps the
    context as long as the graph."""

    def __init__(self, device: int = 0):
        self.device = torch.device("cuda", device)
        self.index = device
        nbytes = als_predict_workspace_bytes(device)
        if nbytes == 0:
            raise RuntimeError(f"als_predict_workspace_bytes failed for device {device} (not gfx950?)")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        h = ctypes.c_void_p()
        _check("als_predict_init", _lib.als_predict_init(ctypes.byref(h), device,
                                                         ctypes.c_void_p(self.workspace.data_ptr()), nbytes))
        self.handle = h
        self._start(torch.cuda.current_stream(self.device))

    def _start(self, stream):
        super()._start(stream)
        self._scores, self._given = _Scores(), _Given()
        self._scores_ref, self._given_ref = ctypes.byref(self._scores), ctypes.byref(self._given)

    def close(self):
        if getattr(self, "handle", None):
            _lib.als_predict_destroy(self.handle)
            self.handle = None


# Results are allocated as other tensors' kin (new_empty), which takes half of torch.empty's time: a small call's allocations
# take longer than its kernel.


def _count(ctx: Context, t, name, dtypes):
    """A tensor's elements; what is no tensor is refused."""
    try:
        return t.numel()
    except AttributeError:
        _use(ctx, t, name, dtypes)


def _like(ctx: Context, t, shape, dtype, other):
    """Allocated on the call's stream; t is a tensor on the context's device."""
    if other is None:
        return t.new_empty(shape) if t.dtype == dtype else t.new_empty(shape, dtype=dtype)
    return _empty(ctx, shape, dtype, other)      # (a number is a vector's length)


def als_predict(ctx: Context, x, theta, users=None, user_offset=None, item_offset=None, activation="none",
                low=None, high=None, residual=None, out=None, dtype=torch.float32, stream=None):
    """out[i, j] = act(x[u] . theta[j] + user_offset[u] + item_offset[j]) + residual[i, j] with u = users[i] (int32), or
    i.  x and theta are matrices of one type (f32, f16 or bf16), the offsets vectors (float32) with an element for each row
    of x and of theta; `activation` is a name of ACTIVATIONS, "clip" between `low` and `high` (None: no bound); `residual`
    has the type of out, and may be it.  out (f32, f16 or bf16, `dtype` where it is not given) may have any row stride."""
    handle, other = _stream(ctx, stream)
    px, ldx, of, f = _matrix(ctx, x, "x", _FLOATS, None, None, other)
    pt, ldt, n, _ = _matrix(ctx, theta, "theta", (x.dtype,), None, f, other)
    m, pu = of, None
    if users is not None:
        m = _count(ctx, users, "users", _I32)
        pu = _vector(ctx, users, "users", _I32, m, other)
    pa = None if user_offset is None else _vector(ctx, user_offset, "user_offset", _F32, of, other)
    pb = None if item_offset is None else _vector(ctx, item_offset, "item_offset", _F32, n, other)
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}, got {activation!r}")
    if activation != "clip" and not (low is None and high is None):
        raise ValueError("low and high are clip's")
    if out is None:
        if dtype not in _DTYPES:
            raise TypeError(f"dtype must be {' or '.join(map(str, _DTYPES))}, got {dtype}")
        out = _like(ctx, x, (m, n), dtype, other)
        po, ldo = out.data_ptr(), n
    else:
        po, ldo, _, _ = _matrix(ctx, out, "out", _FLOATS, m, n, other)
        dtype = out.dtype
    pr, ldr = None, n
    if residual is not None:
        pr, ldr, _, _ = _matrix(ctx, residual, "residual", (dtype,), m, n, other)
    ctx._use_workspace(handle, other)
    rc = _lib.als_predict(ctx.handle, px, of, ldx, pu, m, pt, n, ldt, _DTYPES[x.dtype],
                          f if f <= ALS_PREDICT_F_MAX else ALS_PREDICT_F_MAX + 1, pa, pb, ACTIVATIONS[activation],
                          float("-inf") if low is None else low, float("inf") if high is None else high, pr, ldr, po,
                          ldo, _DTYPES[dtype], handle)
    if rc:
        _check("als_predict", rc, ctx.handle)
    return out


class LogProb(NamedTuple):
    """What als_log_prob gives: log has the given columns' shape, stats is rows x 2, entropy one value a row; the best
    columns and their log p are rows x top (None where top is 0)."""
    log: torch.Tensor
    stats: torch.Tensor
    entropy: torch.Tensor
    top_index: torch.Tensor | None
    top_log: torch.Tensor | None


def _of_rows(ctx, scores, given, temperature, rated, users, other):
    """Fills in the context's als_scores and als_given; (rows, columns, the shape of a value for each given column)."""
    s, g = ctx._scores, ctx._given
    s.z, s.ldz, rows, n = _matrix(ctx, scores, "scores", _FLOATS, None, None, other)
    s.rows, s.n, s.dtype = rows, n, _DTYPES[scores.dtype]
    if isinstance(temperature, torch.Tensor):
        s.temperature = _vector(ctx, temperature, "temperature", _F32, rows, other)
    else:
        s.temperature, s.temperature_all = None, temperature
    s.rated_ptr = s.rated_idx = s.users = None
    s.of = 0
    if rated is not None:
        rowptr, colidx = rated
        of = _count(ctx, rowptr, "rated[0]", _I64) - 1
        s.of = of
        s.rated_ptr = _vector(ctx, rowptr, "rated[0]", _I64, of + 1, other)
        # (of a CSR without entries nothing is read)
        s.rated_idx = _vector(ctx, colidx, "rated[1]", _I32, _count(ctx, colidx, "rated[1]", _I32), other) or s.rated_ptr
        if users is not None:
            s.users = _vector(ctx, users, "users", _I32, rows, other)
        elif of < rows:
            raise ValueError(f"rated has {of} rows, scores {rows}")
    elif users is not None:
        raise ValueError("users without rated")
    if isinstance(given, tuple):
        ptr, idx = given
        entries = _count(ctx, idx, "given[1]", _I32)
        shape = (entries,)
        g.ptr = _vector(ctx, ptr, "given[0]", _I64, rows + 1, other)
        g.idx = _vector(ctx, idx, "given[1]", _I32, entries, other)
        g.entries, g.each = entries, 0
    else:
        try:
            shape, entries = given.shape, given.numel()
        except AttributeError:
            _use(ctx, given, "given", _I32)
        if len(shape) not in (1, 2) or shape[0] != rows:
            raise ValueError(f"given must be a value or a row of them for each of {rows} rows, has shape {tuple(shape)}")
        g.ptr = None
        g.idx = _shaped(ctx, given, "given", shape, other, _I32)
        g.entries, g.each = entries, entries // rows if rows else 0
    return rows, n, shape


def _shaped(ctx, t, name, shape, other, dtypes=_F32):
    """Pointer of a contiguous tensor of that shape."""
    try:
        if t.dtype in dtypes and t.get_device() == ctx.index and t.shape == shape and t.is_contiguous():
            if other is not None:
                t.record_stream(other)
            return t.data_ptr()
    except AttributeError:
        pass
    _use(ctx, t, name, dtypes)
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, has {tuple(t.shape)}")
    raise ValueError(f"{name} must be contiguous")


def _apart(fn, results, rated):
    """Refuses results on the left-out columns, of which the library does not know how many there are."""
    if rated is None:
        return
    start, end = rated[1].data_ptr(), rated[1].data_ptr() + 4 * rated[1].numel()
    for p, words in results:
        if p < end and start < p + 4 * words:
            raise ALSError(fn, ALS_ERR_ALIAS)


def als_log_prob(ctx: Context, scores, given, temperature=1.0, top=0, rated=None, users=None, log=None, stream=None):
    """LogProb of rows of `scores` (f32, f16 or bf16) as distributions over their columns, softmax(scores /
    temperature).  `given` (int32) are the columns asked about: one a row, a matrix with a row of them each (contiguous), or
    (rowptr, colidx), a CSR with a row for each row of scores.  temperature is a number or a tensor with one value a row
    (float32); `rated` = (rowptr, colidx) is a CSR of columns to leave out, row users[r] (int32) of it for row r, or row
    r.  `top` best columns are given beside them.  See als_log_prob in include/als_predict.h for the definition."""
    handle, other = _stream(ctx, stream)
    rows, _, shape = _of_rows(ctx, scores, given, temperature, rated, users, other)
    top = int(top)
    if not 0 <= top <= ALS_PREDICT_TOP_MAX:
        raise ValueError(f"top must be 0 to {ALS_PREDICT_TOP_MAX}, is {top}")
    stats = _like(ctx, scores, (rows, 2), torch.float32, other)
    if log is None:
        log = _like(ctx, stats, shape, torch.float32, other)
        pl = log.data_ptr()
    else:
        pl = _shaped(ctx, log, "log", shape, other)
        _apart("als_log_prob", ((pl, log.numel()),), rated)
    entropy = _like(ctx, stats, rows, torch.float32, other)
    top_index = top_log = pi = pt = None
    if top:
        top_log = _like(ctx, stats, (rows, top), torch.float32, other)
        top_index = _like(ctx, given[1] if isinstance(given, tuple) else given, (rows, top), torch.int32, other)
        pi, pt = top_index.data_ptr(), top_log.data_ptr()
    ctx._use_workspace(handle, other)
    rc = _lib.als_log_prob(ctx.handle, ctx._scores_ref, ctx._given_ref, pl, stats.data_ptr(), entropy.data_ptr(), top,
                           pi, pt, handle)
    if rc:
        _check("als_log_prob", rc, ctx.handle)
    return LogProb(log, stats, entropy, top_index, top_log)


def als_log_prob_grad(ctx: Context, scores, given, forward: LogProb, grad_log, grad_entropy=None, temperature=1.0,
                      rated=None, users=None, grad=True, columns=False, stream=None):
    """(grad, columns): the gradient of sum(grad_log * log) + sum(grad_entropy * entropy) with respect to the scores, in
    their type, and its sums over the rows in float32 -- the gradient of offsets that are added to every row.  `forward`
    is what als_log_prob gave for the same scores, given, temperature, rated and users; grad_log has the shape of its log,
    grad_entropy one value a row.  `grad` and `columns` are True, False, or the tensor to write to (`grad` may be `scores`
    itself); what is False is not computed, and None is in its place."""
    handle, other = _stream(ctx, stream)
    rows, n, shape = _of_rows(ctx, scores, given, temperature, rated, users, other)
    pl = _shaped(ctx, forward.log, "forward.log", shape, other)
    ps = _shaped(ctx, forward.stats, "forward.stats", (rows, 2), other)
    pg = _shaped(ctx, grad_log, "grad_log", shape, other)
    pe = ph = None
    if grad_entropy is not None:
        pe = _vector(ctx, forward.entropy, "forward.entropy", _F32, rows, other)
        ph = _vector(ctx, grad_entropy, "grad_entropy", _F32, rows, other)
    po, ldg, pc = None, n, None
    if isinstance(grad, torch.Tensor):
        po, ldg, _, _ = _matrix(ctx, grad, "grad", (scores.dtype,), rows, n, other)
        if rows and n:
            _apart("als_log_prob_grad", ((po, (((rows - 1) * ldg + n) * grad.element_size() + 3) // 4),), rated)
    elif grad:
        grad = _like(ctx, scores, (rows, n), scores.dtype, other)
        po = grad.data_ptr()
    else:
        grad = None
    if isinstance(columns, torch.Tensor):
        pc = _vector(ctx, columns, "columns", _F32, n, other)
        _apart("als_log_prob_grad", ((pc, n),), rated)
    elif columns:
        columns = _like(ctx, forward.stats, n, torch.float32, other)
        pc = columns.data_ptr()
    else:
        columns = None
    if pc:
        ctx._use_workspace(handle, other)
    rc = _lib.als_log_prob_grad(ctx.handle, ctx._scores_ref, ctx._given_ref, pl, ps, pe, pg, ph, po, ldg, pc, handle)
    if rc:
        _check("als_log_prob_grad", rc, ctx.handle)
    return grad, columns


class Predictor:
    """A trained model's predictions and what they say of items: factors x and theta, an offset for each user and item
    (float32, or None), and `rated`, the CSR of the training ratings, which its users are not recommended again.  The offsets
    belong to the scores whatever they are for: those that fit_offsets leaves are part of what predict gives from then on."""

    def __init__(self, ctx: Context, x, theta, user_offset=None, item_offset=None, rated=None):
        self.ctx, self.x, self.theta, self.rated = ctx, x, theta, rated
        self.user_offset, self.item_offset = user_offset, item_offset

    def predict(self, users=None, low=None, high=None, dtype=torch.float32, stream=None):
        """The predicted ratings of `users` (int32 rows of X; all of them) for every item, between `low` and `high`.  (Where the
        items' offsets were fitted to choices, by fit_offsets, these are scores of choice and no longer ratings: predict ratings
        with a Predictor of the offsets before.)"""
        clip = low is not None or high is not None
        return als_predict(self.ctx, self.x, self.theta, users, self.user_offset, self.item_offset,
                           "clip" if clip else "none", low, high, dtype=dtype, stream=stream)

    def _left_out(self, users):
        return dict(rated=self.rated, users=None if self.rated is None else users)

    def log_prob(self, users, given, temperature=1.0, top=0, log=None, stream=None):
        """LogProb of the items `given` (see als_log_prob) among those that `users` (int32) have not rated.  For a user that is
        no row of x no item is allowed (log p -inf); for one that `rated` has no row of, all results are NaN."""
        z = als_predict(self.ctx, self.x, self.theta, users, None, self.item_offset, stream=stream)
        return als_log_prob(self.ctx, z, given, temperature, top, log=log, stream=stream, **self._left_out(users))

    def fit_offsets(self, users, given, temperature=1.0, steps=20, rate=1.0, batch=1024):
        """Raises the mean log probability of `given` (int32, an item for each of `users`) by the items' offsets, and
        returns that mean before each of `steps` steps.  A step compares how often an item is given (c) with how often
        the model expects it (e), whose difference is T times the gradient, and moves its offset by rate T (c - e) / max(c, e):
        at most by T.  Users are taken `batch` at a time.  Items that a user has rated are left out for them; given
        ones among those count for nothing, and so does what is given for a user that there is not (no row of x, or none of
        `rated`).  The temperature is one number; one that is not above 0 leaves the offsets as they are."""
        if isinstance(temperature, torch.Tensor):
            raise TypeError("temperature must be a number")
        n, count = self.theta.shape[0], _count(self.ctx, users, "users", _I32)
        _count(self.ctx, given, "given", _I32)
        if users.dim() != 1 or count == 0 or given.shape != users.shape:
            raise ValueError(f"given must have an item for each of {count} users (one at least), has shape {tuple(given.shape)}")
        # (a row of a user that there is not has NaN in every column of its gradient)
        of = self.x.shape[0] if self.rated is None else min(self.x.shape[0], self.rated[0].numel() - 1)
        there = (users >= 0) & (users < of)
        users, given = users[there], given[there]
        count = users.numel()
        # the gradient of an offset is up to count / T, a step up to rate T
        largest = torch.finfo(torch.float32).max
        if not (abs(temperature) * max(1.0, abs(rate)) <= largest and (temperature <= 0 or count <= temperature * largest)):
            raise ValueError(f"temperature, rate times it and {count} / temperature must be in float32's range, is {temperature}")
        if self.item_offset is None:
            self.item_offset = torch.zeros(n, dtype=torch.float32, device=self.theta.device)
        means = []
        for _ in range(steps):
            short, counts = torch.zeros_like(self.item_offset), torch.zeros_like(self.item_offset)
            total = torch.zeros((), dtype=torch.float64, device=users.device)
            used = torch.zeros((), dtype=torch.int64, device=users.device)
            for k in range(0, count, batch):
                u, g = users[k:k + batch], given[k:k + batch]
                z = als_predict(self.ctx, self.x, self.theta, u, None, self.item_offset)
                r = als_log_prob(self.ctx, z, g, temperature, **self._left_out(u))
                _, columns = als_log_prob_grad(self.ctx, z, g, r, torch.ones_like(r.log), temperature=temperature,
                                               grad=False, columns=True, **self._left_out(u))
                there = r.log > float("-inf")
                short += columns
                counts.index_add_(0, g.clamp(0, n - 1), there.float())
                total = total + torch.where(there, r.log, 0.0).double().sum()
                used = used + there.sum()
            means.append(total / used.clamp(min=1))
            short *= temperature
            most = torch.maximum(counts, counts - short).clamp_(min=1e-6)
            self.item_offset = self.item_offset + (rate * temperature) * (short / most)
        return [float(m) for m in means]
