"""Plain 64-bit forms of the prediction operators (numpy and math, on the host), and the bounds that their results have
to keep.  Each bound is a count of roundings of fp32 (half a unit in the last place is 2^-24 of a value), and the
output's own where it has fewer bits."""
import math

import numpy as np

HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}     # the least positive value
U = 2.0 ** -24

_erf = np.vectorize(math.erf, otypes=[np.float64])
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def activate(y, name, low=-np.inf, high=np.inf):
    with np.errstate(over="ignore", invalid="ignore"):
        if name == "none":
            return y
        if name == "clip":
            return np.minimum(np.maximum(y, low), high)
        if name == "relu":
            return np.maximum(y, 0.0)
        if name == "gelu":
            return np.where(y == -np.inf, -0.0, 0.5 * y * _erfc(-y / math.sqrt(2.0)))
        if name == "silu":
            return np.where(y == -np.inf, -0.0, y / (1.0 + np.exp(-y)))
        if name == "sigmoid":
            return 1.0 / (1.0 + np.exp(-y))
        assert name == "tanh"
        return np.tanh(y)


def predict(x, theta, users=None, user_offset=None, item_offset=None, activation="none", low=-np.inf, high=np.inf,
            residual=None):
    """(the result, the sums of the products' magnitudes and the offsets') in 64 bits; rows of users that do not exist
    are NaN."""
    x, theta = np.asarray(x, np.float64), np.asarray(theta, np.float64)
    users = np.arange(x.shape[0]) if users is None else np.asarray(users)
    there = (users >= 0) & (users < x.shape[0])
    xs = np.where(there[:, None], x[np.where(there, users, 0)], np.nan) if x.shape[0] else np.full((users.size, x.shape[1]), np.nan)
    y, size = xs @ theta.T, np.abs(xs) @ np.abs(theta).T
    if user_offset is not None and x.shape[0]:
        a = np.asarray(user_offset, np.float64)[np.where(there, users, 0)][:, None]
        y, size = y + a, size + np.abs(a)
    if item_offset is not None:
        b = np.asarray(item_offset, np.float64)
        with np.errstate(invalid="ignore"):
            y, size = y + b, size + np.abs(b)
    out = activate(y, activation, low, high)
    if residual is not None:
        out = out + np.asarray(residual, np.float64)
    return out, size


def predict_bound(out, size, f, dtype, out_dtype, activation="none", residual=None):
    """How far a result may be off: f additions of products (2^-23 each of the magnitudes' sum, as a matrix
    instruction's inner additions need not round to nearest), two for the offsets; fp32's products, six for each, lack
    2^-7 2^-16 of them twice and 2^-32, and their parts' own products are exact.  An activation's slope is at most
    1.13, its own error 16 units of its value and 2^-22 where GELU's argument, rounded, goes into an exponential; the
    residual's sum rounds once, then the output."""
    products = 6 if dtype == "f32" else 1
    off = size * ((products * f + 2) * 2 * U + (2.0 ** -22 + 2.0 ** -32 if dtype == "f32" else 0.0))
    if activation not in ("none", "clip", "relu"):
        off = 1.13 * off + 16 * 2 * U * np.abs(out if residual is None else out - residual) + 2.0 ** -22
    if residual is not None:
        off = off + U * np.abs(out)
    half = 0.0 if out_dtype == "f32" else HALF_ULP[out_dtype]
    return off * (1 + half) + half * np.abs(out) * (1 + 2.0 ** -7) + TINY[out_dtype]


class Row:
    """One row's distribution: `log_p` of every column (-inf where it is left out), entropy, the order of the allowed
    columns, and bounds on what fp32 makes of them."""

    def __init__(self, z, temperature=1.0, rated=(), there=True):
        z = np.asarray(z, np.float64)
        self.n, self.there = z.size, there
        allowed = z > -np.inf
        for c in rated:
            if 0 <= c < z.size:
                allowed[c] = False
        cols = np.nonzero(allowed)[0]
        self.cols = cols[np.lexsort((cols, -z[cols]))]
        self.t = temperature
        self.greedy = not temperature > 0
        self.log_p = np.full(z.size, -np.inf)
        self.entropy = 0.0
        self.best, self.size = -np.inf, -np.inf
        self.off_size = self.off_entropy = 0.0
        self.d = np.zeros(z.size)
        if cols.size == 0:
            return
        self.best = z[self.cols[0]]
        if self.greedy:
            self.log_p[self.cols[0]] = 0.0
            self.size = 0.0
            return
        with np.errstate(invalid="ignore", over="ignore"):
            diff = np.where(z[cols] == self.best, 0.0, z[cols] - self.best)
            diff = np.where(np.abs(diff) > np.finfo(np.float32).max, -np.inf, diff)     # past fp32 it weighs nothing
            y = np.where(diff == -np.inf, -np.inf, diff / temperature)
            y = np.where(np.abs(y) > np.finfo(np.float32).max, -np.inf, y)
        w = np.exp(y)
        self.size = math.log(w.sum())
        self.log_p[cols] = y - self.size
        p = w / w.sum()
        self.entropy = -(p[p > 0] * self.log_p[cols][p > 0]).sum()
        # a weight: difference, rate and their product of an exponent (in bits), the exponential's unit and the sums' (33
        # in a thread, 6 and 4 across it, as many across segments)
        bits = np.where(p > 0, np.abs(np.where(p > 0, y, 0.0)) / math.log(2.0), 0.0)
        off_w = 3 * U * bits * math.log(2.0) + 2.0 ** -22
        sums = 64 * U
        self.off_size = (p * off_w).sum() + sums + 2 * U * abs(self.size) + 2.0 ** -40 * z.size
        self.off_entropy = 2 * self.off_size + (p * bits * (off_w + sums + 4 * U)).sum() + 4 * U * (abs(self.size) + (p * bits).sum())
        self.d[cols] = np.where(np.isfinite(y), y, 0.0)

    def log(self, column):
        if not self.there:
            return np.nan
        return self.log_p[column] if 0 <= column < self.n else -np.inf

    def off_log(self, column):
        """Difference and quotient, then the size and the last difference."""
        if not 0 <= column < self.n or not np.isfinite(self.log_p[column]):
            return 0.0
        return 2 * U * abs(self.d[column]) + self.off_size + 2 * U * abs(self.log_p[column])

    def top(self, k):
        index = np.full(k, -1, np.int64)
        log = np.full(k, -np.inf if self.there else np.nan)
        if self.there:
            some = self.cols[:k]
            index[:some.size] = some
            log[:some.size] = self.log_p[some]
        return index, log

    def loss(self, given, g, h):
        log = np.array([self.log(c) for c in given], np.float64)
        kept = log > -np.inf
        return (np.asarray(g, np.float64)[kept] * log[kept]).sum() + h * self.entropy

    def gradient(self, given, g, h):
        """(gradient, bound) of loss."""
        grad, off = np.zeros(self.n), np.zeros(self.n)
        if not self.there:
            return np.full(self.n, np.nan), off
        if self.greedy or self.cols.size == 0:
            return grad, off
        p = np.exp(self.log_p)
        kept = [(c, w) for c, w in zip(given, np.asarray(g, np.float64)) if self.log(c) > -np.inf]
        total, weight = sum(w for _, w in kept), sum(abs(w) for _, w in kept)
        log_p = np.where(p > 0, self.log_p, 0.0)
        grad = -p * (total + h * (log_p + self.entropy))
        # p: the size's error, four roundings of an exponent and of the size beside it, the exponential's
        off_p = self.off_size + 4 * U * (np.abs(self.d) + abs(self.size)) + 2.0 ** -22
        inner = abs(total) + abs(h) * (np.abs(log_p) + self.entropy)
        off = p * (inner * (off_p + 4 * U) + (len(kept) + 8) * U * weight
                   + abs(h) * (self.off_entropy + off_p + 4 * U * (np.abs(log_p) + self.entropy)))
        per = np.zeros(self.n)
        for c, w in kept:
            grad[c] += w
            per[c] += abs(w)
        off += (len(kept) + 2) * U * per
        off = off + 4 * U * np.abs(grad) + 2.0 ** -126      # weights below 2^-126 are 0
        return grad / self.t, off / self.t
