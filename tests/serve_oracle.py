"""Plain 64-bit forms of the serving operators (numpy, on the host), and the bounds that their results have to
keep.  Each bound is a count of roundings: half a unit in the last place is 2^-24 of a value in fp32, 2^-11 in f16,
2^-8 in bf16 (9 and 12 significant bits less)."""
import numpy as np

HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}     # the least positive value


def quantize(x):
    """(q, scale) of float32 rows, with the definition's roundings."""
    x = np.asarray(x, dtype=np.float32)
    q = np.zeros(x.shape, dtype=np.int8)
    scale = np.zeros(x.shape[0], dtype=np.float32)
    for r, row in enumerate(x):
        if not np.all(np.isfinite(row)):
            scale[r] = np.nan
            continue
        a = np.abs(row).max() if row.size else np.float32(0)
        scale[r] = a * (np.float32(1) / np.float32(127))
        if a > 0:
            # past 1e36 both sides shrink by 2^8, which changes no quotient
            down = np.float32(2.0 ** -8) if a > 1e36 else np.float32(1)
            q[r] = np.rint((row * down) * np.float32(127) / (a * down)).astype(np.int8)
    return q, scale


def score(xq, xs, tq, ts):
    """Exact sums (64-bit integers) times both scales in 64-bit floats."""
    s = np.asarray(xq, dtype=np.int64) @ np.asarray(tq, dtype=np.int64).T
    return s.astype(np.float64) * np.asarray(xs, np.float64)[:, None] * np.asarray(ts, np.float64)


def score_bound(exact, dtype):
    """The sum's conversion and two products in fp32 (three roundings), then the output's: one more of its
    own type, or half its least value."""
    half = HALF_ULP[dtype]
    one = 3 * 2.0 ** -24 + (0 if dtype == "f32" else half)
    return np.abs(exact) * one * (1 + 2.0 ** -7) + TINY[dtype]


class Draw:
    """One row's draw in 64-bit floats.  ``accepts(index, log)`` allows for what the weights' roundings can move: a
    weight is off by at most EPS (difference, 1 / T, their product -- 2^-24 each of an exponent of at most 28 --
    and the exponential's 2^-23), and by 2^-40 of the largest for the rounding down."""

    EPS = 3 * 28 * 2.0 ** -24 + 2.0 ** -23
    STEP = 2.0 ** -40

    def __init__(self, z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, rated=()):
        z = np.asarray(z, dtype=np.float64)
        n = z.size
        allowed = z > -np.inf
        for c in rated:
            if 0 <= c < n:
                allowed[c] = False
        cols = np.nonzero(allowed)[0]
        self.none = cols.size == 0
        self.greedy = not temperature > 0
        if self.none:
            return
        order = cols[np.lexsort((cols, -z[cols]))]
        self.best = order[0]
        if self.greedy:
            return
        if 0 < top_k < order.size:
            order = order[:top_k]
        top = z[order[0]]
        with np.errstate(invalid="ignore", over="ignore"):
            e = np.where(z[order] == top, 1.0, np.exp((z[order] - top) / temperature))
        if top == np.inf:
            e = (z[order] == top).astype(np.float64)
        e[e < self.STEP * (1 - self.EPS)] = 0.0
        slack = self.EPS * e.sum() + self.STEP * e.size
        before = np.cumsum(e) - e
        surely, maybe = np.ones(e.size, bool), np.ones(e.size, bool)
        if top_p < 1:
            goal = max(0.0, top_p) * e.sum()
            off = 2 * slack + 2.0 ** -23 * e.sum()
            surely = before + off < goal
            maybe = before - off < goal
            surely[0] = maybe[0] = True
        if min_p > 0:
            least = min(min_p, 1.0)
            surely &= e >= least * (1 + self.EPS)
            maybe &= e >= least * (1 - self.EPS)
            surely[0] = maybe[0] = True
        self.u = min(max(u, 0.0), 1 - 2.0 ** -24)
        back = np.argsort(order, kind="stable")
        self.order, self.e = order[back], e[back]
        self.surely, self.maybe = surely[back], maybe[back]
        self.slack = slack

    def accepts(self, index, log):
        if self.none:
            return index == -1 and log == -np.inf
        if self.greedy:
            return index == self.best and log == 0
        at = np.nonzero(self.order == index)[0]
        if at.size == 0 or not self.maybe[at[0]] or self.e[at[0]] <= 0:
            return False
        at = at[0]
        least, most = self.e[self.surely].sum(), self.e[self.maybe].sum()
        front = self.e[:at][self.surely[:at]].sum() - self.slack
        end = self.e[:at + 1][self.maybe[:at + 1]].sum() + self.slack
        if not (front <= self.u * (most + self.slack) and
                end >= (self.u - 2.0 ** -23) * (least - self.slack)):
            return False
        # of the logarithm: the exponent's and the sum's errors, and two roundings of a value of at most 50
        off = 2 * self.EPS + self.slack / least + 100 * 2.0 ** -24
        w = np.log(self.e[at])
        return w - np.log(most) - off <= log <= w - np.log(least) + off
