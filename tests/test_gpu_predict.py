"""The prediction operators on the GPU against their plain 64-bit forms (tests/predict_oracle.py)."""
import ctypes

import numpy as np
import pytest
import torch

from tests import predict_oracle
from tests.gpu_util import log

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
D = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    from paper_1603_03820_amd import predict
    c = predict.Context(0)
    yield c
    c.close()


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(D)
    return t if dtype is None else t.to(dtype)


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def strided(t, extra, offset=0):
    """The matrix t as a view of rows that lie `extra` elements further apart, from element `offset` on, in
    memory that holds other values."""
    rows, cols = t.shape
    big = torch.full((rows * (cols + extra) + offset,), 77, dtype=t.dtype, device=t.device)
    v = big[offset:].view(rows, cols + extra)[:, :cols]
    v.copy_(t)
    return v


# ------------------------------------------------------------------------------- predict --

# users, items, f: one of each, below and above every tile's sides, f below, at and past a step
SHAPES = [(1, 1, 1), (1, 300, 7), (3, 65, 8), (16, 64, 64), (17, 63, 32), (15, 129, 33), (64, 64, 65), (70, 130, 100),
          (130, 257, 128), (5, 1000, 1000), (1, 70, 8192), (129, 128, 31), (200, 5000, 40), (1030, 6000, 16),
          (300, 17_770, 100), (33, 20_000, 130), (2, 3, 20_000)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,f", SHAPES)
def test_predict_whole_numbers(ctx, dtype, m, n, f):
    """Sums of products of whole numbers that fp32 holds: every bit has to be there, at any size."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(m * 31 + n * 7 + f)
    most = 3 if f > 1000 else 16
    x, t = rng.integers(-most, most + 1, (m, f)), rng.integers(-most, most + 1, (n, f))
    if dtype == "f32" and f <= 130:      # more bits than one part holds
        x = x * 129
    want = x.astype(np.int64) @ t.astype(np.int64).T
    assert np.abs(want).max() < 2 ** 24
    log(f"predict whole numbers {dtype} {m}x{n}x{f}")
    out = predict.als_predict(ctx, dev(x.astype(np.float32), TYPES[dtype]), dev(t.astype(np.float32), TYPES[dtype]))
    assert np.array_equal(f64(out), want.astype(np.float64))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,f", [(4101, 4105, 520), (4101, 4105, 515), (2300, 2100, 64), (2300, 2100, 200), (1100, 2100, 1000),
                                   (1500, 1400, 72), (600, 900, 4100), (20, 300, 9000), (16, 8192, 2048), (4096, 4097, 512),
                                   (31, 9000, 200), (32, 5000, 96), (310, 20_000, 520), (100, 20_000, 136)])
def test_predict_large(ctx, dtype, m, n, f):
    """Enough tiles for every shape of them, and few that are cut along f: whole numbers against 64-bit products, rows taken
    by index and in order."""
    from paper_1603_03820_amd import predict
    gen = torch.Generator(device=D).manual_seed(m + n + f)
    x, t = (torch.randint(-3, 4, (r, f), device=D, generator=gen).to(TYPES[dtype]) for r in (m + 3, n))
    users = torch.randint(0, m + 3, (m,), device=D, generator=gen, dtype=torch.int32)
    log(f"predict {dtype} {m}x{n}x{f}")
    want = x.double() @ t.double().t()
    assert torch.equal(predict.als_predict(ctx, x, t).double(), want)
    assert torch.equal(predict.als_predict(ctx, x, t, users=users).double(), want[users.long()])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("extra,offset", [(0, 1), (1, 0), (3, 5), (4, 8), (8, 0), (7, 2)])
@pytest.mark.parametrize("f", [5, 64, 100, 130])
def test_predict_strides(ctx, dtype, f, extra, offset):
    """Rows at every alignment of their elements, whose neighbours in memory are NaN; results, residuals and users too."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(f + extra)
    m, n = 37, 150
    x, t = rng.integers(-9, 10, (m, f)), rng.integers(-9, 10, (n, f))
    res = rng.integers(-9, 10, (20, n))
    users = rng.integers(0, m, 20).astype(np.int32)
    users[3], users[19] = -1, m
    want = (x.astype(np.int64) @ t.astype(np.int64).T)[np.where((users < 0) | (users >= m), 0, users)] + res
    xd, td = strided(dev(x.astype(np.float32), TYPES[dtype]), extra, offset), strided(dev(t.astype(np.float32), TYPES[dtype]), extra, offset)
    for v, keep in ((xd, x), (td, t)):
        whole = torch.as_strided(v, (v.untyped_storage().nbytes() // v.element_size(),), (1,), 0)
        whole.fill_(float("nan"))
        v.copy_(dev(keep.astype(np.float32)))
    log(f"predict strides {dtype} f {f} + {extra} from {offset}")
    out = strided(torch.zeros(20, n, device=D), extra, offset)
    rd = strided(dev(res.astype(np.float32)), 2 * extra, offset)
    got = predict.als_predict(ctx, xd, td, users=dev(users), residual=rd, out=out)
    assert got is out
    got = f64(out)
    bad = (users < 0) | (users >= m)
    assert np.isnan(got[bad]).all() and np.array_equal(got[~bad], want[~bad].astype(np.float64))
    whole = torch.as_strided(out, (out.untyped_storage().nbytes() // 4,), (1,), 0)
    beside = torch.ones_like(whole, dtype=torch.bool)
    torch.as_strided(beside, (20, n), (n + extra, 1), offset).fill_(False)
    assert bool((whole[beside] == 77).all())


@pytest.mark.parametrize("dtype,out_dtype", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("m,n,f", [(1, 50, 1), (19, 130, 16), (70, 200, 100), (3, 100, 3000), (130, 140, 128)])
def test_predict_values(ctx, dtype, out_dtype, m, n, f):
    """Real values with offsets, in every type; at f = 1 the bound is a few units of fp32."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(f * 3 + m)
    x = dev((rng.standard_normal((m, f)) * np.exp(rng.standard_normal((m, 1)))).astype(np.float32), TYPES[dtype])
    t = dev(rng.standard_normal((n, f)).astype(np.float32), TYPES[dtype])
    a, b = rng.standard_normal(m).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    log(f"predict values {dtype} to {out_dtype} {m}x{n}x{f}")
    got = f64(predict.als_predict(ctx, x, t, user_offset=dev(a), item_offset=dev(b), dtype=TYPES[out_dtype]))
    want, size = predict_oracle.predict(f64(x), f64(t), None, a, b)
    assert np.all(np.abs(got - want) <= predict_oracle.predict_bound(want, size, f, dtype, out_dtype))


@pytest.mark.parametrize("out_dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("name", ["none", "clip", "relu", "gelu", "silu", "sigmoid", "tanh"])
@pytest.mark.parametrize("m", [3, 40])
def test_predict_activations(ctx, name, out_dtype, m):
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(m)
    n, f = 210, 20
    x = rng.standard_normal((m, f)).astype(np.float32)
    t = (rng.standard_normal((n, f)) * np.exp(rng.uniform(-3, 1.5, (n, 1)))).astype(np.float32)
    b = rng.standard_normal(n).astype(np.float32)
    res = dev(rng.standard_normal((m, n)).astype(np.float32), TYPES[out_dtype])
    limits = dict(low=-0.75, high=2.5) if name == "clip" else {}
    for residual in (None, res):
        log(f"predict {name} to {out_dtype}, residual {residual is not None}, {m} users")
        got = predict.als_predict(ctx, dev(x), dev(t), item_offset=dev(b), activation=name, residual=residual,
                                  dtype=TYPES[out_dtype], **limits)
        r = None if residual is None else f64(residual)
        want, size = predict_oracle.predict(x, t, None, None, b, name, residual=r, **limits)
        assert np.all(np.abs(f64(got) - want) <= predict_oracle.predict_bound(want, size, f, "f32", out_dtype, name, r))


def test_predict_in_place_and_one_bound(ctx):
    """A residual that is the result's own memory, and clips with one bound."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(9)
    x, t = dev(rng.standard_normal((50, 24)).astype(np.float32)), dev(rng.standard_normal((90, 24)).astype(np.float32))
    old = dev(rng.standard_normal((50, 90)).astype(np.float32))
    log("predict in place")
    want = predict.als_predict(ctx, x, t, residual=old, activation="relu")
    got = old.clone()
    predict.als_predict(ctx, x, t, residual=got, out=got, activation="relu")
    assert torch.equal(got, want)
    plain = predict.als_predict(ctx, x, t)
    assert torch.equal(predict.als_predict(ctx, x, t, activation="clip", low=0.5), plain.clamp(min=0.5))
    assert torch.equal(predict.als_predict(ctx, x, t, activation="clip", high=0.5), plain.clamp(max=0.5))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_predict_not_finite(ctx, dtype):
    """NaN and infinities stay in their rows and columns; offsets of -inf; the limits of the activations."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(2)
    m, n, f = 20, 140, 40
    x, t = rng.standard_normal((m, f)).astype(np.float32), rng.standard_normal((n, f)).astype(np.float32)
    x[4, 7], t[11, 39] = np.nan, np.inf
    b = np.zeros(n, np.float32)
    b[5], b[6] = -np.inf, np.inf
    log(f"predict with values that are not finite, {dtype}")
    xd, td = dev(x, TYPES[dtype]), dev(t, TYPES[dtype])
    got = f64(predict.als_predict(ctx, xd, td, item_offset=dev(b)))
    assert np.isnan(got[4]).all()
    rest = np.delete(np.arange(m), 4)
    if dtype == "f32":
        assert np.isnan(got[:, 11]).all()
    else:
        assert np.array_equal(got[rest, 11], np.sign(x[rest, 39]) * np.inf)
    assert np.all(got[rest, 5] == -np.inf) and np.all(got[rest, 6] == np.inf)
    clean = [c for c in range(n) if c not in (5, 6, 11)]
    want, size = predict_oracle.predict(f64(xd)[rest], f64(td)[clean])
    assert np.all(np.abs(got[np.ix_(rest, clean)] - want) <= predict_oracle.predict_bound(want, size, f, dtype, "f32"))
    for name, low, high in (("relu", 0, np.inf), ("gelu", 0, np.inf), ("silu", 0, np.inf), ("sigmoid", 0, 1), ("tanh", -1, 1)):
        got = f64(predict.als_predict(ctx, xd, td, item_offset=dev(b), activation=name))
        assert np.all(got[rest, 5] == low) and np.all(got[rest, 6] == high) and np.isnan(got[4]).all(), name


def test_predict_fp32_range(ctx):
    """The largest and small fp32 values: products of parts neither overflow on their own nor lose their lower parts."""
    from paper_1603_03820_amd import predict
    big = np.finfo(np.float32).max
    x = np.array([[big, 0], [-big, 0], [1.0000001, 0], [2.0 ** -60 * 1.2345678, 0]], np.float32)
    t = np.array([[1, 5], [0.25, 5], [1.0000001, 5], [2.0 ** -40 * 1.7654321, 5]], np.float32)
    log("predict over fp32's range")
    got = f64(predict.als_predict(ctx, dev(x), dev(t)))
    want = x.astype(np.float64) @ t.astype(np.float64).T
    want = np.where(np.abs(want) > big, np.sign(want) * np.inf, want)
    for i in range(4):
        for j in range(4):
            assert got[i, j] == want[i, j] or abs(got[i, j] - want[i, j]) <= 2.0 ** -21 * abs(want[i, j]), (i, j)


def test_predict_empty(ctx):
    from paper_1603_03820_amd import predict
    x, t = torch.ones(3, 8, device=D), torch.ones(5, 8, device=D)
    log("predict of nothing")
    assert predict.als_predict(ctx, x[:0], t).shape == (0, 5)
    assert predict.als_predict(ctx, x, t[:0]).shape == (3, 0)
    assert predict.als_predict(ctx, x, t, users=torch.zeros(0, dtype=torch.int32, device=D)).shape == (0, 5)
    got = predict.als_predict(ctx, x[:0], t, users=torch.zeros(2, dtype=torch.int32, device=D))
    assert bool(torch.isnan(got).all()) and got.shape == (2, 5)


# ------------------------------------------------------------------------------ log_prob --


def lists(rng, rows, n, most, repeats=False):
    """A CSR of columns, some of them outside [0, n)."""
    parts = [rng.integers(-2, n + 3, rng.integers(0, most + 1)) if repeats else
             rng.permutation(n)[:rng.integers(0, min(most, n) + 1)] for _ in range(rows)]
    ptr = np.zeros(rows + 1, np.int64)
    ptr[1:] = np.cumsum([p.size for p in parts])
    return ptr, (np.concatenate(parts) if rows else np.zeros(0)).astype(np.int32)


def row_of(pair, r):
    return pair[1][pair[0][r]:pair[0][r + 1]]


def check(ctx, z, given, temperature, top, rated=None, users=None, what="", grad=True, seed=0):
    """als_log_prob and als_log_prob_grad on a device matrix z, against the oracle row by row."""
    from paper_1603_03820_amd import predict
    rows, n = z.shape
    host = f64(z)
    rd = None if rated is None else (dev(rated[0]), dev(rated[1]))
    ud = None if users is None else dev(users)
    ragged = isinstance(given, tuple)
    gd = (dev(given[0]), dev(given[1])) if ragged else dev(given)
    td = dev(temperature) if isinstance(temperature, np.ndarray) else temperature
    log(f"log_prob {what} {z.dtype} {rows}x{n} top {top}")
    r = predict.als_log_prob(ctx, z, gd, td, top, rd, ud)
    torch.cuda.synchronize()
    got, stats, entropy = f64(r.log).reshape(-1), f64(r.stats), f64(r.entropy)
    rng = np.random.default_rng(seed)
    g = rng.standard_normal(got.size).astype(np.float32)
    h = rng.standard_normal(rows).astype(np.float32)
    oracle, entries = [], []
    for i in range(rows):
        u = i if users is None else users[i]
        there = rated is None or 0 <= u < rated[0].size - 1
        t = float(temperature[i]) if isinstance(temperature, np.ndarray) else np.float32(temperature).item()
        o = predict_oracle.Row(host[i], t, row_of(rated, u) if rated is not None and there else (), there)
        oracle.append(o)
        if ragged:
            e = np.arange(given[0][i], given[0][i + 1])
            cols = given[1][e]
        else:
            per = given.size // rows
            e = np.arange(i * per, (i + 1) * per)
            cols = given.reshape(-1)[e]
        entries.append((e, cols))
        for k, c in zip(e, cols):
            want = o.log(c)
            assert got[k] == want or (np.isnan(want) and np.isnan(got[k])) or abs(got[k] - want) <= o.off_log(c), (i, c, got[k], want)
        if not there:
            assert np.isnan(entropy[i]) and np.isnan(stats[i]).all()
            continue
        assert abs(entropy[i] - o.entropy) <= o.off_entropy, (i, entropy[i], o.entropy, o.off_entropy)
        assert stats[i, 0] == o.best
        assert stats[i, 1] == o.size or abs(stats[i, 1] - o.size) <= o.off_size, (i, stats[i], o.size)
    if top:
        index, best = r.top_index.cpu().numpy(), f64(r.top_log)
        for i, o in enumerate(oracle):
            want_i, want_l = o.top(top)
            assert np.array_equal(index[i], want_i), (i, index[i], want_i)
            for k in range(top):
                same = best[i, k] == want_l[k] or (np.isnan(want_l[k]) and np.isnan(best[i, k]))
                assert same or abs(best[i, k] - want_l[k]) <= o.off_log(want_i[k]), (i, k)
    else:
        assert r.top_index is None and r.top_log is None
    if not grad:
        return r
    name = {v: k for k, v in TYPES.items()}[z.dtype]
    for with_entropy in (False, True):
        log(f"  gradient, entropy {with_entropy}")
        gl = dev(g).view(r.log.shape)
        d, columns = predict.als_log_prob_grad(ctx, z, gd, r, gl, dev(h) if with_entropy else None, td, rd, ud, True, True)
        torch.cuda.synchronize()
        d, columns = f64(d), f64(columns)
        total, off_total, size = np.zeros(n), np.zeros(n), np.zeros(n)
        for i, (o, (e, cols)) in enumerate(zip(oracle, entries)):
            want, off = o.gradient(cols, g[e], float(h[i]) if with_entropy else 0.0)
            if not o.there:
                assert np.isnan(d[i]).all()
            else:
                half = 0.0 if name == "f32" else predict_oracle.HALF_ULP[name]
                want = np.where(np.abs(want) > torch.finfo(z.dtype).max, np.copysign(np.inf, want), want)
                with np.errstate(invalid="ignore"):
                    err = np.where(d[i] == want, 0.0, np.abs(d[i] - want))
                assert np.all(err <= off * (1 + half) + half * np.abs(want) * 1.01 + predict_oracle.TINY[name]), (i, err.max())
            total += want
            off_total += off
            size += np.abs(want)
        with np.errstate(invalid="ignore"):
            same = (columns == total) | (np.isnan(columns) & np.isnan(total))
            assert np.all(same | (np.abs(columns - total) <= off_total + (rows + 4) * 2.0 ** -24 * size + 2.0 ** -149))
    return r


def scores(rng, rows, n, dtype, scale=2.0):
    return dev((scale * rng.standard_normal((rows, n)) + 3).astype(np.float32), TYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,n", [(1, 1), (2, 2), (3, 7), (1, 500), (9, 511), (4, 513), (5, 1024), (3, 1025), (2, 4099), (3, 16_385),
                                    (2, 17_770), (2, 32_768), (2, 32_769), (1, 70_001)])
def test_log_prob_sizes(ctx, dtype, rows, n):
    rng = np.random.default_rng(rows + n)
    z = scores(rng, rows, n, dtype)
    t = (0.3 + rng.random(rows)).astype(np.float32)
    check(ctx, z, rng.integers(0, n, rows).astype(np.int32), t, min(20, n + 2), what="one given")
    check(ctx, z, lists(rng, rows, n, 12, repeats=True), t, 3, lists(rng, rows, n, n // 3 + 1), what="ragged, left out", seed=1)


@pytest.mark.parametrize("top", [0, 1, 2, 63, 64, 65, 128])
@pytest.mark.parametrize("n", [90, 300, 2000, 20_000, 50_000])
def test_log_prob_top(ctx, n, top):
    """Equal scores (bf16 has few) go by their columns; rows in order, so that the best stand side by side."""
    rng = np.random.default_rng(n + top)
    z = scores(rng, 4, n, "bf16")
    z[1] = 1.5
    z[2] = torch.sort(z[2], descending=True).values
    z[3] = torch.sort(z[3]).values
    check(ctx, z, rng.integers(0, n, (4, 3)).astype(np.int32), 0.7, top, lists(rng, 4, n, 30), what="top", grad=False)


@pytest.mark.parametrize("n", [40, 3000, 40_000])
def test_log_prob_special_rows(ctx, n):
    """Rows with nothing left, with infinities, NaN and the type's lowest value; temperatures of 0, NaN, infinity and the
    extremes; given columns that are left out, repeated or outside; users that do not exist."""
    rng = np.random.default_rng(n)
    rows = 16
    z = scores(rng, rows, n, "f32")
    lowest, inf, nan = float(np.finfo(np.float32).min), float("inf"), float("nan")
    z[0] = -inf
    z[1] = nan
    z[2, 1:] = -inf
    z[3, [5, 9, n - 1]] = inf
    z[4, ::2] = nan
    z[5, 3:] = lowest
    z[6] = lowest
    z[7, 7] = inf
    z[8, 4], z[8, 5:] = -lowest, lowest
    t = np.full(rows, 0.5, np.float32)
    t[9], t[10], t[11], t[12], t[13], t[14] = 0.0, np.nan, np.inf, -1.0, 1e-42, 1e30
    z[9, [n - 1, 17]] = 50.0
    given = rng.integers(0, n, (rows, 6)).astype(np.int32)
    given[:, 0], given[:, 1], given[:, 2], given[:, 3] = 0, -1, n, 2 ** 31 - 1
    given[:, 4] = given[:, 5]
    given[3], given[9] = [5, 9, n - 1, 0, 5, 5], [n - 1, 17, 17, 3, -2 ** 31, 2]
    check(ctx, z, given, t, 9, what="special rows")
    rated = lists(rng, 12, n, 25)
    everything = (np.concatenate([rated[0], [rated[0][-1] + n]]), np.concatenate([rated[1], np.arange(n, dtype=np.int32)]))
    users = rng.integers(0, 12, rows).astype(np.int32)
    users[4] = 12
    check(ctx, z, given, t, 9, everything, users, what="special rows, users")
    users[5], users[6] = 13, -1
    check(ctx, z, given, t, 9, everything, users, what="special rows, users that do not exist")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("extra,offset", [(1, 0), (3, 1), (8, 3)])
@pytest.mark.parametrize("n", [333, 33_000])
def test_log_prob_strides(ctx, dtype, n, extra, offset):
    """Rows at every alignment; gradients to such rows leave what lies between them alone; in place."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(n + extra)
    rows = 5
    z = strided(scores(rng, rows, n, dtype), extra, offset)
    given = rng.integers(0, n, rows).astype(np.int32)
    r = check(ctx, z, given, 0.8, 5, what=f"stride + {extra} from {offset}")
    gl = torch.ones(rows, device=D)
    want, _ = predict.als_log_prob_grad(ctx, z, dev(given), r, gl, temperature=0.8)
    into = strided(torch.zeros(rows, n, dtype=z.dtype, device=D), extra + 2, offset)
    got, none = predict.als_log_prob_grad(ctx, z, dev(given), r, gl, temperature=0.8, grad=into)
    assert got is into and none is None and torch.equal(into, want)
    whole = torch.as_strided(into, (into.untyped_storage().nbytes() // into.element_size(),), (1,), 0)
    beside = torch.ones(whole.shape, dtype=torch.bool, device=D)
    torch.as_strided(beside, (rows, n), (n + extra + 2, 1), offset).fill_(False)
    assert bool((whole[beside] == 77).all())
    predict.als_log_prob_grad(ctx, z, dev(given), r, gl, temperature=0.8, grad=z)
    assert torch.equal(z, want)


def test_gradient_against_differences(ctx):
    """The gradient against central differences of the 64-bit loss."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(4)
    rows, n, t = 3, 12, 0.6
    z = rng.standard_normal((rows, n)).astype(np.float32)
    given, g, h = rng.integers(0, n, (rows, 4)).astype(np.int32), rng.standard_normal((rows, 4)).astype(np.float32), rng.standard_normal(rows).astype(np.float32)
    rated = lists(rng, rows, n, 3)
    rd = (dev(rated[0]), dev(rated[1]))
    log("gradient against differences")
    r = predict.als_log_prob(ctx, dev(z), dev(given), t, rated=rd)
    d, _ = predict.als_log_prob_grad(ctx, dev(z), dev(given), r, dev(g), dev(h), t, rd)
    d, step = f64(d), 1e-6
    for i in range(rows):
        for j in range(n):
            at = [z[i].astype(np.float64) for _ in range(2)]
            at[0][j] += step
            at[1][j] -= step
            up, down = (predict_oracle.Row(a, np.float32(t).item(), row_of(rated, i)).loss(given[i], g[i], float(h[i])) for a in at)
            # of the difference: its third derivative's share (1e-12 times some tens) and 1e-16 of the losses over a step
            assert abs(d[i, j] - (up - down) / (2 * step)) <= 1e-5 * (1 + abs(d[i, j]))


def test_offsets_past_32_bits(ctx):
    """Rows that lie billions of elements apart, users far into a large factor, results past 4 GiB."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(1)
    far = 2 ** 31 + 8
    memory = torch.zeros(2 * far + 40_000, dtype=torch.bfloat16, device=D)
    z = torch.as_strided(memory, (3, 33_000), (far, 1))
    z.copy_(scores(rng, 3, 33_000, "bf16"))
    given = rng.integers(0, 33_000, 3).astype(np.int32)
    check(ctx, z, given, 0.8, 5, what="rows far apart")
    check(ctx, z[:, :900], given % 900, 0.8, 5, what="short rows far apart")
    r = predict.als_log_prob(ctx, z, dev(given))
    want, _ = predict.als_log_prob_grad(ctx, z, dev(given), r, torch.ones(3, device=D))
    predict.als_log_prob_grad(ctx, z, dev(given), r, torch.ones(3, device=D), grad=z)
    assert torch.equal(z, want)
    del memory, z
    for dtype in ("f32", "bf16"):
        log(f"predict of far users, {dtype}")
        f = 104
        x = torch.zeros(11_000_000, f, dtype=TYPES[dtype], device=D)
        users = torch.tensor([10_999_999, 0, 5_500_000, 11_000_000, 10_999_999] * 8, dtype=torch.int32, device=D)
        x[users[:3].long()] = dev(rng.integers(-9, 10, (3, f)).astype(np.float32), TYPES[dtype])
        t = dev(rng.integers(-9, 10, (200, f)).astype(np.float32), TYPES[dtype])
        got = predict.als_predict(ctx, x, t, users=users)
        there = users < 11_000_000
        assert torch.equal(got[there].double(), x[users[there].long()].double() @ t.double().t())
        assert bool(torch.isnan(got[~there]).all())
        del x
    log("predict to rows past 4 GiB")
    x, t = (torch.randint(-3, 4, (r, 8), device=D).float() for r in (40_000, 40_000))
    got = predict.als_predict(ctx, x, t)
    for rows in (slice(0, 3), slice(20_000, 20_003), slice(39_997, 40_000)):
        assert torch.equal(got[rows].double(), x[rows].double() @ t.double().t())
    del got
    wide = torch.zeros(2 * far + 300, device=D, dtype=torch.float16)
    out = torch.as_strided(wide, (3, 300), (far, 1))
    predict.als_predict(ctx, x[:3], t[:300], out=out)
    assert torch.equal(out.double(), x[:3].double() @ t[:300].double().t()) and int((wide != 0).sum()) == int((out != 0).sum())


def test_log_prob_shapes(ctx):
    """No rows, no columns, no given columns; a batch's part of a CSR; entries past the list's end."""
    from paper_1603_03820_amd import predict
    log("log_prob of nothing")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=D)  # noqa: E731
    r = predict.als_log_prob(ctx, torch.zeros(0, 9, device=D), i32(0), top=2)
    assert r.log.shape == (0,) and r.top_index.shape == (0, 2)
    _, c = predict.als_log_prob_grad(ctx, torch.zeros(0, 9, device=D), i32(0), r, r.log, grad=False, columns=True)
    assert c.shape == (9,) and not c.any()
    z = torch.zeros(3, 0, device=D)
    r = predict.als_log_prob(ctx, z, i32(3), top=2)
    assert bool((r.log == float("-inf")).all()) and bool((r.top_index == -1).all()) and not r.entropy.any()
    d, c = predict.als_log_prob_grad(ctx, z, i32(3), r, torch.ones(3, device=D), columns=True)
    assert d.shape == (3, 0) and c.shape == (0,)
    rng = np.random.default_rng(0)
    z = scores(rng, 6, 50, "f32")
    check(ctx, z, np.zeros((6, 0), np.int32), 1.0, 2, what="none given")
    ptr, idx = lists(rng, 20, 50, 6)
    whole = torch.full((idx.size,), 5.0, device=D)
    part = predict.als_log_prob(ctx, z, (dev(ptr[7:14]), dev(idx)), log=whole)
    assert part.log is whole
    inside = np.zeros(idx.size, bool)
    inside[ptr[7]:ptr[13]] = True
    assert bool((whole[dev(~inside)] == 5).all())
    for i in range(6):
        for e in range(ptr[7 + i], ptr[8 + i]):
            o = predict_oracle.Row(f64(z)[i])
            assert abs(whole[e].item() - o.log(idx[e])) <= o.off_log(idx[e])
    log("entries that lie outside their list")
    wrong = np.array([-5, 2, 9, 9, 900, 4, 4], np.int64)
    short = torch.zeros(9, dtype=torch.int32, device=D)
    buffer = torch.full((40,), 5.0, device=D)
    predict.als_log_prob(ctx, z, (dev(wrong), short), log=buffer[10:19])
    assert bool((buffer[:10] == 5).all()) and bool((buffer[19:] == 5).all())


def test_one_of_many_rows(ctx):
    """A row's results do not depend on the rows beside it, nor on how often it is asked."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(8)
    for n in (700, 17_770, 40_000):
        z = scores(rng, 300, n, "f32")
        given = rng.integers(0, n, 300).astype(np.int32)
        log(f"rows alone and together, {n} columns")
        r = predict.als_log_prob(ctx, z, dev(given), 0.3, 10)
        again = predict.als_log_prob(ctx, z, dev(given), 0.3, 10)
        for a, b in zip(r, again):
            assert torch.equal(a, b)
        d, c = predict.als_log_prob_grad(ctx, z, dev(given), r, torch.ones(300, device=D), temperature=0.3, columns=True)
        d2, c2 = predict.als_log_prob_grad(ctx, z, dev(given), r, torch.ones(300, device=D), temperature=0.3, columns=True)
        assert torch.equal(d, d2) and torch.equal(c, c2)
        only = predict.als_log_prob_grad(ctx, z, dev(given), r, torch.ones(300, device=D), temperature=0.3, grad=False, columns=True)
        assert only[0] is None and torch.equal(only[1], c)
        for i in (0, 150, 299):
            one = predict.als_log_prob(ctx, z[i:i + 1], dev(given[i:i + 1]), 0.3, 10)
            assert torch.equal(one.top_index[0], r.top_index[i]) and torch.equal(one.log[0], r.log[i])


def test_the_most_columns(ctx):
    """Rows of ALS_PREDICT_N_MAX columns, against the 64-bit forms, and more of them than the workspace holds at a time,
    against the same rows alone; the offsets' gradient in as few groups as the workspace holds."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(11)
    n = predict.ALS_PREDICT_N_MAX
    check(ctx, scores(rng, 2, n, "f32"), rng.integers(0, n, (2, 5)).astype(np.int32), 0.9, 128, lists(rng, 2, n, 300), what="the most columns")
    rows = 700
    gen = torch.Generator(device=D).manual_seed(3)
    z = torch.empty(rows, n, dtype=torch.bfloat16, device=D)
    for r in range(0, rows, 100):
        z[r:r + 100] = torch.randn(100, n, device=D, generator=gen)
    given = torch.randint(0, n, (rows,), device=D, generator=gen, dtype=torch.int32)
    log(f"log_prob {rows}x{n}")
    r = predict.als_log_prob(ctx, z, given, top=128)
    for i in (0, 314, 628, 629, 630, 699):
        one = predict.als_log_prob(ctx, z[i:i + 1], given[i:i + 1], top=128)
        for a, b in zip(one, r):
            assert torch.equal(a[0], b[i])
    log("and its gradient")
    some = z[:40]
    part = predict.LogProb(r.log[:40], r.stats[:40], r.entropy[:40], None, None)
    g = torch.rand(40, device=D, generator=gen)
    d, c = predict.als_log_prob_grad(ctx, some, given[:40], part, g, columns=True)
    p = torch.softmax(some.double(), 1)
    want = -(p * g.double()[:, None])
    want[torch.arange(40, device=D), given[:40].long()] += g.double()
    size = want.abs().sum(0)
    # of p: the sum's error (as in tests/predict_oracle.py, below 2^-17 here), of 40 rows' sum as many roundings
    assert bool(((c.double() - want.sum(0)).abs() <= size * (2.0 ** -17 + 44 * 2.0 ** -24) + 2.0 ** -126).all())
    assert bool(((d.double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -17) + 2.0 ** -126).all())


def test_scores_and_draws_agree(ctx):
    """The log probability of what als_sample draws is the one that it gives: predictions, draw and log probability
    together, as a recommender uses them, captured into a graph and replayed on other users."""
    from paper_1603_03820_amd import predict, serve
    sctx = serve.Context(0)
    rng = np.random.default_rng(6)
    x, t = dev(rng.standard_normal((400, 30)).astype(np.float32)), dev(rng.standard_normal((900, 30)).astype(np.float32))
    b = dev(rng.standard_normal(900).astype(np.float32))
    b[7] = float("-inf")
    rated = tuple(dev(a) for a in lists(rng, 400, 900, 60))
    users, u = dev(rng.integers(0, 400, 64).astype(np.int32)), dev(rng.random(64).astype(np.float32))

    def step():
        z = predict.als_predict(ctx, x, t, users=users, item_offset=b)
        item, lg = serve.als_sample(sctx, z, u, temperature=0.8, rated=rated, users=users)
        r = predict.als_log_prob(ctx, z, item, 0.8, 5, rated, users)
        d, c = predict.als_log_prob_grad(ctx, z, item, r, torch.ones_like(r.log), temperature=0.8, rated=rated, users=users, columns=True)
        return item, lg, r, d, c
    log("predict, draw, log_prob, gradient")
    item, lg, r, d, c = step()
    assert bool((item >= 0).all()) and bool((item != 7).all())
    # both are fp32 forms of one number: the draw's bounds (100 roundings of values of at most 50) cover both
    assert torch.allclose(lg, r.log, rtol=0, atol=200 * 2.0 ** -24 * 50)
    assert bool((r.top_log[:, 0] >= r.log - 1e-5).all())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for k in range(4):
        users.copy_(dev(rng.integers(0, 400, 64).astype(np.int32)))
        u.copy_(dev(rng.random(64).astype(np.float32)))
        log(f"replay {k}")
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (held[0], held[1], *held[2], held[3], held[4])]
        now = step()
        for a, w in zip(got, (now[0], now[1], *now[2], now[3], now[4])):
            assert torch.equal(a, w)
    sctx.close()


def test_captured_in_the_workspace(ctx):
    """Calls that work in the workspace, captured: a product that is cut along its rows, rows in segments, columns' sums.
    Replays on other inputs, with eager calls between them, against the eager results."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(7)
    x, t = dev(rng.standard_normal((4, 3000)).astype(np.float32), torch.bfloat16), dev(rng.standard_normal((50_000, 3000)).astype(np.float32), torch.bfloat16)
    few = t[:200].contiguous()
    given = dev(rng.integers(0, 50_000, (4, 3)).astype(np.int32))

    def step():
        y = predict.als_predict(ctx, x, few, activation="silu")
        z = predict.als_predict(ctx, x, t, dtype=torch.float32)
        r = predict.als_log_prob(ctx, z, given, 40.0, 12)
        d, c = predict.als_log_prob_grad(ctx, z, given, r, r.log, r.entropy, 40.0, columns=True)
        return [y, z, *r, d, c]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for k in range(3):
        x.copy_(dev(rng.standard_normal((4, 3000)).astype(np.float32), torch.bfloat16))
        given.copy_(dev(rng.integers(0, 50_000, (4, 3)).astype(np.int32)))
        log(f"replay {k}")
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in held]
        for a, w in zip(got, step()):
            assert torch.equal(a, w)
        torch.cuda.synchronize()


def test_other_streams(ctx):
    """Calls on a stream that is not the current one, whose tensors are dropped at once; two streams in turn."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(3)
    x, t = dev(rng.standard_normal((200, 64)).astype(np.float32)), dev(rng.standard_normal((50_000, 64)).astype(np.float32))
    given = dev(rng.integers(0, 50_000, 200).astype(np.int32))

    def step(stream):
        z = predict.als_predict(ctx, x, t, stream=stream)
        r = predict.als_log_prob(ctx, z, given, top=7, stream=stream)
        _, c = predict.als_log_prob_grad(ctx, z, given, r, r.log, grad=False, columns=True, stream=stream)
        return r, c
    want, want_c = step(None)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    log("two streams in turn")
    got = [step(streams[k % 2]) for k in range(6)]
    torch.cuda.synchronize()
    for r, c in got:
        assert torch.equal(c, want_c)
        for a, b in zip(r, want):
            assert torch.equal(a, b)


def test_fit_offsets_raises_the_log_probability(ctx):
    """Offsets of a Predictor: every step's mean log probability is above the last one's, and the model's own gradient
    at the end is that of the formula; what is fitted is then what it predicts with."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(12)
    users, n = 300, 80
    x, t = dev((0.3 * rng.standard_normal((users, 8))).astype(np.float32)), dev(rng.standard_normal((n, 8)).astype(np.float32))
    popular = rng.zipf(1.5, 2000) % n
    who, what = dev(rng.integers(0, users, 2000).astype(np.int32)), dev(popular.astype(np.int32))
    model = predict.Predictor(ctx, x, t)
    log("fit offsets")
    means = model.fit_offsets(who, what, temperature=0.7, steps=8, rate=0.5, batch=700)
    assert len(means) == 8 and all(np.isfinite(means))
    before = predict.Predictor(ctx, x, t).log_prob(who, what, 0.7).log.double().mean().item()
    after = model.log_prob(who, what, 0.7).log.double().mean().item()
    assert means[0] == pytest.approx(before, abs=1e-5) and after > before
    z = model.predict(who)
    want = predict.als_predict(ctx, x, t, users=who, item_offset=model.item_offset)
    assert torch.equal(z, want)
    assert float(model.predict(who, low=1, high=2).min()) >= 1


# ------------------------------------------------------------------------------ refusals --


def test_refusals(ctx):
    from paper_1603_03820_amd import predict
    from paper_1603_03820_amd.als import ALSError
    log("refusals")
    x, t = torch.zeros(4, 32, device=D), torch.zeros(6, 32, device=D)
    g = torch.zeros(4, dtype=torch.int32, device=D)
    for error, call in (
            (TypeError, lambda: predict.als_predict(ctx, x.cpu(), t)),
            (TypeError, lambda: predict.als_predict(ctx, x.double(), t.double())),
            (TypeError, lambda: predict.als_predict(ctx, x, t.half())),
            (TypeError, lambda: predict.als_predict(ctx, x, t, dtype=torch.float64)),
            (TypeError, lambda: predict.als_predict(ctx, x, t, users=g.long())),
            (TypeError, lambda: predict.als_predict(ctx, x, t, residual=torch.zeros(4, 6, dtype=torch.float16, device=D))),
            (ValueError, lambda: predict.als_predict(ctx, x, t[:, :31])),
            (ValueError, lambda: predict.als_predict(ctx, x, t.t())),
            (ValueError, lambda: predict.als_predict(ctx, x, t, user_offset=torch.zeros(6, device=D))),
            (ValueError, lambda: predict.als_predict(ctx, x, t, item_offset=torch.zeros(4, device=D))),
            (ValueError, lambda: predict.als_predict(ctx, x, t, activation="swish")),
            (ValueError, lambda: predict.als_predict(ctx, x, t, low=1.0)),
            (ValueError, lambda: predict.als_predict(ctx, x, t, out=torch.zeros(1, 6, device=D).expand(4, 6))),
            (ALSError, lambda: predict.als_predict(ctx, x, t, activation="clip", low=2.0, high=1.0)),
            (ALSError, lambda: predict.als_predict(ctx, x[:, :0], t[:, :0])),
            (TypeError, lambda: predict.als_log_prob(ctx, x, g.long())),
            (TypeError, lambda: predict.als_log_prob(ctx, x, [0, 1, 2, 3])),
            (ValueError, lambda: predict.als_log_prob(ctx, x, g[:3])),
            (ValueError, lambda: predict.als_log_prob(ctx, x, torch.zeros(4, 6, dtype=torch.int32, device=D)[:, ::2])),
            (ValueError, lambda: predict.als_log_prob(ctx, x, g, top=129)),
            (ValueError, lambda: predict.als_log_prob(ctx, x, g, top=-1)),
            (ValueError, lambda: predict.als_log_prob(ctx, x, (torch.zeros(4, dtype=torch.int64, device=D), g))),
            (ValueError, lambda: predict.als_log_prob(ctx, x, g, users=g)),
            (ValueError, lambda: predict.als_log_prob(ctx, x, g, rated=(torch.zeros(4, dtype=torch.int64, device=D), g))),
            (ValueError, lambda: predict.als_log_prob(ctx, x, g, temperature=torch.ones(3, device=D))),
            (ValueError, lambda: predict.als_log_prob(ctx, x, g, log=torch.zeros(5, device=D)))):
        with pytest.raises(error):
            call()
    r = predict.als_log_prob(ctx, x, g)
    for error, call in (
            (ValueError, lambda: predict.als_log_prob_grad(ctx, x, g, r, torch.ones(5, device=D))),
            (TypeError, lambda: predict.als_log_prob_grad(ctx, x, g, r, torch.ones(4, dtype=torch.float64, device=D))),
            (ValueError, lambda: predict.als_log_prob_grad(ctx, x, g, r, r.log, grad_entropy=torch.ones(3, device=D))),
            (TypeError, lambda: predict.als_log_prob_grad(ctx, x, g, r, r.log, grad=x.half())),
            (ValueError, lambda: predict.als_log_prob_grad(ctx, x, g, r, r.log, columns=torch.ones(31, device=D))),
            (ALSError, lambda: predict.als_log_prob_grad(ctx, x, g, r, r.log, columns=x.view(-1)[:32])),
            (ValueError, lambda: predict.als_log_prob_grad(ctx, x[:3], g[:3], r, r.log[:3]))):
        with pytest.raises(error):
            call()
    with pytest.raises(ALSError) as e:
        predict.als_predict(ctx, x, t, residual=torch.zeros(64, device=D)[:24].view(4, 6), out=torch.zeros(64, device=D)[:24].view(4, 6),
                            activation="clip", low=float("nan"))
    assert e.value.code == -1
    c = predict.Context(0)
    c.close()
    with pytest.raises(ValueError):
        predict.als_predict(c, x, t)


def test_refusals_of_the_library(ctx):
    """The C boundary's own."""
    from paper_1603_03820_amd import predict
    lib, P, h = predict._lib, ctypes.c_void_p, ctx.handle
    p = lambda t, off=0: P(t.data_ptr() + off)  # noqa: E731
    log("refusals of the library")
    x, t, o = torch.zeros(4096, device=D), torch.zeros(4096, device=D), torch.zeros(4096, device=D)
    small, ints = torch.zeros(64, device=D), torch.zeros(64, dtype=torch.int32, device=D)

    def product(x=p(x), of=4, ldx=32, users=None, m=4, theta=p(t), n=6, ldt=32, dtype=0, f=32, ua=None, ib=None, act=0,
                low=0.0, high=0.0, res=None, ldr=6, out=p(o), ldo=6, od=0):
        return lib.als_predict(h, x, of, ldx, users, m, theta, n, ldt, dtype, f, ua, ib, act, low, high, res, ldr, out, ldo, od, None)
    assert product() == 0 and product(m=0, out=None) == 0 and product(n=0, theta=None) == 0
    assert product(res=p(o), ldr=6) == 0 and product(users=p(ints), m=60, n=1) == 0
    for bad in (dict(x=None), dict(theta=None), dict(out=None), dict(m=5), dict(m=-1), dict(n=-1), dict(of=-1), dict(dtype=3),
                dict(od=-1), dict(ldx=31), dict(ldt=31), dict(ldo=5), dict(act=7), dict(act=-1), dict(act=1, low=1.0, high=0.0),
                dict(act=1, low=float("nan")), dict(res=p(small), ldr=5)):
        assert product(**bad) == -1, bad
    assert product(f=0) == -2 and product(f=1_048_577, ldx=1 << 21, ldt=1 << 21) == -2
    for bad in (dict(x=p(x, 2)), dict(theta=p(t, 1)), dict(out=p(o, 2)), dict(ua=p(small, 2)), dict(ib=p(small, 1)),
                dict(users=p(ints, 2)), dict(res=p(small, 2))):
        assert product(**bad) == -4, bad
    for bad in (dict(out=p(x)), dict(out=p(t, 64)), dict(ua=p(o)), dict(ib=p(o)), dict(users=p(o)), dict(res=p(o, 4)),
                dict(res=p(o), ldr=7)):
        assert product(**bad) == -6, bad

    lg, st, en, ti, tl = (torch.zeros(64, device=D) for _ in range(5))
    rp = torch.zeros(9, dtype=torch.int64, device=D)

    def structs(z=p(x), dtype=0, rows=4, n=32, ldz=32, t=None, ptr=None, col=None, users=None, of=0, gptr=None, idx=p(ints), entries=4,
                each=1):
        return (predict._Scores(z=z, dtype=dtype, rows=rows, n=n, ldz=ldz, temperature=t, temperature_all=1.0, rated_ptr=ptr,
                                rated_idx=col, users=users, of=of), predict._Given(ptr=gptr, idx=idx, entries=entries, each=each))

    def log_prob(log=p(lg), stats=p(st), entropy=p(en), top=2, index=p(ti), top_log=p(tl), **more):
        s, g = structs(**more)
        return lib.als_log_prob(h, ctypes.byref(s), ctypes.byref(g), log, stats, entropy, top, index, top_log, None)

    def gradient(log=p(lg), stats=p(st), entropy=p(en), gl=p(small), ge=p(small, 64), grad=p(o), ldg=32, columns=p(tl), **more):
        s, g = structs(**more)
        return lib.als_log_prob_grad(h, ctypes.byref(s), ctypes.byref(g), log, stats, entropy, gl, ge, grad, ldg, columns, None)
    assert log_prob() == 0 and log_prob(stats=None, entropy=None, index=None, top_log=None) == 0
    assert log_prob(rows=0, z=None, entries=0, idx=None) == 0 and log_prob(n=0, z=None) == 0
    assert log_prob(entries=0, each=0, idx=None, log=None) == 0 and log_prob(ptr=p(rp), col=p(ints), of=4) == 0
    assert gradient() == 0 and gradient(grad=None) == 0 and gradient(columns=None) == 0 and gradient(ge=None, entropy=None) == 0
    assert gradient(grad=p(x)) == 0 and gradient(grad=None, columns=None) == 0
    for bad in (dict(z=None), dict(rows=-1), dict(n=-1), dict(n=4_194_305, ldz=4_194_305), dict(ldz=31), dict(dtype=3), dict(ptr=p(rp)),
                dict(col=p(ints)), dict(users=p(ints)), dict(ptr=p(rp), col=p(ints), of=3), dict(of=-1), dict(log=None), dict(idx=None),
                dict(entries=5), dict(entries=8), dict(each=2), dict(entries=-4), dict(entries=-1, gptr=p(rp)), dict(each=-1)):
        assert log_prob(**bad) == -1 and gradient(**bad) == -1, bad
    assert log_prob(top=129) == -1 and log_prob(top=-1) == -1
    assert gradient(stats=None) == -1 and gradient(gl=None) == -1 and gradient(entropy=None) == -1 and gradient(ldg=31) == -1
    for bad in (dict(z=p(x, 2)), dict(t=p(small, 1)), dict(ptr=p(rp, 4), col=p(ints), of=4), dict(gptr=p(rp, 4)), dict(idx=p(ints, 2)),
                dict(log=p(lg, 2)), dict(stats=p(st, 1))):
        assert log_prob(**bad) == -4 and gradient(**bad) == -4, bad
    assert log_prob(index=p(ti, 2)) == -4 and gradient(grad=p(o, 2)) == -4 and gradient(columns=p(tl, 2)) == -4
    for bad in (dict(log=p(x, 16)), dict(stats=p(x)), dict(log=p(ints)), dict(entropy=p(st)), dict(index=p(tl)), dict(top_log=p(lg)),
                dict(t=p(en)), dict(gptr=p(rp), stats=p(rp), entries=4)):
        assert log_prob(**bad) == -6, bad
    for bad in (dict(grad=p(x, 4)), dict(grad=p(x), ldg=33), dict(columns=p(x)), dict(columns=p(lg)), dict(columns=p(st)),
                dict(columns=p(en)), dict(columns=p(small)), dict(grad=p(o), columns=p(o, 256)), dict(t=p(o))):
        assert gradient(**bad) == -6, bad
    torch.cuda.synchronize()


def test_evaluate_command():
    """The command's evaluation on the tiny workload against the 64-bit forms: means over the held-out items of every
    second user."""
    import synth
    from paper_1603_03820_amd import als, driver, recommend
    log("train, evaluate and fit, tiny workload")
    before, after, means = recommend.evaluate("tiny", iters=3, batch=300, temperature=0.2, steps=4)
    again = recommend.evaluate("tiny", iters=3, batch=1000, temperature=0.2, steps=0)[0]
    assert len(means) == 4 and all(np.isfinite(means)) and all(np.isfinite(v) for v in after.values())
    assert before["hits"] == again["hits"] and before["log_prob"] == pytest.approx(again["log_prob"], abs=1e-9)
    p = synth.config("tiny")
    train, test = synth.split(p.rowptr, p.colidx, p.vals, 0.1, p.recipe["seed"])
    c = als.Context(0, p.f)
    dp = driver.DeviceProblem.from_host_csr(c, p.m, p.n, p.f, p.lam, *train)
    x, theta, _ = driver.train(c, dp, torch.from_numpy(p.theta0).to(D), 3)
    z = (x @ theta.t()).float().cpu().numpy()
    logs, hits, entropy = [], [], []
    for u in range(1, p.m, 2):
        row = predict_oracle.Row(z[u], np.float32(0.2).item(), train[1][train[0][u]:train[0][u + 1]])
        items = test[1][test[0][u]:test[0][u + 1]]
        logs += [row.log(i) for i in items]
        hits += [i in row.top(20)[0] for i in items]
        entropy.append(row.entropy)
    # z from another product: 1e-6 of scores up to some units, five times that in y
    assert before["log_prob"] == pytest.approx(np.mean(logs), abs=1e-4)
    assert before["entropy"] == pytest.approx(np.mean(entropy), abs=1e-4)
    assert abs(before["hits"] - np.mean(hits)) <= 3 / len(hits)


def test_fit_leaves_out_what_is_rated(ctx):
    """Given items that their users have rated, or that are no items, count for nothing in a fit."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(5)
    x, t = dev(rng.standard_normal((40, 8)).astype(np.float32)), dev(rng.standard_normal((60, 8)).astype(np.float32))
    rated = lists(rng, 40, 60, 20)
    rd = tuple(dev(a) for a in rated)
    who, what = rng.integers(0, 40, 200).astype(np.int32), rng.integers(0, 60, 200).astype(np.int32)
    clean = np.array([w not in row_of(rated, u) for u, w in zip(who, what)])
    log("fit with and without entries that do not count")
    a, b = (predict.Predictor(ctx, x, t, rated=rd) for _ in range(2))
    more = np.concatenate([what, [-1, 60, 2 ** 31 - 1]]).astype(np.int32)
    with_all = a.fit_offsets(dev(np.concatenate([who, [0, 1, 2]]).astype(np.int32)), dev(more), 0.5, 3)
    with_clean = b.fit_offsets(dev(who[clean]), dev(what[clean]), 0.5, 3)
    # rows of nothing that counts still expect nothing: their weight is 0
    assert np.allclose(with_all, with_clean, atol=1e-5)
    assert torch.allclose(a.item_offset, b.item_offset, atol=1e-4)
    nothing = predict.Predictor(ctx, x, t, rated=rd)
    for bad in (what[:0], what[:5]):
        with pytest.raises(ValueError):
            a.fit_offsets(dev(who[:bad.size // 2]), dev(bad))
    assert nothing.fit_offsets(dev(who[~clean][:3]), dev(what[~clean][:3]), 0.5, 1) == [0.0] and not nothing.item_offset.any()
