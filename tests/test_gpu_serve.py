"""The serving operators on the GPU against their plain 64-bit forms (tests/serve_oracle.py)."""
import ctypes

import numpy as np
import pytest
import torch

from tests import serve_oracle
from tests.gpu_util import log

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    from paper_1603_03820_amd import serve
    c = serve.Context(0)
    yield c
    c.close()


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")
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


# ------------------------------------------------------------------------------ quantize --


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,f,extra,offset", [(1, 1, 0, 0), (1, 100, 0, 0), (3, 7, 0, 0), (5, 16, 3, 1),
                                                 (300, 100, 0, 0), (17, 127, 5, 3), (9, 1000, 1, 7),
                                                 (33, 128, 0, 1), (4, 8192, 0, 0), (3, 8191, 2, 5), (2, 131071, 0, 0)])
def test_quantize(ctx, dtype, rows, f, extra, offset):
    from paper_1603_03820_amd import serve
    rng = np.random.default_rng(rows * 7 + f)
    x = rng.standard_normal((rows, f)) * np.exp(rng.standard_normal((rows, 1)))
    xd = strided(dev(x.astype(np.float32), TYPES[dtype]), extra, offset)
    log(f"quantize {dtype} {rows}x{f} stride {xd.stride(0)} offset {offset}")
    q, s = serve.als_quantize(ctx, xd)
    x32 = xd.float().cpu().numpy()
    want_q, want_s = serve_oracle.quantize(x32)
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(s.cpu().numpy(), want_s)
    # half a step, and the two fp32 roundings of a quotient of at most 127
    err = np.abs(f64(q) * f64(s)[:, None] - x32.astype(np.float64))
    assert np.all(err <= f64(s)[:, None] * (0.5 + 127 * 2 * 2.0 ** -24 + 127 * 2.0 ** -23))
    # what lies between a row's end and the next multiple of 16 is zero
    pad = torch.as_strided(q, (rows, q.stride(0)), (q.stride(0), 1))[:, f:]
    assert q.stride(0) % 16 == 0 and not pad.any()


def test_quantize_takes_rows(ctx):
    from paper_1603_03820_amd import serve
    rng = np.random.default_rng(5)
    x = rng.standard_normal((50, 37)).astype(np.float32)
    users = np.array([3, 3, 0, 49, -1, 50, 7], dtype=np.int32)
    log("quantize of rows taken by index")
    q, s = serve.als_quantize(ctx, dev(x), users=dev(users))
    want_q, want_s = serve_oracle.quantize(x)
    for r, u in enumerate(users):
        if 0 <= u < 50:
            assert np.array_equal(q[r].cpu().numpy(), want_q[u]) and s[r].item() == want_s[u]
        else:
            assert torch.isnan(s[r]) and not q[r].any()


@pytest.mark.parametrize("f", [5, 64, 300, 5000])
def test_quantize_edge_values(ctx, f):
    """Zeros, one value, the largest and the least of the type, infinities and NaN."""
    from paper_1603_03820_amd import serve
    big = np.finfo(np.float32).max
    rows = [np.zeros(f), np.full(f, -3.0), np.r_[np.ones(f - 1), -big], np.full(f, 2.0 ** -149),
            np.r_[2.0 ** -140, np.zeros(f - 1)], np.r_[np.ones(f - 1), np.inf], np.r_[np.nan, np.ones(f - 1)],
            np.r_[-np.inf, np.zeros(f - 1)], np.r_[-0.0, np.zeros(f - 1)], np.linspace(-1, 1, f) * big]
    x = np.array(rows).astype(np.float32)
    log(f"quantize of edge values, f {f}")
    q, s = serve.als_quantize(ctx, dev(x))
    want_q, want_s = serve_oracle.quantize(x)
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(s.cpu().numpy(), want_s, equal_nan=True)


def test_quantize_into_given_rows(ctx):
    """A given q of any stride: nothing past a row's padding is written; an empty call writes nothing."""
    from paper_1603_03820_amd import serve
    rng = np.random.default_rng(6)
    x = rng.standard_normal((7, 21)).astype(np.float32)
    for stride in (21, 22, 40):
        buf = torch.full((7, stride), 99, dtype=torch.int8, device="cuda:0")
        log(f"quantize into rows of stride {stride}")
        serve.als_quantize(ctx, dev(x), q=buf[:, :21])
        assert np.array_equal(buf[:, :21].cpu().numpy(), serve_oracle.quantize(x)[0])
        assert not buf[:, 21:min(stride, 32)].any() and bool((buf[:, 32:] == 99).all())
    q, s = serve.als_quantize(ctx, dev(x)[:0])
    assert q.shape == (0, 21) and s.shape == (0,)


# --------------------------------------------------------------------------------- score --


def int8_rows(rng, rows, f, extra=0, offset=0):
    return strided(dev(rng.integers(-128, 128, (rows, f)).astype(np.int8)), extra, offset)


SCORE_SHAPES = [(1, 1, 1), (1, 3, 1000), (2, 17, 5), (16, 64, 64), (15, 63, 63), (17, 65, 65), (1, 500, 100),
                (33, 129, 100), (64, 300, 128), (70, 301, 127), (5, 700, 1024), (130, 260, 200), (257, 513, 320),
                (300, 1000, 16), (3, 2000, 4096), (1, 40, 70000), (20, 40, 131071), (128, 256, 192), (1000, 70, 96),
                (513, 770, 1088), (256, 512, 2048), (7, 9000, 37), (260, 1030, 129)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,f", SCORE_SHAPES)
def test_score(ctx, dtype, m, n, f):
    from paper_1603_03820_amd import serve
    rng = np.random.default_rng(m + 3 * n + 7 * f)
    for layout in range(3):
        # rows as als_quantize leaves them, dense rows, rows of odd stride at an odd address
        extra, offset = ((f + 15) // 16 * 16 - f, 0) if layout == 0 else ((0, 0) if layout == 1 else (3, 5))
        xq, tq = int8_rows(rng, m, f, extra, offset), int8_rows(rng, n, f, extra, offset)
        xs = dev((rng.uniform(0.5, 2.0, m) / np.sqrt(f) / 100).astype(np.float32))
        ts = dev((rng.uniform(0.5, 2.0, n) / 100).astype(np.float32))
        out = torch.full((m, n + (0, 5, 1)[layout]), 9.0, dtype=TYPES[dtype], device="cuda:0")
        log(f"score {dtype} m {m} n {n} f {f} layout {layout}")
        serve.als_score(ctx, xq, xs, tq, ts, out=out[:, :n])
        exact = serve_oracle.score(xq.cpu().numpy(), xs.cpu().numpy(), tq.cpu().numpy(), ts.cpu().numpy())
        err = np.abs(f64(out[:, :n]) - exact)
        assert np.all(err <= serve_oracle.score_bound(exact, dtype)), err.max()
        assert bool((out[:, n:] == 9.0).all())


@pytest.mark.parametrize("m,n,f", [(9, 260_000, 300), (260_000, 9, 300), (900, 1100, 100_003)])
def test_score_of_odd_strides_past_the_workspace(ctx, m, n, f):
    """Rows that are laid out anew, more of them than the workspace holds at a time."""
    from paper_1603_03820_amd import serve
    assert max(m, n) * f > ctx.workspace.numel() // 2
    g = torch.Generator("cuda:0").manual_seed(m)
    xq = torch.randint(-128, 128, (m, f + 1), dtype=torch.int8, device="cuda:0", generator=g)[:, 1:]
    tq = torch.randint(-128, 128, (n, f + 3), dtype=torch.int8, device="cuda:0", generator=g)[:, :f]
    xs, ts = torch.rand(m, device="cuda:0", generator=g), torch.rand(n, device="cuda:0", generator=g)
    log(f"score of odd strides, m {m} n {n} f {f}")
    out = serve.als_score(ctx, xq, xs, tq, ts)
    # a sample of users and items, the ends of the parts among them
    part = ctx.workspace.numel() // 2 // ((f + 15) // 16 * 16)
    pick = lambda k: sorted({0, k - 1, k // 2} | {c for c in (part - 1, part, 2 * part) if 0 <= c < k})  # noqa: E731
    us, it = pick(m), pick(n)
    exact = serve_oracle.score(xq[us].cpu().numpy(), xs[us].cpu().numpy(), tq[it].cpu().numpy(), ts[it].cpu().numpy())
    assert np.all(np.abs(f64(out[us][:, it]) - exact) <= serve_oracle.score_bound(exact, "f32"))
    a = serve.als_score(ctx, *serve_aligned(xq, xs), *serve_aligned(tq, ts))
    assert torch.equal(a, out)


def serve_aligned(q, s):
    rows, f = q.shape
    wide = torch.zeros(rows, (f + 15) // 16 * 16, dtype=torch.int8, device=q.device)
    wide[:, :f] = q
    return wide[:, :f], s


def test_score_sums_at_their_limit(ctx):
    """128^2 times the longest row stays exact."""
    from paper_1603_03820_amd import serve
    f = serve.ALS_SERVE_F_MAX
    one = torch.full((2, f), -128, dtype=torch.int8, device="cuda:0")
    log("score of the longest rows of -128")
    out = serve.als_score(ctx, one, torch.ones(2, device="cuda:0"), one, torch.ones(2, device="cuda:0"))
    assert bool((out == np.float32(128 * 128 * f)).all())


def test_score_not_finite_scales(ctx):
    """A scale of NaN (a row that was not finite) or infinity touches its row and column only; what overflows the
    output's type is infinite."""
    from paper_1603_03820_amd import serve
    rng = np.random.default_rng(3)
    xq, tq = int8_rows(rng, 40, 64), int8_rows(rng, 90, 64)
    xs, ts = torch.ones(40, device="cuda:0"), torch.ones(90, device="cuda:0")
    xs[7], ts[11] = float("nan"), float("inf")
    log("score with scales that are not finite")
    out = f64(serve.als_score(ctx, xq, xs, tq, ts, dtype=torch.float16))
    exact = serve_oracle.score(xq.cpu().numpy(), np.ones(40), tq.cpu().numpy(), np.ones(90))
    assert np.all(np.isnan(out[7]))
    rest = np.delete(np.arange(40), 7)
    assert np.all(~np.isfinite(out[rest, 11]))
    cols = np.delete(np.arange(90), 11)
    got, want = out[np.ix_(rest, cols)], exact[np.ix_(rest, cols)]
    over = np.abs(want) >= 65520
    assert np.all(np.isinf(got[over]) & (np.sign(got[over]) == np.sign(want[over])))
    assert np.all(np.abs(got - want)[~over] <= serve_oracle.score_bound(want, "f16")[~over])


def test_score_far_rows(ctx):
    """Rows whose offsets pass 2^31, in every matrix."""
    from paper_1603_03820_amd import serve
    rng = np.random.default_rng(4)
    far = 1_200_000_016
    for m, n, f in ((3, 40, 100), (3, 40, 2000)):
        xq, tq = rng.integers(-127, 128, (m, f)).astype(np.int8), rng.integers(-127, 128, (n, f)).astype(np.int8)
        big = torch.zeros(2 * far + 4096, dtype=torch.int8, device="cuda:0")
        bx = torch.as_strided(big, (m, f), (far, 1))
        bx.copy_(dev(xq))
        out = torch.empty(2 * far + 4096, dtype=torch.float16, device="cuda:0")
        bo = torch.as_strided(out, (m, n), (far, 1))
        s1, s2 = torch.full((m,), 0.01, device="cuda:0"), torch.full((n,), 0.01, device="cuda:0")
        log(f"score with rows 1.2e9 apart, f {f}")
        serve.als_score(ctx, bx, s1, dev(tq), s2, out=bo)
        exact = serve_oracle.score(xq, s1.cpu().numpy(), tq, s2.cpu().numpy())
        assert np.all(np.abs(f64(bo) - exact) <= serve_oracle.score_bound(exact, "f16"))
        # and as the items
        o2 = serve.als_score(ctx, dev(tq), s2, bx, s1)
        assert np.all(np.abs(f64(o2) - exact.T) <= serve_oracle.score_bound(exact.T, "f32"))
        del big, out, bx, bo


# -------------------------------------------------------------------------------- sample --


def draw_rows(ctx, z, u, rated=None, users=None, **limits):
    from paper_1603_03820_amd import serve
    rows = z.shape[0]
    args = {k: dev(np.asarray(v, np.int32 if k == "top_k" else np.float32)) if np.ndim(v) else v
            for k, v in limits.items()}
    r = None if rated is None else (dev(np.asarray(rated[0], np.int64)), dev(np.asarray(rated[1], np.int32)))
    idx, lg = serve.als_sample(ctx, z, dev(np.asarray(u, np.float32)), rated=r,
                               users=None if users is None else dev(np.asarray(users, np.int32)), **args)
    idx, lg = idx.cpu().numpy(), f64(lg)
    zz = f64(z)
    for i in range(rows):
        mine = {k: float(np.float32(v[i] if np.ndim(v) else v)) for k, v in limits.items()}
        if "top_k" in mine:
            mine["top_k"] = int(mine["top_k"])
        left = ()
        if rated is not None:
            s = i if users is None else users[i]
            left = np.asarray(rated[1])[rated[0][s]:rated[0][s + 1]]
        d = serve_oracle.Draw(zz[i], float(np.float32(u[i])), rated=left, **mine)
        assert d.accepts(idx[i], lg[i]), (i, idx[i], lg[i], mine, u[i])
    return idx, lg


LIMITS = [dict(), dict(temperature=0.25), dict(top_k=1), dict(top_k=7), dict(top_k=300), dict(top_p=0.5),
          dict(top_p=0.95, temperature=0.4), dict(min_p=0.1), dict(top_k=40, top_p=0.8, min_p=0.05, temperature=0.5),
          dict(temperature=0.0), dict(top_p=0.0), dict(temperature=0.02, top_p=0.9), dict(temperature=50.0, top_p=0.3)]


@pytest.mark.parametrize("limits", LIMITS, ids=lambda d: "-".join(f"{k}{v}" for k, v in d.items()) or "none")
@pytest.mark.parametrize("n", [1, 2, 3, 63, 65, 500, 1023, 4097, 17770, 40001])
def test_sample(ctx, n, limits):
    rng = np.random.default_rng(n)
    rows = 6
    u = np.r_[0.0, 1 - 2.0 ** -24, rng.random(rows - 2)].astype(np.float32)
    for t, dtype in enumerate(TYPES.values()):
        z = dev((3.5 + rng.standard_normal((rows, n))).astype(np.float32), dtype)
        z = strided(z, (0, 3, 1)[t], (0, 1, 3)[t])
        log(f"sample n {n} {dtype} {limits}")
        draw_rows(ctx, z, u, **limits)


@pytest.mark.parametrize("n", [100_003, 625_000, 1_048_581])
def test_sample_long_rows(ctx, n):
    rng = np.random.default_rng(n)
    z = dev((3.5 + 0.7 * rng.standard_normal((3, n))).astype(np.float32))
    ptr = np.array([0, 400, 400, 900])
    idx = rng.integers(0, n, 900)
    for limits in (dict(temperature=0.3), dict(top_k=500, top_p=0.9), dict(top_p=0.7, min_p=0.01),
                   dict(temperature=[0.0, 0.1, 1.0], top_k=[0, 3, 100_000], top_p=[1.0, 0.9, 0.99])):
        for zz in (z, z.to(torch.bfloat16)):
            log(f"sample n {n} {zz.dtype} {limits}")
            draw_rows(ctx, zz, [0.2, 0.5, 0.99], rated=(ptr, idx), **limits)


@pytest.mark.parametrize("n", [16_000, 60_000, 131_073, 4_194_304])
def test_sample_longest_and_between(ctx, n):
    """The longest row there may be, and lengths at which rows are held in other ways."""
    rng = np.random.default_rng(n)
    rows = 2
    z = dev((3.5 + 0.7 * rng.standard_normal((rows, n))).astype(np.float32))
    idx = rng.integers(0, n, 300)
    for zz in (z, z.to(torch.bfloat16)):
        for limits in (dict(temperature=0.3), dict(temperature=0.2, top_p=0.9), dict(top_k=200, top_p=0.8),
                       dict(top_k=3000), dict(temperature=0.3, top_p=0.95, min_p=0.05), dict(temperature=0.0)):
            log(f"sample n {n} {zz.dtype} {limits}")
            draw_rows(ctx, zz, [0.3, 0.97], rated=(np.array([0, 300, 300]), idx), **limits)


@pytest.mark.parametrize("rows,n", [(300, 400), (300, 1_000), (300, 3_000), (300, 9_000), (300, 16_000), (900, 100_003)])
def test_sample_rows_alone_and_together(ctx, rows, n):
    """A row's draw does not depend on the rows beside it (how many there are chooses how they are held, and
    many long rows go through the workspace in batches)."""
    from paper_1603_03820_amd import serve
    g = torch.Generator("cuda:0").manual_seed(n)
    z = (3.5 + 0.7 * torch.randn(rows, n, device="cuda:0", generator=g)).to(torch.float16)
    u = torch.rand(rows, device="cuda:0", generator=g)
    k = torch.randint(0, 400, (rows,), device="cuda:0", generator=g, dtype=torch.int32)
    p = 0.8 + 0.3 * torch.rand(rows, device="cuda:0", generator=g)
    t = torch.rand(rows, device="cuda:0", generator=g) * 0.5
    log(f"sample {rows} x {n} together")
    index, lg = serve.als_sample(ctx, z, u, temperature=t, top_k=k, top_p=p)
    for r in range(0, rows, 97):
        log(f"row {r} alone")
        i, l1 = serve.als_sample(ctx, z[r:r + 1], u[r:r + 1], temperature=t[r:r + 1], top_k=k[r:r + 1], top_p=p[r:r + 1])
        assert i.item() == index[r].item() and l1.item() == lg[r].item()
    draw_rows(ctx, z[-3:], u[-3:].cpu().numpy(), temperature=t[-3:].cpu().numpy(), top_k=k[-3:].cpu().numpy(),
              top_p=p[-3:].cpu().numpy())


def test_sample_sorted_scores(ctx):
    """Best columns next to one another: they crowd one wave, one segment."""
    for n in (5_000, 17_770, 200_000):
        z = torch.linspace(5, 0, n, device="cuda:0").expand(3, n).contiguous()
        z[1] = z[1].flip(0)
        for limits in (dict(top_k=300), dict(temperature=0.2, top_p=0.9), dict(top_k=2000, top_p=0.5), dict(top_p=0.99)):
            log(f"sample of sorted scores n {n} {limits}")
            draw_rows(ctx, z, [0.1, 0.6, 0.95], **limits)


def test_sample_limits_by_row(ctx):
    rng = np.random.default_rng(8)
    rows, n = 64, 3000
    z = dev(rng.standard_normal((rows, n)).astype(np.float32))
    limits = dict(temperature=np.where(rng.random(rows) < 0.2, 0, rng.uniform(0.1, 2, rows)).astype(np.float32),
                  top_k=rng.integers(-1, 60, rows), top_p=rng.uniform(0.3, 1.2, rows).astype(np.float32),
                  min_p=rng.uniform(-0.1, 0.3, rows).astype(np.float32))
    log("sample with limits of each row")
    draw_rows(ctx, z, rng.random(rows).astype(np.float32), **limits)


def equal_rows(n, kind):
    z = np.zeros((1, n), np.float32)
    if kind == "steps":
        z[0] = -(np.arange(n) % 3)
    elif kind == "zeros":
        z[0, ::2] = -0.0
    elif kind == "lowest":
        z[0] = np.finfo(np.float32).min
    elif kind == "inf":
        z[0, ::5] = np.inf
    return z


@pytest.mark.parametrize("kind", ["same", "zeros", "lowest"])
@pytest.mark.parametrize("n", [2, 64, 1000, 5000, 70_000])
def test_sample_of_equal_scores_is_exact(ctx, n, kind):
    """Equal scores have equal weights, so the column is known exactly: floor(u k) among the k that are left."""
    from paper_1603_03820_amd import serve
    z = dev(equal_rows(n, kind)).expand(8, n).contiguous()
    u = np.array([0, 0.124, 0.25, 0.5, 0.625, 0.75, 0.999, 1 - 2.0 ** -24], np.float32)
    for top_k, top_p in ((0, 1.0), (2, 1.0), (1500, 1.0), (0, 0.5), (1024, 0.25), (0, 0.75)):
        kept = min(n, top_k) if top_k else n
        if top_p < 1:
            kept = int(np.ceil(kept * top_p))
        log(f"sample of {n} equal scores ({kind}), k {top_k} p {top_p}")
        idx, lg = serve.als_sample(ctx, z, dev(u), top_k=top_k, top_p=top_p)
        want = np.floor(u.astype(np.float64) * kept).astype(np.int32)
        assert np.array_equal(idx.cpu().numpy(), want)
        assert np.allclose(f64(lg), -np.log(kept), rtol=0, atol=1e-6 * max(1.0, np.log(kept)))


@pytest.mark.parametrize("n", [50, 4097, 66_000])
def test_sample_of_ties_cuts_by_column(ctx, n):
    """Many columns share each of three scores; the cut falls inside a score and keeps its lower columns."""
    z = dev(equal_rows(n, "steps")).expand(5, n).contiguous()
    for limits in (dict(top_k=n // 2), dict(top_p=0.9), dict(top_p=0.5), dict(top_k=n // 2, top_p=0.97),
                   dict(top_k=n // 3 + 1)):
        log(f"sample of ties n {n} {limits}")
        draw_rows(ctx, z, [0.0, 0.3, 0.6, 0.9, 0.99999], **limits)


@pytest.mark.parametrize("n", [7, 2000, 70_001])
def test_sample_special_values(ctx, n):
    rng = np.random.default_rng(n)
    z = rng.standard_normal((12, n)).astype(np.float32)
    low = np.finfo(np.float32).min
    z[0] = -np.inf
    z[1] = np.nan
    z[2, 1:] = -np.inf
    z[3, rng.random(n) < 0.5] = np.nan
    z[4, rng.random(n) < 0.7] = -np.inf
    z[5, rng.random(n) < 0.5] = low
    z[6] = low
    z[7, [0, n // 2, n - 1]] = np.inf
    z[8] = np.r_[np.zeros(n - 1), 1e38]
    z[9] *= 1e-40
    z[10] *= 1e30
    z[11] = np.where(rng.random(n) < 0.5, low, np.nan)
    u = rng.random(12).astype(np.float32)
    ptr = np.concatenate(([0], np.full(12, n)))      # the first row's columns are all left out
    for limits in (dict(), dict(top_k=3), dict(top_p=0.9), dict(top_k=1000, top_p=0.5, min_p=0.2), dict(temperature=0),
                   dict(temperature=np.inf), dict(temperature=1e-30), dict(temperature=np.nan)):
        log(f"sample of special values n {n} {limits}")
        idx, _ = draw_rows(ctx, dev(z), u, **limits)
        assert idx[0] == -1 and idx[1] == -1 and idx[2] == 0
        idx, _ = draw_rows(ctx, dev(z[2:].repeat(2, 0)[:12]), u, rated=(ptr, np.arange(n)), **limits)
        assert idx[0] == -1
    # numbers outside their range
    log("sample with u and p outside their ranges")
    draw_rows(ctx, dev(z[3:8]), [-1.0, 1.0, 2.0, 0.5, 1.5], top_p=[-1.0, 2.0, np.inf, -np.inf, 1.0],
              min_p=[2.0, -1.0, 0.0, 0.5, 1.0])


@pytest.mark.parametrize("n", [40, 900, 17_770, 80_000])
def test_sample_leaves_out(ctx, n):
    """Columns of the row's own or another CSR row are left out, in any order, repeated or past the row; a row that
    leaves all out draws nothing; a user that does not exist draws nothing."""
    from paper_1603_03820_amd import serve
    rng = np.random.default_rng(n)
    rows, of = 9, 20
    lens = rng.integers(0, min(n, 700), of)
    lens[3], lens[4] = 0, n
    lists = [rng.choice(n, k, replace=False) for k in lens]
    lists[5] = np.r_[lists[5], lists[5], n, n + 31, -1, 2 ** 31 - 1].astype(np.int64)
    ptr = np.r_[0, np.cumsum([len(x) for x in lists])]
    idx = np.concatenate(lists)
    z = dev(rng.standard_normal((rows, n)).astype(np.float32))
    u = rng.random(rows).astype(np.float32)
    for limits in (dict(), dict(top_k=5), dict(top_p=0.6, top_k=400), dict(temperature=0)):
        log(f"sample leaving out, n {n} {limits}")
        got, _ = draw_rows(ctx, z, u, rated=(ptr, idx), **limits)
        assert got[4] == -1
        users = np.array([4, 5, 3, 3, 19, 0, 5, 11, 4])
        got, _ = draw_rows(ctx, z, u, rated=(ptr, idx), users=users, **limits)
        assert got[0] == -1 and got[8] == -1
        for r in range(rows):
            assert got[r] not in lists[users[r]]
    bad = dev(np.array([0, -1, 20, 3, 1, 1, 1, 1, 1], np.int32))
    got, lg = serve.als_sample(ctx, z, dev(u), rated=(dev(ptr.astype(np.int64)), dev(idx.astype(np.int32))), users=bad)
    assert got[1] == -1 and got[2] == -1 and torch.isnan(lg[1:3]).all() and bool((got[3:] >= 0).all())
    # a CSR without any entry
    none = (torch.zeros(rows + 1, dtype=torch.int64, device="cuda:0"), torch.empty(0, dtype=torch.int32, device="cuda:0"))
    a = serve.als_sample(ctx, z, dev(u), rated=none)
    b = serve.als_sample(ctx, z, dev(u))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_sample_empty_shapes(ctx):
    from paper_1603_03820_amd import serve
    log("sample of rows without columns, and without rows")
    i, lg = serve.als_sample(ctx, torch.empty(3, 0, device="cuda:0"), torch.rand(3, device="cuda:0"))
    assert i.tolist() == [-1] * 3 and lg.tolist() == [-np.inf] * 3
    i, lg = serve.als_sample(ctx, torch.empty(0, 9, device="cuda:0"), torch.rand(0, device="cuda:0"))
    assert i.numel() == 0


def test_sample_far_rows(ctx):
    """Rows whose offsets pass 2^31."""
    far = 1_200_000_001
    big = torch.empty(2 * far + 5000, dtype=torch.bfloat16, device="cuda:0")
    z = torch.as_strided(big, (3, 5000), (far, 1))
    z.copy_(torch.randn(3, 5000, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(1)))
    log("sample with rows 1.2e9 apart")
    draw_rows(ctx, z, [0.1, 0.5, 0.9], top_k=50, top_p=0.9)


def test_same_bits_every_time(ctx):
    """Every operator gives the same bits again, beside other work on other streams."""
    from paper_1603_03820_amd import serve
    g = torch.Generator("cuda:0").manual_seed(2)
    x = torch.randn(200, 96, device="cuda:0", generator=g)
    t = torch.randn(70_000, 96, device="cuda:0", generator=g)
    u = torch.rand(200, device="cuda:0", generator=g)
    results = []
    for _ in range(3):
        log("the whole path again")
        xq, xs = serve.als_quantize(ctx, x)
        tq, ts = serve.als_quantize(ctx, t)
        z = serve.als_score(ctx, xq, xs, tq, ts, dtype=torch.bfloat16)
        i, lg = serve.als_sample(ctx, z, u, temperature=2.0, top_k=2000, top_p=0.95)
        results.append([xq.clone(), xs, tq.clone(), ts, z, i, lg])
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)


# ------------------------------------------------------------- streams, graphs, refusals --


def test_other_stream_and_graph(ctx):
    """The whole path on a stream of its own, and captured and replayed on changing inputs, equals the
    eager calls."""
    from paper_1603_03820_amd import serve
    g = torch.Generator("cuda:0").manual_seed(3)
    for rows, n in ((5, 300), (40, 17_770), (3, 100_000)):
        x = torch.randn(rows, 100, device="cuda:0", generator=g)
        t = torch.randn(n, 100, device="cuda:0", generator=g)
        u = torch.rand(rows, device="cuda:0", generator=g)
        rec = serve.Recommender(ctx, x, t)
        users = torch.arange(rows, dtype=torch.int32, device="cuda:0")
        want = rec.recommend(users, u, top_k=100, top_p=0.9)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        log(f"the path on another stream, {rows} x {n}")
        got = rec.recommend(users, u, top_k=100, top_p=0.9, stream=s)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = rec.recommend(users, u, top_k=100, top_p=0.9)
        for k in range(4):
            u.copy_(torch.rand(rows, device="cuda:0", generator=g))
            x.mul_(1.1 if k else 0.9)
            log(f"graph replay {k}, {rows} x {n}")
            graph.replay()
            torch.cuda.synchronize()
            want = rec.recommend(users, u, top_k=100, top_p=0.9)
            torch.cuda.synchronize()
            assert torch.equal(want[0], out[0]) and torch.equal(want[1], out[1])


def test_recommender_end_to_end(ctx):
    """Items in 8 bits, users by index, rated items left out: against the 64-bit forms."""
    from paper_1603_03820_amd import serve
    rng = np.random.default_rng(12)
    m, n, f = 300, 4000, 100
    x, t = (rng.standard_normal((k, f)).astype(np.float32) + 1 for k in (m, n))
    x, t = x / 10, t / 10
    lens = rng.integers(0, 200, m)
    ptr = np.r_[0, np.cumsum(lens)]
    idx = np.concatenate([np.sort(rng.choice(n, k, replace=False)) for k in lens])
    users = rng.integers(0, m, 64).astype(np.int32)
    u = rng.random(64).astype(np.float32)
    rec = serve.Recommender(ctx, dev(x), dev(t), rated=(dev(ptr.astype(np.int64)), dev(idx.astype(np.int32))))
    log("recommend end to end")
    items, lg = rec.recommend(dev(users), dev(u), temperature=0.1, top_k=100, top_p=0.9)
    z = rec.scores(dev(users))
    xq, xs = serve_oracle.quantize(x)
    tq, ts = serve_oracle.quantize(t)
    exact = serve_oracle.score(xq[users], xs[users], tq, ts)
    assert np.all(np.abs(f64(z) - exact) <= serve_oracle.score_bound(exact, "f32"))
    # the 8-bit scores are those of the factors up to half a step of either side in every product
    both = (np.abs(x[users]) @ (np.ones((f, n)) * ts / 2) + (np.ones((64, f)) * xs[users, None] / 2) @ np.abs(t).T
            + f * np.outer(xs[users], ts) / 4)
    assert np.all(np.abs(exact - x[users].astype(np.float64) @ t.T.astype(np.float64)) <= both * 1.001)
    zz = f64(z)
    for r in range(64):
        left = idx[ptr[users[r]]:ptr[users[r] + 1]]
        d = serve_oracle.Draw(zz[r], float(u[r]), 0.1, 100, float(np.float32(0.9)), rated=left)
        assert d.accepts(items[r].item(), lg[r].item()) and items[r].item() not in left


def test_refusals(ctx):
    from paper_1603_03820_amd import serve
    from paper_1603_03820_amd.als import ALSError
    d = "cuda:0"
    x = torch.zeros(4, 32, device=d)
    q, s = serve.als_quantize(ctx, x)
    with pytest.raises(TypeError):
        serve.als_quantize(ctx, x.cpu())
    with pytest.raises(TypeError):
        serve.als_quantize(ctx, x.double())
    with pytest.raises(ValueError):
        serve.als_quantize(ctx, x.t())
    with pytest.raises(ValueError):
        serve.als_quantize(ctx, x[:, 0])
    with pytest.raises(TypeError):
        serve.als_quantize(ctx, x, users=torch.zeros(2, dtype=torch.int64, device=d))
    with pytest.raises(ValueError):
        serve.als_quantize(ctx, x, q=torch.empty(3, 32, dtype=torch.int8, device=d))
    with pytest.raises(ValueError):
        serve.als_score(ctx, q, s, q[:, :31], s)
    with pytest.raises(ValueError):
        serve.als_score(ctx, q, s[:3], q, s)
    with pytest.raises(TypeError):
        serve.als_score(ctx, q, s, q, s, dtype=torch.float64)
    with pytest.raises(ValueError):
        serve.als_score(ctx, q, s, q, s, out=torch.empty(1, 4, device=d).expand(4, 4))
    u = torch.rand(4, device=d)
    ptr, col = torch.zeros(4, dtype=torch.int64, device=d), torch.zeros(1, dtype=torch.int32, device=d)
    with pytest.raises(ValueError):
        serve.als_sample(ctx, x, u[:3])
    with pytest.raises(ValueError):
        serve.als_sample(ctx, x, u, rated=(ptr, col))          # three CSR rows for four rows
    with pytest.raises(ValueError):
        serve.als_sample(ctx, x, u, users=torch.zeros(4, dtype=torch.int32, device=d))
    with pytest.raises(TypeError):
        serve.als_sample(ctx, x, u, top_k=torch.zeros(4, device=d))
    with pytest.raises(ALSError) as e:
        serve.als_quantize(ctx, torch.zeros(2, 0, device=d))
    assert e.value.code == -2
    # the C boundary's own
    lib, P, h = serve._lib, ctypes.c_void_p, ctx.handle
    p = lambda t, off=0: P(t.data_ptr() + off)  # noqa: E731
    f32 = torch.zeros(4096, device=d)
    i8 = torch.zeros(4096, dtype=torch.int8, device=d)
    sc = torch.zeros(64, device=d)

    def quantize(x=p(f32), dtype=0, of=4, ldx=32, users=None, rows=4, f=32, q=p(i8), ldq=32, scale=p(sc)):
        return lib.als_quantize(h, x, dtype, of, ldx, users, rows, f, q, ldq, scale, None)
    assert quantize() == 0 and quantize(rows=0, q=None, scale=None) == 0
    assert quantize(x=None) == -1 and quantize(q=None) == -1 and quantize(scale=None) == -1
    assert quantize(dtype=3) == -1 and quantize(dtype=-1) == -1 and quantize(rows=-1) == -1
    assert quantize(ldx=31) == -1 and quantize(ldq=31) == -1 and quantize(rows=5) == -1
    assert quantize(f=0) == -2 and quantize(f=131_072, ldx=1 << 20, ldq=1 << 20) == -2
    assert quantize(x=p(f32, 2)) == -4 and quantize(scale=p(sc, 1)) == -4
    assert quantize(q=p(f32, 64)) == -6 and quantize(scale=p(f32)) == -6 and quantize(scale=p(i8, 64)) == -6

    def score(xq=p(i8), ldx=32, xs=p(sc), m=4, tq=p(i8), ldt=32, ts=p(sc), n=4, f=32, out=p(f32), dtype=0, ldo=4):
        return lib.als_score(h, xq, ldx, xs, m, tq, ldt, ts, n, f, out, dtype, ldo, None)
    assert score() == 0 and score(m=0, xq=None) == 0 and score(n=0, out=None) == 0
    assert score(xq=None) == -1 and score(ts=None) == -1 and score(out=None) == -1 and score(m=-1) == -1
    assert score(ldx=31) == -1 and score(ldt=31) == -1 and score(ldo=3) == -1 and score(dtype=7) == -1
    assert score(f=0) == -2 and score(f=131_072, ldx=1 << 20, ldt=1 << 20) == -2
    assert score(xs=p(sc, 2)) == -4 and score(out=p(f32, 2)) == -4 and score(out=p(f32, 1), dtype=1) == -4
    assert score(out=p(i8, 64)) == -6 and score(out=p(sc)) == -6

    idx, lg, uu = torch.zeros(8, dtype=torch.int32, device=d), torch.zeros(8, device=d), torch.zeros(8, device=d)
    rp, rc = torch.zeros(9, dtype=torch.int64, device=d), torch.zeros(8, dtype=torch.int32, device=d)
    lim = serve._Limits(temperature_all=1.0, top_p_all=1.0)

    def sample(z=p(f32), dtype=0, rows=4, n=32, ldz=32, limits=lim, u=p(uu), ptr=None, col=None, users=None, of=0,
               index=p(idx), log=p(lg)):
        return lib.als_sample(h, z, dtype, rows, n, ldz, None if limits is None else ctypes.byref(limits), u, ptr, col,
                              users, of, index, log, None)
    assert sample() == 0 and sample(rows=0, z=None, u=None) == 0 and sample(log=None) == 0
    assert sample(n=0, z=None) == 0 and sample(ptr=p(rp), col=p(rc), of=4) == 0
    assert sample(z=None) == -1 and sample(u=None) == -1 and sample(index=None) == -1 and sample(limits=None) == -1
    assert sample(ldz=31) == -1 and sample(n=4_194_305, ldz=4_194_305) == -1 and sample(dtype=3) == -1
    assert sample(ptr=p(rp)) == -1 and sample(col=p(rc)) == -1 and sample(users=p(rc)) == -1
    assert sample(ptr=p(rp), col=p(rc), of=3) == -1 and sample(rows=-1) == -1
    assert sample(z=p(f32, 2)) == -4 and sample(ptr=p(rp, 4), col=p(rc), of=4) == -4 and sample(index=p(idx, 2)) == -4
    assert sample(index=p(f32)) == -6 and sample(log=p(uu)) == -6 and sample(log=p(idx)) == -6
    torch.cuda.synchronize()
    assert bool((idx[:4] >= 0).all())
    c = serve.Context(0)
    c.close()
    with pytest.raises(ValueError):
        serve.als_quantize(c, x)


def test_recommend_command():
    """The command's run on the tiny workload: every user gets an item it has not rated, within the best 50 of the
    8-bit scores, the same on every run."""
    import synth
    from paper_1603_03820_amd import recommend
    p = synth.config("tiny")
    log("train and recommend, tiny workload")
    rmse, items, lg, _ = recommend.run("tiny", iters=3, batch=300)
    assert len(rmse) == 3 and rmse[2] < rmse[0]
    items = items.cpu().numpy()
    assert items.shape == (p.m,) and items.min() >= 0 and items.max() < p.n
    assert bool((lg <= 0).all()) and bool((lg >= -np.log(50) - 20).all())
    for u in range(p.m):
        assert items[u] not in p.colidx[p.rowptr[u]:p.rowptr[u + 1]]
    log("and with other batches")
    _, again, lg2, _ = recommend.run("tiny", iters=3, batch=1000)
    assert np.array_equal(items, again.cpu().numpy()) and torch.equal(lg, lg2)
