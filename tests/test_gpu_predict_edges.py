"""The prediction operators on the GPU at the ends of what their definitions allow, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

from tests import predict_oracle
from tests.gpu_util import log
from tests.test_gpu_predict import D, TYPES, ctx, dev, f64, lists, row_of, strided  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,f", [(2, 5, 8), (2, 5, 72), (1, 70, 1000), (16, 300, 128), (31, 900, 200), (70, 200, 520), (600, 9000, 64)])
def test_users_of_a_model_without_any(ctx, dtype, m, n, f):  # noqa: F811
    """X without rows, whose memory need not be there: every user's predictions are NaN, and nothing of X is read."""
    from paper_1603_03820_amd import predict
    x, t = torch.empty(0, f, dtype=TYPES[dtype], device=D), torch.ones(n, f, dtype=TYPES[dtype], device=D)
    users = torch.arange(-1, m - 1, dtype=torch.int32, device=D)
    log(f"predict of an empty X, {dtype} {m}x{n}x{f}")
    for activation in ("none", "gelu"):
        got = predict.als_predict(ctx, x, t, users=users, user_offset=torch.empty(0, device=D), item_offset=torch.ones(n, device=D),
                                  activation=activation, residual=torch.ones(m, n, device=D))
        assert got.shape == (m, n) and bool(torch.isnan(got).all())


@pytest.mark.parametrize("with_rated", [False, True])
def test_fit_with_users_that_do_not_exist(ctx, with_rated):  # noqa: F811
    """They count for nothing, with and without a CSR of rated items."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(14)
    x, t = dev(rng.standard_normal((40, 8)).astype(np.float32)), dev(rng.standard_normal((60, 8)).astype(np.float32))
    rated = tuple(dev(a) for a in lists(rng, 40, 60, 20)) if with_rated else None
    who, what = rng.integers(0, 40, 200).astype(np.int32), rng.integers(0, 60, 200).astype(np.int32)
    bad = np.array([-1, 40, 2 ** 31 - 1, -2 ** 31], np.int32)
    log(f"fit with users that do not exist, rated {with_rated}")
    a, b, c = (predict.Predictor(ctx, x, t, rated=rated) for _ in range(3))
    got = a.fit_offsets(dev(np.concatenate([bad[:2], who, bad[2:]])), dev(np.concatenate([what[:2], what, what[:2]])), 0.5, 3)
    want = b.fit_offsets(dev(who), dev(what), 0.5, 3)
    assert bool(torch.isfinite(a.item_offset).all()) and torch.allclose(a.item_offset, b.item_offset, atol=1e-5)
    assert got == pytest.approx(want, abs=4e-5)
    assert c.fit_offsets(dev(bad), dev(what[:4]), 0.5, 2) == [0.0, 0.0] and not c.item_offset.any()


def fit64(x, t, who, what, temperature, steps, rate, rated=None):
    """fit_offsets in 64 bits: (the means before each step, the offsets after each)."""
    n, b, means, offsets = t.shape[0], np.zeros(t.shape[0]), [], []
    for _ in range(steps):
        expected, counts, total = np.zeros(n), np.zeros(n), []
        for u, g in zip(who, what):
            row = predict_oracle.Row(x[u].astype(np.float64) @ t.T.astype(np.float64) + b, temperature,
                                     () if rated is None else row_of(rated, u))
            if row.log(g) > -np.inf:
                total.append(row.log(g))
                expected += np.exp(row.log_p)
                counts[g] += 1
        means.append(np.mean(total))
        b = b + rate * temperature * (counts - expected) / np.maximum(np.maximum(counts, expected), 1e-6)
        offsets.append(b)
    return means, offsets


@pytest.mark.parametrize("with_rated", [False, True])
@pytest.mark.parametrize("batch", [1000, 150])
def test_fit_offsets_against_64_bits(ctx, with_rated, batch):  # noqa: F811
    """Each step's mean, which rises (a step is no longer than iterative scaling's, T log(c / e)), and the offsets."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(21)
    users, n, count, t = 100, 50, 400, 0.7
    x, theta = (0.3 * rng.standard_normal((users, 8))).astype(np.float32), rng.standard_normal((n, 8)).astype(np.float32)
    rated = lists(rng, users, n, 10) if with_rated else None
    who, what = rng.integers(0, users, count).astype(np.int32), (rng.zipf(1.5, count) % n).astype(np.int32)
    want, offsets = fit64(x, theta, who, what, t, 8, 0.5, rated)
    assert all(b > a + 1e-4 for a, b in zip(want, want[1:]))
    log(f"fit against 64 bits, rated {with_rated}, batch {batch}")
    rd = None if rated is None else tuple(dev(a) for a in rated)
    short, whole = (predict.Predictor(ctx, dev(x), dev(theta), rated=rd) for _ in range(2))
    means = short.fit_offsets(dev(who), dev(what), t, 3, 0.5, batch)
    # a score is off by at most 2.2e-5 (predict_bound at sizes up to 3.5), log p and the share of an expected count by 2 / T
    # of that; the sums over 400 rows by 400 units: 1.2e-4 of a step of at most rate T, which each later step doubles at most
    off = 0.5 * t * 1.2e-4 * 7
    assert np.abs(f64(short.item_offset) - offsets[2]).max() <= off
    assert means == pytest.approx(want[:3], abs=2 * off / t + 1e-4)
    means = whole.fit_offsets(dev(who), dev(what), t, 8, 0.5, batch)
    assert all(b > a for a, b in zip(means, means[1:]))


@pytest.mark.parametrize("dtype,nans", [("f32", [0x7F800001, 0x7FC00000, 0x7F80FFFF, -1, -0x7FFFFF, -0x400000]),
                                        ("f16", [0x7C01, 0x7E00, 0x7FFF, -1, -0x3FF]), ("bf16", [0x7F81, 0x7FC0, 0x7FFF, -1, -0x7F])])
@pytest.mark.parametrize("n", [300, 20_000, 40_000])
def test_every_kind_of_nan_is_left_out(ctx, dtype, nans, n):  # noqa: F811
    """Quiet and signalling ones of both signs, at the best columns of a row and in most of another, give the bits that
    -inf gives in their places."""
    from paper_1603_03820_amd import predict
    rng = np.random.default_rng(n)
    z = dev((2 * rng.standard_normal((3, n))).astype(np.float32), TYPES[dtype])
    least = z.clone()
    bits = z.view(torch.int32 if dtype == "f32" else torch.int16)
    values = torch.tensor(nans, dtype=bits.dtype, device=D)
    at = [torch.topk(z[0].float(), 40).indices, torch.arange(n - 5, device=D), torch.arange(0, n, 2, device=D)]
    for row, columns in enumerate(at):
        bits[row, columns] = values[torch.arange(columns.numel(), device=D) % values.numel()]
        least[row, columns] = float("-inf")
    given = dev(rng.integers(0, n, (3, 5)).astype(np.int32))
    given[:, 0] = torch.stack([c[0] for c in at]).int()
    log(f"NaN of every kind, {dtype}, {n} columns")
    got, want = (predict.als_log_prob(ctx, s, given, 0.7, 9) for s in (z, least))
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    ones, h = torch.ones(3, 5, device=D), torch.ones(3, device=D)
    got, want = (predict.als_log_prob_grad(ctx, s, given, want, ones, h, 0.7, columns=True) for s in (z, least))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
