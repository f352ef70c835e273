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
