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
