"""als_sample on rows with NaN of every kind: each leaves its column out, as -inf does."""
import numpy as np
import pytest
import torch

from tests.gpu_util import log
from tests.test_gpu_predict import D, TYPES, dev, lists

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_1603_03820_amd import serve
    c = serve.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype,nans", [("f32", [0x7F800001, 0x7FC00000, 0x7F80FFFF, -1, -0x7FFFFF, -0x400000]),
                                        ("f16", [0x7C01, 0x7E00, 0x7FFF, -1, -0x3FF]), ("bf16", [0x7F81, 0x7FC0, 0x7FFF, -1, -0x7F])])
@pytest.mark.parametrize("n", [60, 300, 5000, 20_000, 60_000, 100_000])
def test_every_kind_of_nan_is_left_out(ctx, dtype, nans, n):
    """Quiet and signalling ones of both signs, at the best columns of a row, at the last of one and in half of another; the
    draws are those of rows with -inf there."""
    from paper_1603_03820_amd import serve
    rng = np.random.default_rng(n)
    z = dev((2 * rng.standard_normal((4, n))).astype(np.float32), TYPES[dtype])
    least = z.clone()
    bits = z.view(torch.int32 if dtype == "f32" else torch.int16)
    values = torch.tensor(nans, dtype=bits.dtype, device=D)
    for row, columns in enumerate((torch.topk(z[0].float(), 40).indices, torch.arange(n - 5, device=D), torch.arange(0, n, 2, device=D),
                                   torch.arange(n - 7, n, device=D))):
        bits[row, columns] = values[torch.arange(columns.numel(), device=D) % values.numel()]
        least[row, columns] = float("-inf")
    rated = tuple(dev(a) for a in lists(rng, 4, n, 20))
    for k, limits in enumerate((dict(), dict(top_k=5), dict(top_k=5, top_p=0.7), dict(top_p=0.6), dict(min_p=0.05), dict(temperature=0.0))):
        u = dev(rng.random(4).astype(np.float32))
        log(f"als_sample of NaN of every kind, {dtype}, {n} columns, {limits}")
        got, want = (serve.als_sample(ctx, s, u, rated=rated if k % 2 else None, **limits) for s in (z, least))
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert bool((want[0][[0, 2, 3]] >= 0).all())
