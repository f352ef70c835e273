"""als_quantize over the whole range of fp32, against the definition with roundings to 24 bits that know no largest
or least exponent (the library and tests/serve_oracle.py scale rows past 1e36 down before 127 x overflows)."""
import numpy as np
import pytest

from tests import serve_oracle


def rounded(v):
    """Float64 values to 24 significant bits, ties to even, whatever their exponent."""
    mantissa, exponent = np.frexp(v)
    return np.ldexp(np.rint(np.ldexp(mantissa, 24)), exponent - 24)


def quantize(x):
    """127 x has 31 bits, which float64 holds; a quotient of two numbers of 24 bits that is rounded to 53 and then to 24
    is the one rounded to 24."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x).max(axis=1, keepdims=True)
    return np.rint(rounded(rounded(x * 127.0) / a)).astype(np.int8)


def rows(f, seed=1):
    """Rows whose largest magnitudes spread over fp32's range, those around the library's bounds among them; values
    at and beside the ties of a row (k + 1/2 of 127 steps)."""
    rng = np.random.default_rng(seed)
    largest = np.float32(np.r_[np.finfo(np.float32).max, 3e38, 2.7e38, 2.6e36, 1.01e36, 1e36, 0.99e36, 1.0, 1e-30, 1.01e-36,
                               1e-36, 0.99e-36, 1.2e-38, 1e-40, 3 * 2.0 ** -149, 2.0 ** -149,
                               2.0 ** rng.uniform(-149, 128, 200)])
    part = rng.uniform(-1, 1, (largest.size, f))
    ties = (rng.integers(-127, 127, part.shape) + 0.5) / 127
    part = np.where(rng.random(part.shape) < 0.4, ties * (1 + rng.integers(-1, 2, part.shape) * 2.0 ** -23), part)
    x = (part * largest[:, None].astype(np.float64)).astype(np.float32)
    x[:, 0] = largest * rng.choice([-1, 1], largest.size)
    return x


def test_the_oracle_rounds_as_the_definition():
    x = rows(300)
    assert np.array_equal(serve_oracle.quantize(x)[0], quantize(x))


@pytest.mark.gpu
@pytest.mark.parametrize("f", [1, 5, 100, 300, 2000, 10_000])
def test_quantize_rounds_as_the_definition(f):
    import torch
    from paper_1603_03820_amd import serve
    from tests.gpu_util import log
    ctx = serve.Context(0)
    x = rows(f, f)
    log(f"quantize over the range of fp32, f {f}")
    q, s = serve.als_quantize(ctx, torch.from_numpy(x).to("cuda:0"))
    assert np.array_equal(q.cpu().numpy(), quantize(x))
    assert np.array_equal(s.cpu().numpy(), np.abs(x).max(axis=1) * (np.float32(1) / np.float32(127)))
