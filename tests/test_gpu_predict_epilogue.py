"""What follows a product of als_predict -- offsets, activation, residual, users that do not exist -- in every shape of its
tiles, and the activations over the range of their arguments, against 64-bit forms on the device."""
import math

import pytest
import torch

from tests import predict_oracle
from tests.gpu_util import log
from tests.test_gpu_predict import D, TYPES, ctx, strided  # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LEAST = 2.0 ** -126      # exponentials below it are 0
# Roundings of fp32 in an activation's value, as a share of it.  An exponential is off by 3.1 (the instruction's unit is 2, a
# product rounds), a reciprocal by 1.1 after its Newton step.
#   sigmoid, silu  1 + e: half of the exponential's, and 1; reciprocal; product with e; with y: 3.1 + 2.6 + 1.1 + 1 + 1
#   gelu           t by 3.1 (constant, sum, reciprocal), which moves t q(t) by at most 3.8 times as much; Horner's steps and
#                  coefficients 6.7; the exponential 3.1; the polynomial's own 0.7; three products: 25.3
#   tanh           the library's, 5 units of 2
OFF = {"none": 0, "clip": 0, "relu": 0, "sigmoid": 9, "silu": 9, "gelu": 26, "tanh": 10}
# of 16-bit results: an exponent's three roundings count |y| (or y^2 / 2, up to 85) times: 2^-16 up to |y| = 87, and with
# GELU's polynomial (1e-5) 2^-15
OFF16 = dict(OFF, sigmoid=2 ** 8, silu=2 ** 8, gelu=2 ** 9)


def activated(y, name, low=-math.inf, high=math.inf):
    if name == "clip":
        return y.clamp(low, high)
    if name == "relu":
        return y.clamp(min=0.0)
    if name == "gelu":
        return 0.5 * y * torch.special.erfc(y * -math.sqrt(0.5))
    if name == "silu":
        return y * torch.special.expit(y)
    if name == "sigmoid":
        return torch.special.expit(y)
    return torch.tanh(y) if name == "tanh" else y


def bound(act, name, out, residual=None):
    """For an exact y: the activation's roundings, the residual's sum, the result's rounding to its type."""
    off = (OFF if out == "f32" else OFF16)[name] * U * act.abs() + (LEAST if OFF[name] else 0.0)
    want = act if residual is None else act + residual
    if residual is not None:
        off = off + U * want.abs()
    half = 0.0 if out == "f32" else predict_oracle.HALF_ULP[out]
    return want, off * (1 + half) + half * want.abs() + (predict_oracle.TINY[out] if half else 0.0)


def agree(got, act, name, out, residual=None):
    want, off = bound(act, name, out, residual)
    return bool(((got.double() - want).abs() <= off).all())


# users, items, f: rows of 16 bits at multiples of 16 bytes in each shape of tiles, with f whole and cut; others in theirs
SHAPES = [
    (5, 900, 264), (13, 300, 4096),           # 16 x 64; f cut
    (31, 9000, 200), (32, 500, 1032),         # 32 x 128; f cut
    (200, 900, 104), (70, 300, 2000),         # 64 x 64; f cut
    (2300, 2100, 64), (1100, 6000, 128),      # 64 x 128 in steps of 32 values
    (1100, 2900, 200), (3001, 1203, 136),     # 64 x 128 in steps of 64
    (3000, 3001, 200),                        # 128 x 128
    (4101, 4105, 520), (4096, 4096, 1024),    # 256 x 256
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("m,n,f", SHAPES)
def test_ways_out(ctx, dtype, odd, m, n, f):  # noqa: F811
    """Values whose sums fp32 holds, so that an activation's argument is exact.  `odd`: rows that are not at multiples of
    16 bytes, which other kernels take."""
    from paper_1603_03820_amd import predict
    gen = torch.Generator(device=D).manual_seed(m + n + f)

    def whole(*size, most=3):
        return torch.randint(-most, most + 1, size, device=D, generator=gen)
    unit = 2.0 ** -round(math.log2(4 * math.sqrt(f) / 3))      # arguments of about 3
    x, t = whole(m + 3, f).to(TYPES[dtype]), (whole(n, f) * unit).to(TYPES[dtype])
    a, b = (whole(r, most=64) * unit for r in (m + 3, n))
    if odd:
        x, t = strided(x, 3, 1), strided(t, 3, 1)
    users = torch.randint(0, m + 3, (m,), device=D, generator=gen, dtype=torch.int32)
    bad = torch.tensor([0, m // 2, m - 1], device=D)
    users[bad] = torch.tensor([-1, m + 3, 2 ** 31 - 1], device=D, dtype=torch.int32)
    there = torch.ones(m, dtype=torch.bool, device=D)
    there[bad] = False
    at = torch.where(there, users, 0).long()
    y = x.double()[at] @ t.double().t() + a.double()[at][:, None] + b.double()
    y = y[there]
    other = "f32" if dtype != "f32" else "bf16"
    for name, out, mode in (("gelu", dtype, "strided"), ("silu", dtype, "in place"), ("sigmoid", other, "none"), ("clip", other, "strided"),
                            ("none", dtype, "strided"), ("relu", dtype, "none"), ("gelu", other, "in place"), ("tanh", dtype, "none")):
        log(f"{dtype} odd {odd} {m}x{n}x{f} {name} to {out}, residual {mode}")
        limits = dict(low=-2.0, high=1.5) if name == "clip" else {}
        r = None if mode == "none" else (whole(m, n, most=40) * unit).to(TYPES[out])
        kept = r
        if mode == "strided":
            r = strided(r, 5, 3)
        to = {"strided": strided(torch.zeros(m, n, dtype=TYPES[out], device=D), 2, 1), "in place": r.clone() if r is not None else None}.get(mode)
        got = predict.als_predict(ctx, x, t, users, a, b, name, residual=to if mode == "in place" else r, out=to, dtype=TYPES[out], **limits)
        assert bool(torch.isnan(got[~there]).all())
        got = got[there]
        act = activated(y, name, **limits)
        res = None if kept is None else kept[there].double()
        if OFF[name] == 0:
            assert torch.equal(got, (act if res is None else act + res).to(TYPES[out]))
        else:
            assert agree(got, act, name, out, res)
        if mode == "strided":      # nothing beside the results
            flat = torch.as_strided(to, (to.untyped_storage().nbytes() // to.element_size(),), (1,), 0)
            beside = torch.ones(flat.shape, dtype=torch.bool, device=D)
            torch.as_strided(beside, (m, n), (n + 2, 1), 1).fill_(False)
            assert bool((flat[beside] == 77).all())


RANGES = {"gelu": (-13.0, math.inf), "silu": (-87.0, math.inf), "sigmoid": (-87.0, math.inf), "tanh": (-math.inf, math.inf),
          "relu": (-math.inf, math.inf)}


def below(got, act):
    """Past the range in which an exponential is at least 2^-126 a result may be 0, but is no larger than the formula's."""
    return bool((got.double().abs() <= act.abs() * 1.01 + LEAST).all())


@pytest.mark.parametrize("name", sorted(RANGES))
@pytest.mark.parametrize("m", [1, 40, 300])
def test_activations_over_their_range(ctx, name, m):  # noqa: F811
    """fp32: arguments as they are (f = 1, times 1), down to the least normal result."""
    from paper_1603_03820_amd import predict
    gen = torch.Generator(device=D).manual_seed(m)
    n = 40_000
    y = torch.empty(n, device=D).uniform_(-13, 13, generator=gen)
    y[:10_000] = torch.empty(10_000, device=D).uniform_(-87, 87, generator=gen)
    y[10_000:20_000] = torch.exp(torch.empty(10_000, device=D).uniform_(-60, 2.5, generator=gen)) * torch.sign(y[10_000:20_000])
    y[20_000:21_000] = torch.empty(1000, device=D).uniform_(-1e4, 1e4, generator=gen)
    scale = torch.ones(m, 1, device=D)
    scale[m // 2] = 0.5
    for out in ("f32", "f16", "bf16"):
        log(f"{name} of {n} arguments, {m} users, to {out}")
        got = predict.als_predict(ctx, scale, y[:, None].contiguous(), activation=name, dtype=TYPES[out])
        for s in {0, m // 2}:
            arg = y.double() * scale[s].double()
            inside = (arg >= RANGES[name][0]) & (arg <= RANGES[name][1])
            act = activated(arg, name)
            if out == "f16":
                inside &= act.abs() < 60_000
            assert agree(got[s][inside], act[inside], name, out)
            rest = arg < RANGES[name][0]
            assert below(got[s][rest], act[rest])


@pytest.mark.parametrize("name", sorted(RANGES))
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("m", [1, 40, 300])
def test_activations_of_every_16_bit_argument(ctx, name, dtype, m):  # noqa: F811
    """Every finite value of the type as an argument, from rows at multiples of 16 bytes whose other values are NaN."""
    from paper_1603_03820_amd import predict
    y = torch.arange(-2 ** 15, 2 ** 15, device=D).to(torch.int16).view(TYPES[dtype])
    y = y[torch.isfinite(y)]
    y = y[y.abs() <= 1e4]
    t = torch.full((y.numel(), 8), float("nan"), dtype=TYPES[dtype], device=D)
    t[:, 0] = y
    x = torch.full((m, 8), float("nan"), dtype=TYPES[dtype], device=D)
    x[:, 0] = 1
    for out in (dtype, "f32"):
        log(f"{name} of every {dtype} argument up to 1e4, {m} users, to {out}")
        got = predict.als_predict(ctx, x[:, :1], t[:, :1], activation=name, dtype=TYPES[out])
        assert torch.equal(got[0], got[m // 2]) and torch.equal(got[0], got[m - 1])
        arg = y.double()
        act = activated(arg, name)
        inside = (arg >= RANGES[name][0]) & (arg <= RANGES[name][1])
        assert agree(got[0][inside], act[inside], name, out)
        assert below(got[0][~inside], act[~inside])
