"""als_score in every tile shape that its rule picks, every output against the exact product, in each output type.
Which kernel ran is asked of the profiler, so that a changed rule cannot leave a shape untested."""
import re

import pytest
import torch

from tests.gpu_util import log
from tests.serve_oracle import HALF_ULP, TINY

pytestmark = pytest.mark.gpu
D = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}

# waves of users x waves of items, fragments of 16 a wave: the tile's users and items are their products times 16
CASES = [("16x64", TYPES, 1, 20_000, 100), ("16x64", TYPES, 100, 700, 300), ("16x64", TYPES, 16, 9_001, 1_111),
         ("64x64", TYPES, 1_030, 1_030, 130), ("64x64", TYPES, 1_001, 1_103, 37), ("64x64", TYPES, 1_500, 1_031, 1_040),
         ("64x128", TYPES, 2_100, 2_100, 130), ("64x128", TYPES, 2_047, 2_090, 100), ("64x128", TYPES, 4_097, 1_025, 1_030),
         ("128x128", TYPES, 3_000, 3_000, 200), ("128x128", TYPES, 2_999, 3_077, 1_100),
         ("128x128", ["f32"], 6_000, 6_000, 100), ("128x128", ["f32"], 6_001, 5_999, 128), ("128x128", ["f32"], 5_905, 5_889, 5),
         ("32x256", ["f16", "bf16"], 2_060, 8_200, 100), ("32x256", ["f16", "bf16"], 6_001, 5_999, 128),
         ("32x256", ["f16", "bf16"], 40_003, 513, 37),
         ("256x256", TYPES, 4_100, 4_100, 1_100), ("256x256", TYPES, 4_097, 4_351, 1_025), ("256x256", TYPES, 3_845, 4_111, 2_048)]


@pytest.fixture(scope="module")
def ctx():
    from paper_1603_03820_amd import serve
    c = serve.Context(0)
    yield c
    c.close()


def tile_of(kernel):
    wu, wi, fu, fi = map(int, re.search(r"k_score_tiles<[^,]+, (\d+), (\d+), (\d+), (\d+), \d+>", kernel).groups())
    return f"{16 * wu * fu}x{16 * wi * fi}"


def tiles_run(call):
    """The tiles of the kernels that a call queued."""
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        call()
        torch.cuda.synchronize()
    return {tile_of(e.key) for e in prof.key_averages() if "k_score_tiles" in e.key}


@pytest.mark.parametrize("tile,types,m,n,f", CASES)
def test_score_in_every_tile(ctx, tile, types, m, n, f):
    from paper_1603_03820_amd import serve
    g = torch.Generator(D).manual_seed(m + 3 * n + 7 * f)

    def rows(k, layout):
        # as als_quantize leaves them (other values up to the stride), or rows that are laid out anew
        ld = ((f + 15) // 16 + 1) * 16 if layout == 0 else f + 3
        return torch.randint(-128, 128, (k, ld), dtype=torch.int8, device=D, generator=g)[:, :f]
    xs = (0.5 + torch.rand(m, device=D, generator=g)) / f ** 0.5 / 100
    ts = (0.5 + torch.rand(n, device=D, generator=g)) / 100
    for layout in (0, 1):
        xq, tq = rows(m, layout), rows(n, layout)
        # whole numbers below 2^53: exact in 64-bit floats
        exact = torch.mm(xq.double(), tq.double().t().contiguous()).mul_(xs.double()[:, None]).mul_(ts.double())
        for dtype in types:
            out = torch.full((m, n + 3 * layout), 9.0, dtype=TYPES[dtype], device=D)
            log(f"score {dtype} {m} x {n} x {f} layout {layout}, tile {tile}")
            ran = tiles_run(lambda: serve.als_score(ctx, xq, xs, tq, ts, out=out[:, :n]))
            assert ran == {tile}
            # the sum's conversion and two products in fp32, then the output's own rounding
            one = (3 * 2.0 ** -24 + (0 if dtype == "f32" else HALF_ULP[dtype])) * (1 + 2.0 ** -7)
            off = (out[:, :n].double() - exact).abs_().sub_(exact.abs() * one)
            assert off.max().item() <= TINY[dtype]
            assert bool((out[:, n:] == 9.0).all())


def test_every_tile_of_the_library_is_here():
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    source = open(os.path.join(root, "paper_1603_03820_amd", "csrc", "serve.hip")).read()
    shapes = {tuple(map(int, s)) for s in re.findall(r"launch_tiles<T, (\d+), (\d+), (\d+), (\d+), \d+>\(a\)", source)}
    assert {f"{16 * wu * fu}x{16 * wi * fi}" for wu, wi, fu, fi in shapes} == {c[0] for c in CASES}
