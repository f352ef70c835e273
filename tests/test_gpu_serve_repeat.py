"""The serving operators' bits beside other work on the card."""
import pytest
import torch

from tests.gpu_util import log

pytestmark = pytest.mark.gpu
D = "cuda:0"


def test_same_bits_beside_other_work():
    """Every operator in a row, short and long rows, while products and copies run on another stream: the bits of the
    same calls alone."""
    from paper_1603_03820_amd import serve
    g = torch.Generator(D).manual_seed(2)
    x = torch.randn(200, 96, device=D, generator=g)
    items = [torch.randn(n, 96, device=D, generator=g) for n in (900, 17_770, 70_000)]
    u = torch.rand(200, device=D, generator=g)
    a, b = torch.randn(2048, 2048, device=D, generator=g), torch.empty(2048, 2048, device=D)
    big, copy = torch.empty(1 << 28, dtype=torch.uint8, device=D), torch.empty(1 << 28, dtype=torch.uint8, device=D)
    ctx = serve.Context(0)

    def path():
        results = []
        for t in items:
            xq, xs = serve.als_quantize(ctx, x)
            tq, ts = serve.als_quantize(ctx, t)
            z = serve.als_score(ctx, xq, xs, tq, ts, dtype=torch.bfloat16)
            results += [xq, xs, tq, ts, z]
            for limits in (dict(temperature=2.0, top_k=100, top_p=0.95), dict(temperature=2.0, top_p=0.9),
                           dict(temperature=1.0), dict(top_k=5000)):
                results += serve.als_sample(ctx, z, u, **limits)
        return results
    alone = path()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    beside = 0
    for turn in range(5):
        log(f"beside other work, turn {turn}")
        with torch.cuda.stream(side):
            for _ in range(60):
                torch.mm(a, a, out=b)
                copy.copy_(big)
        again = path()
        done = torch.cuda.Event()
        done.record()
        done.synchronize()
        beside += not side.query()
        torch.cuda.synchronize()
        assert len(again) == len(alone) and all(torch.equal(p, q) for p, q in zip(alone, again))
    assert beside        # the other stream was still at work after the path's end, at least once
