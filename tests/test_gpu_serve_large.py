"""Calls of more rows than one launch of 2^32 threads takes: every row is answered, those past the first launch as
the others.  The answers are known exactly."""
import pytest
import torch

from tests.gpu_util import log

pytestmark = pytest.mark.gpu
D = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    from paper_1603_03820_amd import serve
    c = serve.Context(0)
    yield c
    c.close()
    torch.cuda.empty_cache()


def pattern(rows, period, dtype):
    """r % period for r < rows."""
    return torch.arange(period, device=D).to(dtype).repeat((rows + period - 1) // period)[:rows]


@pytest.mark.parametrize("rated", ["none", "by_users", "by_rows"])
def test_sample_of_many_rows(ctx, rated):
    from paper_1603_03820_amd import serve
    rows, n = 2 ** 26 + 5, 5
    at = pattern(rows, 3, torch.int8)
    z = torch.zeros(rows, n, dtype=torch.float16, device=D)
    z.scatter_(1, at[:, None].long(), 2.0)
    z[:, 4] = 1.0                                            # the best column of a row that leaves out its own
    u = torch.full((rows,), 0.5, device=D)
    t = pattern(rows, 2, torch.float32).mul_(2.0 ** -8)      # the best column; and a temperature that leaves no other
    index = torch.full((rows,), -7, dtype=torch.int32, device=D)
    args, want = {}, at
    if rated == "by_users":
        # CSR row 1 leaves out columns 0 to 3, row 0 nothing, and there is no row 2
        users = pattern(rows, 7, torch.int32).clamp_(max=2)
        args = dict(rated=(torch.tensor([0, 0, 4], device=D), torch.arange(4, dtype=torch.int32, device=D)), users=users)
        want = torch.where(users == 0, at.int(), torch.where(users == 1, 4, -1))
    elif rated == "by_rows":
        # the last row leaves out all but column 4
        ptr = torch.zeros(rows + 1, dtype=torch.int64, device=D)
        ptr[rows] = 4
        args = dict(rated=(ptr, torch.arange(4, dtype=torch.int32, device=D)))
        want = at.int()
        want[rows - 1] = 4
    log(f"sample {rows} x {n}, rated {rated}")
    serve.als_sample(ctx, z, u, temperature=t, index=index, **args)
    assert torch.equal(index, want.int())


def test_quantize_of_many_rows(ctx):
    from paper_1603_03820_amd import serve
    rows = 2 ** 30 + 5
    x = pattern(rows, 5, torch.float16)[:, None]
    q = torch.full((rows, 1), 99, dtype=torch.int8, device=D)
    scale = torch.full((rows,), -7.0, device=D)
    log(f"quantize {rows} x 1")
    serve.als_quantize(ctx, x, q=q, scale=scale)
    assert torch.equal(q[:, 0], pattern(rows, 5, torch.int8).clamp_(max=1).mul_(127))
    table = torch.arange(5, dtype=torch.float32, device=D) * (torch.ones((), device=D) / 127)
    assert torch.equal(scale, table.repeat((rows + 4) // 5)[:rows])


def test_quantize_of_many_wide_rows_by_index(ctx):
    from paper_1603_03820_amd import serve
    rows, f = 2 ** 24 + 5, 1100
    x = torch.arange(-3, 0, device=D).float()[:, None].repeat(1, f)
    users = pattern(rows, 4, torch.int32)                    # row 3 does not exist
    scale = torch.full((rows,), -7.0, device=D)
    q = torch.full((rows, f), 99, dtype=torch.int8, device=D)
    log(f"quantize {rows} x {f} by index")
    serve.als_quantize(ctx, x, users=users, q=q, scale=scale)
    want = torch.tensor([3, 2, 1, float("nan")], device=D) * (torch.ones((), device=D) / 127)
    assert torch.equal(scale.nan_to_num(nan=-1), want.nan_to_num(nan=-1).repeat((rows + 3) // 4)[:rows])
    rowwise = torch.where(users == 3, 0, -127).to(torch.int8)
    for first in range(0, rows, 2 ** 22):
        some = slice(first, min(rows, first + 2 ** 22))
        assert bool((q[some] == rowwise[some, None]).all())


@pytest.mark.parametrize("m,n", [(1, 2 ** 31 + 70), (65_600, 262_300), (2 ** 20 + 3, 16_500)])
def test_score_of_many_rows(ctx, m, n):
    """More items than a launch takes; more of both; more users."""
    from paper_1603_03820_amd import serve

    def rows(k, period):       # of stride 16, as als_quantize leaves them
        q = torch.zeros(k, 16, dtype=torch.int8, device=D)
        q[:, 0] = pattern(k, period, torch.int8) - 1
        return q[:, :1], torch.ones(k, device=D)
    xq, xs = rows(m, 5)
    tq, ts = rows(n, 3)
    out = torch.full((m, n), 99.0, dtype=torch.float16, device=D)
    log(f"score {m} x {n} x 1")
    serve.als_score(ctx, xq, xs, tq, ts, out=out)
    step = max(1, 2 ** 29 // n)
    for i in range(0, m, step):
        for j in range(0, n, 2 ** 28):
            part = out[i:i + step, j:j + 2 ** 28]
            assert torch.equal(part, xq[i:i + step].half() * tq[j:j + 2 ** 28, 0].half())
    del out, xq, tq, xs, ts
    torch.cuda.empty_cache()
