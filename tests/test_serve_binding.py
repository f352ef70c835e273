"""The serving binding without a GPU: what it hands to the library for tensors of every layout.  The library is a
stand-in that keeps the arguments; tensors are the host's."""
import ctypes

import pytest
import torch

from paper_1603_03820_amd import serve


class Library:
    """Accepts every call and keeps its arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    stand_in = Library()
    monkeypatch.setattr(serve, "_lib", stand_in)
    stand_in.current = Stream(0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: stand_in.current.cuda_stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stand_in.current)
    monkeypatch.setattr(serve, "_capturing", lambda stream: stream.capturing, raising=False)
    return stand_in


class Stream:
    """Keeps the streams that it was told to wait for."""

    def __init__(self, handle, capturing=False):
        self.cuda_stream, self.capturing, self.waits = handle, capturing, []

    def wait_stream(self, stream):
        self.waits.append(stream.cuda_stream)


class Workspace:
    """Keeps the streams that it is recorded on."""

    def __init__(self):
        self.recorded = []

    def record_stream(self, stream):
        self.recorded.append(stream.cuda_stream)


class HostContext(serve.Context):
    """A context whose device is the host (whose tensors are on device -1), created on stream 0."""

    def __init__(self):
        self.handle, self.index, self.device = 1, -1, torch.device("cpu")
        self.workspace = Workspace()
        self._start(Stream(0))

    def close(self):
        pass


def context():
    return HostContext()


def quantize_writes(call):
    """(first byte, bytes) of every row that a call of als_quantize or als_quantize_into writes, as the header says."""
    name, args = call
    rows, f, q, ldq = args[6:10]
    if name == "als_quantize_into":
        width = args[10]
        assert f <= width <= min(ldq, (f + 15) // 16 * 16)
    else:
        assert name == "als_quantize"
        width = min(ldq, (f + 15) // 16 * 16)
    return [(q + r * ldq, width) for r in range(rows)]


@pytest.mark.parametrize("columns,first,f", [(200, 0, 100), (200, 100, 100), (32, 11, 21), (64, 16, 21), (42, 0, 21),
                                             (42, 21, 21), (21, 0, 21), (300, 1, 16), (130, 2, 128), (23, 1, 21)])
def test_quantize_writes_no_neighbour(lib, columns, first, f):
    """Columns of a wider buffer: those beside them, and what lies behind the buffer, are not written."""
    rows = 6
    buffer = torch.zeros(rows, columns, dtype=torch.int8)
    q = buffer[:, first:first + f]
    serve.als_quantize(context(), torch.zeros(rows, f), q=q, scale=torch.zeros(rows))
    start = buffer.data_ptr()
    for r, (at, width) in enumerate(quantize_writes(lib.calls[-1])):
        assert start + r * columns + first <= at and at + width <= start + r * columns + first + f


@pytest.mark.parametrize("stride", [22, 30, 32, 40])
def test_quantize_writes_nothing_past_the_storage(lib, stride):
    """Rows whose last one ends with its storage."""
    rows, f = 5, 21
    flat = torch.zeros((rows - 1) * stride + f, dtype=torch.int8)
    q = torch.as_strided(flat, (rows, f), (stride, 1))
    serve.als_quantize(context(), torch.zeros(rows, f), q=q, scale=torch.zeros(rows))
    for at, width in quantize_writes(lib.calls[-1]):
        assert flat.data_ptr() <= at and at + width <= flat.data_ptr() + flat.numel()


def test_quantize_pads_its_own_rows(lib):
    """Rows that the call allocates are zero up to their stride, which is a multiple of 16."""
    q, _ = serve.als_quantize(context(), torch.zeros(4, 21))
    assert q.stride() == (32, 1)
    assert quantize_writes(lib.calls[-1]) == [(q.data_ptr() + 32 * r, 32) for r in range(4)]


def sample(ctx, n):
    return serve.als_sample(ctx, torch.zeros(2, n), torch.zeros(2))


def score(ctx, extra=0):
    q = torch.zeros(2, 32 + extra, dtype=torch.int8)[:, :32]
    return serve.als_score(ctx, q, torch.zeros(2), q, torch.zeros(2))


def test_the_bounds_are_the_librarys(lib):
    """Up to which calls do without the workspace."""
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    header = open(os.path.join(root, "include", "als_serve.h")).read()
    assert int(re.search(r"#define ALS_SERVE_HELD_MAX (\d+)", header).group(1)) == serve.ALS_SERVE_HELD_MAX
    source = open(os.path.join(root, "paper_1603_03820_amd", "csrc", "serve.hip")).read()
    assert "constexpr int64_t kTileStride = 1 << 22;" in source
    assert "return aligned(q, 16) && ld % 16 == 0 && ld < kTileStride;" in source
    memory = torch.empty((1 << 23) + 64, dtype=torch.int8)
    near = torch.zeros(2, 32, dtype=torch.int8)
    assert memory.data_ptr() % 16 == 0 and near.data_ptr() % 16 == 0
    for start, ld, there in ((0, 32, True), (1, 32, False), (0, 33, False), (16, (1 << 22) - 16, True), (0, 1 << 22, False)):
        rows = torch.as_strided(memory, (2, 32), (ld, 1), start)
        for xq, tq in ((rows, near), (near, rows)):
            ctx = context()
            lib.current = Stream(5)
            serve.als_score(ctx, xq, torch.zeros(2), tq, torch.zeros(2))
            assert (ctx.workspace.recorded == []) == there


def test_the_workspace_is_recorded_where_it_is_used(lib):
    """Its memory must not be handed out again while a call on another stream than its own still works in it."""
    ctx = context()
    sample(ctx, 70_000)
    score(ctx, 1)
    assert ctx.workspace.recorded == []
    lib.current = Stream(5)
    sample(ctx, 65_536)          # these do without it
    score(ctx)
    assert ctx.workspace.recorded == []
    sample(ctx, 65_537)
    assert ctx.workspace.recorded == [5]
    lib.current = Stream(6)
    score(ctx, 1)
    assert ctx.workspace.recorded == [5, 6]
    sample(ctx, 70_000)
    lib.current = Stream(0)
    score(ctx, 1)
    assert ctx.workspace.recorded == [5, 6]      # once is enough


def test_calls_in_the_workspace_follow_one_another(lib):
    """On whatever streams they are; a captured call waits for nobody, and nobody for it."""
    ctx = context()
    a, b, captured = Stream(5), Stream(6), Stream(7, capturing=True)
    lib.current = a
    score(ctx, 1)
    assert a.waits == [0]          # the memory's own stream, which may have used it before
    sample(ctx, 70_000)
    assert a.waits == [0]
    lib.current = b
    sample(ctx, 100)
    score(ctx)
    assert b.waits == []           # without the workspace
    sample(ctx, 70_000)
    assert b.waits == [5]
    lib.current = captured
    sample(ctx, 70_000)
    assert captured.waits == [] and ctx.workspace.recorded == [5, 6, 7]
    lib.current = b
    sample(ctx, 70_000)
    assert b.waits == [5]
    lib.current = a
    sample(ctx, 70_000)
    assert a.waits == [0, 6]


@pytest.mark.parametrize("f", [2 ** 31, 2 ** 32 + 5])
def test_rows_past_32_bits_are_not_cut(lib, f):
    """A row length goes to the library as a 32-bit number; one that does not fit must not arrive as another that
    does (the library refuses all past ALS_SERVE_F_MAX)."""
    ctx = context()
    rows = torch.empty(1, f, dtype=torch.int8)       # (never touched)

    def length(call):
        name, args = call
        return ctypes.c_int32(args[{"als_quantize_into": 7, "als_score": 9}[name]]).value
    serve.als_score(ctx, rows, torch.zeros(1), rows, torch.zeros(1))
    assert length(lib.calls[-1]) > serve.ALS_SERVE_F_MAX
    x = torch.empty(1, f, dtype=torch.float16)
    serve.als_quantize(ctx, x, q=rows)
    assert length(lib.calls[-1]) > serve.ALS_SERVE_F_MAX


@pytest.mark.parametrize("first,fits", [(8, True), (9, False), (20, False), (29, False), (30, True)])
def test_results_on_the_rated_columns_are_refused(lib, first, fits):
    """`index` or `log` on the CSR's columns, whose number the library does not know."""
    from paper_1603_03820_amd.als import ALSError
    memory = torch.zeros(64, dtype=torch.int32)
    rated = (torch.zeros(3, dtype=torch.int64), memory[10:30])
    for kind in ("index", "log"):
        result = memory[first:first + 2]
        given = {kind: result if kind == "index" else result.view(torch.float32)}
        if fits:
            serve.als_sample(context(), torch.zeros(2, 9), torch.zeros(2), rated=rated, **given)
        else:
            with pytest.raises(ALSError) as e:
                serve.als_sample(context(), torch.zeros(2, 9), torch.zeros(2), rated=rated, **given)
            assert e.value.code == -6
