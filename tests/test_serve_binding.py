"""The serving binding without a GPU: what it hands to the library for tensors of every layout.  The library is a
stand-in that keeps the arguments; tensors are the host's."""
import types

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
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0)
    return stand_in


def context():
    """A context whose device is the host (whose tensors are on device -1)."""
    return types.SimpleNamespace(handle=1, index=-1, device=torch.device("cpu"), _limits=serve._Limits(),
                                 _limits_ref=None)


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
