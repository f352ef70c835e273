"""The prediction binding without a GPU: what it hands to the library for tensors of every layout, and what it refuses.
The library is a stand-in that keeps the arguments; tensors are the host's."""
import ctypes

import pytest
import torch

from paper_1603_03820_amd import predict
from paper_1603_03820_amd.als import ALSError
from tests.test_serve_binding import Stream, Workspace


class Library:
    """Accepts every call and keeps its arguments, structures as dicts."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            kept = [{k: getattr(a._obj, k) for k, _ in a._obj._fields_} if hasattr(a, "_obj") else a for a in args]
            self.calls.append((name, kept))
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    from paper_1603_03820_amd import serve
    stand_in = Library()
    monkeypatch.setattr(predict, "_lib", stand_in)
    stand_in.current = Stream(0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: stand_in.current.cuda_stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stand_in.current)
    monkeypatch.setattr(serve, "_capturing", lambda stream: stream.capturing)
    return stand_in


class HostContext(predict.Context):
    """A context whose device is the host (whose tensors are on device -1), created on stream 0."""

    def __init__(self):
        self.handle, self.index, self.device = 1, -1, torch.device("cpu")
        self.workspace = Workspace()
        self._start(Stream(0))

    def close(self):
        pass


def test_predict_passes_its_layouts(lib):
    wide = torch.zeros(9, 40)
    x, t = wide[:, 3:23], torch.zeros(7, 20)
    users = torch.zeros(5, dtype=torch.int32)
    a, b, res = torch.zeros(9), torch.zeros(7), torch.zeros(5, 12)[:, :7]
    out = predict.als_predict(HostContext(), x, t, users, a, b, "clip", 1, 5, res)
    name, args = lib.calls[-1]
    assert name == "als_predict" and out.shape == (5, 7) and out.dtype == torch.float32
    assert args == [1, x.data_ptr(), 9, 40, users.data_ptr(), 5, t.data_ptr(), 7, 20, 0, 20, a.data_ptr(), b.data_ptr(), 1, 1, 5,
                    res.data_ptr(), 12, out.data_ptr(), 7, 0, 0]
    half = predict.als_predict(HostContext(), x.bfloat16(), t.bfloat16(), activation="clip", high=2.0, dtype=torch.float16)
    args = lib.calls[-1][1]
    assert half.dtype == torch.float16 and args[9] == 2 and args[20] == 1 and args[13:16] == [1, float("-inf"), 2.0]
    assert args[4] is None and args[11] is None and args[16] is None


def test_log_prob_passes_its_layouts(lib):
    z = torch.zeros(4, 30, dtype=torch.bfloat16)[:, :25]
    given = torch.zeros(4, 3, dtype=torch.int32)
    ptr, col, users = torch.zeros(7, dtype=torch.int64), torch.zeros(9, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    r = predict.als_log_prob(HostContext(), z, given, 0.5, 6, (ptr, col), users)
    name, (_, s, g, *rest) = lib.calls[-1]
    assert name == "als_log_prob"
    assert s == dict(z=z.data_ptr(), dtype=2, rows=4, n=25, ldz=30, temperature=None, temperature_all=0.5, rated_ptr=ptr.data_ptr(),
                     rated_idx=col.data_ptr(), users=users.data_ptr(), of=6)
    assert g == dict(ptr=None, idx=given.data_ptr(), entries=12, each=3)
    assert rest == [r.log.data_ptr(), r.stats.data_ptr(), r.entropy.data_ptr(), 6, r.top_index.data_ptr(), r.top_log.data_ptr(), 0]
    assert r.log.shape == (4, 3) and r.stats.shape == (4, 2) and r.top_index.shape == (4, 6)
    t, gp, gi = torch.ones(4), torch.zeros(5, dtype=torch.int64), torch.zeros(11, dtype=torch.int32)
    r = predict.als_log_prob(HostContext(), z, (gp, gi), t)
    _, (_, s, g, *rest) = lib.calls[-1]
    assert s["temperature"] == t.data_ptr() and s["rated_ptr"] is None and s["users"] is None and s["of"] == 0
    assert g == dict(ptr=gp.data_ptr(), idx=gi.data_ptr(), entries=11, each=0) and r.log.shape == (11,)
    assert r.top_index is None and rest[3:6] == [0, None, None]
    # the gradient, whose context had another call's arguments in its structures
    d, c = predict.als_log_prob_grad(HostContext(), z, (gp, gi), r, torch.ones(11), temperature=2.0)
    _, (_, s, g, *rest) = lib.calls[-1]
    assert s["temperature"] is None and s["temperature_all"] == 2.0 and c is None and d.shape == (4, 25) and d.dtype == z.dtype
    assert rest[2] is None and rest[4] is None and rest[5:8] == [d.data_ptr(), 25, None]


def test_a_contexts_calls_leave_nothing_behind(lib):
    """Arguments of one call do not show up in the next one's."""
    ctx = HostContext()
    z, given = torch.zeros(2, 9), torch.zeros(2, dtype=torch.int32)
    rated = (torch.zeros(3, dtype=torch.int64), torch.zeros(1, dtype=torch.int32))
    predict.als_log_prob(ctx, z, (torch.zeros(3, dtype=torch.int64), given), torch.ones(2), 4, rated, given)
    predict.als_log_prob(ctx, z, given)
    _, (_, s, g, *rest) = lib.calls[-1]
    assert s["temperature"] is None and s["rated_ptr"] is None and s["rated_idx"] is None and s["users"] is None and s["of"] == 0
    assert g["ptr"] is None and g["each"] == 1 and rest[3] == 0


@pytest.mark.parametrize("f", [2 ** 31, 2 ** 32 + 5])
def test_rows_past_32_bits_are_not_cut(lib, f):
    x = torch.empty(1, f, dtype=torch.float16)       # (never touched)
    predict.als_predict(HostContext(), x, x)
    assert ctypes.c_int32(lib.calls[-1][1][10]).value > predict.ALS_PREDICT_F_MAX


@pytest.mark.parametrize("first,fits", [(8, True), (9, False), (20, False), (29, False), (30, True)])
def test_results_on_the_rated_columns_are_refused(lib, first, fits):
    """`log`, `grad` or `columns` on the CSR's columns, whose number the library does not know."""
    memory = torch.zeros(64, dtype=torch.int32)
    rated = (torch.zeros(3, dtype=torch.int64), memory[10:30])
    result = memory[first:first + 2].view(torch.float32)
    z, given = torch.zeros(2, 1), torch.zeros(2, dtype=torch.int32)
    r = predict.LogProb(torch.zeros(2), torch.zeros(2, 2), torch.zeros(2), None, None)
    calls = (lambda: predict.als_log_prob(HostContext(), z, given, rated=rated, log=result),
             lambda: predict.als_log_prob_grad(HostContext(), z, given, r, r.log, rated=rated, grad=result.view(2, 1)),
             lambda: predict.als_log_prob_grad(HostContext(), torch.zeros(2, 2), given, r, r.log, rated=rated, grad=False, columns=result))
    for call in calls:
        if fits:
            call()
        else:
            with pytest.raises(ALSError) as e:
                call()
            assert e.value.code == -6


def test_calls_follow_one_another_and_keep_the_workspace(lib):
    """Each call works in the workspace, so on another stream it waits for the last one, which keeps its memory."""
    ctx = HostContext()
    z, given = torch.zeros(2, 9), torch.zeros(2, dtype=torch.int32)
    a, b = Stream(5), Stream(6)
    lib.current = a
    predict.als_predict(ctx, z, z)
    assert a.waits == [0] and ctx.workspace.recorded == [5]
    lib.current = b
    r = predict.als_log_prob(ctx, z, given)
    assert b.waits == [5] and ctx.workspace.recorded == [5, 6]
    predict.als_log_prob_grad(ctx, z, given, r, r.log, columns=True)
    lib.current = a
    predict.als_log_prob_grad(ctx, z, given, r, r.log)       # (without columns' sums it does without)
    assert a.waits == [0]
    predict.als_log_prob(ctx, z, given)
    assert a.waits == [0, 6]


@pytest.mark.parametrize("call,error", [
    (lambda c, z, g: predict.als_predict(c, z, z.half()), TypeError),
    (lambda c, z, g: predict.als_predict(c, z, z[:, :8]), ValueError),
    (lambda c, z, g: predict.als_predict(c, z, z, activation="swish"), ValueError),
    (lambda c, z, g: predict.als_predict(c, z, z, high=3.0), ValueError),
    (lambda c, z, g: predict.als_predict(c, z, z, residual=torch.zeros(2, 2, dtype=torch.float16)), (TypeError, ValueError)),
    (lambda c, z, g: predict.als_log_prob(c, z, g[:1]), ValueError),
    (lambda c, z, g: predict.als_log_prob(c, z, g.long()), TypeError),
    (lambda c, z, g: predict.als_log_prob(c, z, g, users=g), ValueError),
    (lambda c, z, g: predict.als_log_prob(c, z, g, top=129), ValueError),
    (lambda c, z, g: predict.als_log_prob(c, z, (torch.zeros(2, dtype=torch.int64), g)), ValueError),
])
def test_refusals(lib, monkeypatch, call, error):
    from paper_1603_03820_amd import serve

    def use(ctx, t, name, dtypes):      # (the host's tensors stand for the device's)
        if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
            raise TypeError(name)
    monkeypatch.setattr(serve, "_use", use)
    monkeypatch.setattr(predict, "_use", use)
    with pytest.raises(error):
        call(HostContext(), torch.zeros(2, 9), torch.zeros(2, dtype=torch.int32))
    assert not lib.calls


@pytest.mark.parametrize("call,name", [
    (lambda c, z, g: predict.als_predict(c, z, z, users=[0, 1]), "users"),
    (lambda c, z, g: predict.als_predict(c, z, z, out=[0.0]), "out"),
    (lambda c, z, g: predict.als_predict(c, [[0.0]], z), "x"),
    (lambda c, z, g: predict.als_predict(c, z, z, residual=[0.0]), "residual"),
    (lambda c, z, g: predict.als_predict(c, z, z, item_offset=[0.0] * 2), "item_offset"),
    (lambda c, z, g: predict.als_log_prob(c, z, [0, 0]), "given"),
    (lambda c, z, g: predict.als_log_prob(c, z, ([0, 1, 2], g)), "given[0]"),
    (lambda c, z, g: predict.als_log_prob(c, z, (torch.zeros(3, dtype=torch.int64), [0, 0])), "given[1]"),
    (lambda c, z, g: predict.als_log_prob(c, z, g, rated=([0, 0, 0], g)), "rated[0]"),
    (lambda c, z, g: predict.als_log_prob(c, z, g, rated=(torch.zeros(3, dtype=torch.int64), [0])), "rated[1]"),
    (lambda c, z, g: predict.als_log_prob(c, z, g, rated=(torch.zeros(3, dtype=torch.int64), g), users=[0, 1]), "users"),
    (lambda c, z, g: predict.als_log_prob(c, z, g, log=[0.0, 0.0]), "log"),
])
def test_lists_in_place_of_tensors_are_refused_by_name(lib, call, name):
    with pytest.raises(TypeError, match=name.replace("[", r"\[").replace("]", r"\]") + " must be a device tensor"):
        call(HostContext(), torch.zeros(2, 9), torch.zeros(2, dtype=torch.int32))
    assert not lib.calls
