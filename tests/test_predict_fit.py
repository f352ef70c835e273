"""Fitting a Predictor's offsets without a GPU: the operators are their 64-bit forms (tests/predict_oracle.py), tensors are the
host's."""
import numpy as np
import pytest
import torch

from tests import predict_oracle


@pytest.fixture
def predict(monkeypatch):
    from paper_1603_03820_amd import predict

    def rows(z, temperature, rated, users):
        for i, row in enumerate(z.double().numpy()):
            u = i if users is None else int(users[i])
            there = rated is None or 0 <= u < rated[0].numel() - 1
            yield predict_oracle.Row(row, temperature, rated[1][rated[0][u]:rated[0][u + 1]].tolist() if rated and there else (), there)

    def product(ctx, x, theta, users=None, user_offset=None, item_offset=None):
        return torch.from_numpy(predict_oracle.predict(x, theta, users, user_offset, item_offset)[0]).float()

    def log_prob(ctx, z, given, temperature=1.0, rated=None, users=None):
        logs = [row.log(int(g)) for row, g in zip(rows(z, temperature, rated, users), given)]
        return predict.LogProb(torch.tensor(logs, dtype=torch.float32), None, None, None, None)

    def gradient(ctx, z, given, forward, grad_log, temperature=1.0, rated=None, users=None, grad=True, columns=False):
        assert not grad and columns
        sums = sum(row.gradient([int(g)], [float(w)], 0.0)[0] for row, g, w in zip(rows(z, temperature, rated, users), given, grad_log))
        return None, torch.from_numpy(sums).float()
    monkeypatch.setattr(predict, "als_predict", product)
    monkeypatch.setattr(predict, "als_log_prob", log_prob)
    monkeypatch.setattr(predict, "als_log_prob_grad", gradient)
    return predict


def problem(seed, users=30, n=12, count=80):
    """(x, theta, a CSR of rated items, users and items to fit to)"""
    rng = np.random.default_rng(seed)
    x, theta = (torch.from_numpy(rng.standard_normal((r, 4)).astype(np.float32)) for r in (users, n))
    lens = rng.integers(0, 4, users)
    ptr = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int64))
    idx = torch.from_numpy(np.concatenate([rng.permutation(n)[:k] for k in lens]).astype(np.int32))
    who, what = (torch.from_numpy(rng.integers(0, r, count).astype(np.int32)) for r in (users, n))
    return x, theta, (ptr, idx), who, what


@pytest.mark.parametrize("with_rated", [False, True])
@pytest.mark.parametrize("batch", [1024, 7])
def test_users_that_do_not_exist_count_for_nothing(predict, with_rated, batch):
    x, theta, rated, who, what = problem(1)
    rated = rated if with_rated else None
    bad = torch.tensor([-1, 30, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    at = torch.tensor([0, 5, 40, 79])
    mixed_who, mixed_what = who.clone(), what.clone()
    mixed_who[at] = bad
    kept = torch.ones(80, dtype=torch.bool)
    kept[at] = False
    a, b = (predict.Predictor(None, x, theta, rated=rated) for _ in range(2))
    means = a.fit_offsets(mixed_who, mixed_what, 0.7, 3, batch=batch)
    want = b.fit_offsets(who[kept], what[kept], 0.7, 3, batch=batch)
    # sums of other batches: some roundings of values of at most some tens; log p moves by at most 2 / T times the offsets
    assert torch.isfinite(a.item_offset).all() and torch.allclose(a.item_offset, b.item_offset, rtol=0, atol=1e-5)
    assert means == pytest.approx(want, abs=2e-5 / 0.7)
    nobody = predict.Predictor(None, x, theta, rated=rated)
    assert nobody.fit_offsets(bad, what[:4], 0.7, 2) == [0.0, 0.0] and not nobody.item_offset.any()


def test_a_csr_of_fewer_users_than_rows(predict):
    """A user behind the CSR's last row has no list, and counts for nothing either."""
    x, theta, (ptr, idx), who, what = problem(2)
    short = (ptr[:21].contiguous(), idx)
    a, b = (predict.Predictor(None, x, theta, rated=short) for _ in range(2))
    assert a.fit_offsets(who, what, 0.7, 2) == pytest.approx(b.fit_offsets(who[who < 20], what[who < 20], 0.7, 2), abs=2e-5 / 0.7)
    assert torch.isfinite(a.item_offset).all() and torch.allclose(a.item_offset, b.item_offset, rtol=0, atol=1e-5)


def test_lists_that_are_no_vectors_are_refused(predict):
    x, theta, rated, who, what = problem(3)
    model = predict.Predictor(None, x, theta)
    for w, g in ((who.view(2, 40), what.view(2, 40)), (who[:0], what[:0]), (who, what[:5])):
        with pytest.raises(ValueError):
            model.fit_offsets(w, g)
    assert model.item_offset is None


@pytest.mark.parametrize("temperature", [float("nan"), float("inf"), float("-inf"), 1e-42, 1e-37, 1e39])
def test_temperatures_without_a_gradient_are_refused(predict, temperature):
    """Those of no finite gradient: its product with T would be no number, and the offsets with it."""
    x, theta, rated, who, what = problem(4)
    for offset in (None, torch.ones(12)):
        model = predict.Predictor(None, x, theta, item_offset=offset, rated=rated)
        with pytest.raises(ValueError):
            model.fit_offsets(who, what, temperature, 2)
        assert model.item_offset is offset


def test_a_temperature_for_each_user_is_refused(predict):
    x, theta, rated, who, what = problem(5, n=1, count=30)
    with pytest.raises(TypeError):
        predict.Predictor(None, x, theta).fit_offsets(who, what, torch.ones(30), 2)


@pytest.mark.parametrize("temperature", [0.0, -1.0])
def test_a_greedy_fit_moves_nothing(predict, temperature):
    x, theta, rated, who, what = problem(6)
    model = predict.Predictor(None, x, theta)
    model.fit_offsets(who, what, temperature, 2)
    assert not model.item_offset.any()


def test_a_cold_fit_is_finite(predict):
    x, theta, rated, who, what = problem(7)
    model = predict.Predictor(None, x, theta, rated=rated)
    model.fit_offsets(who, what, 1e-30, 2)
    assert torch.isfinite(model.item_offset).all()


def test_lists_in_place_of_tensors_are_refused(predict):
    x, theta, rated, who, what = problem(8)
    model = predict.Predictor(None, x, theta)
    for w, g, name in (([0, 1], what, "users"), (who, [0, 1], "given")):
        with pytest.raises(TypeError, match=name + " must be a device tensor"):
            model.fit_offsets(w, g)
