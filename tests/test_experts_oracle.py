"""Pins of the oracle for layers of experts and clipped gradients: against torch's sorting, autograd, the oracle of one layer, and values
worked by hand."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as eo
from oracle import kfac_oracle as ko


def test_sort_by_hand():
    # experts of three tokens, two choices each; 5 and -1 are none of the three experts
    offsets, order, place = eo.expert_sort(np.array([[2, 0], [5, 2], [0, -1]]), 3)
    assert offsets.tolist() == [0, 2, 2, 4]
    assert order.tolist() == [1, 4, 0, 3, -1, -1]
    assert place.tolist() == [[2, 0], [-1, 3], [1, -1]]


def test_sort_is_a_stable_sort():
    rng = np.random.default_rng(3)
    expert = rng.integers(0, 7, (50, 3))
    offsets, order, place = eo.expert_sort(expert, 7)
    want = torch.argsort(torch.from_numpy(expert.reshape(-1)), stable=True).numpy()
    np.testing.assert_array_equal(order, want)
    np.testing.assert_array_equal(place.reshape(-1)[order], np.arange(150))
    np.testing.assert_array_equal(np.diff(offsets), np.bincount(expert.reshape(-1), minlength=7))


def test_there_and_back_and_gradients_against_autograd():
    rng = np.random.default_rng(4)
    T, K, E, D = 6, 3, 4, 5
    expert = rng.integers(-1, E, (T, K))
    _, order, place = eo.expert_sort(expert, E)
    x = torch.tensor(rng.standard_normal((T, D)), requires_grad=True)
    w = torch.tensor(rng.standard_normal((T, K)), requires_grad=True)
    gate = torch.tensor(rng.standard_normal((T * K, D)))
    there = torch.tensor(place >= 0)
    at = torch.tensor(np.maximum(place, 0))
    # the experts multiply by `gate`, row by row
    pick = torch.zeros(T * K, T, dtype=torch.float64)
    for t in range(T):
        for k in range(K):
            if place[t, k] >= 0:
                pick[place[t, k], t] = 1
    xs = pick @ x
    ys = xs * gate
    ys.retain_grad()
    y = (torch.where(there, w, 0)[:, :, None] * ys[at]).sum(1)
    np.testing.assert_allclose(eo.expert_dispatch(x.detach().numpy(), place, np.zeros((T * K, D))), xs.detach().numpy())
    np.testing.assert_allclose(eo.expert_combine(ys.detach().numpy(), w.detach().numpy(), place, D), y.detach().numpy(), atol=1e-14)
    dy = rng.standard_normal((T, D))
    y.backward(torch.tensor(dy))
    dys, dw = eo.expert_combine_backward(dy, ys.detach().numpy(), w.detach().numpy(), place, np.zeros((T * K, D)))
    np.testing.assert_allclose(dys, ys.grad.numpy(), atol=1e-14)
    np.testing.assert_allclose(dw, w.grad.numpy(), atol=1e-14)
    # the gradient of dispatch is a sum without weights
    np.testing.assert_allclose(eo.expert_combine(dys * gate.numpy(), None, place, D), x.grad.numpy(), atol=1e-14)


def test_rows_that_nothing_goes_to_stay():
    place = np.array([[1, -1], [-1, 7]])
    xs = eo.expert_dispatch(np.ones((2, 3)), place, np.full((4, 3), 9.0))
    np.testing.assert_array_equal(xs, [[9] * 3, [1] * 3, [9] * 3, [9] * 3])


def test_factor_of_one_expert_is_a_layers_factor():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((12, 4))
    offsets = np.array([0, 5, 5, 12])
    F = eo.expert_factor(x, offsets, has_bias=True)
    for e, rows in ((0, x[:5]), (2, x[5:])):
        want = ko.factor_A(rows[:, :, None, None], 1, 1, 1, 0, True, ko.ORDER_KH_KW_C)
        np.testing.assert_allclose(F[e], want, atol=1e-14)
    assert not F[1].any()
    G = eo.expert_factor(x, offsets, scale=0.5)
    np.testing.assert_allclose(G[0], 0.5 * sum(np.outer(r, r) for r in x[:5]), atol=1e-14)
    S = rng.standard_normal((3, 5, 5))
    new = eo.expert_factor(x, offsets, has_bias=True, running=S, decay=0.75)
    np.testing.assert_allclose(new[2], 0.75 * S[2] + 0.25 * F[2], atol=1e-14)
    np.testing.assert_array_equal(new[1], S[1])


@pytest.mark.parametrize("max_norm,want", [(13.0, 1.0), (26.0, 1.0), (6.5, 0.5), (0.0, 0.0)])
def test_clipping_by_hand(max_norm, want):
    g = [np.array([3.0, 4.0]), np.zeros((0,)), np.array([[12.0]])]                # norm 13
    out, norm = eo.grad_clip(g, max_norm)
    assert norm == 13.0
    for a, b in zip(out, g):
        np.testing.assert_array_equal(a, want * b)
    assert eo.grad_clip(g, 6.5, norm=52.0)[0][0].tolist() == [3 / 8, 0.5]


def test_a_norm_that_is_not_finite_clips_nothing():
    for bad in (np.nan, np.inf):
        out, norm = eo.grad_clip([np.array([1.0, bad])], 0.5)
        assert not np.isfinite(norm) and out[0][0] == 1.0


def test_a_norm_beyond_the_largest_float_clips_nothing():
    top = float(np.finfo(np.float32).max)
    out, norm = eo.grad_clip([np.array([top, top])], 0.5)
    assert norm == np.inf and out[0].tolist() == [top, top]
    assert eo.grad_norm([np.array([top, top])]) == np.inf
    out, norm = eo.grad_clip([np.array([top, 1e30])], top / 2)                    # rounds to the largest float
    assert np.isfinite(norm) and out[0][0] == top / 2
