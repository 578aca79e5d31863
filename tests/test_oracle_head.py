"""Pins of the head's oracle on the CPU: closed forms, library autograd, finite differences."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as H


def _num_grad(f, a, at, h=1e-6):
    b = a.copy()
    b[at] = a[at] + h
    up = f(b)
    b[at] = a[at] - h
    return (up - f(b)) / (2 * h)


def test_recurrence_closed_forms():
    x = np.random.default_rng(0).standard_normal((2, 6, 3))
    keep_all, keep_none = np.full_like(x, np.inf), np.full_like(x, -np.inf)
    h0 = np.full((2, 3), 2.5)
    assert np.array_equal(H.recur_fwd(x, keep_all, h0), np.broadcast_to(h0[:, None], x.shape))
    assert np.array_equal(H.recur_fwd(x, keep_none, h0), x)
    # constant gate 0.5: h_T = 2^-T h0 + sum 2^-(T-t) x_t
    want = h0 / 64 + sum(x[:, t] / 2.0 ** (6 - t) for t in range(6))
    assert np.allclose(H.recur_fwd(x, np.zeros_like(x), h0)[:, -1], want, rtol=1e-14)


def test_recurrence_gradients_against_differences():
    rng = np.random.default_rng(1)
    x, g, dy = (rng.standard_normal((2, 5, 3)) for _ in range(3))
    h0, dl = rng.standard_normal((2, 3)), rng.standard_normal((2, 3))

    def loss(x, g, h0):
        h = H.recur_fwd(x, g, h0)
        return (h * dy).sum() + (h[:, -1] * dl).sum()
    dx, dg, dh0 = H.recur_bwd(x, g, h0, dy, dl)
    for at in np.ndindex(x.shape):
        assert abs(dx[at] - _num_grad(lambda v: loss(v, g, h0), x, at)) < 1e-8
        assert abs(dg[at] - _num_grad(lambda v: loss(x, v, h0), g, at)) < 1e-8
    for at in np.ndindex(h0.shape):
        assert abs(dh0[at] - _num_grad(lambda v: loss(x, g, v), h0, at)) < 1e-8


def test_layernorm_against_library():
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((7, 11)) * 2 + 1, rng.standard_normal((7, 11))
    gamma, beta = rng.standard_normal(11), rng.standard_normal(11)
    tx, tg, tb = (torch.tensor(v, requires_grad=True) for v in (x, gamma, beta))
    ty = torch.nn.functional.layer_norm(tx, (11,), tg, tb, 1e-5)
    ty.backward(torch.tensor(dy))
    assert np.allclose(H.layernorm_fwd(x, gamma, beta, 1e-5)[0], ty.detach().numpy(), atol=1e-12)
    for got, want in zip(H.layernorm_bwd(x, dy, gamma, 1e-5), (tx, tg, tb)):
        assert np.allclose(got, want.grad.numpy(), atol=1e-12)


@pytest.mark.parametrize("biased", [False, True])
def test_cross_entropy_against_library(biased):
    rng = np.random.default_rng(3)
    x, w = rng.standard_normal((6, 5)), rng.standard_normal((9, 5))
    b = rng.standard_normal(9) if biased else None
    labels, up = np.array([0, 8, 3, -1, 9, 4]), rng.standard_normal(6)
    tx, tw = torch.tensor(x, requires_grad=True), torch.tensor(w, requires_grad=True)
    tb = torch.tensor(b, requires_grad=True) if biased else None
    tl = torch.tensor(np.where(labels > 8, -1, labels))
    per_row = torch.nn.functional.cross_entropy(torch.nn.functional.linear(tx, tw, tb), tl, ignore_index=-1, reduction="none")
    (per_row * torch.tensor(up)).sum().backward()
    assert np.allclose(H.xent_fwd(x, w, b, labels)[0], per_row.detach().numpy(), atol=1e-12)
    dx, dw, db = H.xent_bwd(x, w, b, labels, up)
    assert np.allclose(dx, tx.grad.numpy(), atol=1e-12) and np.allclose(dw, tw.grad.numpy(), atol=1e-12)
    if biased:
        assert np.allclose(db, tb.grad.numpy(), atol=1e-12)


def test_cross_entropy_gradient_against_differences():
    rng = np.random.default_rng(4)
    x, w, b = rng.standard_normal((3, 4)), rng.standard_normal((5, 4)), rng.standard_normal(5)
    labels, up = np.array([1, 4, 7]), rng.standard_normal(3)
    dx, dw, db = H.xent_bwd(x, w, b, labels, up)

    def f(x, w, b):
        return (H.xent_fwd(x, w, b, labels)[0] * up).sum()
    for at in np.ndindex(x.shape):
        assert abs(dx[at] - _num_grad(lambda v: f(v, w, b), x, at)) < 1e-8
    for at in np.ndindex(w.shape):
        assert abs(dw[at] - _num_grad(lambda v: f(x, v, b), w, at)) < 1e-8
    for at in np.ndindex(b.shape):
        assert abs(db[at] - _num_grad(lambda v: f(x, w, v), b, at)) < 1e-8


def test_cross_entropy_with_classes_taken_out():
    x, w = np.ones((2, 2)), np.ones((3, 2))
    b = np.array([0.0, -np.inf, 0.0])
    loss, lse = H.xent_fwd(x, w, b, np.array([0, 1]))
    assert np.isclose(lse[0], 2 + np.log(2)) and np.isclose(loss[0], np.log(2)) and loss[1] == np.inf
    g = H.xent_grad(x, w, b, np.array([0, 1]), np.ones(2))
    assert np.allclose(g, [[-0.5, 0, 0.5], [0.5, -1, 0.5]])
