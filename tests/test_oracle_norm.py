"""Pins of the norm's oracle: unit mean square, invariance, and the gradient against automatic and finite differences."""
import numpy as np
import torch

from oracle import norm


def test_rows_have_unit_mean_square_and_do_not_depend_on_their_scale():
    rng = np.random.default_rng(0)
    h, w = rng.standard_normal((5, 37)), np.ones(37)
    rstd, y = norm.forward(h, w, 0.0)
    assert np.allclose((y ** 2).mean(1), 1.0, atol=1e-14)
    assert np.allclose(norm.forward(1000 * h, w, 0.0)[1], y, atol=1e-13)
    assert np.allclose(norm.forward(np.zeros((1, 4)), np.ones(4), 1e-5)[0], 1e-5 ** -0.5)


def test_gradient_is_that_of_the_formula_and_of_differences():
    rng = np.random.default_rng(1)
    h, w, dy, dres = rng.standard_normal((4, 29)), rng.standard_normal(29), rng.standard_normal((4, 29)), rng.standard_normal((4, 29))
    rstd, y = norm.forward(h, w, 1e-3)
    dx, dw = norm.backward(dy, h, w, rstd, dres)
    th, tw = torch.tensor(h, requires_grad=True), torch.tensor(w, requires_grad=True)
    ty = th * (th.square().mean(1, keepdim=True) + 1e-3).rsqrt() * tw
    ((ty * torch.tensor(dy)).sum() + (th * torch.tensor(dres)).sum()).backward()
    assert np.allclose(th.grad.numpy(), dx, atol=1e-12) and np.allclose(tw.grad.numpy(), dw, atol=1e-12)
    loss = lambda a, b: np.sum(dy * norm.forward(a, b, 1e-3)[1]) + np.sum(dres * a)  # noqa: E731
    for i, j in ((0, 0), (3, 28)):
        e = np.zeros_like(h)
        e[i, j] = 1e-6
        assert abs((loss(h + e, w) - loss(h - e, w)) / 2e-6 - dx[i, j]) < 1e-7
        assert abs((loss(h, w + e[i]) - loss(h, w - e[i])) / 2e-6 - dw[j]) < 1e-7
