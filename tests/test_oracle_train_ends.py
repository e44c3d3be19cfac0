"""Pins for the oracle's ends of a training step: the language-model loss, the norm's gain gradient, clipping.
Gradients against central differences and torch's automatic ones in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import hero_oracle as O
from tests.test_oracle_backward import _close, _fd

RNG = np.random.default_rng


@pytest.mark.parametrize("mean", [True, False])
def test_lm_loss_gradients_are_the_differences_of_the_loss(mean):
    rng = RNG(0)
    x, w = rng.standard_normal((5, 6)), rng.standard_normal((9, 6))
    y = np.array([3, -1, 0, 8, 9])          # two tokens without a target among the rows of w
    r = O.lm_loss(x, w, y, 0.7, mean)
    _close(r.dx, _fd(lambda: O.lm_loss(x, w, y, 0.7, mean).loss, x))
    _close(r.dw, _fd(lambda: O.lm_loss(x, w, y, 0.7, mean).loss, w))
    assert np.all(r.dx[[1, 4]] == 0) and np.all(r.token_loss[[1, 4]] == 0)


@pytest.mark.parametrize("size", [1.0, 30.0, 300.0])
def test_lm_loss_equals_torch(size):
    rng = RNG(1)
    x = torch.tensor(rng.standard_normal((11, 8)) * size, requires_grad=True)
    w = torch.tensor(rng.standard_normal((17, 8)), requires_grad=True)
    y = rng.integers(-1, 17, 11)
    loss = torch.nn.functional.cross_entropy(x @ w.T, torch.tensor(np.where(y < 0, -100, y)))
    loss.backward()
    r = O.lm_loss(x.detach().numpy(), w.detach().numpy(), y)
    assert abs(r.loss - loss.item()) <= 1e-12 * max(1.0, loss.item())
    _close(r.dx, x.grad.numpy(), 1e-10)
    _close(r.dw, w.grad.numpy(), 1e-10)


def test_lm_loss_of_a_sure_token_keeps_its_digits():
    # logits 40 and 0: the loss is log(1 + e^-40), far below a step of 1
    r = O.lm_loss(np.array([[1.0]]), np.array([[40.0], [0.0]]), np.array([0]))
    assert abs(r.loss / np.exp(-40.0) - 1) < 1e-12
    assert abs(r.dx[0, 0] / (-40.0 * np.exp(-40.0)) - 1) < 1e-12


def test_lm_loss_without_counted_tokens_is_zero():
    r = O.lm_loss(np.ones((3, 2)), np.ones((4, 2)), np.array([-1, 4, 99]))
    assert r.loss == 0 and not r.dx.any() and not r.dw.any()


def test_rmsnorm_gain_gradient():
    rng = RNG(2)
    h, g, du = rng.standard_normal((6, 5)), rng.standard_normal(5), rng.standard_normal((6, 5))
    f = lambda: float(np.sum(du * O.rmsnorm(h, g, 1e-5)))  # noqa: E731
    _close(O.rmsnorm_gain_grad(h, 1e-5, du), _fd(f, g))
    _close(O.rmsnorm_backward(h, g, 1e-5, du), _fd(f, h))


def test_grad_clip():
    g = [np.array([3.0, 0.0]), np.array([[4.0]])]
    norm, out = O.grad_clip(g, 1.0)
    assert norm == 5.0 and np.allclose(out[0], [0.6, 0]) and np.allclose(out[1], 0.8)
    norm, out = O.grad_clip(g, 5.0)
    assert np.array_equal(out[0], g[0]) and np.array_equal(out[1], g[1])
