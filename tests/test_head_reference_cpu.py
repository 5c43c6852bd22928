"""The formulas that the GPU tests compare with, against differences of the functions that they are the gradients of."""
import math

import pytest
import torch

import head_reference as R


def directional(f, x, u, step):
    return (f(x + step * u) - f(x - step * u)) / (2 * step)


@pytest.mark.parametrize("layer", [True, False])
def test_norm_gradient_is_the_slope(layer):
    g = torch.Generator().manual_seed(1)
    h, dy, u = (torch.randn((5, 37), generator=g, dtype=torch.float64) for _ in range(3))
    h += 0.7
    w, b, uw = (torch.randn(37, generator=g, dtype=torch.float64) for _ in range(3))
    dx, dw, db = R.norm_grad(dy, h, w, layer=layer)
    # central differences of 1e-5: error of the order of 1e-10, rounding 1e-16 / 1e-5
    value = lambda h_, w_, b_: float((R.norm_of(h_, w_, b_, 1e-5, layer)[0] * dy).sum())
    assert directional(lambda t: value(t, w, b), h, u, 1e-5) == pytest.approx(float((dx * u).sum()), abs=1e-7)
    assert directional(lambda t: value(h, t, b), w, uw, 1e-5) == pytest.approx(float((dw * uw).sum()), abs=1e-7)
    assert directional(lambda t: value(h, w, t), b, uw, 1e-5) == pytest.approx(float((db * uw).sum()), abs=1e-7)


def test_token_gradient_is_the_slope():
    g = torch.Generator().manual_seed(2)
    x, u = (torch.randn((4, 23), generator=g, dtype=torch.float64) for _ in range(2))
    x[1, 5] = -math.inf
    u[1, 5] = 0.0
    targets = torch.tensor([3, -1, 22, 0])
    gl, gh = (torch.randn(4, generator=g, dtype=torch.float64) for _ in range(2))

    def value(t):
        lp, _ = R.log_softmax(t, 1.7)
        given = targets >= 0
        picked = torch.where(given, lp[torch.arange(4), targets.clamp(min=0)], torch.zeros(4, dtype=torch.float64))
        return float((gl * picked).sum() + (gh * R.entropy(lp)).sum())
    want = float((R.token_grad(x, targets, gl, gh, 1.7) * u).sum())
    assert directional(value, x, u, 1e-5) == pytest.approx(want, abs=1e-7)


@pytest.mark.parametrize("rest", [True, False])
def test_distillation_gradient_is_the_slope(rest):
    g = torch.Generator().manual_seed(3)
    x, u = (torch.randn((4, 23), generator=g, dtype=torch.float64) for _ in range(2))
    index = torch.stack([torch.randperm(23, generator=g)[:6] for _ in range(4)])
    value = torch.log_softmax(torch.randn((4, 9), generator=g, dtype=torch.float64), -1)[:, :6]
    index[1, 2], index[2, 4], index[3, 5] = -1, index[2, 1], 23     # padding, the same token again, no token
    loss = lambda t: float(R.distill(t, index, value, rest, 0.6)[0].sum())
    want = float((R.distill(x, index, value, rest, 0.6)[1] * u).sum())
    assert directional(loss, x, u, 1e-5) == pytest.approx(want, abs=1e-7)


def test_distillation_from_everything_is_the_divergence():
    """All tokens listed: the divergence of two distributions, zero for equal ones."""
    g = torch.Generator().manual_seed(4)
    x, t = (torch.randn((3, 8), generator=g, dtype=torch.float64) for _ in range(2))
    index = torch.arange(8).expand(3, 8)
    lq, lp = torch.log_softmax(t, -1), torch.log_softmax(x, -1)
    for rest in (True, False):
        loss, grad = R.distill(x, index, lq, rest, 1.0)
        torch.testing.assert_close(loss, (lq.exp() * (lq - lp)).sum(-1))
        torch.testing.assert_close(grad, lp.exp() - lq.exp(), atol=1e-12, rtol=0)
        assert float(R.distill(t, index, lq, rest, 1.0)[0].abs().max()) < 1e-12
