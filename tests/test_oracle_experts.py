"""The plain definitions of the experts' operators against differences and hand-worked values."""
import math

import pytest
import torch

from oracle import experts as plain


def test_sort_by_hand():
    ids = torch.tensor([[2, 0], [0, 5], [2, 2], [-1, 1]])
    gates = torch.tensor([[1.0, 0.5], [0.0, 1.0], [1.0, -0.0], [1.0, float("nan")]])
    offsets, places = plain.sort(ids, gates, 3)
    assert offsets.tolist() == [0, 1, 2, 4]
    assert places.tolist() == [[2, 0], [-1, -1], [3, -1], [-1, 1]]


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_slopes_are_differences(act):
    v = torch.linspace(-6, 6, 241, dtype=torch.float64) + 0.013
    h = 1e-5
    diff = (plain.activation(v + h, act) - plain.activation(v - h, act)) / (2 * h)
    assert (plain.slope(v, act) - diff).abs().max() < 1e-8          # h^2 times a third derivative below 10, and 1e-16 / h


def test_gelu_is_the_form_with_tanh():
    v = torch.linspace(-5, 5, 101, dtype=torch.float64)
    want = 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    assert (plain.activation(v, "gelu") - want).abs().max() < 1e-14


def test_gradients_are_differences():
    """The whole way there and back: L = sum(dy * y) in 64 bits against central differences."""
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    T, k, E, d, F = 5, 2, 3, 4, 6
    ids = torch.randint(0, E, (T, k), generator=g)
    x, w1, b1, w2, gates, res, dy = r(T, d), r(E, F, d), r(E, F), r(E, d, F), r(T, k), r(T, d), r(T, d)
    gates[1] = 0
    offsets, places = plain.sort(ids, gates, E)
    bounds = offsets.tolist()
    group = torch.bucketize(torch.arange(bounds[-1]), offsets[1:].long(), right=True)

    def forward(x, w1, b1, w2, gates):
        xr = plain.rows(x, places, torch.zeros(bounds[-1], d))
        pre = plain.product(xr, w1, bounds)[0] + b1[group]
        h = plain.activation(pre, "gelu")
        yr = plain.product(h, w2, bounds)[0]
        return plain.combine(yr, places, gates, res, d), (xr, pre, h, yr)

    _, (xr, pre, h, yr) = forward(x, w1, b1, w2, gates)
    dyr, d_gates = plain.combine_backward(dy, yr, places, gates, torch.zeros_like(yr))
    dw2 = plain.weights_gradient(dyr, h, bounds)[0]
    dpre = plain.input_gradient(dyr, w2, bounds)[0] * plain.slope(pre, "gelu")
    dw1, _, db1, _ = plain.weights_gradient(dpre, xr, bounds)
    dx = plain.combine(plain.input_gradient(dpre, w1, bounds)[0], places, None, None, d)
    eps = 1e-6
    for at, (value, grad) in enumerate(((x, dx), (w1, dw1), (b1, db1), (w2, dw2), (gates, d_gates))):
        for i in range(min(value.numel(), 24)):
            args = [x, w1, b1, w2, gates]
            ends = []
            for sign in (1, -1):
                moved = value.clone()
                moved.view(-1)[i] += sign * eps
                args[at] = moved
                ends.append(float((forward(*args)[0] * dy).sum()))
            if at == 4 and not value.view(-1)[i]:
                assert grad.view(-1)[i] == 0                        # a pair without a part
                continue
            assert abs((ends[0] - ends[1]) / (2 * eps) - float(grad.view(-1)[i])) < 1e-6
