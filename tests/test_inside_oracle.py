"""The 64-bit forms of the operators inside the sublayers (CPU): each against something worked out another way."""
import math

import numpy as np
import pytest
import torch

from oracle import step

KINDS = ["silu", "gelu", "gelu_tanh", "relu2"]


@pytest.mark.parametrize("kind", KINDS)
def test_activations(kind):
    """Against torch's in 64 bits, and the slope against differences."""
    g = np.concatenate([np.linspace(-12, 12, 4001), [0.0, 1e-9, -1e-9, 700.0]])
    t = torch.from_numpy(g)
    f = torch.nn.functional
    want = {"silu": lambda: f.silu(t), "gelu": lambda: f.gelu(t), "gelu_tanh": lambda: f.gelu(t, approximate="tanh"),
            "relu2": lambda: f.relu(t).square()}[kind]().numpy()
    a, slope = step.act(g, kind)
    assert np.allclose(a, want, rtol=1e-13, atol=1e-15)
    d = 1e-6
    near = (np.abs(g) > 2 * d) & (np.abs(g) < 100)
    # differences err by d^2 and by rounding of a (at most 144) over d
    assert np.allclose(slope[near], ((step.act(g + d, kind)[0] - step.act(g - d, kind)[0]) / (2 * d))[near], atol=1e-7)


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotation(adjacent):
    """By hand, its inverse, and that products of two turned vectors depend on the distance alone."""
    x = np.array([[[3.0, 1.0, 2.0, 5.0, 7.0]]])
    p = np.array([2])
    f = np.array([0.25, 0.5])
    y = step.turned(x, p, f, adjacent)[0, 0]
    first, second = ((3.0, 1.0), (2.0, 5.0)) if adjacent else ((3.0, 2.0), (1.0, 5.0))
    at = ((0, 1), (2, 3)) if adjacent else ((0, 2), (1, 3))
    for (a, b), (i, j), t in ((first, at[0], 0.5), (second, at[1], 1.0)):
        assert math.isclose(y[i], a * math.cos(t) - b * math.sin(t)) and math.isclose(y[j], b * math.cos(t) + a * math.sin(t))
    assert y[4] == 7.0
    assert np.allclose(step.turned(y[None, None], p, f, adjacent, back=True), x)
    rng = np.random.default_rng(1)
    q, k = rng.normal(size=(1, 1, 8)), rng.normal(size=(1, 1, 8))
    f = np.array([1.0, 0.1, 0.01])
    dots = [(step.turned(q, [n + 5], f, adjacent) * step.turned(k, [n], f, adjacent)).sum() for n in (0, 3, 1000)]
    assert np.allclose(dots, dots[0])


@pytest.mark.parametrize("adjacent", [False, True])
def test_gradient_of_heads_against_differences(adjacent):
    rng = np.random.default_rng(2)
    x, w, dout = rng.normal(size=(3, 2, 9)), 1 + 0.2 * rng.normal(size=9), rng.normal(size=(3, 2, 9))
    rest = (np.array([0, 7, 100]), np.array([1.0, 0.3]), 1e-5, adjacent)
    dx, dw = step.heads_backward(dout, x, w, *rest)
    t = 1e-6
    for which, grad in ((0, dx), (1, dw)):
        for _ in range(5):
            to = rng.normal(size=grad.shape)
            ends = []
            for sign in (t, -t):
                args = [x, w]
                args[which] = args[which] + sign * to
                ends.append((step.heads_forward(*args, *rest) * dout).sum())
            slope = (ends[0] - ends[1]) / (2 * t)
            assert abs(slope - (grad * to).sum()) <= 1e-7 * np.abs(grad * to).sum()


@pytest.mark.parametrize("kind", KINDS)
def test_gradient_of_the_gate_against_differences(kind):
    rng = np.random.default_rng(3)
    g, u, dy = rng.normal(size=(2, 50)), rng.normal(size=(2, 50)), rng.normal(size=(2, 50))
    dg, du, y = step.gate_backward(dy, g, u, kind)
    assert np.allclose(y, step.act(g, kind)[0] * u)
    t = 1e-6
    assert np.allclose(dg, dy * u * (step.act(g + t, kind)[0] - step.act(g - t, kind)[0]) / (2 * t), atol=1e-7)
    assert np.allclose(du, dy * step.act(g, kind)[0])
    alone = step.gate_backward(dy, g, None, kind)
    assert alone[1] is None and np.allclose(alone[0] * u, dg) and np.allclose(alone[2] * u, y)


def test_transpose():
    """Powers of two that differ along a row of the result: values keep their bits until they are subnormal."""
    q = np.array([[1.75, -448.0], [0.875, 1.0]])
    scales = np.full((1, 2, 4), 127, dtype=np.uint8)
    scales[0, 1, 0] = 137
    t, e = step.transpose(q, scales, "e4m3")
    # columns: 1.75 and 0.875 2^10 = 896; -448 and 2^10
    assert e[:, 0].tolist() == [128, 129]
    assert t.tolist() == [[0.875, 448.0], [-112.0, 256.0]]
