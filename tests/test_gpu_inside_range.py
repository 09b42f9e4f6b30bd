"""GPU tests of the magnitudes for which include/reft.h states the operators' formulas inside the sublayers, and of what it states beyond them."""
import numpy as np
import pytest
import torch

import paper_2310_12670_amd as reft
from oracle import step
from test_gpu_inside import EPS, angles
from test_gpu_step import DT, U, dev, f64, normal  # noqa: F401

pytestmark = pytest.mark.gpu


def both(dev, x, dout, weight, positions, freqs, eps):  # noqa: F811
    out, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(x.shape[2], device=dev)
    ws = torch.empty(reft.reft_heads_backward_workspace(x.shape[0], x.shape[1], 0, x.shape[2]), dtype=torch.uint8, device=dev)
    reft.reft_heads_forward(x, None, weight, None, positions, freqs, eps, out)
    reft.reft_heads_backward(dout, None, x, None, weight, None, positions, freqs, eps, dq=dx, dq_weight=dw, workspace=ws)
    return out, dx, dw


@pytest.mark.parametrize("cols,pairs", [(64, 32), (128, 32), (80, 10)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [-62, 58])
def test_heads_of_large_and_small_numbers(dev, cols, pairs, dtype, power):  # noqa: F811
    """Magnitudes from 1 to 2 times an even power of two: squares and sums stay normal, and with eps == 0 each result is the same times a power."""
    rows, heads = 11, 3
    x = normal(dev, 1, rows, heads, cols).sign() * (1 + torch.rand(rows, heads, cols, device=dev))
    x = x.to(DT[dtype])
    dout, weight = normal(dev, 2, rows, heads, cols, dtype=DT[dtype]), (1 + normal(dev, 3, cols, std=0.2)).to(DT[dtype])
    rest = (dout, weight, *angles(dev, rows, pairs), 0.0)
    out, dx, dw = both(dev, x, *rest)
    far, dfar, dwfar = both(dev, x * 2.0 ** power, *rest)
    assert torch.equal(far, out) and torch.equal(dwfar, dw) and torch.equal(dfar * 2.0 ** power, dx) and torch.isfinite(dx).all() and dx.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [2.0 ** 64, 1e30, 3e38])
def test_heads_whose_squares_leave_fp32(dev, dtype, size):  # noqa: F811
    """Their x' counts as zero: in the results, their gradient and their part of the weights' gradient."""
    rows, heads, cols = 40, 3, 128
    x, dout = normal(dev, 1, rows, heads, cols, dtype=DT[dtype]), normal(dev, 2, rows, heads, cols, dtype=DT[dtype])
    rest = (None, *angles(dev, rows, 32), EPS)
    large = torch.zeros(rows, heads, dtype=torch.bool, device=dev)
    large[3, 1] = large[17, 0] = large[39, 2] = True
    x[large] = 0
    none, _, sums = both(dev, x, dout, *rest)
    x[17, 0], x[39, 2, 5], x[3, 1, 0] = size, size, -size
    out, dx, dw = both(dev, x, dout, *rest)
    assert not out[large].any() and not dx[large].any() and torch.equal(dw, sums)
    assert torch.equal(out[~large], none[~large]) and torch.isfinite(dx).all()


def test_heads_whose_squares_vanish(dev):  # noqa: F811
    """With eps == 0 as a head of zeroes; with more each value counts."""
    x = normal(dev, 1, 5, 2, 64).sign() * 2.0 ** -80
    out = torch.empty_like(x)
    reft.reft_heads_forward(x, None, None, None, None, None, 0.0, out)
    assert not torch.isfinite(out).any()
    reft.reft_heads_forward(x, None, None, None, None, None, 2.0 ** -20, out)
    assert torch.equal(out, x * 2.0 ** 10)
    x.zero_()
    reft.reft_heads_forward(x, None, None, None, None, None, 0.0, out)
    assert torch.isnan(out).all()


@pytest.mark.parametrize("kind,ends,exponent", [("silu", (-87, 20), lambda g: 1.25 * np.abs(g)), ("gelu", (-13, 6), lambda g: 2.25 * g * g / 2),
                                                ("gelu_tanh", (-9, 5), lambda g: 6 * np.sqrt(8 / np.pi) * np.abs(g + 0.044715 * g ** 3))])
def test_errors_of_small_activations(dev, kind, ends, exponent):  # noqa: F811
    """Relative to the value: the exponent's roundings, and the steps that each operation beside it counts (a tail's polynomial in gelu)."""
    g = torch.linspace(*ends, 100003, device=dev).view(1, -1)
    y = torch.empty_like(g)
    reft.reft_gate_forward(g, None, kind, y=y)
    want, _ = step.act(f64(g), kind)
    assert (np.abs(f64(y) - want) <= (exponent(f64(g)) + (40 if kind == "gelu" else 8)) * U * np.abs(want) + 2.0 ** -126).all()
