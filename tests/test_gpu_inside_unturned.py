"""GPU tests of the columns of heads that do not turn: out[c] = z[c] and its gradient, whatever stands in the columns beside them."""
import pytest
import torch

import paper_2310_12670_amd as reft
from test_gpu_inside import EPS, angles
from test_gpu_step import DT, dev, normal  # noqa: F401

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
SHAPES = [(128, 32), (80, 16), (80, 10), (81, 10), (64, 8), (64, 1), (40, 0), (260, 64), (512, 101), (72, 20)]


@pytest.mark.parametrize("cols,pairs", SHAPES)
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_a_weight_reaches_its_own_column_alone(dev, cols, pairs, adjacent, dtype):  # noqa: F811
    rows, heads, T = 9, 3, DT[dtype]
    x = normal(dev, 1, rows, heads, cols, dtype=T)
    x[x == 0] = 1
    positions, freqs = angles(dev, rows, pairs)
    weight = (1 + normal(dev, 2, cols, std=0.2)).to(T)
    want, got = torch.empty_like(x), torch.empty_like(x)
    reft.reft_heads_forward(x, None, weight, None, positions, freqs, EPS, want, adjacent=adjacent)
    spoilt = weight.clone()
    at = {2 * pairs: INF, 2 * pairs + 3: NAN, 2 * pairs + 4: -INF, cols - 1: INF}
    for c, v in at.items():
        spoilt[c] = v
        want[..., c] = x[..., c] * v
    reft.reft_heads_forward(x, None, spoilt, None, positions, freqs, EPS, got, adjacent=adjacent)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(nan=7.0), want.nan_to_num(nan=7.0))


@pytest.mark.parametrize("cols,pairs", SHAPES)
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_a_gradient_reaches_its_own_column_of_the_weights_alone(dev, cols, pairs, adjacent, dtype):  # noqa: F811
    rows, heads, T = 9, 3, DT[dtype]
    x, dout = normal(dev, 1, rows, heads, cols, dtype=T), normal(dev, 2, rows, heads, cols, dtype=T)
    x[x == 0] = 1
    positions, freqs = angles(dev, rows, pairs)
    ws = torch.empty(reft.reft_heads_backward_workspace(rows, heads, 0, cols), dtype=torch.uint8, device=dev)
    at = {2 * pairs: INF, 2 * pairs + 3: NAN, 2 * pairs + 4: -INF, cols - 1: INF}
    got = []
    for spoilt in (False, True):
        for (r, h), (c, v) in zip(((0, 0), (3, 2), (3, 1), (8, 2)), at.items()):
            dout[r, h, c] = v if spoilt else 0
        dx, dw = torch.empty_like(x), torch.empty(cols, device=dev)
        reft.reft_heads_backward(dout, None, x, None, None, None, positions, freqs, EPS, adjacent=adjacent, dq=dx, dq_weight=dw, workspace=ws)
        got.append((dx, dw))
    (dx, dw), (other, sums) = got
    for (r, h), (c, v) in zip(((0, 0), (3, 2), (3, 1), (8, 2)), at.items()):
        dw[c] = float(x[r, h, c]) * v
        assert not torch.isfinite(other[r, h]).any()                         # the mean of u weight x' of that head is no number
        dx[r, h] = other[r, h] = 0
    assert torch.equal(dx, other) and torch.isfinite(dx).all()
    assert torch.equal(torch.isnan(sums), torch.isnan(dw)) and torch.equal(sums.nan_to_num(nan=7.0), dw.nan_to_num(nan=7.0))
