"""GPU tests of the weights' gradients of heads, to the last bit: sums of whole numbers, which fp32 holds in any order.

Inputs are 1 and -1, so that 1 / sqrt(mean(x^2)) is 1 (the widths are those whose rounded inverse times the width rounds to 1), positions are 0, so that no
pair turns by more than nothing, and the outputs' gradients are whole numbers from 1 to 8 of either sign: each head of each row counts in
every column, and one that is left out, taken twice or added to another's column or kind shows."""
import numpy as np
import pytest
import torch

import paper_2310_12670_amd as reft
from test_gpu_step import DT, dev  # noqa: F401

pytestmark = pytest.mark.gpu


def whole(dev, seed, *shape, top=8):  # noqa: F811
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    size = torch.randint(1, top + 1, shape, device=dev, generator=gen)
    return size * (torch.randint(0, 2, shape, device=dev, generator=gen) * 2 - 1)


# one row and one head; a unit, a block, 512 blocks and more, in one round and several; heads of 8, 16, 32 and 64 lanes; more keys than queries
SIZES = [(1, 1, 1, 8, 4), (1, 64, 8, 128, 64), (3, 5, 2, 40, 10), (7, 200, 65, 16, 8), (1001, 9, 3, 80, 10), (1024, 72, 8, 128, 64), (2049, 9, 3, 128, 32),
         (2500, 32, 8, 80, 40), (4096, 8, 1, 128, 64), (5000, 3, 7, 64, 16), (9001, 1, 1, 40, 20), (2600, 3, 1, 512, 256), (3000, 2, 12, 200, 100),
         (16384, 4, 1, 128, 64), (16411, 1, 2, 72, 30), (70000, 1, 1, 8, 2), (2048, 64, 8, 96, 48)]


@pytest.mark.parametrize("rows,q_heads,k_heads,cols,pairs", SIZES)
@pytest.mark.parametrize("adjacent,dtype", [(False, "bf16"), (True, "f16"), (False, "f32")])
def test_every_head_counts_once(dev, rows, q_heads, k_heads, cols, pairs, adjacent, dtype):  # noqa: F811
    assert np.float32(cols) * (np.float32(1) / np.float32(cols)) == 1 and rows * max(q_heads, k_heads) * 8 < 1 << 24
    T = DT[dtype]
    x, g = zip(*((whole(dev, s, rows, n, cols, top=1), whole(dev, s + 9, rows, n, cols)) for s, n in ((1, q_heads), (2, k_heads))))
    want = [(a * b).sum((0, 1)).float() for a, b in zip(x, g)]
    x, g = ([t.to(T) for t in pair] for pair in (x, g))
    weight = (1 + torch.arange(cols, device=dev) / cols).to(T)
    positions, freqs = torch.zeros(rows, dtype=torch.int64, device=dev), torch.ones(pairs, device=dev)
    dw = torch.full((2, cols), float("nan"), device=dev)
    ws = torch.full((reft.reft_heads_backward_workspace(rows, q_heads, k_heads, cols),), 0xFF, dtype=torch.uint8, device=dev)
    reft.reft_heads_backward(*g, *x, weight, weight, positions, freqs, 0.0, adjacent=adjacent, dq_weight=dw[0], dk_weight=dw[1], workspace=ws)
    assert torch.equal(dw[0], want[0]) and torch.equal(dw[1], want[1])
