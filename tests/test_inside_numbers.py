"""Numbers of activations (no GPU): one that is none is refused, also where its lowest 32 bits are those of one."""
import pytest
import torch

import paper_2310_12670_amd as reft


def pair(rows, cols):
    return torch.zeros(rows, cols, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(-(-cols // 512), rows, 4, dtype=torch.uint8)


@pytest.mark.parametrize("act", [4, 255, 256, -1, 2 ** 31, 2 ** 32, 2 ** 32 + 1, -2 ** 32, 2 ** 64, 2 ** 70 + 2])
def test_an_activation_that_is_none(act):
    x = torch.zeros(4, 8)
    for call in (lambda: reft.reft_gate_forward(x, None, act, y=x), lambda: reft.reft_gate_backward(x, pair(4, 8), None, act, dg=x)):
        with pytest.raises(reft.ReftError, match="unknown activation") as e:
            call()
        assert e.value.code == reft.REFT_EINVAL
