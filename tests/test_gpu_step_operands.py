"""GPU tests of operands in other memory than the GPU's own: pinned host memory works, other host memory is refused."""
import pytest
import torch

import paper_2310_12670_amd as reft

pytestmark = pytest.mark.gpu


def test_pinned_host_memory():
    dev = torch.device("cuda:0")
    torch.cuda.set_device(dev)
    x = torch.randn(37, 130, pin_memory=True)
    y, want = torch.empty(37, 130, pin_memory=True), torch.empty(37, 130, device=dev)
    reft.reft_dropout(x, y, 0.3, 5, 6)
    reft.reft_dropout(x.to(dev), want, 0.3, 5, 6)
    torch.cuda.synchronize()
    assert torch.equal(y, want.cpu()) and y.any()


@pytest.mark.parametrize("which", range(3))
def test_one_operand_in_host_memory(which):
    dev = torch.device("cuda:0")
    torch.cuda.set_device(dev)
    x, w, y = torch.randn(5, 64, device=dev), torch.ones(64, device=dev), torch.full((5, 64), 3.0, device=dev)
    operands = [x, w, y]
    operands[which] = operands[which].cpu()
    with pytest.raises(reft.ReftError) as e:
        reft.reft_norm_forward(operands[0], None, operands[1], 1e-5, y=operands[2])
    assert e.value.code == reft.REFT_EINVAL and ("x", "weight", "y")[which] + " is on cpu" in e.value.message
    torch.cuda.synchronize()
    assert (y == 3).all()
