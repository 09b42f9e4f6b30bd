"""GPU test of the example that trains with the operators, loses its state, restores it and repeats the steps."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "this test needs the GPU"
    spec = importlib.util.spec_from_file_location("resume_training", os.path.join(ROOT, "examples", "resume_training.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_steps_after_a_restore_repeat_to_the_same_bits(example):
    before, after, again, same = example.run(steps=12, snapshot=5)
    assert same and after == again
    # and it trains: Adam's first steps of 1e-3 on 256-wide weights lower a mean square error of about 2
    assert after[-1] < before[0]
    assert all(0 < v < 10 for v in before + after)


def test_gradients_of_the_example_agree_with_autograd(example):
    """One step's gradients, by what they did to the first moment (0.1 g), against autograd in fp32 without 8 bits: as near as the
    8-bit operands allow (each product rounds both to 2^-4 at most, 3 % in the mean)."""
    import numpy as np
    from oracle import step as oracle_step
    dev = torch.device("cuda:0")
    model = example.Model(dev)
    gen = torch.Generator(device=dev)
    gen.manual_seed(3)
    x = torch.randn(128, 256, device=dev, generator=gen).to(torch.bfloat16)
    target = torch.randn(128, 256, device=dev, generator=gen)
    weights = [p.float().cpu().requires_grad_(True) for p in model.param]
    h, s = x.float().cpu(), torch.zeros(128, 256)
    seed = 0x5EED

    def joined(h, s, offset):
        keep, scale = oracle_step.keep_mask(128, 256, example.DROP, seed, offset)
        return h + torch.where(torch.from_numpy(np.ascontiguousarray(keep)), s * scale, torch.zeros(()))

    def norm(h, w):
        return h * torch.rsqrt(h.square().mean(1, keepdim=True) + example.EPS) * w

    for i in range(model.layers):
        h = joined(h, s, i)
        s = torch.relu(norm(h, weights[3 * i]) @ weights[3 * i + 1].t()).square() @ weights[3 * i + 2].t()
    loss = (norm(joined(h, s, model.layers), weights[-1]) - target.cpu()).square().mean()
    loss.backward()
    got = model.step(x, target)
    assert abs(got - float(loss.detach())) <= 0.02 * float(loss.detach())
    for m, w in zip(model.first, weights):
        g = m.cpu() / 0.1
        assert float((g - w.grad).norm()) <= 0.15 * float(w.grad.norm())
