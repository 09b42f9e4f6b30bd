"""Operands that a kernel must not be given, through the binding and without a GPU: tensors in host memory or on another GPU."""
import pytest
import torch

import paper_2310_12670_amd as reft

E4 = torch.float8_e4m3fn


def eight(rows, cols):
    return torch.zeros(rows, cols, dtype=torch.uint8).view(E4)


def words(rows, cols):
    return torch.zeros(-(-cols // 512), rows, 4, dtype=torch.uint8)


def calls():
    x, w, r = torch.zeros(4, 32), torch.ones(32), torch.ones(4)
    bytes_ = torch.zeros(1 << 16, dtype=torch.uint8)
    return {
        "dropout": lambda: reft.reft_dropout(x, x, 0.1, 1),
        "norm_forward": lambda: reft.reft_norm_forward(x, None, w, 1e-5, y=x),
        "norm_forward, 8 bits": lambda: reft.reft_norm_forward(x, x, w, 1e-5, h=x, rstd=r, q=eight(4, 32), scales=words(4, 32)),
        "norm_backward": lambda: reft.reft_norm_backward(x, x, x, r, w, dres=x, dx=x, dweight=w, workspace=bytes_),
        "quantize": lambda: reft.reft_quantize(x, eight(4, 32), words(4, 32), eight(32, 4), words(32, 4)),
        "quantize, blocks": lambda: reft.reft_quantize(x, eight(4, 32), words(1, 32), blocks=True),
        "product": lambda: reft.reft_product(eight(4, 32), words(4, 32), eight(6, 32), words(6, 32), torch.zeros(4, 6), bytes_),
    }


@pytest.mark.parametrize("name", list(calls()))
def test_host_memory_is_refused(name):
    """Right in everything else: the call must not come to a launch, which would read host addresses on the GPU."""
    for _ in range(2):                                       # the second time the types are known to the binding's C part
        with pytest.raises(reft.ReftError) as e:
            calls()[name]()
        assert e.value.code == reft.REFT_EINVAL and "cpu" in e.value.message


class Elsewhere:
    """A tensor's attributes with another GPU's memory behind them."""

    device = "cuda:77"

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 77


def test_another_gpus_memory_is_refused():
    x, q, s = Elsewhere(torch.zeros(4, 32)), Elsewhere(eight(4, 32)), Elsewhere(words(4, 32))
    for call in (lambda: reft.reft_dropout(x, x, 0.1, 1), lambda: reft.reft_quantize(x, q, s)):
        for _ in range(2):
            with pytest.raises(reft.ReftError) as e:
                call()
            assert e.value.code == reft.REFT_EINVAL and "cuda:77" in e.value.message


def test_what_else_is_wrong_is_said_first():
    x, w = torch.zeros(4, 32), torch.ones(32)
    with pytest.raises(reft.ReftError) as e:
        reft.reft_norm_backward(x, None, x, torch.ones(4), w, dweight=w, workspace=torch.zeros(8, dtype=torch.uint8))
    assert e.value.code == reft.REFT_ESIZE
    reft.reft_dropout(torch.zeros(0, 32), torch.zeros(0, 32), 0.1, 1)          # nothing to read: nothing to refuse


@pytest.mark.parametrize("workspace", [torch.zeros(1 << 16, dtype=torch.uint8)[::2], torch.zeros(256, 256, dtype=torch.uint8).t(),
                                       torch.zeros(128, 256, dtype=torch.uint8)[:, :128], torch.zeros(1 << 14)[::3]])
def test_a_workspace_with_gaps_is_refused(workspace):
    """Its bytes are counted without the gaps, but would be written into them."""
    x, w = torch.zeros(4, 32), torch.ones(32)
    for call in (lambda: reft.reft_norm_backward(x, None, x, torch.ones(4), w, dweight=w, workspace=workspace),
                 lambda: reft.reft_product(eight(60, 2000), words(60, 2000), eight(520, 2000), words(520, 2000), torch.zeros(60, 520), workspace)):
        with pytest.raises(reft.ReftError) as e:
            call()
        assert e.value.code == reft.REFT_EINVAL and "contiguous" in e.value.message


def refused(code, fn, *args, **kw):
    with pytest.raises(reft.ReftError) as e:
        fn(*args, **kw)
    assert e.value.code == code
    return e.value.message


def test_workspaces_that_do_not_hold_what_is_written():
    """A product whose K is cut writes its parts there, the norm's gradient its blocks' sums: nothing else keeps them inside."""
    M, N, K = 60, 520, 2000
    need = reft.reft_product_workspace(M, N, K)
    assert need == 2 * M * N * 4
    a, sa, b, sb, c = eight(M, K), words(M, K), eight(N, K), words(N, K), torch.zeros(M, N)
    room = torch.zeros(need + 16, dtype=torch.uint8)
    assert room.data_ptr() % 16 == 0
    product = (a, sa, b, sb, c)
    assert "no workspace" in refused(reft.REFT_EINVAL, reft.reft_product, *product)
    assert "16 bytes" in refused(reft.REFT_EINVAL, reft.reft_product, *product, room[8:])
    assert "too small" in refused(reft.REFT_ESIZE, reft.reft_product, *product, room[:need - 1])
    assert "cpu" in refused(reft.REFT_EINVAL, reft.reft_product, *product, room[:need])          # right but for the memory
    assert "cpu" in refused(reft.REFT_EINVAL, reft.reft_product, eight(4, 32), words(4, 32), eight(6, 32), words(6, 32), torch.zeros(4, 6))
    rows, cols = 700, 264
    need = reft.reft_norm_backward_workspace(rows, cols)
    assert need > cols * 4 and need % (cols * 4) == 0
    x, r, w = torch.zeros(rows, cols), torch.ones(rows), torch.ones(cols)
    room = torch.zeros(need + 16, dtype=torch.uint8)
    norm = lambda room: reft.reft_norm_backward(x, None, x, r, w, dweight=w, workspace=room)      # noqa: E731
    assert "no workspace" in refused(reft.REFT_EINVAL, norm, None)
    assert "16 bytes" in refused(reft.REFT_EINVAL, norm, room[4:])
    assert "too small" in refused(reft.REFT_ESIZE, norm, room[:need - 1])
    assert "cpu" in refused(reft.REFT_EINVAL, norm, room[:need])


@pytest.mark.parametrize("wrong", [1 << 40, 3.5, "x", [1.0], None])
def test_operands_that_are_no_tensors(wrong):
    x, w, r, q, s = torch.zeros(4, 32), torch.ones(32), torch.ones(4), eight(4, 32), words(4, 32)
    refused(reft.REFT_EINVAL, reft.reft_dropout, wrong, x, 0.1, 1)
    refused(reft.REFT_EINVAL, reft.reft_dropout, x, wrong, 0.1, 1)
    refused(reft.REFT_EINVAL, reft.reft_norm_forward, wrong, None, w, 1e-5, y=x)
    refused(reft.REFT_EINVAL, reft.reft_norm_forward, x, None, wrong, 1e-5, y=x)
    refused(reft.REFT_EINVAL, reft.reft_norm_backward, x, None, wrong, r, w, dres=x)
    refused(reft.REFT_EINVAL, reft.reft_norm_backward, x, None, x, wrong, w, dres=x)
    refused(reft.REFT_EINVAL, reft.reft_quantize, wrong, q, s)
    refused(reft.REFT_EINVAL, reft.reft_quantize, x, q, wrong)
    refused(reft.REFT_EINVAL, reft.reft_product, q, s, q, s, wrong)
    refused(reft.REFT_EINVAL, reft.reft_product, q, wrong, q, s, torch.zeros(4, 4))
    refused(reft.REFT_EINVAL, reft.reft_product, eight(60, 2000), words(60, 2000), eight(520, 2000), words(520, 2000), torch.zeros(60, 520), wrong)


@pytest.mark.parametrize("wrong", [1 << 64, -(1 << 63) - 1, 1 << 80])
def test_seeds_and_offsets_have_64_bits(wrong):
    """More would be cut off without a word: two counters that differ would give one mask."""
    x, r, w = torch.zeros(4, 32), torch.ones(4), torch.ones(32)
    for seed, offset in ((wrong, 0), (0, wrong)):
        assert "64 bits" in refused(reft.REFT_EINVAL, reft.reft_dropout, x, x, 0.1, seed, offset)
        assert "64 bits" in refused(reft.REFT_EINVAL, reft.reft_norm_forward, x, None, w, 1e-5, 0.1, seed, offset, y=x)
        assert "64 bits" in refused(reft.REFT_EINVAL, reft.reft_norm_backward, x, None, x, r, w, 0.1, seed, offset, dres=x)
    for seed in ((1 << 64) - 1, -1, -(1 << 63)):
        assert "cpu" in refused(reft.REFT_EINVAL, reft.reft_dropout, x, x, 0.1, seed, seed)          # right but for the memory
