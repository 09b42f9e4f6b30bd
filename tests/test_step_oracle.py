"""The 64-bit forms of the training step's operators (CPU): each against something worked out another way."""
import numpy as np
import pytest
import torch

from oracle import step


def test_philox_known_answers():
    """Counter and key all zeros and all ones, as published with the generator."""
    def words(c, k):
        return [int(w) for w in step.philox4x32([np.uint64(x) for x in c], k)]
    assert words([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert words([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_mask_depends_on_place_and_counter_only():
    whole, _ = step.keep_mask(9, 100, 0.3, 2 ** 63 + 5, 2 ** 40 + 1)
    part, _ = step.keep_mask(4, 37, 0.3, 2 ** 63 + 5, 2 ** 40 + 1)
    assert np.array_equal(whole[:4, :37], part)
    other, _ = step.keep_mask(9, 100, 0.3, 2 ** 63 + 5, 2 ** 40 + 2)
    assert 0.2 < (whole != other).mean() < 0.65


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_share_of_kept_elements(p):
    keep, scale = step.keep_mask(400, 500, p, 11, 3)
    # five standard deviations of 200,000 draws
    assert abs(keep.mean() - (1 - p)) <= 5 * np.sqrt(p * (1 - p) / keep.size) + 1 / 65536
    assert scale == (65536 / (65536 - round(p * 65536)) if p < 1 else 0.0)


@pytest.mark.parametrize("fmt,dtype", [("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)])
def test_rounding_to_8_bits(fmt, dtype):
    """Every value of the format, halves between neighbours and what lies next to them, against torch's conversion."""
    every = torch.arange(256, dtype=torch.uint8).view(dtype).double()
    v = np.unique(every[torch.isfinite(every)].numpy())
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid.astype(np.float32), np.float32(0)).astype(np.float64)])
    got = step.round_to(x, fmt)
    assert np.array_equal(got, torch.from_numpy(x).float().to(dtype).double().numpy())


def test_scales_are_the_smallest_that_fit():
    x = np.array([[448.0, 1.0], [448.0001, 0.0], [0.0, 0.0], [1e-45, 0.0], [3.4e38, 1.0], [np.inf, 1.0], [np.nan, 1.0]])
    q, e = step.quantize(x, "e4m3", False)
    assert e[:, 0].tolist() == [127, 128, 1, 1, 247, 255, 255]
    assert q[0, 0] == 448 and q[1, 0] == 224 and np.isnan(q[5]).all() and np.isnan(q[6]).all()


def test_gradient_of_the_norm_against_differences():
    rng = np.random.default_rng(4)
    x, res, w = rng.normal(size=(5, 33)), rng.normal(size=(5, 33)), 1 + 0.1 * rng.normal(size=33)
    dy, dh = rng.normal(size=(5, 33)), rng.normal(size=(5, 33))
    args = (1e-5, 0.3, 77, 5)

    def loss(x, res, w):
        h, _, y = step.norm_forward(x, res, w, *args)
        return (y * dy).sum() + (h * dh).sum()

    h, rstd, _ = step.norm_forward(x, res, w, *args)
    dres, dx, dw = step.norm_backward(dy, dh, h, rstd, w, *args[1:])
    t = 1e-6
    for which, grad in ((0, dx), (1, dres), (2, dw)):
        for _ in range(5):
            to = rng.normal(size=grad.shape)
            up, down = [x, res, w], [x, res, w]
            up[which], down[which] = up[which] + t * to, down[which] - t * to
            slope = (loss(*up) - loss(*down)) / (2 * t)
            # eps makes the formula exact only up to eps * rstd^2, which rstd itself holds; differences err by about 1e-8
            assert abs(slope - (grad * to).sum()) <= 1e-6 * np.abs(grad * to).sum()
