"""GPU tests of the training step's operators: what should not matter - where rows lie and how far apart - changes no bit, and every
kernel that sizes and alignment choose between is compared with the definition."""
import numpy as np
import pytest
import torch

import paper_2310_12670_amd as reft
from oracle import step

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E4 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "these tests need the GPU"
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


def normal(dev, seed, *shape, std=1.0, dtype=torch.float32):
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    return (torch.randn(*shape, device=dev, generator=gen) * std).to(dtype)


def rows_at(dev, values, ld, lead):
    """The same 8-bit values in rows that lie ld apart and begin `lead` bytes into their memory; what lies between is no number."""
    rows, cols = values.shape
    raw = torch.full((lead + rows * ld + 16,), 0x7F, dtype=torch.uint8, device=dev)
    view = torch.as_strided(raw, (rows, cols), (ld, 1), lead)
    view.copy_(values.view(torch.uint8))
    return view.view(E4)


# K cut into parts (with its end in a chunk, at a chunk's end, at a block's end), not cut, and the largest tiles; rows of few tokens
@pytest.mark.parametrize("M,N,K", [(40, 300, 4097), (64, 512, 2048), (130, 300, 4097), (200, 300, 9001), (128, 1024, 11008), (1001, 770, 5128),
                                   (300, 700, 896), (2900, 3000, 3712), (5, 700, 1000)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_product_where_rows_lie_changes_no_bit(dev, M, N, K, out):
    a, b = normal(dev, 1, M, K).to(E4), normal(dev, 2, N, K).to(E4)
    gen = torch.Generator(device=dev)
    gen.manual_seed(3)
    sa, sb = (torch.randint(120, 135, (-(-K // 512), n, 4), dtype=torch.uint8, device=dev, generator=gen) for n in (M, N))
    ws = torch.empty(reft.reft_product_workspace(M, N, K), dtype=torch.uint8, device=dev)
    even = -(-K // 16) * 16
    want = None
    # rows on 16 bytes; one byte on; an odd row length on one side; rows too far apart for offsets of 32 bits in a tile
    for ld_a, lead_a, ld_b, lead_b in [(even, 0, even, 0), (even, 1, even, 0), (even, 0, even + 1, 0), (1 << 23, 0, even, 0)][:4 if M < 300 else 3]:
        c = torch.empty(M, N, dtype=DT[out], device=dev)
        reft.reft_product(rows_at(dev, a, ld_a, lead_a), sa, rows_at(dev, b, ld_b, lead_b), sb, c, ws)
        assert torch.isfinite(c).all() and c.any()
        want = c if want is None else want
        assert torch.equal(c, want), (ld_a, lead_a, ld_b, lead_b)


# ---- the largest sizes that the header allows ---------------------------------------------------------------------
def test_quantize_of_the_most_rows(dev):
    rows, half = (1 << 26) - 1, 1 << 25
    x = normal(dev, 1, rows, 1)
    q, s = torch.empty(rows, 1, dtype=torch.uint8, device=dev).view(E4), torch.empty(1, rows, 4, dtype=torch.uint8, device=dev)
    reft.reft_quantize(x, q, s)
    for at in (slice(0, half), slice(half, rows)):
        n = at.stop - at.start
        r, t = torch.empty(n, 1, dtype=torch.uint8, device=dev).view(E4), torch.empty(1, n, 4, dtype=torch.uint8, device=dev)
        reft.reft_quantize(x[at], r, t)
        assert torch.equal(q[at].view(torch.uint8), r.view(torch.uint8)) and torch.equal(s[:, at], t)
    assert q.view(torch.uint8).any()


def test_product_of_few_rows_and_the_most_columns(dev):
    M, N, K, half = 3, (1 << 26) - 1, 16, 1 << 25
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)
    few = torch.arange(-2, 3, device=dev).to(torch.float32).to(E4).view(torch.uint8)
    a, b = (few[torch.randint(0, 5, (n, K), device=dev, generator=gen, dtype=torch.int32)].view(E4) for n in (M, N))
    sa, sb = torch.full((1, M, 4), 127, dtype=torch.uint8, device=dev), torch.full((1, -(-N // 128), 4), 126, dtype=torch.uint8, device=dev)
    c = torch.empty(M, N, dtype=torch.bfloat16, device=dev)
    reft.reft_product(a, sa, b, sb, c, b_blocks=True)
    for at in (slice(0, half), slice(half, N)):
        n = at.stop - at.start
        d, scales = torch.empty(M, n, dtype=torch.bfloat16, device=dev), sb[:, :-(-n // 128)]
        reft.reft_product(a, sa, b[at], scales.contiguous(), d, b_blocks=True)
        assert torch.equal(c[:, at], d) and d.any()


# ---- the kernels of ordinary layers: rows on cache lines, blocks that take several rows one after the other -------------------------
U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}          # half a step, of the value
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def f64(t):
    return t.detach().double().cpu().numpy()


def lines(dev, rows, cols, dtype, fill=None):
    """A matrix whose rows all begin on 128 bytes."""
    ld = -(-cols * SIZE[dtype] // 128) * 128 // SIZE[dtype]
    t = torch.empty(rows, ld, dtype=DT[dtype], device=dev)[:, :cols]
    assert t.data_ptr() % 128 == 0
    if fill is not None:
        t.copy_(fill)
    return t


@pytest.mark.parametrize("rows,cols,dtype", [(257, 4096, "bf16"), (61, 1056, "f32"), (700, 1000, "f16"), (3, 64, "bf16"), (2049, 2048, "bf16")])
def test_dropout_of_rows_on_lines(dev, rows, cols, dtype):
    x, y = lines(dev, rows, cols, dtype, normal(dev, rows, rows, cols)), lines(dev, rows, cols, dtype)
    reft.reft_dropout(x, y, 0.2, 2 ** 64 - 9, 2 ** 32 + 3)
    keep, scale = step.keep_mask(rows, cols, 0.2, 2 ** 64 - 9, 2 ** 32 + 3)
    want = torch.where(torch.from_numpy(keep).to(dev), x.float() * np.float32(scale), torch.zeros((), device=dev)).to(DT[dtype])
    assert torch.equal(y, want)
    reft.reft_dropout(x, x, 0.2, 2 ** 64 - 9, 2 ** 32 + 3)
    assert torch.equal(x, want)


@pytest.mark.parametrize("half_steps", [1, 3, 5, 65535, 65537, 131069, 131071])
def test_dropout_of_shares_between_two_thresholds(dev, half_steps):
    """p = half_steps / 131072 lies in the middle of two thresholds: the even one is taken, forward, backward and in the norm."""
    p, rows, cols = half_steps / 131072, 1000, 1200
    x = 1 + normal(dev, 1, rows, cols).abs()
    y, h = torch.empty_like(x), torch.empty_like(x)
    reft.reft_dropout(x, y, p, 11, 12)
    reft.reft_norm_forward(x, None, None, 1e-5, p, 11, 12, h=h)
    keep, _ = step.keep_mask(rows, cols, p, 11, 12)
    assert torch.equal(y != 0, torch.from_numpy(keep).to(dev)) and torch.equal(h, y)


def norm_back(dev, rows, cols, dtype, residual, place, p):
    """The gradients against the definition; err as in test_gpu_step.py: a sum of n terms errs by n U of their magnitudes."""
    dy, dh = place(dev, rows, cols, dtype, normal(dev, 1, rows, cols)), place(dev, rows, cols, residual, normal(dev, 2, rows, cols))
    h, w = place(dev, rows, cols, residual, normal(dev, 3, rows, cols, std=2.0)), 1 + normal(dev, 4, cols, std=0.3, dtype=DT[dtype])
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-5)
    want = step.norm_backward(f64(dy), f64(dh), f64(h), f64(rstd), f64(w), p, 77, 2 ** 40)
    dres, dx, dw = place(dev, rows, cols, residual), place(dev, rows, cols, dtype), torch.empty(cols, device=dev)
    ws = torch.empty(reft.reft_norm_backward_workspace(rows, cols), dtype=torch.uint8, device=dev)
    reft.reft_norm_backward(dy, dh, h, rstd, w, p, 77, 2 ** 40, dres=dres, dx=dx, dweight=dw, workspace=ws)
    xhat, g = f64(h) * f64(rstd)[:, None], f64(dy) * f64(w)
    dot = (g * xhat).mean(1, keepdims=True)
    # the mean: up to 64 products of three rounded factors a lane (each U times three), six steps in the wave, 16 waves
    dot_err = (64 + 6 + 16 + 6) * U * np.abs(g * xhat).mean(1, keepdims=True)
    err = f64(rstd)[:, None] * (4 * U * np.abs(g) + np.abs(xhat) * (dot_err + 4 * U * np.abs(dot))) + 2 * U * np.abs(want[0]) + U * np.abs(f64(dh))
    assert (np.abs(f64(dres) - want[0]) <= err + HALF[residual] * 1.01 * np.abs(want[0]) + TINY[residual]).all()
    factor = 65536 / (65536 - round(p * 65536))
    assert (np.abs(f64(dx) - want[1]) <= err * factor + (HALF[dtype] * 1.01 + 2 * U) * np.abs(want[1]) + TINY[dtype]).all()
    # each row is in one block's sum once
    assert (np.abs(f64(dw) - want[2]) <= (rows + 4) * U * np.abs(f64(dy) * xhat).sum(0)).all()
    kept = dres.clone(), dx.clone(), dw.clone()
    reft.reft_norm_backward(dy, dh, h, rstd, w, p, 77, 2 ** 40, dres=dh, dx=dy, dweight=dw, workspace=ws)
    assert torch.equal(dh, kept[0]) and torch.equal(dy, kept[1]) and torch.equal(dw, kept[2])


def odd(dev, rows, cols, dtype, fill=None):
    """Rows of an odd length that begin three elements into their memory."""
    t = torch.empty(rows * (cols | 1) + 3 + cols, dtype=DT[dtype], device=dev)
    t = torch.as_strided(t, (rows, cols), (cols | 1, 1), 3)
    if fill is not None:
        t.copy_(fill)
    return t


# eight columns a lane (1, 2, 4 and 16 waves a row), twice eight, and more than 16384 columns; each with several passes of a block's loop
ROWS = [(5000, 512), (3100, 1024), (4000, 2048), (1100, 8192), (1100, 2047), (2500, 2047), (700, 8200), (700, 16384), (600, 16392)]


@pytest.mark.parametrize("rows,cols", ROWS)
@pytest.mark.parametrize("dtype,residual,place", [("bf16", "bf16", lines), ("f16", "f32", lines), ("bf16", "f32", odd)])
def test_norm_backward_blocks_of_several_rows(dev, rows, cols, dtype, residual, place):
    blocks = reft.reft_norm_backward_workspace(rows, cols) // (4 * cols)
    assert rows > blocks * (1 if cols > 1024 else 2 if cols > 512 else 4)            # rows that a block takes side by side: 1, 2, 4
    norm_back(dev, rows, cols, dtype, residual, place, 0.1)


def test_norm_forward_in_two_launches(dev):
    """More than 2^21 rows; every row against the definition."""
    rows, cols, p = (1 << 21) + 5, 3, 0.25
    x, res, w = normal(dev, 1, rows, cols), normal(dev, 2, rows, cols), 1 + normal(dev, 3, cols, std=0.3)
    h, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device=dev)
    reft.reft_norm_forward(x, res, w, 1e-5, p, 7, 8, h=h, rstd=rstd, y=y)
    h64, rstd64, y64 = step.norm_forward(f64(x), f64(res), f64(w), 1e-5, p, 7, 8)
    drop = np.abs(step.dropout(f64(x), p, 7, 8))
    h_err = U * (3 * drop + 2 * np.abs(h64))                  # the factor, the product and the sum
    assert (np.abs(f64(h) - h64) <= h_err).all()
    rel = (16 / 2 + 4) * U + np.sqrt((h_err ** 2).mean(1)) * rstd64          # at most 8 squares and their sums, half of it by the root
    assert (np.abs(f64(rstd) - rstd64) <= rel * rstd64).all()
    assert (np.abs(f64(y) - y64) <= np.abs(y64) * (rel + 4 * U)[:, None] + h_err * np.abs(rstd64[:, None] * f64(w))).all()


@pytest.mark.parametrize("rows,cols", [(128, 128), (256, 384), (384, 1280), (250, 500), (1000, 900)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("blocks", [False, True])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_quantize_into_rows_on_lines(dev, rows, cols, dtype, blocks, fmt):
    F8 = torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2
    x = (normal(dev, rows, rows, cols) * torch.exp2(normal(dev, 2, rows, 1) * 4)).to(DT[dtype])
    q, q_t = (torch.full((n, -(-m // 128) * 128), 0x5A, dtype=torch.uint8, device=dev) for n, m in ((rows, cols), (cols, rows)))
    tall, wide = (-(-rows // 128), -(-cols // 128)) if blocks else (rows, cols)
    s, s_t = (torch.empty(-(-m // 512), n, 4, dtype=torch.uint8, device=dev) for n, m in ((tall, cols), (wide, rows)))
    reft.reft_quantize(x, q.view(F8)[:, :cols], s, q_t.view(F8)[:, :rows], s_t, blocks=blocks)
    for got, scales, value, m in ((q, s, f64(x), cols), (q_t, s_t, f64(x).T, rows)):
        want, e = step.quantize(np.ascontiguousarray(value), fmt, blocks)
        assert np.array_equal(scales.cpu().numpy(), step.words_of(e))
        assert np.array_equal(f64(got.view(F8)[:, :m].float()), want) and (got[:, m:] == 0x5A).all()
