"""GPU tests of the training step's operators: what should not matter - where rows lie and how far apart - changes no bit, and every
kernel that sizes and alignment choose between is compared with the definition."""
import pytest
import torch

import paper_2310_12670_amd as reft

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
