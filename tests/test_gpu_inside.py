"""GPU tests of the operators inside the sublayers: each against its definition in 64 bits, at the sizes, layouts, types and values where
it can go wrong.  Tolerances come from the formats: U is half a step of fp32 at one, a sum of n terms errs by at most n U of the sum
of their magnitudes, hardware's exponential and reciprocal by a step (2 U)."""
import numpy as np
import pytest
import torch

import paper_2310_12670_amd as reft
from oracle import step
from test_gpu_step import DT, F8, HALF, TINY, U, dev, f64, near_eight, normal, padded, scales_like, untouched  # noqa: F401

pytestmark = pytest.mark.gpu

EPS = 1e-5


# ------------------------------------------------------------------------------------------------
# heads
# ------------------------------------------------------------------------------------------------
class Heads:
    """[rows][heads][cols] somewhere in memory that holds 0x5A around it.  layout: "token" (a row's heads one after the other), "head" (a head's
    rows), "wide" (heads and rows with gaps, off alignment)."""

    def __init__(self, dev, rows, heads, cols, dtype, layout, fill=None):
        self.size = torch.empty((), dtype=dtype).element_size()
        row, head, lead = {"token": (heads * cols, cols, 0), "head": (cols, rows * cols, 0),
                           "wide": (heads * (cols + 3) + 5, cols + 3, 1)}[layout]
        span = lead + (rows - 1) * row + (heads - 1) * head + cols
        self.raw = torch.full(((span + 64) * self.size,), 0x5A, dtype=torch.uint8, device=dev)
        self.t = torch.as_strided(self.raw.view(dtype), (rows, heads, cols), (row, head, 1), lead)
        if fill is not None:
            self.t.copy_(fill)

    def alone_written(self):
        flags = torch.zeros(self.raw.numel() // self.size, dtype=torch.bool, device=self.raw.device)
        torch.as_strided(flags, self.t.shape, self.t.stride(), self.t.storage_offset()).fill_(True)
        return bool((self.raw[~flags.repeat_interleave(self.size)] == 0x5A).all())


def angles(dev, rows, pairs, seed=0, far=4000):
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed + 77)
    positions = torch.randint(0, far, (rows,), device=dev, generator=gen)
    return positions, (10000.0 ** (-torch.arange(pairs, device=dev, dtype=torch.float64) / max(1, pairs))).float()


def partners(x, pairs, adjacent):
    """Each column's partner's value, itself behind the pairs."""
    out = x.copy()
    if adjacent:
        out[..., 0:2 * pairs:2], out[..., 1:2 * pairs:2] = x[..., 1:2 * pairs:2], x[..., 0:2 * pairs:2]
    else:
        out[..., :pairs], out[..., pairs:2 * pairs] = x[..., pairs:2 * pairs], x[..., :pairs]
    return out


# 1 / rms: eight squares a lane and up to six additions, half of that through the root; mean, addition, root, quotient
RSTD = ((8 + 6) / 2 + 4) * U
# of each of a result's two terms: weight, 1 / rms and cosine multiplied in (one each), the cosine's own error of 2^-22, the addition
TURN = (3 + 4 + 1) * U


def check_forward(got, x, w, positions, freqs, adjacent, dtype):
    x, w = f64(x), f64(w)
    want = step.heads_forward(x, w, f64(positions), f64(freqs), EPS, adjacent)
    z = np.abs(x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * w)
    err = (RSTD + TURN) * (z + partners(z, len(freqs), adjacent)) + HALF[dtype] * 1.01 * np.abs(want) + (TINY if dtype == "f16" else 0)
    assert (np.abs(f64(got) - want) <= err).all()


def check_backward(dx, dw, dout, x, w, positions, freqs, adjacent, dtype):
    dout, x, w = f64(dout), f64(x), f64(w)
    n = len(freqs)
    want, want_w = step.heads_backward(dout, x, w, f64(positions), f64(freqs), EPS, adjacent)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
    xhat, u = x * r, step.turned(dout, f64(positions), f64(freqs), adjacent, back=True)
    u_err = (1 + 4 + 1) * U * (np.abs(dout) + partners(np.abs(dout), n, adjacent))        # product, cosine, addition
    # the mean of three factors: their roundings, eight a lane and six additions; the statistics twice
    dot = (u * w * xhat).mean(-1, keepdims=True)
    dot_err = (np.abs(w * xhat) * u_err).mean(-1, keepdims=True) + (8 + 6 + 4) * U * np.abs(u * w * xhat).mean(-1, keepdims=True) + \
        2 * RSTD * np.abs(dot)
    if dx is not None:
        err = r * (np.abs(w) * u_err + 3 * U * np.abs(u * w) + np.abs(xhat) * (dot_err + (RSTD + 4 * U) * np.abs(dot))) + (RSTD + 2 * U) * np.abs(want)
        assert (np.abs(f64(dx) - want) <= err + HALF[dtype] * 1.01 * np.abs(want) + (TINY if dtype == "f16" else 0)).all()
    if dw is not None:
        terms = np.abs(u * xhat).sum((0, 1))
        err = (u_err * np.abs(xhat)).sum((0, 1)) + (RSTD + (x.shape[0] * x.shape[1] + 40) * U) * terms
        assert (np.abs(f64(dw) - want_w) <= err).all()


def check_heads(dev, rows, q_heads, k_heads, cols, pairs, adjacent, dtype, weight, layout, out_layout):
    T, W = DT[dtype], DT[weight] if weight else None
    sides = []
    positions, freqs = angles(dev, rows, pairs, rows)
    for seed, heads in ((1, q_heads), (2, k_heads)):
        if not heads:
            sides.append(None)
            continue
        x = Heads(dev, rows, heads, cols, T, layout, normal(dev, seed, rows, heads, cols) * torch.exp(normal(dev, seed + 9, rows, heads, 1)))
        w = (1 + normal(dev, seed + 20, cols, std=0.3)).to(W) if weight else None
        sides.append((x, w, w if weight else torch.ones(cols, device=dev), Heads(dev, rows, heads, cols, T, out_layout),
                      Heads(dev, rows, heads, cols, T, out_layout, normal(dev, seed + 30, rows, heads, cols)),
                      Heads(dev, rows, heads, cols, T, layout)))
    q, k = sides
    nothing = (None,) * 6
    xk, wk, _, ok, dok, dk = k or nothing
    t = lambda h: None if h is None else h.t                                             # noqa: E731
    reft.reft_heads_forward(q[0].t, t(xk), q[1], wk, positions, freqs, EPS, q[3].t, t(ok), adjacent=adjacent)
    dw = torch.full((2, cols), float("nan"), device=dev)
    ws = torch.empty(reft.reft_heads_backward_workspace(rows, q_heads, k_heads, cols), dtype=torch.uint8, device=dev)
    rest = dict(adjacent=adjacent, workspace=ws)
    args = (q[4].t, t(dok), q[0].t, t(xk), q[1], wk, positions, freqs, EPS)
    reft.reft_heads_backward(*args, dq=q[5].t, dk=t(dk), dq_weight=dw[0], dk_weight=dw[1] if k else None, **rest)
    for side, g in ((q, dw[0]), (k, dw[1])):
        if side is None:
            continue
        x, w, w1, out, dout, dx = side
        check_forward(out.t, x.t, w1, positions, freqs, adjacent, dtype)
        check_backward(dx.t, g, dout.t, x.t, w1, positions, freqs, adjacent, dtype)
        assert out.alone_written() and dx.alone_written()
    # each result alone, and in the place of what it is computed from: the same bits
    alone = torch.empty(2, cols, device=dev)
    reft.reft_heads_backward(*args, dq_weight=alone[0], **rest)
    assert torch.equal(alone[0], dw[0])
    if k:
        reft.reft_heads_backward(*args, dk_weight=alone[1], **rest)
        assert torch.equal(alone[1], dw[1])
        here = Heads(dev, rows, k_heads, cols, T, layout)
        reft.reft_heads_backward(*args, dk=here.t, adjacent=adjacent)
        assert torch.equal(here.t, dk.t)
    kept = [h.t.clone() for h in (q[5], dk) if h is not None]
    reft.reft_heads_backward(*args, dq=q[4].t, dk=t(dok), dq_weight=alone[0], **rest)
    assert all(torch.equal(h.t, x) for h, x in zip((q[4], dok), kept)) and torch.equal(alone[0], dw[0])
    reft.reft_heads_forward(q[0].t, t(xk), q[1], wk, positions, freqs, EPS, q[0].t, t(xk), adjacent=adjacent)
    assert torch.equal(q[0].t, q[3].t) and (not k or torch.equal(xk.t, ok.t))


SHAPES = [(1, 1, 0, 1, 0), (1, 64, 8, 128, 64), (3, 2, 1, 7, 3), (5, 3, 3, 64, 32), (2, 5, 1, 80, 16), (37, 9, 3, 80, 10), (4, 2, 2, 128, 32),
          (19, 4, 4, 96, 48), (6, 3, 1, 129, 64), (3, 7, 1, 192, 96), (2, 2, 2, 256, 128), (2, 3, 2, 260, 65), (2, 2, 1, 511, 255),
          (3, 1, 1, 512, 256), (700, 12, 4, 64, 32), (1, 200, 3, 8, 4), (2, 1, 1, 16, 8), (9, 4, 2, 72, 36)]


@pytest.mark.parametrize("rows,q_heads,k_heads,cols,pairs", SHAPES)
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dtype,weight,layout,out_layout", [("bf16", "bf16", "token", "head"), ("f16", "f32", "wide", "token"),
                                                            ("f32", "f32", "head", "wide"), ("bf16", None, "wide", "wide")])
def test_heads(dev, rows, q_heads, k_heads, cols, pairs, adjacent, dtype, weight, layout, out_layout):  # noqa: F811
    check_heads(dev, rows, q_heads, k_heads, cols, pairs, adjacent, dtype, weight, layout, out_layout)


@pytest.mark.parametrize("rows,q_heads,k_heads,cols,pairs", [(4096, 8, 1, 128, 64), (5000, 3, 3, 64, 16), (9001, 1, 1, 40, 20), (2500, 32, 8, 80, 40)])
@pytest.mark.parametrize("adjacent", [False, True])
def test_heads_of_many_rows(dev, rows, q_heads, k_heads, cols, pairs, adjacent):  # noqa: F811
    check_heads(dev, rows, q_heads, k_heads, cols, pairs, adjacent, "bf16", "bf16", "token", "head")


def test_one_weight_and_no_pairs(dev):  # noqa: F811
    x, w = normal(dev, 1, 5, 3, 40), normal(dev, 2, 40)
    out, other = torch.empty_like(x), torch.empty_like(x)
    reft.reft_heads_forward(x, x, None, w, None, None, EPS, out, other)
    nothing = torch.empty(0, device=dev)
    for got, weight in ((out, torch.ones(40, device=dev)), (other, w)):
        check_forward(got, x, weight, torch.zeros(5), nothing.cpu(), False, "f32")
    again = torch.empty_like(x)
    reft.reft_heads_forward(x, None, w, None, None, nothing, EPS, again)
    assert torch.equal(again, other)


def test_angles_of_far_positions(dev):  # noqa: F811
    """To 2^-22 of the exact sine and cosine, wherever the position: every quarter turn, both signs."""
    freqs = torch.cat((torch.ones(1), torch.rand(31, generator=torch.Generator().manual_seed(3)))).to(dev)
    positions = torch.tensor([0, 1, -1, 2, 3, 4, 5, 6, 7, 22, 355, 1000003, -1000003, 2 ** 24 + 1, 2 ** 29 - 1, -(2 ** 29) + 1, 245850922],
                             device=dev)
    x = torch.zeros(positions.numel(), 1, 64, device=dev)
    x[..., :32] = 1                                          # pairs (1, 0): norm 2^0.5, results sine and cosine times that
    out = torch.empty_like(x)
    reft.reft_heads_forward(x, None, None, None, positions, freqs, 0.0, out)
    angle = positions.cpu().numpy().astype(np.longdouble)[:, None] * f64(freqs).astype(np.longdouble)
    want = np.concatenate([np.cos(angle), np.sin(angle)], -1) * np.sqrt(np.longdouble(2))
    assert np.abs(f64(out)[:, 0] - want).max() <= np.sqrt(2) * (2.0 ** -22 + RSTD + 3 * U)


def test_heads_of_zeros_infinities_and_nan(dev):  # noqa: F811
    rows, heads, cols = 5, 6, 128
    x = normal(dev, 1, rows, heads, cols)
    positions, freqs = angles(dev, rows, 64)
    x[0, 0], x[1, 1, 3], x[2, 2, 70] = 0, float("nan"), float("inf")
    x[3, 3], x[4, 4] = 1e-30, 1e30
    out, dx = torch.empty_like(x), torch.empty_like(x)
    dout = normal(dev, 2, rows, heads, cols)
    reft.reft_heads_forward(x, None, None, None, positions, freqs, EPS, out)
    reft.reft_heads_backward(dout, None, x, None, None, None, positions, freqs, EPS, dq=dx)
    assert not out[0, 0].any() and torch.isnan(out[1, 1]).all() and torch.isnan(out[2, 2, [6, 70]]).all()
    assert not out[4, 4].any() and torch.isfinite(dx[0, 0]).all() and torch.isnan(dx[1, 1]).all()
    fine = torch.ones(rows, heads, dtype=torch.bool, device=dev)
    fine[1, 1] = fine[2, 2] = fine[4, 4] = False
    clean = torch.where(fine[..., None], x, torch.ones_like(x))
    again = torch.empty_like(x)
    reft.reft_heads_forward(clean, None, None, None, positions, freqs, EPS, again)
    assert torch.equal(out[fine], again[fine]) and torch.isfinite(out[fine]).all()
    reft.reft_heads_backward(dout, None, clean, None, None, None, positions, freqs, EPS, dq=again)
    assert torch.equal(dx[fine], again[fine]) and torch.isfinite(dx[fine]).all()


@pytest.mark.parametrize("adjacent", [False, True])
def test_heads_gradient_against_differences(dev, adjacent):  # noqa: F811
    """The slope of sum(out g) along random directions, from the forward kernel itself, in fp32."""
    rows, heads, cols, pairs = 4, 3, 32, 12
    x, w, g = normal(dev, 1, rows, heads, cols), 1 + normal(dev, 2, cols, std=0.2), normal(dev, 3, rows, heads, cols)
    positions, freqs = angles(dev, rows, pairs)
    dx, dw = torch.empty_like(x), torch.empty(cols, device=dev)
    ws = torch.empty(reft.reft_heads_backward_workspace(rows, heads, 0, cols), dtype=torch.uint8, device=dev)
    reft.reft_heads_backward(g, None, x, None, w, None, positions, freqs, EPS, adjacent=adjacent, dq=dx, dq_weight=dw, workspace=ws)
    t = 2.0 ** -7
    for at, grad in enumerate((dx, dw)):
        for k in range(4):
            to = normal(dev, 50 + 10 * at + k, *grad.shape)
            to /= to.norm()
            ends = []
            for sign in (t, -t):
                args = [x, w]
                args[at] = args[at] + sign * to
                out = torch.empty_like(x)
                reft.reft_heads_forward(args[0], None, args[1], None, positions, freqs, EPS, out, adjacent=adjacent)
                ends.append((f64(out) * f64(g)).sum())
            slope, want = (ends[0] - ends[1]) / (2 * t), (f64(grad) * f64(to)).sum()
            # the forward's rounding over 2 t: 384 values of order one, sqrt(384) * 6 U / (2 t) < 5e-4, three times that; the
            # cubic term, t^2 times a third derivative of order |g| = 20, over 6: 2e-4
            assert abs(slope - want) <= 1.8e-3


def test_heads_without_rows(dev):  # noqa: F811
    empty = torch.empty(0, 2, 40, device=dev)
    none = torch.empty(0, dtype=torch.int64, device=dev)
    freqs = torch.ones(4, device=dev)
    reft.reft_heads_forward(empty, empty, None, None, none, freqs, EPS, empty, empty)
    dw = torch.full((2, 40), 3.0, device=dev)
    reft.reft_heads_backward(empty, empty, empty, empty, None, None, none, freqs, EPS, dq_weight=dw[0], dk_weight=dw[1],
                             workspace=torch.empty(16, dtype=torch.uint8, device=dev))
    assert not dw.any()


def test_inputs_that_share_elements(dev):  # noqa: F811
    """One head expanded to all, and one row: as if it had been copied."""
    one = normal(dev, 1, 7, 1, 64, dtype=torch.bfloat16)
    positions, freqs = angles(dev, 7, 32)
    for x in (one.expand(7, 5, 64), one[:1].expand(7, 5, 64)):
        a, b = torch.empty(7, 5, 64, dtype=torch.bfloat16, device=dev), torch.empty(7, 5, 64, dtype=torch.bfloat16, device=dev)
        reft.reft_heads_forward(x, None, None, None, positions, freqs, EPS, a)
        reft.reft_heads_forward(x.contiguous(), None, None, None, positions, freqs, EPS, b)
        assert torch.equal(a, b)
        reft.reft_heads_backward(x, None, x, None, None, None, positions, freqs, EPS, dq=a)
        reft.reft_heads_backward(x.contiguous(), None, x.contiguous(), None, None, None, positions, freqs, EPS, dq=b)
        assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------
# gate
# ------------------------------------------------------------------------------------------------
def act_err(g, kind):
    """(error of act(g), error of its slope): the exponent is rounded (its value in U of the result), then a step each for the exponential
    and the reciprocal, and a rounding for each operation.  What is below 2^-126 is lost."""
    a, slope = step.act(g, kind)
    low = 2.0 ** -125
    if kind == "relu2":
        return U * a + low, 0 * a
    if kind == "gelu":
        # the exponent g^2 / 2 log2(e) is rounded as the square and as the product, and log2(e) itself is off by 0.23 U: each rounding
        # of U of the exponent is one of g^2 / 2 U of the result
        expo = 2.25 * g * g / 2
        # the tail beyond |g|: its exponential, the polynomial's fit (9.4e-8) and Horner's roundings (eight, of terms that
        # add up to less than twice the result), and what the rounding of 1 / (1 + 0.23 |g|), 3 U, makes of that (at most 4 times)
        tail = step._erfc(np.abs(g) / np.sqrt(2)) / 2
        p = np.where(g < 0, tail, 1 - tail)
        p_err = tail * (expo + 2 + 2 + 16 + 12 + 3) * U + U * p
        bell = np.abs(g) * np.exp(-g * g / 2) / np.sqrt(2 * np.pi)
        return np.abs(g) * p_err + U * np.abs(a) + low * (1 + np.abs(g)), p_err + bell * (expo + 6) * U + U * (np.abs(slope) + bell) + low * (1 + np.abs(g))
    if kind == "silu":
        arg, inner = np.abs(g), np.abs(g)
        p = 1 / (1 + np.exp(-g))
        arg_err = 2 * arg
    else:
        c = 2 * np.sqrt(2 / np.pi)
        arg = np.abs(c * (g + 0.044715 * g ** 3))
        inner = np.abs(g) * c * (1 + 0.134145 * np.minimum(g * g, 1e4))
        p = 1 / (1 + np.exp(-c * (g + 0.044715 * g ** 3)))
        arg_err = 6 * arg
    p_err = p * ((1 - p) * (arg_err + 2) + 3) * U + low
    second = inner * p * (1 - p)
    s_err = p_err + inner * (p_err * (1 - p) + p * (p_err + U)) + 8 * U * second + U * np.abs(slope)
    return np.abs(g) * p_err + U * np.abs(a) + low, s_err + low


KINDS = ["silu", "gelu", "gelu_tanh", "relu2"]
SIZES = [(1, 1), (1, 28672), (3, 7), (5, 128), (129, 257), (300, 1000), (17, 1537), (130, 24), (256, 512), (1001, 136)]


def eight(dev, rows, cols, fmt, pad=0, lead=0):
    raw, q = padded(dev, rows, cols, F8[fmt], pad, lead)
    return raw, (q, scales_like(dev, rows, cols))


def exactly(pair, value, fmt):
    want, e = step.quantize(np.ascontiguousarray(value), fmt, False)
    return np.array_equal(pair[1].cpu().numpy(), step.words_of(e)) and np.array_equal(f64(pair[0].float()), want, equal_nan=True)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype,gated,fmt,kept,pad,lead", [("bf16", True, "e4m3", "e4m3", 0, 0), ("f16", True, "e5m2", "e4m3", 5, 3),
                                                           ("f32", False, "e4m3", "e5m2", 3, 1), ("f32", True, "e4m3", "e4m3", 0, 0)])
def test_gate_forward(dev, rows, cols, kind, dtype, gated, fmt, kept, pad, lead):  # noqa: F811
    T = DT[dtype]
    _, g = padded(dev, rows, cols, T, pad, lead, normal(dev, rows + cols, rows, cols, std=3.0))
    u = padded(dev, rows, cols, T, pad + 1, lead, normal(dev, cols, rows, cols))[1] if gated else None
    raw_y, y = padded(dev, rows, cols, T, pad + 2, lead)
    (raw_8, y8), (raw_g, g8), (raw_u, u8) = (eight(dev, rows, cols, f, pad + 3, lead) for f in (fmt, kept, kept))
    reft.reft_gate_forward(g, u, kind, y=y, y8=y8, g8=g8, u8=u8 if gated else None)
    a, _ = step.act(f64(g), kind)
    by = np.abs(f64(u)) if gated else 1.0
    want = a * f64(u) if gated else a
    err = act_err(f64(g), kind)[0] * by + U * np.abs(want)
    assert (np.abs(f64(y) - want) <= err + HALF[dtype] * 1.01 * np.abs(want) + (TINY if dtype == "f16" else 0)).all()
    near_eight(*y8, want, err, fmt, cols)
    assert exactly(g8, f64(g), kept) and untouched(raw_y, y) and untouched(raw_8, y8[0]) and untouched(raw_g, g8[0])
    assert not gated or (exactly(u8, f64(u), kept) and untouched(raw_u, u8[0]))
    # each output alone, and y in the place of either input
    for name, pair in (("y8", y8), ("g8", g8), ("u8", u8 if gated else None)):
        if pair is not None:
            alone = eight(dev, rows, cols, fmt if name == "y8" else kept)[1]
            reft.reft_gate_forward(g, u, kind, **{name: alone})
            assert torch.equal(alone[0].view(torch.uint8), pair[0].view(torch.uint8)) and torch.equal(alone[1], pair[1])
    for over in (u, g):
        if over is not None:
            keep = over.clone()
            reft.reft_gate_forward(g, u, reft.binding._ACTS[kind], y=over)
            assert torch.equal(over, y)
            over.copy_(keep)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype,gated,grad,kept,pad,lead", [("bf16", True, "e4m3", "e4m3", 0, 0), ("f16", True, "e5m2", "e4m3", 5, 3),
                                                            ("f32", False, "e4m3", "e5m2", 3, 1)])
def test_gate_backward(dev, rows, cols, kind, dtype, gated, grad, kept, pad, lead):  # noqa: F811
    T = DT[dtype]
    _, dy = padded(dev, rows, cols, T, pad, lead, normal(dev, 7, rows, cols) * torch.exp(normal(dev, 8, rows, 1)))
    inputs = []
    for seed, std in ((1, 2.0), (2, 1.0)):
        value = normal(dev, seed + rows, rows, cols, std=std)
        pair = eight(dev, rows, cols, kept, pad + 1, lead)[1]
        reft.reft_quantize(value, *pair)
        inputs.append((pair, step.scaled(f64(pair[0].float()), pair[1].cpu().numpy(), False)))
    (g8, g), (u8, u) = inputs
    if not gated:
        u8 = u = None
    dg, du, y = step.gate_backward(f64(dy), g, u, kind)
    a_err, s_err = act_err(g, kind)
    by = np.abs(u) if gated else 1.0
    want = {"dg": (dg, np.abs(f64(dy)) * by * s_err + 3 * U * np.abs(dg)), "y": (y, by * a_err + U * np.abs(y))}
    if gated:
        want["du"] = (du, np.abs(f64(dy)) * a_err + U * np.abs(du))
    outs, raws = {}, []
    for name in want:
        if name != "y":
            raw, outs[name] = padded(dev, rows, cols, T, pad + 2, lead)
            raws.append((raw, outs[name]))
            raw, outs[name + "8"] = eight(dev, rows, cols, grad, pad + 3, lead)
            raws.append((raw, outs[name + "8"][0]))
        raw, outs[name + "8_t"] = eight(dev, cols, rows, grad if name != "y" else "e4m3", pad + 1, lead)
        raws.append((raw, outs[name + "8_t"][0]))
    reft.reft_gate_backward(dy, g8, u8, kind, **outs)
    for name, (value, err) in want.items():
        if name != "y":
            assert (np.abs(f64(outs[name]) - value) <= err + HALF[dtype] * 1.01 * np.abs(value) + (TINY if dtype == "f16" else 0)).all()
            near_eight(*outs[name + "8"], value, err, grad, cols)
        near_eight(*outs[name + "8_t"], np.ascontiguousarray(value.T), np.ascontiguousarray(err.T), grad if name != "y" else "e4m3", rows)
    assert all(untouched(raw, view) for raw, view in raws)
    # each output alone, and the gradients in the place of dy
    for name, out in outs.items():
        if isinstance(out, tuple):
            alone = eight(dev, *out[0].shape, {v: k for k, v in F8.items()}[out[0].dtype])[1]
            reft.reft_gate_backward(dy, g8, u8, kind, **{name: alone})
            assert torch.equal(alone[0].view(torch.uint8), out[0].view(torch.uint8)) and torch.equal(alone[1], out[1])
    for name in ("dg", "du"):
        if name in outs:
            keep = dy.clone()
            reft.reft_gate_backward(dy, g8, u8, kind, **{name: dy})
            assert torch.equal(dy, outs[name])
            dy.copy_(keep)


@pytest.mark.parametrize("kind", KINDS)
def test_gate_of_infinities_and_nan(dev, kind):  # noqa: F811
    """A value that is no number takes its block of 128 along, in rows and in columns, and nothing else."""
    rows, cols = 260, 700
    g, u = normal(dev, 1, rows, cols), normal(dev, 2, rows, cols)
    g[3, 5], u[130, 300], g[259, 699] = float("nan"), float("nan"), float("inf")
    y, y8, g8, u8 = torch.empty_like(g), *(eight(dev, rows, cols, "e4m3")[1] for _ in range(3))
    reft.reft_gate_forward(g, u, kind, y=y, y8=y8, g8=g8, u8=u8)
    assert exactly(g8, f64(g), "e4m3") and exactly(u8, f64(u), "e4m3")
    off = torch.zeros(rows, cols, dtype=torch.bool, device=dev)
    off[3, 5] = off[130, 300] = off[259, 699] = True
    assert torch.isnan(y[3, 5]) and torch.isnan(y[130, 300]) and torch.isinf(y[259, 699]) and torch.isfinite(y[~off]).all()
    bad = torch.zeros(rows, cols, dtype=torch.bool, device=dev)
    bad[3, :128] = bad[130, 256:384] = bad[259, 640:] = True
    assert torch.equal(torch.isnan(y8[0].float()), bad) and torch.equal(torch.isnan(g8[0].float()) | torch.isnan(u8[0].float()), bad)
    dy = normal(dev, 3, rows, cols)
    dg, t8 = torch.empty_like(g), eight(dev, cols, rows, "e4m3")[1]
    reft.reft_gate_backward(dy, g8, u8, kind, dg=dg, dg8_t=t8)
    assert torch.equal(torch.isnan(dg), bad)
    column = torch.cat([bad[i:i + 128].any(0).expand(min(128, rows - i), cols) for i in range(0, rows, 128)])
    assert torch.equal(torch.isnan(t8[0].float()).t(), column)


@pytest.mark.parametrize("kind", KINDS)
def test_gate_of_large_values(dev, kind):  # noqa: F811
    """Far from zero the activation is its input or nothing, and its slope one or nothing (but the square's)."""
    g = torch.tensor([[-3e38, -1e19, -1e5, -200.0, -0.0, 0.0, 200.0, 1e5, 1e18]], device=dev)
    y = torch.empty_like(g)
    reft.reft_gate_forward(g, None, kind, y=y)
    above = torch.where(g > 0, g, torch.zeros_like(g))
    assert torch.equal(y, above.square() if kind == "relu2" else above)
    g8 = eight(dev, 1, 9, "e5m2")[1]
    g8[0].view(torch.uint8).copy_(torch.tensor([[0xFB, 0xF0, 0xE0, 0xD8, 0x80, 0x00, 0x58, 0x60, 0x7B]], dtype=torch.uint8, device=dev))
    for byte in (127, 237, 1):
        g8[1].fill_(byte)
        value = g8[0].float() * 2.0 ** (byte - 127)
        dg, dy = torch.empty_like(g), torch.ones_like(g)
        reft.reft_gate_backward(dy, g8, None, kind, dg=dg)
        _, slope = step.act(np.clip(f64(value), -600, 600), kind)
        want = 2 * torch.clamp(value, min=0) if kind == "relu2" else torch.from_numpy(slope).to(dev).float()
        assert torch.allclose(dg, want, rtol=1e-5, atol=1e-6), (byte, dg, want)


def test_gradient_of_the_gate_against_differences(dev):  # noqa: F811
    """With values that 8 bits hold, the forward kernel's differences are the backward kernel's slope."""
    g, u = (normal(dev, s, 16, 130).to(F8["e4m3"]).float().clamp(-3.5, 3.5) for s in (1, 2))
    dy = normal(dev, 3, 16, 130)
    for kind in ("silu", "gelu", "gelu_tanh"):
        kept = [eight(dev, 16, 130, "e4m3")[1] for _ in range(2)]
        for pair, v in zip(kept, (g, u)):
            pair[0].copy_(v.to(F8["e4m3"]))
            pair[1].fill_(127)
        dg, du = torch.empty_like(g), torch.empty_like(g)
        reft.reft_gate_backward(dy, *kept, kind, dg=dg, du=du)
        t = 2.0 ** -6
        for at, grad in ((0, dg), (1, du)):
            ends = []
            for sign in (t, -t):
                x = [g, u]
                x[at] = x[at] + sign
                y = torch.empty_like(g)
                reft.reft_gate_forward(*x, kind, y=y)
                ends.append(f64(y))
            slope = (ends[0] - ends[1]) / (2 * t) * f64(dy)
            # rounding: |y| (|g| + 8) U / t <= 12.3 * 12 * U / t < 6e-4 ; the cubic term: t^2 / 6 times a third derivative below 2
            # times |u|: 3e-4; both times |dy|
            assert (np.abs(slope - f64(grad)) <= 9e-4 * np.abs(f64(dy)) + 1e-6).all()


# ------------------------------------------------------------------------------------------------
# transpose
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 700), (700, 1), (5, 127), (128, 128), (129, 257), (300, 1000), (17, 1537), (1000, 24), (520, 384)])
@pytest.mark.parametrize("fmt,to", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("pad,lead", [(0, 0), (3, 5)])
def test_transpose(dev, rows, cols, fmt, to, pad, lead):  # noqa: F811
    value = normal(dev, rows, rows, cols) * torch.exp2(normal(dev, 2, rows, 1) * 4)
    value[:, : cols // 3] *= 2.0 ** -30
    _, x8 = eight(dev, rows, cols, fmt, pad, lead)
    reft.reft_quantize(value, *x8)
    raw, t8 = eight(dev, cols, rows, to, pad + 2, lead)
    reft.reft_transpose(*x8, *t8)
    want, e = step.transpose(f64(x8[0].float()), x8[1].cpu().numpy(), to)
    assert np.array_equal(t8[1].cpu().numpy(), step.words_of(e)) and np.array_equal(f64(t8[0].float()), want)
    assert untouched(raw, t8[0])


def test_transpose_of_every_value(dev):  # noqa: F811
    """All bytes, NaN and e5m2's infinities among them, with scales at both ends."""
    for fmt in F8:
        for byte in (0, 1, 2, 127, 230, 253, 254, 255):
            q = torch.arange(256, dtype=torch.uint8, device=dev).view(2, 128).view(F8[fmt])
            s = torch.full((1, 2, 4), byte, dtype=torch.uint8, device=dev)
            for to in F8:
                t8 = eight(dev, 128, 2, to)[1]
                reft.reft_transpose(q, s, *t8)
                value = q.double() * (float("nan") if byte == 255 else 2.0 ** (byte - 127))
                value = np.where(np.abs(f64(value)) >= 2.0 ** 128, np.inf, f64(value))      # the widened value is fp32
                assert exactly(t8, value.T, to), (fmt, byte, to)


# ------------------------------------------------------------------------------------------------
# all
# ------------------------------------------------------------------------------------------------
def test_rows_further_apart_than_32_bits_count(dev):  # noqa: F811
    """Three rows of 2^32 bytes and more between them, through each operator's strides."""
    ld, cols = (1 << 31) + 24, 300
    big = torch.empty(2 * ld + 2 * cols, dtype=torch.bfloat16, device=dev)
    far = torch.as_strided(big, (3, 2, 150), (ld, 150, 1))
    near = normal(dev, 1, 3, 2, 150, dtype=torch.bfloat16)
    far.copy_(near)
    positions, freqs = angles(dev, 3, 75)
    a, b = torch.empty_like(near), torch.empty_like(near)
    reft.reft_heads_forward(far, far, None, None, positions, freqs, EPS, a, b)
    c, d = torch.empty_like(near), torch.empty_like(near)
    reft.reft_heads_forward(near, near, None, None, positions, freqs, EPS, c, d)
    assert torch.equal(a, c) and torch.equal(b, d)
    reft.reft_heads_backward(far, None, far, None, None, None, positions, freqs, EPS, dq=far)
    reft.reft_heads_backward(near, None, near, None, None, None, positions, freqs, EPS, dq=c)
    assert torch.equal(far, c)
    heads = torch.as_strided(big, (2, 3, 150), (150, ld, 1))                 # far heads
    heads.copy_(near.transpose(0, 1))
    reft.reft_heads_forward(heads, None, None, None, positions[:2], freqs, EPS, heads)
    reft.reft_heads_forward(near.transpose(0, 1).contiguous(), None, None, None, positions[:2], freqs, EPS, c.view(2, 3, 150))
    assert torch.equal(heads, c.view(2, 3, 150))
    x = torch.as_strided(big, (3, cols), (ld, 1))
    x.copy_(near.view(3, cols))
    near = near.view(3, cols)
    y, y8 = torch.empty(2, 3, cols, dtype=torch.bfloat16, device=dev), [eight(dev, 3, cols, "e4m3")[1] for _ in range(2)]
    reft.reft_gate_forward(x, x, "silu", y=y[0], g8=y8[0])
    reft.reft_gate_forward(near, near, "silu", y=y[1], g8=y8[1])
    assert torch.equal(y[0], y[1]) and torch.equal(y8[0][0].view(torch.uint8), y8[1][0].view(torch.uint8))
    q = torch.as_strided(big.view(torch.uint8).view(F8["e4m3"]), (3, cols), (2 * ld, 1))
    q.view(torch.uint8).copy_(y8[1][0].view(torch.uint8))
    t8 = [eight(dev, cols, 3, "e4m3")[1] for _ in range(4)]
    reft.reft_transpose(q, y8[1][1], *t8[0])
    reft.reft_transpose(*y8[1], *t8[1])
    reft.reft_gate_backward(near, (q, y8[1][1]), None, "gelu", dg=y[0], dg8_t=t8[2])
    reft.reft_gate_backward(near, y8[1], None, "gelu", dg=y[1], dg8_t=t8[3])
    assert torch.equal(y[0], y[1])
    for i in (0, 2):
        assert torch.equal(t8[i][0].view(torch.uint8), t8[i + 1][0].view(torch.uint8)) and torch.equal(t8[i][1], t8[i + 1][1])


class Layer:
    """A feed-forward and its queries and keys in 8 bits, forward and backward, by the library: weights [width -> inner] for g and u, [inner ->
    width] down, [width -> 4 heads of 64] for queries, [width -> 2 heads] for keys.  All room is made once."""

    def __init__(self, dev, rows, width, inner, seed=0):
        self.rows, self.width, self.inner, self.dev = rows, width, inner, dev
        bf16 = torch.bfloat16
        make = lambda s, *shape: normal(dev, seed + s, *shape, std=shape[1] ** -0.5, dtype=bf16)     # noqa: E731
        self.w = {"g": make(1, inner, width), "u": make(2, inner, width), "d": make(3, width, inner), "q": make(4, 256, width),
                  "k": make(5, 128, width)}
        self.x = normal(dev, seed + 6, rows, width, dtype=bf16)
        self.dout, self.dq_out, self.dk_out = (normal(dev, seed + 7 + i, rows, n, dtype=bf16) for i, n in enumerate((width, 256, 128)))
        self.norms = [(1 + normal(dev, seed + 20 + i, n, std=0.1)).to(bf16) for i, n in enumerate((width, 64, 64))]
        self.positions, self.freqs = angles(dev, rows, 32)
        self.room = {}
        self.scratch = torch.empty(1 << 24, dtype=torch.uint8, device=dev)

    def eight(self, name, rows, cols, blocks=False):
        if name not in self.room:
            q = torch.empty(rows, -(-cols // 16) * 16, dtype=torch.uint8, device=self.dev).view(F8["e4m3"])[:, :cols]
            self.room[name] = (q, torch.empty(-(-cols // 512), -(-rows // 128) if blocks else rows, 4, dtype=torch.uint8, device=self.dev))
        return self.room[name]

    def wide(self, name, *shape, dtype=torch.bfloat16):
        if name not in self.room:
            self.room[name] = torch.empty(*shape, dtype=dtype, device=self.dev)
        return self.room[name]

    def product(self, name, a, b, dtype=torch.bfloat16, blocks=False, stream=None):
        c = self.wide(name, a[0].shape[0], b[0].shape[0], dtype=dtype)
        reft.reft_product(*a, *b, c, self.scratch, b_blocks=blocks, stream=stream)
        return c

    def run(self, stream=None):
        R, W, N, s = self.rows, self.width, self.inner, dict(stream=stream)
        w, wt = {}, {}
        for name, v in self.w.items():
            w[name], wt[name] = self.eight("w" + name, *v.shape, True), self.eight("wt" + name, v.shape[1], v.shape[0], True)
            reft.reft_quantize(v, *w[name], *wt[name], blocks=True, **s)
        n8 = self.eight("n8", R, W)
        reft.reft_norm_forward(self.x, None, self.norms[0], EPS, q=n8[0], scales=n8[1], **s)
        q, k = (self.product(name, n8, w[name], blocks=True, **s).view(R, -1, 64) for name in "qk")
        qo, ko = self.wide("qo", 4, R, 64).transpose(0, 1), self.wide("ko", 2, R, 64).transpose(0, 1)
        reft.reft_heads_forward(q, k, *self.norms[1:], self.positions, self.freqs, EPS, qo, ko, **s)
        g, u = (self.product(name, n8, w[name], blocks=True, **s) for name in "gu")
        y8, g8, u8 = (self.eight(name, R, N) for name in ("y8", "g8", "u8"))
        reft.reft_gate_forward(g, u, "silu", y8=y8, g8=g8, u8=u8, **s)
        out = self.product("out", y8, w["d"], blocks=True, **s)
        # backward
        d8, d8_t = self.eight("d8", R, W), self.eight("d8_t", W, R)
        reft.reft_quantize(self.dout, *d8, *d8_t, **s)
        dy = self.product("dy", d8, wt["d"], blocks=True, **s)
        grads = {name: self.eight(name, *((N, R) if name.endswith("_t") else (R, N))) for name in ("dg8", "du8", "dg8_t", "du8_t", "y8_t")}
        reft.reft_gate_backward(dy, g8, u8, "silu", **grads, **s)
        n8_t = self.eight("n8_t", W, R)
        reft.reft_transpose(*n8, *n8_t, **s)
        f32 = torch.float32
        got = {"q": qo, "k": ko, "out": out, "dwd": self.product("dwd", d8_t, grads["y8_t"], f32, **s),
               "dwg": self.product("dwg", grads["dg8_t"], n8_t, f32, **s), "dwu": self.product("dwu", grads["du8_t"], n8_t, f32, **s),
               "dng": self.product("dng", grads["dg8"], wt["g"], blocks=True, **s), "dnu": self.product("dnu", grads["du8"], wt["u"], blocks=True, **s)}
        dq, dk = self.wide("dq", R, 4, 64), self.wide("dk", R, 2, 64)
        dw = self.wide("dw", 2, 64, dtype=f32)
        reft.reft_heads_backward(self.dq_out.view(R, 4, 64), self.dk_out.view(R, 2, 64), q, k, *self.norms[1:], self.positions, self.freqs, EPS,
                                 dq=dq, dk=dk, dq_weight=dw[0], dk_weight=dw[1], workspace=self.scratch, **s)
        return got | {"dq": dq, "dk": dk, "dw": dw}

    def plain(self):
        """The same in 64 bits without any rounding between."""
        d = lambda t: f64(t)                                                               # noqa: E731
        w = {name: d(v) for name, v in self.w.items()}
        x = d(self.x)
        n = x / np.sqrt((x * x).mean(1, keepdims=True) + EPS) * d(self.norms[0])
        q, k = ((n @ w[name].T).reshape(self.rows, -1, 64) for name in "qk")
        rest = (d(self.positions), d(self.freqs), EPS, False)
        g, u = n @ w["g"].T, n @ w["u"].T
        y = step.act(g, "silu")[0] * u
        dout = d(self.dout)
        dg, du, _ = step.gate_backward(dout @ w["d"], g, u, "silu")
        got = {"q": step.heads_forward(q, d(self.norms[1]), *rest), "k": step.heads_forward(k, d(self.norms[2]), *rest), "out": y @ w["d"].T,
               "dwd": dout.T @ y, "dwg": dg.T @ n, "dwu": du.T @ n, "dng": dg @ w["g"], "dnu": du @ w["u"]}
        dq, dwq = step.heads_backward(d(self.dq_out).reshape(self.rows, 4, 64), q, d(self.norms[1]), *rest)
        dk, dwk = step.heads_backward(d(self.dk_out).reshape(self.rows, 2, 64), k, d(self.norms[2]), *rest)
        return got | {"dq": dq, "dk": dk, "dw": np.stack([dwq, dwk])}


def test_a_layer(dev):  # noqa: F811
    """The operators together, as a layer uses them, against the layer in 64 bits: 8 bits (e4m3) bring 2^-4 / sqrt(3) = 3.6 % root mean square
    at most into each operand, uncorrelated; a gradient of weights has gone through at most five such roundings on its longest way (weights,
    norm; g and u; dout and dy's product; dg; n) of which each product joins two: sqrt(8) 3.6 % = 10 %."""
    layer = Layer(dev, 500, 256, 648)
    got, want = layer.run(), layer.plain()
    for name, v in want.items():
        off = np.linalg.norm(f64(got[name]) - v) / np.linalg.norm(v)
        assert off <= 0.10, (name, off)


def test_the_same_bits_again_and_on_another_stream(dev):  # noqa: F811
    layer = Layer(dev, 700, 256, 648)
    first = {name: v.clone() for name, v in layer.run().items()}
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (None, s, s):
        for v in layer.room.values():
            for t in v if isinstance(v, tuple) else (v,):
                t.view(torch.uint8).fill_(0xFF)
        torch.cuda.synchronize()
        got = layer.run(stream)
        torch.cuda.synchronize()
        assert all(torch.equal(first[name].contiguous().view(torch.uint8), v.contiguous().view(torch.uint8)) for name, v in got.items())


def test_captured_and_replayed(dev):  # noqa: F811
    """One graph of a whole layer, replayed on new inputs between eager work; each replay as the eager call on the same inputs."""
    layer, eager = Layer(dev, 300, 256, 400), Layer(dev, 300, 256, 400)
    layer.run()
    torch.cuda.synchronize()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        got = layer.run(torch.cuda.current_stream())
    for seed in (1, 2, 3, 4):
        for a in (layer, eager):
            a.x.copy_(normal(dev, seed, 300, 256))
            a.dout.copy_(normal(dev, seed + 50, 300, 256))
            a.positions.add_(17)
        torch.cuda.synchronize()
        graph.replay()
        want = eager.run()
        torch.cuda.synchronize()
        assert all(torch.equal(got[name].contiguous().view(torch.uint8), v.contiguous().view(torch.uint8)) for name, v in want.items())


def test_two_streams_at_once(dev):  # noqa: F811
    """Two layers side by side, each with its own room: as one after the other."""
    a, b = Layer(dev, 600, 256, 648, 0), Layer(dev, 600, 256, 648, 100)
    want = [{name: v.clone() for name, v in layer.run().items()} for layer in (a, b)]
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        got = [layer.run(s) for layer, s in zip((a, b), streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(w[name], g[name]) for w, g in zip(want, got) for name in w)
