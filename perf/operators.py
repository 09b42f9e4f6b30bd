"""The operators of a training step whose speed is measured, over their range of sizes, types and directions.

A step at the boundary of a residual sublayer, in 8 bits: dropout of the sublayer's output, its addition to the
residual stream, root-mean-square norm, 8-bit copies of what the matrix cores multiply, and the products of the forward pass
and of both gradients.  After a restore such a step has to repeat to the same bits, so masks come from a counter that
the training state holds.  Operations, each through the public entry points:

  norm           reft_norm_forward: h = residual + dropout(x), 1 / rms(h), and the norm's output in the inputs' type or in 8 bits
  norm_back      reft_norm_backward: the gradients of residual, x and weight
  dropout        reft_dropout: forward or, on a gradient, backward
  quantize       reft_quantize: a matrix in 8 bits with a power of two for each 128 values or 128 x 128 block, and its transpose
  product        reft_product: C[M, N] = A[M, K] B[N, K]^T of 8-bit matrices with their scales

Scales are bytes [ceil(K / 512)][rows][4] (blocks 4 w to 4 w + 3 of a row in one word), exponents of two with bias 127; places behind the last
block hold 127 (one).  Masks: 16 bits for each element from Philox4x32-10 (Salmon et al., 2011), key = seed, counter = (column / 8, row,
offset).  An element is kept where its bits are at least t = round(65536 p), and kept ones are scaled by 65536 / (65536 - t).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 8, "e5m2": 15}             # the largest value of a format is 1.75 * 2 ** TOP
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
MOST_VALUES = 16384 * 11008               # of a drawn matrix
MOST_PRODUCT = 8192 * 28672 * 8192        # of a drawn product


def listed():
    return [
        # One token of a 70B-shaped decoder on its way into a product: the call's latency counts.
        dict(name="norm_token", op="norm", rows=1, cols=8192, dtype="bf16", residual="bf16", p=0.0, out="e4m3"),
        # A micro-batch of four sequences of 4096 tokens, 13B-shaped, in training: fp32 residual stream, dropout, 8-bit output.
        dict(name="norm_train", op="norm", rows=16384, cols=5120, dtype="bf16", residual="f32", p=0.1, out="e4m3"),
        # An odd number of tokens of an adapter's odd width, in half precision.
        dict(name="norm_back_odd", op="norm_back", rows=1001, cols=1155, dtype="f16", residual="f16", p=0.2),
        # The gradient of a norm of a 70B-shaped decoder for 16384 tokens.
        dict(name="norm_back_train", op="norm_back", rows=16384, cols=8192, dtype="bf16", residual="bf16", p=0.1),
        # A classifier head's dropout on a small batch.
        dict(name="dropout_small", op="dropout", rows=61, cols=1000, dtype="f32", p=0.5, pad=0),
        # Dropout behind the activation of a 7B-shaped feed-forward for 16384 tokens.
        dict(name="dropout_train", op="dropout", rows=16384, cols=11008, dtype="bf16", p=0.1, pad=0),
        # A gradient of an odd number of tokens, in both orders: for the product of the inputs' gradient and that of the weights'.
        dict(name="quantize_grad", op="quantize", rows=4099, cols=4096, dtype="bf16", blocks=False, format="e5m2", both=True),
        # A tensor-parallel share of a 70B-shaped up projection laid out anew after an optimizer step, for both directions.
        dict(name="quantize_weight", op="quantize", rows=3584, cols=8192, dtype="bf16", blocks=True, format="e4m3", both=True),
        # One token through a 7B-shaped up projection: the weights' bytes count.
        dict(name="product_token", op="product", M=1, N=11008, K=4096, a="e4m3", b="e4m3", blocks=True, out="bf16"),
        # A share of a 13B-shaped down projection (13824 / 8 inputs: 13 and a half blocks) for an odd number of tokens.
        dict(name="product_ragged", op="product", M=1001, N=5120, K=1728, a="e4m3", b="e4m3", blocks=True, out="bf16"),
        # The gradient of a 7B-shaped up projection's weights over 8192 tokens, summed up in fp32.
        dict(name="product_weights", op="product", M=11008, N=4096, K=8192, a="e5m2", b="e4m3", blocks=False, out="f32"),
        # A 70B-shaped up projection of 8192 tokens.
        dict(name="product_train", op="product", M=8192, N=28672, K=8192, a="e4m3", b="e4m3", blocks=True, out="bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_back", "norm_back", "dropout", "quantize", "product", "product", "product"])
    if op == "product":
        kind = rng.choice(["token", "any", "any", "long"])
        M = _log(rng, 1, 64) if kind == "token" else _log(rng, 64, 16384)
        N = _log(rng, 16, 28672)
        K = _log(rng, 16, 16384 if kind != "long" else 28672)
        if rng.random() < 0.5:              # widths of layers are mostly round
            N, K = max(16, N // 64 * 64), max(16, K // 64 * 64)
        while M * N * K > MOST_PRODUCT:
            M, N = max(1, M // 2), max(16, N * 3 // 4)
        return dict(op=op, M=M, N=N, K=K, a=rng.choice(["e4m3", "e4m3", "e5m2"]), b=rng.choice(["e4m3", "e4m3", "e5m2"]),
                    blocks=rng.random() < 0.6, out=rng.choice(["bf16", "bf16", "f16", "f32"]))
    cols = _log(rng, 64, 16384)
    if rng.random() < 0.5:
        cols = max(64, cols // 64 * 64)
    rows = min(_log(rng, 1, 16384), MOST_VALUES // 2 // cols)
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    p = rng.choice([0.0, 0.05, 0.1, 0.1, 0.2, 0.5])
    if op in ("norm", "norm_back"):
        case = dict(op=op, rows=rows, cols=cols, dtype=dtype, residual=rng.choice([dtype, "f32"]), p=p)
        if op == "norm":
            case["out"] = rng.choice(["same", "e4m3", "e4m3", "e5m2"])
        return case
    if op == "dropout":
        return dict(op=op, rows=rows, cols=cols, dtype=dtype, p=max(p, 0.05), pad=rng.choice([0, 0, 8, 13]))
    return dict(op=op, rows=rows, cols=cols, dtype=dtype, blocks=rng.random() < 0.4, format=rng.choice(["e4m3", "e4m3", "e5m2"]),
                both=rng.random() < 0.6)


def _up(n, m):
    return -(-n // m) * m


def _scales_like(rows, cols, dev):
    """Room for the scales of `rows` rows (or rows of blocks) of `cols` values."""
    return torch.empty(-(-cols // 512), rows, 4, dtype=torch.float8_e8m0fnu, device=dev)


def _eight_like(rows, cols, fmt, dev):
    """Room for an 8-bit matrix whose rows begin at multiples of 16 bytes."""
    return torch.empty(rows, _up(cols, 16), dtype=torch.uint8, device=dev).view(FORMATS[fmt])[:, :cols]


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.randn(*shape, device=dev, generator=gen).mul_(std).to(dtype)

    op = case["op"]
    s = dict(case, seed=(seed * 0x9E3779B97F4A7C15 + 0x1234567) & (2 ** 64 - 1), offset=seed * 4 + (1 << 33))
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        for side, rows, fmt, blocks in (("a", M, case["a"], False), ("b", N, case["b"], case["blocks"])):
            x = normal(rows, K)
            if not blocks:
                x *= torch.exp(normal(rows, 1))          # tokens and gradients differ in size
            q = _eight_like(rows, K, fmt, dev)
            values, e = _quantized(x, fmt, blocks)
            q.copy_(values)
            s[side], s[side + "_scales"] = q, _in_words(e)
        s["c"] = torch.empty(M, N, dtype=DTYPES[case["out"]], device=dev)
        s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device=dev)
        return s
    rows, cols, dt = case["rows"], case["cols"], DTYPES[case["dtype"]]
    if op == "dropout":
        width = cols + case["pad"]
        s["x"] = normal(rows, width, dtype=dt)[:, :cols]
        s["y"] = torch.empty(rows, width, dtype=dt, device=dev)[:, :cols]
        return s
    if op == "quantize":
        s["x"] = normal(rows, cols).mul_(torch.exp(normal(rows, 1))).mul_(0.02).to(dt)
        tall = -(-rows // 128) if case["blocks"] else rows
        wide = -(-cols // 128) if case["blocks"] else cols
        s["q"], s["scales"] = _eight_like(rows, cols, case["format"], dev), _scales_like(tall, cols, dev)
        if case["both"]:
            s["q_t"], s["scales_t"] = _eight_like(cols, rows, case["format"], dev), _scales_like(wide, rows, dev)
        return s
    rt = DTYPES[case["residual"]]
    s["weight"] = (1 + normal(cols, std=0.2)).to(dt)
    if op == "norm":
        s["x"], s["residual_in"] = normal(rows, cols, dtype=dt), normal(rows, cols, std=2.0, dtype=rt)
        s["h"], s["rstd"] = torch.empty(rows, cols, dtype=rt, device=dev), torch.empty(rows, device=dev)
        if case["out"] == "same":
            s["y"] = torch.empty(rows, cols, dtype=dt, device=dev)
        else:
            s["q"], s["scales"] = _eight_like(rows, cols, case["out"], dev), _scales_like(rows, cols, dev)
        return s
    s["h"] = normal(rows, cols, std=2.0, dtype=rt)
    s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + EPS)
    s["dy"] = normal(rows, cols, std=1e-2, dtype=dt)
    s["dh"] = normal(rows, cols, std=1e-2, dtype=rt)
    s["dres"], s["dx"] = torch.empty(rows, cols, dtype=rt, device=dev), torch.empty(rows, cols, dtype=dt, device=dev)
    s["dweight"] = torch.empty(cols, device=dev)
    s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device=dev)
    return s


# ---- the plain form ---------------------------------------------------------------------------------------
def _keep(rows, cols, p, seed, offset, dev):
    """(which elements are kept, the factor of those) in whole-number tensor operations."""
    t = round(p * 65536)
    low = 0xFFFFFFFF
    group = torch.arange(-(-cols // 8), device=dev)
    c = [group.repeat(rows, 1), torch.arange(rows, device=dev)[:, None].expand(rows, group.numel()),
         torch.full((1, 1), offset & low, device=dev), torch.full((1, 1), offset >> 32, device=dev)]
    k = [seed & low, seed >> 32]
    for _ in range(10):
        u, v = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((v >> 32) & low) ^ c[1] ^ k[0], v & low, ((u >> 32) & low) ^ c[3] ^ k[1], u & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    c = torch.broadcast_tensors(*c)
    bits = torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], dim=-1)
    return bits.reshape(rows, -1)[:, :cols] >= t, 65536 / (65536 - t)


def _dropped(x, s):
    if s["p"] == 0:
        return x
    keep, scale = _keep(*x.shape, s["p"], s["seed"], s["offset"], x.device)
    return torch.where(keep, x * scale, 0.0)


def _quantized(x, fmt, blocks):
    """(8-bit values, biased exponents [rows or rows of blocks, blocks of columns]) of an fp32 matrix."""
    rows, cols = x.shape
    tall = 128 if blocks else 1
    padded = torch.nn.functional.pad(x, (0, _up(cols, 128) - cols, 0, _up(rows, tall) - rows))
    tiles = padded.view(padded.shape[0] // tall, tall, padded.shape[1] // 128, 128)
    amax = tiles.abs().amax(dim=(1, 3))
    e = (((amax.view(torch.int32) + 0x1FFFFF) >> 23) - TOP[fmt]).clamp(min=1)
    e = torch.where(torch.isfinite(amax), e, 255)
    back = torch.where(e == 255, math.nan, ((254 - e) << 23).view(torch.float32))
    q = (tiles * back[:, None, :, None]).view_as(padded)[:rows, :cols]
    return q.to(FORMATS[fmt]), e


def _in_words(e):
    """Exponents [rows, blocks] as scales [ceil(blocks / 4)][rows][4]."""
    e = torch.nn.functional.pad(e, (0, _up(e.shape[1], 4) - e.shape[1]), value=127)
    return e.view(e.shape[0], -1, 4).transpose(0, 1).contiguous().to(torch.uint8).view(torch.float8_e8m0fnu)


def _factors(scales, rows, cols, blocks, kind):
    """Scales as factors of the elements of a [rows, cols] matrix."""
    f = scales.to(kind).transpose(0, 1).reshape(scales.shape[1], -1)[:, :-(-cols // 128)]
    if blocks:
        f = f.repeat_interleave(128, 0)[:rows]
    return f.repeat_interleave(128, 1)[:, :cols]


def _plain(s):
    op = s["op"]
    if op == "product":
        a = s["a"].float() * _factors(s["a_scales"], s["M"], s["K"], False, torch.float32)
        b = s["b"].float() * _factors(s["b_scales"], s["N"], s["K"], s["blocks"], torch.float32)
        return (a @ b.t()).to(s["c"].dtype)
    if op == "dropout":
        return _dropped(s["x"].float(), s).to(s["x"].dtype)
    if op == "quantize":
        x = s["x"].float()
        q, e = _quantized(x, s["format"], s["blocks"])
        got = {"q": q, "scales": _in_words(e)}
        if s["both"]:
            q, e = _quantized(x.t().contiguous(), s["format"], s["blocks"])
            got |= {"q_t": q, "scales_t": _in_words(e)}
        return got
    w = s["weight"].float()
    if op == "norm":
        h = s["residual_in"].float() + _dropped(s["x"].float(), s)
        rstd = torch.rsqrt((h * h).mean(1) + EPS)
        y = h * rstd[:, None] * w
        got = {"h": h.to(s["h"].dtype), "rstd": rstd}
        if s["out"] == "same":
            return got | {"y": y.to(s["x"].dtype)}
        q, e = _quantized(y, s["out"], False)
        return got | {"q": q, "scales": _in_words(e)}
    dy, r = s["dy"].float(), s["rstd"][:, None]
    xhat, g = s["h"].float() * r, dy * w
    dres = r * (g - xhat * (g * xhat).mean(1, keepdim=True)) + s["dh"].float()
    dx = _dropped(dres, s)
    return {"dres": dres.to(s["dres"].dtype), "dx": dx.to(s["dx"].dtype), "dweight": (dy * xhat).sum(0)}


# ---- the framework's operators ------------------------------------------------------------------------------
def run(state):
    if not own:
        return _plain(state)
    import paper_2310_12670_amd as reft

    s, op = state, state["op"]
    if op == "product":
        reft.reft_product(s["a"], s["a_scales"], s["b"], s["b_scales"], s["c"], s["workspace"], b_blocks=s["blocks"])
        return s["c"]
    if op == "dropout":
        reft.reft_dropout(s["x"], s["y"], s["p"], s["seed"], s["offset"])
        return s["y"]
    if op == "quantize":
        if s["both"]:
            reft.reft_quantize(s["x"], s["q"], s["scales"], s["q_t"], s["scales_t"], blocks=s["blocks"])
            return {"q": s["q"], "scales": s["scales"], "q_t": s["q_t"], "scales_t": s["scales_t"]}
        reft.reft_quantize(s["x"], s["q"], s["scales"], blocks=s["blocks"])
        return {"q": s["q"], "scales": s["scales"]}
    if op == "norm":
        got = {"h": s["h"], "rstd": s["rstd"]}
        if s["out"] == "same":
            reft.reft_norm_forward(s["x"], s["residual_in"], s["weight"], EPS, s["p"], s["seed"], s["offset"],
                                   h=s["h"], rstd=s["rstd"], y=s["y"])
            return got | {"y": s["y"]}
        reft.reft_norm_forward(s["x"], s["residual_in"], s["weight"], EPS, s["p"], s["seed"], s["offset"],
                               h=s["h"], rstd=s["rstd"], q=s["q"], scales=s["scales"])
        return got | {"q": s["q"], "scales": s["scales"]}
    reft.reft_norm_backward(s["dy"], s["dh"], s["h"], s["rstd"], s["weight"], s["p"], s["seed"], s["offset"],
                            dres=s["dres"], dx=s["dx"], dweight=s["dweight"], workspace=s["workspace"])
    return {"dres": s["dres"], "dx": s["dx"], "dweight": s["dweight"]}


def work(case):
    op = case["op"]
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        words = -(-K // 512) * 4
        out = M * N * (4 if case["out"] == "f32" else 2)
        return {"bytes": M * K + N * K + out + words * (M + (-(-N // 128) if case["blocks"] else N)), "flops": 2 * M * N * K}
    rows, cols = case["rows"], case["cols"]
    n, size = rows * cols, SIZE[case["dtype"]]
    if op == "dropout":
        return {"bytes": 2 * n * size, "flops": n}
    if op == "quantize":
        tall, wide = (-(-rows // 128), -(-cols // 128)) if case["blocks"] else (rows, cols)
        one = n + -(-cols // 512) * 4 * tall
        other = n + -(-rows // 512) * 4 * wide if case["both"] else 0
        return {"bytes": n * size + one + other, "flops": 2 * n}
    wide = SIZE[case["residual"]]
    if op == "norm":
        out = n * size if case["out"] == "same" else n + -(-cols // 512) * 4 * rows
        return {"bytes": n * (size + 2 * wide) + out + cols * size + rows * 4, "flops": 6 * n}
    return {"bytes": n * (2 * size + 3 * wide) + cols * (size + 4) + rows * 4, "flops": 12 * n}


# ---- the same from the definitions, in 64 bits --------------------------------------------------------------------
def _mask64(rows, cols, p, seed, offset, dev):
    """1 / (1 - p) where an element is kept and 0 where not, from whole numbers of 64 bits on the host, some rows at a time."""
    t = np.uint64(round(p * 65536))
    groups, out = (cols + 7) // 8, np.empty((rows, cols), dtype=bool)
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    step = max(1, (1 << 20) // groups)
    for first in range(0, rows, step):
        n = min(step, rows - first)
        x0 = np.tile(np.arange(groups, dtype=np.uint64), n)
        x1 = np.repeat(np.arange(first, first + n, dtype=np.uint64), groups)
        x2 = np.full(n * groups, offset % 2 ** 32, dtype=np.uint64)
        x3 = np.full(n * groups, offset // 2 ** 32, dtype=np.uint64)
        for i in range(10):
            k0 = np.uint64((seed % 2 ** 32 + i * 0x9E3779B9) % 2 ** 32)
            k1 = np.uint64((seed // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32)
            a, b = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
            x0, x1, x2, x3 = (b >> half) ^ x1 ^ k0, b & low, (a >> half) ^ x3 ^ k1, a & low
        words = np.stack([x0, x1, x2, x3], axis=1).astype("<u4")
        out[first:first + n] = (words.view("<u2").reshape(n, groups * 8)[:, :cols] >= t)
    return torch.from_numpy(out).to(dev).double() * (65536 / (65536 - int(t)))


def _eight64(y, fmt, blocks):
    """What the 8 bits of a matrix stand for before they are rounded, and the powers of two, from logarithms of exact values."""
    m, n = y.shape
    tall = 128 if blocks else 1
    up, left = -(-m // tall), -(-n // 128)
    full = torch.zeros(up * tall, left * 128, dtype=torch.float64, device=y.device)
    full[:m, :n] = y
    most = full.abs().reshape(up, tall, left, 128).transpose(1, 2).reshape(up, left, -1).max(dim=2).values
    mantissa, power = torch.frexp(most / 1.75)            # most = 1.75 * mantissa * 2 ** power with mantissa in [0.5, 1)
    power = torch.where(mantissa == 0.5, power - 1, power).double() - TOP[fmt]
    power = torch.where(most == 0, torch.full_like(power, -126), power).clamp(min=-126)
    scale = torch.exp2(power)
    per = scale.repeat_interleave(tall, 0).repeat_interleave(128, 1)[:m, :n]
    words = torch.ones(up, -(-left // 4) * 4, dtype=torch.float64, device=y.device)
    words[:, :left] = scale
    return y / per, words.reshape(up, -1, 4).permute(1, 0, 2).contiguous()


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "product":
        def whole(q, scales, rows, tall):
            value = q.double()
            for block in range(-(-case["K"] // 128)):
                f = scales[block // 4, :, block % 4].double()
                value[:, block * 128:block * 128 + 128] *= f.repeat_interleave(tall)[:rows, None]
            return value
        a = whole(s["a"], s["a_scales"], case["M"], 1)
        b = whole(s["b"], s["b_scales"], case["N"], 128 if case["blocks"] else 1)
        return torch.mm(a, b.t())
    rows, cols = case["rows"], case["cols"]

    def mask(dev):
        return _mask64(rows, cols, case["p"], s["seed"], s["offset"], dev) if case["p"] else 1.0

    if op == "dropout":
        return s["x"].double() * mask(s["x"].device)
    if op == "quantize":
        x = s["x"].double()
        q, scales = _eight64(x, case["format"], case["blocks"])
        got = {"q": q, "scales": scales}
        if case["both"]:
            got["q_t"], got["scales_t"] = _eight64(x.t(), case["format"], case["blocks"])
        return got
    w = s["weight"].double()
    if op == "norm":
        h = s["x"].double() * mask(w.device) + s["residual_in"].double()
        rstd = 1 / torch.sqrt(h.pow(2).sum(1) / cols + EPS)
        y = torch.einsum("rc,r,c->rc", h, rstd, w)
        got = {"h": h, "rstd": rstd}
        if case["out"] == "same":
            return got | {"y": y}
        q, scales = _eight64(y, case["out"], False)
        return got | {"q": q, "scales": scales}
    h, dy, r = s["h"].double(), s["dy"].double(), s["rstd"].double()
    dot = (dy * w * h).sum(1) * r.pow(3) / cols
    dres = dy * w * r[:, None] - h * dot[:, None] + s["dh"].double()
    return {"dres": dres, "dx": dres * mask(w.device), "dweight": torch.mv((dy * h).t(), r)}
