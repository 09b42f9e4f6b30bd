"""Training in 8 bits that resumes to the same bits.

A few residual sublayers (norm, two products with a squared ReLU between them, dropout) are trained on synthetic data with the
library's operators; PyTorch does the elementwise rest.  The training state - per weight a bf16 parameter and fp32
master, first and second moment, and dropout's seed and step (16 bytes) - is snapshotted to pinned host memory
after some steps.  Later all of it is lost, restored from the snapshot, and the steps since then are run again: losses and
state come out as they were, bit for bit.

    python examples/resume_training.py [--steps 6] [--snapshot 3]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2310_12670_amd as reft  # noqa: E402

EPS, DROP, RATE = 1e-5, 0.1, 1e-3


class Eight:
    """Room for a matrix in 8 bits, with its scales: rows on 16 bytes, as the products like them."""

    def __init__(self, rows, cols, dev, blocks=False):
        self.q = torch.empty(rows, -(-cols // 16) * 16, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)[:, :cols]
        self.scales = torch.empty(-(-cols // 512), -(-rows // 128) if blocks else rows, 4, dtype=torch.uint8, device=dev)
        self.blocks = blocks


def quantize(x, blocks=False, which="both"):
    """x and its transpose in 8 bits ("both"), or one of them ("q", "t")."""
    q = Eight(*x.shape, x.device, blocks) if which != "t" else None
    t = Eight(x.shape[1], x.shape[0], x.device, blocks) if which != "q" else None
    reft.reft_quantize(x, q and q.q, q and q.scales, t and t.q, t and t.scales, blocks=blocks)
    return (q, t) if which == "both" else q or t


def product(a, b, dtype):
    M, K = a.q.shape
    N = b.q.shape[0]
    c = torch.empty(M, N, dtype=dtype, device=a.q.device)
    scratch = torch.empty(reft.reft_product_workspace(M, N, K), dtype=torch.uint8, device=a.q.device)
    reft.reft_product(a.q, a.scales, b.q, b.scales, c, scratch, b_blocks=b.blocks)
    return c


class Model:
    """Sublayers of s = W2 relu(W1 norm(h))^2, joined by h <- h + dropout(s), and a norm at the end."""

    def __init__(self, dev, width=256, inner=640, layers=2, seed=1):
        gen = torch.Generator(device=dev)
        gen.manual_seed(seed)
        shapes = []
        for _ in range(layers):
            shapes += [(width,), (inner, width), (width, inner)]
        self.layers, self.dev = layers, dev
        self.master = [torch.ones(s, device=dev) if len(s) == 1 else
                       torch.randn(s, device=dev, generator=gen) * s[1] ** -0.5 for s in shapes + [(width,)]]
        self.param = [t.to(torch.bfloat16) for t in self.master]
        self.first = [torch.zeros_like(t) for t in self.master]
        self.second = [torch.zeros_like(t) for t in self.master]
        self.counter = torch.tensor([0x5EED, 0], dtype=torch.int64, device=dev)         # dropout's seed, steps done

    def state(self):
        """The tensors of a snapshot, in order."""
        return self.param + self.master + self.first + self.second + [self.counter]

    def _norm(self, at, x, residual, seed, offset, out):
        """h = residual + dropout(x) and what the backward pass needs of the norm; its output in 8 bits too if `out` says so."""
        rows, cols = residual.shape
        h, y = torch.empty_like(residual), torch.empty_like(residual)
        rstd, e = torch.empty(rows, device=self.dev), Eight(rows, cols, self.dev) if out == "eight" else None
        reft.reft_norm_forward(x, residual, self.param[at], EPS, DROP, seed, offset, h=h, rstd=rstd, y=y,
                               q=e and e.q, scales=e and e.scales)
        return h, rstd, y, e

    def _norm_back(self, at, dy, dh, h, rstd, seed, offset):
        dres, dx, dw = torch.empty_like(h), torch.empty_like(h), torch.empty(h.shape[1], device=self.dev)
        scratch = torch.empty(reft.reft_norm_backward_workspace(*h.shape), dtype=torch.uint8, device=self.dev)
        reft.reft_norm_backward(dy, dh, h, rstd, self.param[at], DROP, seed, offset, dres=dres, dx=dx, dweight=dw, workspace=scratch)
        return dres, dx, dw

    def step(self, x, target):
        """One step of Adam on the mean square error; returns the loss."""
        seed, done = self.counter.tolist()
        offset = [done * (self.layers + 1) + i for i in range(self.layers + 1)]          # a mask of its own for every use
        bf16, kept = torch.bfloat16, []
        h, s = x, torch.zeros_like(x)
        for i in range(self.layers):
            w1, w1_t = quantize(self.param[3 * i + 1], blocks=True)
            w2, w2_t = quantize(self.param[3 * i + 2], blocks=True)
            h, rstd, y, y8 = self._norm(3 * i, s, h, seed, offset[i], "eight")
            u = product(y8, w1, bf16)
            a, a_t = quantize(torch.relu(u).square())
            s = product(a, w2, bf16)
            kept.append((h, rstd, y, u, a_t, w1_t, w2_t))
        h, rstd, y, _ = self._norm(-1, s, h, seed, offset[-1], "same")
        error = y.float() - target
        loss = error.square().mean()
        grads = [None] * len(self.param)
        dh, ds, grads[-1] = self._norm_back(-1, (error * (2 / error.numel())).to(bf16), None, h, rstd, seed, offset[-1])
        for i in reversed(range(self.layers)):
            h, rstd, y, u, a_t, w1_t, w2_t = kept[i]
            ds8, ds_t = quantize(ds)
            grads[3 * i + 2] = product(ds_t, a_t, torch.float32)
            du = product(ds8, w2_t, bf16) * (2 * torch.relu(u))
            du8, du_t = quantize(du)
            grads[3 * i + 1] = product(du_t, quantize(y, which="t"), torch.float32)
            dh, ds, grads[3 * i] = self._norm_back(3 * i, product(du8, w1_t, bf16), dh, h, rstd, seed, offset[i])
        t = done + 1
        for p, w, m, v, g in zip(self.param, self.master, self.first, self.second, grads):
            m.mul_(0.9).add_(g, alpha=0.1)
            v.mul_(0.99).addcmul_(g, g, value=0.01)
            w.sub_(RATE * (m / (1 - 0.9 ** t)) / ((v / (1 - 0.99 ** t)).sqrt() + 1e-12))
            p.copy_(w)
        self.counter[1] += 1
        return float(loss)


def run(steps=6, snapshot=3, rows=384, dev=None):
    """(losses up to the snapshot, losses after it, the same again after the restore, whether the states are equal)"""
    dev = dev or torch.device("cuda:0")
    torch.cuda.set_device(dev)
    model = Model(dev)
    gen = torch.Generator(device=dev)
    gen.manual_seed(2)
    x = torch.randn(rows, 256, device=dev, generator=gen).to(torch.bfloat16)
    target = torch.randn(rows, 256, device=dev, generator=gen)

    spans = model.state()
    plan = reft.reft_plan_create([t.numel() * t.element_size() for t in spans], None, 1 << 20)
    try:
        size = reft.reft_plan_stream_bytes(plan)
        host = torch.empty(size, dtype=torch.uint8, pin_memory=True)
        staging = torch.empty(2 * reft.reft_plan_staging_slot_bytes(plan), dtype=torch.uint8, device=dev)
        before = [model.step(x, target) for _ in range(snapshot)]
        reft.reft_snapshot_pack(plan, spans, staging, host)
        reft.reft_snapshot_wait(plan)
        after = [model.step(x, target) for _ in range(steps - snapshot)]
        final = [t.clone() for t in spans]
        for t in spans:                                                                 # the state is lost
            t.view(torch.uint8).fill_(0xFF)
        reft.reft_restore(plan, host, staging, spans)
        reft.reft_restore_wait(plan)
        again = [model.step(x, target) for _ in range(steps - snapshot)]
        same = all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(spans, final))
    finally:
        torch.cuda.synchronize()
        reft.reft_plan_destroy(plan)
    return before, after, again, same


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=6)
    ap.add_argument("--snapshot", type=int, default=3)
    args = ap.parse_args()
    before, after, again, same = run(args.steps, args.snapshot)
    print("losses up to the snapshot:", *("%.6f" % v for v in before))
    print("losses after it:          ", *("%.6f" % v for v in after))
    print("after the restore:        ", *("%.6f" % v for v in again))
    print("same bits:", same and after == again)
    return 0 if same and after == again else 1


if __name__ == "__main__":
    sys.exit(main())
