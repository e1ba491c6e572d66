#!/usr/bin/env python3
"""One data-parallel worker's training step, from activations to the gradient it sends.

A gated feed-forward block with a residual (y = x + W2 (silu(Wg n) * (Wu n)), n = gamma * rmsnorm(x)) runs forward on 8-bit
products and keeps 8-bit checkpoints; its backward pass takes them and writes the weight gradients into one flat
binary32 buffer; that buffer is compressed at the ratio the network-sensing controller picks, as the worker would send it,
decompressed, and applied to the weights.

    python examples/worker_step.py [--tokens 4096 --hidden 1024 --inner 2816 --steps 20]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2506_16235_amd import binding as nsml  # noqa: E402
from paper_2506_16235_amd import workloads as W  # noqa: E402


class Block:
    """Weights and gradients are views of two flat buffers, a bucket each: gamma [K], W1 = (Wg; Wu) [2F, K], W2 [K, F]."""

    def __init__(self, hidden: int, inner: int, seed: int = 0, device="cuda:0"):
        self.K, self.F, self.dev = hidden, inner, torch.device(device)
        self.off = W.offsets_of([hidden, 2 * inner * hidden, hidden * inner])
        n = int(self.off[-1])
        self.flat = torch.empty(n, dtype=torch.float32, device=self.dev)
        self.grad = torch.zeros(n, dtype=torch.float32, device=self.dev)
        gen = torch.Generator(device=self.dev)
        gen.manual_seed(seed)
        self.gamma, self.w1, self.w2 = self._views(self.flat)
        self.dgamma, self.dw1, self.dw2 = self._views(self.grad)
        self.gamma.fill_(1.0)
        for w in (self.w1, self.w2):
            w.copy_(torch.randn(w.shape, generator=gen, device=self.dev) * w.shape[1] ** -0.5)
        self.laid_out()

    def _views(self, flat):
        o, K, F = [int(v) for v in self.off], self.K, self.F
        return flat[:o[1]], flat[o[1]:o[2]].view(2 * F, K), flat[o[2]:o[3]].view(K, F)

    def laid_out(self):
        """The weights in 8 bits, by output channel, and their codes the other way round: once per update."""
        self.q1, self.q2 = nsml.q8_rows(self.w1), nsml.q8_rows(self.w2)
        self.t1, self.t2 = nsml.q8_transposed(self.q1), nsml.q8_transposed(self.q2)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        F = self.F
        self.norm = nsml.rmsnorm_q8(x, self.gamma, checkpoint=True)
        z = nsml.q8_matmul(self.norm.y, self.q1, x.dtype)
        self.glu = nsml.swiglu_q8(z[:, :F], z[:, F:], checkpoint=True)
        return x + nsml.q8_matmul(self.glu.a, self.q2, x.dtype)

    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        """Gradients of the weights into self.grad; -> the gradient of x."""
        F, norm, glu = self.F, self.norm, self.glu
        nsml.ckpt8_wgrad(dy, glu.held, out=self.dw2)
        da = nsml.q8_matmul(nsml.q8_rows(dy, self.q2.scale), self.t2, dy.dtype)
        dz = torch.empty(dy.shape[0], 2 * F, dtype=dy.dtype, device=dy.device)
        nsml.swiglu_backward(da, glu.gate, glu.up, dgate=dz[:, :F], dup=dz[:, F:])
        nsml.ckpt8_wgrad(dz, norm.xhat, col_scale=self.gamma, out=self.dw1)
        dn = nsml.q8_matmul(nsml.q8_rows(dz, self.q1.scale), self.t1, dy.dtype)
        dx, _ = nsml.rmsnorm_backward(dn, norm.xhat, norm.rstd, self.gamma, dres=dy, dgamma=self.dgamma)
        return dx

    def kept_bytes(self) -> int:
        """What the backward pass needs to be kept of the forward pass."""
        return sum(t.numel() for c in (self.norm.xhat, self.glu.gate, self.glu.up, self.glu.held) for t in c) + 4 * self.norm.rstd.numel()


class Worker:
    """A block, the controller, and what earlier steps did not send."""

    def __init__(self, block: Block):
        self.block, self.ctl = block, nsml.Controller()
        n = block.flat.numel()
        self.ctx = nsml.Context(n, len(block.off) - 1, 2048, device=block.dev.index or 0)
        self.residual = torch.zeros(n, dtype=torch.float32, device=block.dev)
        self.last = (0.0, 0.0)

    def step(self, x, target, lr: float, link_bits_per_s: float = 1e10):
        """-> (loss, ratio, bits, payload bytes)."""
        b, off = self.block, self.block.off
        err = b.forward(x).float() - target.float()
        b.backward((err * (2.0 / err.numel())).to(x.dtype))
        ratio, bits = self.ctl.choose_ratio(*self.last, 4.0 * b.flat.numel())
        idx, val, sc = self.ctx.compress(b.grad, self.residual, off, ratio, bits)
        sent = idx.numel() * 4 + val.numel() + (sc.numel() * 4 if bits <= 8 else 0)
        b.flat.sub_(self.ctx.decompress(idx, val, sc, b.flat.numel(), off, ratio, bits), alpha=lr)
        b.laid_out()
        self.last = (float(sent), W.simulated_tx_seconds(sent, link_bits_per_s))
        return err.square().mean(), ratio, bits, sent


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--inner", type=int, default=2816)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--lr", type=float, default=200.0)
    a = ap.parse_args()
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(1)
    teacher, worker = Block(a.hidden, a.inner, seed=2), Worker(Block(a.hidden, a.inner, seed=3))
    x = torch.randn(a.tokens, a.hidden, generator=gen, device="cuda:0").bfloat16()
    target = teacher.forward(x)
    t0 = time.perf_counter()
    for s in range(a.steps):
        loss, ratio, bits, sent = worker.step(x, target, a.lr)
        print(f"step {s:3d}  loss {loss.item():.5f}  ratio {ratio:.3f}  {bits} bits  sent {sent / 1e6:.2f} MB", flush=True)
    torch.cuda.synchronize()
    dt = (time.perf_counter() - t0) / a.steps
    plain = a.tokens * (2 * a.hidden + 3 * 2 * a.inner)      # x, gate, up and the activation in 16 bits
    print(f"{dt * 1e3:.2f} ms a step; kept for the backward pass {worker.block.kept_bytes() / 1e6:.1f} MB, in 16 bits {plain / 1e6:.1f} MB")


if __name__ == "__main__":
    main()
