"""The operators together, as examples/worker_step.py runs them: a block's gradients against automatic differentiation in 64 bits of the
same block without 8-bit values, and a worker that learns through them and the compressed gradient.

Tolerance: every value passed on in 8 bits is off by at most half a step, absmax / 254 of its row (or of its 32 neighbours, up
to 1 / 128), uniformly spread: for near-normal rows of this width (absmax about 3.5 sigma) a relative error of the norm of
3.5 / 127 / sqrt(12) = 0.8 %.  A weight gradient sees at most five such factors one after the other (norm, product's
weights, activation, incoming gradient, checkpoint), so 5 * 0.8 % = 4 % if they all added up; 16-bit results add 0.4 % each."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def off(a, b):
    return float((a.double().cpu() - b).norm() / b.norm())


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("m,K,F", [(300, 256, 320), (77, 130, 201)])
def test_gradients_of_a_block(dt, m, K, F):
    from worker_step import Block
    b = Block(K, F, seed=5)
    gen = torch.Generator()
    gen.manual_seed(1)
    x = torch.randn(m, K, generator=gen).to(dt)
    dy = torch.randn(m, K, generator=gen).to(dt)
    b.gamma.copy_(1 + 0.2 * torch.randn(K, generator=gen))
    y = b.forward(x.cuda())
    dx = b.backward(dy.cuda())
    ref = {n: getattr(b, n).detach().double().cpu().requires_grad_() for n in ("gamma", "w1", "w2")}
    xr = x.double().requires_grad_()
    n = ref["gamma"] * xr / torch.sqrt(xr.square().mean(1, keepdim=True) + 1e-5)
    z = n @ ref["w1"].t()
    out = xr + (z[:, :F] * torch.sigmoid(z[:, :F]) * z[:, F:]) @ ref["w2"].t()
    out.backward(dy.double())
    assert off(y, out.detach()) < 0.05
    assert off(dx, xr.grad) < 0.05
    assert off(b.dw2, ref["w2"].grad) < 0.05
    assert off(b.dw1, ref["w1"].grad) < 0.05
    assert off(b.dgamma, ref["gamma"].grad) < 0.05


def test_a_worker_learns():
    from worker_step import Block, Worker
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(1)
    teacher, worker = Block(128, 256, seed=2), Worker(Block(128, 256, seed=3))
    x = torch.randn(512, 128, generator=gen, device="cuda:0").bfloat16()
    target = teacher.forward(x)
    loss = [float(worker.step(x, target, 20.0)[0]) for _ in range(30)]
    assert loss[-1] < 0.7 * loss[0] and all(v == v for v in loss)
    assert worker.block.kept_bytes() < 0.6 * 2 * 512 * (128 + 3 * 256)
