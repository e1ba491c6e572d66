"""Checkpoints whose exponents have a row stride of their own: read and written where they lie, with nothing between the rows touched or used."""
import pytest
import torch

from paper_2506_16235_amd import binding as nsml

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
types = pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16], ids=["f32", "bf16", "f16"])


def rand(seed, *shape):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g)


def room(m, k, gap):
    """-> (checkpoint to write into, all of its exponents' memory, all of its codes')."""
    e = torch.full((m, (k + 31) // 32 + gap), 251, dtype=torch.uint8, device=DEV)
    q = torch.full((m, (k + 15) // 16 * 16 + 32), 99, dtype=torch.int8, device=DEV)
    return nsml.Ckpt8(q[:, :k], e[:, :(k + 31) // 32]), e, q


@types
@pytest.mark.parametrize("m,k,gap", [(1, 5, 3), (9, 64, 1), (70, 333, 5), (200, 1100, 13), (520, 4100, 2), (40, 9000, 7), (30, 20000, 1)])
def test_exponents_with_gaps(dt, m, k, gap):
    x, dy = rand(1, m, k).to(dt).to(DEV), rand(2, m, k).to(dt).to(DEV)
    c, e, q = room(m, k, gap)
    tight = nsml.ckpt8_pack(x)
    assert nsml.ckpt8_pack(x, out=c) is c
    assert torch.equal(c.q, tight.q) and torch.equal(c.e, tight.e)
    assert (e[:, (k + 31) // 32:] == 251).all() and (q[:, (k + 15) // 16 * 16:] == 99).all()
    assert torch.equal(nsml.ckpt8_unpack(c), nsml.ckpt8_unpack(tight))
    rstd = 1 / x.float().square().mean(1).sqrt()
    for a, b in zip(nsml.rmsnorm_backward(dy, c, rstd), nsml.rmsnorm_backward(dy, tight, rstd)):
        assert torch.equal(a, b)
    for a, b in zip(nsml.swiglu_backward(dy, c, c), nsml.swiglu_backward(dy, tight, tight)):
        assert torch.equal(a, b)
    d = rand(3, m, 37).to(dt).to(DEV)
    assert torch.equal(nsml.ckpt8_wgrad(d, c), nsml.ckpt8_wgrad(d, tight))


@types
@pytest.mark.parametrize("m,n,k", [(300, 700, 900), (4000, 600, 520), (64, 3000, 2950)])
def test_weight_gradients_with_gaps(dt, m, n, k):
    x, d = rand(4, m, k).to(DEV), rand(5, m, n).to(dt).to(DEV)
    c, _, _ = room(m, k, 11)
    nsml.ckpt8_pack(x, out=c)
    assert torch.equal(nsml.ckpt8_wgrad(d, c), nsml.ckpt8_wgrad(d, nsml.ckpt8_pack(x)))
