"""Results of the 8-bit layer written over what they are made from, where that is allowed, equal those written elsewhere."""
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


@types
@pytest.mark.parametrize("m,k", [(1, 5), (7, 300), (2000, 520), (700, 2048), (1100, 4096), (600, 8200), (90, 32768)])
def test_gradients_over_what_they_come_from(dt, m, k):
    x, dy, dres = rand(1, m, k).to(dt).to(DEV), rand(2, m, k).to(dt).to(DEV), rand(3, m, k).to(dt).to(DEV)
    c = nsml.ckpt8_pack(x)
    rstd = 1 / x.float().square().mean(1).sqrt()
    want, dgamma = nsml.rmsnorm_backward(dy, c, rstd, dres=dres)
    for same in ("dy", "dres"):
        t = {"dy": dy.clone(), "dres": dres.clone()}
        got, dg = nsml.rmsnorm_backward(t["dy"], c, rstd, dres=t["dres"], out=t[same])
        assert got is t[same] and torch.equal(got, want) and torch.equal(dg, dgamma)
    g, u = nsml.swiglu_backward(dy, c, c)
    for same in ("dgate", "dup"):
        da = dy.clone()
        a, b = nsml.swiglu_backward(da, c, c, **{same: da})
        assert torch.equal(a, g) and torch.equal(b, u)


@types
@pytest.mark.parametrize("m,k", [(1, 5), (7, 300), (700, 2048), (600, 8200), (90, 32768)])
def test_norm_over_its_input(dt, m, k):
    x, r = rand(1, m, k).to(dt).to(DEV), rand(2, m, k).to(dt).to(DEV)
    o = nsml.rmsnorm_q8(x, None, 1e-5, residual=r)
    for same in (0, 1):
        t = [x.clone(), r.clone()]
        q, s = nsml._new_codes(m, k, t[0].device), torch.empty(m, device=DEV)
        rstd = torch.empty(m, device=DEV)
        rc = nsml.raw().nsml_rmsnorm_q8(t[0].data_ptr(), k, t[1].data_ptr(), k, None, 1e-5, nsml._TYPE[dt], m, k, t[same].data_ptr(), k,
                                        q.data_ptr(), (k + 15) // 16 * 16, s.data_ptr(), rstd.data_ptr(), None, torch.cuda.current_stream().cuda_stream)
        assert rc == nsml.OK
        assert torch.equal(t[same], o.h) and torch.equal(q, o.y.q) and torch.equal(s, o.y.scale) and torch.equal(rstd, o.rstd)


def test_results_that_reach_into_other_buffers_are_refused():
    k = 64
    flat = rand(1, 3 * k, k).to(DEV)
    before = flat.clone()
    c, rstd = nsml.ckpt8_pack(flat[:20]), torch.ones(20, device=DEV)
    for call in (lambda: nsml.rmsnorm_backward(flat[:20], c, rstd, out=flat[1:21]),
                 lambda: nsml.rmsnorm_backward(flat[:20], c, rstd, out=flat[20:40], dgamma=flat[39]),
                 lambda: nsml.swiglu_backward(flat[:20], c, c, dgate=flat[20:40], dup=flat[39:59]),
                 lambda: nsml.ckpt8_pack(flat[:20], out=nsml.Ckpt8(flat[:20].view(torch.int8)[:, :k], c.e)),
                 lambda: nsml.ckpt8_wgrad(flat[:20], c, out=flat[19:19 + k]),
                 lambda: nsml.ckpt8_wgrad(flat[:20], c, add=flat[20:20 + k], out=flat[21:21 + k])):
        with pytest.raises(nsml.NsmlError):
            call()
    torch.cuda.synchronize()
    assert torch.equal(flat, before)
