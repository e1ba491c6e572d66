"""Codes the other way round, by the library's own kernel, byte for byte."""
import pytest
import torch

from paper_2506_16235_amd import binding as nsml

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def codes(m, k, gap=0, seed=0, fill=None):
    g = torch.Generator()
    g.manual_seed(seed + m * 3 + k)
    whole = torch.randint(-128, 128, (m, (k + 15) // 16 * 16 + gap), generator=g, dtype=torch.int8) if fill is None else \
        torch.full((m, (k + 15) // 16 * 16 + gap), fill, dtype=torch.int8)
    whole = whole.to(DEV)
    return whole, whole[:, :k]


@pytest.mark.parametrize("m,k", [(1, 1), (1, 300), (300, 1), (15, 16), (16, 17), (64, 64), (127, 129), (128, 128), (129, 127), (200, 1021), (1543, 1021),
                                 (2048, 768), (11008, 4096), (100, 70000), (70000, 33)])
def test_transposed(m, k):
    _, q = codes(m, k, 32)
    want = q.t().contiguous()
    t = nsml.q8_transposed(nsml.Q8(q, None))
    assert t.scale is None and t.q.shape == (k, m) and t.q.stride(0) % 16 == 0 and torch.equal(t.q, want)
    # into a part of something wider: nothing behind a row's own bytes is touched
    whole, out = codes(k, m, 48, fill=99)
    rc = nsml.raw().nsml_q8_transpose(q.data_ptr(), q.stride(0), m, k, out.data_ptr(), out.stride(0), torch.cuda.current_stream().cuda_stream)
    assert rc == nsml.OK and torch.equal(out, want) and (whole[:, (m + 15) // 16 * 16:] == 99).all()


def test_more_tiles_than_workgroups():
    """A workgroup takes more than one tile; offsets pass 2^32."""
    m, k = 128 * (1 << 20) + 300, 40
    q = torch.zeros(m, 48, dtype=torch.int8, device=DEV)[:, :k]
    _, tail = codes(1000, k)
    q[:500], q[-500:] = tail[:500], tail[500:]
    t = nsml.q8_transposed(nsml.Q8(q, None)).q
    assert torch.equal(t[:, :500], tail[:500].t()) and torch.equal(t[:, -500:], tail[500:].t())
    assert not bool(t[:, 500:-500].any())


def test_on_another_stream_and_in_a_graph():
    _, q = codes(300, 200)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        held = nsml.q8_transposed(nsml.Q8(q, None)).q
    for turn in range(3):
        q.copy_(codes(300, 200, seed=turn + 5)[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, q.t())
