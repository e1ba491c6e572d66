"""delta = do o has the rounding of o in it, e of it, and the gradient shows that where a query's weight is nearly all on one key: its ds are then far smaller than
e.  The sum of ds over a query's keys, 0 but for e, tells what e is.  So dk is made with a delta that is right in 32 bits; and dq too, unless e is
below two steps of the type, 4 U, of the root of the sum of ds^2 (of keys with normal scores it is 0.6 U in the mean square).

Bounds, beside those of attention_util (u, U, U16, the relative error of a weight w = 2 e_s + 8 u, e_s that of its score; line = (dim + 8) u sum |do|(|v| + |o|)):

  e          at most E = sum |do| bound(o)
  delta      (w + (n + 8) u) (sum p |dp - delta| + E) + the largest line, D: weights that do not quite add up to 1, a sum of n, dp and delta themselves
  ds         p ((w + U16) |dp - delta| + line + D)
  dq         scale sum bound(ds) |k| + scale sum p |k| 4 U |ds| / (1 - 4 U), |ds| the root of the sum; for heads of up to 64 elements, whose ds are rounded with e in them, which
             is taken off with weights that are rounded, scale sum p |k| 2 U E more; then as there
  dk         scale sum bound(ds) |q|, then as there
"""
import math

import pytest
import torch

from attention_util import DEV, HALF, NAME, inside, mask_of, u
from paper_2506_16235_amd import binding as nsml
from test_gpu_attention import gen, offsets, say

pytestmark = pytest.mark.gpu
types = pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16], ids=NAME.get)


def one_head(q, k, v, do, seen, scale, dt):
    """-> dq, dk and their bounds, and the median of the largest weights."""
    U, dim, (m, n) = HALF[dt], q.shape[1], seen.shape
    tiny, low = (2.0 ** -25, 2.0 ** -30) if dt == torch.float16 else (2.0 ** -140, 0.0)
    s = torch.where(seen, scale * (q @ k.t().contiguous()), -math.inf)
    p = torch.softmax(s, 1)
    off_s = torch.where(seen, (dim + 8) * u * scale * (q.abs() @ k.abs().t().contiguous()) + 4 * u * (torch.where(seen, s.abs(), 0.0) + s.amax(1, keepdim=True).abs()), 0.0)
    w = 2 * off_s.amax(1, keepdim=True) + 8 * u
    o, av = p @ v, p @ v.abs()
    off_o = (U + w + (n + 8) * u) * av + U * o.abs() + low * (seen.double() @ v.abs()) + tiny
    dp, delta = do @ v.t().contiguous(), (do * o).sum(1, keepdim=True)
    ds = torch.where(seen, p * (dp - delta), 0.0)
    line = torch.where(seen, (dim + 8) * u * (do.abs() @ v.abs().t().contiguous() + (do.abs() * o.abs()).sum(1, keepdim=True)), 0.0)
    E = (do.abs() * off_o).sum(1, keepdim=True)
    D = (w + (n + 8) * u) * (ds.abs().sum(1, keepdim=True) + E) + line.amax(1, keepdim=True)
    bad = torch.where(seen, p * ((w + U) * (dp - delta).abs() + line + D), 0.0)
    if low:
        bad = bad + seen * 2.0 ** -32 * float(ds.abs().max())
    root = ds.square().sum(1, keepdim=True).sqrt()
    more = 4 * U * root / (1 - 4 * U) + (2 * U * E if dim <= 64 else 0.0)
    dq, dk = scale * (ds @ k), scale * (ds.t().contiguous() @ q)
    off_q = scale * ((bad + (n + 8) * u * ds.abs() + more * p) @ k.abs()) + U * dq.abs() + tiny
    off_k = scale * ((bad + (m + 8) * u * ds.abs()).t().contiguous() @ q.abs())
    return dq, dk, off_q, off_k, float(p.amax(1).median())


def contents(g, lens, heads, kv, dim, dt, sink):
    """Keys with a mean, and in each sequence one of `sink` times that; queries that share its direction."""
    n = sum(lens)
    q, k, v, do = (torch.randn(n, h, dim, generator=g, device=DEV) for h in (heads, kv, kv, heads))
    k += 0.5
    for i in range(len(lens)):
        k[sum(lens[:i]) + lens[i] // 3] = sink
    # the sink's score is sink * sqrt(dim) * 0.25, the others' are around sqrt(dim) * 0.125
    q = 0.3 * q + 0.25
    return [x.to(dt) for x in (q, k, v, 0.01 * do)]


@types
@pytest.mark.parametrize("dim", [64, 96, 121, 128])
@pytest.mark.parametrize("lens,heads,kv,causal,window", [((200,), 2, 2, True, None), ((700,), 2, 1, False, None), ((1500,), 1, 1, True, None), ((530, 800), 4, 2, True, None),
                                                         ((1200,), 2, 2, True, 600), ((40, 3, 1100), 6, 2, False, None)])
@pytest.mark.parametrize("peak", [0.0, 5.0, 9.0])
def test_a_key_with_nearly_all_weight(dt, dim, lens, heads, kv, causal, window, peak):
    """peak: how far the sink's score lies above the others' (in natural units, about)."""
    scale, sink = dim ** -0.5, 0.5 + peak / (0.25 * dim ** 0.5)
    q, k, v, do = contents(gen(dim + sum(lens)), lens, heads, kv, dim, dt, sink)
    seqs, how = nsml.Seqs(offsets(lens)), dict(causal=causal, window=window)
    r = nsml.attention(q, k, v, seqs, **how)
    dq, dk, _ = nsml.attention_backward(do, q, k, v, r.o, r.lse, seqs, **how)
    torch.cuda.synchronize()
    worst, peaks = [0.0, 0.0], []
    tiny = 2.0 ** -25 if dt == torch.float16 else 2.0 ** -140
    for i, n in enumerate(lens):
        part, seen = slice(sum(lens[:i]), sum(lens[:i + 1])), mask_of(n, n, causal, window)
        for c in range(kv):
            kk, vv = (t[part, c].double().contiguous() for t in (k, v))
            sum_k = sum_off = 0.0
            for h in range(c * heads // kv, (c + 1) * heads // kv):
                a, b, off_a, off_b, top = one_head(q[part, h].double().contiguous(), kk, vv, do[part, h].double().contiguous(), seen, scale, dt)
                worst[0] = max(worst[0], inside(dq[part, h], a, off_a, f"dq of sequence {i}, head {h}"))
                sum_k, sum_off = sum_k + b, sum_off + off_b
                peaks.append(round(top, 4))
            worst[1] = max(worst[1], inside(dk[part, c], sum_k, sum_off * (1 + heads * u) + HALF[dt] * sum_k.abs() + tiny, f"dk of sequence {i}, head {c}"))
    say(NAME[dt], dim, lens, "weights", peaks[:3], "of the bounds: dq %.3f dk %.3f" % tuple(worst))
