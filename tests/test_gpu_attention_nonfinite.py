"""Values that are not finite, one at a time and in one tensor alone, at every place of the first two tiles of keys or queries: whoever sees one shows it, in its
column at least, wherever it lies in a tile; whoever does not has the very bits of the run without it.

A pack holds a sequence for each place, all with the same contents but for the one value.  Runs of one sequence have their keys split."""
import math

import pytest
import torch

from attention_util import DEV, NAME, TYPES, inside, mask_of, reference
from paper_2506_16235_amd import binding as nsml
from test_gpu_attention import gen, offsets, say, tensor

pytestmark = pytest.mark.gpu
types = pytest.mark.parametrize("dt", TYPES, ids=NAME.get)
dims = pytest.mark.parametrize("dim", [64, 128])
groups = pytest.mark.parametrize("heads,kv", [(2, 2), (4, 2), (4, 1)])
VALUES = (math.nan, math.inf, -math.inf)
# queries, keys, causal, window: a prompt, no mask, a window, a chunk behind an odd number of keys, single tokens
SHAPES = [(256, 256, True, None), (200, 200, False, None), (256, 256, True, 70), (150, 283, True, None)]
TOKENS = [(1, 100, True, None), (1, 800, True, None), (2, 100, True, None), (1, 333, True, 100)]
shapes = pytest.mark.parametrize("m,n,causal,window", SHAPES)


class Pack:
    """Sequences alike, of m queries and n keys each."""

    def __init__(self, dt, dim, heads, kv, m, n, causal, window, places):
        c, g = len(places), gen(dim + m)
        self.m, self.n, self.c, self.places, self.group = m, n, c, places, heads // kv
        self.q, self.k, self.v, self.do = (tensor(g, r, h, dim, dt, "plain", s).repeat(c, 1, 1) for r, h, s in ((m, heads, 1.0), (n, kv, 1.0), (n, kv, 1.0), (m, heads, 0.01)))
        self.seqs, self.how = nsml.Seqs(offsets([m] * c), offsets([n] * c)), dict(causal=causal, window=window)
        self.clean = nsml.attention(self.q, self.k, self.v, self.seqs, **self.how)
        self.seen = mask_of(m, n, causal, window)
        self.col = [(7 * i + 3) % dim for i in range(c)]
        want, off = reference(self.q[:m], self.k[:n], self.v[:n], None, [(0, m, 0, n)], causal, window, dim ** -0.5, dt)
        for name in ("o", "lse"):
            inside(getattr(self.clean, name)[:m], want[name], off[name], name)

    def spoiled(self, t, rows, head):
        """t with a value that is not finite at the place of each sequence, in one head."""
        t = t.clone()
        for i, (at, col) in enumerate(zip(self.places, self.col)):
            t[i * rows + at, head, col] = VALUES[i % 3]
        return t

    def column(self, t, rows):
        """Of each sequence's part of t the column that was spoiled: [sequences, rows, heads]."""
        at = torch.tensor(self.col, device=DEV).view(-1, 1, 1, 1)
        return t.view(self.c, rows, *t.shape[1:]).gather(3, at.expand(self.c, rows, t.shape[1], 1))[..., 0]

    def shown(self, got, clean, rows, affected, what):
        """affected, [sequences, rows, heads]: not finite in the column; all else the bits of the clean run."""
        bad = affected & torch.isfinite(self.column(got, rows))
        assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {int(affected.sum())} lost, first at {tuple(int(x) for x in bad.nonzero()[0])}"
        self.kept(got, clean, rows, affected, what)

    def kept(self, got, clean, rows, affected, what):
        same = (got == clean).view(self.c, rows, got.shape[1], -1).all(3)
        assert bool((same | affected).all()), f"{what}: {int((~same & ~affected).sum())} differ"

    def of_head(self, seen, heads, hit):
        """seen [sequences, rows] for the heads that are hit."""
        which = torch.zeros(heads, dtype=torch.bool, device=DEV)
        which[hit] = True
        return seen[..., None] & which

    def who_sees(self):
        """[sequences, queries]: whether a query sees the key of the place."""
        return self.seen[:, self.places].t()

    def who_is_seen(self):
        """[sequences, keys]: whether the query of the place sees a key."""
        return self.seen[self.places]


def packs(n, more=()):
    """Every place of the first 128 rows in one pack, which is worked through in order; some of them in a pack that is not; the rest alone."""
    first = [*range(min(n, 128)), *more]
    return [first, first[1::3][-60:], *[[p] for p in (0, 31, 40, 63, 70, 95, 99, 127, *more[-1:]) if p < n]]


@types
@dims
@groups
@pytest.mark.parametrize("m,n,causal,window", SHAPES + TOKENS)
def test_a_value_shows_in_results(dt, dim, heads, kv, m, n, causal, window):
    for places in packs(n, range(max(128, n - 64), n)):
        p = Pack(dt, dim, heads, kv, m, n, causal, window, places)
        got = nsml.attention(p.q, p.k, p.spoiled(p.v, n, kv - 1), p.seqs, **p.how)
        p.shown(got.o, p.clean.o, m, p.of_head(p.who_sees(), heads, slice((kv - 1) * p.group, None)), f"o, {len(places)} sequences")


@types
@dims
@groups
@pytest.mark.parametrize("m,n,causal,window", SHAPES + TOKENS)
def test_a_value_has_no_part_in_lse(dt, dim, heads, kv, m, n, causal, window):
    """lse is made of scores alone."""
    for places in packs(n, range(max(128, n - 64), n)):
        p = Pack(dt, dim, heads, kv, m, n, causal, window, places)
        got = nsml.attention(p.q, p.k, p.spoiled(p.v, n, 0), p.seqs, **p.how)
        assert torch.equal(got.lse, p.clean.lse), (len(places), int((got.lse != p.clean.lse).sum()))


def gradients(p, **spoiled):
    """Of the clean run's result and lse, with one of its tensors spoiled."""
    t = {"do": p.do, "q": p.q, "k": p.k, "v": p.v, **spoiled}
    return nsml.attention_backward(t["do"], t["q"], t["k"], t["v"], *p.clean, p.seqs, **p.how)


@types
@dims
@groups
@shapes
@pytest.mark.parametrize("which", ["do", "q"])
def test_a_query_or_its_gradient_shows_in_the_gradients_of_keys(dt, dim, heads, kv, m, n, causal, window, which):
    for places in packs(m):
        p = Pack(dt, dim, heads, kv, m, n, causal, window, places)
        head = heads - 1
        clean, got = gradients(p), gradients(p, **{which: p.spoiled(getattr(p, which), m, head)})
        hit = p.of_head(p.who_is_seen(), kv, head // p.group)
        if which == "do":
            p.shown(got[2], clean[2], n, hit, "dv")
            p.kept(got[1], clean[1], n, hit, "dk")
        else:
            p.shown(got[1], clean[1], n, hit, "dk")
            p.kept(got[2], clean[2], n, hit, "dv")
        own = torch.zeros(p.c, m, dtype=torch.bool, device=DEV)
        own[range(p.c), places] = True
        p.kept(got[0], clean[0], m, p.of_head(own, heads, head), "dq")


@types
@dims
@groups
@shapes
@pytest.mark.parametrize("which", ["k", "v"])
def test_a_key_or_its_value_shows_in_the_gradient_of_queries(dt, dim, heads, kv, m, n, causal, window, which):
    for places in packs(n):
        p = Pack(dt, dim, heads, kv, m, n, causal, window, places)
        clean, got = gradients(p), gradients(p, **{which: p.spoiled(getattr(p, which), n, kv - 1)})
        p.shown(got[0], clean[0], m, p.of_head(p.who_sees(), heads, slice((kv - 1) * p.group, None)), "dq")


@types
@dims
@shapes
def test_a_value_goes_through_a_step(dt, dim, m, n, causal, window):
    """Forward and backward together: what belongs to queries that do not see it, and keys that none of those sees that do, stays."""
    p = Pack(dt, dim, 2, 2, m, n, causal, window, [*range(0, 128, 3)])
    v = p.spoiled(p.v, n, 1)
    r = nsml.attention(p.q, p.k, v, p.seqs, **p.how)
    got, clean = nsml.attention_backward(p.do, p.q, p.k, v, *r, p.seqs, **p.how), gradients(p)
    sees = p.who_sees()
    p.shown(got[0], clean[0], m, p.of_head(sees, 2, 1), "dq")
    with_it = (sees.double() @ p.seen.double()) > 0
    p.shown(got[1], clean[1], n, p.of_head(with_it, 2, 1), "dk")
    assert torch.equal(got[2], clean[2])                # the weights do not know of values
    say(NAME[dt], dim, m, n, int(sees.sum()), int(with_it.sum()))


@types
@pytest.mark.parametrize("n", [40, 5000])
def test_a_value_shows_where_every_weight_is_0(dt, n):
    """Scores of -infinity alone: weights of 0, of which the product with what is not finite is NaN, whether the keys are split or not."""
    q, k, v = tensor(gen(n), 1, 2, 64, dt).abs() + 0.1, tensor(gen(n + 1), n, 2, 64, dt), tensor(gen(n + 2), n, 2, 64, dt)
    k[:, :, 7] = -math.inf
    r = nsml.attention(q, k, v)
    assert bool((r.o == 0).all()) and bool((r.lse == -math.inf).all())
    v[n - 3, 1, 5] = math.inf
    o = nsml.attention(q, k, v).o
    assert bool(torch.isnan(o[0, 1, 5])) and bool((o[0, 0] == 0).all())
