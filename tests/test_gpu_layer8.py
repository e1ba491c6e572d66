"""The 8-bit layer's operators against their definitions in 64 bits (numpy on the host), at the sizes and contents where
they can go wrong.

Tolerances, derived beforehand.  u = 2^-24 (half a unit in the last place of binary32), U = 2^-8 (bfloat16), 2^-11 (float16): their units of rounding.
  codes of rows     t = x * col is one rounding, absmax / 127 one, t * inv two more: a code may differ from the exact one only
                    where the exact quotient is within 127 * 4u of a half; for inputs of 16 bits without col_scale t is exact
  checkpoints       exact: powers of two
  products          the sum is exact; at most four roundings (of the sum, two scales, bias), then the type's
  sums              n terms in binary32: error <= n * u * sum |terms| (far from reached), used with n = depth of the sum
"""
import numpy as np
import pytest
import torch

from paper_2506_16235_amd import binding as nsml

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
u32 = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
NAME = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}
types = pytest.mark.parametrize("dt", TYPES, ids=NAME.get)


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def acts(seed, m, k, dt=torch.float32, scale=1.0):
    g = gen(seed)
    x = torch.randn(m, k, generator=g) * torch.exp(0.5 * torch.randn(1, k, generator=g)) * scale
    return x.to(dt)


def strided(x, extra=0, shift=0):
    """x on the GPU with `extra` elements between rows and `shift` before the first; the gaps hold NaN."""
    m, k = x.shape
    flat = torch.full((shift + m * (k + extra) + 8,), float("nan"), dtype=x.dtype, device=DEV)
    v = flat[shift:shift + m * (k + extra)].view(m, k + extra)[:, :k]
    v.copy_(x)
    return v


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def padded_codes(q, fill=77):
    """int8 codes with a row stride that is a multiple of 16; what lies between rows is not zero."""
    m, k = q.shape
    out = torch.full((m, (k + 15) // 16 * 16 + 16), fill, dtype=torch.int8, device=DEV)
    out[:, :k] = q
    return out[:, :k]


# ---------------------------------------------------------------- definitions in 64 bits

def rows_ref(t):
    """t (float64 of binary32 values) -> codes, scales, and where a code may be either neighbour."""
    top = np.abs(t).max(1)
    bad = ~np.isfinite(t).all(1)
    zero = top < 2.0 ** -112
    with np.errstate(all="ignore"):
        scale = np.where(bad, np.nan, np.where(zero, 0.0, top / 127))
        x = np.where((bad | zero)[:, None], 0.0, t / np.where(zero | bad, 1.0, top / 127)[:, None])
    q = np.rint(x)
    return q, scale, np.abs(np.abs(x - np.floor(x)) - 0.5) < 127 * 8 * u32


def blocks_ref(x):
    m, k = x.shape
    nb = (k + 31) // 32
    full = np.zeros((m, nb * 32))
    full[:, :k] = x
    full = full.reshape(m, nb, 32)
    bad = ~np.isfinite(full).all(2)
    top = np.where(bad, 1.0, np.abs(np.where(np.isfinite(full), full, 0)).max(2))
    e = np.frexp(np.where(top == 0, 2.0 ** -200, top))[1] - 1 - 6 + 127
    e = np.where(bad, 255, np.maximum(e, 1))
    with np.errstate(all="ignore"):
        q = np.clip(np.rint(np.where(bad[:, :, None], 0.0, full) * np.exp2(127.0 - e)[:, :, None]), -127, 127)
        v = np.where(bad[:, :, None], np.nan, q * np.exp2(e - 127.0)[:, :, None])
    return q.reshape(m, -1)[:, :k], e, v.reshape(m, -1)[:, :k]


def same_codes(got, ref, either=None):
    d = np.abs(got.cpu().numpy().astype(np.int64) - ref)
    if either is not None:
        assert (d[either] <= 1).all()
        d = d[~either]
    assert (d == 0).all(), f"{int((d != 0).sum())} codes differ"


def close(got, ref, tol, floor=0.0):
    """|got - ref| <= tol * |ref| + floor elementwise, NaN where ref has NaN."""
    got = f64(got) if isinstance(got, torch.Tensor) else got
    assert (np.isnan(got) == np.isnan(ref)).all()
    ok = np.isfinite(ref)
    err = np.abs(got - ref)
    lim = tol * np.abs(ref) + floor
    bad = ok & ~(err <= lim)
    assert not bad.any(), f"{int(bad.sum())} of {ref.size} off, worst {np.nanmax(np.where(ok, err / np.maximum(lim, 1e-300), 0)):.3g} of the bound"
    assert (got[~ok & ~np.isnan(ref)] == ref[~ok & ~np.isnan(ref)]).all()


def same_values(got, want):
    """Equal, with NaN where the other has it."""
    got = got.cpu()
    return bool(((got == want) | (torch.isnan(got) & torch.isnan(want))).all())


WIDTHS = [1, 7, 8, 31, 33, 64, 127, 512, 513, 1021, 1024, 1030, 2048, 2056, 4096, 4100, 8192, 8200, 11008, 16384, 16392, 32768]


# ---------------------------------------------------------------- coding by rows

@types
@pytest.mark.parametrize("k", WIDTHS + [32776, 131072])
def test_rows(dt, k):
    m = 5 if k <= 4100 else 2
    x = acts(k, m, k, dt)
    x[0] = 0
    g = strided(x, 3, 1)
    r = nsml.q8_rows(g)
    q, s, either = rows_ref(f64(x))
    same_codes(r.q, q, either)
    close(r.scale, s, 2 * u32)
    v = nsml.q8_values(r, dt)
    with np.errstate(all="ignore"):
        close(v, r.q.cpu().numpy() * f64(r.scale)[:, None], HALF[dt] + 2 * u32, 2.0 ** -24 if dt == torch.float16 else 0)


@types
def test_rows_with_column_scales_and_special_rows(dt):
    m, k = 9, 777
    x, col = acts(3, m, k, dt), torch.exp(torch.randn(k, generator=gen(4)))
    x[1, 5], x[2, 776], x[3, 0] = float("inf"), float("nan"), float("-inf")
    x[4] = 0
    x[5] = torch.finfo(dt).tiny                     # below what is coded, in 32 and bfloat16
    x[6] = torch.finfo(dt).max / 512
    x[7] = -x[7].abs()
    r = nsml.q8_rows(x.to(DEV), col.to(DEV))
    t = (x.float() * col).double().numpy()
    q, s, either = rows_ref(t)
    same_codes(r.q, q, either)
    close(r.scale, s, 3 * u32)
    v = nsml.q8_values(r)
    assert torch.isnan(v[1:4]).all() and torch.isfinite(v[4:]).all() and torch.isfinite(v[0]).all()
    assert (v[4] == 0).all()
    if dt != torch.float16:
        assert (v[5] == 0).all()


# ---------------------------------------------------------------- checkpoints

@types
@pytest.mark.parametrize("m,k", [(1, 1), (3, 31), (2, 32), (5, 33), (300, 64), (7, 1000), (129, 2049), (4, 11008), (70000, 5)])
def test_checkpoint_is_exact(dt, m, k):
    x = acts(m + k, m, k, dt) * torch.exp2(torch.randint(-20, 14, (m, 1), generator=gen(9)).float()).to(dt)
    if k > 8:
        x[0, 1:k // 2] = 0
    c = nsml.ckpt8_pack(strided(x, 5, 3))
    q, e, v = blocks_ref(f64(x))
    same_codes(c.q, q)
    assert (c.e.cpu().numpy() == e).all()
    for to in TYPES:
        y = nsml.ckpt8_unpack(c, to)
        want = torch.from_numpy(v).float().to(to)       # exact in bfloat16 and binary32
        assert same_values(y, want)
    out = strided(torch.zeros(m, k), 7, 1)
    nsml.ckpt8_unpack(c, out=out)
    assert same_values(out.double(), torch.from_numpy(v))


def test_checkpoint_of_extremes():
    big, sub = torch.finfo(torch.float32).max, 2.0 ** -149
    rows = [[0.0] * 70, [big] * 70, [sub] * 70, [2.0 ** -126] * 70, [127.49, 127.5, 127.51, -127.9] + [1.0] * 66,
            [63.999, -64.0, 0.5, 1.5, 2.5, -0.5] + [0.25] * 64, [-0.0] * 70]
    x = torch.tensor(rows)
    x = torch.cat([x, x])
    x[7, 40], x[8, 0], x[9, 69], x[10, 31] = float("nan"), float("inf"), float("-inf"), float("nan")
    c = nsml.ckpt8_pack(x.to(DEV))
    q, e, v = blocks_ref(f64(x))
    same_codes(c.q, q)
    assert (c.e.cpu().numpy() == e).all()
    y = nsml.ckpt8_unpack(c).cpu().double().numpy()
    assert (np.isnan(y) == np.isnan(v)).all() and (y[~np.isnan(v)] == v[~np.isnan(v)]).all()


# ---------------------------------------------------------------- products

def product_ref(qa, sa, qb, sb, bias):
    c = qa.astype(np.float64) @ qb.astype(np.float64).T          # exact: below 2^53
    c = c * sa[:, None] * (1.0 if sb is None else sb)
    return c if bias is None else c + bias


def product_case(m, n, k, dt, seed=0, with_b=True, with_bias=True):
    g = gen(seed + m * 7 + n * 3 + k)
    qa, qb = (torch.randint(-127, 128, (r, k), generator=g, dtype=torch.int8) for r in (m, n))
    sa, sb, bias = torch.rand(m, generator=g) + 0.1, torch.rand(n, generator=g) * 0.01 + 1e-3, torch.randn(n, generator=g)
    out = strided(torch.full((m, n), 7.0, dtype=dt), 3, 1)
    A = nsml.Q8(padded_codes(qa), sa.to(DEV))
    B = nsml.Q8(padded_codes(qb), sb.to(DEV) if with_b else None)
    got = nsml.q8_matmul(A, B, bias=bias.to(DEV) if with_bias else None, out=out)
    whole = out.as_strided((m, n + 3), (n + 3, 1))
    ref = product_ref(qa.numpy(), sa.double().numpy(), qb.numpy(), sb.double().numpy() if with_b else None,
                      bias.double().numpy() if with_bias else None)
    mid = np.abs(product_ref(qa.numpy(), sa.double().numpy(), qb.numpy(), sb.double().numpy() if with_b else None, None))
    if dt == torch.float16:
        ok = np.abs(ref) < 65000
        ref, got = np.where(ok, ref, 0), np.where(ok, f64(got), 0)
    close(got, ref, HALF[dt] + u32, 4 * u32 * mid + (2.0 ** -25 if dt == torch.float16 else 0))
    assert m < 2 or torch.isnan(whole[:-1, n:]).all(), "written between rows"


@types
@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 32, 33, 64, 65, 100, 128, 129, 256, 300])
@pytest.mark.parametrize("n,k", [(1, 1), (17, 63), (64, 64), (100, 129), (33, 255), (16, 4096), (130, 1000), (257, 272)])
def test_product(dt, m, n, k):
    product_case(m, n, k, dt, 1, with_b=(m + n) % 2 == 0, with_bias=(m + k) % 2 == 0)


@pytest.mark.parametrize("m,n,k", [(1, 11008, 4096), (48, 4096, 11008), (1000, 1543, 1021), (2048, 2048, 384), (2049, 4100, 130),
                                   (4096, 5000, 513), (3, 40, 131072), (70, 65, 131072), (5000, 130, 100), (520, 9000, 1031)])
def test_product_large(m, n, k):
    product_case(m, n, k, torch.float32, 2)


def test_product_of_the_largest_sums():
    """127 * 127 * 131072 in every place: the sum is whole and fits."""
    for m in (2, 100):
        k = nsml.Q8_MAX_COLS
        a = torch.full((m, k), 127, dtype=torch.int8, device=DEV)
        b = torch.cat([a[:1], -a[:1]]).contiguous()
        one = torch.ones(m, device=DEV)
        c = nsml.q8_matmul(nsml.Q8(a, one), nsml.Q8(b, None), torch.float32)
        assert (c[:, 0].double() == np.float32(127 * 127 * k)).all() and (c[:, 1] == -c[:, 0]).all()


@pytest.mark.parametrize("m", [3, 100, 400])
def test_product_keeps_bad_rows_apart(m):
    """A row of scale NaN and an output channel of scale infinity reach their own row and column only."""
    g = gen(5)
    a, b = torch.randint(-127, 128, (m, 100), generator=g, dtype=torch.int8), torch.randint(-127, 128, (70, 100), generator=g, dtype=torch.int8)
    sa, sb = torch.ones(m), torch.ones(70)
    sa[1], sb[7], sa[2] = float("nan"), float("nan"), 0.0
    c = nsml.q8_matmul(nsml.Q8(padded_codes(a), sa.to(DEV)), nsml.Q8(padded_codes(b), sb.to(DEV)), torch.float32).cpu()
    bad = torch.zeros(m, 70, dtype=torch.bool)
    bad[1], bad[:, 7] = True, True
    assert torch.equal(torch.isnan(c), bad)
    assert (c[2][~bad[2]] == 0).all()


# ---------------------------------------------------------------- weight gradient

def wgrad_case(m, n, k, dt, col=True, add="apart", seed=0):
    g = gen(seed + m + n + k)
    dy = (torch.randn(m, n, generator=g) * 1e-3 * torch.exp(torch.randn(m, 1, generator=g))).to(dt)
    x = acts(seed + 1, m, k) if m else torch.zeros(0, k)
    if m > 3:
        dy[3], x[2] = 0, 0
    q, e, v = blocks_ref(x.double().numpy()) if m else (np.zeros((0, k)), np.zeros((0, (k + 31) // 32)), np.zeros((0, k)))
    c = nsml.Ckpt8(padded_codes(torch.from_numpy(q).to(torch.int8)), torch.from_numpy(e).to(torch.uint8).to(DEV))
    gam = 1 + 0.3 * torch.randn(k, generator=g) if col else None
    base = torch.randn(n, k, generator=g) * 1e-3 if add else None
    out = strided(torch.full((n, k), 7.0), 5, 1)
    kw = {"col_scale": gam.to(DEV) if col else None, "out": out}
    if add == "apart":
        kw["add"] = strided(base, 5, 3)
    elif add == "self":
        out.copy_(base)
        kw["add"] = out
    got = nsml.ckpt8_wgrad(strided(dy, 1, 1) if m else dy.to(DEV), c, **kw)
    d = f64(dy)
    ref = d.T @ v * (f64(gam) if col else 1.0) + (f64(base) if add else 0.0)
    size = np.abs(d).T @ np.abs(v) * (np.abs(f64(gam)) if col else 1.0)
    # a random walk of rounding errors: sqrt(depth) * u of the terms' sum is already generous, the split into parts adds two
    close(got, ref, 4 * u32, (4 + 2 * np.sqrt(m)) * u32 * size)
    whole = out.as_strided((n, k + 5), (k + 5, 1))
    assert n < 2 or torch.isnan(whole[:-1, k:]).all(), "written between rows"


@types
@pytest.mark.parametrize("m,n,k", [(0, 5, 40), (1, 1, 1), (1, 130, 33), (7, 8, 64), (63, 100, 31), (64, 128, 128), (65, 129, 130), (200, 257, 96),
                                   (1027, 64, 65), (1000, 1, 300), (513, 300, 1), (130, 768, 770)])
def test_wgrad(dt, m, n, k):
    wgrad_case(m, n, k, dt, col=(n + k) % 2 == 0, add=("apart", "self", None)[(m + n) % 3])


@types
def test_wgrad_larger(dt):
    wgrad_case(1500, 700, 1100, dt, seed=3)


def test_wgrad_many_rows():
    wgrad_case(40000, 70, 100, torch.bfloat16, seed=4, add=None)


@types
def test_wgrad_of_infinities(dt):
    """An infinity or NaN in dy reaches its output channel, a bad block of the checkpoint its 32 columns, nothing else."""
    m, n, k = 100, 70, 100
    dy, x = (torch.randn(m, n, generator=gen(1)) * 0.1).to(dt), acts(2, m, k) + 3.0
    dy[5, 7], dy[6, 9] = float("inf"), float("nan")
    x[8, 40] = float("nan")
    got = nsml.ckpt8_wgrad(dy.to(DEV), nsml.ckpt8_pack(x.to(DEV))).cpu()
    bad = torch.zeros(n, k, dtype=torch.bool)
    bad[7], bad[9], bad[:, 32:64] = True, True, True
    assert not torch.isfinite(got[bad]).any()
    assert torch.isfinite(got[~bad]).all()


def test_wgrad_twice_is_the_same():
    dy, x = (torch.randn(777, 300, generator=gen(1)) * 1e-3).bfloat16().to(DEV), acts(2, 777, 200).to(DEV)
    c = nsml.ckpt8_pack(x)
    a, b = nsml.ckpt8_wgrad(dy, c), nsml.ckpt8_wgrad(dy, c)
    assert torch.equal(a, b)


# ---------------------------------------------------------------- norm

def norm_ref(x, r, gamma, eps, dt):
    h = x.double().numpy() if r is None else (x.float() + r.float()).to(dt).double().numpy()
    rstd = 1 / np.sqrt((h * h).mean(1) + eps)
    return h, rstd, h if gamma is None else (torch.from_numpy(h).float() * gamma).double().numpy()


@types
@pytest.mark.parametrize("k", WIDTHS)
def test_norm(dt, k):
    m = 5 if k <= 4100 else 2
    x, r, gamma = acts(k, m, k, dt), acts(k + 1, m, k, dt), 1 + 0.3 * torch.randn(k, generator=gen(k))
    x[1], r[1] = 0, 0
    res = k % 2 == 0
    o = nsml.rmsnorm_q8(strided(x, 3, 1), gamma.to(DEV), 1e-5, residual=strided(r, 1, 1) if res else None, checkpoint=True)
    h, rstd, t = norm_ref(x, r if res else None, gamma, 1e-5, dt)
    assert (f64(o.h) == h).all()
    close(o.rstd, rstd, (8 + np.sqrt(k)) * u32)
    q, s, either = rows_ref(t)
    same_codes(o.y.q, q, either)
    close(o.y.scale, s * rstd, (12 + np.sqrt(k)) * u32)
    # the checkpoint is that of h * rstd as rounded: a value may fall to the other side of a half, or of a power of two
    v = h * rstd[:, None]
    _, e, _ = blocks_ref(v)
    step = np.exp2(np.repeat(np.maximum(e, 1), 32, 1)[:, :k] - 127.0)
    got = f64(nsml.ckpt8_unpack(o.xhat))
    assert (np.abs(got - v) <= 0.5 * step * (1 + 1e-4) + (np.abs(v) > 126.99 * step) * step).all()
    assert (np.abs(o.xhat.e.cpu().numpy().astype(int) - e) <= 1).all()


@types
def test_norm_special_rows(dt):
    m, k = 8, 333
    x = acts(1, m, k, dt)
    x[0, 3], x[1, 3], x[2, 3] = float("nan"), float("inf"), float("-inf")
    x[3] = 0
    x[4] = 0
    x[4, 9] = 1
    o = nsml.rmsnorm_q8(x.to(DEV), None, 0.0, checkpoint=True)
    y = nsml.q8_values(o.y)
    assert torch.isnan(y[:3]).all() and torch.isfinite(y[4:]).all()
    ok = [4, 5, 6, 7]
    h, rstd, t = norm_ref(x[ok], None, None, 0.0, dt)
    q, s, either = rows_ref(t)
    same_codes(o.y.q[ok], q, either)
    close(o.y.scale[ok], s * rstd, 40 * u32)
    xh = nsml.ckpt8_unpack(o.xhat)
    assert torch.isnan(xh[0]).all() and torch.isnan(xh[1, :32]).all() and torch.isfinite(xh[4:]).all()


def back_ref(dy, xh, rstd, gamma, dres):
    g = dy if gamma is None else dy * gamma
    return rstd[:, None] * (g - xh * (g * xh).mean(1, keepdims=True)) + (0 if dres is None else dres)


@types
@pytest.mark.parametrize("k", WIDTHS)
@pytest.mark.parametrize("m", [1, 6, 700])
def test_norm_backward(dt, k, m):
    if m * k > 3000000:
        m = 40
    g = gen(k)
    x = acts(k, m, k)
    rstd = 1 / torch.sqrt(x.square().mean(1) + 1e-5)
    c = nsml.ckpt8_pack((x * rstd[:, None]).to(DEV))
    xh = f64(nsml.ckpt8_unpack(c))
    dy, dres = (torch.randn(m, k, generator=g) * 1e-2).to(dt), (torch.randn(m, k, generator=g) * 1e-2).to(dt)
    gamma = 1 + 0.3 * torch.randn(k, generator=g) if k % 2 else None
    res = k % 3 != 0
    dx, dgamma = nsml.rmsnorm_backward(strided(dy, 3, 1), c, rstd.to(DEV), None if gamma is None else gamma.to(DEV),
                                       dres=strided(dres, 1, 1) if res else None, out=strided(torch.zeros(m, k, dtype=dt), 5, 1))
    ga = None if gamma is None else f64(gamma)
    ref = back_ref(f64(dy), xh, f64(rstd), ga, f64(dres) if res else None)
    gg = np.abs(f64(dy) * (1 if ga is None else ga))
    size = f64(rstd)[:, None] * (gg + np.abs(xh) * (gg * np.abs(xh)).mean(1, keepdims=True)) + (np.abs(f64(dres)) if res else 0)
    close(dx, ref, HALF[dt], (8 + np.sqrt(k)) * u32 * size + (2.0 ** -25 if dt == torch.float16 else 0))
    close(dgamma, (f64(dy) * xh).sum(0), 0, (4 + np.sqrt(m)) * u32 * (np.abs(f64(dy)) * np.abs(xh)).sum(0) + 1e-300)


def test_norm_backward_against_differences():
    """The gradient of sum(w * gamma * norm(x)), by central differences in 64 bits at points that a checkpoint holds exactly."""
    m, k, eps = 3, 96, 1e-5
    g = gen(11)
    x = torch.randint(-127, 128, (m, k), generator=g).double() / 32
    w, gamma = torch.randn(m, k, generator=g), 1 + 0.3 * torch.randn(k, generator=g)

    def f(v, ga):
        return (w.double() * ga * v / torch.sqrt(v.square().mean(1, keepdim=True) + eps)).sum()

    rstd = 1 / torch.sqrt(x.square().mean(1) + eps)
    # eps enters the derivative through rstd alone: x-hat is x * rstd
    xh = nsml.ckpt8_pack((x * rstd[:, None]).float().to(DEV))
    err = np.abs(f64(nsml.ckpt8_unpack(xh)) - (x * rstd[:, None]).numpy()).max()
    dx, dgamma = nsml.rmsnorm_backward(w.to(DEV), xh, rstd.float().to(DEV), gamma.to(DEV))
    step = 1e-6
    for i, j in ((0, 0), (0, 95), (1, 31), (2, 32), (2, 64)):
        d = torch.zeros_like(x)
        d[i, j] = step
        num = (f(x + d, gamma.double()) - f(x - d, gamma.double())) / (2 * step)
        # the checkpoint's error enters through x-hat times the mean and the mean itself
        lim = float(rstd[i]) * err * (float((w[i] * gamma).abs().mean()) * 8 + float((w[i] * gamma).norm()) / k * 8)
        assert abs(float(dx[i, j]) - float(num)) <= lim + 1e-5
    for j in (0, 50, 95):
        d = torch.zeros(k, dtype=torch.float64)
        d[j] = step
        num = (f(x, gamma.double() + d) - f(x, gamma.double() - d)) / (2 * step)
        assert abs(float(dgamma[j]) - float(num)) <= err * float(w[:, j].abs().sum()) + 1e-6


def test_norm_backward_of_no_rows():
    c = nsml.Ckpt8(torch.empty(0, 48, dtype=torch.int8, device=DEV), torch.empty(0, 2, dtype=torch.uint8, device=DEV))
    dx, dgamma = nsml.rmsnorm_backward(torch.empty(0, 48, device=DEV), c, torch.empty(0, device=DEV), dgamma=torch.full((48,), 3.0, device=DEV))
    assert dx.shape == (0, 48) and (dgamma == 0).all()


# ---------------------------------------------------------------- gated activation

def glu64(g, u):
    with np.errstate(over="ignore"):
        s = 1 / (1 + np.exp(-g))
    return s, g * s * u


@types
@pytest.mark.parametrize("k", WIDTHS + [32776])
def test_swiglu(dt, k):
    m = 4 if k <= 4100 else 2
    gate, up = acts(k, m, k, dt, 2.0), acts(k + 5, m, k, dt)
    gate[0, 0], gate[0, k // 2] = 100.0, -100.0
    gate[1] = 0
    o = nsml.swiglu_q8(strided(gate, 3, 1), strided(up, 1, 1), checkpoint=True)
    _, a = glu64(f64(gate), f64(up))
    # a's own error: product with log2 e and exponential |g| * 2u + 2u, reciprocal and two products 4u
    rel = (8 + 2 * np.abs(f64(gate))) * u32
    q, s, _ = rows_ref(a)
    close(o.a.scale, s, 2.0 ** -16)
    step = np.where(s == 0, 1, s)[:, None]
    exact = np.where(s[:, None] == 0, 0, a / step)
    assert (np.abs(o.a.q.cpu().numpy() - exact) <= 0.5 + np.abs(exact) * (rel + 2.0 ** -15)).all()
    for c, want in ((o.gate, gate), (o.up, up)):
        q, e, _ = blocks_ref(f64(want))
        same_codes(c.q, q)
        assert (c.e.cpu().numpy() == e).all()
    _, e, _ = blocks_ref(a)
    st = np.exp2(np.repeat(np.maximum(e, 1), 32, 1)[:, :k] - 127.0)
    got = f64(nsml.ckpt8_unpack(o.held))
    assert (np.abs(got - a) <= 0.5 * st * (1 + 2.0 ** -10) + (np.abs(a) > 126.9 * st) * st).all()
    plain = nsml.swiglu_q8(gate.to(DEV), up.to(DEV))
    assert plain.gate is None and torch.equal(plain.a.q, o.a.q) and torch.equal(plain.a.scale, o.a.scale)


@types
@pytest.mark.parametrize("m,k", [(1, 1), (3, 33), (70, 100), (9, 4097), (2, 11008)])
def test_swiglu_backward(dt, m, k):
    gate, up = acts(k, m, k, dt, 2.0), acts(k + 5, m, k, dt)
    gate[0, 0] = 60.0
    da = (torch.randn(m, k, generator=gen(k)) * 1e-2).to(dt)
    kg, ku = nsml.ckpt8_pack(gate.to(DEV)), nsml.ckpt8_pack(up.to(DEV))
    both = torch.full((m, 2 * k + 3), 9.0, dtype=dt, device=DEV)
    dg, du = nsml.swiglu_backward(strided(da, 3, 1), kg, ku, dgate=both[:, :k], dup=both[:, k:2 * k])
    g, u, d = f64(nsml.ckpt8_unpack(kg)), f64(nsml.ckpt8_unpack(ku)), f64(da)
    s, _ = glu64(g, u)
    rel = (12 + 2 * np.abs(g)) * u32
    floor = 2.0 ** -25 if dt == torch.float16 else 1e-37
    close(du, d * g * s, HALF[dt], rel * np.abs(d * g * s) + floor)
    size = np.abs(d * u * s) * (1 + np.abs(g) * (1 - s + u32 * 4))
    close(dg, d * u * s * (1 + g * (1 - s)), HALF[dt], 2 * rel * size + floor)
    assert (both[:, 2 * k:] == 9).all()


def test_swiglu_gradient_against_differences():
    g = torch.tensor([[-8.0, -2.0, -1.0, -0.25, 0.0, 0.25, 1.0, 2.0, 4.0, 8.0]])          # held exactly: eighths up to 8
    u = torch.tensor([[1.0, -2.0, 0.5, 3.0, 1.0, -1.0, 2.0, 0.25, 1.5, -1.0]])
    da = torch.tensor([[1.0, 0.5, -1.0, 2.0, 1.0, 1.0, -0.5, 1.0, 1.0, 2.0]])
    kg, ku = nsml.ckpt8_pack(g.to(DEV)), nsml.ckpt8_pack(u.to(DEV))
    assert torch.equal(nsml.ckpt8_unpack(kg).cpu(), g) and torch.equal(nsml.ckpt8_unpack(ku).cpu(), u)
    dg, du = nsml.swiglu_backward(da.to(DEV), kg, ku)
    h = 1e-5
    num_g = (glu64(f64(g) + h, f64(u))[1] - glu64(f64(g) - h, f64(u))[1]) / (2 * h) * f64(da)
    num_u = (glu64(f64(g), f64(u) + h)[1] - glu64(f64(g), f64(u) - h)[1]) / (2 * h) * f64(da)
    assert np.abs(f64(dg) - num_g).max() < 2e-6 and np.abs(f64(du) - num_u).max() < 2e-6


# ---------------------------------------------------------------- calls as a program makes them

def test_no_rows_at_all():
    x = torch.empty(0, 40, dtype=torch.bfloat16, device=DEV)
    assert nsml.q8_values(nsml.q8_rows(x)).shape == (0, 40)
    assert nsml.ckpt8_unpack(nsml.ckpt8_pack(x)).shape == (0, 40)
    o = nsml.rmsnorm_q8(x, torch.ones(40, device=DEV), residual=x, checkpoint=True)
    w = nsml.q8_rows(torch.ones(24, 40, device=DEV))
    assert nsml.q8_transposed(w).q.shape == (40, 24)
    assert nsml.q8_matmul(o.y, w).shape == (0, 24)
    s = nsml.swiglu_q8(x, x, checkpoint=True)
    assert nsml.swiglu_backward(x, s.gate, s.up)[0].shape == (0, 40)
    torch.cuda.synchronize()


def test_on_another_stream_and_in_a_graph():
    m, n, k = 70, 96, 128
    x, gamma = acts(1, m, k, torch.bfloat16).to(DEV), torch.ones(k, device=DEV)
    w = nsml.q8_rows(acts(2, n, k).to(DEV))
    dy = (torch.randn(m, n, generator=gen(3)) * 1e-3).bfloat16().to(DEV)

    def step():
        o = nsml.rmsnorm_q8(x, gamma, residual=x, checkpoint=True)
        c = nsml.q8_matmul(o.y, w)
        dw = nsml.ckpt8_wgrad(dy, o.xhat, gamma)
        dx, dg = nsml.rmsnorm_backward(o.h, o.xhat, o.rstd, gamma)
        return [c, dw, dx, dg]

    want = [t.clone() for t in step()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        held = step()
    for turn in range(3):
        x.copy_(acts(10 + turn, m, k, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, step()))


# ---------------------------------------------------------------- both sides of the sizes at which another launch is chosen

@pytest.mark.parametrize("m,n,k", [(10, 6000, 70), (10, 20000, 300), (16, 24500, 48), (16, 24600, 48), (20, 6000, 520), (20, 9000, 257), (32, 20000, 1030),
                                   (33, 8100, 300), (40, 6000, 515), (48, 8200, 100), (60, 6000, 999), (64, 8128, 40), (64, 8130, 1100),
                                   (65, 4096, 100), (70, 2000, 333), (1000, 300, 64), (1030, 200, 64), (1000, 2600, 200), (1000, 2400, 81),
                                   (3000, 3600, 140), (2500, 2500, 65), (2300, 2500, 127), (5100, 1290, 190)])
def test_product_at_every_launch(m, n, k):
    product_case(m, n, k, TYPES[(m + n + k) % 3], 3, with_b=n % 3 != 0, with_bias=k % 2 == 0)


@types
@pytest.mark.parametrize("m,n,k", [(2560, 2560, 192), (2500, 4096, 130), (4096, 4096, 77)])
def test_product_whole_lines(dt, m, n, k):
    """Large results whose rows are whole lines take another kind of store."""
    g = gen(m + k)
    a, b = torch.randint(-127, 128, (m, k), generator=g, dtype=torch.int8), torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8)
    sa, sb = torch.rand(m, generator=g) + 0.1, torch.rand(n, generator=g) * 0.01 + 1e-3
    c = nsml.q8_matmul(nsml.Q8(padded_codes(a), sa.to(DEV)), nsml.Q8(padded_codes(b), sb.to(DEV)), dt)
    ref = (a.to(DEV).double() @ b.to(DEV).double().t().contiguous()) * sa.to(DEV).double()[:, None] * sb.to(DEV).double()
    lim = (HALF[dt] + 4 * u32) * ref.abs() + (2.0 ** -25 if dt == torch.float16 else 0)
    assert bool(((c.double() - ref).abs() <= lim).all())


@pytest.mark.parametrize("m,n,k,col,add", [(70, 2944, 3328, True, None), (200, 3001, 3300, False, "apart"), (64, 3100, 2950, True, "self"),
                                           (130, 2048, 4096, True, "apart"), (130, 2304, 4096, False, None), (1, 3000, 3001, True, None)])
def test_wgrad_large_tiles(m, n, k, col, add):
    wgrad_case(m, n, k, torch.bfloat16, col=col, add=add, seed=6)


def test_wgrad_whole_lines_and_a_second_call():
    m, n, k = 320, 3200, 3200
    dy, x = (torch.randn(m, n, generator=gen(1)) * 1e-3).bfloat16().to(DEV), acts(2, m, k).to(DEV)
    c = nsml.ckpt8_pack(x)
    dw = nsml.ckpt8_wgrad(dy, c)
    v = nsml.ckpt8_unpack(c).double()
    ref, size = dy.double().t().contiguous() @ v, dy.double().abs().t().contiguous() @ v.abs()
    assert bool(((dw.double() - ref).abs() <= 4 * u32 * ref.abs() + (4 + 2 * m ** 0.5) * u32 * size).all())
    both = nsml.ckpt8_wgrad(dy, c, add=dw, out=dw)
    assert both is dw and bool(((dw.double() - 2 * ref).abs() <= 8 * u32 * ref.abs() + (8 + 4 * m ** 0.5) * u32 * size).all())


def test_rows_beyond_32_bits_of_bytes():
    """Offsets of a long matrix pass 2^32."""
    m, k = (1 << 32) // 4096 + 70, 4096
    x = torch.zeros(m, k, dtype=torch.bfloat16, device=DEV)
    tail = acts(1, 100, k, torch.bfloat16).to(DEV)
    x[-100:] = tail
    c, q = nsml.ckpt8_pack(x), nsml.q8_rows(x)
    ct, qt = nsml.ckpt8_pack(tail), nsml.q8_rows(tail)
    assert torch.equal(c.q[-100:], ct.q) and torch.equal(c.e[-100:], ct.e) and torch.equal(q.q[-100:], qt.q) and torch.equal(q.scale[-100:], qt.scale)
    w = nsml.q8_rows(acts(2, 40, k).to(DEV))
    assert torch.equal(nsml.q8_matmul(q, w)[-100:], nsml.q8_matmul(qt, w))
    dy = torch.zeros(m, 8, dtype=torch.bfloat16, device=DEV)
    dy[-100:] = torch.randn(100, 8, generator=gen(3)).to(torch.bfloat16).to(DEV)
    a, b = nsml.ckpt8_wgrad(dy, c), nsml.ckpt8_wgrad(dy[-100:], ct)
    assert bool(((a - b).abs() <= 64 * u32 * (dy[-100:].float().abs().t().contiguous() @ nsml.ckpt8_unpack(ct).abs())).all())


@types
@pytest.mark.parametrize("m,n,k", [(33, 3, 33000), (40, 1, 65700), (64, 100, 34000), (20, 34000, 3), (70, 33100, 60)])
def test_wgrad_long_and_narrow(dt, m, n, k):
    """Many tiles of a matrix with few rows or columns."""
    wgrad_case(m, n, k, dt, col=n < k, add=None, seed=7)


@pytest.mark.parametrize("dt", [torch.float16, torch.float32], ids=["f16", "f32"])
@pytest.mark.parametrize("m,n,k,col,add", [(70, 2944, 3328, True, None), (201, 3001, 3300, False, "apart"), (32, 3100, 2950, True, "self"), (1, 3000, 3001, True, None)])
def test_wgrad_large_tiles_in_parts(dt, m, n, k, col, add):
    wgrad_case(m, n, k, dt, col=col, add=add, seed=8)


@types
@pytest.mark.parametrize("m,n,k", [(3501, 3001, 900), (2100, 1300, 1100), (4001, 300, 1100), (700, 3000, 520), (3000, 129, 140), (3333, 1030, 260)])
def test_wgrad_slices(dt, m, n, k):
    """Slices of the rows that do not divide them, of tiles of both sides."""
    wgrad_case(m, n, k, dt, col=k % 3 == 1, add="apart" if n % 2 else None, seed=9)


@pytest.mark.parametrize("m,n,k", [(70, 19300, 700), (20000, 61, 700), (20000, 100, 700), (2300, 1177, 71), (130, 2000, 400), (260, 1300, 384), (260, 1300, 385),
                                   (5600, 704, 97), (279, 6592, 641), (4900, 900, 700), (19000, 150, 650)])
def test_product_at_more_launches(m, n, k):
    product_case(m, n, k, TYPES[(m + n + k) % 3], 3, with_b=n % 3 != 0, with_bias=k % 2 == 0)
