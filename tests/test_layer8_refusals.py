"""What the 8-bit layer's entry points and their binding refuse, before any kernel is launched (no GPU needed: the library's own
checks come before its first HIP call, and CPU tensors stand in for device tensors in the binding's)."""
import ctypes as C

import pytest
import torch

from paper_2506_16235_amd import binding as nsml

L = nsml.raw()
P = 1 << 12                 # an address that is aligned to everything; nothing is read from it


def ck(q=P, e=P, ldq=64, lde=2):
    return C.byref(nsml._CkptArg(q, e, ldq, lde))


def refused(rc, code=None):
    assert rc == (nsml.EINVAL if code is None else code)


def test_rows_and_values():
    def rows(x=P, type=0, ldx=64, m=3, k=64, col=None, q=P, ldq=64, s=P):
        return L.nsml_q8_rows(x, type, ldx, m, k, col, q, ldq, s, None)
    for bad in ({"x": None}, {"x": P + 2}, {"type": 3}, {"type": -1}, {"ldx": 63}, {"k": 0}, {"col": P + 1}, {"q": None}, {"q": P + 8},
                {"ldq": 72}, {"ldq": 48}, {"s": None}, {"s": P + 2}):
        refused(rows(**bad))
    refused(rows(k=131073, ldx=1 << 20, ldq=1 << 20), nsml.ECAP)

    def values(q=P, ldq=64, s=P, m=3, k=64, out=P, type=1, ldo=64):
        return L.nsml_q8_values(q, ldq, s, m, k, out, type, ldo, None)
    for bad in ({"q": None}, {"ldq": 65}, {"s": P + 1}, {"k": 0}, {"out": None}, {"out": P + 1}, {"type": 9}, {"ldo": 10}):
        refused(values(**bad))
    refused(values(k=(1 << 32) - 1, ldq=1 << 32, ldo=1 << 32), nsml.ECAP)


def test_matmul():
    def mm(a=P, lda=64, sa=P, b=P, ldb=64, sb=P, bias=None, m=3, n=5, k=64, c=P, type=1, ldc=5):
        return L.nsml_q8_matmul(a, lda, sa, b, ldb, sb, bias, m, n, k, c, type, ldc, None)
    for bad in ({"a": None}, {"a": P + 4}, {"lda": 60}, {"sa": None}, {"b": None}, {"ldb": 63}, {"sb": P + 2}, {"bias": P + 3}, {"n": 0},
                {"k": 0}, {"c": None}, {"c": P + 1}, {"type": 5}, {"ldc": 4}):
        refused(mm(**bad))
    refused(mm(k=131088, lda=131088, ldb=131088), nsml.ECAP)
    refused(mm(lda=(1 << 22) + 16), nsml.ECAP)
    refused(mm(n=(1 << 32) - 1, ldc=1 << 33), nsml.ECAP)


def test_checkpoints():
    for bad in (ck(q=None), ck(q=P + 8), ck(e=None), ck(ldq=72), ck(ldq=48), ck(lde=1), None):
        refused(L.nsml_ckpt8_pack(P, 0, 64, 3, 64, bad, None))
        refused(L.nsml_ckpt8_unpack(bad, 3, 64, P, 0, 64, None))
        refused(L.nsml_ckpt8_wgrad(P, 0, 8, bad, None, 3, 8, 64, None, P, 64, None, 0, None))
        refused(L.nsml_rmsnorm_backward(P, 64, bad, P, None, None, 0, 0, 3, 64, P, 64, None, None, 0, None))
        refused(L.nsml_swiglu_backward(P, 64, bad, ck(), 0, 3, 64, P, 64, P, 64, None))
        refused(L.nsml_swiglu_backward(P, 64, ck(), bad, 0, 3, 64, P, 64, P, 64, None))
        if bad is not None:
            refused(L.nsml_rmsnorm_q8(P, 64, None, 0, None, 0.0, 0, 3, 64, None, 0, P, 64, P, P, bad, None))
            refused(L.nsml_swiglu_q8(P, 64, P, 64, 0, 3, 64, P, 64, P, bad, None, None, None))
    refused(L.nsml_ckpt8_pack(P, 7, 64, 3, 64, ck(), None))
    refused(L.nsml_ckpt8_pack(P + 1, 1, 64, 3, 64, ck(), None))
    refused(L.nsml_ckpt8_unpack(ck(), 3, 0, P, 0, 64, None))


def test_wgrad():
    def wg(dy=P, type=1, lddy=1000, col=None, m=4000, n=1000, k=64, add=None, dw=P, ld=64, work=P, size=1 << 40):
        return L.nsml_ckpt8_wgrad(dy, type, lddy, ck(), col, m, n, k, add, dw, ld, work, size, None)
    for bad in ({"dy": None}, {"dy": P + 1}, {"type": 4}, {"lddy": 999}, {"col": P + 2}, {"n": 0}, {"k": 0}, {"add": P + 1}, {"dw": None},
                {"ld": 63}, {"work": None}, {"work": P + 8}, {"size": L.nsml_ckpt8_wgrad_work(4000, 1000, 64) - 1}):
        refused(wg(**bad))
    refused(wg(n=1 << 31, lddy=1 << 31), nsml.ECAP)
    refused(wg(lddy=1 << 23), nsml.ECAP)
    assert L.nsml_ckpt8_wgrad_work(4000, 1000, 64) > 0 and L.nsml_ckpt8_wgrad_work(0, 1000, 64) == 0


def test_norm():
    def nq(x=P, ldx=64, r=None, ldr=0, g=None, eps=1e-5, type=0, m=3, k=64, h=None, ldh=0, q=P, ldq=64, s=P, rstd=P):
        return L.nsml_rmsnorm_q8(x, ldx, r, ldr, g, eps, type, m, k, h, ldh, q, ldq, s, rstd, None, None)
    for bad in ({"x": None}, {"ldx": 3}, {"r": P, "ldr": 64}, {"h": P, "ldh": 64}, {"r": P, "ldr": 63, "h": P, "ldh": 64},
                {"r": P, "ldr": 64, "h": P, "ldh": 63}, {"g": P + 2}, {"eps": -1.0}, {"eps": float("nan")}, {"type": 3}, {"k": 0}, {"q": None},
                {"ldq": 16}, {"s": None}, {"rstd": None}):
        refused(nq(**bad))
    refused(nq(k=32769, ldx=40000, ldq=40000), nsml.ECAP)

    def nb(dy=P, ld=64, rstd=P, g=None, dres=None, ldr=0, type=0, k=64, dx=P, ldx=64, dg=P, work=P, size=1 << 40):
        return L.nsml_rmsnorm_backward(dy, ld, ck(), rstd, g, dres, ldr, type, 3, k, dx, ldx, dg, work, size, None)
    for bad in ({"dy": None}, {"ld": 1}, {"rstd": None}, {"g": P + 1}, {"dres": P, "ldr": 60}, {"type": 8}, {"k": 0}, {"dx": None},
                {"ldx": 2}, {"dg": P + 2}, {"work": None}, {"work": P + 4}, {"size": L.nsml_rmsnorm_backward_work(3, 64) - 1}):
        refused(nb(**bad))


def test_swiglu():
    def sg(g=P, ldg=64, u=P, ldu=64, type=0, k=64, q=P, ldq=64, s=P):
        return L.nsml_swiglu_q8(g, ldg, u, ldu, type, 3, k, q, ldq, s, None, None, None, None)
    for bad in ({"g": None}, {"ldg": 63}, {"u": None}, {"u": P + 2}, {"ldu": 1}, {"type": 3}, {"k": 0}, {"q": P + 1}, {"ldq": 68}, {"s": None}):
        refused(sg(**bad))
    for bad in ({"da": None}, {"dg": None}, {"du": P + 2}, {"ld": 63}):
        a = {"da": P, "dg": P, "du": P, "ld": 64, **bad}
        refused(L.nsml_swiglu_backward(a["da"], a["ld"], ck(), ck(), 0, 3, 64, a["dg"], 64, a["du"], 64, None))


# ---------------------------------------------------------------- the binding's own checks

CPU = torch.device("cpu")


def test_binding_wants_tensors_on_a_gpu():
    x = torch.zeros(4, 32)
    q = nsml.Q8(torch.zeros(4, 32, dtype=torch.int8), torch.ones(4))
    c = nsml.Ckpt8(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8))
    for call in (lambda: nsml.q8_rows(x), lambda: nsml.q8_values(q), lambda: nsml.q8_matmul(q, q), lambda: nsml.ckpt8_pack(x),
                 lambda: nsml.ckpt8_unpack(c), lambda: nsml.ckpt8_wgrad(x, c), lambda: nsml.rmsnorm_q8(x),
                 lambda: nsml.rmsnorm_backward(x, c, torch.ones(4)), lambda: nsml.swiglu_q8(x, x),
                 lambda: nsml.swiglu_backward(x, c, c), lambda: nsml.q8_rows(None)):
        with pytest.raises(ValueError):
            call()


def test_binding_checks_matrices():
    ok = torch.zeros(4, 40)
    assert nsml._matrix("x", ok, CPU)[1:] == (40, 4, 40)
    assert nsml._matrix("x", ok[:, :30], CPU)[1:] == (40, 4, 30)
    assert nsml._matrix("x", ok[:1, :30], CPU)[1] >= 30
    for bad, kw in ((ok.t(), {}), (ok[0], {}), (ok.double(), {}), (ok.half(), {"dtype": torch.float32}), (ok, {"rows": 5}), (ok, {"cols": 39}),
                    (ok[:, :0], {}), (ok[:, ::2], {}), (ok[:1].expand(4, 40), {}), ([1, 2], {}), (torch.zeros(2, 2, 2), {})):
        with pytest.raises(ValueError):
            nsml._matrix("x", bad, CPU, kw.get("dtype"), kw.get("rows"), kw.get("cols"))
    with pytest.raises(ValueError):
        nsml._matrix("x", ok, torch.device("cuda", 0))


def _aligned(*shape):
    n = 1
    for s in shape:
        n *= s
    flat = torch.zeros(n + 16, dtype=torch.int8)
    lead = -flat.data_ptr() % 16
    return flat[lead:lead + n].view(shape), flat, lead


def test_binding_checks_codes():
    q, flat, lead = _aligned(4, 48)
    assert nsml._codes("q", q, CPU)[1:] == (48, 4, 48)
    assert nsml._codes("q", q[:, :40], CPU)[1:] == (48, 4, 40)
    with pytest.raises(ValueError):
        nsml._codes("q", q[:, 1:41], CPU)                                   # does not start at a multiple of 16
    with pytest.raises(ValueError):
        nsml._codes("q", torch.zeros(4, 40, dtype=torch.int8), CPU)         # stride 40
    with pytest.raises(ValueError):
        nsml._codes("q", q.to(torch.uint8), CPU)
    short = torch.zeros(lead + 3 * 48 + 40 + 16, dtype=torch.int8)
    lead = -short.data_ptr() % 16
    short = torch.empty(0, dtype=torch.int8).set_(short.untyped_storage()[:lead + 3 * 48 + 40], lead, (4, 40), (48, 1))
    with pytest.raises(ValueError):
        nsml._codes("q", short, CPU)                                        # the last row's 16-byte chunk is not its own


def test_binding_checks_vectors_and_pairs():
    assert nsml._vector("v", None, CPU, 5) is None
    for bad in (torch.zeros(4), torch.zeros(5, dtype=torch.float64), torch.zeros(10)[::2], torch.zeros(5, 1), 3.0):
        with pytest.raises(ValueError):
            nsml._vector("v", bad, CPU, 5)
    q, _, _ = _aligned(4, 48)
    with pytest.raises(ValueError):
        nsml._rows_of("a", (q, torch.ones(4)), CPU)
    with pytest.raises(ValueError):
        nsml._rows_of("a", nsml.Q8(q, torch.ones(3)), CPU)
    with pytest.raises(ValueError):
        nsml._ckpt("c", nsml.Ckpt8(q, torch.zeros(4, 1, dtype=torch.uint8)), CPU)       # needs two exponents a row
    with pytest.raises(ValueError):
        nsml._ckpt("c", nsml.Q8(q, torch.ones(4)), CPU)


def test_results_of_more_tiles_than_a_launch_has():
    for m, n in ((1, 1 << 30), (64, (1 << 30) - 32768 + 1), (1 << 31, 1), (1 << 29, 1024)):
        refused(L.nsml_q8_matmul(P, 16, P, P, 16, P, None, m, n, 16, P, 1, n, None), nsml.ECAP)
    refused(L.nsml_ckpt8_wgrad(P, 1, 1 << 21, ck(ldq=1 << 21, lde=1 << 16), None, 3, 1 << 21, 1 << 21, None, P, 1 << 21, P, 1 << 40, None), nsml.ECAP)


@pytest.mark.parametrize("m,n", [(1 << 30, 1), (1 << 30, 64), ((1 << 30) - 63, 64), ((1 << 31) - 65800, 1), ((1 << 31) - 65800, 64)])
def test_tall_products_of_few_columns_beyond_a_launch(m, n):
    """Up to 64 columns take tiles of 64 rows however many rows there are: 2^24 of them have 2^32 threads."""
    refused(L.nsml_q8_matmul(P, 16, P, P, 16, P, None, m, n, 16, P, 1, n, None), nsml.ECAP)


@pytest.mark.parametrize("n,k", [(1 << 20, 1 << 19), ((1 << 19) + 1, 1 << 20), (1 << 20, (1 << 20) - 256)])
def test_weight_gradients_beyond_a_launch(n, k):
    """2^23 tiles of 256 have 2^32 threads."""
    refused(L.nsml_ckpt8_wgrad(P, 1, n, ck(ldq=k, lde=k // 32), None, 3, n, k, None, P, k, P, 1 << 40, None), nsml.ECAP)


# ---------------------------------------------------------------- buffers that share bytes

A = [1 << 20 << i for i in range(12)]       # addresses far apart; nothing is read from them


def free(rc):
    """Not refused: without a GPU the launch itself fails.  (Never run where there is one: the addresses are nobody's.)"""
    assert rc == nsml.EHIP


CALLS = {
    # name of each buffer: bytes from row to row, rows, bytes of a row; then which are written, and the call
    "q8_rows": ({"x": 128, "col": 256, "q": 64, "s": 12}, "q s",
                lambda b: L.nsml_q8_rows(b["x"], 1, 64, 3, 64, b["col"], b["q"], 64, b["s"], None)),
    "q8_values": ({"q": 64, "s": 12, "out": 128}, "out", lambda b: L.nsml_q8_values(b["q"], 64, b["s"], 3, 64, b["out"], 1, 64, None)),
    "q8_matmul": ({"a": 64, "sa": 12, "b": 64, "sb": 20, "bias": 20, "c": 10}, "c",
                  lambda b: L.nsml_q8_matmul(b["a"], 64, b["sa"], b["b"], 64, b["sb"], b["bias"], 3, 5, 64, b["c"], 1, 5, None)),
    "ckpt8_pack": ({"x": 128, "q": 64, "e": 2}, "q e", lambda b: L.nsml_ckpt8_pack(b["x"], 1, 64, 3, 64, ck(b["q"], b["e"]), None)),
    "ckpt8_unpack": ({"q": 64, "e": 2, "out": 128}, "out", lambda b: L.nsml_ckpt8_unpack(ck(b["q"], b["e"]), 3, 64, b["out"], 1, 64, None)),
    "ckpt8_wgrad": ({"dy": 2000, "q": 64, "e": 2, "col": 256, "dw": 256, "work": 1 << 16}, "dw work",
                    lambda b: L.nsml_ckpt8_wgrad(b["dy"], 1, 1000, ck(b["q"], b["e"]), b["col"], 4000, 1000, 64, None, b["dw"], 64, b["work"], 1 << 40, None)),
    "rmsnorm_q8": ({"x": 128, "r": 128, "g": 256, "h": 128, "q": 64, "s": 12, "rstd": 12, "xq": 64, "xe": 2}, "h q s rstd xq xe",
                   lambda b: L.nsml_rmsnorm_q8(b["x"], 64, b["r"], 64, b["g"], 1e-5, 1, 3, 64, b["h"], 64, b["q"], 64, b["s"], b["rstd"], ck(b["xq"], b["xe"]), None)),
    "rmsnorm_backward": ({"dy": 128, "q": 64, "e": 2, "rstd": 12, "g": 256, "dres": 128, "dx": 128, "dg": 256, "work": 256}, "dx dg work",
                         lambda b: L.nsml_rmsnorm_backward(b["dy"], 64, ck(b["q"], b["e"]), b["rstd"], b["g"], b["dres"], 64, 1, 3, 64, b["dx"], 64, b["dg"],
                                                           b["work"], 1 << 40, None)),
    "swiglu_q8": ({"g": 128, "u": 128, "q": 64, "s": 12, "gq": 64, "ge": 2, "uq": 64, "ue": 2, "aq": 64, "ae": 2}, "q s gq ge uq ue aq ae",
                  lambda b: L.nsml_swiglu_q8(b["g"], 64, b["u"], 64, 1, 3, 64, b["q"], 64, b["s"], ck(b["gq"], b["ge"]), ck(b["uq"], b["ue"]), ck(b["aq"], b["ae"]), None)),
    "swiglu_backward": ({"da": 128, "gq": 64, "ge": 2, "uq": 64, "ue": 2, "dg": 128, "du": 128}, "dg du",
                        lambda b: L.nsml_swiglu_backward(b["da"], 64, ck(b["gq"], b["ge"]), ck(b["uq"], b["ue"]), 1, 3, 64, b["dg"], 64, b["du"], 64, None)),
}


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are not refused have addresses of nobody's")
@pytest.mark.parametrize("name", CALLS)
def test_buffers_that_share_bytes(name):
    width, written, call = CALLS[name]
    apart = dict(zip(width, A))
    free(call(apart))
    for w in written.split():
        for other in width:
            if other == w:
                continue
            # what is written begins in the first row of the other one, or ends in it
            last = 16 if width[other] > 16 else 0
            for at in (apart[other] + last, apart[other] - 16 if width[w] > 16 else apart[other]):
                refused(call({**apart, w: at}))


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are not refused have addresses of nobody's")
def test_buffers_that_may_be_the_same_or_lie_side_by_side():
    for name, same in (("rmsnorm_q8", ("h", "x")), ("rmsnorm_q8", ("h", "r")), ("rmsnorm_backward", ("dx", "dy")), ("rmsnorm_backward", ("dx", "dres")),
                       ("swiglu_backward", ("dg", "da")), ("swiglu_backward", ("du", "da"))):
        width, _, call = CALLS[name]
        b = dict(zip(width, A))
        free(call({**b, same[0]: b[same[1]]}))
    # halves of one matrix, in either order, and one half that reaches into the other
    def halves(dg, du, ld, da=A[0]):
        return L.nsml_swiglu_backward(da, 64, ck(A[1], A[2]), ck(A[3], A[4]), 1, 3, 64, dg, ld, du, ld, None)
    free(halves(A[5], A[5] + 128, 128))
    free(halves(A[5] + 128, A[5], 128))
    refused(halves(A[5], A[5] + 128, 127))
    refused(halves(A[5], A[5] + 126, 128))
    # a sum over micro-batches in place, beside it, or shifted
    def wg(add, dw=A[4], lddw=64):
        return L.nsml_ckpt8_wgrad(A[0], 1, 1000, ck(A[1], A[2]), None, 3, 1000, 64, add, dw, lddw, A[6], 1 << 40, None)
    free(wg(A[4]))
    free(wg(A[4] + 256, lddw=128))
    refused(wg(A[4] + 256))
    # a checkpoint whose exponents stand behind the codes of each row, and rows of other pitches between them
    free(L.nsml_ckpt8_pack(A[0], 1, 64, 3, 64, ck(A[1], A[1] + 64, 80, 80), None))
    refused(L.nsml_ckpt8_pack(A[0], 1, 64, 3, 64, ck(A[1], A[1] + 63, 80, 80), None))
    free(L.nsml_ckpt8_pack(A[0], 1, 64, 3, 64, ck(A[1], A[1] + 64, 80, 160), None))
    refused(L.nsml_ckpt8_pack(A[0], 1, 64, 3, 64, ck(A[1], A[1] + 64, 80, 60), None))
    # scales in the gap behind the only row that they meet
    free(L.nsml_q8_rows(A[0], 1, 64, 3, 64, None, A[1], 80, A[1] + 64, None))
    refused(L.nsml_q8_rows(A[0], 1, 64, 3, 64, None, A[1], 64, A[1] + 64, None))


def test_transpose():
    def tr(q=P, ldq=64, m=48, k=64, out=1 << 20, ldo=48):
        return L.nsml_q8_transpose(q, ldq, m, k, out, ldo, None)
    for bad in ({"q": None}, {"q": P + 8}, {"ldq": 48}, {"ldq": 72}, {"k": 0}, {"out": None}, {"out": P + 4}, {"ldo": 32}, {"ldo": 56}, {"out": P}, {"out": P + 48 * 64 - 16}):
        refused(tr(**bad))
    refused(tr(k=(1 << 32) - 1, ldq=1 << 32), nsml.ECAP)
    refused(tr(m=1 << 31, ldo=1 << 31), nsml.ECAP)
    assert L.nsml_q8_transpose(None, 0, 0, 64, None, 0, None) == nsml.OK


def test_binding_refuses_what_wants_a_graph():
    """Results have none: a gradient would be missing without a word."""
    m, v = torch.zeros(4, 40, requires_grad=True), torch.zeros(5, requires_grad=True)
    for t in (m, m[:, :30], m * 2):
        with pytest.raises(ValueError, match="requires a gradient"):
            nsml._matrix("x", t, CPU)
    with pytest.raises(ValueError, match="requires a gradient"):
        nsml._vector("v", v, CPU, 5)
    with torch.no_grad():
        assert nsml._matrix("x", m, CPU)[1:] == (40, 4, 40) and nsml._vector("v", v, CPU, 5) == v.data_ptr()
    assert nsml._matrix("x", m.detach(), CPU)[0] == m.data_ptr()

    class Norm(torch.autograd.Function):            # how a training program calls them
        @staticmethod
        def forward(ctx, x):
            nsml._matrix("x", x, CPU)
            return x.clone()

        @staticmethod
        def backward(ctx, dy):
            nsml._matrix("dy", dy, CPU)
            return dy
    (Norm.apply(m) * torch.ones(4, 40)).sum().backward()
    assert (m.grad == 1).all()


def test_binding_tells_torch_what_it_writes(monkeypatch):
    """A tensor that torch has kept for a backward pass and the library then writes has to fail there, not to give a wrong gradient."""
    monkeypatch.setattr(nsml, "_device_of", lambda name, t: t.device)
    monkeypatch.setattr(nsml, "_enqueue", lambda dev, fn, *args: None)
    x, f32 = torch.zeros(4, 48), torch.float32
    q, _, _ = _aligned(4, 48)
    c, r = nsml.Ckpt8(q, torch.zeros(4, 2, dtype=torch.uint8)), nsml.Q8(q, torch.ones(4))

    def rises(call, *tensors):
        before = [t._version for t in tensors]
        call(*tensors)
        assert all(t._version > v for t, v in zip(tensors, before))
    code, scale, e = _aligned(4, 48)[0], torch.zeros(4), torch.zeros(4, 2, dtype=torch.uint8)
    rises(lambda *_: nsml.q8_rows(x, out=nsml.Q8(code, scale)), code, scale)
    rises(lambda *_: nsml.ckpt8_pack(x, out=nsml.Ckpt8(code, e)), code, e)
    rises(lambda o: nsml.q8_values(r, out=o), torch.zeros(4, 48))
    rises(lambda o: nsml.ckpt8_unpack(c, out=o), torch.zeros(4, 48))
    rises(lambda o: nsml.q8_matmul(r, r, out=o), torch.zeros(4, 4))
    rises(lambda o: nsml.ckpt8_wgrad(x, c, out=o), torch.zeros(48, 48))
    rises(lambda o, d: nsml.rmsnorm_backward(x, c, torch.ones(4), out=o, dgamma=d), torch.zeros(4, 48), torch.zeros(48))
    rises(lambda a, b: nsml.swiglu_backward(x, c, c, dgate=a, dup=b), torch.zeros(4, 48), torch.zeros(4, 48))
    flat = torch.zeros(2 * 48 * 48)
    rises(lambda f: nsml.ckpt8_wgrad(x, c, out=f[48 * 48:].view(48, 48)), flat)
    # and in earnest
    w = torch.ones(4, 4, requires_grad=True)
    kept = torch.ones(4, 4)
    loss = (w * kept).sum()
    nsml.q8_matmul(r, r, out=kept, dtype=f32)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_binding_refuses_other_things_with_its_own_error(monkeypatch):
    x = torch.zeros(4, 32)
    for call in (lambda: nsml.q8_values(x), lambda: nsml.q8_transposed(x), lambda: nsml.q8_matmul(x, x), lambda: nsml.ckpt8_unpack(x), lambda: nsml.q8_values(None)):
        with pytest.raises(ValueError, match="must be a (Q8|Ckpt8)"):
            call()
    monkeypatch.setattr(nsml, "_device_of", lambda name, t: t.device)
    q, _, _ = _aligned(4, 32)
    c = nsml.Ckpt8(q, torch.zeros(4, 1, dtype=torch.uint8))
    for call in (lambda: nsml.ckpt8_wgrad(x, c, out="out"), lambda: nsml.rmsnorm_backward(x, c, torch.ones(4), out=3.0),
                 lambda: nsml.swiglu_backward(x, c, c, dgate=[1]), lambda: nsml.swiglu_backward(x, c, c, dup=(x, x))):
        with pytest.raises(ValueError):
            call()
