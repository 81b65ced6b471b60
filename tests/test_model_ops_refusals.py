"""What the products of trained models refuse, found on the host before anything
is enqueued (no GPU: the addresses given are never read), and what their
scratch memory comes to."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2609_05419_amd as o2m  # noqa: E402
from paper_2609_05419_amd import model_ops as M  # noqa: E402

L = o2m._L
PTR = 1 << 20          # a 16-byte aligned address that no call reads
SIZE, WORKSPACE, STEPS = -25, -22, -28


def operand(**kw):
    f = dict(values=PTR, ld=64, scales=PTR, s_row=1, s_blk=64, block=1, format=0, scale_type=0)
    f.update(kw)
    return M._Operand(**f)


BAD_OPERANDS = [dict(values=0), dict(values=PTR + 8), dict(ld=72), dict(ld=16), dict(scales=0), dict(s_row=-1),
                dict(s_blk=-1), dict(block=2), dict(block=64), dict(format=2), dict(format=-1), dict(scale_type=2),
                dict(scales=PTR + 2, scale_type=1)]


def quantize(rows=8, k=40, X=PTR, t=0, order=b"R", ld=64, Q=None, Qt=None, both=False):
    ref = lambda o: ctypes.byref(o) if o is not None else None  # noqa: E731
    if Q is None and not both:
        Q = operand()
    return L.o2m_quantize_fp8(rows, k, X, t, order, ld, ref(Q), ref(Qt), None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), -1), (dict(k=-1), -2), (dict(X=0), -3), (dict(X=PTR + 2), -3), (dict(X=PTR + 1, t=1), -3),
    (dict(t=3), -4), (dict(t=-1), -4), (dict(order=b"X"), -5), (dict(ld=39), -6), (dict(order=b"C", ld=7), -6),
    (dict(both=True), -7)])
def test_quantize_refuses(kw, code):
    assert quantize(**kw) == code


@pytest.mark.parametrize("bad", BAD_OPERANDS)
def test_quantize_refuses_operands(bad):
    assert quantize(Q=operand(**bad)) == -7
    assert quantize(rows=40, Qt=operand(**bad)) == -8


@pytest.mark.parametrize("bad", [dict(s_row=0), dict(s_blk=0), dict(s_row=1, s_blk=7), dict(s_row=2, s_blk=2),
                                 dict(s_row=0, block=128), dict(s_blk=0, block=128), dict(s_row=2, s_blk=2, block=128)])
def test_quantize_refuses_scales_on_one_another(bad):
    """300 x 300 entries: 300 or 3 by 3 scales."""
    q = operand(ld=304, **{**dict(s_blk=300), **bad})
    other = operand(ld=304, values=2 * PTR, scales=2 * PTR, s_blk=300)
    assert quantize(300, 300, ld=300, Q=q) == -7
    assert quantize(300, 300, ld=300, Q=other, Qt=q) == -8


def test_quantize_refuses_one_operand_for_both():
    q = operand(ld=304, s_blk=300)
    for same in (dict(values=PTR, scales=2 * PTR), dict(values=2 * PTR, scales=PTR)):
        assert quantize(300, 300, ld=300, Q=q, Qt=operand(ld=304, s_blk=300, **same)) == -8


def test_sizes_past_the_last_tile():
    n, far = (1 << 31) - 1, operand(ld=1 << 31, s_row=1, s_blk=1 << 31)
    assert quantize(n, 40, ld=64, Q=operand(s_blk=n)) == SIZE
    assert quantize(8, n, ld=n, Q=far) == SIZE
    assert gemm(m=n) == SIZE and gemm(n=n, ld=n) == SIZE
    assert linear(tokens=n) == SIZE and linear(n=n, ldy=n) == SIZE


def gemm(m=8, n=9, k=40, A=None, B=None, C=PTR, t=2, order=b"R", ld=64, add=0):
    a, b = A or operand(), B or operand()
    return L.o2m_gemm_fp8(m, n, k, ctypes.byref(a), ctypes.byref(b), C, t, order, ld, add, None, 0, None)


@pytest.mark.parametrize("kw,code", [
    (dict(m=-1), -1), (dict(n=-1), -2), (dict(k=-1), -3), (dict(C=0), -6), (dict(C=PTR + 1), -6),
    (dict(C=PTR + 2, t=0), -6), (dict(t=3), -7), (dict(order=b"?"), -8), (dict(ld=8), -9),
    (dict(order=b"C", ld=7), -9), (dict(A=operand(ld=1 << 23)), SIZE), (dict(B=operand(ld=1 << 24)), SIZE)])
def test_gemm_refuses(kw, code):
    assert gemm(**kw) == code


@pytest.mark.parametrize("bad", BAD_OPERANDS)
def test_gemm_refuses_operands(bad):
    assert gemm(A=operand(**bad)) == -4
    assert gemm(B=operand(**bad)) == -5


def test_gemm_refuses_two_kinds_of_scales():
    assert gemm(B=operand(scale_type=1)) == -5


def linear(tokens=3, n=9, k=40, X=PTR, t=2, ldx=40, W=None, Y=PTR, ldy=16, ws=None, nbytes=0):
    w = W or operand()
    return L.o2m_linear_fp8(tokens, n, k, X, t, ldx, ctypes.byref(w), Y, ldy, ws, nbytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), -1), (dict(n=-1), -2), (dict(k=-1), -3), (dict(X=0), -4), (dict(X=PTR + 1), -4), (dict(t=5), -5),
    (dict(ldx=39), -6), (dict(Y=0), -8), (dict(Y=PTR + 1), -8), (dict(ldy=8), -9), (dict(W=operand(ld=1 << 23)), SIZE)])
def test_linear_refuses(kw, code):
    assert linear(**kw) == code


@pytest.mark.parametrize("bad", BAD_OPERANDS)
def test_linear_refuses_operands(bad):
    assert linear(W=operand(**bad)) == -7


def test_linear_refuses_too_little_scratch():
    tokens, n, k = 300, 900, 1000
    need = L.o2m_linear_fp8_workspace(tokens, n, k)
    assert need >= tokens * k
    big = operand(ld=1008, s_blk=900)
    args = dict(tokens=tokens, n=n, k=k, ldx=k, ldy=n, W=big)
    assert linear(**args) == WORKSPACE
    assert linear(**args, ws=PTR, nbytes=need - 1) == WORKSPACE
    assert linear(**args, ws=PTR + 16, nbytes=need) == WORKSPACE


COEF = (ctypes.c_double * 15)(*[3.4445, -4.775, 2.0315] * 5)


def ortho(batch=1, rows=6, cols=9, G=PTR, og=b"R", ldg=9, sg=0, O=PTR, oo=b"R", ldo=9, so=0, t=0, steps=5, coef=COEF,
          eps=1e-7, ws=None, nbytes=0):
    return L.o2m_orthogonalize(batch, rows, cols, G, og, ldg, sg, O, oo, ldo, so, t, steps,
                               ctypes.addressof(coef) if coef is not None else None, eps, ws, nbytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), -1), (dict(rows=-1), -2), (dict(cols=-1), -3), (dict(G=0), -4), (dict(G=PTR + 2), -4),
    (dict(og=b"x"), -5), (dict(ldg=8), -6), (dict(og=b"C", ldg=5), -6), (dict(sg=-1), -7), (dict(O=0), -8),
    (dict(O=PTR + 1, t=1), -8), (dict(oo=b"x"), -9), (dict(ldo=8), -10), (dict(oo=b"C", ldo=5), -10), (dict(so=-1), -11),
    (dict(batch=2, so=53), -11), (dict(batch=2, oo=b"C", ldo=7, so=61), -11), (dict(t=3), -12), (dict(steps=-1), STEPS),
    (dict(steps=65), STEPS), (dict(coef=None), STEPS), (dict(eps=-1e-9), STEPS), (dict(eps=math.inf), STEPS),
    (dict(eps=math.nan), STEPS), (dict(coef=(ctypes.c_double * 15)(*[math.nan] * 15)), STEPS),
    (dict(cols=(1 << 21) + 1, ldg=1 << 22, ldo=1 << 22), SIZE),
    (dict(batch=65536, so=54), SIZE), (dict(), WORKSPACE), (dict(ws=PTR, nbytes=1), WORKSPACE)])
def test_orthogonalize_refuses(kw, code):
    assert ortho(**kw) == code


def test_nothing_to_do_needs_nothing():
    assert quantize(rows=0) == 0 and quantize(k=0) == 0
    assert gemm(m=0) == 0 and gemm(n=0) == 0
    assert linear(tokens=0) == 0 and linear(n=0) == 0
    assert ortho(batch=0) == 0 and ortho(rows=0) == 0
    assert gemm(k=0, add=1) == 0
    assert L.o2m_gemm_fp8_workspace(0, 5, 5) == 0 and L.o2m_linear_fp8_workspace(5, 0, 5) == 0
    assert L.o2m_orthogonalize_workspace(1, 0, 5, 0) == 0 and L.o2m_orthogonalize_workspace(1, 5, 5, 9) == 0


def test_status_text():
    assert b"o2m_orthogonalize" in L.o2m_status_string(STEPS)


def test_binding_refuses():
    cpu = torch.zeros((4, 32))
    q = (torch.zeros((4, 32), dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros((4, 1)))
    for call in (lambda: o2m.quantize_fp8(cpu), lambda: o2m.quantize_fp8_pair(cpu), lambda: o2m.gemm_fp8(q, q),
                 lambda: o2m.linear_fp8(cpu, q), lambda: o2m.orthogonalize(cpu)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: o2m.quantize_fp8(cpu.double()), lambda: o2m.quantize_fp8(cpu, dtype=torch.float16),
                 lambda: o2m.gemm_fp8((cpu, cpu), q), lambda: o2m.orthogonalize(cpu.double())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: o2m.quantize_fp8(cpu, block=(2, 128)), lambda: o2m.quantize_fp8(cpu, scales="int8"),
                 lambda: o2m.orthogonalize(torch.zeros(5)), lambda: o2m.quantize_fp8_pair(torch.zeros(5))):
        with pytest.raises(ValueError):
            call()
    # entries that all lie in one place, of a single row or column
    for rows, cols, s0, s1 in ((1, 5, 0, 0), (5, 1, 0, 1), (5, 1, 0, 0), (1, 5, 1, 0)):
        with pytest.raises(ValueError):
            M._order(rows, cols, s0, s1, "X")
    assert M._order(1, 5, 0, 2, "X") == (b"C", 2) and M._order(5, 1, 3, 0, "X") == (b"R", 3)
    assert M._order(1, 1, 0, 0, "X") == (b"R", 1) and M._order(0, 7, 0, 0, "X") == (b"R", 7)
