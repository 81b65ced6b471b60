"""What the binding of the products of trained models checks before it allocates
or calls anything (no GPU, and no memory behind the large shapes)."""
import ctypes
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
import paper_2609_05419_amd as o2m  # noqa: E402
from paper_2609_05419_amd import model_ops as M  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ---- sizes past 32 bits ----------------------------------------------------------

FAR = [1 << 31, (1 << 32) - 1, 1 << 32, (1 << 32) + 5]   # as 32-bit numbers: -2^31, -1, 0, 5


def wide(rows, cols, dtype=torch.bfloat16):
    """A matrix of any size in a few bytes."""
    return torch.zeros(1).to(dtype).expand(rows, cols)


@pytest.mark.parametrize("n", FAR)
def test_sizes_past_32_bits(n):
    fp8 = torch.float8_e4m3fn
    long_k, many = (wide(3, n, fp8), wide(3, -(-n // 128), torch.float32)), (wide(n, 16, fp8), wide(n, 1, torch.float32))
    calls = [lambda: o2m.quantize_fp8(wide(1, n)), lambda: o2m.quantize_fp8(wide(n, 1)),
             lambda: o2m.quantize_fp8(wide(n, 1), out=many), lambda: o2m.quantize_fp8_pair(wide(n, 2)),
             lambda: o2m.gemm_fp8(many, many), lambda: o2m.gemm_fp8(long_k, long_k), lambda: o2m.linear_fp8(wide(2, 16), many),
             lambda: M._operand(long_k, "W"), lambda: M._matrix(wide(n, 16), "X"),   # (whichever comes first)
             lambda: o2m.linear_fp8_backward(wide(n, 3), (wide(2, n, fp8), wide(2, -(-n // 128), torch.float32)),
                                             (wide(2, 3, fp8), wide(2, 1, torch.float32))),
             lambda: o2m.orthogonalize(wide(n, 1)), lambda: o2m.orthogonalize(wide(1, n)),
             lambda: o2m.orthogonalize(torch.zeros(1).expand(n, 2, 2))]
    for call in calls:
        with pytest.raises(ValueError, match="2\\^31"):
            call()


def test_steps_past_32_bits():
    for steps in (-1, 65, 1 << 31, (1 << 32) + 5):
        with pytest.raises(o2m.O2MError, match="steps") as e:
            o2m.orthogonalize(torch.zeros((3, 4)), steps=steps)
        assert e.value.status == -28


# ---- operands of a backward step that do not belong together ---------------------

def test_backward_of_operands_of_different_layers():
    """Xt and Wt of different k, of other tokens or outputs than dY, or of two kinds of scales: refused
    before dY is quantized."""
    def op(rows, k, s=torch.float32):
        return torch.zeros((rows, k), dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros((rows, -(-k // 128)), dtype=s)
    dy = torch.zeros((32, 48))   # 32 tokens, n = 48
    for xt, wt, what in ((op(64, 32), op(80, 48), "k rows"), (op(64, 16), op(64, 48), "tokens"),
                         (op(64, 32), op(64, 32), "n = 48"), (op(64, 32, torch.uint8), op(64, 48), "kind of scales"),
                         (op(64, 32), op(64, 48, torch.uint8), "kind of scales")):
        error = TypeError if "scales" in what else ValueError
        with pytest.raises(error, match=what):
            o2m.linear_fp8_backward(dy, xt, wt)
    with pytest.raises(ValueError, match="matrix"):
        o2m.linear_fp8_backward(torch.zeros(48), op(64, 32), op(64, 48))
    for dw in (torch.zeros((48, 65)), torch.zeros((64, 48)), torch.zeros(48)):
        with pytest.raises(ValueError, match="dW"):
            o2m.linear_fp8_backward(dy, op(64, 32), op(64, 48), dW=dw)
    with pytest.raises(ValueError, match="dW"):
        o2m.linear_fp8_backward(dy, op(64, 32), op(64, 48), accumulate=True)


# ---- a torch without the 8-bit types ---------------------------------------------

@pytest.mark.parametrize("lacks", [["float8_e8m0fnu"], ["float8_e8m0fnu", "float8_e4m3fn", "float8_e5m2"]])
def test_import_without_8_bit_types(lacks):
    """The package, the 2M calls with it, needs none of torch's 8-bit types: without them
    scales of powers of two are bytes, and a call that takes 8-bit values says what it lacks."""
    code = f"""
import torch
for name in {lacks!r}:
    delattr(torch, name)
import paper_2609_05419_amd as o2m
from paper_2609_05419_amd import model_ops as M
o2m.moduli(3)
assert M._SCALE_DTYPES["pow2"] == torch.uint8 and M._SCALE_KINDS[torch.uint8] == 0
x = torch.zeros((2, 16))
try:
    o2m.quantize_fp8(x)
except (ValueError if hasattr(torch, "float8_e4m3fn") else TypeError) as e:
    print(e)
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert ("float8_e4m3fn" if len(lacks) == 3 else "current device") in r.stdout


# ---- tensors that require a gradient ---------------------------------------------

def test_gradients_are_not_lost_silently():
    """The results carry no graph, so an input that requires a gradient is refused while
    gradients are recorded; without recording, or detached, it passes (to the next check)."""
    def op(rows, k):
        return torch.zeros((rows, k), dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros((rows, -(-k // 128)))
    x = torch.zeros((4, 32), requires_grad=True)
    w, xt, wt = op(48, 32), op(16, 4), op(16, 32)
    calls = [lambda x: o2m.quantize_fp8(x), lambda x: o2m.quantize_fp8_pair(x), lambda x: o2m.linear_fp8(x, w),
             lambda x: o2m.linear_fp8_backward(x, xt, wt), lambda x: o2m.orthogonalize(x),
             lambda x: o2m.quantize_fp8(2 * x)]
    for call in calls:
        with pytest.raises(RuntimeError, match="gradient"):
            call(x)
        for y in (x.detach(), x):
            with torch.set_grad_enabled(y is not x), pytest.raises(ValueError, match="current device"):
                call(y)


# ---- scratch memory ---------------------------------------------------------------

def test_scratch_of_small_updates():
    """Matrices that one workgroup keeps in LDS need none, however many (21 GB were asked for
    65535 of 96 x 80); others theirs."""
    need = o2m._L.o2m_orthogonalize_workspace
    for t in range(3):
        for rows, cols in ((1, 1), (96, 80), (80, 96), (128, 128), (64, 256), (33, 90)):
            small = (rows, cols) not in ((128, 128), (64, 256)) or t == 2   # (fp32 and fp16 are held twice as long)
            for batch in (1, 65535):
                assert (need(batch, rows, cols, t) <= 256) == small, (t, rows, cols, batch)
        assert need(2, 300, 200, t) > 2 * 2 * 5 * 200 * 200


# ---- launches of more threads than one launch has --------------------------------

def test_more_threads_than_a_launch_has():
    """A launch counts its threads in 32 bits; sizes past that are refused on the host, by the linear layer
    before its tokens are quantized (the addresses are never read)."""
    ptr, L, size = 1 << 20, o2m._L, -25

    def operand(**kw):
        f = dict(values=ptr, ld=16, scales=ptr, s_row=1, s_blk=1 << 31, block=1, format=0, scale_type=0)
        f.update(kw)
        return M._Operand(**f)
    q, tall = operand(), operand(ld=1 << 31)

    def quantize(rows, k, order, ld, Q, Qt):
        return L.o2m_quantize_fp8(rows, k, ptr, 2, order, ld, Q, Qt, None)

    def gemm(m, n, w, t=2):
        return L.o2m_gemm_fp8(m, n, 16, w, w, ptr, t, b"R", 1 << 31, 0, ptr, 1 << 62, None)

    def linear(tokens, n, w, t=2):
        return L.o2m_linear_fp8(tokens, n, 16, ptr, t, 16, w, 1 << 44, 1 << 31, ptr, 1 << 62, None)
    most = (1 << 31) - 1024
    assert quantize(1 << 28, 1, b"R", 1, q, None) == size            # 16 blocks of 1 x 128 to 256 threads
    assert quantize(1 << 30, 1, b"R", 1, operand(block=128), None) == size   # a block of 128 x 128 to 512
    assert quantize(1 << 30, 1, b"R", 1, operand(values=2 * ptr, scales=2 * ptr), tall) == size
    assert gemm(5, 1 << 28, q) == size and gemm(1 << 28, 5, q) == size       # 16 rows to 256
    f32 = operand(scale_type=1)
    assert gemm(most, 300, f32, 0) == size and gemm(300, most, q, 0) == size   # 128 x 128 at most to 256
    assert linear(1, 1 << 28, q) == size and linear(1 << 28, 16, q) == size
    assert linear(200, most, f32, 0) == size   # (the tokens alone would fit)


# ---- results in the memory of inputs ---------------------------------------------

@pytest.mark.parametrize("dx,ldx,dy,ldy,n", [
    (0, 40, 0, 40, 40), (0, 40, 39, 40, 40), (39, 40, 0, 40, 40),       # the same place, the last entry
    (0, 100, 30, 100, 40), (30, 100, 0, 100, 40), (0, 100, 90, 100, 40),   # rows of one pitch that meet
    (0, 100, 50, 90, 40)])
def test_linear_in_one_launch_refuses_its_tokens_memory(dx, ldx, dy, ldy, n):
    """3 tokens of 40 entries, bf16 (the addresses are never read)."""
    ptr = 1 << 20
    w = M._Operand(ptr, 48, ptr, 1, n, 1, 0, 0)
    assert o2m._L.o2m_linear_fp8_workspace(3, n, 40) == 0
    assert o2m._L.o2m_linear_fp8(3, n, 40, ptr + 2 * dx, 2, ldx, w, ptr + 2 * dy, ldy, None, 0, None) == -8


def test_shared_memory_is_seen():
    x = torch.zeros(6, 20)
    for a, b, shares in ((x, x, True), (x[:3], x[3:], False), (x[:3], x[2:], True), (x[5:], x[:5], False),
                         (x[::2], x[1::2], True), (x[:, :10], x[:, 10:], True), (x[:, :0], x, False),
                         (x[0:1, :10], x[0:1, 10:], False), (x, x.clone(), False), (x.t(), x, True)):
        assert M._shares(a, b) == M._shares(b, a) == shares


@pytest.mark.parametrize("dg,og,ldg,sg,do,oo,ldo,so", [
    (0, b"R", 9, 54, 0, b"C", 6, 54),              # in place, but across
    (0, b"R", 9, 54, 5, b"R", 9, 54), (54, b"R", 9, 54, 0, b"R", 9, 54),   # a part of a matrix, or a whole one, on
    (0, b"R", 9, 0, 53, b"R", 9, 54),              # one G for all
    (0, b"R", 20, 240, 3, b"R", 20, 240),          # rows of one pitch that meet
    (0, b"R", 20, 240, 12, b"R", 20, 241)])
def test_a_batch_of_small_updates_refuses_its_own_memory(dg, og, ldg, sg, do, oo, ldo, so):
    """2 matrices of 6 x 9, fp32 (the addresses are never read)."""
    ptr, L = 1 << 20, o2m._L
    assert L.o2m_orthogonalize_workspace(2, 6, 9, 0) == M._SMALL_UPDATE
    coef = (ctypes.c_double * 3)(1.0, 1.0, 1.0)
    assert L.o2m_orthogonalize(2, 6, 9, ptr + 4 * dg, og, ldg, sg, ptr + 4 * do, oo, ldo, so, 0, 1,
                               ctypes.addressof(coef), 0.0, ptr, 256, None) == -8


@pytest.mark.parametrize("oo,ldo,so", [(b"R", 17, 8), (b"R", 26, 9), (b"R", 27, 53), (b"C", 17, 6), (b"C", 62, 5)])
def test_a_batch_refuses_results_that_share_entries(oo, ldo, so):
    """3 matrices of 6 x 9 whose results meet, as rows side by side or one behind the other."""
    ptr, coef = 1 << 20, (ctypes.c_double * 3)(1.0, 1.0, 1.0)
    assert o2m._L.o2m_orthogonalize(3, 6, 9, ptr, b"R", 9, 54, 2 * ptr, oo, ldo, so, 0, 1, ctypes.addressof(coef), 0.0,
                                    ptr, 256, None) == -11
