"""What the binding of the products of trained models checks before it allocates
or calls anything (no GPU, and no memory behind the large shapes)."""
import pytest

torch = pytest.importorskip("torch")
import paper_2609_05419_amd as o2m  # noqa: E402
from paper_2609_05419_amd import model_ops as M  # noqa: E402


# ---- sizes past 32 bits ----------------------------------------------------------

FAR = [1 << 31, (1 << 32) - 1, 1 << 32, (1 << 32) + 5]   # as 32-bit numbers: -2^31, -1, 0, 5


def wide(rows, cols, dtype=torch.bfloat16):
    """A matrix of any size in a few bytes."""
    return torch.zeros(1).to(dtype).expand(rows, cols)


@pytest.mark.parametrize("n", FAR)
def test_sizes_past_32_bits(n):
    fp8 = torch.float8_e4m3fn
    q = (wide(3, 16, fp8), wide(3, 1, torch.float32))
    long_k, many = (wide(3, n, fp8), wide(3, -(-n // 128), torch.float32)), (wide(n, 16, fp8), wide(n, 1, torch.float32))
    calls = [lambda: o2m.quantize_fp8(wide(1, n)), lambda: o2m.quantize_fp8(wide(n, 1)),
             lambda: o2m.quantize_fp8(wide(n, 1), out=many), lambda: o2m.quantize_fp8_pair(wide(n, 2)),
             lambda: o2m.gemm_fp8(many, q), lambda: o2m.gemm_fp8(long_k, q), lambda: o2m.linear_fp8(wide(2, 16), many),
             lambda: M._operand(long_k, "W"), lambda: M._matrix(wide(n, 16), "X"),   # (whichever comes first)
             lambda: o2m.linear_fp8_backward(wide(n, 3), q, q),
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
