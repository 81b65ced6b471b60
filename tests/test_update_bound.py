"""The bound of one step of the orthogonalised update (model_reference.py) tells a step apart
from a wrong one: a simulated step with the held roundings lies within it, one with a changed
coefficient, a left-out term or one held part in place of two does not."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import model_reference as R  # noqa: E402

TRIPLES = [(3.4445, -4.7750, 2.0315), (3.0, -3.2, 1.2), (2.5, -2.0, 0.5), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]


def hold(v, exponent, parts):
    w = v * 2.0 ** exponent
    hi = w.astype(np.float16).astype(np.float64)
    if parts == 2:
        hi = hi + (w - hi).astype(np.float16).astype(np.float64)
    return hi * 2.0 ** -exponent


def held_step(x, coef, parts, add=1.0):
    if x.shape[0] > x.shape[1]:
        return held_step(x.T, coef, parts, add).T
    a, b, c = coef
    x = hold(x, 14, parts)
    t = hold(x @ x.T, 11, parts)
    return hold(a * np.eye(len(t)) + add * b * t + c * (t @ t), 6, parts) @ x


def rounded(v, dtype):
    return torch.from_numpy(np.ascontiguousarray(v)).to(dtype).double().numpy()


@pytest.mark.parametrize("rows,cols", [(1, 200), (96, 80), (33, 90), (64, 64), (100, 140)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_bound_of_a_step(rows, cols, dtype):
    parts = 1 if dtype == torch.bfloat16 else 2
    rng = np.random.default_rng(5)
    v = rng.standard_normal((rows, cols))
    v /= np.linalg.norm(v)
    for a, b, c in TRIPLES:
        x = rounded(v, dtype)
        exact, bound = R.orthogonalize_step(x, (a, b, c)), R.orthogonalize_step_bound(x, (a, b, c), parts, dtype)
        size = np.linalg.norm(exact)
        assert bound < {torch.float32: 3e-4, torch.float16: 4e-3, torch.bfloat16: 4e-2}[dtype] * size
        off = lambda v: np.linalg.norm(rounded(v, dtype) - exact)  # noqa: E731
        v = held_step(x, (a, b, c), parts)
        assert off(v) <= bound
        assert off(held_step(x, (1.05 * a, b, c), parts)) > bound
        assert off(0 * x) > bound
        if (a, b, c) == TRIPLES[0]:   # (the last ones have p(1) = 1, so near the end a step changes little)
            assert off(x) > bound
        if min(rows, cols) > 1 and (a, b, c) != TRIPLES[0]:   # (X is small before the first step)
            assert off(held_step(x, (a, b, c), parts, 0.0)) > bound
            assert off(held_step(x, (a, b, 0.8 * c), parts)) > bound or dtype == torch.bfloat16
        if dtype == torch.float32 and min(rows, cols) > 1:
            assert off(held_step(x, (a, b, c), 1)) > bound
