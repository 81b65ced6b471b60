"""The definitions of the products of trained models in 64 bits on the CPU,
written from the formulas and used by the tests only: quantization in blocks,
products of quantized matrices with a bound of what fp32 sums may be off, and
the orthogonalised update with a bound of what its held roundings may cost."""
import math

import numpy as np
import torch

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
TOP = {E4M3: 448.0, E5M2: 57344.0}
GRID = {E4M3: (3, -6), E5M2: (2, -14)}   # mantissa bits, exponent of the lowest normal number


def round_to(x, dtype):
    """float64 numbers within the format's range, rounded to it, ties to even."""
    mant, low = GRID[dtype]
    _, e = np.frexp(np.maximum(np.abs(x), 2.0 ** low))
    step = np.ldexp(1.0, e - 1 - mant)
    return np.rint(x / step) * step


def quantize(x, block, dtype, scales):
    """(values as float64, scale of each block as float64) of a float32 matrix."""
    x = np.asarray(x, np.float32)
    rows, k = x.shape
    top = np.float32(TOP[dtype])
    rb, kb = -(-rows // block), -(-k // 128)
    s = np.ones((rb, kb))
    q = np.empty((rows, k))
    for i in range(rb):
        for j in range(kb):
            at = np.s_[i * block:(i + 1) * block, j * 128:(j + 1) * 128]
            b = x[at]
            fine = np.isfinite(b)
            amax = np.abs(b[fine]).max() if fine.any() else np.float32(0)
            if amax > 0:
                if scales == "pow2":
                    e = -126
                    while float(top) * 2.0 ** e < float(amax):
                        e += 1
                    s[i, j] = 2.0 ** e
                else:
                    s[i, j] = max(np.float32(amax / top), np.float32(2.0 ** -126))
            with np.errstate(invalid="ignore", over="ignore"):
                y = np.where(fine, b * (np.float32(1) / np.float32(s[i, j])), np.float32(0))
            q[at] = np.where(fine, round_to(np.clip(y.astype(np.float64), -top, top), dtype), np.nan)
    return q, s


def spread(s, block, rows, k):
    return np.repeat(np.repeat(s, block, 0)[:rows], 128, 1)[:, :k]


def scales64(s):
    """An operand's scales as float64."""
    if s.dtype == torch.float32:
        return s.double().cpu().numpy()
    code = s.view(torch.uint8).cpu().numpy().astype(np.int64)
    return np.where(code == 255, np.nan, np.ldexp(1.0, code - 127))


def values64(operand, block):
    """The matrix that an operand stands for."""
    q, s = operand
    return q.float().cpu().double().numpy() * spread(scales64(s), block, *q.shape)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def product_bound(a, b, exact, dtype):
    """How far a product may be from the exact one.  Each of the k additions in
    fp32 and of the at most four roundings of a scaled partial sum is off by at
    most one unit of 2^-23 of what it adds up (the matrix unit need not round to
    nearest), and the result by half a step, or by half the smallest number of
    the type.  16-bit results: the 8-bit matrix unit adds groups of 8 neighbouring
    products cut off 13 bits below the exponent of the largest, so each of the
    other 7 is off by less than 2^-13 of the power of two at or below the largest,
    7 2^-13 < 2^-10 of the largest for the group, which is at most the product of
    the largest factors."""
    k = a.shape[1]
    with np.errstate(invalid="ignore"):
        sums = (k + 4) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)
        if dtype != torch.float32:
            top = lambda x: np.pad(np.abs(x), ((0, 0), (0, -k % 8))).reshape(len(x), -1, 8).max(-1)  # noqa: E731
            sums += 2.0 ** -10 * (top(a) @ top(b).T)
    tiny = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}[dtype]
    return sums + half_step(dtype) * (np.abs(exact) + sums) + tiny


def check_product(got, a, b, dtype, start=None):
    """got (a tensor) against a b^T (+ start)."""
    fine = np.isfinite(a).all(1)[:, None] & np.isfinite(b).all(1)[None, :]
    a0, b0 = np.nan_to_num(a, nan=0.0, posinf=0.0, neginf=0.0), np.nan_to_num(b, nan=0.0, posinf=0.0, neginf=0.0)
    exact = a0 @ b0.T
    bound = product_bound(a0, b0, exact + (0 if start is None else np.abs(start)), dtype)
    if start is not None:
        exact = exact + start
        bound = bound + 2.0 ** -23 * np.abs(exact)
    got = got.double().cpu().numpy()
    assert got.shape == exact.shape
    assert np.isnan(got[~fine]).all()
    off = np.abs(got - exact)[fine]
    assert (off <= bound[fine]).all(), (off / bound[fine]).max()


COEF = (3.4445, -4.7750, 2.0315)


def orthogonalize(g, steps=5, coef=COEF, eps=1e-7):
    """The update of one float64 matrix, and the singular values of X before
    each step and after the last."""
    coef = list(coef) if steps and hasattr(coef[0], "__len__") else [coef] * steps
    x = g / (np.linalg.norm(g) + eps)
    sigma = [np.linalg.svd(x, compute_uv=False)]
    for a, b, c in coef:
        if x.shape[0] <= x.shape[1]:
            t = x @ x.T
            x = a * x + (b * t + c * (t @ t)) @ x
        else:
            t = x.T @ x
            x = a * x + x @ (b * t + c * (t @ t))
        sigma.append(np.linalg.svd(x, compute_uv=False))
    return x, sigma


def orthogonalize_bound(sigma, cols, parts, dtype, steps=5, coef=COEF):
    """Bound of the Frobenius norm of the error, to first order.  A step maps X to
    the matrix with the singular values p(s) = a s + b s^3 + c s^5 and the same
    singular vectors, so an error of X comes out multiplied by at most max |p'| over
    [0, s_max].  A step adds the roundings of what it holds, u relative in each
    entry of A, B = a + b A + c A^2 and X (u: half a step of fp16, or its square for two parts,
    once more for the left-out product of the low parts; and 2 (n + 2) 2^-23 for
    the fp32 sums of n terms, in the norm of the factors): those of A go into B
    through b + 2 c A, those of B into X through X."""
    coef = list(coef) if steps and hasattr(coef[0], "__len__") else [coef] * steps
    u = half_step(torch.float16)
    if parts == 2:
        u = 2 * u * u
    r = len(sigma[0])
    frob = lambda s: math.sqrt(float((s ** 2).sum()))  # noqa: E731
    err = u * frob(sigma[0])
    for t, (a, b, c) in enumerate(coef):
        s, s2 = sigma[t], sigma[t] ** 2
        top = float(s[0])
        grid = np.linspace(0.0, top, 2001)
        gain = np.abs(a + 3 * b * grid ** 2 + 5 * c * grid ** 4).max()
        fp = 2.0 ** -23
        d_a = u * frob(s2) + 2 * (cols + 2) * fp * frob(s) ** 2
        held_b = a + b * s2 + c * s2 ** 2
        d_b = (abs(b) + 2 * abs(c) * top ** 2) * d_a + u * frob(held_b) + 2 * (r + 2) * fp * abs(c) * frob(s2) ** 2
        d_x = top * d_b + u * frob(sigma[t + 1]) + 2 * (r + 2) * fp * frob(held_b) * frob(s)
        err = gain * err + d_x
    return err + half_step(dtype) * frob(sigma[-1])


def orthogonalize_step(x, coef):
    """One step on one float64 matrix."""
    a, b, c = coef
    if x.shape[0] > x.shape[1]:
        return orthogonalize_step(x.T, coef).T
    t = x @ x.T
    return a * x + (b * t + c * (t @ t)) @ x


def orthogonalize_step_bound(x, coef, parts, dtype):
    """Bound of the Frobenius norm of what one step may be off, given the result x (float64) of
    the steps before, rounded to dtype.  The step itself starts from the same numbers in fp32, held in one
    or two fp16 parts, so its start is off x by both roundings; a start that is off by e gives a
    result that is off by at most e max |p'| over the singular values, p(s) = a s + b s^3 + c s^5.  Then
      - A = X X^T, A^2 and B X are summed in fp32: of n terms every one passes a rounding (of at most one
        unit, 2^-23) for each 32 terms of each pass (three with two parts), 32 within such a run and 16 where
        splits are joined, so a sum is off by that of the sum of its terms' magnitudes; with two parts the
        products of the low ones, each below 2^-11 of its number, are left out;
      - A, B = a + b A + c A^2 and X are held, and B is added up from three terms in fp32.
    fp16 numbers end at 2^-24 of X 2^14, A 2^11, B 2^6, so each held entry may be off by half of
    that too.  1.05: what is of second order."""
    if x.shape[0] > x.shape[1]:
        x = x.T
    (r, c), (a, b, k5) = x.shape, coef
    norm = np.linalg.norm
    one = half_step(torch.float16)
    u, low, passes = (one, 0.0, 1) if parts == 1 else (one * one, one * one, 3)
    sums = lambda n: (passes * -(-n // 32) + 48) * 2.0 ** -23 + low  # noqa: E731
    tiny = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}[dtype]
    s = np.linalg.svd(x, compute_uv=False)
    grid = np.linspace(0.0, 1.01 * s[0], 4001)
    gain = np.abs(a + 3 * b * grid ** 2 + 5 * k5 * grid ** 4).max()
    start = (u + half_step(dtype)) * norm(x) + (2.0 ** -39 + tiny) * math.sqrt(r * c)
    t = x @ x.T
    held_b = a * np.eye(r) + b * t + k5 * (t @ t)
    d_a = u * norm(t) + sums(c) * norm(np.abs(x) @ np.abs(x).T) + 2.0 ** -36 * r
    d_b = ((abs(b) + 2 * abs(k5) * s[0] ** 2) * d_a + abs(k5) * sums(r) * norm(np.abs(t) @ np.abs(t)) + 2.0 ** -31 * r
           + u * norm(held_b) + 4 * 2.0 ** -24 * (abs(a) * math.sqrt(r) + abs(b) * norm(t) + abs(k5) * norm(t @ t)))
    exact = orthogonalize_step(x, coef)
    d_x = s[0] * d_b + sums(r) * norm(np.abs(held_b) @ np.abs(x))
    return 1.05 * (gain * start + d_x) + half_step(dtype) * norm(exact) + tiny * math.sqrt(r * c)
