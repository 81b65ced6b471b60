"""Products of trained models on MI355X: matrices held in 8-bit floating point
with a scale for each block of 128, the linear layer made of them, and the
orthogonalised update.

Thin binding, as the package's other calls: every step runs in the library's
HIP kernels, enqueued on the current stream (or ``stream``); nothing is
synchronised, and without the library the import fails.  Tensors live on the
current device.  Outputs and scratch memory come from torch's allocator, from
the pool of the stream that uses them, so that calls on different streams and
captured graphs share none.

An 8-bit operand is a pair ``(values, scales)``: ``values`` of shape (rows, k)
in ``torch.float8_e4m3fn`` or ``torch.float8_e5m2``, k running contiguously and
rows starting at multiples of 16 bytes, ``scales`` of shape (rows, ceil(k /
128)) for blocks of 1 x 128 or (ceil(rows / 128), ceil(k / 128)) for blocks of
128 x 128, in ``torch.float8_e8m0fnu`` (powers of two; or its bytes, in
``torch.uint8``, which are what a torch without that type gets) or
``torch.float32``.  The matrix it stands for is each value times its block's
scale.  ``quantize_fp8`` makes one.  Other matrices may be row-major or
column-major.  There is no autograd here: the backward products are calls of
their own, and an input that requires a gradient is refused while gradients are
recorded (``torch.no_grad()`` or ``detach()`` says that none is wanted).
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

import torch

from . import O2MError, _L, _check, _stream

__all__ = ["Fp8Operand", "quantize_fp8", "quantize_fp8_pair", "gemm_fp8", "linear_fp8", "linear_fp8_backward",
           "orthogonalize"]

_I, _L64, _P, _D, _C, _Z = (ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_double, ctypes.c_char,
                            ctypes.c_size_t)


class _Operand(ctypes.Structure):
    _fields_ = [("values", _P), ("ld", _L64), ("scales", _P), ("s_row", _L64), ("s_blk", _L64), ("block", _I),
                ("format", _I), ("scale_type", _I)]


_O = ctypes.POINTER(_Operand)
_L.o2m_quantize_fp8.argtypes = [_I, _I, _P, _I, _C, _L64, _O, _O, _P]
_L.o2m_gemm_fp8.argtypes = [_I, _I, _I, _O, _O, _P, _I, _C, _L64, _I, _P, _Z, _P]
_L.o2m_linear_fp8.argtypes = [_I, _I, _I, _P, _I, _L64, _O, _P, _L64, _P, _Z, _P]
_L.o2m_orthogonalize.argtypes = [_I, _I, _I, _P, _C, _L64, _L64, _P, _C, _L64, _L64, _I, _I, _P, _D, _P, _Z, _P]
for _f in ("o2m_quantize_fp8", "o2m_gemm_fp8", "o2m_linear_fp8", "o2m_orthogonalize"):
    getattr(_L, _f).restype = _I
_L.o2m_gemm_fp8_workspace.argtypes = [_I, _I, _I]
_L.o2m_linear_fp8_workspace.argtypes = [_I, _I, _I]
_L.o2m_orthogonalize_workspace.argtypes = [_I, _I, _I, _I]
for _f in ("o2m_gemm_fp8_workspace", "o2m_linear_fp8_workspace", "o2m_orthogonalize_workspace"):
    getattr(_L, _f).restype = _Z

_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
# (older releases of torch lack these types, and the package's other calls need none:
# a type that is missing is only missed where it is asked for)
_E4M3, _E5M2, _E8M0 = (getattr(torch, t, None) for t in ("float8_e4m3fn", "float8_e5m2", "float8_e8m0fnu"))
_FORMATS = {t: i for i, t in enumerate((_E4M3, _E5M2)) if t is not None}
_SCALES = {"pow2": 0, "float32": 1}
_SCALE_DTYPES = {"pow2": _E8M0 or torch.uint8, "float32": torch.float32}
_SCALE_KINDS = {_SCALE_DTYPES["pow2"]: 0, torch.uint8: 0, torch.float32: 1}
BLOCK = 128
_LARGEST = (1 << 31) - 1   # what the C calls' sizes hold: ctypes would drop the bits above
_ERR_STEPS, _MOST_STEPS = -28, 64
_SMALL_UPDATE = 256        # scratch bytes of an update in one launch


class Fp8Operand(NamedTuple):
    """A matrix held in 8 bits: values (rows, k) and the scales of its blocks."""
    values: torch.Tensor
    scales: torch.Tensor


# the current device's index without torch.cuda's checks (a device tensor exists)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _here(x: torch.Tensor, name: str) -> None:
    if not x.is_cuda or x.get_device() != _current_device():   # (get_device() is -1 on the CPU)
        raise ValueError(f"{name} must be a tensor on the current device")


def _fits(shape, name: str) -> None:
    if max(shape) > _LARGEST:
        raise ValueError(f"{name}: sizes reach 2^31 - 1 at most, got {tuple(shape)}")


def _type_of(x: torch.Tensor, name: str) -> int:
    """The C code of an input's type; of one whose gradient nobody would get, an error."""
    if x.requires_grad and torch.is_grad_enabled():
        raise RuntimeError(f"{name} requires a gradient, which this call does not pass on: call it under torch.no_grad() "
                           f"or on {name}.detach(), and take the gradients from linear_fp8_backward")
    t = _TYPES.get(x.dtype)
    if t is None:
        raise TypeError(f"{name} must be float32, float16 or bfloat16, got {x.dtype}")
    return t


def _order(rows: int, cols: int, s0: int, s1: int, name: str):
    """(order, leading dimension) of a rows x cols matrix with these strides."""
    if rows <= 1 or cols <= 1:
        if rows * cols <= 1:
            return b"R", max(cols, 1)
        if (s0 if cols == 1 else s1) < 1:
            raise ValueError(f"{name} must hold its entries apart from one another (strides of 1 and more)")
        if cols == 1:
            return b"R", s0                      # entry i at i s0
        return (b"R", cols) if s1 == 1 else (b"C", s1)
    if s1 == 1:
        return b"R", s0
    if s0 == 1:
        return b"C", s1
    raise ValueError(f"{name} must be row-major or column-major")


def _matrix(x: torch.Tensor, name: str):
    shape = x.shape
    if len(shape) != 2:
        raise ValueError(f"{name} must be a matrix, got {len(shape)} dimensions")
    _fits(shape, name)
    _here(x, name)
    s0, s1 = x.stride()
    if s1 == 1 and shape[0] > 1 and shape[1] > 1:
        return b"R", s0
    return _order(shape[0], shape[1], s0, s1, name)


def _operand(x, name: str) -> _Operand:
    """The C struct of an 8-bit operand, its shapes and types checked."""
    q, s = x
    fmt = _FORMATS.get(q.dtype)
    if fmt is None:
        raise TypeError(f"{name}: values must be float8_e4m3fn or float8_e5m2, got {q.dtype}")
    shape, s_shape = q.shape, s.shape
    if len(shape) != 2 or len(s_shape) != 2:
        raise ValueError(f"{name}: values and scales must be matrices")
    _fits(shape, name)
    _here(q, name)
    _here(s, name)
    kind = _SCALE_KINDS.get(s.dtype)
    if kind is None:
        raise TypeError(f"{name}: scales must be float8_e8m0fnu (or its bytes) or float32, got {s.dtype}")
    rows, k = shape
    ld, step = q.stride()
    if k > 1 and rows > 0 and step != 1:
        raise ValueError(f"{name}: the k values of a row must be contiguous (stride(1) == 1)")
    if rows <= 1 or k == 0:
        ld = (k + 15) // 16 * 16
    at = q.data_ptr()
    if ld % 16 or at % 16 or ld < k:
        raise ValueError(f"{name}: rows must start at multiples of 16 bytes, one after another")
    kb, rb = (k + BLOCK - 1) // BLOCK, (rows + BLOCK - 1) // BLOCK
    r, columns = s_shape
    if columns != kb:
        raise ValueError(f"{name}: {k} values a row need {kb} columns of scales, got {columns}")
    if r != rows and r != rb:
        raise ValueError(f"{name}: {rows} rows need {rows} or {rb} rows of scales, got {r}")
    s_row, s_blk = s.stride()
    return _Operand(at, ld, s.data_ptr(), s_row, s_blk, 1 if r == rows else BLOCK, fmt, kind)


def _empty(size, dtype, device, stream):
    """Memory of the pool of the stream that will use it."""
    if stream is None:
        return torch.empty(size, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(size, dtype=dtype, device=device)


def _reach(x: torch.Tensor):
    """First byte of a tensor with entries, and the one behind its last."""
    at = x.data_ptr()
    return at, at + x.element_size() * (1 + sum((n - 1) * s for n, s in zip(x.shape, x.stride())))


def _shares(x: torch.Tensor, y: torch.Tensor) -> bool:
    """Whether two tensors reach into one another's memory."""
    if x.numel() == 0 or y.numel() == 0:
        return False
    (a, b), (c, d) = _reach(x), _reach(y)
    return a < d and c < b


def _copy(x: torch.Tensor, stream) -> torch.Tensor:
    if stream is None:
        return x.clone()
    with torch.cuda.stream(stream):
        return x.clone()


def _scratch(nbytes: int, beside: torch.Tensor, stream):
    """(tensor that holds it, address, bytes) of scratch memory on the device of
    ``beside``; torch's blocks are 512-byte aligned."""
    if nbytes == 0:
        return None, None, 0
    t = _empty((nbytes,), torch.uint8, beside.device, stream)
    return t, t.data_ptr(), nbytes


def _strided(size, strides, dtype, device, stream):
    if stream is None:
        return torch.empty_strided(size, strides, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty_strided(size, strides, dtype=dtype, device=device)


def _fresh_operand(rows: int, k: int, block: int, dtype, scales: str, device, stream):
    """An operand to be written, and its C struct."""
    ld = (k + 15) // 16 * 16
    r, kb = (rows if block == 1 else (rows + BLOCK - 1) // BLOCK), (k + BLOCK - 1) // BLOCK
    q = _strided((rows, k), (ld, 1), dtype, device, stream)
    s = _strided((r, kb), (1, max(r, 1)), _SCALE_DTYPES[scales], device, stream)
    return Fp8Operand(q, s), _Operand(q.data_ptr(), ld, s.data_ptr(), 1, r, block, _FORMATS[dtype], _SCALES[scales])


def _quantize_args(block, dtype, scales):
    if tuple(block) not in ((1, BLOCK), (BLOCK, BLOCK)):
        raise ValueError(f"block must be (1, 128) or (128, 128), got {block!r}")
    if dtype not in _FORMATS:
        raise TypeError(f"dtype must be float8_e4m3fn or float8_e5m2, got {dtype}")
    if scales not in _SCALES:
        raise ValueError(f"unknown kind of scales {scales!r}; expected one of {sorted(_SCALES)}")
    return block[0]


def _written(out, shape, what):
    """The C struct of an operand given to be written."""
    if tuple(out[0].shape) != shape:
        raise ValueError(f"{what}: values must be of shape {shape}, got {tuple(out[0].shape)}")
    return _operand(out, what)


def quantize_fp8(X: torch.Tensor, block=(1, 128), dtype=_E4M3, scales: str = "pow2", out=None,
                 stream=None) -> Fp8Operand:
    """X (rows x k, float32, float16 or bfloat16) as an 8-bit operand: blocks of
    1 x 128 or 128 x 128, the last ones shorter.

    With amax the largest finite magnitude of a block and F the format's largest
    number, ``scales="pow2"`` takes the smallest power of two s >= amax / F (from
    2^-126), ``"float32"`` s = amax / F; entries become x (1 / s), rounded to
    nearest, ties to even, and Inf and NaN become NaN.  ``quantize_fp8(X.t())``
    is the operand of the transpose.  ``out``: an operand to write into, of any
    format and kind of scales (the other arguments are then not used)."""
    t = _type_of(X, "X")
    b = _quantize_args(block, dtype, scales) if out is None else 0
    order, ld = _matrix(X, "X")
    rows, k = X.shape
    if out is None:
        out, q = _fresh_operand(rows, k, b, dtype, scales, X.device, stream)
    else:
        q = _written(out, (rows, k), "out")
    _check(_L.o2m_quantize_fp8(rows, k, X.data_ptr(), t, order, ld, q, None, _stream(stream)), "quantize_fp8")
    return out


def quantize_fp8_pair(X: torch.Tensor, block=(1, 128), dtype=_E4M3, scales: str = "pow2", out=None,
                      stream=None) -> tuple[Fp8Operand, Fp8Operand]:
    """The operands of X and of its transpose from one reading of X (what a
    layer's forward product and its backward products take of X, W or dY).
    ``out``: a pair of operands to write into."""
    t = _type_of(X, "X")
    b = _quantize_args(block, dtype, scales) if out is None else 0
    order, ld = _matrix(X, "X")
    rows, k = X.shape
    if out is None:
        first, q = _fresh_operand(rows, k, b, dtype, scales, X.device, stream)
        second, qt = _fresh_operand(k, rows, b, dtype, scales, X.device, stream)
        out = (first, second)
    else:
        q, qt = _written(out[0], (rows, k), "out"), _written(out[1], (k, rows), "transposed out")
    _check(_L.o2m_quantize_fp8(rows, k, X.data_ptr(), t, order, ld, q, qt, _stream(stream)), "quantize_fp8_pair")
    return out


def gemm_fp8(A, B, dtype=torch.bfloat16, out: torch.Tensor | None = None, accumulate: bool = False,
             stream=None) -> torch.Tensor:
    """C = A B^T for 8-bit operands A (m rows of k) and B (n rows of k) of one
    kind of scales and any formats and blocks, rounded once to ``dtype`` (or that of
    ``out``, which may be row-major or column-major).  float32 results: exact
    products summed in fp32.  16-bit ones: 8 neighbouring products at a time are
    added with 13 bits below the largest, these sums in fp32; some 2e-5 of the
    result's norm where entries are of like size, but where large products cancel,
    2^-10 of them may be left in an entry, and ``dtype=torch.float32`` is the way to
    more.  Products of two blocks' scales have to stay within the range of normal
    fp32 numbers.  ``accumulate``: out += A B^T, rounded once."""
    a, b = _operand(A, "A"), _operand(B, "B")
    m, k = A[0].shape
    n = B[0].size(0)
    if B[0].size(1) != k:
        raise ValueError(f"inner dimensions differ: {tuple(A[0].shape)} and {tuple(B[0].shape)}")
    if a.scale_type != b.scale_type:
        raise TypeError("A and B must have the same kind of scales")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        if dtype not in _TYPES:
            raise TypeError(f"dtype must be float32, float16 or bfloat16, got {dtype}")
        out = _empty((m, n), dtype, A[0].device, stream)
        t, order, ld = _TYPES[dtype], b"R", max(n, 1)
    else:
        if tuple(out.shape) != (m, n):
            raise ValueError(f"out must be of shape {(m, n)}, got {tuple(out.shape)}")
        t = _type_of(out, "out")
        order, ld = _matrix(out, "out")
    ws, at, nbytes = _scratch(_L.o2m_gemm_fp8_workspace(m, n, k), out, stream)
    _check(_L.o2m_gemm_fp8(m, n, k, a, b, out.data_ptr(), t, order, ld, int(accumulate), at,
                           nbytes, _stream(stream)), "gemm_fp8")
    return out


def linear_fp8(X: torch.Tensor, W, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The linear layer Y = X W^T: X (tokens x k, row-major) is quantized to e4m3
    in blocks of 1 x 128 with W's kind of scales and multiplied with the operand
    W (n rows of k); Y (tokens x n, row-major) has X's type, which decides how
    products are summed (gemm_fp8: ``X.float()`` for the most).  ``out`` may lie in
    X's memory."""
    t = _type_of(X, "X")
    w = _operand(W, "W")
    order, ldx = _matrix(X, "X")
    tokens, k = X.shape
    n = W[0].size(0)
    if W[0].size(1) != k:
        raise ValueError(f"inner dimensions differ: {tuple(X.shape)} and {tuple(W[0].shape)}")
    if order != b"R":
        raise ValueError("X must be row-major")
    given = out is not None
    if out is None:
        out = _empty((tokens, n), X.dtype, X.device, stream)
        ldy = max(n, 1)
    else:
        if tuple(out.shape) != (tokens, n) or out.dtype != X.dtype:
            raise ValueError(f"out must be {X.dtype} of shape {(tokens, n)}")
        order, ldy = _matrix(out, "out")
        if order != b"R":
            raise ValueError("out must be row-major")
    nbytes = _L.o2m_linear_fp8_workspace(tokens, n, k)
    if given and nbytes == 0 and _shares(X, out):   # one launch, which writes while it reads
        X = _copy(X, stream)
        _, ldx = _matrix(X, "X")
    ws, at, nbytes = _scratch(nbytes, out, stream)
    _check(_L.o2m_linear_fp8(tokens, n, k, X.data_ptr(), t, ldx, w, out.data_ptr(), ldy, at, nbytes,
                             _stream(stream)), "linear_fp8")
    return out


def linear_fp8_backward(dY: torch.Tensor, Xt, Wt, dtype=_E4M3, dW: torch.Tensor | None = None,
                        accumulate: bool = False, stream=None) -> tuple[torch.Tensor, torch.Tensor]:
    """(dX, dW) of Y = X W^T: dX = dY W (of dY's type) and dW = dY^T X (float32; into
    ``dW`` if given, added to it with ``accumulate``).  Xt and Wt are the operands
    of the transposes, k rows of tokens and k rows of n values, as
    quantize_fp8_pair makes them in the forward pass; dY (tokens x n) is
    quantized to ``dtype`` in blocks of 1 x 128 along both its axes."""
    if dY.dim() != 2:
        raise ValueError(f"dY must be a matrix, got {dY.dim()} dimensions")
    (tokens, n), k = dY.shape, Wt[0].size(0)
    # both products are checked here, so that none is computed when the other cannot be
    if tuple(Xt[0].shape) != (k, tokens) or tuple(Wt[0].shape) != (k, n):
        raise ValueError(f"Xt and Wt must have k rows both, of tokens = {tokens} and n = {n} values, got "
                         f"{tuple(Xt[0].shape)} and {tuple(Wt[0].shape)}")
    if _SCALE_KINDS.get(Xt[1].dtype) != _SCALE_KINDS.get(Wt[1].dtype):
        raise TypeError("Xt and Wt must have the same kind of scales")
    if dW is None:
        if accumulate:
            raise ValueError("accumulate needs dW")
    elif tuple(dW.shape) != (n, k):
        raise ValueError(f"dW must be of shape {(n, k)}, got {tuple(dW.shape)}")
    scales = "float32" if Wt[1].dtype == torch.float32 else "pow2"
    dy, dyt = quantize_fp8_pair(dY, (1, BLOCK), dtype, scales, stream=stream)
    dX = gemm_fp8(dy, Wt, dtype=dY.dtype, stream=stream)
    return dX, gemm_fp8(dyt, Xt, dtype=torch.float32, out=dW, accumulate=accumulate, stream=stream)


def orthogonalize(G: torch.Tensor, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                  out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The orthogonalised update of G (rows x cols, or a batch of such matrices;
    float32, float16 or bfloat16): X = G / (||G|| + eps) in the Frobenius norm, then
    ``steps`` times X <- a X + (b A + c A^2) X with A = X X^T on the shorter side.
    ``coefficients``: (a, b, c), or one such triple for each step.  The result
    (or ``out``, which may lie in G's memory) has G's shape and type.  Between
    products a bfloat16 matrix is held in 11 bits, others in 22 (``G.float()`` gives a
    bfloat16 update that precision); singular values have to stay below 4."""
    t = _type_of(G, "G")
    if G.dim() not in (2, 3):
        raise ValueError(f"G must be a matrix or a batch of matrices, got {G.dim()} dimensions")
    _fits(G.shape, "G")
    if not 0 <= steps <= _MOST_STEPS:
        raise O2MError(_ERR_STEPS, "orthogonalize")
    _here(G, "G")
    rows, cols = G.shape[-2:]
    batch = G.size(0) if G.dim() == 3 else 1
    og, ldg = _order(rows, cols, G.stride(-2), G.stride(-1), "G")
    given = out is not None
    if out is None:
        if og == b"R":
            out = _empty(tuple(G.shape), G.dtype, G.device, stream)
        else:
            out = _empty(tuple(G.shape[:-2]) + (cols, rows), G.dtype, G.device, stream).transpose(-2, -1)
    elif out.shape != G.shape or out.dtype != G.dtype:
        raise ValueError(f"out must be {G.dtype} of shape {tuple(G.shape)}")
    _here(out, "out")
    oo, ldo = _order(rows, cols, out.stride(-2), out.stride(-1), "out")
    flat = [float(c) for k in coefficients for c in (k if hasattr(k, "__len__") else (k,))]
    if len(flat) == 3:
        flat = flat * steps
    if len(flat) != 3 * steps:
        raise ValueError(f"coefficients must be one triple or {steps} of them")
    coef = (ctypes.c_double * max(len(flat), 1))(*flat)
    nbytes = _L.o2m_orthogonalize_workspace(batch, rows, cols, t)
    if (given and batch > 1 and nbytes <= _SMALL_UPDATE and _shares(G, out)
            and (G.data_ptr() != out.data_ptr() or G.stride() != out.stride())):
        G = _copy(G, stream)   # one launch, which writes matrices while it reads others
        og, ldg = _order(rows, cols, G.stride(-2), G.stride(-1), "G")
    ws, at, nbytes = _scratch(nbytes, out, stream)
    _check(_L.o2m_orthogonalize(batch, rows, cols, G.data_ptr(), og, ldg, G.stride(0) if G.dim() == 3 else 0,
                                out.data_ptr(), oo, ldo, out.stride(0) if G.dim() == 3 else 0, t, steps,
                                ctypes.addressof(coef), eps, at, nbytes, _stream(stream)), "orthogonalize")
    return out
