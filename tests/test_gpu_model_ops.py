"""The products of trained models against their definitions in 64 bits: 8-bit
quantization bit for bit, block-scaled products and the linear layer within
the bound of their fp32 sums, the orthogonalised update within that of its
held roundings; odd and empty sizes, both memory orders, padded rows whose
padding holds NaN, and what lies behind the outputs left as it was."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import model_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E4M3, E5M2 = R.E4M3, R.E5M2
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def o2m():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_05419_amd as lib
    return lib


def matrix(rows, k, seed, dtype=torch.float32, order="row", spread=2.0):
    """Entries of unlike sizes, on the device, in either memory order."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, k)) * np.exp(spread * rng.standard_normal((rows, k)))
    x = torch.from_numpy(x).to(dtype)
    return x.to(DEV) if order == "row" else x.t().contiguous().to(DEV).t()


def padded_operand(o2m, x, block, dtype, scales):
    """An operand of x whose rows are 48 bytes longer, filled with NaN behind k, and
    whose scales lie in the other memory order."""
    rows, k = x.shape
    buf = torch.full((rows, (k + 15) // 16 * 16 + 48), 0x7F, dtype=torch.uint8, device=DEV)
    r, kb = (rows if block == 1 else -(-rows // block)), -(-k // 128)
    s = torch.empty((r, kb), dtype=torch.uint8 if scales == "pow2" else torch.float32, device=DEV)
    out = o2m.Fp8Operand(buf[:, :k].view(dtype), s.view(torch.float8_e8m0fnu) if scales == "pow2" else s)
    o2m.quantize_fp8(x, out=out)
    return out, buf


def same_operand(got, x, block, dtype, scales):
    q, s = R.quantize(x.float().cpu().numpy(), block, dtype, scales)
    assert got[0].dtype == dtype and tuple(got[0].shape) == q.shape
    assert np.array_equal(R.scales64(got[1]), s)
    v = got[0].float().cpu().double().numpy()
    assert np.array_equal(v, q, equal_nan=True)


# ---- quantization ------------------------------------------------------------

SHAPES = [(1, 1), (1, 128), (3, 127), (5, 129), (130, 7), (128, 256), (257, 300), (64, 1000), (300, 4096 + 8)]


@pytest.mark.parametrize("rows,k", SHAPES)
@pytest.mark.parametrize("scales", ["pow2", "float32"])
@pytest.mark.parametrize("block", [1, 128])
def test_quantize(o2m, rows, k, scales, block):
    for n, (dtype, fmt, order) in enumerate([(torch.float32, E4M3, "row"), (torch.bfloat16, E5M2, "row"),
                                             (torch.float16, E4M3, "col"), (torch.bfloat16, E4M3, "col")]):
        x = matrix(rows, k, 100 + n, dtype, order)
        same_operand(o2m.quantize_fp8(x, (block, 128), fmt, scales), x, block, fmt, scales)


@pytest.mark.parametrize("rows,k", SHAPES)
@pytest.mark.parametrize("block", [1, 128])
def test_quantize_pair(o2m, rows, k, block):
    for dtype, fmt, order, scales in [(torch.bfloat16, E4M3, "row", "pow2"), (torch.float32, E5M2, "col", "float32")]:
        x = matrix(rows, k, 7, dtype, order)
        q, qt = o2m.quantize_fp8_pair(x, (block, 128), fmt, scales)
        same_operand(q, x, block, fmt, scales)
        same_operand(qt, x.t(), block, fmt, scales)


@pytest.mark.parametrize("scales", ["pow2", "float32"])
@pytest.mark.parametrize("fmt", [E4M3, E5M2])
def test_quantize_extremes(o2m, scales, fmt):
    """Blocks of zeros, of the largest and the smallest numbers, of subnormals,
    next to the limits of a scale, and with Inf and NaN among or alone."""
    big, tiny, top = 3.4028234663852886e38, 2.0 ** -149, R.TOP[fmt]
    x = np.zeros((14, 128), np.float32)
    x[1] = big
    x[2, ::3] = -tiny
    x[3] = np.linspace(-1e-39, 1e-39, 128)
    x[4, 0], x[4, 1] = top, -top
    x[5, 0] = np.nextafter(np.float32(top), np.float32(np.inf))
    x[6, 0] = 1e30
    x[6, 1:] = np.linspace(1e-30, 1e30, 127)
    x[7] = np.arange(128) + 0.5
    x[8, 3], x[8, 4], x[8, 5], x[8, 6] = np.inf, -np.inf, np.nan, 2.0
    x[9] = np.nan
    x[10] = -np.inf
    x[11, :64], x[11, 64:] = 2.0 ** -126, 2.0 ** -130
    x[12] = np.ldexp(1.0, np.arange(128) % 40 - 20) * 1.0625      # halfway between two numbers of e4m3
    x[13] = np.ldexp(1.0, np.arange(128) % 40 - 20) * 1.1875
    t = torch.from_numpy(x).to(DEV)
    for block in (1, 128):
        same_operand(o2m.quantize_fp8(t, (block, 128), fmt, scales), t, block, fmt, scales)
        q, qt = o2m.quantize_fp8_pair(t.t(), (block, 128), fmt, scales)
        same_operand(q, t.t(), block, fmt, scales)
        same_operand(qt, t, block, fmt, scales)


@pytest.mark.parametrize("rows,k,ld", [(37, 75, 83), (129, 130, 136), (5, 128, 129)])
@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_views_and_guards(o2m, rows, k, ld, dtype):
    """Rows at any distance and start; the bytes behind an operand's rows stay."""
    whole = matrix(rows + 2, ld, 5, dtype)
    x = whole[1:1 + rows, 3:3 + k] if k + 3 <= ld else whole[1:1 + rows, :k]
    for v in (x, x.t()):
        got, buf = padded_operand(o2m, v, 1, E4M3, "pow2")
        same_operand(got, v, 1, E4M3, "pow2")
        assert (buf[:, v.size(1):] == 0x7F).all()


# ---- products -----------------------------------------------------------------

PRODUCTS = [(1, 1, 1), (1, 17, 16), (2, 3, 129), (33, 65, 127), (128, 128, 128), (200, 130, 300), (129, 257, 1000),
            (64, 500, 2051), (257, 1, 513), (300, 520, 640)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("scales", ["pow2", "float32"])
def test_gemm(o2m, m, n, k, scales):
    for i, (ba, bb, fa, fb, dtype) in enumerate([(1, 128, E4M3, E4M3, torch.bfloat16), (1, 1, E5M2, E4M3, torch.float32),
                                                 (128, 1, E4M3, E5M2, torch.float16), (128, 128, E5M2, E5M2, torch.float32)]):
        a, b = matrix(m, k, 20 + i, spread=0.5), matrix(n, k, 40 + i, spread=0.5)
        A, _ = padded_operand(o2m, a, ba, fa, scales)
        B = o2m.quantize_fp8(b, (bb, 128), fb, scales)
        print("gemm", m, n, k, scales, ba, bb, flush=True)
        C = o2m.gemm_fp8(A, B, dtype=dtype)
        R.check_product(C, R.values64(A, ba), R.values64(B, bb), dtype)
        assert torch.equal(C, o2m.gemm_fp8(A, B, dtype=dtype))


@pytest.mark.parametrize("m,n,k", [(1290, 1601, 128), (1290, 1601, 97), (1537, 1283, 300), (1536, 2048, 256), (1400, 1900, 1041),
                                   (8, 8200, 700), (9000, 130, 2064), (2100, 2000, 200), (2065, 2100, 333),
                                   (3700, 3601, 128), (3700, 3601, 97), (3601, 3700, 300), (3590, 3800, 1041), (140, 60001, 264),
                                   (2000, 4001, 2051), (1800, 4090, 1930), (4080, 2000, 2304)])
@pytest.mark.parametrize("scales", ["pow2", "float32"])
def test_gemm_large(o2m, m, n, k, scales):
    """Enough tiles for the kernels of larger products: one stage and many, odd and
    even numbers of them, ends of k within 16 bytes, ragged edges."""
    for i, (ba, bb, fa, fb, dtype) in enumerate([(1, 128, E4M3, E4M3, torch.bfloat16), (1, 1, E5M2, E4M3, torch.float16),
                                                 (128, 1, E4M3, E5M2, torch.bfloat16), (128, 128, E5M2, E5M2, torch.float32)]):
        a, b = matrix(m, k, 20 + i, spread=0.5), matrix(n, k, 40 + i, spread=0.5)
        a[m // 2, k // 3], b[n - 1, k - 1] = float("nan"), float("inf")
        A = o2m.quantize_fp8(a, (ba, 128), fa, scales)
        B = o2m.quantize_fp8(b, (bb, 128), fb, scales)
        if i % 2:   # rows behind which NaN lies
            A, _ = padded_operand(o2m, a, ba, fa, scales)
            A = o2m.Fp8Operand(A.values, A.scales.t().contiguous().t())
        print("gemm", m, n, k, scales, ba, bb, flush=True)
        C = o2m.gemm_fp8(A, B, dtype=dtype)
        R.check_product(C, R.values64(A, ba), R.values64(B, bb), dtype)
        again = o2m.gemm_fp8(A, B, dtype=dtype)
        assert torch.equal(C.view(torch.uint8), again.view(torch.uint8))   # NaN as well
        out = torch.ones((n, m), dtype=dtype, device=DEV).t()
        R.check_product(o2m.gemm_fp8(A, B, out=out, accumulate=True), R.values64(A, ba), R.values64(B, bb), dtype,
                        np.ones((m, n)))


@pytest.mark.parametrize("scales", ["pow2", "float32"])
@pytest.mark.parametrize("dtype", TYPES)
def test_gemm_out(o2m, scales, dtype):
    """Into outputs of either order, behind which nothing changes, and added."""
    m, n, k = 77, 150, 270
    A = o2m.quantize_fp8(matrix(m, k, 1, spread=0.5), scales=scales)
    B = o2m.quantize_fp8(matrix(n, k, 2, spread=0.5), (128, 128), scales=scales)
    a, b = R.values64(A, 1), R.values64(B, 128)
    for order in ("row", "col"):
        for add in (False, True):
            buf = torch.full((m + 3, n + 5) if order == "row" else (n + 3, m + 5), 7.0, dtype=dtype, device=DEV)
            out = buf[1:1 + m, 2:2 + n] if order == "row" else buf[1:1 + n, 2:2 + m].t()
            got = o2m.gemm_fp8(A, B, out=out, accumulate=add)
            assert got is out
            R.check_product(out, a, b, dtype, 7.0 * np.ones((m, n)) if add else None)
            out.fill_(7.0)
            assert (buf == 7.0).all()


@pytest.mark.parametrize("m,n,k", [(5, 90, 300), (70, 90, 300), (1900, 2100, 1000), (3700, 3600, 400)])
@pytest.mark.parametrize("scales", ["pow2", "float32"])
def test_gemm_orders_of_scales(o2m, m, n, k, scales):
    """Scales in either order, as bytes, or one for all blocks (strides of 0): the
    same values, so the same product; sizes for the kernels of each tile."""
    a, b = matrix(m, k, 6, spread=0.5), matrix(n, k, 7, spread=0.5)
    A, B = o2m.quantize_fp8(a, scales=scales), o2m.quantize_fp8(b, (128, 128), scales=scales)
    want = o2m.gemm_fp8(A, B)
    R.check_product(want, R.values64(A, 1), R.values64(B, 128), torch.bfloat16)
    wide = torch.empty((m, 2 * A.scales.size(1)), dtype=A.scales.dtype, device=DEV)[:, ::2]
    wide.copy_(A.scales)
    for s in (A.scales.contiguous(), wide, A.scales.t().contiguous().t()):
        for t in (B.scales.contiguous(), B.scales.t().contiguous().t()):
            R.check_product(o2m.gemm_fp8((A.values, s), (B.values, t)), R.values64(A, 1), R.values64(B, 128), torch.bfloat16)
            if scales == "pow2":
                assert torch.equal(o2m.gemm_fp8((A.values, s), (B.values, t)),
                                   o2m.gemm_fp8((A.values, s.view(torch.uint8)), (B.values, t.view(torch.uint8))))
    one = torch.full((1, 1), 0.5, device=DEV).to(A.scales.dtype)
    s, t = one.expand(m, A.scales.size(1)), one.expand(B.scales.shape)
    full = o2m.gemm_fp8((A.values, s.contiguous()), (B.values, t.contiguous()), dtype=torch.float32)
    assert torch.equal(o2m.gemm_fp8((A.values, s), (B.values, t), dtype=torch.float32), full)
    R.check_product(full, R.values64(o2m.Fp8Operand(A.values, s), 1), R.values64(o2m.Fp8Operand(B.values, t), 128),
                    torch.float32)


def test_gemm_ends_of_the_scales(o2m):
    """Scales that are NaN, and the smallest and largest that leave scaled entries
    normal, against ones of the other end."""
    m, n, k = 300, 260, 384
    a, b = matrix(m, k, 8, spread=0.5), matrix(n, k, 9, spread=0.5)
    A, B = o2m.quantize_fp8(a), o2m.quantize_fp8(b, (128, 128))
    low, high = o2m.Fp8Operand(A.values, torch.full_like(A.scales.view(torch.uint8), 127 - 110)), o2m.Fp8Operand(
        B.values, torch.full_like(B.scales.view(torch.uint8), 127 + 110))
    for dtype in TYPES:
        want = R.values64(o2m.Fp8Operand(A.values, torch.ones_like(A.scales, dtype=torch.float32)), 1)
        other = R.values64(o2m.Fp8Operand(B.values, torch.ones_like(B.scales, dtype=torch.float32)), 128)
        if dtype != torch.float16:   # (beyond fp16's range)
            R.check_product(o2m.gemm_fp8(low, high, dtype=dtype), want, other, dtype)
        s = A.scales.view(torch.uint8).clone()
        s[37, 1] = 255
        C = o2m.gemm_fp8(o2m.Fp8Operand(A.values, s), B, dtype=dtype)
        assert torch.isnan(C[37]).all() and torch.isfinite(C[:37]).all() and torch.isfinite(C[38:]).all()


def test_gemm_non_finite_rows(o2m):
    m, n, k = 40, 50, 200
    for scales in ("pow2", "float32"):
        a, b = matrix(m, k, 3, spread=0.5), matrix(n, k, 4, spread=0.5)
        a[3, 7], a[20, 199], b[11, 130] = float("nan"), float("inf"), float("-inf")
        A, B = o2m.quantize_fp8(a, scales=scales), o2m.quantize_fp8(b, scales=scales)
        R.check_product(o2m.gemm_fp8(A, B, dtype=torch.float32), R.values64(A, 1), R.values64(B, 1), torch.float32)


def test_gemm_empty(o2m):
    q = lambda r, k: o2m.quantize_fp8(torch.ones((r, k), device=DEV))  # noqa: E731
    assert o2m.gemm_fp8(q(0, 5), q(3, 5)).shape == (0, 3)
    C = o2m.gemm_fp8(q(4, 0), q(3, 0), dtype=torch.float32)
    assert C.shape == (4, 3) and (C == 0).all()
    out = torch.ones((4, 3), device=DEV)
    assert (o2m.gemm_fp8(q(4, 0), q(3, 0), out=out, accumulate=True) == 1).all()
    assert o2m.linear_fp8(torch.ones((2, 0), device=DEV), q(3, 0)).eq(0).all()
    assert o2m.linear_fp8(torch.ones((0, 8), device=DEV), q(3, 8)).shape == (0, 3)


# ---- the linear layer -----------------------------------------------------------

LINEAR = [(1, 1, 1), (1, 64, 128), (1, 333, 2051), (2, 257, 512), (5, 48, 4096), (16, 130, 700), (17, 100, 260),
          (33, 200, 129), (65, 300, 1024), (200, 129, 384)]


@pytest.mark.parametrize("tokens,n,k", LINEAR)
@pytest.mark.parametrize("scales", ["pow2", "float32"])
def test_linear(o2m, tokens, n, k, scales):
    for i, (dtype, block, fmt) in enumerate([(torch.bfloat16, 128, E4M3), (torch.float16, 1, E4M3),
                                             (torch.float32, 128, E5M2)]):
        x = matrix(tokens, k, 60 + i, dtype, spread=0.5)
        W, _ = padded_operand(o2m, matrix(n, k, 80 + i, spread=0.5), block, fmt, scales)
        print("linear", tokens, n, k, scales, dtype, flush=True)
        buf = torch.full((tokens + 1, n + 3), 7.0, dtype=dtype, device=DEV)
        y = o2m.linear_fp8(x, W, out=buf[:tokens, :n])
        q, s = R.quantize(x.float().cpu().numpy(), 1, E4M3, scales)
        R.check_product(y, q * R.spread(s, 1, tokens, k), R.values64(W, block), dtype)
        assert (buf[:, n:] == 7).all() and (buf[tokens:] == 7).all()
        assert torch.equal(y, o2m.linear_fp8(x, W))


def test_linear_non_finite_tokens(o2m):
    for tokens in (1, 3, 40):
        x = matrix(tokens, 300, 5, torch.bfloat16, spread=0.5)
        x[tokens - 1, 299] = float("nan")
        W = o2m.quantize_fp8(matrix(70, 300, 6), (128, 128))
        y = o2m.linear_fp8(x, W)
        assert torch.isnan(y[tokens - 1]).all() and torch.isfinite(y[:tokens - 1]).all()


@pytest.mark.parametrize("tokens,n,k", [(1, 1, 1), (40, 33, 130), (200, 129, 257), (130, 300, 64)])
@pytest.mark.parametrize("scales,fmt,dtype", [("pow2", E4M3, torch.bfloat16), ("float32", E5M2, torch.float16)])
def test_linear_backward(o2m, tokens, n, k, scales, fmt, dtype):
    x, w, dy = matrix(tokens, k, 1, spread=0.3), matrix(n, k, 2, spread=0.3), matrix(tokens, n, 3, dtype, spread=0.3)
    _, xt = o2m.quantize_fp8_pair(x, scales=scales)
    _, wt = o2m.quantize_fp8_pair(w, (128, 128), scales=scales)
    dx, dw = o2m.linear_fp8_backward(dy, xt, wt, dtype=fmt)
    d = dy.float().cpu().numpy()
    q, s = R.quantize(d, 1, fmt, scales)
    qt, st = R.quantize(d.T, 1, fmt, scales)
    R.check_product(dx, q * R.spread(s, 1, tokens, n), R.values64(wt, 128), dtype)
    held = qt * R.spread(st, 1, n, tokens)
    R.check_product(dw, held, R.values64(xt, 1), torch.float32)
    assert dw.dtype == torch.float32 and dx.dtype == dtype
    # the next micro-batch adds to the same gradient
    first = dw.double().cpu().numpy()
    _, again = o2m.linear_fp8_backward(dy, xt, wt, dtype=fmt, dW=dw, accumulate=True)
    assert again is dw
    R.check_product(dw, held, R.values64(xt, 1), torch.float32, first)


def test_linear_backward_against_differences(o2m):
    """dX and dW of L = sum(Y T) against differences of L over the unquantized
    layer.  Each of the two factors of a product is held within half a step of
    e4m3 of itself, or of the lowest number that its block's scale gives (2^-10
    of at least 448 / 2 of the scale, below 2^-17 of the block's largest), so the
    products are off by at most (2 h + h^2) |a| |b| with h = 2^-4, and 2^-17 of the
    largest twice for the small ones."""
    tokens, n, k = 24, 40, 56
    rng = np.random.default_rng(9)
    x, w, t = (rng.standard_normal(s) for s in ((tokens, k), (n, k), (tokens, n)))
    dev = lambda v: torch.from_numpy(v).float().to(DEV)  # noqa: E731
    _, xt = o2m.quantize_fp8_pair(dev(x))
    _, wt = o2m.quantize_fp8_pair(dev(w), (128, 128))
    dx, dw = (v.double().cpu().numpy() for v in o2m.linear_fp8_backward(dev(t), xt, wt))
    h = R.half_step(E4M3)

    def bound(a, b):   # of a @ b
        return (2 * h + h * h) * (np.abs(a) @ np.abs(b)) + 2.0 ** -16 * a.shape[1] * np.abs(a).max() * np.abs(b).max()
    loss = lambda x, w: ((x @ w.T) * t).sum()  # noqa: E731
    for _ in range(20):
        i, j, c, d = rng.integers(tokens), rng.integers(n), rng.integers(k), 0.5   # L is linear in each entry
        e = np.zeros_like(x)
        e[i, c] = d
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * d) - dx[i, c]) <= bound(t, w)[i, c]
        e = np.zeros_like(w)
        e[j, c] = d
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * d) - dw[j, c]) <= bound(t.T, x)[j, c]


# ---- the orthogonalised update ---------------------------------------------------

def check_orthogonalize(got, g, dtype, steps=5, coef=R.COEF, eps=1e-7):
    exact, sigma = R.orthogonalize(g.double().cpu().numpy(), steps, coef, eps)
    bound = R.orthogonalize_bound(sigma, max(g.shape), 1 if dtype == torch.bfloat16 else 2, dtype, steps, coef)
    got = got.double().cpu().numpy()
    assert got.shape == exact.shape
    off = np.linalg.norm(got - exact)
    assert off <= bound, (off, bound, np.linalg.norm(exact))


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 200), (96, 80), (64, 64), (128, 128), (130, 129), (33, 500), (300, 256),
                                       (257, 900), (17, 250), (127, 33), (64, 256), (90, 101), (112, 112), (513, 700)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("order", ["row", "col"])
def test_orthogonalize(o2m, rows, cols, dtype, order):
    g = matrix(rows, cols, 11, torch.float32, order, spread=0.3) * 1e-3
    g = (g.to(dtype) if order == "row" else g.t().contiguous().to(dtype).t())
    print("orthogonalize", rows, cols, dtype, order, flush=True)
    x = o2m.orthogonalize(g)
    assert x.dtype == dtype and x.shape == g.shape and x.stride() == g.stride()
    check_orthogonalize(x, g, dtype)
    assert torch.equal(x, o2m.orthogonalize(g))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,rows,cols,order", [(1, 1100, 3900, "row"), (1, 2300, 1400, "col"), (40, 260, 300, "row"),
                                                   (16, 900, 1101, "row"), (1, 2000, 5001, "col"), (15, 1000, 1300, "col"),
                                                   (18, 1000, 1399, "row")])
def test_orthogonalize_large(o2m, batch, rows, cols, order, dtype):
    """Enough tiles for the kernels of large products, the last ones beside the
    matrix; a step or two, which the bound tells apart from anything else."""
    g = torch.stack([matrix(rows, cols, 50 + i % 3, torch.float32, order, spread=0.3) for i in range(batch)]).to(dtype)
    if order == "col":
        g = g.transpose(1, 2).contiguous().transpose(1, 2)
    print("orthogonalize", batch, rows, cols, dtype, order, flush=True)
    x = o2m.orthogonalize(g, steps=2)
    assert x.stride() == g.stride()
    for i in (0, batch - 1):
        check_orthogonalize(x[i], g[i], dtype, 2)
    assert torch.equal(x, o2m.orthogonalize(g, steps=2))
    turned = o2m.orthogonalize(g, steps=2, out=torch.empty_like(g.transpose(1, 2).contiguous()).transpose(1, 2))
    assert torch.equal(x, turned)


@pytest.mark.parametrize("dtype", TYPES)
def test_orthogonalize_batch_views_and_orders(o2m, dtype):
    """A batch, in rows at a distance, into outputs of the other order, behind
    which nothing changes; and in place."""
    b, rows, cols = 3, 70, 150
    whole = torch.stack([matrix(rows + 1, cols + 9, 30 + i, dtype, spread=0.3) for i in range(b)])
    g = whole[:, 1:, 4:4 + cols]
    one = o2m.orthogonalize(g)
    for i in range(b):
        check_orthogonalize(one[i], g[i], dtype)
        assert torch.equal(one[i], o2m.orthogonalize(g[i]))
    buf = torch.full((b, cols + 2, rows + 6), 7.0, dtype=dtype, device=DEV)
    out = buf[:, 1:1 + cols, 3:3 + rows].transpose(1, 2)
    assert torch.equal(o2m.orthogonalize(g, out=out), one)
    out.fill_(7.0)
    assert (buf == 7).all()
    o2m.orthogonalize(g, out=g)
    assert torch.equal(g, one)


@pytest.mark.parametrize("dtype", TYPES)
def test_orthogonalize_steps_and_coefficients(o2m, dtype):
    g = matrix(100, 140, 17, dtype, spread=0.3)
    for steps, coef in ((0, R.COEF), (1, R.COEF), (3, [(3.0, -3.2, 1.2), (2.5, -2.0, 0.5), (1.875, -1.25, 0.375)])):
        check_orthogonalize(o2m.orthogonalize(g, steps=steps, coefficients=coef), g, dtype, steps, coef)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_orthogonalize_sizes_of_entries(o2m, dtype):
    """The norm of entries whose squares leave fp32, zeros, and Inf or NaN."""
    g = matrix(60, 90, 18, torch.float32, spread=0.3)
    for scale in (1e30, 1e-30):
        h = (g * scale).to(dtype)
        check_orthogonalize(o2m.orthogonalize(h, eps=0.0), h, dtype, eps=0.0)
    assert (o2m.orthogonalize(torch.zeros((60, 90), dtype=dtype, device=DEV)) == 0).all()
    for bad in (float("inf"), float("nan")):
        h = g.to(dtype).repeat(2, 1, 1)
        h[0, 59, 3] = bad
        x = o2m.orthogonalize(h)
        assert torch.isnan(x[0]).all() and torch.isfinite(x[1]).all()


# ---- together, streams, graphs --------------------------------------------------

def training_step(o2m, x, w, target, lr=0.02):
    """Forward, backward, orthogonalised update and the next operands of one
    linear layer with the loss |Y - T|^2 / 2."""
    xq, xt = o2m.quantize_fp8_pair(x)
    wq, wt = o2m.quantize_fp8_pair(w, (128, 128))
    y = o2m.gemm_fp8(xq, wq, dtype=torch.bfloat16)
    dx, dw = o2m.linear_fp8_backward(y - target, xt, wt)
    u = o2m.orthogonalize(dw)
    w.sub_(u, alpha=lr)
    return y, dx, dw, u


def test_a_training_step(o2m):
    tokens, n, k = 200, 96, 160
    x, w = matrix(tokens, k, 1, torch.bfloat16, spread=0.1), matrix(n, k, 2, spread=0.1) * k ** -0.5
    target = matrix(tokens, n, 3, torch.bfloat16, spread=0.1)
    for _ in range(3):
        w0 = w.clone()
        y, dx, dw, u = training_step(o2m, x, w, target)
        q = lambda v, b, f=E4M3: (lambda p: p[0] * R.spread(p[1], b, *v.shape))(  # noqa: E731
            R.quantize(v, b, f, "pow2"))
        xs, ws, dy = x.float().cpu().numpy(), w0.cpu().numpy(), (y - target).float().cpu().numpy()
        R.check_product(y, q(xs, 1), q(ws, 128), torch.bfloat16)
        R.check_product(dx, q(dy, 1), q(ws.T, 128), torch.bfloat16)
        R.check_product(dw, q(dy.T, 1), q(xs.T, 1), torch.float32)
        check_orthogonalize(u, dw, torch.float32)
        assert torch.equal(w, w0.sub(u, alpha=0.02))
        # the layer in use: the same product from the new weights
        R.check_product(o2m.linear_fp8(x[:1], o2m.quantize_fp8(w, (128, 128))), q(xs[:1], 1),
                        q(w.cpu().numpy(), 128), torch.bfloat16)


def test_streams_beside_each_other(o2m):
    """The same calls on two streams at once, one of them given as an argument."""
    data = [(matrix(150, 300, i, torch.bfloat16, spread=0.3), matrix(200, 300, 10 + i, spread=0.3)) for i in range(2)]
    W = [o2m.quantize_fp8(w, (128, 128)) for _, w in data]
    want = [(o2m.linear_fp8(x, w), o2m.orthogonalize(v)) for (x, v), w in zip(data, W)]
    torch.cuda.synchronize()
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        with torch.cuda.stream(s[0]):
            got.append((o2m.linear_fp8(data[0][0], W[0]), o2m.orthogonalize(data[0][1])))
        got.append((o2m.linear_fp8(data[1][0], W[1], stream=s[1]), o2m.orthogonalize(data[1][1], stream=s[1])))
        torch.cuda.synchronize()
        for (y, u), (y0, u0) in zip(got, want):
            assert torch.equal(y, y0) and torch.equal(u, u0)


def test_graphs(o2m):
    """Two graphs captured on one stream without a call before, replayed in turn on
    fresh inputs with eager work between, each with its own scratch memory."""
    shapes = [(130, 96, 200), (1, 256, 700)]
    graphs = []
    o2m.linear_fp8(torch.ones((1, 16), device=DEV), o2m.quantize_fp8(torch.ones((16, 16), device=DEV)))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i, (t, n, k) in enumerate(shapes):
        x = torch.zeros((t, k), dtype=torch.bfloat16, device=DEV)
        w = torch.zeros((n, k), device=DEV)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            wq = o2m.quantize_fp8(w, (128, 128))
            out = (o2m.linear_fp8(x, wq), o2m.orthogonalize(w))
        graphs.append((g, x, w, out))
    for seed in range(4):
        for i, (g, x, w, _) in enumerate(graphs):
            x.copy_(matrix(*x.shape, 70 + 2 * seed + i, torch.bfloat16, spread=0.3))
            w.copy_(matrix(*w.shape, 90 + 2 * seed + i, spread=0.3))
        eager = [(o2m.linear_fp8(x, o2m.quantize_fp8(w, (128, 128))), o2m.orthogonalize(w)) for _, x, w, _ in graphs]
        torch.cuda.synchronize()
        for g, *_ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (_, _, _, out), want in zip(graphs, eager):
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), seed


# ---- beyond 2^31 entries, and the largest update ----------------------------------

def same_bits(a, b):
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


def test_quantize_past_32_bits(o2m):
    """Rows and columns at the end of a matrix of more than 2^31 entries."""
    rows, k = 66000, 33000
    x = torch.randn((rows, k), dtype=torch.bfloat16, device=DEV)
    q, qt = o2m.quantize_fp8_pair(x)
    assert same_bits((q.values[-200:], q.scales[-200:]), o2m.quantize_fp8(x[-200:]))
    assert same_bits((qt.values[-200:], qt.scales[-200:]), o2m.quantize_fp8(x[:, -200:].t()))
    only = o2m.quantize_fp8(x)
    assert same_bits((only.values[-200:], only.scales[-200:]), (q.values[-200:], q.scales[-200:]))


@pytest.mark.parametrize("scales,dtype", [("pow2", torch.bfloat16), ("float32", torch.float16), ("pow2", torch.float32)])
def test_gemm_past_32_bits(o2m, scales, dtype):
    """A result of more than 2^31 entries, in either order: its first and last rows."""
    m, n, k = 66000, 33000, 40
    A = o2m.quantize_fp8(matrix(m, k, 61, spread=0.5), scales=scales)
    B = o2m.quantize_fp8(matrix(n, k, 62, spread=0.5), scales=scales)
    a, b = R.values64(A, 1), R.values64(B, 1)
    for out in (torch.empty((m, n), dtype=dtype, device=DEV), torch.empty((n, m), dtype=dtype, device=DEV).t()):
        o2m.gemm_fp8(A, B, out=out)
        for part in (slice(0, 30), slice(m - 30, m)):
            R.check_product(out[part], a[part], b, dtype)


def test_orthogonalize_largest(o2m):
    """2^29 entries, one per row not zero: X stays such a matrix, of the scalars x <-
    a x + b x^3 + c x^5.  All sums have one term, so what is off is the roundings of
    held numbers, u = 2^-21 relative each (two fp16 parts): X before the first
    step, with the norm's inverse below u / 4, and in a step B (A, of at most 0.02
    in B, adds below 0.05 u) and X, with three fp32 roundings of u / 4: below 3 u a
    step, 8 u in all with the last rounding."""
    r, c = 16384, 32768
    g = torch.zeros((r, c), device=DEV)
    g.diagonal().fill_(3.0)
    x = o2m.orthogonalize(g, steps=2)
    s = 1.0 / 128
    for _ in range(2):
        s = R.COEF[0] * s + R.COEF[1] * s ** 3 + R.COEF[2] * s ** 5
    assert (x.diagonal().double() - s).abs().max().item() <= 8 * 2.0 ** -21 * s
    x.diagonal().zero_()
    assert not x.any()
