"""The products of trained models at their edges: calls at the limits of a kernel's
range, results and inputs in one memory, and steps of the update one by one."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import model_reference as R  # noqa: E402
from fp8_shapes import SPLIT, SPLIT_LINEAR  # noqa: E402
from test_gpu_model_ops import DEV, E4M3, TYPES, matrix, o2m, padded_operand  # noqa: E402,F401

pytestmark = pytest.mark.gpu


# ---- the update of small matrices: one workgroup each ------------------------------

@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 200), (96, 80), (33, 90), (64, 64), (150, 60)])
@pytest.mark.parametrize("dtype", TYPES)
def test_small_update_without_steps(o2m, rows, cols, dtype):  # noqa: F811
    """X = G / (||G|| + eps), held in one or two fp16 parts of X 2^14 and rounded to the type: half a
    step of each of the two roundings, and one of 2^-23 for the quotient in fp32; the numbers that fp16
    holds end at 2^-24, so an entry may be off by half of that, 2^-39 of X."""
    for order in ("row", "col"):
        g = matrix(rows, cols, 13, torch.float32, order, spread=1.0)
        g = g.to(dtype) if order == "row" else g.t().contiguous().to(dtype).t()
        print("no steps", rows, cols, dtype, order, flush=True)
        got = o2m.orthogonalize(g, steps=0).double().cpu().numpy()
        exact = g.double().cpu().numpy()
        exact = exact / (np.linalg.norm(exact) + 1e-7)
        one = R.half_step(torch.float16)
        u = (one if dtype == torch.bfloat16 else 2 * one * one) + R.half_step(dtype) + 2.0 ** -23
        tiny = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}[dtype] + 2.0 ** -39
        assert (np.abs(got - exact) <= 1.01 * u * np.abs(exact) + tiny).all()


@pytest.mark.parametrize("steps", [0, 2])
def test_most_small_updates(o2m, steps):  # noqa: F811
    """65535 matrices in one call, each as if it were alone, and next to no scratch memory."""
    g = torch.randn((65535, 20, 33), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    x = o2m.orthogonalize(g, steps=steps)
    torch.cuda.synchronize()
    assert torch.cuda.max_memory_allocated() - before <= x.numel() * 4 + (4 << 20)
    for i in (0, 1, 40000, 65534):
        assert torch.equal(x[i], o2m.orthogonalize(g[i], steps=steps))


# ---- results in the memory of inputs ------------------------------------------------

@pytest.mark.parametrize("tokens", [1, 3, 16, 40])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_into_its_tokens(o2m, tokens, dtype):  # noqa: F811
    """The layer's result in its tokens' place, over a part of them, beside them and behind them: as if
    it were elsewhere, for sizes of one launch and of several."""
    k, n = 700, 700
    W = o2m.quantize_fp8(matrix(n, k, 5, spread=0.3), (128, 128))
    x0 = matrix(tokens, k, 6, dtype, spread=0.3)
    want = o2m.linear_fp8(x0, W)
    for first, width in ((0, k), (300, 1000), (k, 2 * k)):   # the output's first column, a row's entries
        buf = torch.zeros((tokens, width), dtype=dtype, device=DEV)
        buf[:, :k] = x0
        out = buf[:, first:first + n]
        assert o2m.linear_fp8(buf[:, :k], W, out=out) is out
        assert torch.equal(out, want)
        assert torch.equal(buf[:, :min(first, k)], x0[:, :min(first, k)])
    flat = torch.zeros(2 * tokens * k, dtype=dtype, device=DEV)
    x, out = flat[:tokens * k].view(tokens, k), flat[tokens * k:].view(tokens, n)
    x.copy_(x0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2m.linear_fp8(x, W, out=out, stream=side)
    o2m.linear_fp8(x, W, out=x, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(x, want)


@pytest.mark.parametrize("n", [24, 70, 300])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_updates_into_their_own_memory(o2m, n, dtype):  # noqa: F811
    """A batch into its own memory in the same layout, across, a matrix further on, and beside itself in
    rows of one pitch: as if it were elsewhere, for sizes of one launch and of several."""
    b = 40
    g0 = torch.stack([matrix(n, n, 40 + i, dtype, spread=0.3) for i in range(b)])
    want = o2m.orthogonalize(g0)
    for into in (lambda g: g, lambda g: g.transpose(1, 2)):
        g = g0.clone()
        out = into(g)
        assert o2m.orthogonalize(g, out=out) is out
        assert torch.equal(out, want)
    buf = torch.zeros((b + 1, n, n), dtype=dtype, device=DEV)
    for g, out in ((buf[:b], buf[1:]), (buf[1:], buf[:b])):
        g.copy_(g0)
        assert torch.equal(o2m.orthogonalize(g, out=out), want)
    for first in (n, n // 2):
        wide = torch.zeros((b, n, 2 * n), dtype=dtype, device=DEV)
        g, out = wide[:, :, :n], wide[:, :, first:first + n]
        g.copy_(g0)
        assert torch.equal(o2m.orthogonalize(g, out=out), want)
        assert torch.equal(wide[:, :, :first], g0[:, :, :first])


# ---- the update step by step ----------------------------------------------------------

TRIPLES = [(3.4445, -4.7750, 2.0315), (3.0, -3.2, 1.2), (2.5, -2.0, 0.5), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 200), (96, 80), (33, 90), (64, 64), (60, 150), (100, 140), (130, 129),
                                       (64, 500), (513, 300), (900, 1000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_update_step_by_step(o2m, rows, cols, dtype):  # noqa: F811
    """The update of no, one, .. five steps, each against one step of the definition on the result of the
    one before, within a bound that is far below the result (test_update_bound.py): matrices of one
    launch and of several, coefficients of their own for each step."""
    parts = 1 if dtype == torch.bfloat16 else 2
    g = torch.stack([matrix(rows, cols, 21 + i, dtype, spread=0.3) for i in range(2)])
    x = g[1].double().cpu().numpy()
    x = x / (np.linalg.norm(x) + 1e-7)
    got = o2m.orthogonalize(g, steps=0)[1].double().cpu().numpy()
    one = R.half_step(torch.float16)
    u = (one if parts == 1 else one * one) + R.half_step(dtype) + 2.0 ** -23
    tiny = 2.0 ** -39 + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    assert (np.abs(got - x) <= 1.01 * u * np.abs(x) + tiny).all()
    for t, coef in enumerate(TRIPLES):
        print("step", t + 1, rows, cols, dtype, flush=True)
        x = got
        got = o2m.orthogonalize(g, steps=t + 1, coefficients=TRIPLES[:t + 1])[1].double().cpu().numpy()
        exact = R.orthogonalize_step(x, coef)
        bound = R.orthogonalize_step_bound(x, coef, parts, dtype)
        off = np.linalg.norm(got - exact)
        assert off <= bound, (t, off / bound, bound / np.linalg.norm(exact))
    # one triple for all steps
    assert torch.equal(o2m.orthogonalize(g, steps=3, coefficients=TRIPLES[1]),
                       o2m.orthogonalize(g, steps=3, coefficients=[TRIPLES[1]] * 3))


# ---- products split along k (test_fp8_plan.py: that they are) ----------------------------

def check_outputs(o2m, m, n, k, scales, dtype):  # noqa: F811
    """Either order of the result, fresh or added to, rows of odd pitch behind which nothing changes, a row
    of NaN and a column of it."""
    a, b = matrix(m, k, 71, spread=0.5), matrix(n, k, 72, spread=0.5)
    a[m // 2, k // 3], b[n - 1, k - 1] = float("nan"), float("inf")
    A, _ = padded_operand(o2m, a, 1, E4M3, scales)
    B = o2m.quantize_fp8(b, (128, 128), R.E5M2 if m % 2 else E4M3, scales)
    print("outputs", m, n, k, scales, dtype, flush=True)
    want = (R.values64(A, 1), R.values64(B, 128), dtype)
    C = o2m.gemm_fp8(A, B, dtype=dtype)
    R.check_product(C, *want)
    for order in ("row", "col"):
        for add in (False, True):
            buf = torch.full((m + 3, n + 5) if order == "row" else (n + 3, m + 5), 7.0, dtype=dtype, device=DEV)
            out = buf[1:1 + m, 2:2 + n] if order == "row" else buf[1:1 + n, 2:2 + m].t()
            assert o2m.gemm_fp8(A, B, out=out, accumulate=add) is out
            R.check_product(out, *want, 7.0 * np.ones((m, n)) if add else None)
            if order == "row" and not add:
                assert torch.equal(out.contiguous().view(torch.uint8), C.view(torch.uint8))   # NaN as well
            out.fill_(7.0)
            assert (buf == 7.0).all()


@pytest.mark.parametrize("m,n,k,splits", SPLIT)
@pytest.mark.parametrize("scales", ["pow2", "float32"])
@pytest.mark.parametrize("dtype", TYPES)
def test_gemm_in_splits(o2m, m, n, k, splits, scales, dtype):  # noqa: F811
    """Sums of splits joined."""
    check_outputs(o2m, m, n, k, scales, dtype)


@pytest.mark.parametrize("m,n,k", [(1, 77, 300), (5, 90, 300), (90, 31, 1041), (77, 150, 270), (1290, 1601, 97), (1800, 4090, 300),
                                   (3700, 3601, 200)])
@pytest.mark.parametrize("scales", ["pow2", "float32"])
@pytest.mark.parametrize("dtype", TYPES)
def test_gemm_into_outputs(o2m, m, n, k, scales, dtype):  # noqa: F811
    """The same for few rows on one side and for tiles of every size."""
    check_outputs(o2m, m, n, k, scales, dtype)


@pytest.mark.parametrize("tokens,n,k", SPLIT_LINEAR)
@pytest.mark.parametrize("scales", ["pow2", "float32"])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_in_splits(o2m, tokens, n, k, scales, dtype):  # noqa: F811
    """The scratch memory holds the quantized tokens and, behind them, the splits' sums."""
    x = matrix(tokens, k, 73, dtype, spread=0.5)
    W, _ = padded_operand(o2m, matrix(n, k, 74, spread=0.5), 128, E4M3, scales)
    buf = torch.full((tokens + 1, n + 3), 7.0, dtype=dtype, device=DEV)
    y = o2m.linear_fp8(x, W, out=buf[:tokens, :n])
    q, s = R.quantize(x.float().cpu().numpy(), 1, E4M3, scales)
    R.check_product(y, q * R.spread(s, 1, tokens, k), R.values64(W, 128), dtype)
    assert (buf[:, n:] == 7).all() and (buf[tokens:] == 7).all()


@pytest.mark.parametrize("scales,fmt", [("pow2", E4M3), ("float32", R.E5M2)])
def test_weight_gradient_over_many_tokens(o2m, scales, fmt):  # noqa: F811
    """dW of 10007 tokens, in splits, added to the gradient of the batch before."""
    tokens, n, k = 10007, 99, 131
    _, xt = o2m.quantize_fp8_pair(matrix(tokens, k, 75, torch.bfloat16, spread=0.3), scales=scales)
    _, wt = o2m.quantize_fp8_pair(matrix(n, k, 76, spread=0.3), (128, 128), scales=scales)
    dw = None
    for i in range(3):
        dy = matrix(tokens, n, 77 + i, torch.bfloat16, spread=0.3)
        first = None if dw is None else dw.double().cpu().numpy()
        _, dw = o2m.linear_fp8_backward(dy, xt, wt, dtype=fmt, dW=dw, accumulate=dw is not None)
        qt, st = R.quantize(dy.float().cpu().numpy().T, 1, fmt, scales)
        R.check_product(dw, qt * R.spread(st, 1, n, tokens), R.values64(xt, 1), torch.float32, first)


@pytest.mark.parametrize("m,n,k", [(5, 90, 512), (70, 90, 512), (301, 299, 8200), (1900, 2100, 512), (3700, 3600, 400)])
@pytest.mark.parametrize("scales", ["pow2", "float32"])
def test_gemm_of_cancelling_channels(o2m, m, n, k, scales):  # noqa: F811
    """Two outlier channels in different groups of 8 whose products cancel exactly: what is left is the
    sum of the small ones, each entry within the bound that the largest of every group gives for 16-bit
    results, and within fp32's for fp32 ones."""
    a, b = matrix(m, k, 81, spread=0.3), matrix(n, k, 82, spread=0.3)
    a[:, 17], a[:, k - 3] = 256.0, 256.0
    b[:, 17], b[:, k - 3] = 256.0, -256.0
    A, B = o2m.quantize_fp8(a, scales=scales), o2m.quantize_fp8(b, scales=scales)
    for dtype in TYPES:
        R.check_product(o2m.gemm_fp8(A, B, dtype=dtype), R.values64(A, 1), R.values64(B, 1), dtype)


# ---- batches whose matrices lie side by side ---------------------------------------------

@pytest.mark.parametrize("rows,cols", [(20, 33), (33, 20), (300, 200), (1, 50)])
@pytest.mark.parametrize("dtype", TYPES)
def test_updates_side_by_side(o2m, rows, cols, dtype):  # noqa: F811
    """Heads that share their rows' memory, (rows, heads, cols) as (heads, rows, cols), in and out and in place."""
    b = 5
    g0 = torch.stack([matrix(rows, cols, 60 + i, dtype, spread=0.3) for i in range(b)])
    want = o2m.orthogonalize(g0)
    side = torch.full((rows + 1, b, cols + 3), 7.0, dtype=dtype, device=DEV)
    out = side[:rows, :, :cols].transpose(0, 1)
    assert o2m.orthogonalize(g0, out=out) is out
    assert torch.equal(out, want)
    out.copy_(g0)
    assert torch.equal(o2m.orthogonalize(out), want)
    assert torch.equal(o2m.orthogonalize(out, out=out), want)
    out.fill_(7.0)
    assert (side == 7.0).all()


# ---- graphs and streams -------------------------------------------------------------------

def test_graphs_of_a_training_step(o2m):  # noqa: F811
    """Two captured training steps of layers whose products are split and whose updates take one launch and
    several, replayed in turn with eager work between; each replay as the eager step on the same inputs."""
    def step(x, w, dy, total):
        xq, xt = o2m.quantize_fp8_pair(x)
        wq, wt = o2m.quantize_fp8_pair(w, (128, 128))
        y = o2m.gemm_fp8(xq, wq)
        dx, dw = o2m.linear_fp8_backward(dy, xt, wt, dW=total, accumulate=True)
        return y, o2m.linear_fp8(x[:1], wq), dx, dw, o2m.orthogonalize(dw)

    shapes = [(8200, 65, 90), (70, 501, 4096)]   # tokens, n, k
    side, graphs = torch.cuda.Stream(), []
    for i, (t, n, k) in enumerate(shapes):
        args = [torch.zeros((t, k), dtype=torch.bfloat16, device=DEV), torch.zeros((n, k), device=DEV),
                torch.zeros((t, n), dtype=torch.bfloat16, device=DEV), torch.zeros((n, k), device=DEV)]
        step(*args)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            out = step(*args)
        graphs.append((g, args, out))
    for seed in range(4):
        want = []
        for i, (g, args, _) in enumerate(graphs):
            for j, a in enumerate(args):
                a.copy_(matrix(*a.shape, 100 + 10 * seed + 5 * i + j, a.dtype, spread=0.3))
            want.append([v.clone() for v in step(*args[:3], args[3].clone())])
        torch.cuda.synchronize()
        for g, *_ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (_, _, out), ref in zip(graphs, want):
            for a, b in zip(out, ref):
                assert torch.equal(a, b), seed


# ---- the longest rows ---------------------------------------------------------------------

@pytest.mark.parametrize("m,n", [(3, 40), (40, 65), (2100, 2049)])
@pytest.mark.parametrize("scales", ["pow2", "float32"])
def test_gemm_of_the_longest_rows(o2m, m, n, scales):  # noqa: F811
    """Rows of 2^23 - 16 values, the pitch at which offsets within a tile come closest to 2^31: row i holds
    one power of two throughout, so every sum is exact and a result is rounded once."""
    k = (1 << 23) - 16
    code = torch.tensor([0x38, 0x30, 0x40, 0xB8], dtype=torch.uint8, device=DEV)      # 1, 1/2, 2, -1 in e4m3
    value = torch.tensor([1.0, 0.5, 2.0, -1.0], dtype=torch.float64, device=DEV)

    def operand(rows):
        kind = (torch.arange(rows, device=DEV) * 7 // 3) % 4
        q = torch.empty((rows, k), dtype=torch.uint8, device=DEV)
        q.copy_(code[kind][:, None])
        s = torch.full((-(-k // 128), rows), 127, dtype=torch.uint8, device=DEV) if scales == "pow2" else \
            torch.ones((-(-k // 128), rows), device=DEV)
        return (q.view(E4M3), s.t()), value[kind]
    (A, a), (B, b) = operand(m), operand(n)
    exact = k * a[:, None] * b[None, :]
    for dtype in (torch.bfloat16, torch.float32):
        print("longest", m, n, scales, dtype, flush=True)
        C = o2m.gemm_fp8(A, B, dtype=dtype)
        assert torch.equal(C, exact.to(dtype))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("r", [1, 256])
def test_update_of_the_longest_rows(o2m, r, dtype):  # noqa: F811
    """Rows of 2^21 entries, up to 2^29 in all, one per row not zero: X stays such a matrix, of the scalars
    x <- a x + b x^3 + c x^5.  All sums have one term, so what is off is the roundings of held numbers,
    u relative each (2^-11 in one fp16 part, 2^-21 in two), and of fp32, u / 8.  An error of x comes out of a step
    multiplied by |p'| x / p; the step adds A's, by |b A + 2 c A^2| / |B|, B's, those of B's three terms, by the
    largest one / |B| and 3 / 8, and X's.  One row: x is 1, 0.70, 1.11.  First step 1.03 + 1.02 + 1 + 2.6 + 1 = 6.7 u,
    second 0.72 * 6.7 + 0.86 + 1 + 0.8 + 1 = 8.5 u, below 20.  256 rows: x is 1/16, 0.21, 0.69.  First 1 + 0.01 + 1 +
    0.4 + 1 = 3.4 u, second 0.9 * 3.4 + 0.1 + 1 + 0.4 + 1 = 5.6 u, below 8.  Then the result's rounding."""
    c = 1 << 21
    u = 2.0 ** (-11 if dtype == torch.bfloat16 else -21)
    g = torch.zeros((r, c), dtype=dtype, device=DEV)
    g[:, 1000:1000 + r].diagonal().fill_(3.0)
    x = o2m.orthogonalize(g, steps=2)
    s = 1.0 / r ** 0.5
    for _ in range(2):
        s = R.COEF[0] * s + R.COEF[1] * s ** 3 + R.COEF[2] * s ** 5
    d = x[:, 1000:1000 + r].diagonal()
    assert (d.double() - s).abs().max().item() <= ((20 if r == 1 else 8) * u + R.half_step(dtype)) * abs(s)
    d.zero_()
    assert not x.any()
