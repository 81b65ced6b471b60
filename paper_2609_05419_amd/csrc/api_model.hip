// C-ABI entry points of the products of trained models (include/o2m.h):
// argument checks on the host, then kernels on the caller's stream.  Scratch
// memory is the caller's, so nothing here keeps state between calls.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include "model_internal.h"

using namespace o2m;

namespace {

o2m_status hip_fail(hipError_t e) {
    if (e == hipSuccess) return O2M_OK;
    if (getenv("O2M_LOG")) fprintf(stderr, "o2m: HIP error %d (%s)\n", (int)e, hipGetErrorString(e));
    return e == hipErrorInvalidValue ? O2M_ERR_SIZE : O2M_ERR_HIP;
}

bool type_ok(int t) { return t == O2M_TYPE_F32 || t == O2M_TYPE_F16 || t == O2M_TYPE_BF16; }
int type_bytes(int t) { return t == O2M_TYPE_F32 ? 4 : 2; }

// 'R' and 'C' in either case; 0 otherwise
char order_of(char c) { return c == 'R' || c == 'r' ? 'R' : c == 'C' || c == 'c' ? 'C' : 0; }

bool aligned(const void *p, size_t q) { return reinterpret_cast<uintptr_t>(p) % q == 0; }

// An operand of rows of k values.  Row pitches stay below 2^23 bytes, so that
// every offset within a tile of 256 rows fits 31 bits.
constexpr int64_t kMaxPitch = 1 << 23;
bool operand_ok(const o2m_fp8_operand *o, int k) {
    return o && o->values && aligned(o->values, 16) && o->ld >= k && o->ld % 16 == 0 && o->scales && o->s_row >= 0 &&
           o->s_blk >= 0 && (o->block == 1 || o->block == kBlockK) &&
           (o->format == O2M_FP8_E4M3 || o->format == O2M_FP8_E5M2) &&
           (o->scale_type == O2M_SCALES_POW2 || (o->scale_type == O2M_SCALES_F32 && aligned(o->scales, 4)));
}

// Scales to be written have a place each.
bool scales_apart(const o2m_fp8_operand *o, int rows, int k) {
    const int64_t r = o->block == 1 ? rows : ceil_div(rows, kBlockK), b = ceil_div(k, kBlockK);
    return (r == 1 || o->s_row >= 1) && (b == 1 || o->s_blk >= 1) &&
           (r == 1 || b == 1 || o->s_row > (b - 1) * o->s_blk || o->s_blk > (r - 1) * o->s_row);
}

// Sizes up to here, so that a row past the last tile is still an int.
constexpr int kMaxSize = 0x7FFFFFFF - 1023;

// `lines` runs of `bytes` bytes, `pitch` apart.
struct Runs {
    const void *at;
    int64_t lines, pitch, bytes;
};
// Whether two such sets may share a byte: not if they lie one behind the other, or
// side by side in rows of one pitch.
bool may_meet(const Runs &x, const Runs &y) {
    const int64_t d = static_cast<const char *>(y.at) - static_cast<const char *>(x.at);
    if (d >= (x.lines - 1) * x.pitch + x.bytes || -d >= (y.lines - 1) * y.pitch + y.bytes) return false;
    if (x.pitch != y.pitch || x.pitch <= 0) return true;
    const int64_t in = (d % x.pitch + x.pitch) % x.pitch;
    return in < x.bytes || x.pitch - in < y.bytes;
}

o2m_status check_workspace(size_t need, const void *ws, size_t bytes) {
    if (need == 0) return O2M_OK;
    return ws && bytes >= need && aligned(ws, 256) ? O2M_OK : O2M_ERR_WORKSPACE;
}

// Quantized X of a linear layer, in the workspace: values, then scales.
o2m_fp8_operand kept_x(int tokens, int k, int scale_type, void *ws) {
    o2m_fp8_operand q;
    q.values = ws;
    q.ld = round_up64(k, 16);
    q.scales = ws ? static_cast<char *>(ws) + round_up64((int64_t)tokens * q.ld, 256) : nullptr;
    q.s_row = 1;
    q.s_blk = tokens;
    q.block = 1;
    q.format = O2M_FP8_E4M3;
    q.scale_type = scale_type;
    return q;
}
size_t kept_x_bytes(int tokens, int k) {
    return (size_t)(round_up64((int64_t)tokens * round_up64(k, 16), 256) +
                    round_up64(4 * (int64_t)tokens * ceil_div(k, kBlockK), 256));
}

}  // namespace

extern "C" {

o2m_status o2m_quantize_fp8(int rows, int k, const void *X, int x_type, char x_order, int64_t ldx,
                            const o2m_fp8_operand *Q, const o2m_fp8_operand *Qt, void *stream) {
    if (rows < 0) return -1;
    if (k < 0) return -2;
    const bool any = rows > 0 && k > 0;
    if (any && !X) return -3;
    if (!type_ok(x_type)) return -4;
    if (any && !aligned(X, type_bytes(x_type))) return -3;
    const char order = order_of(x_order);
    if (!order) return -5;
    if (ldx < (order == 'R' ? k : rows) || ldx < 1) return -6;
    if (!Q && !Qt) return -7;
    if (!any) return O2M_OK;
    if (Q && (!operand_ok(Q, k) || !scales_apart(Q, rows, k))) return -7;
    if (Qt && (!operand_ok(Qt, rows) || !scales_apart(Qt, k, rows))) return -8;
    if (Q && Qt && (Q->values == Qt->values || Q->scales == Qt->scales)) return -8;
    if (rows > kMaxSize || k > kMaxSize) return O2M_ERR_SIZE;
    const hipStream_t st = (hipStream_t)stream;
    return hip_fail(order == 'R' ? launch_quantize(rows, k, X, x_type, ldx, Q, Qt, st)
                                 : launch_quantize(k, rows, X, x_type, ldx, Qt, Q, st));
}

size_t o2m_gemm_fp8_workspace(int m, int n, int k) { return m > 0 && n > 0 && k > 0 ? gemm_fp8_workspace(m, n, k) : 0; }

o2m_status o2m_gemm_fp8(int m, int n, int k, const o2m_fp8_operand *A, const o2m_fp8_operand *B, void *C, int c_type,
                        char c_order, int64_t ldc, int accumulate, void *workspace, size_t workspace_bytes,
                        void *stream) {
    if (m < 0) return -1;
    if (n < 0) return -2;
    if (k < 0) return -3;
    const bool any = m > 0 && n > 0;
    if (any && k > 0) {
        if (!operand_ok(A, k)) return -4;
        if (!operand_ok(B, k) || B->scale_type != A->scale_type) return -5;
    }
    if (any && !C) return -6;
    if (!type_ok(c_type)) return -7;
    if (any && !aligned(C, type_bytes(c_type))) return -6;
    const char order = order_of(c_order);
    if (!order) return -8;
    if (ldc < (order == 'R' ? n : m) || ldc < 1) return -9;
    if (!any) return O2M_OK;
    const hipStream_t st = (hipStream_t)stream;
    const bool swap = order == 'C';
    if (k == 0) {
        if (accumulate) return O2M_OK;
        return hip_fail(launch_zero_out(C, swap ? m : n, swap ? n : m, ldc, type_bytes(c_type), st));
    }
    if (A->ld >= kMaxPitch || B->ld >= kMaxPitch || m > kMaxSize || n > kMaxSize) return O2M_ERR_SIZE;
    const o2m_status s = check_workspace(gemm_fp8_workspace(m, n, k), workspace, workspace_bytes);
    if (s != O2M_OK) return s;
    return hip_fail(swap ? launch_gemm_fp8(n, m, k, *B, *A, C, c_type, ldc, accumulate != 0, workspace, st)
                         : launch_gemm_fp8(m, n, k, *A, *B, C, c_type, ldc, accumulate != 0, workspace, st));
}

size_t o2m_linear_fp8_workspace(int tokens, int n, int k) {
    if (tokens <= 0 || n <= 0 || k <= 0 || linear_is_fused(tokens, k)) return 0;
    return kept_x_bytes(tokens, k) + gemm_fp8_workspace(tokens, n, k);
}

o2m_status o2m_linear_fp8(int tokens, int n, int k, const void *X, int x_type, int64_t ldx, const o2m_fp8_operand *W,
                          void *Y, int64_t ldy, void *workspace, size_t workspace_bytes, void *stream) {
    if (tokens < 0) return -1;
    if (n < 0) return -2;
    if (k < 0) return -3;
    const bool any = tokens > 0 && n > 0;
    if (any && k > 0 && !X) return -4;
    if (!type_ok(x_type)) return -5;
    if (any && k > 0 && !aligned(X, type_bytes(x_type))) return -4;
    if (ldx < k || ldx < 1) return -6;
    if (any && k > 0 && !operand_ok(W, k)) return -7;
    if (any && (!Y || !aligned(Y, type_bytes(x_type)))) return -8;
    if (ldy < n || ldy < 1) return -9;
    if (!any) return O2M_OK;
    const hipStream_t st = (hipStream_t)stream;
    if (k == 0) return hip_fail(launch_zero_out(Y, n, tokens, ldy, type_bytes(x_type), st));
    if (W->ld >= kMaxPitch || round_up64(k, 16) >= kMaxPitch || tokens > kMaxSize || n > kMaxSize) return O2M_ERR_SIZE;
    const o2m_status s = check_workspace(o2m_linear_fp8_workspace(tokens, n, k), workspace, workspace_bytes);
    if (s != O2M_OK) return s;
    const bool fused = linear_is_fused(tokens, k);
    const int64_t size = type_bytes(x_type);
    // (every workgroup reads the tokens, others may have written by then)
    if (fused && may_meet({X, tokens, ldx * size, k * size}, {Y, tokens, ldy * size, n * size})) return -8;
    if (fused) return hip_fail(launch_linear_fused(tokens, n, k, X, x_type, ldx, *W, Y, ldy, st));
    // (the product is checked before the tokens are quantized)
    if (!gemm_fp8_fits(tokens, n, k, W->scale_type, x_type)) return O2M_ERR_SIZE;
    const o2m_fp8_operand q = kept_x(tokens, k, W->scale_type, workspace);
    const hipError_t e = launch_quantize(tokens, k, X, x_type, ldx, &q, nullptr, st);
    if (e != hipSuccess) return hip_fail(e);
    return hip_fail(launch_gemm_fp8(tokens, n, k, q, *W, Y, x_type, ldy, false,
                                    static_cast<char *>(workspace) + kept_x_bytes(tokens, k), st));
}

size_t o2m_orthogonalize_workspace(int batch, int rows, int cols, int type) {
    if (batch <= 0 || rows <= 0 || cols <= 0 || !type_ok(type)) return 0;
    return ortho_workspace(batch, rows < cols ? rows : cols, rows < cols ? cols : rows, type);
}

o2m_status o2m_orthogonalize(int batch, int rows, int cols, const void *G, char order_g, int64_t ldg, int64_t stride_g,
                             void *O, char order_o, int64_t ldo, int64_t stride_o, int type, int steps,
                             const double *coef, double eps, void *workspace, size_t workspace_bytes, void *stream) {
    if (batch < 0) return -1;
    if (rows < 0) return -2;
    if (cols < 0) return -3;
    const bool any = batch > 0 && rows > 0 && cols > 0;
    if (!type_ok(type)) return -12;
    if (any && (!G || !aligned(G, type_bytes(type)))) return -4;
    const char og = order_of(order_g), oo = order_of(order_o);
    if (!og) return -5;
    if (ldg < (og == 'R' ? cols : rows) || ldg < 1) return -6;
    if (stride_g < 0) return -7;
    if (any && (!O || !aligned(O, type_bytes(type)))) return -8;
    if (!oo) return -9;
    if (ldo < (oo == 'R' ? cols : rows) || ldo < 1) return -10;
    // the matrices of a batch must not share entries: they lie one behind the other, or side by side
    // within a row of ldo
    const int64_t lines_o = oo == 'R' ? rows : cols, len_o = oo == 'R' ? cols : rows;
    if (stride_o < 0 || (any && batch > 1 && stride_o < ldo * (lines_o - 1) + len_o &&
                         (stride_o < len_o || ldo < stride_o * (batch - 1) + len_o)))
        return -11;
    if (steps < 0 || steps > 64 || (steps > 0 && !coef) || !(eps >= 0.0) || !isfinite(eps)) return O2M_ERR_STEPS;
    for (int i = 0; i < 3 * steps; ++i)
        if (!isfinite(coef[i])) return O2M_ERR_STEPS;
    if (!any) return O2M_OK;
    const bool tall = rows > cols;
    const int r = tall ? cols : rows, c = tall ? rows : cols;
    // offsets within a tile, and within the two parts of a matrix; the tiles of a launch
    const int64_t rt = ceil_div(r, 64), ct = ceil_div(c, 64);
    if (c > (1 << 21) || (rt * ct) << 12 > (1 << 29) || batch > 65535 || 256 * rt * ct > 0x7FFFFFFF / (int64_t)batch) return O2M_ERR_SIZE;
    const o2m_status s = check_workspace(ortho_workspace(batch, r, c, type), workspace, workspace_bytes);
    if (s != O2M_OK) return s;
    // Workgroups that have a matrix each finish while others still read theirs.  (Longer
    // updates, and one matrix alone, are read in full before anything is written.)
    const bool same = G == O && og == oo && ldg == ldo && stride_g == stride_o;
    if (batch > 1 && !same && ortho_is_small(r, c, type)) {
        const int64_t size = type_bytes(type);
        auto whole = [&](const void *at, char order, int64_t ld, int64_t stride) {
            const int64_t lines = order == 'R' ? rows : cols, len = order == 'R' ? cols : rows;
            return Runs{at, batch, stride * size, (ld * (lines - 1) + len) * size};
        };
        auto lines = [&](const void *at, char order, int64_t ld, int64_t stride) {
            return Runs{at, stride / ld * (batch - 1) + (order == 'R' ? rows : cols), ld * size, (order == 'R' ? cols : rows) * size};
        };
        const bool one_pitch = ldg == ldo && stride_g % ldg == 0 && stride_o % ldo == 0;
        if (may_meet(whole(G, og, ldg, stride_g), whole(O, oo, ldo, stride_o)) &&
            !(one_pitch && !may_meet(lines(G, og, ldg, stride_g), lines(O, oo, ldo, stride_o))))
            return -8;
    }
    OrthoArgs a;
    a.batch = batch;
    a.rows = r;
    a.cols = c;
    a.G = G;
    a.g_row = (og == 'R') != tall ? ldg : 1;
    a.g_col = (og == 'R') != tall ? 1 : ldg;
    a.g_batch = stride_g;
    a.O = O;
    a.o_row = (oo == 'R') != tall ? ldo : 1;
    a.o_col = (oo == 'R') != tall ? 1 : ldo;
    a.o_batch = stride_o;
    a.type = type;
    a.steps = steps;
    a.coef = coef;
    a.eps = eps;
    return hip_fail(launch_ortho(a, workspace, (hipStream_t)stream));
}

}  // extern "C"
