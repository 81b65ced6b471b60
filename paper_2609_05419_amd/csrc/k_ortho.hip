// The orthogonalised update (include/o2m.h: o2m_orthogonalize):
//
//   X = G / (||G|| + eps);  steps x:  A = X X^T, B = b A + c A^2, X <- a X + B X
//
// on the work matrix X (r x c, r <= c, G transposed where it is tall).  Three
// products per step: A and A^2 symmetric, so half their tiles are computed and
// mirrored, then B X with a X added as it is stored.
//
// Held numbers.  Entries of X are of the size 1 / sqrt(c) in the end, those of A
// and B up to 1 and 3: matrices are held in fp16, as X 2^s with 2^s next to
// sqrt(c), A 2^8 and B 2^7, which keeps them within fp16's normal range.  For bf16
// updates one fp16 part is kept, whose 11 bits put the held matrices'
// roundings below the result's own; fp32 and fp16 updates keep a second part,
// lo = (x - hi) 2^11, also fp16, and multiply hi hi + 2^-11 (hi lo + lo hi): the
// cross terms are summed first, scaled once, and the main product is summed on
// top, all in fp32.  What is left out, lo lo, is 2^-24 of the product.
//
// Layout.  All held matrices are padded with zeros to multiples of 128, so no
// product has a ragged edge.  X is kept both as it is (the rows that A
// multiplies) and transposed (the rows that B X multiplies); the product that
// makes it writes both.
//
// Bound: fp16 MFMA, 2 r^2 c + (r^2 c + r^3) / 1 products of a step.
#include "mfma_tiles.h"
#include "model_internal.h"

#include <algorithm>
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <math.h>

namespace o2m {
namespace {

typedef _Float16 f16;
typedef f16 v8f16 __attribute__((ext_vector_type(8)));

constexpr int kPad = 128;
constexpr int kScaleA = 8, kScaleB = 7, kLowBits = 11;
constexpr int kParts = 256;   // partial sums of the norm, per matrix

struct Planes {
    f16 *hi, *lo;     // lo: null when one part is kept
    int64_t pitch;    // elements of a row
    int64_t batch;    // elements of a matrix
};

__device__ inline float load_any(const void *p, int64_t i, int type) {
    if (type == O2M_TYPE_F32) return static_cast<const float *>(p)[i];
    if (type == O2M_TYPE_F16) return __half2float(static_cast<const __half *>(p)[i]);
    return __bfloat162float(static_cast<const __hip_bfloat16 *>(p)[i]);
}
__device__ inline void store_any(void *p, int64_t i, int type, float v) {
    if (type == O2M_TYPE_F32) static_cast<float *>(p)[i] = v;
    else if (type == O2M_TYPE_F16) static_cast<__half *>(p)[i] = __float2half(v);
    else static_cast<__hip_bfloat16 *>(p)[i] = __float2bfloat16(v);
}

template <bool SPLIT>
__device__ inline float held(const Planes &m, int64_t i) {
    float v = (float)m.hi[i];
    if (SPLIT) v += (float)m.lo[i] * (1.0f / (1 << kLowBits));
    return v;
}
template <bool SPLIT>
__device__ inline void hold(const Planes &m, int64_t i, float v) {
    const f16 hi = (f16)v;
    m.hi[i] = hi;
    if (SPLIT) m.lo[i] = (f16)((v - (float)hi) * (float)(1 << kLowBits));
}

// Sums of squares in fp64, a fixed part per workgroup, so that every run adds
// in the same order.
struct NormArgs {
    const void *G;
    int64_t g_outer, g_batch;
    int outer, inner, type;
    double *parts;
};
__global__ __launch_bounds__(256) void norm_parts(NormArgs g) {
    __shared__ double sums[256];
    const int64_t total = (int64_t)g.outer * g.inner, base = (int64_t)blockIdx.y * g.g_batch;
    double s = 0.0;
    for (int64_t t = blockIdx.x * 256LL + threadIdx.x; t < total; t += kParts * 256LL) {
        const double v = load_any(g.G, base + t / g.inner * g.g_outer + t % g.inner, g.type);
        s += v * v;
    }
    sums[threadIdx.x] = s;
    __syncthreads();
    for (int w = 128; w > 0; w >>= 1) {
        if (threadIdx.x < w) sums[threadIdx.x] += sums[threadIdx.x + w];
        __syncthreads();
    }
    if (threadIdx.x == 0) g.parts[(int64_t)blockIdx.y * kParts + blockIdx.x] = sums[0];
}

struct PrepArgs {
    const void *G;
    int64_t g_row, g_col, g_batch;
    int r, c, type;
    const double *parts;
    double eps;
    double scale;    // 2^s
    Planes x, t;     // X (r x c) and its transpose, padded
    int tiles_c;
};
// X 2^s and its transpose, 64 x 64 entries per workgroup.
template <bool SPLIT>
__global__ __launch_bounds__(256) void prepare_x(PrepArgs g) {
    __shared__ float tile[64][65];
    __shared__ double sums[256];
    const int tid = threadIdx.x, b = blockIdx.y;
    sums[tid] = g.parts[(int64_t)b * kParts + tid];
    __syncthreads();
    for (int w = 128; w > 0; w >>= 1) {
        if (tid < w) sums[tid] += sums[tid + w];
        __syncthreads();
    }
    const double norm = sqrt(sums[0]);
    // Inf and NaN anywhere: NaN everywhere
    const double inv = norm <= 1.7e308 ? g.scale / (norm + g.eps) : (double)NAN;
    const int i0 = blockIdx.x / g.tiles_c * 64, j0 = blockIdx.x % g.tiles_c * 64;
    const bool along_c = g.g_col == 1;
    for (int t = tid; t < 64 * 64; t += 256) {
        const int i = along_c ? t >> 6 : t & 63, j = along_c ? t & 63 : t >> 6;
        float v = 0.0f;
        if (i0 + i < g.r && j0 + j < g.c)
            v = (float)((double)load_any(g.G, b * g.g_batch + (i0 + i) * g.g_row + (j0 + j) * g.g_col, g.type) * inv);
        tile[i][j] = v;
    }
    __syncthreads();
    for (int t = tid; t < 64 * 64; t += 256) {
        const int p = t >> 6, q = t & 63;
        hold<SPLIT>(g.x, b * g.x.batch + (i0 + p) * g.x.pitch + j0 + q, tile[p][q]);
        hold<SPLIT>(g.t, b * g.t.batch + (j0 + p) * g.t.pitch + i0 + q, tile[q][p]);
    }
}

enum Product { kGram, kPoly, kUpdate, kLast };

struct ProductArgs {
    Planes p, q;        // rows multiplied: D = P Q^T
    Planes e;           // kPoly: A, kUpdate, kLast: X, of D's layout (added)
    Planes d, dt;       // D and its transpose (kGram, kPoly: d alone, both halves)
    int kblocks;        // stages of 64
    int mt, nt, tiles;  // tiles of 128 x 128; per matrix
    float add, mul;     // D = add e + mul P Q^T
    void *O;            // kLast
    int64_t o_row, o_col, o_batch;
    int r, c, type;
    float out_scale;
};

// D[i, j] = add e[i, j] + mul sum_k P[i, k] Q[j, k], 128 x 128 per workgroup of 2 x
// 2 waves, 4 x 4 blocks of 16 x 16 each; two stage buffers.
template <bool SPLIT, Product KIND>
__global__ __launch_bounds__(256) void product_tile(ProductArgs g) {
    constexpr int T = kPad, kBuf = 2 * T * kStageRowBytes;
    constexpr bool SYM = KIND == kGram || KIND == kPoly;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kBuf];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = blockIdx.x / g.tiles, t = blockIdx.x % g.tiles;
    int ti, tj;
    if (SYM) {   // the tiles at and below the diagonal, row after row
        ti = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
        while (ti * (ti + 1) / 2 > t) --ti;
        while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
        tj = t - ti * (ti + 1) / 2;
    } else {
        ti = t % g.mt;
        tj = t / g.mt;
    }
    const int i0 = ti * T, j0 = tj * T;
    const CopyLane cl = copy_lane(lane);
    const int ldp = (int)g.p.pitch * 2, ldq = (int)g.q.pitch * 2, kbytes = g.kblocks * kStageRowBytes;
    auto rows = [&](const f16 *m, const Planes &of, int row0, int ld) {
        return rows_of(reinterpret_cast<const uint8_t *>(m + b * of.batch + row0 * of.pitch), T, ld, kbytes);
    };
    const int passes = SPLIT ? 3 : 1;   // lo hi, hi lo, hi hi
    const int total = passes * g.kblocks;
    auto copy = [&](int s) {
        uint8_t *buf = lds + (s & 1) * kBuf;
        const int pass = SPLIT ? s / g.kblocks : 2, kb = SPLIT ? s % g.kblocks : s;
        const auto rp = rows(pass == 0 ? g.p.lo : g.p.hi, g.p, i0, ldp);
        const auto rq = rows(pass == 1 ? g.q.lo : g.q.hi, g.q, j0, ldq);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            copy_rows(rp, buf + (wave * 4 + q) * 1024, cl, wave * 4 + q, ldp, kb, kStageRowBytes);
            copy_rows(rq, buf + T * kStageRowBytes + (wave * 4 + q) * 1024, cl, wave * 4 + q, ldq, kb, kStageRowBytes);
        }
    };
    const int wi = (wave >> 1) * 64, wj = (wave & 1) * 64;
    v4f acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = v4f{0, 0, 0, 0};
    copy(0);
    for (int s = 0; s < total; ++s) {
        wait_vmem<0>();
        lds_barrier();
        const uint8_t *buf = lds + (s & 1) * kBuf;
        if (s + 1 < total) copy(s + 1);
        if (SPLIT && s == 2 * g.kblocks) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] *= 1.0f / (1 << kLowBits);
        }
        v8i fa[4], fb[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fa[i] = read_fragment(buf, wi + 16 * i, lane);
            fb[i] = read_fragment(buf + T * kStageRowBytes, wj + 16 * i, lane);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    typedef int v4i_ __attribute__((ext_vector_type(4)));
                    const v4i_ x = h ? fa[i].hi : fa[i].lo, y = h ? fb[j].hi : fb[j].lo;
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8f16, x),
                                                                       __builtin_bit_cast(v8f16, y), acc[i][j], 0, 0, 0);
                }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = i0 + wi + 16 * i + 4 * (lane >> 4) + e, col = j0 + wj + 16 * j + (lane & 15);
                // a diagonal tile computes each pair twice, not to the same bits:
                // its lower half counts
                if (SYM && row < col) continue;
                float v = g.mul * acc[i][j][e];
                if (KIND != kGram) v = fmaf(g.add, held<SPLIT>(g.e, b * g.e.batch + row * g.e.pitch + col), v);
                if (KIND == kLast) {
                    if (row < g.r && col < g.c)
                        store_any(g.O, b * g.o_batch + row * g.o_row + col * g.o_col, g.type, v * g.out_scale);
                } else {
                    hold<SPLIT>(g.d, b * g.d.batch + row * g.d.pitch + col, v);
                    if (SYM) hold<SPLIT>(g.d, b * g.d.batch + col * g.d.pitch + row, v);
                    else hold<SPLIT>(g.dt, b * g.dt.batch + col * g.dt.pitch + row, v);
                }
            }
}

// No steps: X itself.
template <bool SPLIT>
__global__ __launch_bounds__(256) void write_x(Planes x, ProductArgs g) {
    const int64_t total = (int64_t)g.r * g.c;
    for (int64_t t = blockIdx.x * 256LL + threadIdx.x; t < total; t += gridDim.x * 256LL) {
        const int64_t i = t / g.c, j = t % g.c, b = blockIdx.y;
        store_any(g.O, b * g.o_batch + i * g.o_row + j * g.o_col, g.type,
                  held<SPLIT>(x, b * x.batch + i * x.pitch + j) * g.out_scale);
    }
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

struct Buffers {
    double *parts;
    Planes x, t[2], a, b;
};

// One part per held matrix for bf16, two otherwise.
bool split_of(int type) { return type != O2M_TYPE_BF16; }

size_t carve(int batch, int r, int c, bool split, void *base, Buffers *out) {
    const int64_t rp = round_up64(r, kPad), cp = round_up64(c, kPad);
    char *at = static_cast<char *>(base);
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char *p = at ? at + off : nullptr;
        off += align256(bytes);
        return p;
    };
    auto planes = [&](int64_t rows, int64_t cols) {
        Planes m;
        m.pitch = cols;
        m.batch = rows * cols;
        const size_t bytes = sizeof(f16) * (size_t)m.batch * batch;
        m.hi = reinterpret_cast<f16 *>(take(bytes));
        m.lo = split ? reinterpret_cast<f16 *>(take(bytes)) : nullptr;
        return m;
    };
    Buffers b;
    b.parts = reinterpret_cast<double *>(take(sizeof(double) * kParts * (size_t)batch));
    b.x = planes(rp, cp);
    b.t[0] = planes(cp, rp);
    b.t[1] = planes(cp, rp);
    b.a = planes(rp, rp);
    b.b = planes(rp, rp);
    if (out) *out = b;
    return off;
}

template <bool SPLIT, Product KIND>
void launch_product(ProductArgs &g, int batch, hipStream_t st) {
    g.tiles = KIND == kGram || KIND == kPoly ? g.mt * (g.mt + 1) / 2 : g.mt * g.nt;
    product_tile<SPLIT, KIND><<<(unsigned)(g.tiles * batch), 256, 0, st>>>(g);
}

template <bool SPLIT>
hipError_t run_ortho(const OrthoArgs &o, const Buffers &b, hipStream_t st) {
    const int r = o.rows, c = o.cols;
    const int rt = (int)ceil_div(r, kPad), ct = (int)ceil_div(c, kPad);
    const int s = (int)lrint(0.5 * log2((double)c));
    const bool along_c = o.g_col == 1;
    norm_parts<<<dim3(kParts, o.batch), 256, 0, st>>>(
        {o.G, along_c ? o.g_row : o.g_col, o.g_batch, along_c ? r : c, along_c ? c : r, o.type, b.parts});
    PrepArgs p = {o.G, o.g_row, o.g_col, o.g_batch, r, c, o.type, b.parts, o.eps, ldexp(1.0, s), b.x, b.t[0], ct * 2};
    prepare_x<SPLIT><<<dim3(rt * 2 * ct * 2, o.batch), 256, 0, st>>>(p);
    ProductArgs g = {};
    g.O = o.O;
    g.o_row = o.o_row;
    g.o_col = o.o_col;
    g.o_batch = o.o_batch;
    g.r = r;
    g.c = c;
    g.type = o.type;
    g.out_scale = (float)ldexp(1.0, -s);
    if (o.steps == 0) {
        write_x<SPLIT><<<dim3(std::min<int64_t>(1024, ceil_div((int64_t)r * c, 256)), o.batch), 256, 0, st>>>(b.x, g);
        return hipGetLastError();
    }
    for (int step = 0; step < o.steps; ++step) {
        const double *k = o.coef + 3 * step;
        const Planes &t = b.t[step & 1], &t_next = b.t[(step + 1) & 1];
        g.p = g.q = b.x;
        g.d = b.a;
        g.kblocks = ct * 2;
        g.mt = g.nt = rt;
        g.mul = (float)ldexp(1.0, kScaleA - 2 * s);
        launch_product<SPLIT, kGram>(g, o.batch, st);
        g.p = g.q = g.e = b.a;
        g.d = b.b;
        g.kblocks = rt * 2;
        g.add = (float)ldexp(k[1], kScaleB - kScaleA);
        g.mul = (float)ldexp(k[2], kScaleB - 2 * kScaleA);
        launch_product<SPLIT, kPoly>(g, o.batch, st);
        g.p = b.b;
        g.q = t;
        g.e = g.d = b.x;
        g.dt = t_next;
        g.nt = ct;
        g.add = (float)k[0];
        g.mul = (float)ldexp(1.0, -kScaleB);
        if (step + 1 < o.steps) launch_product<SPLIT, kUpdate>(g, o.batch, st);
        else launch_product<SPLIT, kLast>(g, o.batch, st);
    }
    return hipGetLastError();
}

}  // namespace

size_t ortho_workspace(int batch, int rows, int cols, int type) {
    return carve(batch, rows, cols, split_of(type), nullptr, nullptr);
}

hipError_t launch_ortho(const OrthoArgs &o, void *ws, hipStream_t st) {
    Buffers b;
    const bool split = split_of(o.type);
    carve(o.batch, o.rows, o.cols, split, ws, &b);
    return split ? run_ortho<true>(o, b, st) : run_ortho<false>(o, b, st);
}

}  // namespace o2m
