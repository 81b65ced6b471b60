// The orthogonalised update (include/o2m.h: o2m_orthogonalize):
//
//   X = G / (||G|| + eps);  steps x:  A = X X^T, B = b A + c A^2, X <- a X + B X
//
// on the work matrix X (r x c, r <= c, G transposed where it is tall).  Three
// products per step: A and A^2 symmetric, so half their tiles are computed and
// mirrored, then B X with a X added as it is stored.
//
// Held numbers.  |X| <= s_max in every entry, A <= s_max^2, and of the size of 1 /
// sqrt(c) in the end: matrices are held in fp16, as X 2^14, A 2^11 and B 2^6, which
// leaves room for singular values up to 4 and keeps fp16's smallest numbers
// 2^-24 far below what counts.  For bf16 updates one fp16 part is kept, whose 11
// bits put the held matrices' roundings below the result's own; fp32 and fp16
// updates keep the rest in a second fp16 part, and multiply lo hi + hi lo + hi
// hi, all summed in fp32.  What is left out, lo lo, is 2^-24 of the product.
//
// Layout.  All held matrices are padded with zeros to multiples of 128, so no
// product has a ragged edge.  X is kept both as it is (the rows that A
// multiplies) and transposed (the rows that B X multiplies); the product that
// makes it writes both.
//
// Products with enough 256 x 256 tiles to go round take the pipeline of
// mfma_pipe.h and write from it; the others take tiles of 128 x 128, split along
// k until they fill the part, whose fp32 sums a second kernel adds up and writes.
//
// Bound: fp16 MFMA; 3 r^2 c + r^3 multiply-adds a step, halves counted once, and
// three times that for two parts.
#include "mfma_pipe.h"
#include "mfma_tiles.h"
#include "model_internal.h"
#include "tile_schedule.h"

#include <algorithm>
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <math.h>

namespace o2m {
namespace {

typedef _Float16 f16;
typedef f16 v8f16 __attribute__((ext_vector_type(8)));
typedef __bf16 v8bf16 __attribute__((ext_vector_type(8)));

constexpr int kPad = 128;
constexpr int kScaleX = 14, kScaleA = 11, kScaleB = 6;
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

// An entry held in one or two parts, and 8 neighbouring ones.
template <bool SPLIT>
__device__ inline float held(const Planes &m, int64_t i) {
    return SPLIT ? (float)m.hi[i] + (float)m.lo[i] : (float)m.hi[i];
}
template <bool SPLIT>
__device__ inline void hold(const Planes &m, int64_t i, float v) {
    const f16 hi = (f16)v;
    m.hi[i] = hi;
    if (SPLIT) m.lo[i] = (f16)(v - (float)hi);
}
template <bool SPLIT>
__device__ inline v8f held8(const Planes &m, int64_t i) {
    v8f v = __builtin_convertvector(*reinterpret_cast<const v8f16 *>(m.hi + i), v8f);
    if (SPLIT) v += __builtin_convertvector(*reinterpret_cast<const v8f16 *>(m.lo + i), v8f);
    return v;
}
template <bool SPLIT>
__device__ inline void hold8(const Planes &m, int64_t i, const v8f &v) {
    const v8f16 hi = __builtin_convertvector(v, v8f16);
    *reinterpret_cast<v8f16 *>(m.hi + i) = hi;
    if (SPLIT)
        *reinterpret_cast<v8f16 *>(m.lo + i) = __builtin_convertvector(v - __builtin_convertvector(hi, v8f), v8f16);
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
constexpr bool symmetric(Product k) { return k == kGram || k == kPoly; }

// D = add E + mul P Q^T, of rows x cols entries (padded).
struct ProductArgs {
    Planes p, q;
    Planes e, et;       // kPoly: A twice; kUpdate, kLast: X and its transpose
    Planes d, dt;       // D and its transpose (kGram, kPoly: the same matrix)
    int rows, cols;
    int kblocks;        // stages of 64
    int mt, nt, tiles;  // tiles of the launch's size; per matrix
    int batch, chunk;   // chunk: tiles of the whole launch per XCD
    float add, mul;
    float *parts;       // split launches: sums [split][batch][rows][cols]
    int splits, per;    // stages of a split
    void *O;            // kLast: where the r x c result goes
    int64_t o_row, o_col, o_batch;
    int r, c, type;
    float out_scale;
};

// Tile t of a symmetric product: those at and below the diagonal, row after row.
__device__ inline void triangle_tile(int t, int &ti, int &tj) {
    ti = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
    while (ti * (ti + 1) / 2 > t) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
    tj = t - ti * (ti + 1) / 2;
}

// Matrix and tile of slot t of a launch; tiles of one matrix in groups of 8
// tile-rows (tile_schedule.h), or a triangle.
template <Product KIND>
__device__ inline bool tile_at(const ProductArgs &g, int64_t t, int &b, int &ti, int &tj) {
    b = (int)(t / g.tiles);
    if (b >= g.batch) return false;
    const int in = (int)(t % g.tiles);
    if (symmetric(KIND)) {
        triangle_tile(in, ti, tj);
        return true;
    }
    const TileCoord c = tile_of(0, in, g.mt, g.nt, g.tiles, 0);
    ti = c.ti;
    tj = c.tj;
    return true;
}

// The stages of a product: kblocks of hi hi, before them, with two parts, those
// of lo hi and hi lo.
template <bool SPLIT>
struct HalfSrc {
    __amdgpu_buffer_rsrc_t p_hi, p_lo, q_hi, q_lo;
    int ld_a, ld_b, kblocks, total;
    __device__ inline HalfSrc(const ProductArgs &g, int b, int i0, int j0, int tile) {
        kblocks = g.kblocks;
        total = SPLIT ? 3 * kblocks : kblocks;
        ld_a = (int)g.p.pitch * 2;
        ld_b = (int)g.q.pitch * 2;
        auto rows = [&](const f16 *m, const Planes &of, int row0, int all, int ld) {
            return rows_of(reinterpret_cast<const uint8_t *>(m + b * of.batch + row0 * of.pitch), min(tile, all - row0), ld,
                           kblocks * kStageRowBytes);
        };
        p_hi = rows(g.p.hi, g.p, i0, g.rows, ld_a);
        q_hi = rows(g.q.hi, g.q, j0, g.cols, ld_b);
        if (SPLIT) {
            p_lo = rows(g.p.lo, g.p, i0, g.rows, ld_a);
            q_lo = rows(g.q.lo, g.q, j0, g.cols, ld_b);
        }
    }
    __device__ inline __amdgpu_buffer_rsrc_t a(int s) const { return SPLIT && s < kblocks ? p_lo : p_hi; }
    __device__ inline __amdgpu_buffer_rsrc_t b(int s) const {
        return SPLIT && s >= kblocks && s < 2 * kblocks ? q_lo : q_hi;
    }
    __device__ inline int k(int s) const { return !SPLIT || s < kblocks ? s : s < 2 * kblocks ? s - kblocks : s - 2 * kblocks; }
    __device__ inline int left(int s) const { return s < total ? kStageRowBytes : 0; }
};

// Two fp16 MFMAs of 32 per stage of 64.  (In assembly, as the 8-bit ones, to keep
// the accumulators in place.)
struct HalfOp {
    static constexpr int kParts = 2;
    __device__ inline void fetch(int) {}
    __device__ inline void begin(int) {}
    __device__ inline void mask(v8i &, int) {}
    template <int I, int J, int P>
    __device__ __forceinline__ void mma(v4f &d, const v8i &x, const v8i &y) {
        if constexpr (P == 0) mfma(d, x.lo, y.lo);
        else mfma(d, x.hi, y.hi);
    }
    __device__ static inline void mfma(v4f &d, const v4i &x, const v4i &y) {
        asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(d) : "v"(x), "v"(y) : "memory");
    }
};

// The first n of eight values.
template <class T, class V>
__device__ inline void store_some(T *p, const V &v, int n) {
    if (n >= 8 && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
        *reinterpret_cast<V *>(p) = v;
    } else {
        each<8>([&](auto J) {
            if (J < n) p[J] = v[(int)J];
        });
    }
}

// Eight outputs of row `row`, columns col .. col + 7 (T: of column `col`, rows row ..
// row + 7), given the sums.
template <bool SPLIT, Product KIND, bool T>
__device__ inline void emit(const ProductArgs &g, int b, int row, int col, v8f v) {
    const int first = T ? row : col, line = T ? col : row;
    if (row >= g.rows || col >= g.cols) return;
    v *= g.mul;
    if (KIND != kGram) {
        const Planes &e = T ? g.et : g.e;
        v += g.add * held8<SPLIT>(e, b * e.batch + line * e.pitch + first);
    }
    if (KIND != kLast) {
        const Planes &d = T ? g.dt : g.d;
        hold8<SPLIT>(d, b * d.batch + line * d.pitch + first, v);
        return;
    }
    const int lines = T ? g.c : g.r, n = min(8, (T ? g.r : g.c) - first);
    if (line >= lines) return;
    const int64_t at = b * g.o_batch + row * g.o_row + col * g.o_col;
    v *= g.out_scale;
    if (g.type == O2M_TYPE_F32) store_some(static_cast<float *>(g.O) + at, v, n);
    else if (g.type == O2M_TYPE_F16) store_some(static_cast<f16 *>(g.O) + at, __builtin_convertvector(v, v8f16), n);
    else store_some(static_cast<__bf16 *>(g.O) + at, __builtin_convertvector(v, v8bf16), n);
}

template <bool SPLIT, Product KIND>
__global__ __launch_bounds__(256, 1) void product_pipe(ProductArgs g) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kPipeLds];
    const PipeWave w = pipe_wave(lds);
    int b, ti, tj;
    if (!tile_at<KIND>(g, (int64_t)(blockIdx.x & 7) * g.chunk + (blockIdx.x >> 3), b, ti, tj)) return;
    const int i0 = ti * kPipeTile, j0 = tj * kPipeTile;
    const HalfSrc<SPLIT> src(g, b, i0, j0, kPipeTile);
    HalfOp op;
    v4f acc[8][8];
    pipe_run(w, op, src, src.total, acc);
    // a diagonal tile holds both halves already, an off-diagonal one is mirrored
    const bool rows = KIND != kLast || g.o_col == 1;
    const bool across = symmetric(KIND) ? ti != tj : KIND != kLast || !rows;
    if (rows)
        pipe_results<false>(w, acc, [&](int row, int col, const v8f &v) { emit<SPLIT, KIND, false>(g, b, i0 + row, j0 + col, v); });
    if (across)
        pipe_results<true>(w, acc, [&](int row, int col, const v8f &v) { emit<SPLIT, KIND, true>(g, b, i0 + row, j0 + col, v); });
}

// fp32 sums of a part of the stages on 128 x 128, by 2 x 2 waves of 4 x 4 blocks;
// two stage buffers, two workgroups per CU.  Columns of a wave are 4 q + j (block
// j, q = lane % 16), so that a lane's 4 blocks are 4 neighbouring columns.
template <bool SPLIT, Product KIND>
__global__ __launch_bounds__(256, 2) void product_parts(ProductArgs g) {
    constexpr int T = kPad, kBuf = 2 * T * kStageRowBytes;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kBuf];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int z = blockIdx.x % g.splits;
    int b, ti, tj;
    if (!tile_at<KIND>(g, blockIdx.x / g.splits, b, ti, tj)) return;
    const int i0 = ti * T, j0 = tj * T;
    const HalfSrc<SPLIT> src(g, b, i0, j0, T);
    const int s0 = z * g.per, s1 = min(src.total, s0 + g.per);
    auto copy = [&](int s) {
        uint8_t *buf = lds + (s & 1) * kBuf;
        const auto rp = src.a(s), rq = src.b(s);
        const int kb = src.k(s);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            copy_rows<0>(rp, buf + (wave * 4 + q) * 1024, lane, wave * 4 + q, src.ld_a, kb, kStageRowBytes);
            copy_rows<2>(rq, buf + T * kStageRowBytes + (wave * 4 + q) * 1024, lane, wave * 4 + q, src.ld_b, kb,
                         kStageRowBytes);
        }
    };
    const int wi = (wave >> 1) * 64, wj = (wave & 1) * 64, q = lane & 15;
    v4f acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = v4f{0, 0, 0, 0};
    if (s0 < s1) copy(s0);
    for (int s = s0; s < s1; ++s) {
        wait_vmem<0>();
        lds_barrier();
        const uint8_t *buf = lds + (s & 1) * kBuf;
        if (s + 1 < s1) copy(s + 1);
        v8i fa[4], fb[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fa[i] = read_fragment<0>(buf, wi + 16 * i + q, lane);
            fb[i] = read_fragment<2>(buf + T * kStageRowBytes, wj + 4 * q + i, lane);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const v4i x = h ? fa[i].hi : fa[i].lo, y = h ? fb[j].hi : fb[j].lo;
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8f16, x),
                                                                       __builtin_bit_cast(v8f16, y), acc[i][j], 0, 0, 0);
                }
    }
    float *out = g.parts + ((int64_t)z * g.batch + b) * g.rows * g.cols;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = i0 + wi + 16 * i + 4 * (lane >> 4) + e, col = j0 + wj + 4 * q;
            *reinterpret_cast<v4f *>(out + (int64_t)row * g.cols + col) = v4f{acc[i][0][e], acc[i][1][e], acc[i][2][e], acc[i][3][e]};
        }
}

// Adds up the splits in their order and writes D and its transpose, 64 x 64 per
// workgroup, a quarter of a tile of product_parts.
template <bool SPLIT, Product KIND>
__global__ __launch_bounds__(256) void product_join(ProductArgs g) {
    __shared__ float tile[64][65];
    const int tid = threadIdx.x, quarter = blockIdx.x & 3;
    int b, ti, tj;
    if (!tile_at<KIND>(g, blockIdx.x >> 2, b, ti, tj)) return;
    const int i0 = ti * kPad + (quarter >> 1) * 64, j0 = tj * kPad + (quarter & 1) * 64;
    const bool rows = KIND != kLast || g.o_col == 1;
    const bool across = symmetric(KIND) ? ti != tj : KIND != kLast || !rows;
    const int64_t plane = (int64_t)g.rows * g.cols;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = 32 * h + (tid >> 3), col = (tid & 7) * 8;
        const float *at = g.parts + b * plane + (int64_t)(i0 + row) * g.cols + j0 + col;
        v4f lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
        for (int z = 0; z < g.splits; ++z) {
            lo += *reinterpret_cast<const v4f *>(at + z * g.batch * plane);
            hi += *reinterpret_cast<const v4f *>(at + z * g.batch * plane + 4);
        }
        const v8f v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        if (rows) emit<SPLIT, KIND, false>(g, b, i0 + row, j0 + col, v);
        if (across)
#pragma unroll
            for (int j = 0; j < 8; ++j) tile[row][col + j] = v[j];
    }
    if (!across) return;   // uniform over the workgroup
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int col = 32 * h + (tid >> 3), row = (tid & 7) * 8;
        v8f v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = tile[row + i][col];
        emit<SPLIT, KIND, true>(g, b, i0 + row, j0 + col, v);
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
    float *sums;
};

// How a product of rows x cols (padded) and `stages` stages is launched.
struct ProductPlan {
    bool pipe;
    int mt, nt, tiles;   // per matrix
    int splits, per;
};
// 256 x 256 tiles from half a tile per CU on: they take twice as long as four of 128
// x 128 on a CU of their own, but feed the MFMA pipe 1.5 times as well.  Smaller
// tiles are split until two for each CU are in flight, from 4 stages each.
ProductPlan plan_product(int batch, int rows, int cols, int stages, bool sym) {
    auto count = [&](int q, int &mt, int &nt) {
        mt = (int)ceil_div(rows, q);
        nt = (int)ceil_div(cols, q);
        return sym ? mt * (mt + 1) / 2 : mt * nt;
    };
    ProductPlan p;
    p.tiles = count(kPipeTile, p.mt, p.nt);
    p.pipe = (int64_t)p.tiles * batch >= kCus / 2;
    p.splits = 1;
    p.per = stages;
    if (p.pipe) return p;
    p.tiles = count(kPad, p.mt, p.nt);
    const int64_t want = std::min<int64_t>(ceil_div(2 * kCus, (int64_t)p.tiles * batch), std::max(1, stages / 4));
    p.per = (int)ceil_div(stages, want);
    p.splits = (int)ceil_div(stages, p.per);
    return p;
}

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
    // fp32 sums of the split products: those of X (r x c) and of A and B
    int64_t sums = 0;
    const int passes = split ? 3 : 1;
    auto room = [&](int64_t rows, int64_t cols, int64_t k, bool sym) {
        const ProductPlan p = plan_product(batch, (int)rows, (int)cols, passes * (int)(k / 64), sym);
        if (!p.pipe) sums = std::max(sums, p.splits * rows * cols);
    };
    room(rp, rp, cp, true);
    room(rp, rp, rp, true);
    room(rp, cp, rp, false);
    b.sums = reinterpret_cast<float *>(take(sizeof(float) * (size_t)sums * batch));
    if (out) *out = b;
    return off;
}

template <bool SPLIT, Product KIND>
void launch_product(ProductArgs &g, int batch, hipStream_t st) {
    const int stages = (SPLIT ? 3 : 1) * g.kblocks;
    const ProductPlan p = plan_product(batch, g.rows, g.cols, stages, symmetric(KIND));
    g.mt = p.mt;
    g.nt = p.nt;
    g.tiles = p.tiles;
    g.batch = batch;
    g.splits = p.splits;
    g.per = p.per;
    const int64_t all = (int64_t)p.tiles * batch;
    if (p.pipe) {
        g.chunk = (int)ceil_div(all, kXcds);
        product_pipe<SPLIT, KIND><<<(unsigned)(kXcds * g.chunk), 256, 0, st>>>(g);
    } else {
        product_parts<SPLIT, KIND><<<(unsigned)(all * p.splits), 256, 0, st>>>(g);
        product_join<SPLIT, KIND><<<(unsigned)(all * 4), 256, 0, st>>>(g);
    }
}

template <bool SPLIT>
hipError_t run_ortho(const OrthoArgs &o, const Buffers &b, hipStream_t st) {
    const int r = o.rows, c = o.cols;
    const int rt = (int)ceil_div(r, kPad), ct = (int)ceil_div(c, kPad);
    const bool along_c = o.g_col == 1;
    norm_parts<<<dim3(kParts, o.batch), 256, 0, st>>>(
        {o.G, along_c ? o.g_row : o.g_col, o.g_batch, along_c ? r : c, along_c ? c : r, o.type, b.parts});
    PrepArgs p = {o.G, o.g_row, o.g_col, o.g_batch, r, c, o.type, b.parts, o.eps, ldexp(1.0, kScaleX), b.x, b.t[0], ct * 2};
    prepare_x<SPLIT><<<dim3(rt * 2 * ct * 2, o.batch), 256, 0, st>>>(p);
    ProductArgs g = {};
    g.O = o.O;
    g.o_row = o.o_row;
    g.o_col = o.o_col;
    g.o_batch = o.o_batch;
    g.r = r;
    g.c = c;
    g.type = o.type;
    g.out_scale = (float)ldexp(1.0, -kScaleX);
    if (o.steps == 0) {
        write_x<SPLIT><<<dim3(std::min<int64_t>(1024, ceil_div((int64_t)r * c, 256)), o.batch), 256, 0, st>>>(b.x, g);
        return hipGetLastError();
    }
    const int rp = rt * kPad, cp = ct * kPad;
    g.parts = b.sums;
    for (int step = 0; step < o.steps; ++step) {
        const double *k = o.coef + 3 * step;
        const Planes &t = b.t[step & 1], &t_next = b.t[(step + 1) & 1];
        g.rows = g.cols = rp;
        g.p = g.q = b.x;
        g.d = g.dt = b.a;
        g.kblocks = cp / 64;
        g.mul = (float)ldexp(1.0, kScaleA - 2 * kScaleX);
        launch_product<SPLIT, kGram>(g, o.batch, st);
        g.p = g.q = g.e = g.et = b.a;
        g.d = g.dt = b.b;
        g.kblocks = rp / 64;
        g.add = (float)ldexp(k[1], kScaleB - kScaleA);
        g.mul = (float)ldexp(k[2], kScaleB - 2 * kScaleA);
        launch_product<SPLIT, kPoly>(g, o.batch, st);
        g.p = b.b;
        g.q = g.et = t;
        g.e = g.d = b.x;
        g.dt = t_next;
        g.cols = cp;
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
