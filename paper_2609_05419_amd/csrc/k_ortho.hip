// The orthogonalised update (include/o2m.h: o2m_orthogonalize):
//
//   X = G / (||G|| + eps);  steps x:  A = X X^T, B = a I + b A + c A^2, X <- B X
//
// on the work matrix X (r x c, r <= c, G transposed where it is tall).  Three
// products per step: A and A^2 symmetric, so half their tiles are computed and
// mirrored, then B X.  (With a in B rather than a X added to the last product, that
// one reads nothing but its operands, and B's rounding, relative to a + b s^2 + c
// s^4 rather than to b s^2 + c s^4, is if anything the smaller one.)
//
// Held numbers.  |X| <= s_max in every entry, A <= s_max^2, and X of the size of 1 /
// sqrt(c) in the end: matrices are held in fp16, as X 2^14, A 2^11 and B 2^6, which
// leaves room for singular values up to 4 (and B up to 1000) and keeps fp16's
// smallest numbers 2^-24 far below what counts.  For bf16 updates one fp16 part is kept, whose 11
// bits put the held matrices' roundings below the result's own; fp32 and fp16
// updates keep the rest in a second fp16 part, and multiply lo hi + hi lo + hi
// hi, all summed in fp32.  What is left out, lo lo, is 2^-24 of the product.
//
// Layout.  All held matrices are padded with zeros to multiples of 64, so no
// product has a ragged edge within a stage.  X is kept both as it is (the rows that A
// multiplies) and transposed (the rows that B X multiplies); the product that
// makes it writes both.
//
// Products take the pipeline of mfma_pipe.h or smaller tiles (plan_product); those
// with too few tiles are split along k, and a second kernel adds the fp32 sums
// up and writes.
//
// Bound: fp16 MFMA; 1.5 r^2 c + 0.5 r^3 multiply-adds a step, halves counted once, and
// three times that for two parts.
#include "ortho_shared.h"
#include "tile_schedule.h"

#include <algorithm>
#include <math.h>

namespace o2m {
namespace {

constexpr int kPad = 64;
constexpr int kParts = 1024;   // partial sums of the norm, at most, per matrix

struct Planes {
    f16 *hi;
    int64_t lo;       // the second part, elements after the first; 0 when one is kept
    int64_t pitch;    // elements of a row
    int64_t batch;    // from matrix to matrix, both parts
};

// An entry held in one or two parts.
template <bool SPLIT>
__device__ inline float held(const Planes &m, int64_t i) {
    return SPLIT ? (float)m.hi[i] + (float)m.hi[i + m.lo] : (float)m.hi[i];
}
// N neighbouring entries.
template <bool SPLIT, int N, class V>
__device__ inline V held_run(const Planes &m, int64_t i) {
    typedef f16 vf16 __attribute__((ext_vector_type(N)));
    V v = __builtin_convertvector(*reinterpret_cast<const vf16 *>(m.hi + i), V);
    if (SPLIT) v += __builtin_convertvector(*reinterpret_cast<const vf16 *>(m.hi + m.lo + i), V);
    return v;
}
template <bool SPLIT, int N, class V>
__device__ inline void hold_run(const Planes &m, int64_t i, const V &v) {
    typedef f16 vf16 __attribute__((ext_vector_type(N)));
    const vf16 hi = __builtin_convertvector(v, vf16);
    *reinterpret_cast<vf16 *>(m.hi + i) = hi;
    if (SPLIT) *reinterpret_cast<vf16 *>(m.hi + m.lo + i) = __builtin_convertvector(v - __builtin_convertvector(hi, V), vf16);
}
// Sums of squares in fp64: part z adds up the runs of 8 entries z, z + parts, ..,
// its threads in a fixed order, so that every run of the call adds in the same one.
__global__ __launch_bounds__(256) void norm_parts(Lines g, int parts, double *out) {
    __shared__ double sums[256];
    const unsigned per_line = (unsigned)(g.len + 7) / 8;
    const int64_t runs = (int64_t)per_line * g.lines, base = blockIdx.y * g.batch;
    double s = 0.0;
    for (int64_t t = blockIdx.x * 256LL + threadIdx.x; t < runs; t += parts * 256LL) {
        // (the quotient of a line's runs: 32 bits where they suffice)
        const int64_t p = runs <= 0xFFFFFFFFLL ? (int64_t)((unsigned)t / per_line) : t / per_line;
        const int q = (int)(t - p * per_line) * 8;
        const v8f v = load_some(g.G, base + p * g.line + q, g.len - q, g.type);
#pragma unroll
        for (int j = 0; j < 8; ++j) s += (double)v[j] * (double)v[j];
    }
    sums[threadIdx.x] = s;
    __syncthreads();
    for (int w = 128; w > 0; w >>= 1) {
        if (threadIdx.x < w) sums[threadIdx.x] += sums[threadIdx.x + w];
        __syncthreads();
    }
    if (threadIdx.x == 0) out[(int64_t)blockIdx.y * kParts + blockIdx.x] = sums[0];
}

// scale / (norm + eps) from the parts, for the whole workgroup; NaN when the norm is
// not finite.
__device__ inline double inverse_norm(const double *parts, int count, double eps, double scale, double *sums) {
    const int tid = threadIdx.x;
    double s = 0.0;
    for (int i = tid; i < count; i += 256) s += parts[i];
    sums[tid] = s;
    __syncthreads();
    for (int w = 128; w > 0; w >>= 1) {
        if (tid < w) sums[tid] += sums[tid + w];
        __syncthreads();
    }
    const double norm = sqrt(sums[0]);
    return norm <= 1.7e308 ? scale / (norm + eps) : (double)NAN;
}

struct PrepArgs {
    Lines g;
    const double *parts;
    int count;
    double eps, scale;   // scale: 2^kScaleX
    Planes along, across;   // the lines of G, and their transpose, padded
    int tiles_q;
};
// G / (norm + eps) held, and its transpose, 64 x 64 entries per workgroup.
template <bool SPLIT>
__global__ __launch_bounds__(256) void prepare_x(PrepArgs g) {
    __shared__ float tile[64][65];
    __shared__ double sums[256];
    const int tid = threadIdx.x, b = blockIdx.y;
    const double inv = inverse_norm(g.parts + (int64_t)b * kParts, g.count, g.eps, g.scale, sums);
    const int p0 = blockIdx.x / g.tiles_q * 64, q0 = blockIdx.x % g.tiles_q * 64;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int p = 32 * h + (tid >> 3), q = (tid & 7) * 8;
        const int n = p0 + p < g.g.lines ? min(8, g.g.len - q0 - q) : 0;
        v8f v = load_some(g.g.G, b * g.g.batch + (p0 + p) * g.g.line + q0 + q, n, g.g.type);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = j < n ? (float)((double)v[j] * inv) : 0.0f;   // (padding stays zero under a NaN)
            tile[p][q + j] = v[j];
        }
        hold_run<SPLIT, 8>(g.along, b * g.along.batch + (p0 + p) * g.along.pitch + q0 + q, v);
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int q = 32 * h + (tid >> 3), p = (tid & 7) * 8;
        v8f v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = tile[p + i][q];
        hold_run<SPLIT, 8>(g.across, b * g.across.batch + (q0 + q) * g.across.pitch + p0 + p, v);
    }
}

enum Product { kGram, kPoly, kUpdate, kLast };
constexpr bool symmetric(Product k) { return k == kGram || k == kPoly; }

// D = diag I + add E + mul P Q^T (kPoly; the others: mul P Q^T), of rows x cols
// entries (padded).
struct ProductArgs {
    Planes p, q;
    Planes e;           // kPoly: A
    Planes d, dt;       // D and its transpose (kGram, kPoly: the same matrix)
    int rows, cols;
    int kblocks;        // stages of 64
    int mt, nt, tiles;  // tiles of the launch's size; per matrix
    int tm, tn;         // that size
    int batch;
    float diag, add, mul;
    // Workgroups: one for each of the first `whole` tiles, then `splits` for each of the
    // `rest`, `per` stages each, whose sums go to parts [rest][splits][tm][tn].
    int64_t whole, rest;
    int whole_chunk, rest_chunk;   // workgroups of each kind per XCD
    int splits, per;
    float *parts;
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

// Matrix and place of tile t of a launch; tiles of one matrix in groups of 8
// tile-rows (tile_schedule.h), or a triangle.
template <Product KIND>
__device__ inline void tile_at(const ProductArgs &g, int64_t t, int &b, int &ti, int &tj) {
    b = (int)(t / g.tiles);
    const int in = (int)(t % g.tiles);
    if (symmetric(KIND)) {
        triangle_tile(in, ti, tj);
        return;
    }
    const TileCoord c = tile_of(0, in, g.mt, g.nt, g.tiles, 0);
    ti = c.ti;
    tj = c.tj;
}

// What a workgroup computes.  An XCD has neighbouring tiles, and of split ones those of
// the same stages.
struct Share {
    int b, ti, tj;
    int first, total;   // stages
    float *part;        // where the sums go; null: the whole product
};
template <Product KIND>
__device__ inline bool share_of(const ProductArgs &g, int stages, Share &w) {
    const int xcd = blockIdx.x % kXcds, slot = blockIdx.x / kXcds;
    int64_t t;
    if (slot < g.whole_chunk) {
        t = (int64_t)xcd * g.whole_chunk + slot;
        if (t >= g.whole) return false;
        w.first = 0;
        w.total = stages;
        w.part = nullptr;
    } else {
        t = (int64_t)xcd * g.rest_chunk + slot - g.whole_chunk;
        if (t >= g.rest * g.splits) return false;
        const int64_t z = t / g.rest, u = t % g.rest;
        w.first = (int)z * g.per;
        w.total = min(g.per, stages - w.first);
        w.part = g.parts + (u * g.splits + z) * g.tm * g.tn;
        t = g.whole + u;
    }
    tile_at<KIND>(g, t, w.b, w.ti, w.tj);
    return true;
}

// The stages [first, first + total) of a product: kblocks of hi hi, before them,
// with two parts, those of lo hi and hi lo.
template <bool SPLIT>
struct HalfSrc {
    // one descriptor for both parts: the second lies a fixed distance on (so rows
    // past the last one read what follows, which only rows that are not written
    // see, and not zeros)
    __amdgpu_buffer_rsrc_t rp, rq;
    int ld_a, ld_b, lo_a, lo_b, kblocks, first, total;
    __device__ inline HalfSrc(const ProductArgs &g, const Share &w, int i0, int j0, int tile_m, int tile_n) {
        const int b = w.b;
        kblocks = g.kblocks;
        first = w.first;
        total = w.total;
        ld_a = (int)g.p.pitch * 2;
        ld_b = (int)g.q.pitch * 2;
        lo_a = (int)g.p.lo * 2;
        lo_b = (int)g.q.lo * 2;
        auto rows = [&](const Planes &of, int row0, int all, int tile, int ld, int lo) {
            // (2^31 at most, of 256 rows of 2^21 entries in two parts)
            const uint32_t extent = (uint32_t)lo + (uint32_t)((min(tile, all - row0) - 1) * ld) + kblocks * kStageRowBytes;
            return __builtin_amdgcn_make_buffer_rsrc(of.hi + b * of.batch + row0 * of.pitch, (short)0, (int)extent, 0x00020000);
        };
        rp = rows(g.p, i0, g.rows, tile_m, ld_a, SPLIT ? lo_a : 0);
        rq = rows(g.q, j0, g.cols, tile_n, ld_b, SPLIT ? lo_b : 0);
    }
    __device__ inline __amdgpu_buffer_rsrc_t a(int) const { return rp; }
    __device__ inline __amdgpu_buffer_rsrc_t b(int) const { return rq; }
    // byte offsets of stage s: passes lo hi, hi lo, hi hi
    __device__ inline int at_a(int s) const {
        const int at = first + s, pass = SPLIT ? (at >= kblocks) + (at >= 2 * kblocks) : 2;
        return (SPLIT ? at - pass * kblocks : at) * kStageRowBytes + (SPLIT && pass == 0 ? lo_a : 0);
    }
    __device__ inline int at_b(int s) const {
        const int at = first + s, pass = SPLIT ? (at >= kblocks) + (at >= 2 * kblocks) : 2;
        return (SPLIT ? at - pass * kblocks : at) * kStageRowBytes + (SPLIT && pass == 1 ? lo_b : 0);
    }
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

// The first n of N values of the result.
template <int N, class T, class V>
__device__ inline void store_some(T *p, const V &v, int n) {
    if (n >= N) {
        __builtin_memcpy(p, &v, sizeof(T) * N);
    } else {
        each<N>([&](auto J) {
            if (J < n) p[J] = v[(int)J];
        });
    }
}

// N outputs of row `row`, columns col .. (T: of column `col`, rows row ..), given the
// sums.
template <bool SPLIT, Product KIND, bool T, int N, class V>
__device__ inline void emit(const ProductArgs &g, int b, int row, int col, V v) {
    typedef f16 vf16 __attribute__((ext_vector_type(N)));
    typedef __bf16 vbf16 __attribute__((ext_vector_type(N)));
    const int first = T ? row : col, line = T ? col : row;
    if (row >= g.rows || col >= g.cols) return;
    v *= g.mul;
    if (KIND == kPoly) {
        v += g.add * held_run<SPLIT, N, V>(g.e, b * g.e.batch + line * g.e.pitch + first);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] += first + j == line ? g.diag : 0.0f;
    }
    if (KIND != kLast) {
        const Planes &d = T ? g.dt : g.d;
        hold_run<SPLIT, N, V>(d, b * d.batch + line * d.pitch + first, v);
        return;
    }
    const int n = min(N, (T ? g.r : g.c) - first);
    if (line >= (T ? g.c : g.r) || n <= 0) return;
    const int64_t at = b * g.o_batch + row * g.o_row + col * g.o_col;
    v *= g.out_scale;
    if (g.type == O2M_TYPE_F32) store_some<N>(static_cast<float *>(g.O) + at, v, n);
    else if (g.type == O2M_TYPE_F16) store_some<N>(static_cast<f16 *>(g.O) + at, __builtin_convertvector(v, vf16), n);
    else store_some<N>(static_cast<__bf16 *>(g.O) + at, __builtin_convertvector(v, vbf16), n);
}

// Which directions a product is written in.  A symmetric one: a tile on the
// diagonal holds both halves already, another is mirrored; X: both ways, the
// result in the one in which it is contiguous.
template <Product KIND>
__device__ inline bool writes_rows(const ProductArgs &g) { return KIND != kLast || g.o_col == 1; }
template <Product KIND>
__device__ inline bool writes_across(const ProductArgs &g, int ti, int tj) {
    return symmetric(KIND) ? ti != tj : KIND != kLast || g.o_col != 1;
}

template <bool SPLIT, Product KIND, int N>
__global__ __launch_bounds__(256, 1) void product_pipe(ProductArgs g) {
    static_assert(N == 8 || !symmetric(KIND), "triangles of squares");
    typedef PipeShape<N> T;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
    const PipeWave w = pipe_wave<N>(lds);
    Share of;
    if (!share_of<KIND>(g, (SPLIT ? 3 : 1) * g.kblocks, of)) return;   // whole workgroup
    const int b = of.b, i0 = of.ti * kPipeTile, j0 = of.tj * T::kTn;
    const HalfSrc<SPLIT> src(g, of, i0, j0, kPipeTile, T::kTn);
    HalfOp op;
    v4f acc[8][N];
    pipe_run<N>(w, op, src, src.total, acc);
    if (of.part) {
        pipe_results<false, N>(w, acc, [&](int row, int col, const auto &v) {
            __builtin_memcpy(of.part + row * T::kTn + col, &v, sizeof v);
        });
        return;
    }
    if (writes_rows<KIND>(g))
        pipe_results<false, N>(w, acc, [&](int row, int col, const auto &v) { emit<SPLIT, KIND, false, N>(g, b, i0 + row, j0 + col, v); });
    if (writes_across<KIND>(g, of.ti, of.tj))
        pipe_results<true, N>(w, acc, [&](int row, int col, const auto &v) { emit<SPLIT, KIND, true, 8>(g, b, i0 + row, j0 + col, v); });
}

// Smaller tiles: WR x WC waves of M x 4 blocks, a ring of S stage buffers with S - 1
// stages on their way.  Rows of a wave are 16 i + q (block i, q = lane % 16),
// columns 4 q + j: a lane holds 4 neighbouring columns (its blocks j) of 4
// neighbouring rows (an accumulator), so it writes 8 bytes in either direction.
template <bool SPLIT, Product KIND, int WR, int WC, int M, int S, int OCC>
__global__ __launch_bounds__(64 * WR * WC, OCC) void product_tile(ProductArgs g) {
    constexpr int kWaves = WR * WC, kTm = WR * M * 16, kTn = WC * 64, kBuf = (kTm + kTn) * kStageRowBytes;
    constexpr int kCopyA = kTm / 8 / kWaves, kCopyB = kTn / 8 / kWaves;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S * kBuf];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    Share of;
    if (!share_of<KIND>(g, (SPLIT ? 3 : 1) * g.kblocks, of)) return;   // whole workgroup
    const int b = of.b, i0 = of.ti * kTm, j0 = of.tj * kTn;
    const HalfSrc<SPLIT> src(g, of, i0, j0, kTm, kTn);
    auto copy = [&](int s, uint8_t *buf) {
        const int at_a = src.at_a(s), at_b = src.at_b(s);
#pragma unroll
        for (int c = 0; c < kCopyA; ++c) {
            const int q = wave * kCopyA + c;
            copy_rows<1>(src.rp, buf + q * 1024, lane, q, src.ld_a, at_a, kStageRowBytes);
        }
#pragma unroll
        for (int c = 0; c < kCopyB; ++c) {
            const int q = wave * kCopyB + c;
            copy_rows<2>(src.rq, buf + kTm * kStageRowBytes + q * 1024, lane, q, src.ld_b, at_b, kStageRowBytes);
        }
    };
    const int wi = wave / WC * (M * 16), wj = wave % WC * 64, q = lane & 15;
    v4f acc[M][4];
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < S - 1; ++u)
        if (u < src.total) copy(u, lds + u * kBuf);
    int u = 0;   // s % S
    for (int s = 0; s < src.total; ++s) {
        // this stage has landed; those after it, if there are S - 2, need not
        if (S > 2 && s + S - 1 <= src.total) wait_vmem<(S - 2) * (kCopyA + kCopyB)>();
        else wait_vmem<0>();
        lds_barrier();
        const uint8_t *buf = lds + u * kBuf;
        if (s + S - 1 < src.total) copy(s + S - 1, lds + (u == 0 ? S - 1 : u - 1) * kBuf);
        v8i fb[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) fb[j] = read_fragment<2>(buf + kTm * kStageRowBytes, wj + 4 * q + j, lane);
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const v8i fa = read_fragment<1>(buf, wi + 16 * i + q, lane);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const v4i x = h ? fa.hi : fa.lo, y = h ? fb[j].hi : fb[j].lo;
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8f16, x),
                                                                       __builtin_bit_cast(v8f16, y), acc[i][j], 0, 0, 0);
                }
        }
        u = u + 1 == S ? 0 : u + 1;
    }
    const bool rows = of.part || writes_rows<KIND>(g), across = !of.part && writes_across<KIND>(g, of.ti, of.tj);
#pragma unroll
    for (int i = 0; i < M; ++i) {
        const int row = i0 + wi + 16 * i + 4 * (lane >> 4), col = j0 + wj + 4 * q;
        if (rows)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const v4f v = {acc[i][0][e], acc[i][1][e], acc[i][2][e], acc[i][3][e]};
                if (of.part) *reinterpret_cast<v4f *>(of.part + (row + e - i0) * kTn + col - j0) = v;
                else emit<SPLIT, KIND, false, 4>(g, b, row + e, col, v);
            }
        if (across)
#pragma unroll
            for (int j = 0; j < 4; ++j) emit<SPLIT, KIND, true, 4>(g, b, row, col + j, acc[i][j]);
    }
}

// Adds up the splits in their order and writes D and its transpose, 32 x 64 of a tile
// per workgroup.
template <bool SPLIT, Product KIND>
__global__ __launch_bounds__(256) void product_join(ProductArgs g) {
    __shared__ float tile[32][65];
    const int tid = threadIdx.x, across_tile = g.tn / 64, per_tile = g.tm / 32 * across_tile;
    const int64_t u = blockIdx.x / per_tile;
    const int in = blockIdx.x % per_tile, di = in / across_tile * 32, dj = in % across_tile * 64;
    int b, ti, tj;
    tile_at<KIND>(g, g.whole + u, b, ti, tj);
    const int i0 = ti * g.tm + di, j0 = tj * g.tn + dj;
    if (i0 >= g.rows || j0 >= g.cols) return;   // whole workgroup
    const bool rows = writes_rows<KIND>(g), across = writes_across<KIND>(g, ti, tj);
    const int row = tid >> 3, col = (tid & 7) * 8, plane = g.tm * g.tn;
    const float *at = g.parts + u * g.splits * plane + (di + row) * g.tn + dj + col;
    v4f lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
#pragma unroll 4
    for (int z = 0; z < g.splits; ++z) {
        lo += *reinterpret_cast<const v4f *>(at + (int64_t)z * plane);
        hi += *reinterpret_cast<const v4f *>(at + (int64_t)z * plane + 4);
    }
    const v8f v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    if (rows) emit<SPLIT, KIND, false, 8>(g, b, i0 + row, j0 + col, v);
    if (!across) return;   // uniform over the workgroup
#pragma unroll
    for (int j = 0; j < 8; ++j) tile[row][col + j] = v[j];
    __syncthreads();
    const int down = (tid & 3) * 8;
    v8f t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = tile[down + i][tid >> 2];
    emit<SPLIT, KIND, true, 8>(g, b, i0 + down, j0 + (tid >> 2), t);
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
    int tm, tn;                   // tiles: 256 x 256, 256 x 128 (the pipeline), 128 x 128, 64 x 64
    int resident;                 // workgroups a CU holds (64 x 64: 2 with four stage buffers, 4 with two)
    int mt, nt, tiles;            // per matrix
    int64_t whole, rest;          // tiles with one workgroup, and split ones
    int splits, per;
};
// The tiles, and how many of them are split along k: all, or those of the last round
// that leaves CUs idle, or none, whichever has the least estimated time (us).  A size
// has `fixed`, then per stage `one` while a CU has one workgroup and `full` with all of
// `resident` (of one resident: while few CUs work, and when all do); then the
// writing, or the sums' way through memory and their joining.  Fitted to the best of
// 10 to 60 launches each of 54 products (64 x 64 tiles a, with two stage buffers and
// four workgroups a CU a', 128 x 128 b, 256 x 128 c, 256 x 256 d; /n: split in n, +/n:
// the last round's); what it takes is 0.5% slower than the best on average, 12% at
// most.  Measured (us):
//   r = c = 4096, one part, A    d 93, b 100, b/2 102, b+/8 77, b+/2 87
//                           X    d 108, b 123, c 126
//   r = c = 2048, one part, A    a' 20, b 25, a 27, b/2 24, a+/8 24;  two parts: b/3 45, d/6 54
//   8 of 768 x 768, one part, A  a' 11, a 13, b 13
//   r = c = 1024, one part, A    a 9, a' 12
//   1024 x 8192, two parts, A    b/12 47, b/8 56, d/12 65;  X: c 62, b 64, d 93
//   r = c = 1024, two parts, A   a/3 18, a'/6 16, b/4 18, a 29
//   320 x 896, two parts, A      a/4 11, a 22, b/4 16
// 16 splits are the most, a bound that no measurement set: an update of 128 x 131072
// bf16 takes 377 us, with A in 48 workgroups.
ProductPlan plan_product(int batch, int rows, int cols, int stages, bool sym) {
    struct Size {
        int tm, tn, resident;
        double fixed, one, full;
    };
    constexpr Size sizes[] = {{64, 64, 2, 3.7, 0.40, 0.48}, {64, 64, 4, 3.4, 0.48, 0.78}, {128, 128, 2, 4.1, 0.74, 0.95},
                              {256, 128, 1, 4.9, 0.93, 0.93}, {256, 256, 1, 10.2, 1.22, 1.65}};
    const double entries = (double)batch * rows * cols * (sym ? 0.5 : 1.0);
    ProductPlan best = {};
    double least = 0.0;
    for (const Size &s : sizes) {
        if (sym && s.tm != s.tn) continue;
        ProductPlan p;
        p.tm = s.tm;
        p.tn = s.tn;
        p.resident = s.resident;
        p.mt = (int)ceil_div(rows, s.tm);
        p.nt = (int)ceil_div(cols, s.tn);
        p.tiles = sym ? p.mt * (p.mt + 1) / 2 : p.mt * p.nt;
        const int64_t all = (int64_t)p.tiles * batch, round = (int64_t)kCus * s.resident;
        auto rounds = [&](int64_t groups) {
            const int64_t left = groups % round;
            const double fill = s.resident == 1 ? (double)left / kCus
                                                : (double)(ceil_div(left, kCus) - 1) / (s.resident - 1);
            return (double)(groups / round) * s.full + (left ? s.one + (s.full - s.one) * fill : 0.0);
        };
        for (int want = 1; want <= 16; ++want)
            for (int some = 0; some <= (want > 1 && all > round); ++some) {
                p.rest = want == 1 ? 0 : some ? all % round : all;
                p.whole = all - p.rest;
                p.per = (int)ceil_div(stages, want);
                p.splits = (int)ceil_div(stages, p.per);
                if (want > 1 && (p.per < 4 || p.rest == 0)) continue;
                double t = s.fixed + stages * rounds(p.whole) + p.per * rounds(p.rest * p.splits) + entries * 0.5e-6;
                if (p.rest > 0) t += 4.2 + p.splits * (0.22 + 1.1e-6 * p.rest * s.tm * s.tn) + (some ? 0.2 * s.fixed : 0.0);
                if (least == 0.0 || t < least) {
                    least = t;
                    best = p;
                }
            }
    }
    return best;
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
        m.lo = split ? rows * cols : 0;
        m.batch = rows * cols + m.lo;
        m.hi = reinterpret_cast<f16 *>(take(sizeof(f16) * (size_t)m.batch * batch));
        return m;
    };
    Buffers b;
    b.parts = reinterpret_cast<double *>(take(sizeof(double) * kParts * (size_t)batch));
    b.x = planes(rp, cp);
    b.t[0] = planes(cp, rp);
    b.t[1] = planes(cp, rp);
    b.a = planes(rp, rp);
    b.b = planes(rp, rp);
    // fp32 sums of the split products
    int64_t sums = 0;
    const int passes = split ? 3 : 1;
    auto room = [&](int64_t rows, int64_t cols, int64_t k, bool sym) {
        const ProductPlan p = plan_product(batch, (int)rows, (int)cols, passes * (int)(k / 64), sym);
        sums = std::max(sums, p.rest * p.splits * p.tm * p.tn);
    };
    room(rp, rp, cp, true);
    room(rp, rp, rp, true);
    room(rp, cp, rp, false);
    b.sums = reinterpret_cast<float *>(take(sizeof(float) * (size_t)sums));
    if (out) *out = b;
    return off;
}

template <bool SPLIT, Product KIND>
void launch_product(ProductArgs &g, const ProductPlan &p, int batch, hipStream_t st) {
    g.mt = p.mt;
    g.nt = p.nt;
    g.tiles = p.tiles;
    g.tm = p.tm;
    g.tn = p.tn;
    g.batch = batch;
    g.whole = p.whole;
    g.rest = p.rest;
    g.splits = p.splits;
    g.per = p.per;
    g.whole_chunk = (int)ceil_div(p.whole, kXcds);
    g.rest_chunk = (int)ceil_div(p.rest * p.splits, kXcds);
    const unsigned grid = (unsigned)(kXcds * (g.whole_chunk + g.rest_chunk));
    if (p.resident == 4) product_tile<SPLIT, KIND, 4, 1, 1, 2, 4><<<grid, 256, 0, st>>>(g);
    else if (p.tm == 64) product_tile<SPLIT, KIND, 4, 1, 1, 4, 2><<<grid, 256, 0, st>>>(g);
    else if (p.tm == 128) product_tile<SPLIT, KIND, 2, 2, 4, 2, 2><<<grid, 256, 0, st>>>(g);
    else if (p.tn == 256) product_pipe<SPLIT, KIND, 8><<<grid, 256, 0, st>>>(g);
    else if constexpr (!symmetric(KIND)) product_pipe<SPLIT, KIND, 4><<<grid, 256, 0, st>>>(g);
    if (p.rest > 0) {
        const int64_t blocks = p.rest * (p.tm / 32) * (p.tn / 64);
        product_join<SPLIT, KIND><<<(unsigned)blocks, 256, 0, st>>>(g);
    }
}

template <bool SPLIT>
hipError_t run_ortho(const OrthoArgs &o, const Buffers &b, hipStream_t st) {
    const int r = o.rows, c = o.cols;
    const int rt = (int)ceil_div(r, kPad), ct = (int)ceil_div(c, kPad);
    const bool along_c = o.g_col == 1;
    const Lines lines = {o.G, along_c ? o.g_row : o.g_col, o.g_batch, along_c ? r : c, along_c ? c : r, o.type};
    const int count = (int)std::min<int64_t>(kParts, ceil_div((int64_t)r * c, 4096));
    norm_parts<<<dim3(count, o.batch), 256, 0, st>>>(lines, count, b.parts);
    const PrepArgs p = {lines, b.parts, count, o.eps, ldexp(1.0, kScaleX), along_c ? b.x : b.t[0], along_c ? b.t[0] : b.x,
                        along_c ? ct : rt};
    prepare_x<SPLIT><<<dim3(rt * ct, o.batch), 256, 0, st>>>(p);
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
    const int rp = rt * kPad, cp = ct * kPad, passes = SPLIT ? 3 : 1;
    const ProductPlan gram = plan_product(o.batch, rp, rp, passes * ct, true),
                      poly = plan_product(o.batch, rp, rp, passes * rt, true),
                      update = plan_product(o.batch, rp, cp, passes * rt, false);
    g.parts = b.sums;
    for (int step = 0; step < o.steps; ++step) {
        const double *k = o.coef + 3 * step;
        const Planes &t = b.t[step & 1], &t_next = b.t[(step + 1) & 1];
        g.rows = g.cols = rp;
        g.p = g.q = b.x;
        g.d = g.dt = b.a;
        g.kblocks = cp / 64;
        g.mul = (float)ldexp(1.0, kScaleA - 2 * kScaleX);
        launch_product<SPLIT, kGram>(g, gram, o.batch, st);
        g.p = g.q = g.e = b.a;
        g.d = g.dt = b.b;
        g.kblocks = rp / 64;
        g.diag = (float)ldexp(k[0], kScaleB);
        g.add = (float)ldexp(k[1], kScaleB - kScaleA);
        g.mul = (float)ldexp(k[2], kScaleB - 2 * kScaleA);
        launch_product<SPLIT, kPoly>(g, poly, o.batch, st);
        g.p = b.b;
        g.q = t;
        g.d = b.x;
        g.dt = t_next;
        g.cols = cp;
        g.mul = (float)ldexp(1.0, -kScaleB);
        if (step + 1 < o.steps) launch_product<SPLIT, kUpdate>(g, update, o.batch, st);
        else launch_product<SPLIT, kLast>(g, update, o.batch, st);
    }
    return hipGetLastError();
}

}  // namespace

bool ortho_is_small(int rows, int cols, int type) { return ortho_fits_lds(rows, cols, split_of(type)); }

// Small matrices stay in LDS: 256 bytes, which nothing uses, so that a caller passes
// a workspace for every size.
size_t ortho_workspace(int batch, int rows, int cols, int type) {
    if (ortho_is_small(rows, cols, type)) return 256;
    return carve(batch, rows, cols, split_of(type), nullptr, nullptr);
}

hipError_t launch_ortho(const OrthoArgs &o, void *ws, hipStream_t st) {
    Buffers b;
    const bool split = split_of(o.type);
    if (ortho_is_small(o.rows, o.cols, o.type)) return launch_ortho_small(o, split, st);
    carve(o.batch, o.rows, o.cols, split, ws, &b);
    return split ? run_ortho<true>(o, b, st) : run_ortho<false>(o, b, st);
}

}  // namespace o2m
