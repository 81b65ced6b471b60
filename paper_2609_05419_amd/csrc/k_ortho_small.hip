// The orthogonalised update of small matrices, whole in one launch: one workgroup
// of 16 waves per matrix, which keeps X (r x c, padded to multiples of 32), its
// transpose and A or B in LDS, held as k_ortho.hip says.
//
// Bound: latency.  Each product is one round of the waves, a wave owning 32 x 32 of
// its outputs (2 x 2 blocks of 16 x 16), between barriers; 15 of them for five
// steps, where separate launches take 3 us and more each (16 matrices of 96 x 80
// in fp32: 43 us, of them 14 to load and write and 5.8 a step, against 105 in 17
// launches).  By count a step is some 2 us: 1024 threads leave a lane 128 registers, of
// which 62 are spilled to scratch memory (28 with one part), and the k loop waits for
// each of its LDS reads.
#include "ortho_shared.h"

#include <math.h>

namespace o2m {
namespace {

constexpr int kWaves = 16, kThreads = 64 * kWaves;
constexpr int kRowPad = 8;          // entries between rows, which spreads them over the banks
constexpr int kLdsBytes = 152 * 1024;
constexpr int kMaxSteps = 64;

struct SmallArgs {
    Lines g;               // along: the lines are rows of X, otherwise its columns
    int along, r, c, rp, cp;
    void *O;
    int64_t o_row, o_col, o_batch;
    int steps;
    double eps;
};
// (by value: the coefficients a, b, c of each step)
struct SmallCoef {
    float k[3 * kMaxSteps];
};

// A matrix in LDS: rows of `pitch` entries, the second part `lo` entries on.
struct Held {
    f16 *hi;
    int pitch, lo;
};

typedef _Float16 v4f16 __attribute__((ext_vector_type(4)));

template <bool SPLIT>
__device__ inline v4f held4(const Held &m, int row, int col) {
    const f16 *p = m.hi + row * m.pitch + col;
    v4f v = __builtin_convertvector(*reinterpret_cast<const v4f16 *>(p), v4f);
    if (SPLIT) v += __builtin_convertvector(*reinterpret_cast<const v4f16 *>(p + m.lo), v4f);
    return v;
}
template <bool SPLIT>
__device__ inline void hold4(const Held &m, int row, int col, const v4f &v) {
    f16 *p = m.hi + row * m.pitch + col;
    const v4f16 hi = __builtin_convertvector(v, v4f16);
    *reinterpret_cast<v4f16 *>(p) = hi;
    if (SPLIT) *reinterpret_cast<v4f16 *>(p + m.lo) = __builtin_convertvector(v - __builtin_convertvector(hi, v4f), v4f16);
}
template <bool SPLIT>
__device__ inline void hold(const Held &m, int row, int col, float v) {
    f16 *p = m.hi + row * m.pitch + col;
    const f16 hi = (f16)v;
    *p = hi;
    if (SPLIT) p[m.lo] = (f16)(v - (float)hi);
}

// D = P Q^T on rows i0 .. i0 + 31 of P and j0 .. of Q, k entries each (a multiple of
// 32): block (x, y) in acc[x][y], entries (row 4 (lane / 16) + e, column lane % 16).
template <bool SPLIT>
__device__ inline void product32(const Held &p, const Held &q, int i0, int j0, int k, int lane, v4f (&acc)[2][2]) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) acc[x][y] = v4f{0, 0, 0, 0};
    const f16 *a = p.hi + (i0 + (lane & 15)) * p.pitch + 8 * (lane >> 4);
    const f16 *b = q.hi + (j0 + (lane & 15)) * q.pitch + 8 * (lane >> 4);
#pragma unroll 1
    for (int at = 0; at < k; at += 32) {
        v8f16 f[2][SPLIT ? 2 : 1], g[2][SPLIT ? 2 : 1];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int s = 0; s < (SPLIT ? 2 : 1); ++s) {
                f[x][s] = *reinterpret_cast<const v8f16 *>(a + 16 * x * p.pitch + at + s * p.lo);
                g[x][s] = *reinterpret_cast<const v8f16 *>(b + 16 * x * q.pitch + at + s * q.lo);
            }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                if (SPLIT) {
                    acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[x][SPLIT], g[y][0], acc[x][y], 0, 0, 0);
                    acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[x][0], g[y][SPLIT], acc[x][y], 0, 0, 0);
                }
                acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[x][0], g[y][0], acc[x][y], 0, 0, 0);
            }
    }
}

template <bool SPLIT>
__global__ __launch_bounds__(kThreads) void ortho_small(SmallArgs g, SmallCoef coef) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[kLdsBytes];
    __shared__ double sums[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t b = blockIdx.x;
    constexpr int kKeep = SPLIT ? 2 : 1;
    const int px = g.cp + kRowPad, pt = g.rp + kRowPad;
    f16 *at = reinterpret_cast<f16 *>(lds);
    const Held x = {at, px, g.rp * px};
    at += kKeep * g.rp * px;
    const Held t = {at, pt, g.cp * pt};
    at += kKeep * g.cp * pt;
    const Held m = {at, pt, g.rp * pt};   // A, then B

    // the norm, summed in a fixed order; the entries are read again below
    const int per_line = (g.g.len + 7) / 8, runs = per_line * g.g.lines;
    double s = 0.0;
    for (int i = tid; i < runs; i += kThreads) {
        const int p = i / per_line, q = (i - p * per_line) * 8;
        const v8f v = load_some(g.g.G, b * g.g.batch + p * g.g.line + q, g.g.len - q, g.g.type);
#pragma unroll
        for (int j = 0; j < 8; ++j) s += (double)v[j] * (double)v[j];
    }
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) s += __shfl_xor(s, w);
    if (lane == 0) sums[wave] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += sums[w];
    const double norm = sqrt(s);
    // Inf and NaN anywhere: NaN everywhere
    const double inv = norm <= 1.7e308 ? (double)(1 << kScaleX) / (norm + g.eps) : (double)NAN;

    // X and its transpose with their padding: lines of `along`'s direction
    const Held &lines = g.along ? x : t, &turned = g.along ? t : x;
    const int plines = g.along ? g.rp : g.cp, plen8 = (g.along ? g.cp : g.rp) / 8;
    for (int i = tid; i < plines * plen8; i += kThreads) {
        const int p = i / plen8, q = (i - p * plen8) * 8;
        const int n = p < g.g.lines ? min(8, g.g.len - q) : 0;
        const v8f v = load_some(g.g.G, b * g.g.batch + p * g.g.line + q, n, g.g.type);
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            y[j] = j < n ? (float)((double)v[j] * inv) : 0.0f;
            hold<SPLIT>(turned, q + j, p, y[j]);
        }
        hold4<SPLIT>(lines, p, q, v4f{y[0], y[1], y[2], y[3]});
        hold4<SPLIT>(lines, p, q + 4, v4f{y[4], y[5], y[6], y[7]});
    }
    __syncthreads();
    if (g.steps == 0) {   // X itself
        for (int i = tid; i < g.r * g.c; i += kThreads) {
            const int row = i / g.c, col = i - row * g.c;
            const f16 *v = x.hi + row * x.pitch + col;
            store_any(g.O, b * g.o_batch + row * g.o_row + col * g.o_col, g.g.type,
                      ((float)v[0] + (SPLIT ? (float)v[x.lo] : 0.0f)) * (1.0f / (1 << kScaleX)));
        }
        return;   // whole workgroup
    }

    const int rt = g.rp / 32, ct = g.cp / 32;
    const int quad = lane >> 4, q = lane & 15;
    // this wave's 32 x 32 of a square product, and of X
    const bool has_a = wave < rt * rt, has_x = wave < rt * ct;   // uniform
    const int ai = wave % rt * 32, aj = wave / rt * 32;
    v4f acc[2][2];
    for (int step = 0; step < g.steps; ++step) {
        const float ka = coef.k[3 * step] * (1 << kScaleB), kb = coef.k[3 * step + 1] * 0x1p-5f,
                    kc = coef.k[3 * step + 2] * 0x1p-16f;
        static_assert(kScaleB - kScaleA == -5 && kScaleB - 2 * kScaleA == -16 && kScaleA - 2 * kScaleX == -17, "scales");
        if (has_a) {
            product32<SPLIT>(x, x, ai, aj, g.cp, lane, acc);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int v = 0; v < 2; ++v)   // (A is its own transpose: 4 rows of a column at once)
                    hold4<SPLIT>(m, aj + 16 * v + q, ai + 16 * u + 4 * quad, acc[u][v] * 0x1p-17f);
        }
        __syncthreads();
        if (has_a) product32<SPLIT>(m, m, ai, aj, g.rp, lane, acc);
        __syncthreads();   // every wave is done with A as an operand
        if (has_a) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    const int row = aj + 16 * v + q, col = ai + 16 * u + 4 * quad;
                    v4f d = kc * acc[u][v] + kb * held4<SPLIT>(m, row, col);
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[e] += col + e == row ? ka : 0.0f;
                    hold4<SPLIT>(m, row, col, d);
                }
        }
        __syncthreads();
        if (has_x) product32<SPLIT>(m, t, ai, aj, g.rp, lane, acc);
        __syncthreads();   // every wave is done with X and B
        if (!has_x) {
        } else if (step + 1 < g.steps) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    const int row = ai + 16 * u + 4 * quad, col = aj + 16 * v + q;
                    const v4f d = acc[u][v] * (1.0f / (1 << kScaleB));
                    hold4<SPLIT>(t, col, row, d);
#pragma unroll
                    for (int e = 0; e < 4; ++e) hold<SPLIT>(x, row + e, col, d[e]);
                }
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int v = 0; v < 2; ++v)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int row = ai + 16 * u + 4 * quad + e, col = aj + 16 * v + q;
                        if (row < g.r && col < g.c)
                            store_any(g.O, b * g.o_batch + row * g.o_row + col * g.o_col, g.g.type,
                                      acc[u][v][e] * (1.0f / (1 << (kScaleB + kScaleX))));
                    }
        }
        __syncthreads();
    }
}

int64_t lds_bytes(int r, int c, bool split) {
    const int64_t rp = round_up64(r, 32), cp = round_up64(c, 32), px = cp + kRowPad, pt = rp + kRowPad;
    return (split ? 2 : 1) * 2 * (rp * px + cp * pt + rp * pt);
}

}  // namespace

// Matrices that fit, whose products are one round of the waves.
bool ortho_fits_lds(int r, int c, bool split) {
    const int64_t rt = ceil_div(r, 32), ct = ceil_div(c, 32);
    return rt * ct <= kWaves && lds_bytes(r, c, split) <= kLdsBytes;
}

hipError_t launch_ortho_small(const OrthoArgs &o, bool split, hipStream_t st) {
    SmallArgs g;
    const bool along = o.g_col == 1;
    g.g = {o.G, along ? o.g_row : o.g_col, o.g_batch, along ? o.rows : o.cols, along ? o.cols : o.rows, o.type};
    g.along = along;
    g.r = o.rows;
    g.c = o.cols;
    g.rp = (int)round_up64(o.rows, 32);
    g.cp = (int)round_up64(o.cols, 32);
    g.O = o.O;
    g.o_row = o.o_row;
    g.o_col = o.o_col;
    g.o_batch = o.o_batch;
    g.steps = o.steps;
    g.eps = o.eps;
    SmallCoef k;
    for (int i = 0; i < 3 * o.steps; ++i) k.k[i] = (float)o.coef[i];
    if (split) ortho_small<true><<<(unsigned)o.batch, kThreads, 0, st>>>(g, k);
    else ortho_small<false><<<(unsigned)o.batch, kThreads, 0, st>>>(g, k);
    return hipGetLastError();
}

}  // namespace o2m
