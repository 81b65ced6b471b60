// Tiles of 8-bit block-scaled products whose partial sums are scaled by the vector
// unit, and small ones of every kind; k_fp8.hip says which product takes what.
#pragma once

#include "fp8_operand.h"
#include "fp8_plan.h"
#include "mfma_pipe.h"
#include "tile_schedule.h"

namespace o2m {

// C = A B^T, entry (i, j) at C[i ldc + j].
struct Fp8Args {
    Side a, b;
    int k, kblocks;
    int mt, nt, chunk;   // tiles; per XCD
    void *C;
    int64_t ldc;
    int type, accumulate;
    float *parts;        // split launches: sums [split][m][pitch]
    int pitch, splits, per;
};

// N (4 or 8) neighbouring outputs of a row, from `col` on, at once where all exist.
// (The accesses need no alignment but the entries' own.)
template <int N, class V>
__device__ inline void store_run(const Fp8Args &g, int row, int col, V v) {
    typedef _Float16 vf16 __attribute__((ext_vector_type(N)));
    typedef __bf16 vbf16 __attribute__((ext_vector_type(N)));
    const int n = g.b.rows - col;
    if (row >= g.a.rows || n <= 0) return;
    const int64_t at = row * g.ldc + col;
    if (n >= N) {
        if (g.type == O2M_TYPE_F32) {
            float *p = static_cast<float *>(g.C) + at;
            V old;
            if (g.accumulate) {
                __builtin_memcpy(&old, p, sizeof old);
                v += old;
            }
            __builtin_memcpy(p, &v, sizeof v);
        } else if (g.type == O2M_TYPE_F16) {
            _Float16 *p = static_cast<_Float16 *>(g.C) + at;
            vf16 h;
            if (g.accumulate) {
                __builtin_memcpy(&h, p, sizeof h);
                v += __builtin_convertvector(h, V);
            }
            h = __builtin_convertvector(v, vf16);
            __builtin_memcpy(p, &h, sizeof h);
        } else {
            __bf16 *p = static_cast<__bf16 *>(g.C) + at;
            vbf16 h;
            if (g.accumulate) {
                __builtin_memcpy(&h, p, sizeof h);
                v += __builtin_convertvector(h, V);
            }
            h = __builtin_convertvector(v, vbf16);
            __builtin_memcpy(p, &h, sizeof h);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j < n) store_out(g.C, at + j, g.type, v[j] + (g.accumulate ? load_out(g.C, at + j, g.type) : 0.0f));
}

// WR x WC waves of M x 4 blocks of 16 x 16 and two stage buffers.  Rows of a
// wave are 16 i + q (block i, q = lane % 16), columns 4 q + j, so that a lane's
// blocks j are neighbouring columns.  WB: B's scale is one for the wave's columns.
template <int WR, int WC, int M>
struct TileOf {
    static constexpr int kWaves = WR * WC, kThreads = 64 * kWaves;
    static constexpr int kTm = WR * M * 16, kTn = WC * 64, kRows = kTm + kTn;
    static constexpr int kCopyA = kTm / 8 / kWaves, kCopyB = kTn / 8 / kWaves;
    static constexpr int kBuf = kRows * kStageRowBytes;
    static_assert(kRows <= kThreads && kCopyA * 8 * kWaves == kTm && kCopyB * 8 * kWaves == kTn, "shares of a stage");
};

// Stage kb lies in buffer (kb - s0) % 2, and the next one is on its way.  Each thread
// fetches the scale of one row of A or B as far ahead, into a register, and passes
// it on in LDS when the stage begins.  What hides the latencies of a stage are the
// OCC workgroups that a CU holds.
template <Sum SUM, int FA, int FB, bool WB, int WR, int WC, int M, int OCC>
__global__ __launch_bounds__(64 * WR * WC, OCC) void fp8_tile(Fp8Args g) {
    typedef TileOf<WR, WC, M> T;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * T::kBuf + 2 * T::kRows * 4];
    uint32_t *const scales = reinterpret_cast<uint32_t *>(lds + 2 * T::kBuf);   // [2][A's rows, B's rows]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int z = blockIdx.x % g.splits, slot = blockIdx.x / g.splits;
    const TileCoord tc = tile_of(slot & 7, slot >> 3, g.mt, g.nt, g.chunk, 0);
    if (!tc.valid) return;   // whole workgroup
    const int i0 = tc.ti * T::kTm, j0 = tc.tj * T::kTn;
    const auto ra = rows_of(g.a.values + i0 * g.a.ld, min(T::kTm, g.a.rows - i0), g.a.ld, g.k);
    const auto rb = rows_of(g.b.values + j0 * g.b.ld, min(T::kTn, g.b.rows - j0), g.b.ld, g.k);
    const int s0 = z * g.per, s1 = min(g.kblocks, s0 + g.per);
    auto copy = [&](int kb, uint8_t *buf) {
        const int left = g.k - kb * kBlockK;
#pragma unroll
        for (int c = 0; c < T::kCopyA; ++c) {
            const int q = wave * T::kCopyA + c;
            copy_rows<1>(ra, buf + q * 1024, lane, q, (int)g.a.ld, kb * kStageRowBytes, left);
        }
#pragma unroll
        for (int c = 0; c < T::kCopyB; ++c) {
            const int q = wave * T::kCopyB + c;
            copy_rows<2>(rb, buf + T::kTm * kStageRowBytes + q * 1024, lane, q, (int)g.b.ld, kb * kStageRowBytes, left);
        }
    };
    // (threads past the rows fetch the last row's)
    const int my_row = min(tid, T::kRows - 1);
    const bool mine_a = my_row < T::kTm;
    const Side &side = mine_a ? g.a : g.b;
    const int64_t scale_row = scale_index(side, mine_a ? i0 + my_row : j0 + my_row - T::kTm, 0);
    auto fetch = [&](int kb) -> uint32_t {
        const int64_t at = scale_row + kb * side.s_blk;
        return side.pow2 ? static_cast<const uint8_t *>(side.scales)[at] : static_cast<const uint32_t *>(side.scales)[at];
    };
    const int wi = wave / WC * (M * 16), wj = wave % WC * 64, q = lane & 15;
    v4f acc[M][4];
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = v4f{0, 0, 0, 0};
    uint32_t ahead = fetch(s0);
    copy(s0, lds);
    for (int kb = s0; kb < s1; ++kb) {
        const int u = (kb - s0) & 1;
        uint8_t *buf = lds + u * T::kBuf;
        const int left = g.k - kb * kBlockK;
        if (tid < T::kRows)
            scales[(kb & 1) * T::kRows + tid] = SUM == kWideScaled ? __float_as_uint(code_value(ahead)) : ahead;
        wait_vmem<0>();   // this stage has landed
        lds_barrier();
        if (left < kBlockK && (left & 15)) {   // uniform: the last stage of an odd k
            if (tid < T::kRows) clear_row_tail(buf, tid, left, mine_a ? 1 : 2);
            lds_barrier();
        }
        if (kb + 1 < s1) {
            ahead = fetch(kb + 1);
            copy(kb + 1, lds + (u ^ 1) * T::kBuf);
        }
        const uint32_t *sc = scales + (kb & 1) * T::kRows;
        const v4i cb = *reinterpret_cast<const v4i *>(sc + T::kTm + wj + 4 * q);   // codes, or floats' bits
        const v4f sb = __builtin_bit_cast(v4f, cb);
        v8i fb[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) fb[j] = read_fragment<2>(buf + T::kTm * kStageRowBytes, wj + 4 * q + j, lane);
        std::conditional_t<SUM == kWideScaled, v8bf16, v8f16> wb[SUM >= kWide ? 4 : 1][4];
        if constexpr (SUM == kWide) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int h = 0; h < 4; ++h) wb[j][h] = widen<FB>(fb[j][2 * h], fb[j][2 * h + 1]);
        } else if constexpr (SUM == kWideScaled) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int h = 0; h < 4; ++h) wb[j][h] = widen_scaled<FB>(fb[j][2 * h], fb[j][2 * h + 1], sb[j]);
        }
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const v8i fa = read_fragment<1>(buf, wi + 16 * i + q, lane);
            if constexpr (SUM == kScaled) {
                const int ca = (int)sc[wi + 16 * i + q];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        fa, fb[j], acc[i][j], FA, FB, 0, ca, 0, cb[j]);
            } else if constexpr (SUM == kWideScaled) {
                const float sa = __uint_as_float(sc[wi + 16 * i + q]);
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const v8bf16 wa = widen_scaled<FA>(fa[2 * h], fa[2 * h + 1], sa);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa, wb[j][h], acc[i][j], 0, 0, 0);
                }
            } else {
                v4f sa = *reinterpret_cast<const v4f *>(sc + wi + 16 * i + 4 * (lane >> 4));
                if (WB) sa *= sb[0];
                v8f16 wa[4];
                if constexpr (SUM == kWide) {
#pragma unroll
                    for (int h = 0; h < 4; ++h) wa[h] = widen<FA>(fa[2 * h], fa[2 * h + 1]);
                }
                v4f p[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) p[j] = v4f{0, 0, 0, 0};
                if constexpr (SUM == kPartial) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        p[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb[j], p[j], FA, FB, 0, 0, 0, 0);
                } else {
#pragma unroll
                    for (int h = 0; h < 4; ++h)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            p[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wa[h], wb[j][h], p[j], 0, 0, 0);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[i][j][e] = fmaf(p[j][e], WB ? sa[e] : sa[e] * sb[j], acc[i][j][e]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = i0 + wi + 16 * i + 4 * (lane >> 4) + e, col = j0 + wj + 4 * q;
            const v4f v = {acc[i][0][e], acc[i][1][e], acc[i][2][e], acc[i][3][e]};
            if (g.splits == 1) store_run<4>(g, row, col, v);
            else if (row < g.a.rows && col < g.pitch)
                *reinterpret_cast<v4f *>(g.parts + ((int64_t)z * g.a.rows + row) * g.pitch + col) = v;
        }
}

template <Sum SUM, int FA, int FB, bool WB, int WR, int WC, int M, int OCC>
hipError_t launch_tile(Fp8Args &g, hipStream_t st) {
    typedef TileOf<WR, WC, M> T;
    g.mt = (int)ceil_div(g.a.rows, T::kTm);
    g.nt = (int)ceil_div(g.b.rows, T::kTn);
    const int64_t chunk = ceil_div((int64_t)g.mt * g.nt, kXcds), grid = kXcds * chunk * g.splits;
    if (!launch_fits(grid, T::kThreads)) return hipErrorInvalidValue;
    g.chunk = (int)chunk;
    fp8_tile<SUM, FA, FB, WB, WR, WC, M, OCC><<<(unsigned)grid, T::kThreads, 0, st>>>(g);
    return hipGetLastError();
}

// Tile sizes: 256 x 256 by 8 waves (kPartial; kScaled has kernels of its own for this
// and 256 x 128), 128 x 128 by 4 (two workgroups per CU), 64 x 64 by 4 (four; two with
// three stages on their way each were never faster: 1537 x 1283 x 2051 with a 16-bit
// result, 525 tiles, 22 against 17 us).
template <Sum SUM, int FA, int FB, bool WB>
hipError_t launch_sizes(Fp8Args &g, TileSize size, hipStream_t st) {
    switch (size) {
    case k64: return launch_tile<SUM, FA, FB, WB, 4, 1, 1, 4>(g, st);
    case k128: return launch_tile<SUM, FA, FB, WB, 2, 2, 4, 2>(g, st);
    default: break;
    }
    if constexpr (SUM == kPartial) return launch_tile<SUM, FA, FB, WB, 2, 4, 8, 2>(g, st);
    return hipErrorInvalidValue;
}

// One file each; format: of A x 2 + of B.
hipError_t launch_fp8_scaled(Fp8Args &g, int format, TileSize size, hipStream_t st);
hipError_t launch_fp8_partial(Fp8Args &g, int format, TileSize size, hipStream_t st);
hipError_t launch_fp8_wide(Fp8Args &g, int format, TileSize size, hipStream_t st);

}  // namespace o2m
