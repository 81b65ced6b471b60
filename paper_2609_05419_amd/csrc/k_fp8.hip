// Products of 8-bit block-scaled operands (include/o2m.h: o2m_gemm_fp8).
//
//   C[i, j] = sum_b sa[i, b] sb[j, b] sum_{k in block b} qa[i, k] qb[j, k]
//
// A block of 128 along k is one v_mfma_f32_16x16x128_f8f6f4, so a scale belongs
// to one MFMA: power-of-two scales go into the scaled form of the instruction,
// fp32 ones multiply the partial sum of the block as it is added up.
//
// That instruction adds 8 neighbouring products at a time with 13 bits below
// the largest of them, and such groups in fp32 (measured: of two products of a
// group the smaller one is lost below 2^-13 of the larger, of different groups
// below 2^-24).  On normal data in blocks a sum is 1.5e-5 to 3e-5 off in the
// 2-norm: far below the rounding of a bf16 (1.7e-3) or fp16 (2.1e-4) result,
// which therefore take it, and far above that of an fp32 one.  Products with an
// fp32 result turn the values to fp16 in registers, which holds both formats
// exactly, and add up with v_mfma_f32_16x16x32_f16 (6e-8), at half the rate.
//
// Bound: 8-bit (fp32 results: fp16) MFMA for large products.
#include "mfma_tiles.h"
#include "model_internal.h"

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

namespace o2m {
namespace {

struct Side {
    const uint8_t *values;
    int64_t ld;
    const void *scales;
    int64_t s_row, s_blk;
    int rows;
    int by_row;   // 1: a scale per row, 0: per 128 rows
    int pow2;
};

struct Fp8Args {
    Side a, b;
    int k, kblocks;
    int mt, nt;
    void *C;
    int64_t ldc;
    int type, accumulate, vec;
};

typedef _Float16 v2f16 __attribute__((ext_vector_type(2)));
typedef _Float16 v8f16 __attribute__((ext_vector_type(8)));

// How a block's products are added up.
enum Sum {
    kScaled,    // 8-bit MFMA with power-of-two scales
    kPartial,   // 8-bit MFMA, then fp32 scales
    kWide,      // fp16 MFMA, then scales of either kind
};

// Eight 8-bit values (two dwords) in fp16, exactly.
template <int F>
__device__ inline v8f16 widen(int x, int y) {
    v2f16 r[4];
    const uint32_t w[2] = {(uint32_t)x, (uint32_t)y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        r[2 * i] = F == O2M_FP8_E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, false)
                                     : __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w[i], 1.0f, false);
        r[2 * i + 1] = F == O2M_FP8_E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, true)
                                         : __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w[i], 1.0f, true);
    }
    return v8f16{r[0][0], r[0][1], r[1][0], r[1][1], r[2][0], r[2][1], r[3][0], r[3][1]};
}

__device__ inline float load_out(const void *C, int64_t i, int type) {
    if (type == O2M_TYPE_F32) return static_cast<const float *>(C)[i];
    if (type == O2M_TYPE_F16) return __half2float(static_cast<const __half *>(C)[i]);
    return __bfloat162float(static_cast<const __hip_bfloat16 *>(C)[i]);
}
__device__ inline void store_out(void *C, int64_t i, int type, float v) {
    if (type == O2M_TYPE_F32) static_cast<float *>(C)[i] = v;
    else if (type == O2M_TYPE_F16) static_cast<__half *>(C)[i] = __float2half(v);
    else static_cast<__hip_bfloat16 *>(C)[i] = __float2bfloat16(v);
}

// The scale of `row` in block kb, as an e8m0 byte or a float.  Rows past the last
// one take its scale (their values are zeros).
__device__ inline int64_t scale_index(const Side &s, int row, int kb) {
    row = min(row, s.rows - 1);
    return (s.by_row ? row : row >> 7) * s.s_row + kb * s.s_blk;
}
__device__ inline int scale_code(const Side &s, int row, int kb) {
    return static_cast<const uint8_t *>(s.scales)[scale_index(s, row, kb)];
}
// 2^(code - 127); 2^-127 (code 0) is half the smallest normal number, 255 is NaN
__device__ inline float code_value(uint32_t code) {
    return code == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(code ? code << 23 : 0x00400000u);
}
template <Sum SUM>
__device__ inline float scale_value(const Side &s, int row, int kb) {
    const int64_t i = scale_index(s, row, kb);
    if (SUM == kWide && s.pow2) return code_value(static_cast<const uint8_t *>(s.scales)[i]);
    return static_cast<const float *>(s.scales)[i];
}

// One tile of 128 x 128 per workgroup of 2 x 2 waves, 4 x 4 blocks of 16 x 16
// each; two stage buffers.
template <Sum SUM, int FA, int FB>
__global__ __launch_bounds__(256) void fp8_tile(Fp8Args g) {
    constexpr int T = 128, kBuf = 2 * T * kStageRowBytes;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kBuf];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ti = blockIdx.x % g.mt, tj = blockIdx.x / g.mt;
    const int i0 = ti * T, j0 = tj * T;
    const auto ra = rows_of(g.a.values + i0 * g.a.ld, min(T, g.a.rows - i0), g.a.ld, g.k);
    const auto rb = rows_of(g.b.values + j0 * g.b.ld, min(T, g.b.rows - j0), g.b.ld, g.k);
    const CopyLane cl = copy_lane(lane);
    auto copy = [&](int kb) {
        uint8_t *buf = lds + (kb & 1) * kBuf;
        const int left = g.k - kb * kBlockK;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            copy_rows(ra, buf + (wave * 4 + q) * 1024, cl, wave * 4 + q, (int)g.a.ld, kb, left);
            copy_rows(rb, buf + T * kStageRowBytes + (wave * 4 + q) * 1024, cl, wave * 4 + q, (int)g.b.ld, kb, left);
        }
    };
    const int wi = (wave >> 1) * 64, wj = (wave & 1) * 64;
    v4f acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = v4f{0, 0, 0, 0};
    copy(0);
    for (int kb = 0; kb < g.kblocks; ++kb) {
        wait_vmem<0>();
        lds_barrier();
        uint8_t *buf = lds + (kb & 1) * kBuf;
        const int left = g.k - kb * kBlockK;
        if (left < kBlockK && (left & 15)) {   // uniform: the last stage of an odd k
            clear_row_tail(buf, tid, left);    // 256 rows: A's, then B's
            lds_barrier();
        }
        if (kb + 1 < g.kblocks) copy(kb + 1);
        int ca[4], cb[4];
        float sa[4][4], sb[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int ra0 = i0 + wi + 16 * i, rb0 = j0 + wj + 16 * i + (lane & 15);
            if (SUM == kScaled) {
                ca[i] = scale_code(g.a, ra0 + (lane & 15), kb);
                cb[i] = scale_code(g.b, rb0, kb);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) sa[i][e] = scale_value<SUM>(g.a, ra0 + 4 * (lane >> 4) + e, kb);
                sb[i] = scale_value<SUM>(g.b, rb0, kb);
            }
        }
        v8i fa[4], fb[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fa[i] = read_fragment(buf, wi + 16 * i, lane);
            fb[i] = read_fragment(buf + T * kStageRowBytes, wj + 16 * i, lane);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (SUM == kScaled) {
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[i], fb[j], acc[i][j], FA, FB, 0,
                                                                                 ca[i], 0, cb[j]);
                    continue;
                }
                v4f p = {0, 0, 0, 0};
                if (SUM == kPartial) {
                    p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[i], fb[j], p, FA, FB, 0, 0, 0, 0);
                } else {
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        p = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen<FA>(fa[i][2 * h], fa[i][2 * h + 1]),
                                                                   widen<FB>(fb[j][2 * h], fb[j][2 * h + 1]), p, 0, 0, 0);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[e], sa[i][e] * sb[j], acc[i][j][e]);
            }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int col = j0 + wj + 16 * j + (lane & 15);
        if (col >= g.b.rows) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = i0 + wi + 16 * i + 4 * (lane >> 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (row + e >= g.a.rows) continue;
                const int64_t at = col * g.ldc + row + e;
                store_out(g.C, at, g.type, acc[i][j][e] + (g.accumulate ? load_out(g.C, at, g.type) : 0.0f));
            }
        }
    }
}

template <class T>
__global__ __launch_bounds__(256) void zero_out(T *C, int64_t m, int64_t total, int64_t ldc) {
    for (int64_t t = blockIdx.x * 256LL + threadIdx.x; t < total; t += gridDim.x * 256LL)
        C[t % m + t / m * ldc] = T(0);
}

Side side_of(const o2m_fp8_operand &o, int rows) {
    return {static_cast<const uint8_t *>(o.values), o.ld, o.scales, o.s_row, o.s_blk, rows, o.block == 1,
            o.scale_type == O2M_SCALES_POW2};
}

template <int FA, int FB>
void launch_formats(const Fp8Args &g, unsigned grid, hipStream_t st) {
    if (g.type == O2M_TYPE_F32) fp8_tile<kWide, FA, FB><<<grid, 256, 0, st>>>(g);
    else if (g.a.pow2) fp8_tile<kScaled, FA, FB><<<grid, 256, 0, st>>>(g);
    else fp8_tile<kPartial, FA, FB><<<grid, 256, 0, st>>>(g);
}

}  // namespace

hipError_t launch_zero_out(void *C, int64_t m, int64_t n, int64_t ldc, int size, hipStream_t st) {
    const int64_t total = m * n;
    if (total <= 0) return hipSuccess;
    const unsigned grid = (unsigned)(ceil_div(total, 256) < 2048 ? ceil_div(total, 256) : 2048);
    if (size == 4) zero_out<uint32_t><<<grid, 256, 0, st>>>(static_cast<uint32_t *>(C), m, total, ldc);
    else zero_out<uint16_t><<<grid, 256, 0, st>>>(static_cast<uint16_t *>(C), m, total, ldc);
    return hipGetLastError();
}

size_t gemm_fp8_workspace(int m, int n, int k) { return 0; }

hipError_t launch_gemm_fp8(int m, int n, int k, const o2m_fp8_operand &A, const o2m_fp8_operand &B, void *C, int type,
                           int64_t ldc, bool accumulate, void *ws, hipStream_t st) {
    Fp8Args g = {};
    g.a = side_of(A, m);
    g.b = side_of(B, n);
    g.k = k;
    g.kblocks = (int)ceil_div(k, kBlockK);
    g.mt = (int)ceil_div(m, 128);
    g.nt = (int)ceil_div(n, 128);
    g.C = C;
    g.ldc = ldc;
    g.type = type;
    g.accumulate = accumulate;
    const int64_t grid = (int64_t)g.mt * g.nt;
    if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
    switch (A.format * 2 + B.format) {
    case 0: launch_formats<0, 0>(g, (unsigned)grid, st); break;
    case 1: launch_formats<0, 1>(g, (unsigned)grid, st); break;
    case 2: launch_formats<1, 0>(g, (unsigned)grid, st); break;
    default: launch_formats<1, 1>(g, (unsigned)grid, st); break;
    }
    return hipGetLastError();
}

}  // namespace o2m
