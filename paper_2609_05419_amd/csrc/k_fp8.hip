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
#include "mfma_pipe.h"
#include "mfma_tiles.h"
#include "model_internal.h"
#include "tile_schedule.h"

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
    int mt, nt, chunk;
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
    auto copy = [&](int kb) {
        uint8_t *buf = lds + (kb & 1) * kBuf;
        const int left = g.k - kb * kBlockK;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            copy_rows<0>(ra, buf + (wave * 4 + q) * 1024, lane, wave * 4 + q, (int)g.a.ld, kb, left);
            copy_rows<0>(rb, buf + T * kStageRowBytes + (wave * 4 + q) * 1024, lane, wave * 4 + q, (int)g.b.ld, kb, left);
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
            fa[i] = read_fragment<0>(buf, wi + 16 * i + (lane & 15), lane);
            fb[i] = read_fragment<0>(buf + T * kStageRowBytes, wj + 16 * i + (lane & 15), lane);
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

// ---- large tiles -------------------------------------------------------------

// D += (A 2^sa) (B 2^sb)^T on one 16 x 16 block, the scales being byte I of sa and
// byte J of sb.  In assembly so that the accumulators stay in their registers
// (with the builtin they are copied to and fro in every stage).
template <int FA, int FB, int I, int J>
__device__ inline void mfma_scaled(v4f &d, const v8i &a, const v8i &b, int sa, int sb) {
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0] cbsz:%9 "
                 "blgp:%10"
                 : "+a"(d)
                 : "v"(a), "v"(b), "v"(sa), "v"(sb), "n"(I & 1), "n"(J & 1), "n"(I >> 1), "n"(J >> 1), "n"(FA), "n"(FB)
                 : "memory");
}

// The scales of one operand for a wave: bytes of its lane's 8 rows, two dwords;
// or, WHOLE, the one byte of its 128 rows.
template <bool WHOLE>
struct ScaleLane {
    typedef uint32_t v2u __attribute__((ext_vector_type(2)));
    const uint8_t *p;    // this lane's first byte in block 0
    int64_t s_blk;
    int shift;           // rows past the last one: bits that the load starts early
    v2u next;
    uint32_t next_one;
    int use[2];
    __device__ inline void init(const Side &s, int row) {
        s_blk = s.s_blk;
        // the last lanes read the last 8 rows' scales and shift them into place
        const int from = min(row, s.rows - 8);
        shift = 8 * min(row - from, 7);
        p = static_cast<const uint8_t *>(s.scales) + (WHOLE ? (int64_t)(min(row, s.rows - 1) >> 7) * s.s_row : from);
    }
    __device__ inline void fetch(int kb) {
        const uint8_t *at = p + kb * s_blk;
        if (WHOLE) next_one = *at;
        else __builtin_memcpy(&next, at, 8);
    }
    __device__ inline void begin() {
        if (WHOLE) {
            use[0] = use[1] = (int)(next_one * 0x01010101u);
        } else {
            const uint64_t v = __builtin_bit_cast(uint64_t, next) >> shift;
            use[0] = (int)v;
            use[1] = (int)(v >> 32);
        }
    }
};

template <int FA, int FB, bool WA, bool WB>
struct ScaledOp {
    ScaleLane<WA> a;
    ScaleLane<WB> b;
    int kblocks, k, lane;
    // (past the last stage: the last one's again, without a branch)
    __device__ inline void fetch(int s) {
        a.fetch(min(s, kblocks - 1));
        b.fetch(min(s, kblocks - 1));
    }
    __device__ inline void begin(int) {
        a.begin();
        b.begin();
        // VALU results before an MFMA of the assembly below reads them
        asm volatile("s_nop 1" : "+v"(a.use[0]), "+v"(a.use[1]), "+v"(b.use[0]), "+v"(b.use[1]));
    }
    static constexpr int kParts = 1;
    template <int I, int J, int P>
    __device__ __forceinline__ void mma(v4f &d, const v8i &x, const v8i &y) {
        mfma_scaled<FA, FB, I & 3, J & 3>(d, x, y, a.use[I >> 2], b.use[J >> 2]);
    }
    // bytes past k in the last stage's fragments (whole chunks past it are zeros
    // already)
    __device__ inline void mask(v8i &f, int s) {
        const int left = k - s * kBlockK - 32 * (lane >> 4);
        if ((k & 15) == 0) return;
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const int n = min(max(left - 4 * d, 0), 4);
            f[d] &= n >= 4 ? -1 : (1 << (8 * n)) - 1;
        }
        asm volatile("s_nop 1" : "+v"(f));
    }
};

struct Fp8Src {
    __amdgpu_buffer_rsrc_t ra, rb;
    int ld_a, ld_b, kbytes;
    __device__ inline __amdgpu_buffer_rsrc_t a(int) const { return ra; }
    __device__ inline __amdgpu_buffer_rsrc_t b(int) const { return rb; }
    __device__ inline int k(int s) const { return s; }
    __device__ inline int left(int s) const { return kbytes - s * kBlockK; }
};

typedef __bf16 v8bf16 __attribute__((ext_vector_type(8)));

// Eight neighbouring outputs of a row, from `col` on: in 16-byte stores where
// all exist and the rows allow it.
__device__ inline void store8(const Fp8Args &g, int row, int col, v8f v) {
    const int n = g.b.rows - col;
    if (row >= g.a.rows || n <= 0) return;
    const int64_t at = row * g.ldc + col;
    if (g.vec && n >= 8) {
        uint16_t *p = static_cast<uint16_t *>(g.C) + at;
        if (g.type == O2M_TYPE_BF16) {
            if (g.accumulate) v += __builtin_convertvector(*reinterpret_cast<const v8bf16 *>(p), v8f);
            *reinterpret_cast<v8bf16 *>(p) = __builtin_convertvector(v, v8bf16);
        } else if (g.type == O2M_TYPE_F16) {
            if (g.accumulate) v += __builtin_convertvector(*reinterpret_cast<const v8f16 *>(p), v8f);
            *reinterpret_cast<v8f16 *>(p) = __builtin_convertvector(v, v8f16);
        } else {
            v8f *q = reinterpret_cast<v8f *>(static_cast<float *>(g.C) + at);
            if (g.accumulate) v += *q;
            *q = v;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) store_out(g.C, at + j, g.type, v[j] + (g.accumulate ? load_out(g.C, at + j, g.type) : 0.0f));
}

template <int FA, int FB, bool WA, bool WB>
__global__ __launch_bounds__(256, 1) void fp8_pipe(Fp8Args g) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kPipeLds];
    const PipeWave w = pipe_wave(lds);
    const TileCoord tc = tile_of(blockIdx.x & 7, blockIdx.x >> 3, g.mt, g.nt, g.chunk, 0);
    if (!tc.valid) return;   // whole workgroup
    const int i0 = tc.ti * kPipeTile, j0 = tc.tj * kPipeTile;
    const Fp8Src src = {rows_of(g.a.values + i0 * g.a.ld, min(kPipeTile, g.a.rows - i0), g.a.ld, g.k),
                        rows_of(g.b.values + j0 * g.b.ld, min(kPipeTile, g.b.rows - j0), g.b.ld, g.k), (int)g.a.ld,
                        (int)g.b.ld, g.k};
    ScaledOp<FA, FB, WA, WB> op;
    op.kblocks = g.kblocks;
    op.k = g.k;
    op.lane = w.lane;
    const int q = w.lane & 15;
    op.a.init(g.a, i0 + w.row_a + 8 * q);
    op.b.init(g.b, j0 + w.row_b + 8 * q);
    v4f acc[8][8];
    pipe_run(w, op, src, g.kblocks, acc);
    pipe_results<false>(w, acc, [&](int row, int col, const v8f &v) { store8(g, i0 + row, j0 + col, v); });
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

// The kernel of one launch.  Large tiles feed the MFMA pipe best and take products
// with enough of them to go round; they read the scales of 8 rows at once.
bool takes_pipe(const Fp8Args &g) {
    auto fits = [](const Side &s) { return !s.by_row || (s.s_row == 1 && s.rows >= 8); };
    return g.type != O2M_TYPE_F32 && g.a.pow2 && fits(g.a) && fits(g.b) &&
           ceil_div(g.a.rows, kPipeTile) * ceil_div(g.b.rows, kPipeTile) >= 32;
}

template <int FA, int FB>
hipError_t launch_formats(Fp8Args &g, hipStream_t st) {
    if (takes_pipe(g)) {
        g.mt = (int)ceil_div(g.a.rows, kPipeTile);
        g.nt = (int)ceil_div(g.b.rows, kPipeTile);
        const int64_t chunk = ceil_div((int64_t)g.mt * g.nt, kXcds);
        if (kXcds * chunk > 0x7FFFFFFF) return hipErrorInvalidValue;
        g.chunk = (int)chunk;
        const unsigned grid = (unsigned)(kXcds * chunk);
        if (g.a.by_row && g.b.by_row) fp8_pipe<FA, FB, false, false><<<grid, 256, 0, st>>>(g);
        else if (g.a.by_row) fp8_pipe<FA, FB, false, true><<<grid, 256, 0, st>>>(g);
        else if (g.b.by_row) fp8_pipe<FA, FB, true, false><<<grid, 256, 0, st>>>(g);
        else fp8_pipe<FA, FB, true, true><<<grid, 256, 0, st>>>(g);
        return hipGetLastError();
    }
    // these write the first operand's rows contiguously
    Fp8Args t = g;
    t.a = g.b;
    t.b = g.a;
    t.mt = (int)ceil_div(t.a.rows, 128);
    t.nt = (int)ceil_div(t.b.rows, 128);
    const int64_t tiles = (int64_t)t.mt * t.nt;
    if (tiles > 0x7FFFFFFF) return hipErrorInvalidValue;
    const unsigned grid = (unsigned)tiles;
    if (g.type == O2M_TYPE_F32) fp8_tile<kWide, FB, FA><<<grid, 256, 0, st>>>(t);
    else if (g.a.pow2) fp8_tile<kScaled, FB, FA><<<grid, 256, 0, st>>>(t);
    else fp8_tile<kPartial, FB, FA><<<grid, 256, 0, st>>>(t);
    return hipGetLastError();
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
    g.C = C;
    g.ldc = ldc;
    g.type = type;
    g.accumulate = accumulate;
    const int size = type == O2M_TYPE_F32 ? 4 : 2;
    g.vec = reinterpret_cast<uintptr_t>(C) % 16 == 0 && ldc * size % 16 == 0;
    switch (A.format * 2 + B.format) {
    case 0: return launch_formats<0, 0>(g, st);
    case 1: return launch_formats<0, 1>(g, st);
    case 2: return launch_formats<1, 0>(g, st);
    default: return launch_formats<1, 1>(g, st);
    }
}

}  // namespace o2m
