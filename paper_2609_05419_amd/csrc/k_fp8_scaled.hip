// 8-bit block-scaled products with power-of-two scales and 16-bit results: the
// scaled MFMA applies them, so that nothing but MFMAs and the feeding of them is
// left.  Large products take the pipeline of mfma_pipe.h (8192^3 393 us, 2.8
// PFLOP/s), 256 x 256 or 256 x 128, small ones tiles of 128 x 128
// and 64 x 64.
#include "fp8_tile.h"

namespace o2m {
namespace {

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

// The scales of one operand for a wave: bytes of its lane's N (8 or 4) rows, in
// dwords; or, WHOLE, the one byte of its rows.
template <bool WHOLE, int N>
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
        // the last lanes read the last N rows' scales and shift them into place
        const int from = min(row, s.rows - N);
        shift = 8 * min(row - from, N - 1);
        p = static_cast<const uint8_t *>(s.scales) + (WHOLE ? (int64_t)(min(row, s.rows - 1) >> 7) * s.s_row : from);
    }
    __device__ inline void fetch(int kb) {
        const uint8_t *at = p + kb * s_blk;
        if (WHOLE) next_one = *at;
        else if (N == 8) __builtin_memcpy(&next, at, 8);
        else __builtin_memcpy(&next_one, at, 4);
    }
    __device__ inline void begin() {
        if (WHOLE) {
            use[0] = use[1] = (int)(next_one * 0x01010101u);
        } else if (N == 4) {
            use[0] = (int)(next_one >> shift);
        } else {
            const uint64_t v = __builtin_bit_cast(uint64_t, next) >> shift;
            use[0] = (int)v;
            use[1] = (int)(v >> 32);
        }
    }
};

template <int FA, int FB, bool WA, bool WB, int N>
struct ScaledOp {
    ScaleLane<WA, 8> a;
    ScaleLane<WB, N> b;
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
        asm volatile("s_nop 1" : "+v"(a.use[0]), "+v"(a.use[1]), "+v"(b.use[0]));
        if constexpr (N == 8) asm volatile("s_nop 1" : "+v"(b.use[1]));
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
    __device__ inline int at_a(int s) const { return s * kStageRowBytes; }
    __device__ inline int at_b(int s) const { return s * kStageRowBytes; }
    __device__ inline int left(int s) const { return kbytes - s * kBlockK; }
};

template <int FA, int FB, bool WA, bool WB, int N>
__global__ __launch_bounds__(256, 1) void fp8_pipe(Fp8Args g) {
    typedef PipeShape<N> T;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[T::kLds];
    const PipeWave w = pipe_wave<N>(lds);
    const TileCoord tc = tile_of(blockIdx.x & 7, blockIdx.x >> 3, g.mt, g.nt, g.chunk, 0);
    if (!tc.valid) return;   // whole workgroup
    const int i0 = tc.ti * kPipeTile, j0 = tc.tj * T::kTn;
    const Fp8Src src = {rows_of(g.a.values + i0 * g.a.ld, min(kPipeTile, g.a.rows - i0), g.a.ld, g.k),
                        rows_of(g.b.values + j0 * g.b.ld, min(T::kTn, g.b.rows - j0), g.b.ld, g.k), (int)g.a.ld,
                        (int)g.b.ld, g.k};
    ScaledOp<FA, FB, WA, WB, N> op;
    op.kblocks = g.kblocks;
    op.k = g.k;
    op.lane = w.lane;
    const int q = w.lane & 15;
    op.a.init(g.a, i0 + w.row_a + 8 * q);
    op.b.init(g.b, j0 + w.row_b + N * q);
    v4f acc[8][N];
    pipe_run<N>(w, op, src, g.kblocks, acc);
    pipe_results<false, N>(w, acc, [&](int row, int col, const auto &v) { store_run<N>(g, i0 + row, j0 + col, v); });
}

template <int FA, int FB, int N>
hipError_t launch_pipe(Fp8Args &g, hipStream_t st) {
    g.mt = (int)ceil_div(g.a.rows, kPipeTile);
    g.nt = (int)ceil_div(g.b.rows, PipeShape<N>::kTn);
    const int64_t chunk = ceil_div((int64_t)g.mt * g.nt, kXcds);
    if (!launch_fits(kXcds * chunk, 256)) return hipErrorInvalidValue;
    g.chunk = (int)chunk;
    const unsigned grid = (unsigned)(kXcds * chunk);
    if (g.a.by_row && g.b.by_row) fp8_pipe<FA, FB, false, false, N><<<grid, 256, 0, st>>>(g);
    else if (g.a.by_row) fp8_pipe<FA, FB, false, true, N><<<grid, 256, 0, st>>>(g);
    else if (g.b.by_row) fp8_pipe<FA, FB, true, false, N><<<grid, 256, 0, st>>>(g);
    else fp8_pipe<FA, FB, true, true, N><<<grid, 256, 0, st>>>(g);
    return hipGetLastError();
}

template <int FA, int FB>
hipError_t launch(Fp8Args &g, TileSize size, hipStream_t st) {
    return size == k256 ? launch_pipe<FA, FB, 8>(g, st) : size == k256x128 ? launch_pipe<FA, FB, 4>(g, st)
                                                                          : launch_sizes<kScaled, FA, FB, false>(g, size, st);
}

}  // namespace

hipError_t launch_fp8_scaled(Fp8Args &g, int format, TileSize size, hipStream_t st) {
    switch (format) {
    case 0: return launch<0, 0>(g, size, st);
    case 1: return launch<0, 1>(g, size, st);
    case 2: return launch<1, 0>(g, size, st);
    default: return launch<1, 1>(g, size, st);
    }
}

}  // namespace o2m
