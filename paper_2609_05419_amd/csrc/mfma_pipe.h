// The pipeline of the large product tile: 256 x 256 outputs per workgroup of 4
// waves (one per SIMD, 2 x 2), each wave 128 x 128 = 8 x 8 accumulators of 16 x
// 16 held in its 256 accumulation registers.
//
// Operands arrive in k-stages of 128 bytes a row (mfma_tiles.h), two stage
// buffers of 64 KB.  One wave per SIMD leaves nothing else to feed the MFMA
// pipe, so every memory instruction is placed between MFMAs by hand: a wave
// holds the stage's whole B strip (8 fragments) in registers, streams A's
// fragments one ahead, and reads the next stage's B strip during the second half
// of a stage.  What a stage has left in LDS is refilled as soon as it is free:
// its B strip at the stage's start (it is in registers by then), the first half
// of its A strip in the middle, the second half at the end, so that with two
// buffers every copy has one to one and a half stages (some 2000 to 3000
// cycles) to land.
//
// Rows.  Fragment i of a wave holds rows 8 q + i, q = lane % 16, rather than 16
// consecutive ones.  A lane then owns 8 consecutive rows of each operand, whose
// 8 e8m0 scales are one load, and 8 consecutive columns (and 32 consecutive
// rows) of the output, which leave as 16-byte stores in either direction.  In
// LDS the rows of i = 0..3 come first (the half that is free first), 4 rows of
// each q together; chunk c of a row lies in slot c ^ (q & 7), which spreads a
// fragment's lanes over the banks.
#pragma once

#include "mfma_tiles.h"

#include <type_traits>
#include <utility>

namespace o2m {

// f(0), f(1), .. f(N - 1) with the index as a compile-time constant.
template <class F, int... I>
__device__ __forceinline__ void each_of(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>()), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F &&f) {
    each_of(f, std::make_integer_sequence<int, N>());
}

typedef float v8f __attribute__((ext_vector_type(8)));

constexpr int kPipeTile = 256;
constexpr int kHalfBytes = 128 * kStageRowBytes;   // half an operand's stage
constexpr int kOperandBytes = 2 * kHalfBytes;
constexpr int kPipeStage = 2 * kOperandBytes;      // A and B
constexpr int kPipeLds = 2 * kPipeStage;

// One wave's place.
struct PipeWave {
    uint8_t *lds;
    int lane, wave;       // wave: uniform
    int row_a, row_b;     // its first row of A and B within the tile
    int chunk16;          // copies: the lane's byte within the stage row
    int copy_row;         // copies: the lane's row within the tile, first copy
    int frag_a, frag_b;   // reads: the lane's byte of fragment 0 within a stage
};

__device__ inline PipeWave pipe_wave(uint8_t *lds) {
    PipeWave w;
    w.lds = lds;
    w.lane = threadIdx.x & 63;
    w.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    w.row_a = (w.wave >> 1) * 128;
    w.row_b = (w.wave & 1) * 128;
    const int lr = w.lane >> 3, slot = w.lane & 7;
    const int q = 2 * w.wave + (lr >> 2);              // of the first copy; + 8 per copy
    w.chunk16 = (slot ^ (q & 7)) << 4;
    w.copy_row = 8 * q + (lr & 3);
    const int fq = w.lane & 15, c = 2 * (w.lane >> 4);
    const int at = 4 * fq * kStageRowBytes + ((c ^ (fq & 7)) << 4);
    w.frag_a = at + w.row_a / 2 * kStageRowBytes;      // 4 LDS rows per 8 rows, in each half
    w.frag_b = at + w.row_b / 2 * kStageRowBytes + kOperandBytes;
    return w;
}

// Copy t (0..3) of half h of an operand's stage, which lies `at` bytes from the
// descriptor's start: 64 t + 4 h rows on.  `left`: the operand's bytes from there on; none are read past them (left <= 0: zeros).
__device__ inline void pipe_copy(const PipeWave &w, __amdgpu_buffer_rsrc_t r, int ld, int at, int left, uint8_t *dst,
                                 int h, int t) {
    int off = (w.copy_row + 64 * t + 4 * h) * ld + w.chunk16;
    if (left < kStageRowBytes) off = w.chunk16 < left ? off : 0x7FFFFFF0;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr *)(dst + h * kHalfBytes + (4 * t + w.wave) * 1024), 16, off,
                                             left > 0 ? at : 0, 0, 0);
}

// Fragment i of the strip at `at`: 32 bytes a lane.
__device__ inline v8i pipe_fragment(const uint8_t *buf, int at, int i) {
    const uint8_t *p = buf + (i >> 2) * kHalfBytes + (i & 3) * kStageRowBytes;
    const v4i lo = *reinterpret_cast<const v4i *>(p + at);
    const v4i hi = *reinterpret_cast<const v4i *>(p + (at ^ 16));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// The accumulators between their last MFMA and the epilogue's reads: 16 passes
// and more, each asm holding a row of them so that no access moves across.
__device__ inline void pipe_settle(v4f (&acc)[8][8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        asm volatile("s_nop 7\n s_nop 7\n s_nop 7" : "+a"(acc[i][0]), "+a"(acc[i][1]), "+a"(acc[i][2]),
                     "+a"(acc[i][3]), "+a"(acc[i][4]), "+a"(acc[i][5]), "+a"(acc[i][6]), "+a"(acc[i][7]));
}
__device__ inline void pipe_zero(v4f (&acc)[8][8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        asm volatile("s_nop 4" : "+a"(acc[i][0]), "+a"(acc[i][1]), "+a"(acc[i][2]), "+a"(acc[i][3]),
                     "+a"(acc[i][4]), "+a"(acc[i][5]), "+a"(acc[i][6]), "+a"(acc[i][7]));
}

// The product of `stages` stages into acc, which is zeroed here.  Src gives the
// operands of a stage: a(s), b(s) descriptors, at_a(s), at_b(s) its place in them,
// left(s) the bytes from there on (<= 0 for s >= stages), ld_a, ld_b; Op the arithmetic:
// fetch(s) asks for what stage s needs besides (it may issue any number of
// loads), begin(s) takes it into use, mma<i, j, p>(acc[i][j], a, b) multiplies, in
// kParts MFMAs of 8 blocks' distance to each other, and mask(f, s) clears what the last stage's fragments hold past the rows' ends.
//
// Waits.  The copies of a wave are issued in the order .. A1(s) B(s+1) | A0(s+1) |
// A1(s+1) B(s+2) | A0(s+2) .. (A0, A1: 4 copies of a half, B: 8), a bar being a
// barrier: at the start of stage s all but the last 12 have landed, so A1(s) has,
// and in the middle again all but 12, so B(s+1) and A0(s+1) have.  Loads of
// fetch() in between only make a wait stricter.
template <class Op, class Src>
__device__ inline void pipe_run(const PipeWave &w, Op &op, const Src &src, int stages, v4f (&acc)[8][8]) {
    constexpr int P = Op::kParts;
    auto buffer = [&](int s) { return w.lds + (s & 1) * kPipeStage; };
    auto copy_a = [&](int s, int h, int t) {
        pipe_copy(w, src.a(s), src.ld_a, src.at_a(s), src.left(s), buffer(s), h, t);
    };
    auto copy_b = [&](int s, int c) {
        pipe_copy(w, src.b(s), src.ld_b, src.at_b(s), src.left(s), buffer(s) + kOperandBytes, c >> 2, c & 3);
    };
    op.fetch(0);   // before the copies, so that its wait is none of theirs
#pragma unroll
    for (int t = 0; t < 4; ++t) copy_a(0, 0, t);
#pragma unroll
    for (int c = 0; c < 8; ++c) copy_b(0, c);
#pragma unroll
    for (int t = 0; t < 4; ++t) copy_a(0, 1, t);
#pragma unroll
    for (int c = 0; c < 8; ++c) copy_b(1, c);
#pragma unroll
    for (int t = 0; t < 4; ++t) copy_a(1, 0, t);
    __builtin_amdgcn_sched_barrier(0);
    pipe_zero(acc);
    wait_vmem<12>();
    lds_barrier();
    v8i b0[8], b1[8], a[2];
#pragma unroll
    for (int j = 0; j < 8; ++j) b0[j] = pipe_fragment(buffer(0), w.frag_b, j);
    a[0] = pipe_fragment(buffer(0), w.frag_a, 0);

    auto stage = [&](int s, v8i(&bc)[8], v8i(&bn)[8]) {
        const uint8_t *cur = buffer(s), *next = buffer(s + 1);
        wait_vmem<12>();
        lds_barrier();
        op.begin(s);
        op.fetch(s + 1);
        // the 32 blocks of i = 0..3, kParts MFMAs each; m counts blocks' worth of
        // MFMAs, after which the memory instructions follow
        each<32 * P>([&](auto T) {
            constexpr int t = T, i = t / (8 * P), p = t / 8 % P, j = (i & 1) ? 7 - (t & 7) : t & 7;
            constexpr int m = t / P, c = m >> 1;
            if constexpr (t % (8 * P) == 0) a[(i + 1) & 1] = pipe_fragment(cur, w.frag_a, i + 1);
            op.template mma<i, j, p>(acc[i][j], a[i & 1], bc[j]);
            if constexpr (t % P == P - 1) {
                if constexpr ((m & 1) && c < 4) copy_a(s + 1, 1, c);
                if constexpr ((m & 1) && c >= 4 && c < 12) copy_b(s + 2, c - 4);
            }
        });
        wait_vmem<12>();
        lds_barrier();
        each<32 * P>([&](auto T) {
            constexpr int t = T, i = 4 + t / (8 * P), p = t / 8 % P, j = (i & 1) ? 7 - (t & 7) : t & 7;
            constexpr int m = t / P;
            if constexpr (t % (8 * P) == 0)
                a[(i + 1) & 1] = i < 7 ? pipe_fragment(cur, w.frag_a, i + 1) : pipe_fragment(next, w.frag_a, 0);
            op.template mma<i, j, p>(acc[i][j], a[i & 1], bc[j]);
            if constexpr (t % P == P - 1) {
                if constexpr ((m & 3) == 1) bn[m >> 2] = pipe_fragment(next, w.frag_b, m >> 2);
                if constexpr ((m & 7) == 3) copy_a(s + 2, 0, m >> 3);
            }
        });
    };
    int s = 0;
    for (; s + 2 < stages; s += 2) {
        stage(s, b0, b1);
        stage(s + 1, b1, b0);
    }
    if (s + 1 < stages) {
        stage(s, b0, b1);
        ++s;
#pragma unroll
        for (int j = 0; j < 8; ++j) b0[j] = b1[j];
    }
    // the last stage: A1 has to land, nothing follows
    wait_vmem<12>();
    lds_barrier();
    op.begin(s);
    const uint8_t *cur = buffer(s);
#pragma unroll
    for (int j = 0; j < 8; ++j) op.mask(b0[j], s);
    each<8>([&](auto I) {
        constexpr int i = I;
        if constexpr (i < 7) a[(i + 1) & 1] = pipe_fragment(cur, w.frag_a, i + 1);
        op.mask(a[i & 1], s);
        each<8 * P>([&](auto J) {
            constexpr int j = J & 7;
            op.template mma<i, j, J / 8>(acc[i][j], a[i & 1], b0[j]);
        });
    });
    wait_vmem<0>();
    pipe_settle(acc);
}

// out(row, col, v): 8 neighbouring outputs of a row of the wave's 128 x 128, for
// all of them; or, ACROSS, 8 neighbouring ones of a column, from `row` on.  The
// accumulators go to LDS straight from their registers and each lane reads its
// own back, 8 x 4 outputs at a time: read as values from a program they would
// all be copied at once, into scratch memory.  (The round trip is some 2% of a
// tile of 64 stages.)
template <bool ACROSS, class Out>
__device__ inline void pipe_results(const PipeWave &w, const v4f (&acc)[8][8], Out out) {
    uint8_t *mine = w.lds + w.wave * (kPipeLds / 4) + w.lane * 16;
    lds_barrier();   // every wave is done with the stages
    each<2>([&](auto H) {
        each<4>([&](auto I) {
            each<8>([&](auto J) {
                *reinterpret_cast<v4f *>(mine + (I * 8 + J) * 1024) = ACROSS ? acc[J][4 * H + I] : acc[4 * H + I][J];
            });
        });
        const int row0 = w.row_a + 32 * (w.lane >> 4), col0 = w.row_b + 8 * (w.lane & 15);
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
            v4f u[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = *reinterpret_cast<const v4f *>(mine + (i * 8 + j) * 1024);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const v8f v = {u[0][e], u[1][e], u[2][e], u[3][e], u[4][e], u[5][e], u[6][e], u[7][e]};
                if (ACROSS) out(row0 + 8 * e, col0 + 4 * H + i, v);
                else out(row0 + 8 * e + 4 * H + i, col0, v);
            }
        }
    });
}

}  // namespace o2m
