// The pipeline of the large product tiles: 256 x 256 (N = 8) or 256 x 128 (N = 4)
// outputs per workgroup of 4 waves (one per SIMD, 2 x 2), each wave 128 x 16 N = 8 x
// N accumulators of 16 x 16 held in accumulation registers.
//
// Operands arrive in k-stages of 128 bytes a row (mfma_tiles.h), two stage
// buffers of 64 KB or three of 48 KB.  One wave per SIMD leaves nothing else to
// feed the MFMA pipe, so every memory instruction is placed between MFMAs by
// hand: a wave holds the stage's whole B strip (N fragments) in registers, streams
// A's fragments one or two ahead, and reads the next stage's B strip during the
// second half of a stage.  What a stage has left in LDS is refilled as soon as it
// is free: its B strip at the stage's start (it is in registers by then), the
// first half of its A strip in the middle, the second half at the end, so that
// with two buffers every copy has one to one and a half stages of 2048 cycles of
// MFMAs to land, with three two to two and a half of 1024.
//
// The larger tile reads 16 fragments for 64 blocks, the smaller 12 for 32, which
// is all that LDS can give (144 KB a stage with the copies, 1150 cycles at 128
// bytes, beside 1024 of MFMAs): it is for products that would leave CUs idle.
//
// Rows.  Fragment i of a wave holds rows 8 q + i of A, fragment j rows N q + j of
// B, q = lane % 16, rather than 16 consecutive ones.  A lane then owns 8 and N
// consecutive rows, whose e8m0 scales are one load, and N consecutive columns
// (and 32 consecutive rows) of the output, which leave as 8- or 16-byte stores in
// either direction.  In LDS the rows of i = 0..3 come first (the half that is free
// first), 4 rows of each q together, in pairs exchanged for q >= 8; chunk c of a row
// lies in slot c ^ (q & 7).  The 16 chunks that 16 lanes of a fragment read at a
// time then fill all 64 banks once.
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

constexpr int kPipeTile = 256;                     // rows of A
constexpr int kHalfBytes = 128 * kStageRowBytes;   // half of A's stage
constexpr int kABytes = 2 * kHalfBytes;

template <int N>
struct PipeShape {
    static_assert(N == 8 || N == 4, "B fragments of a wave");
    static constexpr int kTn = 32 * N;                     // rows of B
    static constexpr int kBuffers = N == 8 ? 2 : 3;
    static constexpr int kStage = kABytes + kTn * kStageRowBytes;
    static constexpr int kLds = kBuffers * kStage;
    static constexpr int kAhead = N == 8 ? 1 : 2;          // A fragments read ahead
    // copies of a wave that may be in flight where a stage begins and in its middle
    static constexpr int kFlying = (kBuffers - 1) * (8 + N) - 4;
};

// One wave's place.
struct PipeWave {
    uint8_t *lds;
    int lane, wave;       // wave: uniform
    int row_a, row_b;     // its first row of A and B within the tile
    int chunk16;          // copies: the lane's byte within the stage row
    int copy_a, copy_b;   // copies: the lane's row within the tile, first copy
    int pair;             // and how far its row of the odd copies is from there
    int frag_a[2], frag_b[2];   // reads: the lane's byte of fragment 0 within a stage,
                                // for the even and the odd fragments
};

template <int N>
__device__ inline PipeWave pipe_wave(uint8_t *lds) {
    PipeWave w;
    w.lds = lds;
    w.lane = threadIdx.x & 63;
    w.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    w.row_a = (w.wave >> 1) * 128;
    w.row_b = (w.wave & 1) * 16 * N;
    const int lr = w.lane >> 3, slot = w.lane & 7;
    const int q = 2 * w.wave + (lr >> 2);              // of the first copy; + 8 per copy
    w.chunk16 = (slot ^ (q & 7)) << 4;
    w.copy_a = 8 * q + (lr & 3);
    w.copy_b = N * q + (lr & 3);
    w.pair = lr & 1 ? -1 : 1;                          // q >= 8 (mod 16) in the odd copies
    const int fq = w.lane & 15, c = 2 * (w.lane >> 4);
    const int at = 4 * fq * kStageRowBytes + ((c ^ (fq & 7)) << 4);
    const int swap = fq >> 3 ? kStageRowBytes : 0;
    w.frag_a[0] = at + w.row_a / 2 * kStageRowBytes + swap;   // 4 LDS rows per 8 rows, in each half
    w.frag_a[1] = w.frag_a[0] - 2 * swap;
    w.frag_b[0] = at + (N == 8 ? w.row_b / 2 : w.row_b) * kStageRowBytes + kABytes + swap;
    w.frag_b[1] = w.frag_b[0] - 2 * swap;
    return w;
}

// Copy t of half h of A's stage (t < 4), or of B's with N = 8; with N = 4 there are no
// halves.  The stage lies `at` bytes from the descriptor's start; `left`: the
// operand's bytes from there on, none are read past them (left <= 0: zeros).
__device__ inline void pipe_copy(const PipeWave &w, __amdgpu_buffer_rsrc_t r, int row, int ld, int at, int left, uint8_t *dst,
                                 int h, int t) {
    int off = row * ld + w.chunk16;
    if (left < kStageRowBytes) off = w.chunk16 < left ? off : 0x7FFFFFF0;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr *)(dst + h * kHalfBytes + (4 * t + w.wave) * 1024), 16, off,
                                             left > 0 ? at : 0, 0, 0);
}

// Fragment i of the strip at `strip`, in halves or not: 32 bytes a lane.
template <bool HALVES>
__device__ inline v8i pipe_fragment(const uint8_t *buf, const int (&strip)[2], int i) {
    const int at = strip[i & 1];
    const uint8_t *p = buf + (HALVES ? (i >> 2) * kHalfBytes : 0) + (i & 3) * kStageRowBytes;
    const v4i lo = *reinterpret_cast<const v4i *>(p + at);
    const v4i hi = *reinterpret_cast<const v4i *>(p + (at ^ 16));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// The accumulators between their last MFMA and the epilogue's reads: 16 passes
// and more, each asm holding a row of them so that no access moves across.
template <int N>
__device__ inline void pipe_row(v4f (&a)[N], bool zeroed) {
    if constexpr (N == 8) {
        if (zeroed)
            asm volatile("s_nop 4" : "+a"(a[0]), "+a"(a[1]), "+a"(a[2]), "+a"(a[3]), "+a"(a[4]), "+a"(a[5]), "+a"(a[6]), "+a"(a[7]));
        else
            asm volatile("s_nop 7\n s_nop 7\n s_nop 7"
                         : "+a"(a[0]), "+a"(a[1]), "+a"(a[2]), "+a"(a[3]), "+a"(a[4]), "+a"(a[5]), "+a"(a[6]), "+a"(a[7]));
    } else {
        if (zeroed) asm volatile("s_nop 4" : "+a"(a[0]), "+a"(a[1]), "+a"(a[2]), "+a"(a[3]));
        else asm volatile("s_nop 7\n s_nop 7\n s_nop 7" : "+a"(a[0]), "+a"(a[1]), "+a"(a[2]), "+a"(a[3]));
    }
}
template <int N>
__device__ inline void pipe_settle(v4f (&acc)[8][N]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) pipe_row<N>(acc[i], false);
}
template <int N>
__device__ inline void pipe_zero(v4f (&acc)[8][N]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[i][j] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) pipe_row<N>(acc[i], true);
}

// The product of `stages` stages into acc, which is zeroed here.  Src gives the
// operands of a stage: a(s), b(s) descriptors, at_a(s), at_b(s) its place in them,
// left(s) the bytes from there on (<= 0 for s >= stages), ld_a, ld_b; Op the arithmetic:
// fetch(s) asks for what stage s needs besides (it may issue any number of
// loads), begin(s) takes it into use, mma<i, j, p>(acc[i][j], a, b) multiplies, in
// kParts MFMAs of 8 blocks' distance to each other, and mask(f, s) clears what the last stage's fragments hold past the rows' ends.
//
// Waits.  With S buffers the copies of a wave are issued in the order
//   .. B(s) A0(s) | A1(s) B(s+1) A0(s+1) | ..
// (A0, A1: the 4 copies of a half, B: N), those of a bar to the next during one
// stage, S - 1 stages before the stage they belong to: where stage s begins, all
// but the last kFlying have landed, so A1(s) has, and in its middle again all but
// kFlying, so B(s+1) and A0(s+1) have.  Loads of fetch() in between only make a
// wait stricter.
template <int N, class Op, class Src>
__device__ inline void pipe_run(const PipeWave &w, Op &op, const Src &src, int stages, v4f (&acc)[8][N]) {
    typedef PipeShape<N> T;
    constexpr int P = Op::kParts, S = T::kBuffers, D = T::kAhead, R = 2 * D;
    int turn = 0;   // the current stage % S
    auto buffer = [&](int d) {   // of the stage d (<= S) after the current one
        const int u = turn + d;
        return w.lds + (u >= S ? u - S : u) * T::kStage;
    };
    auto copy_a = [&](int s, uint8_t *buf, int h, int t) {
        pipe_copy(w, src.a(s), w.copy_a + (t & 1 ? w.pair : 0) + 64 * t + 4 * h, src.ld_a, src.at_a(s), src.left(s), buf, h, t);
    };
    auto copy_b = [&](int s, uint8_t *buf, int c) {
        const int h = N == 8 ? c >> 2 : 0, t = N == 8 ? c & 3 : c;
        pipe_copy(w, src.b(s), w.copy_b + (t & 1 ? w.pair : 0) + 8 * N * t + 4 * h, src.ld_b, src.at_b(s), src.left(s), buf + kABytes, h, t);
    };
    auto fragment_a = [&](const uint8_t *buf, int i) { return pipe_fragment<true>(buf, w.frag_a, i); };
    auto fragment_b = [&](const uint8_t *buf, int j) { return pipe_fragment<N == 8>(buf, w.frag_b, j); };
    op.fetch(0);   // before the copies, so that its wait is none of theirs
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
        for (int c = 0; c < N; ++c) copy_b(s, buffer(s), c);
#pragma unroll
        for (int t = 0; t < 4; ++t) copy_a(s, buffer(s), 0, t);
        if (s + 1 < S)
#pragma unroll
            for (int t = 0; t < 4; ++t) copy_a(s, buffer(s), 1, t);
    }
    __builtin_amdgcn_sched_barrier(0);
    pipe_zero<N>(acc);
    wait_vmem<T::kFlying>();
    lds_barrier();
    v8i b0[N], b1[N], a[R];
#pragma unroll
    for (int j = 0; j < N; ++j) b0[j] = fragment_b(buffer(0), j);
#pragma unroll
    for (int i = 0; i < D; ++i) a[i] = fragment_a(buffer(0), i);

    auto stage = [&](int s, v8i(&bc)[N], v8i(&bn)[N]) {
        const uint8_t *cur = buffer(0), *next = buffer(1);
        uint8_t *after = buffer(S - 1), *same = buffer(S);   // of stages s + S - 1 and s + S
        wait_vmem<T::kFlying>();
        lds_barrier();
        op.begin(s);
        op.fetch(s + 1);
        // the blocks of i = 0..3, kParts MFMAs each; m counts blocks' worth of MFMAs,
        // after which the memory instructions follow
        each<4 * N * P>([&](auto I) {
            constexpr int t = I, i = t / (N * P), p = t / N % P, j = (i & 1) ? N - 1 - t % N : t % N;
            constexpr int m = t / P, c = m >> 1;
            if constexpr (t % (N * P) == 0) a[(i + D) % R] = fragment_a(cur, i + D);
            op.template mma<i, j, p>(acc[i][j], a[i % R], bc[j]);
            if constexpr (t % P == P - 1) {
                if constexpr ((m & 1) && c < 4) copy_a(s + S - 1, after, 1, c);
                if constexpr ((m & 1) && c >= 4 && c < 4 + N) copy_b(s + S, same, c - 4);
            }
        });
        wait_vmem<T::kFlying>();
        lds_barrier();
        each<4 * N * P>([&](auto I) {
            constexpr int t = I, i = 4 + t / (N * P), p = t / N % P, j = (i & 1) ? N - 1 - t % N : t % N;
            constexpr int m = t / P;
            if constexpr (t % (N * P) == 0)
                a[(i + D) % R] = i + D < 8 ? fragment_a(cur, i + D) : fragment_a(next, i + D - 8);
            op.template mma<i, j, p>(acc[i][j], a[i % R], bc[j]);
            if constexpr (t % P == P - 1) {
                // (the last of these reads well before the barrier that waits for it)
                if constexpr (m % 3 == 1 && m / 3 < N) bn[m / 3] = fragment_b(next, m / 3);
                if constexpr (m % N == 3) copy_a(s + S, same, 0, m / N);
            }
        });
        turn = turn + 1 == S ? 0 : turn + 1;
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
        for (int j = 0; j < N; ++j) b0[j] = b1[j];
    }
    // the last stage: A1 has to land, nothing follows
    wait_vmem<T::kFlying>();
    lds_barrier();
    op.begin(s);
    const uint8_t *cur = buffer(0);
#pragma unroll
    for (int j = 0; j < N; ++j) op.mask(b0[j], s);
    each<8>([&](auto I) {
        constexpr int i = I;
        if constexpr (i + D < 8) a[(i + D) % R] = fragment_a(cur, i + D);
        op.mask(a[i % R], s);
        each<N * P>([&](auto J) {
            constexpr int j = J % N;
            op.template mma<i, j, J / N>(acc[i][j], a[i % R], b0[j]);
        });
    });
    wait_vmem<0>();
    pipe_settle<N>(acc);
}

// out(row, col, v): N neighbouring outputs of a row of the wave's 128 x 16 N, for
// all of them; or, ACROSS, 8 neighbouring ones of a column, from `row` on.  The
// accumulators go to LDS straight from their registers and each lane reads its
// own back, 8 x 4 or N x 4 outputs at a time: read as values from a program they
// would all be copied at once, into scratch memory.  (The round trip is some 2% of
// a tile of 64 stages.)
template <bool ACROSS, int N, class Out>
__device__ inline void pipe_results(const PipeWave &w, const v4f (&acc)[8][N], Out out) {
    // lines of 8 or N blocks (of one j or i), as many at a time as 32 KB a wave hold
    constexpr int kLen = ACROSS ? 8 : N, kLines = ACROSS ? N : 8, kAtOnce = 32 / kLen < kLines ? 32 / kLen : kLines;
    typedef float V __attribute__((ext_vector_type(kLen)));
    uint8_t *mine = w.lds + w.wave * (32 * 1024) + w.lane * 16;
    lds_barrier();   // every wave is done with the stages
    const int row0 = w.row_a + 32 * (w.lane >> 4), col0 = w.row_b + N * (w.lane & 15);
    each<kLines / kAtOnce>([&](auto H) {
        each<kAtOnce>([&](auto I) {
            each<kLen>([&](auto J) {
                constexpr int l = H * kAtOnce + I;
                *reinterpret_cast<v4f *>(mine + (I * kLen + J) * 1024) = acc[ACROSS ? (int)J : l][ACROSS ? l : (int)J];
            });
        });
#pragma unroll 1
        for (int i = 0; i < kAtOnce; ++i) {
            v4f u[kLen];
#pragma unroll
            for (int j = 0; j < kLen; ++j) u[j] = *reinterpret_cast<const v4f *>(mine + (i * kLen + j) * 1024);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                V v;
#pragma unroll
                for (int j = 0; j < kLen; ++j) v[j] = u[j][e];
                const int l = H * kAtOnce + i;
                if (ACROSS) out(row0 + 8 * e, col0 + l, v);
                else out(row0 + 8 * e + l, col0, v);
            }
        }
    });
}

}  // namespace o2m
