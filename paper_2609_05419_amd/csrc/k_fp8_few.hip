// Products of 8-bit block-scaled operands with few rows on one side (tokens that
// are decoded), and the linear layer of them in one launch.
//
// Bound: memory, the reading of the long operand W (n k bytes).  A workgroup owns
// 16 rows of W, whose blocks of 128 its waves take in turn straight from memory
// into MFMA fragments, several blocks ahead; nothing is shared, so there is
// nothing to stage.  The tokens are the other side of the MFMA, 16 at a time.  All
// products are summed exactly in fp16 MFMAs with fp32 sums (k_fp8.hip says why
// that matters), which costs nothing here.  The waves' sums are joined in LDS in a
// fixed order.
//
// Tokens of up to 16 KB in 8 bits (two of 8192 entries, 16 of 1024) are quantized by
// each workgroup for itself: reading them again is some 2% of reading W a token,
// from the cache, and a launch of its own would cost as much as 20 MB of W.
//
// 1 x 8192 x 8192 16.2 us (67 MB at 4.1 TB/s; a large copy moves 4.9).
#include "fp8_operand.h"
#include "fp8_round.h"

namespace o2m {
namespace {

constexpr int kAhead = 4;          // blocks of W in flight per wave
constexpr int kFusedBytes = 16384;   // quantized tokens kept in LDS

struct FewArgs {
    Side w, x;          // x.rows: tokens
    int k, kblocks;
    const void *X;      // FUSED: unquantized tokens
    int64_t ldx;
    int x_type;
    void *Y;            // entry (t, r) at t y_tok + r y_row
    int64_t y_tok, y_row;
    int type, accumulate;
};

// 16 bytes at `off` of the rows in r, zeros from byte `k` of a row on.
__device__ inline v4i chunk(__amdgpu_buffer_rsrc_t r, int row_off, int at, int k) {
    v4i v = __builtin_amdgcn_raw_buffer_load_b128(r, at < k ? row_off + at : 0x7FFFFFF0, 0, 0);
    return v;
}
__device__ inline void clear_past(v4i &v, int at, int k) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const int n = min(max(k - at - 4 * d, 0), 4);
        v[d] &= n >= 4 ? -1 : (1 << (8 * n)) - 1;
    }
}

// A lane's part of a block: bytes 16 g .. and 64 + 16 g .. (g = lane / 16) of its
// row, so that a wave reads 64 neighbouring bytes of each row at once.
struct Part {
    v4i lo, hi;
};

template <int F>
__device__ inline v4f block_product(const Part &w, const Part &x, v4f p) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const v4i &a = h < 2 ? w.lo : w.hi, &b = h < 2 ? x.lo : x.hi;
        const int i = 2 * (h & 1);
        p = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen<(F & 1)>(a[i], a[i + 1]), widen<(F >> 1)>(b[i], b[i + 1]), p, 0, 0, 0);
    }
    return p;
}

// T x 16 tokens; F: format of W (bit 0) and of the tokens (bit 1); FUSED: tokens of
// x_type, quantized here to e4m3.
template <int WAVES, int T, int F, bool FUSED>
__global__ __launch_bounds__(WAVES * 64) void few_rows(FewArgs g) {
    constexpr int kJoin = WAVES * T * 16 * 16 * 4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[FUSED ? kFusedBytes + 2048 + kJoin : kJoin];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int q = lane & 15, quad = lane >> 4;
    const int r0 = blockIdx.x * 16;
    const auto rw = rows_of(g.w.values + (int64_t)r0 * g.w.ld, min(16, g.w.rows - r0), g.w.ld, g.k);
    const auto rx = FUSED ? rw : rows_of(g.x.values, g.x.rows, g.x.ld, g.k);
    const int w_off = q * (int)g.w.ld;
    const int kpad = g.kblocks * kBlockK;
    float *x_scale = reinterpret_cast<float *>(lds + kFusedBytes);
    uint8_t *join = lds + (FUSED ? kFusedBytes + 2048 : 0);

    Part w[kAhead];
    // the n-th block that this workgroup takes: each begins elsewhere, so that the
    // rows, often a power of two apart, are not all read at one offset at a time
    const int turn = (int)(blockIdx.x % (unsigned)g.kblocks);
    auto turned = [&](int n) { return n + turn < g.kblocks ? n + turn : n + turn - g.kblocks; };
    auto fetch = [&](int n) {
        const int at = n < g.kblocks ? turned(n) * kBlockK + 16 * quad : g.k;
        return Part{chunk(rw, w_off, at, g.k), chunk(rw, w_off, at + 64, g.k)};
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) w[i] = fetch(wave + WAVES * i);

    if (FUSED) {
        // each 16 lanes quantize a block: 8 entries a lane
        const int blocks = g.x.rows * g.kblocks;
        for (int b = tid >> 4; b < blocks; b += WAVES * 4) {
            const int t = b / g.kblocks, kb = b % g.kblocks, k0 = kb * kBlockK + 8 * q;
            float v[8], m = 0.0f;
            const int64_t at = t * g.ldx + k0;
            if (g.x_type == O2M_TYPE_F32) load8(static_cast<const float *>(g.X) + at, g.k - k0, v);
            else if (g.x_type == O2M_TYPE_F16) load8(static_cast<const __half *>(g.X) + at, g.k - k0, v);
            else load8(static_cast<const __hip_bfloat16 *>(g.X) + at, g.k - k0, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) m = fmaxf(m, magnitude(v[j]));
#pragma unroll
            for (int s = 1; s < 16; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
            const Scale s = scale_of(m, O2M_FP8_E4M3, g.w.pow2 ? O2M_SCALES_POW2 : O2M_SCALES_F32);
            float y[4], z[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                y[j] = scaled(v[j], s.inv, 448.0f);
                z[j] = scaled(v[4 + j], s.inv, 448.0f);
            }
            *reinterpret_cast<uint2 *>(lds + t * kpad + k0) = uint2{pack_fp8(y, O2M_FP8_E4M3), pack_fp8(z, O2M_FP8_E4M3)};
            if (q == 0) x_scale[b] = g.w.pow2 ? code_value(s.held) : __uint_as_float(s.held);
        }
        __syncthreads();
    }

    v4f acc[T];
#pragma unroll
    for (int t = 0; t < T; ++t) acc[t] = v4f{0, 0, 0, 0};
    auto block = [&](int kb, Part &wf) {
        const int at = kb * kBlockK + 16 * quad;
        if (kb + 1 == g.kblocks && (g.k & 15)) {   // bytes past k of W's last chunk
            clear_past(wf.lo, at, g.k);
            clear_past(wf.hi, at + 64, g.k);
        }
        float sw[4];
        if (g.w.by_row) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sw[e] = scale_value<true>(g.w, r0 + 4 * quad + e, kb);
        } else {
            sw[0] = sw[1] = sw[2] = sw[3] = scale_value<true>(g.w, r0, kb);
        }
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const int tok = min(16 * t + q, g.x.rows - 1);   // tokens past the last one: not stored
            Part x;
            float sx;
            if (FUSED) {
                x.lo = *reinterpret_cast<const v4i *>(lds + tok * kpad + at);
                x.hi = *reinterpret_cast<const v4i *>(lds + tok * kpad + at + 64);
                sx = x_scale[tok * g.kblocks + kb];
            } else {
                x = {chunk(rx, tok * (int)g.x.ld, at, g.k), chunk(rx, tok * (int)g.x.ld, at + 64, g.k)};
                sx = scale_value<true>(g.x, tok, kb);
                if (kb + 1 == g.kblocks && (g.k & 15)) {
                    clear_past(x.lo, at, g.k);
                    clear_past(x.hi, at + 64, g.k);
                }
            }
            const v4f p = block_product<F>(wf, x, v4f{0, 0, 0, 0});
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][e] = fmaf(p[e], sw[e] * sx, acc[t][e]);
        }
    };
    for (int n = wave; n < g.kblocks; n += WAVES * kAhead) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int at = n + WAVES * i;
            if (at < g.kblocks) {   // uniform
                Part now = w[i];
                w[i] = fetch(at + WAVES * kAhead);
                block(turned(at), now);
            }
        }
    }

    // the waves' sums in their order: entry (row, token) at [wave][token][row]
#pragma unroll
    for (int t = 0; t < T; ++t)
        *reinterpret_cast<v4f *>(join + (((wave * T + t) * 16 + q) * 16 + 4 * quad) * 4) = acc[t];
    __syncthreads();
    for (int i = tid; i < T * 256; i += WAVES * 64) {
        const int t = i >> 4, r = r0 + (i & 15);
        if (t >= g.x.rows || r >= g.w.rows) continue;
        float v = 0.0f;
#pragma unroll
        for (int u = 0; u < WAVES; ++u) v += reinterpret_cast<const float *>(join)[u * T * 256 + i];
        const int64_t at = t * g.y_tok + r * g.y_row;
        store_out(g.Y, at, g.type, v + (g.accumulate ? load_out(g.Y, at, g.type) : 0.0f));
    }
}

// More waves to a workgroup where there are too few workgroups to keep the memory
// busy (8 waves a CU and more), if k has blocks for them.
template <int T, int F, bool FUSED>
void launch_waves(const FewArgs &g, hipStream_t st) {
    const unsigned grid = (unsigned)ceil_div(g.w.rows, 16);
    if (grid >= 1024 || g.kblocks <= 4) few_rows<4, T, F, FUSED><<<grid, 256, 0, st>>>(g);
    else if (FUSED || grid >= 256 || g.kblocks <= 8) few_rows<8, T, F, FUSED><<<grid, 512, 0, st>>>(g);
    else if constexpr (!FUSED) few_rows<16, T, F, FUSED><<<grid, 1024, 0, st>>>(g);
}

// (256 threads where there are many workgroups)
bool few_fits(int n) { return launch_fits(ceil_div(n, 16), 256); }

template <int F>
void launch_tokens(const FewArgs &g, hipStream_t st) {
    if (g.x.rows <= 16) launch_waves<1, F, false>(g, st);
    else launch_waves<2, F, false>(g, st);
}

}  // namespace

// Tokens for which a workgroup quantizes X itself.
bool linear_is_fused(int tokens, int k) { return tokens <= 16 && tokens * round_up64(k, kBlockK) <= kFusedBytes; }

hipError_t launch_linear_fused(int tokens, int n, int k, const void *X, int x_type, int64_t ldx, const o2m_fp8_operand &W,
                               void *Y, int64_t ldy, hipStream_t st) {
    if (!few_fits(n)) return hipErrorInvalidValue;
    FewArgs g = {};
    g.w = side_of(W, n);
    g.x.rows = tokens;
    g.k = k;
    g.kblocks = (int)ceil_div(k, kBlockK);
    g.X = X;
    g.ldx = ldx;
    g.x_type = x_type;
    g.Y = Y;
    g.y_tok = ldy;
    g.y_row = 1;
    g.type = x_type;
    if (W.format == O2M_FP8_E4M3) launch_waves<1, 0, true>(g, st);
    else launch_waves<1, 1, true>(g, st);
    return hipGetLastError();
}

// W: the operand with the many rows; entry (t, r) of Y at t y_tok + r y_row.
hipError_t launch_few(int tokens, int n, int k, const o2m_fp8_operand &X, const o2m_fp8_operand &W, void *Y, int type,
                      int64_t y_tok, int64_t y_row, bool accumulate, hipStream_t st) {
    if (!few_fits(n)) return hipErrorInvalidValue;
    FewArgs g = {};
    g.w = side_of(W, n);
    g.x = side_of(X, tokens);
    g.k = k;
    g.kblocks = (int)ceil_div(k, kBlockK);
    g.Y = Y;
    g.y_tok = y_tok;
    g.y_row = y_row;
    g.type = type;
    g.accumulate = accumulate;
    switch (W.format + 2 * X.format) {
    case 0: launch_tokens<0>(g, st); break;
    case 1: launch_tokens<1>(g, st); break;
    case 2: launch_tokens<2>(g, st); break;
    default: launch_tokens<3>(g, st); break;
    }
    return hipGetLastError();
}

}  // namespace o2m
