// Quantization into 8-bit floating point with a scale for each block of 1 x
// 128 or 128 x 128 entries (include/o2m.h: o2m_quantize_fp8).
//
// Bound: memory.  One read of X and one write of each operand.
#include "fp8_round.h"
#include "model_internal.h"

namespace o2m {
namespace {

struct Dest {
    uint8_t *values;
    int64_t ld;
    void *scales;
    int64_t s_row, s_blk;
    int block, format, scale_type;
};

struct QuantArgs {
    const void *X;
    int64_t ld;
    int lines, len;
    int tiles_q;      // tiles along a line
    Dest along, across;
};

__device__ inline void store_scale(const Dest &d, int64_t row, int64_t blk, uint32_t held) {
    const int64_t i = row * d.s_row + blk * d.s_blk;
    if (d.scale_type == O2M_SCALES_F32) static_cast<uint32_t *>(d.scales)[i] = held;
    else static_cast<uint8_t *>(d.scales)[i] = (uint8_t)held;
}

__device__ inline void store_bytes(uint8_t *p, uint2 w, int n) {
    if (n >= 8) {
        *reinterpret_cast<uint2 *>(p) = w;
    } else {
        for (int j = 0; j < n; ++j) p[j] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
    }
}

// The largest finite magnitude of eight entries, as bits.
template <class T>
__device__ inline uint32_t largest_finite_of(const Run8<T> &r) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < Run8<T>::kWords; ++i) {
        const uint32_t w = magnitude_bits<T>(r.w[i]), lo = Run8<T>::kHalves ? w & 0xFFFFu : w, hi = Run8<T>::kHalves ? w >> 16 : 0;
        m = max(m, max(bits_finite<T>(lo) ? lo : 0u, bits_finite<T>(hi) ? hi : 0u));
    }
    return m;
}
// Words with Inf and NaN replaced by zeros.
template <class T>
__device__ inline uint32_t finite_word(uint32_t w) {
    w = magnitude_bits<T>(w);
    if (!Run8<T>::kHalves) return bits_finite<T>(w) ? w : 0u;
    return (bits_finite<T>(w & 0xFFFFu) ? w & 0xFFFFu : 0u) | (bits_finite<T>(w >> 16) ? w & 0xFFFF0000u : 0u);
}

// One tile of 128 x 128 entries per workgroup, quantized along its lines, across
// them or both.  Thread (rg, cg) holds the 4 x 8 entries of lines 4 rg .. and
// positions 8 cg ..: 16 lanes share a line, whose maximum is taken by lane
// exchanges; the maxima across lines go through LDS, and so do the bytes of the
// transposed operand, in words of 4 lines: word rg of position q lies at rg ^ 2 (q /
// 8), which spreads both the writes and the reads over the banks.
//
// Bound: memory; the vector unit comes next, which is why maxima are taken on the
// bits as they come and Inf and NaN are looked for once a tile.
constexpr int kTileThreads = 512;
template <class T, bool ALONG, bool ACROSS>
__global__ __launch_bounds__(kTileThreads, 4) void quantize_tile(QuantArgs g) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[ACROSS ? 128 * 128 : 16];
    __shared__ uint32_t part[ACROSS ? 8 : 1][ACROSS ? 128 : 1];   // maxima of each wave's lines
    __shared__ uint32_t wave_max[8];
    constexpr int W = Run8<T>::kWords;
    const int tid = threadIdx.x, cg = tid & 15, rg = tid >> 4, wave = tid >> 6;
    const int tp = blockIdx.x / g.tiles_q, tq = blockIdx.x % g.tiles_q;
    const int p0 = tp * 128 + 4 * rg, q0 = tq * 128 + 8 * cg;
    const int nq = min(8, g.len - q0);
    Run8<T> x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        x[i] = load_run(static_cast<const T *>(g.X) + (int64_t)(p0 + i) * g.ld + q0, p0 + i < g.lines ? nq : 0);

    uint32_t row_max[4], all = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        row_max[i] = largest_of(x[i]);
        all = max(all, row_max[i]);
    }
    const bool fine = !__syncthreads_or(!bits_finite<T>(all));
    if (!fine) {
        all = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            row_max[i] = largest_finite_of(x[i]);
            all = max(all, row_max[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) row_max[i] = largest_of_16(row_max[i]);
    const bool whole = (ALONG && g.along.block == kBlockK) || (ACROSS && g.across.block == kBlockK);
    if (whole) {   // (uniform over the workgroup)
        all = larger_of_rows<float>(largest_of_16(all));
        if ((tid & 63) == 0) wave_max[wave] = all;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) all = max(all, wave_max[w]);
    }

    if (ALONG) {
        const Dest &d = g.along;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Scale s = scale_of(bits_value<T>(d.block == 1 ? row_max[i] : all), d.format, d.scale_type);
            if (p0 + i >= g.lines || nq <= 0) continue;
            const uint2 w = fine ? round_run<true>(x[i], s.inv, d.format) : round_run<false>(x[i], s.inv, d.format);
            store_bytes(d.values + (int64_t)(p0 + i) * d.ld + q0, w, nq);
            if (cg == 0 && d.block == 1) store_scale(d, p0 + i, tq, s.held);
            if (tid == 0 && i == 0 && d.block == kBlockK) store_scale(d, tp, tq, s.held);
        }
    }

    if (ACROSS) {
        const Dest &d = g.across;
        float inv[8];
        if (d.block == 1) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                uint32_t m = 0;
#pragma unroll
                for (int l = 0; l < 4; ++l) m = larger<T>(m, fine ? magnitude_bits<T>(x[l].w[i]) : finite_word<T>(x[l].w[i]));
                m = larger_of_rows<T>(m);
                if ((tid & 63) < 16) {
                    if (Run8<T>::kHalves) {
                        part[wave][8 * cg + 2 * i] = m & 0xFFFFu;
                        part[wave][8 * cg + 2 * i + 1] = m >> 16;
                    } else {
                        part[wave][8 * cg + i] = m;
                    }
                }
            }
            __syncthreads();
            if (tid < 128) {   // a position each: its scale, and the inverse for the others
                uint32_t m = 0;
#pragma unroll
                for (int w = 0; w < 8; ++w) m = max(m, part[w][tid]);
                const Scale s = scale_of(bits_value<T>(m), d.format, d.scale_type);
                part[0][tid] = __float_as_uint(s.inv);   // (only this thread reads this column)
                if (tq * 128 + tid < g.len) store_scale(d, tq * 128 + tid, tp, s.held);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) inv[j] = __uint_as_float(part[0][8 * cg + j]);
        } else {
            const Scale s = scale_of(bits_value<T>(all), d.format, d.scale_type);
#pragma unroll
            for (int j = 0; j < 8; ++j) inv[j] = s.inv;
            if (tid == 0) store_scale(d, tq, tp, s.held);
        }
        const float top = d.format == O2M_FP8_E4M3 ? 448.0f : 57344.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = fine ? entry(x[i], j) * inv[j] : scaled(entry(x[i], j), inv[j], top);
            *reinterpret_cast<uint32_t *>(lds + (8 * cg + j) * 128 + ((rg ^ (2 * cg)) << 2)) = pack_fp8(y, d.format);
        }
        __syncthreads();
        // 8 consecutive threads write the 128 bytes of one operand row
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int q = 64 * i + (tid >> 3), u = tid & 7, turn = q >> 3;   // bytes 16 u ..: words 4 u ..
            const uint2 lo = *reinterpret_cast<const uint2 *>(lds + q * 128 + (((2 * u) ^ turn) << 3));
            const uint2 hi = *reinterpret_cast<const uint2 *>(lds + q * 128 + (((2 * u + 1) ^ turn) << 3));
            const int line = tp * 128 + 16 * u, n = g.lines - line;
            if (tq * 128 + q >= g.len || n <= 0) continue;
            uint8_t *p = d.values + (int64_t)(tq * 128 + q) * d.ld + line;
            if (n >= 16) {
                *reinterpret_cast<uint4 *>(p) = uint4{lo.x, lo.y, hi.x, hi.y};
            } else {
                store_bytes(p, lo, min(8, n));
                store_bytes(p + 8, hi, min(8, n - 8));
            }
        }
    }
}

// Along lines alone, in blocks of 1 x 128: 16 lanes hold a block, 8 entries each, and
// nothing is shared.  PER blocks of a line, 16 lanes apart from one another, keep
// that many loads in flight.
template <class T, int PER>
__global__ __launch_bounds__(256) void quantize_rows(QuantArgs g) {
    const Dest &d = g.along;
    const int lane16 = threadIdx.x & 15;
    const int64_t group = blockIdx.x * 16LL + (threadIdx.x >> 4);   // PER blocks of a line
    const int groups = (g.tiles_q + PER - 1) / PER;
    const int64_t p = group / groups;
    if (p >= g.lines) return;
    const int blk0 = (int)(group % groups) * PER;
    const T *line = static_cast<const T *>(g.X) + p * g.ld;
    Run8<T> x[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int q0 = (blk0 + i) * 128 + 8 * lane16;
        x[i] = load_run(line + q0, min(8, g.len - q0));
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        uint32_t m = largest_of_16(largest_of(x[i]));
        const bool fine = bits_finite<T>(m);
        if (!fine) m = largest_of_16(largest_finite_of(x[i]));   // (the 16 lanes agree)
        const Scale s = scale_of(bits_value<T>(m), d.format, d.scale_type);
        const int q0 = (blk0 + i) * 128 + 8 * lane16, n = g.len - q0;
        if (n <= 0) continue;
        const uint2 w = fine ? round_run<true>(x[i], s.inv, d.format) : round_run<false>(x[i], s.inv, d.format);
        store_bytes(d.values + p * d.ld + q0, w, n);
        if (lane16 == 0) store_scale(d, p, blk0 + i, s.held);
    }
}

Dest dest_of(const o2m_fp8_operand *o) {
    if (!o) return {nullptr, 0, nullptr, 0, 0, 0, 0, 0};
    return {static_cast<uint8_t *>(o->values), o->ld, o->scales, o->s_row, o->s_blk, o->block, o->format, o->scale_type};
}

// Lines of many blocks are taken four at a time where that leaves enough
// workgroups (8 a CU); a token's single line is taken block by block.
template <class T>
hipError_t launch(const QuantArgs &g, int64_t tiles, hipStream_t st) {
    if (g.across.values || g.along.block != 1) {
        if (!launch_fits(tiles, kTileThreads)) return hipErrorInvalidValue;
        if (!g.across.values) quantize_tile<T, true, false><<<(unsigned)tiles, kTileThreads, 0, st>>>(g);
        else if (!g.along.values) quantize_tile<T, false, true><<<(unsigned)tiles, kTileThreads, 0, st>>>(g);
        else quantize_tile<T, true, true><<<(unsigned)tiles, kTileThreads, 0, st>>>(g);
        return hipGetLastError();
    }
    const int64_t by4 = ceil_div(g.lines * ceil_div(g.tiles_q, 4), 16), by1 = ceil_div((int64_t)g.lines * g.tiles_q, 16);
    if (!launch_fits(by4 >= 2048 ? by4 : by1, 256)) return hipErrorInvalidValue;
    if (by4 >= 2048) quantize_rows<T, 4><<<(unsigned)by4, 256, 0, st>>>(g);
    else quantize_rows<T, 1><<<(unsigned)by1, 256, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(int lines, int len, const void *X, int type, int64_t ld, const o2m_fp8_operand *along,
                           const o2m_fp8_operand *across, hipStream_t st) {
    const int64_t tiles_q = ceil_div(len, 128), tiles = tiles_q * ceil_div(lines, 128);
    if (tiles <= 0) return hipSuccess;
    const QuantArgs g = {X, ld, lines, len, (int)tiles_q, dest_of(along), dest_of(across)};
    switch (type) {
    case O2M_TYPE_F32: return launch<float>(g, tiles, st);
    case O2M_TYPE_F16: return launch<__half>(g, tiles, st);
    default: return launch<__hip_bfloat16>(g, tiles, st);
    }
}

}  // namespace o2m
