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

// One tile of 128 x 128 entries per workgroup, quantized along its lines, across
// them or both.  Thread (rg, cg) holds the 8 x 8 entries of lines 8 rg.. and
// positions 8 cg..: 16 threads share a line, whose maximum is taken by lane
// exchanges, and the maxima across lines and the bytes of the transposed operand
// go through LDS (in 8-byte units of 8 lines, unit rg of position q in slot rg ^
// (q / 8), which spreads both the writes and the reads over the banks).
template <class T>
__global__ __launch_bounds__(256) void quantize_tile(QuantArgs g) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[128 * 128];
    __shared__ float tile_max[4];
    const int tid = threadIdx.x, cg = tid & 15, rg = tid >> 4;
    const int tp = blockIdx.x / g.tiles_q, tq = blockIdx.x % g.tiles_q;
    const int p0 = tp * 128 + 8 * rg, q0 = tq * 128 + 8 * cg;
    const int nq = min(8, g.len - q0);
    float x[8][8], row_max[8], col_max[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) col_max[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        load8<T>(static_cast<const T *>(g.X) + (int64_t)(p0 + i) * g.ld + q0, p0 + i < g.lines ? nq : 0, x[i]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float a = magnitude(x[i][j]);
            m = fmaxf(m, a);
            col_max[j] = fmaxf(col_max[j], a);
        }
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
        row_max[i] = m;
    }
    const bool whole = g.along.block == kBlockK || g.across.block == kBlockK;
    float all = 0.0f;
    if (whole) {   // (uniform over the workgroup)
#pragma unroll
        for (int i = 0; i < 8; ++i) all = fmaxf(all, row_max[i]);
        all = fmaxf(all, __shfl_xor(all, 16));
        all = fmaxf(all, __shfl_xor(all, 32));
        if ((tid & 63) == 0) tile_max[tid >> 6] = all;
        __syncthreads();
        all = fmaxf(fmaxf(tile_max[0], tile_max[1]), fmaxf(tile_max[2], tile_max[3]));
    }

    if (g.along.values) {
        const Dest &d = g.along;
        const float top = d.format == O2M_FP8_E4M3 ? 448.0f : 57344.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Scale s = scale_of(d.block == 1 ? row_max[i] : all, d.format, d.scale_type);
            if (p0 + i >= g.lines || nq <= 0) continue;
            float y[4], z[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                y[j] = scaled(x[i][j], s.inv, top);
                z[j] = scaled(x[i][4 + j], s.inv, top);
            }
            store_bytes(d.values + (int64_t)(p0 + i) * d.ld + q0, uint2{pack_fp8(y, d.format), pack_fp8(z, d.format)}, nq);
            if (cg == 0 && d.block == 1) store_scale(d, p0 + i, tq, s.held);
            if (tid == 0 && i == 0 && d.block == kBlockK) store_scale(d, tp, tq, s.held);
        }
    }

    if (g.across.values) {
        const Dest &d = g.across;
        const float top = d.format == O2M_FP8_E4M3 ? 448.0f : 57344.0f;
        Scale s[8];
        if (d.block == 1) {
            float *part = reinterpret_cast<float *>(lds);   // [16][128]
#pragma unroll
            for (int j = 0; j < 8; ++j) part[rg * 128 + 8 * cg + j] = col_max[j];
            __syncthreads();
            float m = 0.0f;
            if (tid < 128) {
                for (int r = 0; r < 16; ++r) m = fmaxf(m, part[r * 128 + tid]);
            }
            __syncthreads();
            if (tid < 128) part[tid] = m;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[j] = scale_of(part[8 * cg + j], d.format, d.scale_type);
                if (rg == 0 && j < nq) store_scale(d, q0 + j, tp, s[j].held);
            }
            __syncthreads();   // before the bytes overwrite the maxima
        } else {
            const Scale t = scale_of(all, d.format, d.scale_type);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = t;
            if (tid == 0) store_scale(d, tq, tp, t.held);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float y[4], z[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i] = scaled(x[i][j], s[j].inv, top);
                z[i] = scaled(x[4 + i][j], s[j].inv, top);
            }
            *reinterpret_cast<uint2 *>(lds + (8 * cg + j) * 128 + ((rg ^ cg) << 3)) =
                uint2{pack_fp8(y, d.format), pack_fp8(z, d.format)};
        }
        __syncthreads();
        // unit u (8 lines) of position q: 16 consecutive threads write the 128
        // bytes of one operand row
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int q = 16 * i + (tid >> 4), u = tid & 15;
            const uint2 w = *reinterpret_cast<const uint2 *>(lds + q * 128 + ((u ^ (q >> 3)) << 3));
            const int line = tp * 128 + 8 * u;
            if (tq * 128 + q < g.len && line < g.lines)
                store_bytes(d.values + (int64_t)(tq * 128 + q) * d.ld + line, w, min(8, g.lines - line));
        }
    }
}

// Along lines alone, in blocks of 1 x 128: 16 lanes hold a block, 8 entries each, and
// nothing is shared.  PER blocks of a line, 16 lanes apart from one another, keep
// that many loads in flight.
template <class T, int PER>
__global__ __launch_bounds__(256) void quantize_rows(QuantArgs g) {
    const Dest &d = g.along;
    const float top = d.format == O2M_FP8_E4M3 ? 448.0f : 57344.0f;
    const int lane16 = threadIdx.x & 15;
    const int64_t group = blockIdx.x * 16LL + (threadIdx.x >> 4);   // PER blocks of a line
    const int groups = (g.tiles_q + PER - 1) / PER;
    const int64_t p = group / groups;
    if (p >= g.lines) return;
    const int blk0 = (int)(group % groups) * PER;
    const T *line = static_cast<const T *>(g.X) + p * g.ld;
    float x[PER][8];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int q0 = (blk0 + i) * 128 + 8 * lane16;
        load8<T>(line + q0, min(8, g.len - q0), x[i]);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, magnitude(x[i][j]));
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
        const Scale s = scale_of(m, d.format, d.scale_type);
        const int q0 = (blk0 + i) * 128 + 8 * lane16, n = g.len - q0;
        if (n <= 0) continue;
        float y[4], z[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            y[j] = scaled(x[i][j], s.inv, top);
            z[j] = scaled(x[i][4 + j], s.inv, top);
        }
        store_bytes(d.values + p * d.ld + q0, uint2{pack_fp8(y, d.format), pack_fp8(z, d.format)}, n);
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
        quantize_tile<T><<<(unsigned)tiles, 256, 0, st>>>(g);
        return hipGetLastError();
    }
    const int64_t by4 = ceil_div(g.lines * ceil_div(g.tiles_q, 4), 16), by1 = ceil_div((int64_t)g.lines * g.tiles_q, 16);
    if (by1 > 0x7FFFFFFF) return hipErrorInvalidValue;
    if (by4 >= 2048) quantize_rows<T, 4><<<(unsigned)by4, 256, 0, st>>>(g);
    else quantize_rows<T, 1><<<(unsigned)by1, 256, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(int lines, int len, const void *X, int type, int64_t ld, const o2m_fp8_operand *along,
                           const o2m_fp8_operand *across, hipStream_t st) {
    const int64_t tiles_q = ceil_div(len, 128), tiles = tiles_q * ceil_div(lines, 128);
    if (tiles <= 0) return hipSuccess;
    if (tiles > 0x7FFFFFFF) return hipErrorInvalidValue;
    const QuantArgs g = {X, ld, lines, len, (int)tiles_q, dest_of(along), dest_of(across)};
    switch (type) {
    case O2M_TYPE_F32: return launch<float>(g, tiles, st);
    case O2M_TYPE_F16: return launch<__half>(g, tiles, st);
    default: return launch<__hip_bfloat16>(g, tiles, st);
    }
}

}  // namespace o2m
