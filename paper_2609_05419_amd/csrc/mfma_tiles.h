// What the product kernels of k_fp8.hip and k_ortho.hip share: operand rows
// staged through LDS in k-stages of 128 bytes (128 8-bit or 64 16-bit values),
// and the 16-row fragments that the MFMAs read from there.
//
// A stage of R rows is R x 128 bytes of LDS, row after row.  It arrives by
// direct buffer->LDS copies of 1 KB per wave: 8 rows, each a whole 128-byte
// line of its operand.  The 16-byte chunk c of row r lies in slot c ^ (r >> S & 7)
// of its row: fragments take one chunk of 16 rows at a time, either 16 neighbouring
// ones (S = 1) or 16 rows 4 apart (S = 2, where rows 32 .. 63 of each 64 are kept in
// exchanged pairs), and these 16 chunks fill all 64 banks once.  The swizzle costs nothing: a copy's
// destination is fixed (lane x 16), its source address is each lane's own.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace o2m {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_ptr;

constexpr int kStageRowBytes = 128;
constexpr int kFragRowCount = 16;

// s_waitcnt on the vector-memory counter only (gfx9 encoding), n <= 63
template <int N>
__device__ inline void wait_vmem() {
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (0xF << 8));
}

// Workgroup barrier that leaves copies in flight: this wave's LDS reads have
// returned (lgkmcnt 0), its copies are waited for by wait_vmem beforehand.
__device__ inline void lds_barrier() {
    __builtin_amdgcn_s_waitcnt(0xC07F);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Descriptor of `rows` operand rows of kbytes each, `ld` bytes apart: reads
// past the last one give zeros.  ld < 2^23 (checked on the host) keeps every
// offset of a tile below 2^31.
__device__ inline __amdgpu_buffer_rsrc_t rows_of(const uint8_t *base, int rows, int64_t ld, int kbytes) {
    const int extent = rows > 0 ? (int)((rows - 1) * ld) + ((kbytes + 15) & ~15) : 0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(base), (short)0, extent, 0x00020000);
}

// Where row r lies among the rows of a stage; its own inverse.
template <int S>
__device__ inline int kept_row(int r) { return S == 2 ? r ^ (r >> 5 & 1) : r; }

// Copy rows [8 q, 8 q + 8) of a stage, which lies `at` bytes from the descriptor's
// start, to dst (wave-uniform, 1 KB; S: as above, of LDS rows).  `left` is the operand's bytes from there on: chunks past it are read as zeros.  S:
// the chunk c of row r lies in slot c ^ (r >> S & 7).
template <int S>
__device__ inline void copy_rows(__amdgpu_buffer_rsrc_t r, uint8_t *dst, int lane, int q, int ld, int at, int left) {
    const int at_row = 8 * q + (lane >> 3), row = kept_row<S>(at_row), chunk16 = ((lane & 7) ^ (row >> S & 7)) << 4;
    int off = row * ld + chunk16;
    if (left < kStageRowBytes) off = chunk16 < left ? off : 0x7FFFFFF0;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr *)dst, 16, off, at, 0, 0);
}

// Zero the bytes of the row at `row` past `left` in the chunk that holds byte `left`.
__device__ inline void clear_row_tail(uint8_t *stage, int row, int left, int s) {
    uint8_t *chunk = stage + row * kStageRowBytes + (((left >> 4) ^ (row >> s & 7)) << 4);
    for (int b = left & 15; b < 16; ++b) chunk[b] = 0;
}

// The 32 bytes of a fragment that one lane holds: of `row`, bytes [32 g, 32 g +
// 32) of the stage row with g = lane / 16.
template <int S>
__device__ inline v8i read_fragment(const uint8_t *stage, int row, int lane) {
    const int slot = (2 * (lane >> 4)) ^ (row >> S & 7);
    const uint8_t *p = stage + kept_row<S>(row) * kStageRowBytes;
    const v4i lo = *reinterpret_cast<const v4i *>(p + (slot << 4));
    const v4i hi = *reinterpret_cast<const v4i *>(p + ((slot ^ 1) << 4));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

}  // namespace o2m
