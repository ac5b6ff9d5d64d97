// What the kernels of the 8-bit block-scaled product share on the device.
//
//   C[i][j] = sum_b sA[i][b] sB[j][b] sum_{l in block b} A[i][l] B[j][l]          (blocks of 128 along k)
//
// A step is one block: one v_mfma_*_16x16x128_f8f6f4 per 16 x 16 of C.  B feeds the instruction's row operand and A its
// column operand, so a lane's four results are four consecutive j of one row of C.  E8M0 scales go into the instruction,
// which multiplies by them exactly; float32 scales are applied to each block's sums, in 32 bits.
#pragma once

#include "oz_scaled_device.h"

namespace oz {

// 64 lanes x 16 (4) bytes from global memory into LDS at lds_addr + 16 (4) * lane; the address is a wave-uniform base and a per-lane
// offset.  The compiler does not see the access: completion is awaited with s_waitcnt vmcnt in the loops.
__device__ __forceinline__ void copy16_to_lds(const uint8_t* base, uint32_t lane_off, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(lds_addr), "v"(lane_off), "s"(base) : "memory");
}
__device__ __forceinline__ void copy4_to_lds(const uint8_t* base, uint32_t lane_off, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, %2" :: "s"(lds_addr), "v"(lane_off), "s"(base) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return uint32_t(uintptr_t((__attribute__((address_space(3))) const uint8_t*)p));
}

// One step of 16 x 16 results: E8M0 scales in the low byte of sb, sa; A_E5M2: A's type (B is e4m3).
template <bool A_E5M2>
__device__ __forceinline__ v4f mfma_e8m0(v8i32 b, v8i32 a, v4f c, uint32_t sb, uint32_t sa) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, A_E5M2 ? 1 : 0, 0, int(sb), 0, int(sa));
}
template <bool A_E5M2>
__device__ __forceinline__ v4f mfma_plain(v8i32 b, v8i32 a) {
    const v4f none = {0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, none, 0, A_E5M2 ? 1 : 0, 0, 0, 0, 0);
}

// The part of a call that a workgroup works on.  Offsets in bytes / elements are 64-bit, what is left inside a tile 32-bit.
struct GemmTile {
    const uint8_t *a, *b;         // first row of the tile, first byte of k
    const uint8_t *sa, *sb;       // scale arrays of the operands (of the group's B)
    int row, rows;                // rows of A and of C
    int col, cols;                // rows of B, columns of C
    int k;                        // bytes of k; 0: C is zero, or left as it is
    int block0;                   // first block of k
    int64_t c;                    // elements from the call's C to this group's
    bool none;
};

// Rows `row` on of group `group`; TM rows, TN columns of C per tile.
template <int TM, int TN>
__device__ __forceinline__ GemmTile locate(const ScaledGemm& g, int tile_m, int tile_n, int group) {
    GemmTile t;
    t.none = false;
    t.row = tile_m * TM;
    t.col = tile_n * TN;
    t.cols = min(TN, g.n - t.col);
    t.k = g.k;
    t.block0 = 0;
    t.c = 0;
    int row_end = g.m, weights = 0;
    if (g.grouping == Grouping::kRows) {
        const GroupPiece p = find_piece<TM>(g.offsets, g.groups, g.m, tile_m);
        if (p.group < 0) { t.none = true; return t; }
        t.row = p.row;
        row_end = p.end;
        weights = p.group;
        if (p.group == g.groups) { weights = 0; t.k = 0; }
    } else if (g.grouping == Grouping::kContraction) {
        const GroupSpan s = group_span(g.offsets, group, g.k);
        t.k = s.count;
        t.block0 = s.blocks_before;
        t.c = int64_t(group) * g.stride_c;
        if (t.block0 + (t.k + kScaleBlock - 1) / kScaleBlock > g.k / kScaleBlock) t.k = 0;       // offsets that do not fit the columns
    }
    t.rows = min(TM, row_end - t.row);
    const int64_t k0 = int64_t(t.block0) * kScaleBlock;
    t.a = g.a.data + int64_t(t.row) * g.a.ld + k0;
    t.b = g.b.data + int64_t(weights) * g.b.stride + int64_t(t.col) * g.b.ld + k0;
    const int64_t esize = g.e8m0 ? 1 : 4;
    t.sa = g.a.scale;
    t.sb = g.b.scale + int64_t(weights) * g.b.scale_stride * esize;
    return t;
}

// Four consecutive results of one row of C.
template <typename T>
__device__ __forceinline__ void put4(T* p, int have, bool vec, bool add, const v4f& x) {
    typedef T vec_t __attribute__((ext_vector_type(4)));
    if (vec && have >= 4) {
        v4f s = x;
        if (add) {
            const vec_t old = *reinterpret_cast<const vec_t*>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += float(old[i]);
        }
        vec_t out;
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = T(s[i]);
        *reinterpret_cast<vec_t*>(p) = out;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) p[i] = T(add ? x[i] + float(p[i]) : x[i]);
    }
}
__device__ __forceinline__ void put4(const ScaledGemm& g, int64_t at, int have, bool vec, const v4f& x) {
    const bool add = g.accumulate != 0;
    if (g.c_type == OZ_F32) put4(static_cast<float*>(g.c) + at, have, vec, add, x);
    else if (g.c_type == OZ_BF16) put4(static_cast<bf16_t*>(g.c) + at, have, vec, add, x);
    else put4(static_cast<f16_t*>(g.c) + at, have, vec, add, x);
}
__device__ __forceinline__ bool aligned_c(const ScaledGemm& g, int64_t offset) {
    const int esize = g.c_type == OZ_F32 ? 4 : 2;
    return ((uintptr_t(g.c) + uintptr_t(offset) * esize) | uintptr_t(g.ldc) * esize) % (4 * esize) == 0;
}

}  // namespace oz
