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

// Rows of a tile as a buffer: loads at lane offset + scalar offset from `base` on; dwords from `bytes` on read as zero and touch no
// memory, so neither rows behind the last nor bytes behind the end of the last row are loaded.
__device__ __forceinline__ v4i32 tile_buffer(const uint8_t* base, uint32_t bytes) {
    const uint64_t a = uint64_t(uintptr_t(base));
    return v4i32{__builtin_amdgcn_readfirstlane(int(uint32_t(a))), __builtin_amdgcn_readfirstlane(int(uint32_t(a >> 32) & 0xFFFFu)),
                 __builtin_amdgcn_readfirstlane(int(bytes)), 0x00020000};
}
// 64 lanes x 16 (4) bytes from memory into LDS at lds_addr + 16 (4) * lane.  The compiler does not see the access: completion is awaited
// with s_waitcnt vmcnt in the loops.
__device__ __forceinline__ void copy16_to_lds(const v4i32& buffer, uint32_t lane_off, uint32_t off, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :: "s"(lds_addr), "v"(lane_off), "s"(buffer), "s"(off) : "memory");
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

// The instruction above adds products by eights and cuts each off, towards zero, at 2^-13 of the largest of its eight (a 1 beside 2^14 and -2^14 is
// lost, in another eight it is not); sums of eights and C keep 32 bits.  Normal data: 1.4e-5 of the result's rms, which a result
// rounded to 16 bits does not show.  Where C is float32, operands are widened to bfloat16, exactly, for v_mfma_f32_16x16x32_bf16,
// whose sums keep 32 bits (8e-9 on the same data) at half the rate.  A fragment's 32 bytes per lane make four operands.
typedef bf16_t v8bf __attribute__((ext_vector_type(8)));
typedef bf16_t v2bf __attribute__((ext_vector_type(2)));
// four bytes: two pairs
template <bool E5M2>
__device__ __forceinline__ void widen4(uint32_t x, float scale, int& lo, int& hi) {
    v2bf p, q;
    if constexpr (E5M2) {
        p = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(x, scale, false);
        q = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(x, scale, true);
    } else {
        p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false);
        q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true);
    }
    lo = __builtin_bit_cast(int, p);
    hi = __builtin_bit_cast(int, q);
}
struct Wide { v4i32 part[4]; };         // pairs of bfloat16
template <bool E5M2>
__device__ __forceinline__ Wide widen(const v8i32& f, float scale) {
    Wide w;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        int lo, hi;
        widen4<E5M2>(uint32_t(f[i]), scale, lo, hi);
        w.part[i >> 1][2 * (i & 1)] = lo;
        w.part[i >> 1][2 * (i & 1) + 1] = hi;
    }
    return w;
}
__device__ __forceinline__ v4f mfma_bf16(const v4i32& b, const v4i32& a, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, b), __builtin_bit_cast(v8bf, a), c, 0, 0, 0);
}
__device__ __forceinline__ v4f mfma_wide(const Wide& b, const Wide& a, v4f c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = mfma_bf16(b.part[i], a.part[i], c);
    return c;
}
// An E8M0 scale as the conversion takes it: a float of that exponent.
__device__ __forceinline__ float scale_float(uint32_t byte) { return __uint_as_float((byte & 0xFFu) << 23); }
// Widening with a scale is exact while no element leaves bfloat16's normal numbers: elements lie in 2^-16 .. 1.75 2^15 (e5m2; e4m3's are
// within), so exponents from -110 to 112 do.  Where another one turns up, or a NaN, operands are widened without scales and both are applied
// to the sums (add_scaled): a sum's factor is a power of two, so that costs no precision, only time.
constexpr uint32_t kWidenLeast = 127 - 110, kWidenMost = 127 + 112;
// x, y: words of four scales, of which the lowest `blocks` count; by a whole wave.
template <int M, int N>
__device__ __forceinline__ bool widens_exactly(const uint32_t (&x)[M], const uint32_t (&y)[N], int blocks) {
    static_assert(kWidenMost == 0xEF, "above are the bytes whose upper four bits are set");
    uint32_t wild = 0;
    // the top bit of a byte: below the least (of a word's first such byte), above the most
    auto look = [&](uint32_t w) { wild |= ((w - kWidenLeast * 0x01010101u) & ~w) | (w & (w << 1) & (w << 2) & (w << 3)); };
    const uint32_t there = blocks >= 4 ? 0xFFFFFFFFu : (1u << (8 * blocks)) - 1;
#pragma unroll
    for (int i = 0; i < M; ++i) look((x[i] & there) | (0x7F7F7F7Fu & ~there));
#pragma unroll
    for (int i = 0; i < N; ++i) look((y[i] & there) | (0x7F7F7F7Fu & ~there));
    return __ballot((wild & 0x80808080u) != 0) == 0;
}
// c + p 2^(ea + eb): the product's exponent is applied at once, whatever the two are.
__device__ __forceinline__ float add_scaled(float c, float p, uint32_t ea, uint32_t eb) {
    const uint32_t a = ea & 0xFFu, b = eb & 0xFFu;
    return c + (max(a, b) == 255 ? __uint_as_float(0x7FC00000u) : __builtin_amdgcn_ldexpf(p, int(a + b) - 254));
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

// Which tile a workgroup takes.  Workgroups are dealt to the XCDs in turn: an XCD gets a contiguous run of tiles, in bands of eight rows of
// tiles, so that those it has at a time share their operands in its L2.  Rows in groups: of the tiles that there are, fewer than the
// launch has workgroups for (8192 rows in 8 groups, the runs counted by the launch 68 us, by the tiles 54: the last XCDs were idle).
struct TilePlace { int m, n; };      // n < 0: none
__device__ __forceinline__ TilePlace tile_place(int tiles_m, int tiles_n) {
    constexpr int kBand = 8;
    const int total = tiles_m * tiles_n, per = total / 8, extra = total % 8, xcd = int(blockIdx.x) & 7, slot = int(blockIdx.x) >> 3;
    if (slot >= per + (xcd < extra ? 1 : 0)) return TilePlace{0, -1};
    const int id = xcd * per + min(xcd, extra) + slot;
    const int band = id / (kBand * tiles_n), in_band = id - band * kBand * tiles_n, high = min(kBand, tiles_m - band * kBand);
    return TilePlace{band * kBand + in_band % high, in_band / high};
}

// The tile at (tile_m, tile_n), TM rows and TN columns of C, of product or part `group`; p: where it is if rows come in groups.
template <int TM, int TN>
__device__ __forceinline__ GemmTile tile_at(const ScaledGemm& g, int tile_m, int tile_n, int group, const GroupPiece& p) {
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
    } else if (g.parts > 1) {             // `group`: a part of k
        const int fours = (g.k + 4 * kScaleBlock - 1) / (4 * kScaleBlock);        // whole words of E8M0 scales
        t.block0 = int(int64_t(fours) * group / g.parts) * 4;
        t.k = min(g.k, int(int64_t(fours) * (group + 1) / g.parts) * 4 * kScaleBlock) - t.block0 * kScaleBlock;
        t.c = int64_t(group) * g.m * g.n;
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
// A workgroup's tile.  DEALT: over the XCDs as above, of tiles_m rows of tiles (with groups: of those that there are), else row by row.
template <int TM, int TN, bool DEALT>
__device__ __forceinline__ GemmTile locate(const ScaledGemm& g, int tiles_m, int tiles_n) {
    TilePlace place{int(blockIdx.x) / tiles_n, int(blockIdx.x) % tiles_n};
    GroupPiece p = {};
    if (g.grouping == Grouping::kRows) {
        GroupPieces<TM> pieces(g.offsets, g.groups, g.m);
        if (DEALT) place = tile_place(pieces.count, tiles_n);
        if (place.n >= 0) p = pieces.template find<false>(place.m);
    } else if (DEALT) {
        place = tile_place(tiles_m, tiles_n);
    }
    GemmTile t = tile_at<TM, TN>(g, place.m, max(place.n, 0), int(blockIdx.y), p);
    if (place.n < 0) t.none = true;
    return t;
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    typedef T pair __attribute__((ext_vector_type(2)));
    union { pair p; uint32_t u; } v;
    v.p = pair{T(lo), T(hi)};
    return v.u;
}
template <typename T>
__device__ __forceinline__ v4f unpack4(uint2 w) {
    typedef T quad __attribute__((ext_vector_type(4)));
    union { uint2 w; quad q; } v;
    v.w = w;
    return v4f{float(v.q[0]), float(v.q[1]), float(v.q[2]), float(v.q[3])};
}

// Four consecutive results of one row of C.
template <typename T>
__device__ __forceinline__ void put4(T* p, int have, bool add, v4f s) {
    typedef T aligned_quad __attribute__((ext_vector_type(4)));
    typedef aligned_quad __attribute__((aligned(2), may_alias)) quad;
    if (have >= 4) {
        quad* at = reinterpret_cast<quad*>(p);
        if (add) {
            const aligned_quad old = *at;
            s += v4f{float(old[0]), float(old[1]), float(old[2]), float(old[3])};
        }
        *at = aligned_quad{T(s[0]), T(s[1]), T(s[2]), T(s[3])};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) p[i] = T(add ? s[i] + float(p[i]) : s[i]);
    }
}
__device__ __forceinline__ void put4(const ScaledGemm& g, int64_t at, int have, const v4f& s) {
    if (g.c_type == OZ_F32) put4(static_cast<float*>(g.c) + at, have, g.accumulate != 0, s);
    else if (g.c_type == OZ_BF16) put4(static_cast<bf16_t*>(g.c) + at, have, g.accumulate != 0, s);
    else put4(static_cast<f16_t*>(g.c) + at, have, g.accumulate != 0, s);
}

// A tile whose k is empty, by all of a workgroup: zero, unless it is added to what is there.
__device__ __forceinline__ void store_nothing(const ScaledGemm& g, const GemmTile& t) {
    if (g.accumulate) return;
    for (int r = 0; r < t.rows; ++r)
        for (int c = threadIdx.x; c < t.cols; c += blockDim.x) {
            const int64_t at = t.c + int64_t(t.row + r) * g.ldc + t.col + c;
            if (g.c_type == OZ_F32) static_cast<uint32_t*>(g.c)[at] = 0;
            else static_cast<uint16_t*>(g.c)[at] = 0;
        }
}

// A wave's results, MT x NT tiles of 16 x 16, to C.  They change places through `lds` (the wave's own, 16 * MT * 16 * NT elements / PARTS,
// 16-byte aligned), so that a lane stores 16 bytes of a row; for `accumulate` C comes in the same way first.  A row's 16-byte
// pieces lie at piece ^ row there: the 16 rows that a wave writes at a time meet different banks.
//   rows, cols: how many of the wave's rows and columns there are;  c: element (0, 0)
template <typename T, bool ADD, int PARTS, int MT, int NT>
__device__ __forceinline__ void store_typed(const ScaledGemm& g, v4f (&acc)[NT][MT], uint8_t* lds, int64_t c, int rows, int cols) {
    constexpr int ES = int(sizeof(T)), kRowBytes = NT * 16 * ES, kPieces = kRowBytes / 16, kMask = kPieces < 16 ? kPieces - 1 : 15;
    constexpr int kPartRows = MT * 16 / PARTS, kPer = 16 / ES;
    static_assert(MT % PARTS == 0 && kPartRows * kPieces % 64 == 0, "whole rounds of the wave");
    const int lane = threadIdx.x & 63, q = lane >> 4, x16 = lane & 15;
    uint8_t* const out = static_cast<uint8_t*>(g.c) + c * ES;
    const int64_t ld = g.ldc * ES;
    const bool whole = rows >= MT * 16 && cols >= NT * 16;
    // piece x of the part, in the order of LDS: row, column, how many of its elements there are
    auto each = [&](int part, auto&& f) {
#pragma unroll 1
        for (int x = lane; x < kPartRows * kPieces; x += 64) {
            const int r = x / kPieces, col = ((x % kPieces) ^ (r & kMask)) * kPer;
            const int have = part * kPartRows + r < rows ? cols - col : 0;
            f(reinterpret_cast<v4i32*>(lds + x * 16), reinterpret_cast<T*>(out + (part * kPartRows + r) * ld) + col, have);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    // where this lane's results of tile (0, j) lie: tile (i, j) is a constant further
    uint32_t at[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
        at[j] = ES == 4 ? uint32_t(x16 * kRowBytes + (((j * 4 + q) ^ (x16 & kMask)) << 4))
                        : uint32_t(x16 * kRowBytes + (((j * 2 + (q >> 1)) ^ (x16 & kMask)) << 4) + (q & 1) * 8);
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
        if constexpr (ADD) {
            each(part, [&](v4i32* piece, const T* p, int have) {
                union { v4i32 v; T e[kPer]; } u;
                u.v = v4i32{0, 0, 0, 0};
                if (have >= kPer) u.v = *reinterpret_cast<const v4i32_any*>(p);
                else
#pragma unroll
                    for (int i = 0; i < kPer; ++i)
                        if (i < have) u.e[i] = p[i];
                *piece = u.v;
            });
        }
#pragma unroll
        for (int i = 0; i < MT / PARTS; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                uint8_t* p = lds + at[j] + i * 16 * kRowBytes;
                v4f s = acc[j][part * (MT / PARTS) + i];
                if constexpr (ES == 4) {
                    if constexpr (ADD) s += *reinterpret_cast<const v4f*>(p);
                    *reinterpret_cast<v4f*>(p) = s;
                } else {
                    if constexpr (ADD) s += unpack4<T>(*reinterpret_cast<const uint2*>(p));
                    *reinterpret_cast<uint2*>(p) = make_uint2(pack2<T>(s[0], s[1]), pack2<T>(s[2], s[3]));
                }
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (whole) {
            // nothing to check, eight pieces of a lane on their way together
            constexpr int kRounds = kPartRows * kPieces / 64, kBatch = kRounds % 8 == 0 ? 8 : kRounds;
            constexpr int kStepRows = 64 / kPieces;
            static_assert(64 % kPieces == 0, "a round is whole rows");
            const int r0 = lane / kPieces;
#pragma unroll 1
            for (int x = 0; x < kRounds; x += kBatch) {
                v4i32 v[kBatch];
#pragma unroll
                for (int u = 0; u < kBatch; ++u) v[u] = *reinterpret_cast<const v4i32*>(lds + (x + u) * 1024 + lane * 16);
#pragma unroll
                for (int u = 0; u < kBatch; ++u) {
                    const int r = (x + u) * kStepRows + r0;
                    *reinterpret_cast<v4i32_any*>(out + (part * kPartRows + r) * ld + (((lane % kPieces) ^ (r & kMask)) << 4)) = v[u];
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        } else {
            each(part, [&](const v4i32* piece, T* p, int have) {
                union { v4i32 v; T e[kPer]; } u;
                u.v = *piece;
                if (have >= kPer) *reinterpret_cast<v4i32_any*>(p) = u.v;
                else
#pragma unroll
                    for (int i = 0; i < kPer; ++i)
                        if (i < have) p[i] = u.e[i];
            });
        }
    }
}
// WIDE: C is float32; else it has 16 bits, or is a plane of float32 for a part of k (CUT: such calls reach this kernel).  `lds` holds
// BYTES.  One copy of the code per type runs: the kernels' own is what fills the instruction cache.
template <bool WIDE, bool CUT, int BYTES, int MT, int NT>
__device__ __forceinline__ void store_results(const ScaledGemm& g, v4f (&acc)[NT][MT], uint8_t* lds, int64_t c, int rows, int cols) {
    constexpr int kSize = MT * NT * 256;
    constexpr int P4 = kSize * 4 <= BYTES ? 1 : kSize * 2 <= BYTES ? 2 : 4, P2 = kSize * 2 <= BYTES ? 1 : 2;
    static_assert(kSize * 4 / P4 <= BYTES && kSize * 2 / P2 <= BYTES, "room for a part");
    const bool add = g.accumulate != 0;
    if constexpr (WIDE) {
        if (add) store_typed<float, true, P4>(g, acc, lds, c, rows, cols);
        else store_typed<float, false, P4>(g, acc, lds, c, rows, cols);
        return;
    }
    constexpr int PARTS = P2;
    if (CUT && g.c_type == OZ_F32) {
        store_typed<float, false, P4>(g, acc, lds, c, rows, cols);
    } else if (g.c_type == OZ_BF16) {
        if (add) store_typed<bf16_t, true, PARTS>(g, acc, lds, c, rows, cols);
        else store_typed<bf16_t, false, PARTS>(g, acc, lds, c, rows, cols);
    } else {
        if (add) store_typed<f16_t, true, PARTS>(g, acc, lds, c, rows, cols);
        else store_typed<f16_t, false, PARTS>(g, acc, lds, c, rows, cols);
    }
}

}  // namespace oz
