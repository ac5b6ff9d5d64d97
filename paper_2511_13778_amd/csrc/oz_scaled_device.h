// Device code that the kernels on 8-bit block-scaled operands and on sorted rows share.
#pragma once

#include "oz_scaled.h"

namespace oz {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i32 __attribute__((ext_vector_type(4)));
typedef int v8i32 __attribute__((ext_vector_type(8)));

// Sums over the lanes up to each, by a whole wave: within rows of 16 lanes, then rows 0 and 2 into the next, then the lower half into the upper.
// Six additions; shuffles go through LDS and take its latency each (groups' offsets loaded and scanned twice, by shuffles: experts' products
// of 2296 rows, 2345 x 334, 13.6 us, once and so 11.2).
__device__ __forceinline__ int sum_up_to(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
    return x;
}

__device__ __forceinline__ int clamp_offset(const int32_t* offsets, int g, int rows) { return min(max(offsets[g], 0), rows); }

// A piece of the rows: the groups are cut into pieces of SIZE rows, each group for itself; group `groups` holds the rows behind the last
// one.  blocks_before: 128-row blocks of the groups before.
struct GroupPiece {
    int group, row, end;      // rows row .. min(row + SIZE, end) - 1; group < 0: no such piece
    int blocks_before;
};

// The pieces of a call, by whole waves: a lane has a group (of the first 64; more are read again).  Offsets that are not ascending
// or pass `rows` give wrong pieces, none outside 0 .. rows.
template <int SIZE>
struct GroupPieces {
    const int32_t* offsets;
    int groups, rows;
    int lo, hi, upto;         // a lane's group: its rows, and the pieces of the groups up to it
    int count;                // of all

    __device__ __forceinline__ void load(int g0, int before) {
        const int g = g0 + int(threadIdx.x & 63);
        lo = clamp_offset(offsets, min(g, groups), rows);
        hi = g < groups ? max(lo, clamp_offset(offsets, min(g + 1, groups), rows)) : rows;
        if (g > groups) lo = hi = 0;
        upto = before + sum_up_to((hi - lo + SIZE - 1) / SIZE);
    }
    __device__ __forceinline__ int last() const { return __builtin_amdgcn_readlane(upto, 63); }
    __device__ __forceinline__ GroupPieces(const int32_t* o, int n, int r) : offsets(o), groups(n), rows(r) {
        load(0, 0);
        count = last();
        if (groups >= 64) {
            for (int g0 = 64; g0 <= groups; g0 += 64) {
                load(g0, count);
                count = last();
            }
            load(0, 0);
        }
    }
    template <bool BLOCKS>
    __device__ __forceinline__ GroupPiece find(int t) {
        int blocks = 0;
        for (int g0 = 0;;) {
            const unsigned long long has = __ballot(upto > t);
            const int blk = (hi - lo + kScaleBlock - 1) / kScaleBlock, blk_upto = BLOCKS ? sum_up_to(blk) : 0;
            if (has) {
                const int src = __builtin_ctzll(has), in = __builtin_amdgcn_readlane(lo, src), out = __builtin_amdgcn_readlane(hi, src);
                const int first = __builtin_amdgcn_readlane(upto, src) - (out - in + SIZE - 1) / SIZE;
                return GroupPiece{g0 + src, in + (t - first) * SIZE, out,
                                  BLOCKS ? blocks + __builtin_amdgcn_readlane(blk_upto, src) - (out - in + kScaleBlock - 1) / kScaleBlock : 0};
            }
            if (BLOCKS) blocks += __builtin_amdgcn_readlane(blk_upto, 63);
            g0 += 64;
            if (g0 > groups) return GroupPiece{-1, 0, 0, 0};
            load(g0, last());
        }
    }
};

// Rows of group g, and the 128-row blocks of the groups before it.
struct GroupSpan { int count, blocks_before; };
__device__ __forceinline__ GroupSpan group_span(const int32_t* __restrict__ offsets, int g, int rows) {
    const int lane = threadIdx.x & 63;
    int blocks = 0, rows_of = 0;
    for (int q0 = 0; q0 <= g; q0 += 64) {
        const int q = q0 + lane;
        const int lo = clamp_offset(offsets, min(q, g), rows), hi = max(lo, clamp_offset(offsets, min(q, g) + 1, rows));
        if (q < g) blocks += (hi - lo + kScaleBlock - 1) / kScaleBlock;
        if (q == g) rows_of = hi - lo;
    }
    return GroupSpan{__builtin_amdgcn_readlane(sum_up_to(rows_of), 63), __builtin_amdgcn_readlane(sum_up_to(blocks), 63)};
}

// ---- elements of 32 and 16 bits; a conversion to fewer bits rounds to nearest even ----------------
typedef __bf16 bf16_t;
typedef _Float16 f16_t;

template <typename T>
__device__ __forceinline__ float to_float(T x) { return static_cast<float>(x); }
template <typename T>
__device__ __forceinline__ void put(T* p, float x) { *p = static_cast<T>(x); }

// 16 bytes of a row that starts at any element: global loads and stores need no more than the element's own alignment.
typedef v4i32 __attribute__((aligned(2), may_alias)) v4i32_any;

// N consecutive elements of a row, from p on, of which `have` are there before its end (any number, also none or less); `cols` is the row's length.
// fetch_row sends for them, settle_row waits for them and puts zeros from `have` on: several rows are on their way together when all are
// fetched first.  16-byte loads throughout; a row's last piece is read from N before its end and moved down (rows shorter than N: element
// by element).  STREAM: read once, past the caches.
template <int N, typename T>
struct RowPiece {
    static constexpr int kVec = N * int(sizeof(T)) / 16, kWords = 4 * kVec;
    static_assert(kVec * 16 == N * int(sizeof(T)), "whole 16-byte loads");
    union { v4i32 v[kVec]; uint32_t w[kWords]; T e[N]; };
};
// cols >= N
template <int N, bool STREAM = false, typename T>
__device__ __forceinline__ void fetch_long_row(const T* __restrict__ p, int have, RowPiece<N, T>& r) {
#pragma unroll
    for (int i = 0; i < r.kVec; ++i) r.v[i] = v4i32{0, 0, 0, 0};
    if (have <= 0) return;
    const v4i32_any* at = reinterpret_cast<const v4i32_any*>(p - max(N - have, 0));
#pragma unroll
    for (int i = 0; i < r.kVec; ++i) r.v[i] = STREAM ? __builtin_nontemporal_load(at + i) : at[i];
}
template <int N, typename T>
__device__ __forceinline__ void fetch_short_row(const T* __restrict__ p, int have, RowPiece<N, T>& r) {
#pragma unroll
    for (int i = 0; i < r.kVec; ++i) r.v[i] = v4i32{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < have) r.e[i] = p[i];
}
template <int N, bool STREAM = false, typename T>
__device__ __forceinline__ void fetch_row(const T* __restrict__ p, int have, int cols, RowPiece<N, T>& r) {
    if (cols >= N) fetch_long_row<N, STREAM>(p, have, r);
    else fetch_short_row(p, have, r);
}
// 0 < have < N <= cols
template <int N, typename T>
__device__ __forceinline__ void move_down(RowPiece<N, T>& r, int have) {
    constexpr int kPer = 4 / int(sizeof(T));
    const int down = (N - have) / kPer;
#pragma unroll
    for (int step = r.kWords / 2; step > 0; step /= 2)
#pragma unroll
        for (int i = 0; i < r.kWords; ++i) r.w[i] = (down & step) ? (i + step < r.kWords ? r.w[i + step] : 0u) : r.w[i];
    if (kPer == 2 && (have & 1)) {                        // N is even
#pragma unroll
        for (int i = 0; i < r.kWords; ++i) r.w[i] = (r.w[i] >> 16) | (i + 1 < r.kWords ? r.w[i + 1] << 16 : 0u);
    }
}
template <int N, typename T>
__device__ __forceinline__ void settle_row(RowPiece<N, T>& r, int have, int cols) {
    if (have > 0 && have < N && cols >= N) move_down(r, have);
}
template <int N, typename T>
__device__ __forceinline__ void as_floats(RowPiece<N, T> r, int have, int cols, float (&x)[N]) {
    settle_row(r, have, cols);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = to_float(r.e[i]);
}
template <int N, bool STREAM = false, typename T>
__device__ __forceinline__ void load_row(const T* __restrict__ p, int have, int cols, float (&x)[N]) {
    RowPiece<N, T> r;
    fetch_row<N, STREAM>(p, have, cols, r);
    as_floats(r, have, cols, x);
}

// N floats to consecutive elements of a row, `have` of them.
template <int N, bool STREAM = false, typename T>
__device__ __forceinline__ void store_row(T* __restrict__ p, int have, const float (&x)[N]) {
    if (have >= N) {
        constexpr int kVec = N * int(sizeof(T)) / 16;
        union { v4i32 v[kVec]; T e[N]; } u;
#pragma unroll
        for (int i = 0; i < N; ++i) put(&u.e[i], x[i]);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            if constexpr (STREAM) __builtin_nontemporal_store(u.v[i], reinterpret_cast<v4i32_any*>(p) + i);
            else reinterpret_cast<v4i32_any*>(p)[i] = u.v[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < have) put(p + i, x[i]);
    }
}

}  // namespace oz
