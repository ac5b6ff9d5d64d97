// Rows sorted by group (tokens by expert), gathered, and combined back with their weights.
//
// Sort: a stable counting sort of the choices by expert.  Within 64 choices the lanes of one expert find each other with one ballot
// per bit of its number; rank = lanes before, plus what the wave, the waves before and the blocks before counted of that
// expert.  The only atomics add whole numbers: the order is the same in every run.  Few choices are bound by a chain of latencies (264:
// 3.8 us), 65536 take 8.3 in two launches.
// Gather and combine move rows; what bounds them is memory: 16384 tokens of 2048 bfloat16 with four choices 53 us each (6.3 and 6.1 TB/s),
// the gradient, which reads dY and the rows and writes rows, 95 (6.4).  Rows that are read or written once are streamed past the
// caches: at that size all three lose 12 to 22 % without, up to 8192 x 2 choices both ways are level.
#include <algorithm>

#include "oz_scaled_device.h"

namespace oz {

namespace {

constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64;
constexpr int kRounds = 8;                // 64s of choices that a wave has on their way at a time

// Choices of a workgroup: all of them up to 4096, which one launch sorts; else 1024 (two rounds of a wave), more where that would be over
// 256 workgroups.  Up to 4096 a wave's choices stay in registers between counting and placing (96 choices of 32 experts 5.4 -> 3.8 us).
int sort_block(int64_t choices) {
    if (choices <= kSortThreads * kRounds) return int((std::max<int64_t>(choices, 1) + kSortThreads - 1) / kSortThreads * kSortThreads);
    const int64_t per = (choices + 255) / 256;
    return int(per <= 2 * kSortThreads ? 2 * kSortThreads : (per + kSortThreads - 1) / kSortThreads * kSortThreads);
}

struct SortArgs {
    const void* chosen;
    int32_t *offsets, *order, *place, *counts;      // counts[block][expert]
    int choices, experts, bits, per_block, blocks;
    bool wide;
};

// Lanes of this wave with the same expert (0 for none).
__device__ __forceinline__ unsigned long long same_expert(int e, int bits) {
    unsigned long long m = __ballot(e >= 0);
    for (int b = 0; b < bits; ++b) {
        const unsigned long long set = __ballot((e >> b) & 1);
        m &= ((e >> b) & 1) ? set : ~set;
    }
    return e >= 0 ? m : 0;
}

// What a wave holds of its choices: 64 per round.
struct Choices {
    int e[kRounds];                          // expert or -1
    unsigned long long same[kRounds];        // lanes with the same expert
};
__device__ __forceinline__ void load_choices(const SortArgs& p, int from, int to, Choices& c) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int u = 0; u < kRounds; ++u) {
        const int i = from + u * 64 + lane;
        int64_t id = -1;
        if (i < to) id = p.wide ? static_cast<const int64_t*>(p.chosen)[i] : int64_t(static_cast<const int32_t*>(p.chosen)[i]);
        c.e[u] = id >= 0 && id < p.experts ? int(id) : -1;
    }
#pragma unroll
    for (int u = 0; u < kRounds; ++u)
        if (from + u * 64 < to) c.same[u] = same_expert(c.e[u], p.bits);
}

// f(index, expert or -1, lanes with the same expert) for this wave's choices, 64 at a time, in their order; all lanes come along, also those
// behind the last.  held: what `c` has of them already (KEEP: they are no more than it holds).
template <bool KEEP, typename F>
__device__ __forceinline__ void each_choice(const SortArgs& p, int from, int to, Choices& c, bool held, F&& f) {
    const int lane = threadIdx.x & 63;
    for (int i0 = from; i0 < to; i0 += 64 * kRounds) {
        if (!KEEP || !held) load_choices(p, i0, to, c);
#pragma unroll
        for (int u = 0; u < kRounds; ++u)
            if (i0 + u * 64 < to) f(i0 + u * 64 + lane, c.e[u], c.same[u]);
        if (KEEP) break;
    }
}

__device__ __forceinline__ void wave_part(const SortArgs& p, int& from, int& to) {
    const int begin = int(blockIdx.x) * p.per_block, end = min(begin + p.per_block, p.choices), per_wave = p.per_block / kSortWaves;
    from = begin + int(threadIdx.x >> 6) * per_wave;
    to = min(from + per_wave, end);
}

// count[wave][expert] of this block's choices; waves take consecutive parts of it
template <bool KEEP>
__device__ __forceinline__ void count_block(const SortArgs& p, int32_t* count, Choices& c) {
    for (int i = threadIdx.x; i < kSortWaves * p.experts; i += kSortThreads) count[i] = 0;
    __syncthreads();
    int from, to;
    wave_part(p, from, to);
    int32_t* mine = count + int(threadIdx.x >> 6) * p.experts;
    const unsigned long long below = (1ull << (threadIdx.x & 63)) - 1;
    each_choice<KEEP>(p, from, to, c, false, [&](int, int e, unsigned long long m) {
        if (m && (m & below) == 0) mine[e] += __popcll(m);       // one lane per expert
        __builtin_amdgcn_wave_barrier();
    });
    __syncthreads();
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortArgs p) {
    extern __shared__ int32_t count[];
    Choices c;
    count_block<false>(p, count, c);
    for (int e = threadIdx.x; e < p.experts; e += kSortThreads) {
        int sum = 0;
        for (int w = 0; w < kSortWaves; ++w) sum += count[w * p.experts + e];
        p.counts[int64_t(blockIdx.x) * p.experts + e] = sum;
    }
}

// Where each choice goes.  Every workgroup adds up the counts of all blocks by itself: its waves take an eighth of the blocks each.
template <bool KEEP>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(SortArgs p) {
    extern __shared__ int32_t count[];                    // [waves][experts], then the tables below
    __shared__ int32_t wave_total[kSortWaves];
    int32_t* total = count + kSortWaves * p.experts;      // all choices of an expert, then its first slot
    int32_t* before = total + p.experts;                  // those in blocks before this one
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, block = blockIdx.x;
    if (p.blocks > 1) {
        for (int e = threadIdx.x; e < 2 * p.experts; e += kSortThreads) total[e] = 0;
        __syncthreads();
        const int share = (p.blocks + kSortWaves - 1) / kSortWaves, b0 = wave * share, b1 = min(b0 + share, p.blocks);
        for (int e = lane; e < p.experts; e += 64) {
            int all = 0, prev = 0;
#pragma unroll 8
            for (int b = b0; b < b1; ++b) {
                const int c = p.counts[int64_t(b) * p.experts + e];
                all += c;
                prev += b < block ? c : 0;
            }
            atomicAdd(&total[e], all);                    // whole numbers: in any order the same
            atomicAdd(&before[e], prev);
        }
    }
    Choices held;
    count_block<KEEP>(p, count, held);
    if (p.blocks == 1) {
        for (int e = threadIdx.x; e < p.experts; e += kSortThreads) {
            int sum = 0;
            for (int w = 0; w < kSortWaves; ++w) sum += count[w * p.experts + e];
            total[e] = sum;
            before[e] = 0;
        }
        __syncthreads();
    }
    // exclusive prefix over the experts, 512 at a time
    int carry = 0;
    for (int e0 = 0; e0 < p.experts; e0 += kSortThreads) {
        const int e = e0 + threadIdx.x;
        const int mine = e < p.experts ? total[e] : 0;
        const int sum = sum_up_to(mine);
        if (lane == 63) wave_total[wave] = sum;
        __syncthreads();
        int base = carry;
        for (int w = 0; w < wave; ++w) base += wave_total[w];
        for (int w = 0; w < kSortWaves; ++w) carry += wave_total[w];
        if (e < p.experts) {
            const int first = base + sum - mine;
            if (block == 0) p.offsets[e] = first;
            // first slot of each wave's choices
            int at = first + before[e];
            for (int w = 0; w < kSortWaves; ++w) {
                const int c = count[w * p.experts + e];
                count[w * p.experts + e] = at;
                at += c;
            }
        }
        __syncthreads();
    }
    const int live = carry;
    if (block == 0 && threadIdx.x == 0) p.offsets[p.experts] = live;
    int32_t* next = count + wave * p.experts;
    int from, to;
    wave_part(p, from, to);
    const unsigned long long below = (1ull << lane) - 1;
    each_choice<KEEP>(p, from, to, held, true, [&](int i, int e, unsigned long long m) {
        int slot = -1;
        if (m) slot = next[e] + __popcll(m & below);
        __builtin_amdgcn_wave_barrier();
        if (m && (m & below) == 0) next[e] += __popcll(m);
        __builtin_amdgcn_wave_barrier();
        if (i < to) {
            p.place[i] = slot;
            if (slot >= 0) p.order[slot] = i;
            if (i >= live) p.order[i] = -1;
        }
    });
}

// ---- rows ---------------------------------------------------------------------------------------

constexpr int kUnitVecs = 4;              // 16-byte loads a lane has in flight: a wave moves 4 KB of a row

struct GatherArgs {
    const uint8_t* x;
    uint8_t* y;
    int64_t ldx, ldy;                     // bytes
    const int32_t *order, *place;
    int tokens, topk, row_bytes, pieces;
    int per;                              // choices of a token that a wave writes
};

// A wave per 4 KB of a token's row, which it reads once and writes for each choice: from the slots' side every choice would read it again,
// long after it has left L2 (65536 slots of 4 KB 76 us that way, 61 this).  Few tokens have a wave per choice (33 tokens with 8
// choices 2.7 us, 5 with one wave for all).  grid.y: choices / per.  T: 16 bytes, at any element's address, or an element where a row is shorter; a row's last 16 bytes may
// overlap those before them, which carry the same there.
template <typename T>
__global__ __launch_bounds__(256) void gather_rows_kernel(GatherArgs p) {
    const uint32_t id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = int(id / uint32_t(p.pieces)), piece = int(id - uint32_t(t) * uint32_t(p.pieces)), lane = threadIdx.x & 63;
    if (t >= p.tokens) return;
    const int slots = p.tokens * p.topk, from = piece * 4096, to = min(from + 4096, p.row_bytes);
    const uint8_t* x = p.x + int64_t(t) * p.ldx;
    constexpr int kStep = 64 * int(sizeof(T));
    for (int at = from + lane * int(sizeof(T)); at < to; at += kStep * kUnitVecs) {
        T v[kUnitVecs];
        int pos[kUnitVecs];
#pragma unroll
        for (int u = 0; u < kUnitVecs; ++u) {
            pos[u] = min(at + u * kStep, p.row_bytes - int(sizeof(T)));
            v[u] = T{};
            if (at + u * kStep < to) v[u] = *reinterpret_cast<const T*>(x + pos[u]);
        }
        for (int j = int(blockIdx.y) * p.per; j < min((int(blockIdx.y) + 1) * p.per, p.topk); ++j) {
            const int c = t * p.topk + j, s = p.place[c];
            if (s >= 0 && s < slots) {
                uint8_t* y = p.y + int64_t(s) * p.ldy;
#pragma unroll
                for (int u = 0; u < kUnitVecs; ++u)
                    if (at + u * kStep < to) __builtin_nontemporal_store(v[u], reinterpret_cast<T*>(y + pos[u]));
            }
            if (p.order[c] < 0) {         // slot c belongs to no choice
                uint8_t* y = p.y + int64_t(c) * p.ldy;
#pragma unroll
                for (int u = 0; u < kUnitVecs; ++u)
                    if (at + u * kStep < to) *reinterpret_cast<T*>(y + pos[u]) = T{};
            }
        }
    }
}

struct CombineArgs {
    const void *x, *dy;
    void *y, *dx;
    int64_t ldx, ldy, lddy, lddx;
    const int32_t *order, *place;
    const float* weights;
    float* dweights;
    int tokens, topk, cols, slots, pieces;
};

// A wave per 512 columns of a token; the choices' rows four at a time, all of which are on their way before the first is added.
template <typename T>
__global__ __launch_bounds__(256) void combine_rows_kernel(CombineArgs p) {
    const uint32_t id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = int(id / uint32_t(p.pieces)), piece = int(id - uint32_t(t) * uint32_t(p.pieces)), lane = threadIdx.x & 63;
    if (t >= p.tokens) return;
    const int col = piece * 512 + lane * 8, have = p.cols - col;
    const T* x = static_cast<const T*>(p.x);
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int j0 = 0; j0 < p.topk; j0 += 4) {
        RowPiece<8, T> v[4];
        float w[4];
        bool live[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t c = int64_t(t) * p.topk + j0 + u;
            const int s = j0 + u < p.topk ? p.place[c] : -1;
            live[u] = s >= 0 && s < p.slots;
            w[u] = live[u] && p.weights ? p.weights[c] : 1.0f;
            fetch_row<8, true>(x + int64_t(live[u] ? s : 0) * p.ldx + col, live[u] ? have : 0, p.cols, v[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (live[u]) {
                float e[8];
                as_floats(v[u], have, p.cols, e);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] = fmaf(w[u], e[i], sum[i]);
            }
    }
    store_row<8>(static_cast<T*>(p.y) + int64_t(t) * p.ldy + col, have, sum);
}

// A wave per choice: the choices of a token lie in one workgroup and find its dY in the cache.  The product of dY and the row is the
// wave's own sum, lane by lane and then over the lanes in one order: no atomics.
template <typename T>
__global__ __launch_bounds__(256) void combine_grad_kernel(CombineArgs p) {
    const uint32_t c = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (c >= uint32_t(p.slots)) return;
    const int s = p.place[c];
    const bool live = s >= 0 && s < p.slots;
    const float w = live && p.weights ? p.weights[c] : 1.0f;
    const T* dy = static_cast<const T*>(p.dy) + int64_t(c / uint32_t(p.topk)) * p.lddy;
    const T* x = static_cast<const T*>(p.x) + int64_t(live ? s : 0) * p.ldx;
    T* dx = static_cast<T*>(p.dx) + int64_t(live ? s : 0) * p.lddx;
    float dot = 0.0f;
    if (live) {
        for (int col = lane * 8; col < p.cols; col += 1024) {
            RowPiece<8, T> gp[2], vp[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int at = col + u * 512;
                fetch_row<8>(dy + at, p.cols - at, p.cols, gp[u]);
                if (p.dweights) fetch_row<8, true>(x + at, p.cols - at, p.cols, vp[u]);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int at = col + u * 512;
                if (at < p.cols) {
                    float g[8], out[8];
                    as_floats(gp[u], p.cols - at, p.cols, g);
                    if (p.dweights) {
                        float v[8];
                        as_floats(vp[u], p.cols - at, p.cols, v);
#pragma unroll
                        for (int i = 0; i < 8; ++i) dot = fmaf(g[i], v[i], dot);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) out[i] = w * g[i];
                    store_row<8, true>(dx + at, p.cols - at, out);
                }
            }
        }
        for (int d = 32; d > 0; d >>= 1) dot += __shfl_xor(dot, d);
    }
    if (p.dweights && lane == 0) p.dweights[c] = dot;
    if (p.order[c] < 0) {                 // slot c belongs to no choice
        const float none[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        T* row = static_cast<T*>(p.dx) + int64_t(c) * p.lddx;
        for (int col = lane * 8; col < p.cols; col += 512) store_row<8>(row + col, p.cols - col, none);
    }
}

template <typename T>
void combine_typed(hipStream_t st, CombineArgs p) {
    p.pieces = (p.cols + 511) / 512;
    const int64_t waves = int64_t(p.tokens) * p.pieces;
    hipLaunchKernelGGL(combine_rows_kernel<T>, dim3(unsigned((waves + 3) / 4)), dim3(256), 0, st, p);
}

template <typename T>
void combine_grad_typed(hipStream_t st, CombineArgs p) {
    hipLaunchKernelGGL(combine_grad_kernel<T>, dim3(unsigned((int64_t(p.slots) + 3) / 4)), dim3(256), 0, st, p);
}

}  // namespace

size_t sort_tokens_bytes(int64_t choices, int64_t experts) {
    const int64_t per = sort_block(choices), blocks = (choices + per - 1) / per;
    return blocks > 1 ? size_t(blocks) * size_t(experts) * 4 : 0;
}

void launch_sort_tokens(hipStream_t st, int choices, int experts, const void* chosen, bool wide, int32_t* offsets, int32_t* order,
                        int32_t* place, int32_t* ws) {
    SortArgs p{chosen, offsets, order, place, ws, choices, experts, 0, sort_block(choices), 0, wide};
    while ((1 << p.bits) < experts) ++p.bits;
    p.blocks = choices > 0 ? (choices + p.per_block - 1) / p.per_block : 1;
    if (p.blocks > 1)
        hipLaunchKernelGGL(sort_count_kernel, dim3(p.blocks), dim3(kSortThreads), size_t(kSortWaves) * experts * 4, st, p);
    const size_t lds = size_t(kSortWaves + 2) * experts * 4;
    if (p.per_block <= kSortThreads * kRounds) hipLaunchKernelGGL(sort_place_kernel<true>, dim3(p.blocks), dim3(kSortThreads), lds, st, p);
    else hipLaunchKernelGGL(sort_place_kernel<false>, dim3(p.blocks), dim3(kSortThreads), lds, st, p);
}

void launch_gather_rows(hipStream_t st, int tokens, int topk, int cols, int elem_bytes, const void* x, int64_t ldx, const int32_t* order,
                        const int32_t* place, void* y, int64_t ldy) {
    GatherArgs p{static_cast<const uint8_t*>(x), static_cast<uint8_t*>(y), ldx * elem_bytes, ldy * elem_bytes, order, place, tokens, topk,
                 cols * elem_bytes, 0, topk};
    p.pieces = (p.row_bytes + 4095) / 4096;
    if (int64_t(tokens) * p.pieces < 4096) p.per = 1;
    const dim3 grid(unsigned((int64_t(tokens) * p.pieces + 3) / 4), unsigned(topk / p.per));
    if (p.row_bytes >= 16) hipLaunchKernelGGL(gather_rows_kernel<v4i32_any>, grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL(gather_rows_kernel<uint16_t>, grid, dim3(256), 0, st, p);
}

void launch_combine_rows(hipStream_t st, int tokens, int topk, int cols, int type, const void* x, int64_t ldx, int slots, const int32_t* place,
                         const float* weights, void* y, int64_t ldy) {
    CombineArgs p{};
    p.x = x; p.ldx = ldx; p.y = y; p.ldy = ldy; p.place = place; p.weights = weights;
    p.tokens = tokens; p.topk = topk; p.cols = cols; p.slots = slots;
    if (type == OZ_F32) combine_typed<float>(st, p);
    else if (type == OZ_BF16) combine_typed<bf16_t>(st, p);
    else combine_typed<f16_t>(st, p);
}

void launch_combine_grad(hipStream_t st, int tokens, int topk, int cols, int type, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                         int slots, const int32_t* order, const int32_t* place, const float* weights, void* dx, int64_t lddx, float* dweights) {
    CombineArgs p{};
    p.dy = dy; p.lddy = lddy; p.x = x; p.ldx = ldx; p.dx = dx; p.lddx = lddx; p.order = order; p.place = place; p.weights = weights;
    p.dweights = dweights; p.tokens = tokens; p.topk = topk; p.cols = cols; p.slots = slots;
    if (type == OZ_F32) combine_grad_typed<float>(st, p);
    else if (type == OZ_BF16) combine_grad_typed<bf16_t>(st, p);
    else combine_grad_typed<f16_t>(st, p);
}

}  // namespace oz
