// Product with weights in 4 bits for few rows of x: what bounds it is the read of the weights.
//
// A workgroup has 16 R rows of W and 16 rows of x; its waves share k, in runs of blocks of 128, and add up their sums through LDS in the waves'
// order.  code - 8 is exact in x's 16-bit type, and goes with x into v_mfma_f32_16x16x32 (float32 x as three bfloat16 parts, exactly); scales
// are applied to each group's sum, in 32 bits, so a result of 16 bits has one rounding, the last.  The sums of x that zero points need are one
// more matrix instruction, with a matrix of ones.  One row of 4096 x 4096 bfloat16: 5.1 us, of which a launch is 2.4; of 8192 x 8192 10 (3.4 TB/s); 96 rows of 32
// experts, 2048 x 2048: 18 (3.9 TB/s).
#pragma once

#include <algorithm>
#include <type_traits>

#include "oz_layer.h"
#include "oz_packed_plan.h"
#include "oz_scaled_device.h"

namespace oz {

namespace {

typedef uint32_t v4u32 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = kPackedBlock;     // of k that a wave takes at a time

// Eight codes as the matrix instruction takes them, in the order 0 4 1 5 2 6 3 7 (x's elements in the same): float16 and EXACT: code - 8;
// bfloat16 else: 128 + code, a third of the instructions, and what is too much comes off the sums.
template <typename W, bool EXACT>
__device__ __forceinline__ void widen_codes(uint32_t codes, uint32_t (&w)[4]) {
    if constexpr (std::is_same_v<W, f16_t>) {
        // 1024 + code, whose last bits are the code's
        const f16x2 less = {f16_t(1032.0f), f16_t(1032.0f)};
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, ((codes >> (4 * i)) & 0x000F000Fu) | 0x64006400u) - less);
    } else if constexpr (EXACT) {
        const uint32_t even = codes & 0x0F0F0F0Fu, odd = (codes >> 4) & 0x0F0F0F0Fu;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t of = i % 2 ? odd : even;
            const float a = float((of >> (i / 2 * 8)) & 0xFFu) - 8.0f, b = float((of >> (i / 2 * 8 + 16)) & 0xFFu) - 8.0f;
            w[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);       // whole numbers: the upper halves hold all of them
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = ((codes >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
    }
}

__device__ __forceinline__ v4f mfma16(const uint32_t (&a)[4], const uint32_t (&b)[4], v4f c, f16_t) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ v4f mfma16(const uint32_t (&a)[4], const uint32_t (&b)[4], v4f c, bf16_t) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight consecutive elements of a row of x, and as the matrix instruction takes them, in the codes' order: one part, three of float32.
template <typename X>
struct Eight {
    static constexpr int kParts = sizeof(X) == 4 ? 3 : 1, kWords = 2 * int(sizeof(X));
    using W = std::conditional_t<sizeof(X) == 4, bf16_t, X>;
    uint32_t e[kWords];
    __device__ __forceinline__ void load(const X* p) { __builtin_memcpy(e, p, sizeof(e)); }
    // What load(row + from) brought, moved down by `down` elements, zeros behind it.
    __device__ __forceinline__ void move_down(int down) {
        constexpr int kPer = 4 / int(sizeof(X));
#pragma unroll
        for (int step = kWords / 2; step > 0; step /= 2)
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                const uint32_t now = e[i], far = i + step < kWords ? e[i + step] : 0u;
                e[i] = (down & (step * kPer)) ? far : now;
            }
        if (kPer == 2) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                const uint32_t now = e[i], odd = (now >> 16) | (i + 1 < kWords ? e[i + 1] << 16 : 0u);
                e[i] = (down & 1) ? odd : now;
            }
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) e[i] = down >= 8 ? 0u : e[i];
    }
    __device__ __forceinline__ void parts(uint32_t (&w)[kParts][4]) const {
        if constexpr (kParts == 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[0][i] = __builtin_amdgcn_perm(e[i / 2 + 2], e[i / 2], i % 2 ? 0x07060302u : 0x05040100u);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t bits[2][3];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    // cut off, not rounded: what is left is exact, and no part is larger than the whole
                    float x = __uint_as_float(e[i + 4 * j]);
                    const bool fine = (e[i + 4 * j] & 0x7F800000u) != 0x7F800000u;
#pragma unroll
                    for (int p = 0; p < 3; ++p) {
                        bits[j][p] = __float_as_uint(x) & 0xFFFF0000u;
                        if (p == 0 && x != x) bits[j][0] = 0x7FC00000u;
                        x = fine ? x - __uint_as_float(bits[j][p]) : 0.0f;
                    }
                }
#pragma unroll
                for (int p = 0; p < 3; ++p) w[p][i] = __builtin_amdgcn_perm(bits[1][p], bits[0][p], 0x07060302u);
            }
        }
    }
};

template <typename T>
__device__ __forceinline__ void store4(T* p, int have, v4f v) {
    T t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) put(t + i, v[i]);
    if (have >= 4) {
        __builtin_memcpy(p, t, sizeof(t));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) p[i] = t[i];
    }
}
__device__ __forceinline__ void store_results(const PackedGemm& g, int64_t at, int have, v4f v) {
    if (g.y_type == OZ_F32) store4(static_cast<float*>(g.y) + at, have, v);
    else if (g.y_type == OZ_BF16) store4(static_cast<bf16_t*>(g.y) + at, have, v);
    else store4(static_cast<f16_t*>(g.y) + at, have, v);
}

// A scale or zero point of any of the three types, without a branch that would wait for what else is on its way: two halves of a float32, or the same 16
// bits twice.
struct ScaleLoad {
    const uint8_t* p;
    int shift, second;
    bool wide, bf16;
    __device__ __forceinline__ ScaleLoad(const void* q, int type)
        : p(static_cast<const uint8_t*>(q)), shift(type == OZ_F32 ? 2 : 1), second(type == OZ_F32 ? 2 : 0), wide(type == OZ_F32), bf16(type == OZ_BF16) {}
    struct Halves { uint16_t lo, hi; };
    __device__ __forceinline__ Halves fetch(int64_t at) const {
        const uint8_t* from = p + (at << shift);
        return Halves{*reinterpret_cast<const uint16_t*>(from), *reinterpret_cast<const uint16_t*>(from + second)};
    }
    __device__ __forceinline__ float value(Halves h) const {
        const float half = to_float(__builtin_bit_cast(f16_t, h.lo));
        return wide ? __uint_as_float(uint32_t(h.lo) | uint32_t(h.hi) << 16) : bf16 ? __uint_as_float(uint32_t(h.lo) << 16) : half;
    }
};

// Sums of code - 8 (or of 128 + code, less what is too much) say nothing where x has an infinity, or leave float32's range on the way to a result that lies
// in it.  Results that are not finite are therefore computed once more as they are defined, in 64 bits: sums of x * (scale * (code - zero)), here of N columns
// of the result from `col` on, over the eight columns of x from l0 on.
template <int N, typename X>
__device__ __forceinline__ void add_defined(const PackedGemm& g, int of, const X* x, int col, int l0, double (&sum)[N]) {
    if (l0 >= g.k) return;
    const ScaleLoad scales(g.w.scale, g.w.type), zeros(g.w.zero, g.w.type);
    uint32_t codes[N];
    double scale[N], zero[N];
#pragma unroll
    for (int c = 0; c < N; ++c) {
        const int64_t row = min(col + c, g.n - 1), at = of * g.w.scale_stride + int64_t(l0 >> g.w.shift) * g.w.scale_ld + row;
        codes[c] = *reinterpret_cast<const uint32_t*>(g.w.data + of * g.w.stride + row * g.w.ld + l0 / 2);
        scale[c] = scales.value(scales.fetch(at));
        zero[c] = g.w.zero ? zeros.value(zeros.fetch(at)) : 8.0f;
    }
    for (int i = 0; i < 8; ++i)
        if (l0 + i < g.k) {
            const double v = to_float(x[l0 + i]);
#pragma unroll
            for (int c = 0; c < N; ++c) sum[c] = fma(v, scale[c] * (double((codes[c] >> (4 * i)) & 15u) - zero[c]), sum[c]);
        }
}
// Every lane of a wave, with `s` the results of its row of x and four columns from `col` on.  One infinity among 64 x 8192 bfloat16 by 8192: 250 us instead of 27,
// one in each row 2260, many 280; a NaN 30.
template <typename X>
__device__ __forceinline__ void mend_results(const PackedGemm& g, int of, bool in, int row, int col, v4f& s) {
    int odd = 0;                              // which of them
#pragma unroll
    for (int i = 0; i < 4; ++i) odd |= in && !__builtin_isfinite(s[i]) ? 1 << i : 0;
    uint64_t left = __ballot(odd != 0);
    if (__builtin_expect(left == 0, true)) return;
    const int lane = threadIdx.x & 63;
    int seen = -1;
    while (left) {
        const int from = __builtin_ctzll(left), r = __builtin_amdgcn_readlane(row, from), c = __builtin_amdgcn_readlane(col, from);
        const int which = __builtin_amdgcn_readlane(odd, from);
        const X* const x = static_cast<const X*>(g.x) + int64_t(r) * g.ldx;
        left &= left - 1;
        if (r != seen) {
            // a NaN in a row of x makes all of its results NaN, which they are
            bool nan = false;
            for (int l0 = 0; l0 < g.k && !__any(nan); l0 += 512)
                for (int i = 0; i < 8; ++i) {
                    const float v = to_float(x[min(l0 + lane * 8 + i, g.k - 1)]);
                    nan = nan || v != v;
                }
            if (__any(nan)) {
                left &= ~__ballot(row == r);
                continue;
            }
            seen = r;
        }
        double sum[4] = {0.0, 0.0, 0.0, 0.0};
        // until all that are asked for are NaN, which they stay
        for (int l0 = 0, open = which; l0 < g.k && open; l0 += 512) {
            add_defined<4>(g, of, x, c, l0 + lane * 8, sum);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (__any(sum[i] != sum[i])) open &= ~(1 << i);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            for (int d = 1; d < 64; d *= 2) sum[i] += __shfl_xor(sum[i], d);
            s[i] = lane == from && (which >> i & 1) ? float(sum[i]) : s[i];
        }
    }
}

// 16 rows of x; R: 16s of rows of W.  PER: groups of columns in a block, whose sums are scaled apart.  EXACT: bfloat16 codes with nothing to come off the sums.
// That 128 + code is multiplied instead of code - 8 makes the sums 136 / 4.6 times as large and their 32-bit roundings with them: 4e-6 of a result, or
// 4e-5 where all of x has one sign, beside a rounding to bfloat16 of 2e-3.
template <typename X, int R, int PER, bool ZEROS, bool EXACT>
struct Shape {
    static constexpr int kAhead = 2;                                               // blocks whose weights are on their way together
    static constexpr int kX = sizeof(X) == 2 ? 2 : 1;                 // of them, those whose x is too
    static constexpr int kLoads = (kAhead * PER * 16 * R + 63) / 64, kScales = kLoads * 64;      // of a wave, in LDS
    static constexpr int kThreads = R * int(sizeof(X)) <= 4 ? 1024 : 512;
    static constexpr int kWaveBytes = std::max(16 * 16 * R, kScales * (ZEROS ? 2 : 1)) * 4;      // scales, and in the end the sums
};

template <typename X, int R, int PER, bool ZEROS, bool EXACT>
__global__ __launch_bounds__((Shape<X, R, PER, ZEROS, EXACT>::kThreads)) void packed_gemm_kernel(PackedGemm g, int strips) {
    using E = Eight<X>;
    using W = typename E::W;
    using S = Shape<X, R, PER, ZEROS, EXACT>;
    constexpr int kPer = PER, kEach = 4 / PER, kAhead = S::kAhead, kX = S::kX;
    constexpr bool SMALL = PER > 1;
    constexpr bool kSums = ZEROS || !EXACT;                           // sums of x are needed
    extern __shared__ __align__(16) float lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = int(blockDim.x) >> 6;
    const int q = lane >> 4, x16 = lane & 15;
    const int strip = int(blockIdx.x % unsigned(strips)), piece = int(blockIdx.x / unsigned(strips)), col0 = strip * 16 * R, cols = min(g.n - col0, 16 * R);
    int row0 = piece * 16, rows = min(g.m - row0, 16), of = 0;
    if (g.offsets) {
        GroupPieces<16> pieces(g.offsets, g.groups, g.m);
        const GroupPiece p = pieces.template find<false>(piece);
        if (p.group < 0) return;
        of = p.group;
        row0 = p.row;
        rows = min(p.end - p.row, 16);
    }
    const bool none = g.offsets && of >= g.groups;                    // rows behind the last group: zeros
    float* mine = lds + wave * (S::kWaveBytes / 4);
    v4f acc[R];
#pragma unroll
    for (int s = 0; s < R; ++s) acc[s] = v4f{0, 0, 0, 0};
    if (!none) {
        const int bytes = (g.k + 31) / 32 * 16;
        const uint8_t* w_row[R];
#pragma unroll
        for (int s = 0; s < R; ++s) w_row[s] = g.w.data + of * g.w.stride + int64_t(col0 + min(s * 16 + x16, cols - 1)) * g.w.ld;
        const X* const x_row = static_cast<const X*>(g.x) + int64_t(row0 + min(x16, rows - 1)) * g.ldx;
        const int blocks = (g.k + kBlock - 1) / kBlock, per = (blocks + waves - 1) / waves, begin = wave * per, end = min(begin + per, blocks);
        const ScaleLoad scales(g.w.scale, g.w.type), zeros(g.w.zero, g.w.type);
        uint32_t ones[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) ones[i] = uint32_t(__builtin_bit_cast(uint16_t, static_cast<W>(1.0f))) * 0x10001u;
        for (int b0 = begin; b0 < end; b0 += kAhead) {
            // What this chunk reads is sent for without a branch, which would wait; blocks behind the end are the last one again, and bytes behind a row's end
            // its last ones, whose columns have zeros in x.  (The next chunk's weights sent for before this one is multiplied: 3 to 14 % slower.)
            v4u32 codes[kAhead][R];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int s = 0; s < R; ++s) codes[u][s] = *reinterpret_cast<const v4u32*>(w_row[s] + min(min(b0 + u, end - 1) * 64 + q * 16, bytes - 16));
            // the blocks' scales, [block, group][row], for this wave alone
            ScaleLoad::Halves scale_bits[S::kLoads], zero_bits[ZEROS ? S::kLoads : 1];
#pragma unroll
            for (int y = 0; y < S::kLoads; ++y) {
                const int z = y * 64 + lane, row = z % (16 * R), p = z / (16 * R);
                const int64_t group = min(((b0 * kPer + p) * (kBlock / kPer)) >> g.w.shift, (g.k - 1) >> g.w.shift);
                const int64_t at = of * g.w.scale_stride + group * g.w.scale_ld + col0 + min(row, cols - 1);
                scale_bits[y] = scales.fetch(at);
                if constexpr (ZEROS) zero_bits[y] = zeros.fetch(at);
            }
            E x[kX][4];
            auto fetch = [&](int u, E (&n)[4]) {
                const int b = min(b0 + u, end - 1);
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    // which of the block's columns lane q's part of instruction v covers: any order that both operands share
                    n[v].load(x_row + min(b * kBlock + (SMALL ? v * 32 + q * 8 : q * 32 + v * 8), g.k - 8));
            };
#pragma unroll
            for (int u = 0; u < kX; ++u) fetch(u, x[u]);
#pragma unroll
            for (int y = 0; y < S::kLoads; ++y) {
                mine[y * 64 + lane] = scales.value(scale_bits[y]);
                if constexpr (ZEROS) mine[S::kScales + y * 64 + lane] = (EXACT ? 8.0f : -128.0f) - zeros.value(zero_bits[y]);
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int b = b0 + u;
                if (b >= end) break;
                E (&now)[4] = x[u % kX];
                if (u >= kX) fetch(u, now);
                uint32_t w[4][4];
                if ((b + 1) * kBlock > g.k) {
#pragma unroll
                    for (int v = 0; v < 4; ++v) now[v].move_down(max(b * kBlock + (SMALL ? v * 32 + q * 8 : q * 32 + v * 8) - (g.k - 8), 0));
                }
                // sums of x, once for all of W's rows
                constexpr bool kOnce = kSums && R > 1;
                v4f all[kOnce ? kPer : 1];
                if constexpr (kOnce) {
#pragma unroll
                    for (int p = 0; p < kPer; ++p) {
                        all[p] = v4f{0, 0, 0, 0};
#pragma unroll
                        for (int v = p * kEach; v < (p + 1) * kEach; ++v) {
                            uint32_t part[E::kParts][4];
                            now[v].parts(part);
#pragma unroll
                            for (int y = E::kParts - 1; y >= 0; --y) all[p] = mfma16(ones, part[y], all[p], W{});
                        }
                    }
                }
#pragma unroll
                for (int s = 0; s < R; ++s) {
                    uint32_t word[4] = {codes[u][s][0], codes[u][s][1], codes[u][s][2], codes[u][s][3]};
                    if constexpr (SMALL) {
                        // instruction v takes 32 consecutive columns: word v of each lane goes to the lanes of the v-th 16 (4 x 4 transposed over q)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const auto two = __builtin_amdgcn_permlane32_swap(word[i], word[i + 2], false, false);
                            word[i] = two[0];
                            word[i + 2] = two[1];
                        }
#pragma unroll
                        for (int i = 0; i < 4; i += 2) {
                            const auto two = __builtin_amdgcn_permlane16_swap(word[i], word[i + 1], false, false);
                            word[i] = two[0];
                            word[i + 1] = two[1];
                        }
                    }
#pragma unroll
                    for (int v = 0; v < 4; ++v) widen_codes<W, EXACT>(word[v], w[v]);
#pragma unroll
                    for (int p = 0; p < kPer; ++p) {
                        const float* of_group = mine + (u * kPer + p) * (16 * R) + s * 16 + q * 4;
                        const v4f scale = *reinterpret_cast<const v4f*>(of_group);
                        v4f less = {-136.0f, -136.0f, -136.0f, -136.0f};
                        if constexpr (ZEROS) less = *reinterpret_cast<const v4f*>(of_group + S::kScales);
                        v4f sum = {0, 0, 0, 0}, here = {0, 0, 0, 0};
                        if constexpr (kOnce) here = all[p];
#pragma unroll
                        for (int v = p * kEach; v < (p + 1) * kEach; ++v) {
                            uint32_t part[E::kParts][4];
                            now[v].parts(part);
#pragma unroll
                            for (int y = E::kParts - 1; y >= 0; --y) {
                                sum = mfma16(w[v], part[y], sum, W{});
                                if constexpr (kSums && !kOnce) here = mfma16(ones, part[y], here, W{});
                            }
                        }
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            float e = sum[r];
                            if constexpr (kSums) e = fmaf(less[r], here[r], e);
                            acc[s][r] = fmaf(scale[r], e, acc[s][r]);
                        }
                    }
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
    // the wave's sums take the place of its scales
#pragma unroll
    for (int s = 0; s < R; ++s) *reinterpret_cast<v4f*>(mine + x16 * (16 * R) + s * 16 + q * 4) = acc[s];
    __syncthreads();
    for (int x = threadIdx.x; x < 64 * R; x += blockDim.x) {
        const int r = x / (4 * R), c = (x % (4 * R)) * 4;
        const bool in = r < rows && c < cols;
        v4f s = {0, 0, 0, 0};
        for (int w = 0; w < waves; ++w) s += *reinterpret_cast<const v4f*>(lds + w * (S::kWaveBytes / 4) + r * (16 * R) + c);
        mend_results<X>(g, of, in, row0 + r, col0 + c, s);
        if (in) store_results(g, int64_t(row0 + r) * g.ldy + col0 + c, cols - c, s);
    }
}

// Rows of less than eight: a thread for each result.
template <typename X>
__global__ __launch_bounds__(256) void packed_gemm_short_kernel(PackedGemm g) {
    const ScaleLoad scales(g.w.scale, g.w.type), zeros(g.w.zero, g.w.type);
    const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x, row = id / g.n, col = id - row * g.n;
    if (row >= g.m) return;
    int of = 0;
    if (g.offsets) {
        of = -1;
        for (int e = 0; e < g.groups; ++e)
            if (row >= clamp_offset(g.offsets, e, g.m) && row < clamp_offset(g.offsets, e + 1, g.m)) of = e;
    }
    float sum = 0.0f;
    if (of >= 0 && g.k > 0) {
        const int64_t at = of * g.w.scale_stride + col;
        const float scale = scales.value(scales.fetch(at)), zero = g.w.zero ? zeros.value(zeros.fetch(at)) : 8.0f;
        const uint8_t* w = g.w.data + of * g.w.stride + col * g.w.ld;
        const X* x = static_cast<const X*>(g.x) + row * g.ldx;
        float all = 0.0f;
        for (int l = 0; l < g.k; ++l) {
            const float v = to_float(x[l]);
            sum = fmaf(float((w[l / 2] >> (4 * (l & 1))) & 15) - 8.0f, v, sum);
            all += v;
        }
        sum = scale * (g.w.zero ? fmaf(8.0f - zero, all, sum) : sum);
        if (!__builtin_isfinite(sum)) {
            double defined[1] = {0.0};
            add_defined<1>(g, of, x, int(col), 0, defined);
            sum = float(defined[0]);
        }
    }
    store_results(g, row * g.ldy + col, 1, v4f{sum, 0, 0, 0});
}

}  // namespace

}  // namespace oz

#include "oz_packed_gemm_staged.h"

namespace oz {

namespace {

// f(groups in a block, zero points or not, exact codes or not)
template <typename X, typename F>
void with_kind(const PackedGemm& g, F&& f) {
    const std::true_type yes;
    const std::false_type no;
    auto of_group = [&](auto zeros, auto exact) {
        if (g.w.shift == 5) f(std::integral_constant<int, 4>{}, zeros, exact);
        else if (g.w.shift == 6) f(std::integral_constant<int, 2>{}, zeros, exact);
        else f(std::integral_constant<int, 1>{}, zeros, exact);
    };
    auto of_shift = [&](auto exact) {
        if (g.w.zero) of_group(yes, exact);
        else of_group(no, exact);
    };
    if constexpr (std::is_same_v<X, bf16_t>) {
        if (g.y_type != OZ_F32) return of_shift(no);
    }
    of_shift(yes);
}

template <typename X, int MT, int R>
void launch_staged(hipStream_t st, const PackedGemm& g, int waves) {
    const int strips = (g.n + 16 * R - 1) / (16 * R);
    const dim3 grid(unsigned(packed_tiles(g.m, g.offsets ? g.groups : 0, MT * 16) * strips)), block(64 * waves);
    with_kind<X>(g, [&](auto per, auto zeros, auto exact) {
        constexpr int kPer = decltype(per)::value;
        constexpr bool kZeros = decltype(zeros)::value, kExact = decltype(exact)::value;
        if constexpr (R < 4 || kPer == 1) {
            const size_t bytes = size_t(waves) * Staged<X, MT, R, kPer, kZeros>::kWaveBytes;
            hipLaunchKernelGGL((packed_gemm_staged_kernel<X, MT, R, kPer, kZeros, kExact>), grid, block, bytes, st, g, strips);
        }
    });
}

template <typename X, int R>
void launch_few(hipStream_t st, const PackedGemm& g, int waves) {
    const int strips = (g.n + 16 * R - 1) / (16 * R);
    const dim3 grid(unsigned(packed_tiles(g.m, g.offsets ? g.groups : 0, 16) * strips)), block(64 * waves);
    with_kind<X>(g, [&](auto per, auto zeros, auto exact) {
        constexpr int kPer = decltype(per)::value;
        constexpr bool kZeros = decltype(zeros)::value, kExact = decltype(exact)::value;
        if constexpr (R < 4 || kPer < 4) {
            const size_t bytes = size_t(waves) * Shape<X, R, kPer, kZeros, kExact>::kWaveBytes;
            hipLaunchKernelGGL((packed_gemm_kernel<X, R, kPer, kZeros, kExact>), grid, block, bytes, st, g, strips);
        }
    });
}

// The kernels with more than 64 KB of LDS to a workgroup.
template <typename X, int MT, int R, int PER, bool ZEROS, bool EXACT>
bool allow_lds() {
    constexpr int bytes = 8 * Staged<X, MT, R, PER, ZEROS>::kWaveBytes;
    static_assert(bytes <= 160 * 1024, "LDS");
    return bytes <= 64 * 1024 || hipFuncSetAttribute(reinterpret_cast<const void*>(packed_gemm_staged_kernel<X, MT, R, PER, ZEROS, EXACT>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess;
}
template <typename X, int MT, int R, bool EXACT>
bool allow_kinds() {
    if constexpr (R == 4) return allow_lds<X, MT, R, 1, false, EXACT>() && allow_lds<X, MT, R, 1, true, EXACT>();
    else return allow_lds<X, MT, R, 1, false, EXACT>() && allow_lds<X, MT, R, 2, false, EXACT>() && allow_lds<X, MT, R, 4, false, EXACT>() &&
                allow_lds<X, MT, R, 1, true, EXACT>() && allow_lds<X, MT, R, 2, true, EXACT>() && allow_lds<X, MT, R, 4, true, EXACT>();
}
template <typename X, bool EXACT>
bool allow_staged() {
    return (sizeof(X) == 4 || allow_kinds<X, 1, 1, EXACT>()) && allow_kinds<X, 1, 2, EXACT>() && allow_kinds<X, 2, 2, EXACT>() && allow_kinds<X, 2, 4, EXACT>();
}

template <typename X>
void launch_typed(hipStream_t st, const PackedGemm& g, int num_cu) {
    if (g.k < 8) {
        hipLaunchKernelGGL(packed_gemm_short_kernel<X>, dim3(unsigned((int64_t(g.m) * g.n + 255) / 256)), dim3(256), 0, st, g);
        return;
    }
    const PackedPlan p = packed_plan(g.m, g.n, g.k, g.offsets ? g.groups : 0, sizeof(X), g.w.shift, num_cu);
    if (p.staged) {
        if (p.strips == 4) return launch_staged<X, 2, 4>(st, g, p.waves);
        if (p.rows == 2) return launch_staged<X, 2, 2>(st, g, p.waves);
        if constexpr (sizeof(X) == 2) {
            if (p.strips == 1) return launch_staged<X, 1, 1>(st, g, p.waves);
        }
        return launch_staged<X, 1, 2>(st, g, p.waves);
    }
    if (p.strips == 4) launch_few<X, 4>(st, g, p.waves);
    else if (p.strips == 2) launch_few<X, 2>(st, g, p.waves);
    else launch_few<X, 1>(st, g, p.waves);
}

}  // namespace

}  // namespace oz
