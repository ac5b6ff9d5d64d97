// Weights in 4 bits with a scale (and a zero point) per group of 32, 64 or 128 along their rows: quantised, read back, and multiplied with few rows.
//
//   value = scale * (code - zero), codes 0 .. 15, zero 8 where none is given
//   y_ij = sum over groups g of s_jg (sum_l (code_jl - 8) x_il + (8 - z_jg) sum_l x_il)
//
// Product: what bounds it is the read of the weights.  A workgroup has 16 rows of W and up to 64 rows of x; its waves share k, 128 at a time, and add up
// their sums through LDS in the waves' order.  code - 8 is exact in x's 16-bit type, and goes with x into v_mfma_f32_16x16x32 (float32
// x as three bfloat16 parts, exactly); scales are applied to each group's sum, in 32 bits, so the results have one rounding of 16 bits, the last.
// The sums of x that zero points need are one more matrix instruction, with a matrix of ones.
#include <algorithm>
#include <type_traits>

#include "oz_layer.h"
#include "oz_scaled_device.h"

namespace oz {

namespace {

typedef uint32_t v4u32 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float load_scale(const void* p, int type, int64_t at) {
    if (type == OZ_F32) return static_cast<const float*>(p)[at];
    if (type == OZ_BF16) return to_float(static_cast<const bf16_t*>(p)[at]);
    return to_float(static_cast<const f16_t*>(p)[at]);
}
__device__ __forceinline__ void store_scale(void* p, int type, int64_t at, float x) {
    if (type == OZ_F32) static_cast<float*>(p)[at] = x;
    else if (type == OZ_BF16) static_cast<bf16_t*>(p)[at] = static_cast<bf16_t>(x);
    else static_cast<f16_t*>(p)[at] = static_cast<f16_t>(x);
}
__device__ __forceinline__ float round_to(int type, float x) {
    return type == OZ_F32 ? x : type == OZ_BF16 ? to_float(static_cast<bf16_t>(x)) : to_float(static_cast<f16_t>(x));
}

// the largest over groups of 4, 8 or 16 lanes
__device__ __forceinline__ uint32_t lanes_max(uint32_t x, int lanes) {
    x = max(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0xB1, 0xF, 0xF, false)));       // the neighbour
    x = max(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x4E, 0xF, 0xF, false)));       // the next two
    if (lanes >= 8) x = max(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x141, 0xF, 0xF, false)));      // eight, mirrored
    if (lanes >= 16) x = max(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x140, 0xF, 0xF, false)));     // sixteen, mirrored
    return x;
}

// A lane has 8 consecutive elements of a row, a wave 512.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(PackCall c, int pieces) {
    const int64_t id = int64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = id / pieces;
    if (row >= c.rows) return;
    const int col = int(id - row * pieces) * 512 + int(threadIdx.x & 63) * 8, have = c.cols - col, lanes = (1 << c.w.shift) / 8;
    const int64_t b = blockIdx.y;
    float x[8];
    load_row<8>(static_cast<const T*>(c.x) + b * c.stride_x + row * c.ldx + col, have, c.cols, x);
    uint32_t top = 0;
    float hi = 0.0f, low = 0.0f;                         // zero is among the values, also behind the end
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
        hi = fmaxf(hi, x[i]);
        low = fmaxf(low, -x[i]);
    }
    top = lanes_max(top, lanes);                         // of magnitudes: whole numbers, and a NaN or an infinity is the largest
    float scale, zero = 8.0f;
    if (c.w.zero) {
        hi = __uint_as_float(lanes_max(__float_as_uint(hi), lanes));
        low = __uint_as_float(lanes_max(__float_as_uint(low), lanes));
        scale = round_to(c.w.type, (hi + low) / 15.0f);
    } else {
        scale = round_to(c.w.type, __uint_as_float(top) / 7.0f);
    }
    const bool fine = top < 0x7F800000u && scale < INFINITY;
    if (!fine) scale = NAN;
    if (c.w.zero && fine) zero = scale > 0.0f ? fminf(rintf(low / scale), 15.0f) : 0.0f;
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = fine && scale > 0.0f ? fminf(fmaxf(rintf(x[i] / scale) + zero, 0.0f), 15.0f) : zero;
        codes |= (i < have ? uint32_t(q) : 0u) << (4 * i);
    }
    if (have > 0 || col / 32 * 32 < c.cols) *reinterpret_cast<uint32_t*>(c.w.data + b * c.w.stride + row * c.w.ld + col / 2) = codes;
    if (have > 0 && (col & ((1 << c.w.shift) - 1)) == 0) {
        const int64_t at = b * c.w.scale_stride + int64_t(col >> c.w.shift) * c.w.scale_ld + row;
        store_scale(c.w.scale, c.w.type, at, scale);
        if (c.w.zero) store_scale(c.w.zero, c.w.type, at, zero);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void unpack_kernel(PackCall c, int pieces) {
    const int64_t id = int64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = id / pieces;
    if (row >= c.rows) return;
    const int col = int(id - row * pieces) * 512 + int(threadIdx.x & 63) * 8, have = c.cols - col;
    const int64_t b = blockIdx.y;
    if (have <= 0) return;
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(c.w.data + b * c.w.stride + row * c.w.ld + col / 2);
    const int64_t at = b * c.w.scale_stride + int64_t(col >> c.w.shift) * c.w.scale_ld + row;
    const float scale = load_scale(c.w.scale, c.w.type, at), zero = c.w.zero ? load_scale(c.w.zero, c.w.type, at) : 8.0f;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = scale * (float((codes >> (4 * i)) & 15u) - zero);
    store_row<8>(static_cast<T*>(const_cast<void*>(c.x)) + b * c.stride_x + row * c.ldx + col, have, x);
}

// ---- product ------------------------------------------------------------------------------------

constexpr int kBlock = 128;              // of k that a wave takes at a time

// code - 8 of eight codes, the lowest first
template <typename W>
__device__ __forceinline__ void widen_codes(uint32_t codes, uint32_t (&w)[4]) {
    const uint32_t even = codes & 0x0F0F0F0Fu, odd = (codes >> 4) & 0x0F0F0F0Fu;
    if constexpr (std::is_same_v<W, f16_t>) {
        // 1024 + code, whose last bits are the code's
        const f16x2 less = {f16_t(1032.0f), f16_t(1032.0f)};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t two = __builtin_amdgcn_perm(odd, even, 0x0C040C00u + 0x00010001u * uint32_t(i)) | 0x64006400u;
            w[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, two) - less);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = float((even >> (8 * i)) & 0xFFu) - 8.0f, b = float((odd >> (8 * i)) & 0xFFu) - 8.0f;
            w[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);       // whole numbers: the upper halves hold all of them
        }
    }
}

__device__ __forceinline__ v4f mfma16(const uint32_t (&a)[4], const uint32_t (&b)[4], v4f c, f16_t) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ v4f mfma16(const uint32_t (&a)[4], const uint32_t (&b)[4], v4f c, bf16_t) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight consecutive elements of a row of x as the matrix instruction takes them: one part, three of float32.
template <typename X>
struct Eight {
    static constexpr int kParts = sizeof(X) == 4 ? 3 : 1;
    using W = std::conditional_t<sizeof(X) == 4, bf16_t, X>;
    X e[8];
    __device__ __forceinline__ void load(const X* p) { __builtin_memcpy(e, p, sizeof(e)); }
    __device__ __forceinline__ void load(const X* p, int have) {
        if (have >= 8) {
            load(p);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = i < have ? p[i] : X(0.0f);
        }
    }
    __device__ __forceinline__ void parts(uint32_t (&w)[kParts][4]) const {
        if constexpr (kParts == 1) {
            __builtin_memcpy(w, e, sizeof(e));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t bits[2][3];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    // cut off, not rounded: what is left is exact, and no part is larger than the whole
                    float x = e[2 * i + j];
                    const bool fine = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
#pragma unroll
                    for (int p = 0; p < 3; ++p) {
                        bits[j][p] = __float_as_uint(x) & 0xFFFF0000u;
                        if (p == 0 && !fine && x != x) bits[j][0] = 0x7FC00000u;
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
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < have) put(p + i, v[i]);
}
__device__ __forceinline__ void store_results(const PackedGemm& g, int64_t at, int have, v4f v) {
    if (g.y_type == OZ_F32) store4(static_cast<float*>(g.y) + at, have, v);
    else if (g.y_type == OZ_BF16) store4(static_cast<bf16_t*>(g.y) + at, have, v);
    else store4(static_cast<f16_t*>(g.y) + at, have, v);
}

// scales of a lane's four rows of W
__device__ __forceinline__ v4f four_scales(const void* p, int type, int64_t at, int have) {
    v4f s;
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] = load_scale(p, type, at + min(r, max(have - 1, 0)));
    return s;
}

// MT: 16s of rows of x.  SHIFT: 2^SHIFT columns share a scale.
template <typename X, int MT, int SHIFT, bool ZEROS>
__global__ __launch_bounds__(MT == 1 ? 1024 : 512) void packed_gemm_kernel(PackedGemm g, int strips) {
    using E = Eight<X>;
    using W = typename E::W;
    constexpr int kPer = kBlock >> SHIFT, kEach = 4 / kPer;           // groups of a block; matrix instructions of a group
    extern __shared__ __align__(16) float sums[];                     // [wave][row][16]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = int(blockDim.x) >> 6;
    const int q = lane >> 4, x16 = lane & 15;
    const int strip = int(blockIdx.x % unsigned(strips)), piece = int(blockIdx.x / unsigned(strips)), col0 = strip * 16, cols = min(g.n - col0, 16);
    int row0 = piece * MT * 16, rows = min(g.m - row0, MT * 16), of = 0;
    if (g.offsets) {
        GroupPieces<MT * 16> pieces(g.offsets, g.groups, g.m);
        const GroupPiece p = pieces.template find<false>(piece);
        if (p.group < 0) return;
        of = p.group;
        row0 = p.row;
        rows = min(p.end - p.row, MT * 16);
    }
    const bool none = g.offsets && of >= g.groups;                    // rows behind the last group: zeros
    v4f acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = v4f{0, 0, 0, 0};
    if (!none) {
        const int my_row = min(x16, cols - 1);
        const uint8_t* w_row = g.w.data + of * g.w.stride + int64_t(col0 + my_row) * g.w.ld;
        const int64_t scale0 = of * g.w.scale_stride + col0 + min(q * 4, cols - 1);
        const X* x_row[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) x_row[i] = static_cast<const X*>(g.x) + int64_t(row0 + min(i * 16 + x16, rows - 1)) * g.ldx;
        const int blocks = (g.k + kBlock - 1) / kBlock, bytes = (g.k + 31) / 32 * 16;
        uint32_t ones[4];
        {
            const W one = static_cast<W>(1.0f);
            const uint32_t two = uint32_t(__builtin_bit_cast(uint16_t, one)) * 0x10001u;
#pragma unroll
            for (int i = 0; i < 4; ++i) ones[i] = two;
        }
        for (int b = wave; b < blocks; b += waves) {
            v4u32 codes = {0, 0, 0, 0};
            if (b * 64 + q * 16 < bytes) codes = *reinterpret_cast<const v4u32*>(w_row + b * 64 + q * 16);
            const bool whole = (b + 1) * kBlock <= g.k;
            E x[MT][4];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    // which of the block's columns lane q's part of instruction u covers: any order that both operands share
                    const int at = b * kBlock + (SHIFT == 7 ? q * 32 + u * 8 : u * 32 + q * 8);
                    if (whole) x[i][u].load(x_row[i] + at);
                    else x[i][u].load(x_row[i] + at, g.k - at);
                }
            v4f scale[kPer], zero[kPer];
#pragma unroll
            for (int p = 0; p < kPer; ++p) {
                const int group = min(b * kPer + p, (g.k - 1) >> SHIFT);
                scale[p] = four_scales(g.w.scale, g.w.type, scale0 + int64_t(group) * g.w.scale_ld, cols - q * 4);
                if constexpr (ZEROS) zero[p] = four_scales(g.w.zero, g.w.type, scale0 + int64_t(group) * g.w.scale_ld, cols - q * 4);
            }
            uint32_t word[4] = {codes[0], codes[1], codes[2], codes[3]};
            if constexpr (SHIFT != 7) {
                // instruction u takes 32 consecutive columns: word u of each lane goes to the lanes of the u-th 16 (4 x 4 transposed over q)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const auto s = __builtin_amdgcn_permlane32_swap(word[i], word[i + 2], false, false);
                    word[i] = s[0];
                    word[i + 2] = s[1];
                }
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const auto s = __builtin_amdgcn_permlane16_swap(word[i], word[i + 1], false, false);
                    word[i] = s[0];
                    word[i + 1] = s[1];
                }
            }
            uint32_t w[4][4];
#pragma unroll
            for (int u = 0; u < 4; ++u) widen_codes<W>(word[u], w[u]);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int p = 0; p < kPer; ++p) {
                    v4f sum = {0, 0, 0, 0}, all = {0, 0, 0, 0};
#pragma unroll
                    for (int u = p * kEach; u < (p + 1) * kEach; ++u) {
                        uint32_t part[E::kParts][4];
                        x[i][u].parts(part);
#pragma unroll
                        for (int s = E::kParts - 1; s >= 0; --s) {
                            sum = mfma16(w[u], part[s], sum, W{});
                            if constexpr (ZEROS) all = mfma16(ones, part[s], all, W{});
                        }
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][r] = fmaf(scale[p][r], ZEROS ? fmaf(8.0f - zero[p][r], all[r], sum[r]) : sum[r], acc[i][r]);
                }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) *reinterpret_cast<v4f*>(sums + ((wave * MT + i) * 16 + x16) * 16 + q * 4) = acc[i];
    __syncthreads();
    for (int x = threadIdx.x; x < MT * 64; x += blockDim.x) {
        const int r = x >> 2, c = (x & 3) * 4;
        v4f s = {0, 0, 0, 0};
        for (int w = 0; w < waves; ++w) s += *reinterpret_cast<const v4f*>(sums + (w * MT * 16 + r) * 16 + c);
        if (r < rows && c < cols) store_results(g, int64_t(row0 + r) * g.ldy + col0 + c, cols - c, s);
    }
}

template <typename X, int MT, int SHIFT>
void launch_rows(hipStream_t st, const PackedGemm& g) {
    const int strips = (g.n + 15) / 16, blocks = (g.k + kBlock - 1) / kBlock;
    const int64_t tiles = g.offsets ? group_pieces(g.m, g.groups, MT * 16) : (g.m + MT * 16 - 1) / (MT * 16);
    const int waves = std::max(std::min(blocks, MT == 1 ? 16 : 8), 1);
    const dim3 grid(unsigned(tiles * strips)), block(64 * waves);
    const size_t lds = size_t(waves) * MT * 16 * 16 * 4;
    if (g.w.zero) hipLaunchKernelGGL((packed_gemm_kernel<X, MT, SHIFT, true>), grid, block, lds, st, g, strips);
    else hipLaunchKernelGGL((packed_gemm_kernel<X, MT, SHIFT, false>), grid, block, lds, st, g, strips);
}

template <typename X, int MT>
void launch_shift(hipStream_t st, const PackedGemm& g) {
    if (g.w.shift == 5) launch_rows<X, MT, 5>(st, g);
    else if (g.w.shift == 6) launch_rows<X, MT, 6>(st, g);
    else launch_rows<X, MT, 7>(st, g);
}

template <typename X>
void launch_typed(hipStream_t st, const PackedGemm& g) {
    const int64_t rows = g.offsets ? (int64_t(g.m) + g.groups - 1) / g.groups : g.m;      // of a group on average
    if (rows <= 16) launch_shift<X, 1>(st, g);
    else if (rows <= 32) launch_shift<X, 2>(st, g);
    else launch_shift<X, 4>(st, g);
}

}  // namespace

void launch_pack(hipStream_t st, const PackCall& c) {
    const int pieces = (c.cols + 511) / 512;
    const dim3 grid(unsigned((int64_t(c.rows) * pieces + 3) / 4), unsigned(c.batch));
    if (c.x_type == OZ_F32) hipLaunchKernelGGL(pack_kernel<float>, grid, dim3(256), 0, st, c, pieces);
    else if (c.x_type == OZ_BF16) hipLaunchKernelGGL(pack_kernel<bf16_t>, grid, dim3(256), 0, st, c, pieces);
    else hipLaunchKernelGGL(pack_kernel<f16_t>, grid, dim3(256), 0, st, c, pieces);
}

void launch_unpack(hipStream_t st, const PackCall& c) {
    const int pieces = (c.cols + 511) / 512;
    const dim3 grid(unsigned((int64_t(c.rows) * pieces + 3) / 4), unsigned(c.batch));
    if (c.x_type == OZ_F32) hipLaunchKernelGGL(unpack_kernel<float>, grid, dim3(256), 0, st, c, pieces);
    else if (c.x_type == OZ_BF16) hipLaunchKernelGGL(unpack_kernel<bf16_t>, grid, dim3(256), 0, st, c, pieces);
    else hipLaunchKernelGGL(unpack_kernel<f16_t>, grid, dim3(256), 0, st, c, pieces);
}

void launch_packed_gemm(hipStream_t st, const PackedGemm& g, int) {
    if (g.x_type == OZ_F32) launch_typed<float>(st, g);
    else if (g.x_type == OZ_BF16) launch_typed<bf16_t>(st, g);
    else launch_typed<f16_t>(st, g);
}

}  // namespace oz
