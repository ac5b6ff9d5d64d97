// Weights in 4 bits with a scale (and a zero point) per group of 32, 64 or 128 along their rows: quantised, and read back.
//
//   value = scale * (code - zero), codes 0 .. 15, zero 8 where none is given
//
// What bounds both is memory: 16 x 2048 x 2048 bfloat16 41 us (4.1 TB/s) to 4 bits and 27 (6.2, writes to the last-level cache among them) back.
#include <type_traits>

#include "oz_layer.h"
#include "oz_scaled_device.h"

namespace oz {

namespace {

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

// rint(x / scale) for eight values whose quotients are at most 15 in magnitude.  A product with the inverse is off by less than 2^-17: only where it lies that
// close to a half can the division's own rounding decide, and there it is done.
__device__ __forceinline__ void quotients(const float (&x)[8], float scale, float (&q)[8]) {
    const float inverse = __builtin_amdgcn_rcpf(scale);
    float far = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = x[i] * inverse;
        q[i] = rintf(t);
        far = fmaxf(far, fabsf(t - q[i]));
    }
    // scales whose inverse has fewer bits, or none
    if (far > 0.5f - 0x1p-17f || !(scale > 0x1p-120f && scale < 0x1p120f)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = rintf(x[i] / scale);
    }
}

// The largest magnitude, as its bits: a NaN or an infinity is above all.  16-bit values two at a time.
template <typename T>
__device__ __forceinline__ uint32_t largest_bits(const RowPiece<8, T>& p) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    if constexpr (sizeof(T) == 4) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, p.w[i] & 0x7FFFFFFFu);
        return top;
    } else {
        u16x2 top = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, p.w[i] & 0x7FFF7FFFu));
        return __float_as_uint(to_float(__builtin_bit_cast(T, uint16_t(max(top[0], top[1])))));
    }
}

// A lane has 8 consecutive elements of a row, a wave 512, of kRows rows that are on their way together.  What bounds it is memory, and close behind it the
// vector instructions: about a hundred for a lane's eight elements, where with a division for each there were two hundred (16 x 2048 x 2048
// bfloat16 56 us).
constexpr int kRows = 2;
template <typename T, bool ZEROS>
__global__ __launch_bounds__(256) void pack_kernel(PackCall c, int pieces) {
    const uint32_t id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), of = id / uint32_t(pieces);
    const int64_t row0 = int64_t(of) * kRows;
    if (row0 >= c.rows) return;
    const int col = int(id - of * uint32_t(pieces)) * 512 + int(threadIdx.x & 63) * 8, have = c.cols - col, lanes = (1 << c.w.shift) / 8;
    const int64_t b = blockIdx.y;
    RowPiece<8, T> raw[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        fetch_row<8>(static_cast<const T*>(c.x) + b * c.stride_x + min(row0 + r, int64_t(c.rows) - 1) * c.ldx + col, have, c.cols, raw[r]);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int64_t row = row0 + r;
        if (row < c.rows) {
            RowPiece<8, T> piece = raw[r];
            settle_row(piece, have, c.cols);
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = to_float(piece.e[i]);
            const uint32_t top = lanes_max(largest_bits(piece), lanes);
            float scale, zero = 8.0f, low = 0.0f;
            if constexpr (ZEROS) {
                float hi = 0.0f;                         // zero is among the values, also behind the end
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    hi = fmaxf(hi, x[i] + 0.0f);
                    low = fmaxf(low, 0.0f - x[i]);
                }
                hi = __uint_as_float(lanes_max(__float_as_uint(hi), lanes));
                low = __uint_as_float(lanes_max(__float_as_uint(low), lanes));      // bit patterns: neither is a negative zero
                scale = round_to(c.w.type, (hi + low) / 15.0f);
            } else {
                scale = round_to(c.w.type, __uint_as_float(top) / 7.0f);
            }
            const bool fine = top < 0x7F800000u && scale < INFINITY, some = fine && scale > 0.0f;
            if (!fine) scale = NAN;
            if (ZEROS && fine) zero = some ? fminf(rintf(low / scale), 15.0f) : 0.0f;
            float q[8];
            quotients(x, some ? scale : 1.0f, q);
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = fminf(fmaxf(q[i] + zero, 0.0f), 15.0f);
            // four codes are a whole number that a float32 holds
            const float first = fmaf(fmaf(fmaf(q[3], 16.0f, q[2]), 16.0f, q[1]), 16.0f, q[0]), last = fmaf(fmaf(fmaf(q[7], 16.0f, q[6]), 16.0f, q[5]), 16.0f, q[4]);
            uint32_t codes = uint32_t(first) | uint32_t(last) << 16;
            if (!fine) codes = 0x88888888u;
            if (have < 8) codes &= (1u << (4 * max(have, 0))) - 1;
            if (have > 0 || col / 32 * 32 < c.cols) *reinterpret_cast<uint32_t*>(c.w.data + b * c.w.stride + row * c.w.ld + col / 2) = codes;
            if (have > 0 && (col & ((1 << c.w.shift) - 1)) == 0) {
                const int64_t at = b * c.w.scale_stride + int64_t(col >> c.w.shift) * c.w.scale_ld + row;
                store_scale(c.w.scale, c.w.type, at, scale);
                if (ZEROS) store_scale(c.w.zero, c.w.type, at, zero);
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void unpack_kernel(PackCall c, int pieces) {
    const uint32_t id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), of = id / uint32_t(pieces);
    const int64_t row = of;
    if (row >= c.rows) return;
    const int col = int(id - of * uint32_t(pieces)) * 512 + int(threadIdx.x & 63) * 8, have = c.cols - col;
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

}  // namespace

void launch_pack(hipStream_t st, const PackCall& c) {
    const int pieces = (c.cols + 511) / 512;
    const dim3 grid(unsigned(((int64_t(c.rows) + kRows - 1) / kRows * pieces + 3) / 4), unsigned(c.batch));
    auto typed = [&](auto zeros) {
        constexpr bool kZeros = decltype(zeros)::value;
        if (c.x_type == OZ_F32) hipLaunchKernelGGL((pack_kernel<float, kZeros>), grid, dim3(256), 0, st, c, pieces);
        else if (c.x_type == OZ_BF16) hipLaunchKernelGGL((pack_kernel<bf16_t, kZeros>), grid, dim3(256), 0, st, c, pieces);
        else hipLaunchKernelGGL((pack_kernel<f16_t, kZeros>), grid, dim3(256), 0, st, c, pieces);
    };
    if (c.w.zero) typed(std::true_type{});
    else typed(std::false_type{});
}

void launch_unpack(hipStream_t st, const PackCall& c) {
    const int pieces = (c.cols + 511) / 512;
    const dim3 grid(unsigned((int64_t(c.rows) * pieces + 3) / 4), unsigned(c.batch));
    if (c.x_type == OZ_F32) hipLaunchKernelGGL(unpack_kernel<float>, grid, dim3(256), 0, st, c, pieces);
    else if (c.x_type == OZ_BF16) hipLaunchKernelGGL(unpack_kernel<bf16_t>, grid, dim3(256), 0, st, c, pieces);
    else hipLaunchKernelGGL(unpack_kernel<f16_t>, grid, dim3(256), 0, st, c, pieces);
}

void launch_packed_gemm(hipStream_t st, const PackedGemm& g, int num_cu) {
    if (g.x_type == OZ_F32) launch_packed_gemm_f32(st, g, num_cu);
    else if (g.x_type == OZ_BF16) launch_packed_gemm_bf16(st, g, num_cu);
    else launch_packed_gemm_f16(st, g, num_cu);
}

}  // namespace oz
