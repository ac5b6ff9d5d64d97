// Weights in 4 bits with a scale (and a zero point) per group of 32, 64 or 128 along their rows: quantised, and read back.
//
//   value = scale * (code - zero), codes 0 .. 15, zero 8 where none is given
//
// What bounds both is memory.
#include <algorithm>

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

void launch_packed_gemm(hipStream_t st, const PackedGemm& g, int num_cu) {
    if (g.x_type == OZ_F32) launch_packed_gemm_f32(st, g, num_cu);
    else if (g.x_type == OZ_BF16) launch_packed_gemm_bf16(st, g, num_cu);
    else launch_packed_gemm_f16(st, g, num_cu);
}

}  // namespace oz
