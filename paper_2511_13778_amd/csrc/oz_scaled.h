// 8-bit block-scaled operands: what their kernels and the C ABI share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ozdgemm.h"

namespace oz {

constexpr int kScaleBlock = 128;      // elements of a row that share a scale

// One operand as the kernels see it.  shift: 0 where every row has scales of its own, 7 where 128 rows share them.
struct ScaledOperand {
    uint8_t* data;
    uint8_t* scale;
    int64_t ld, scale_ld, stride, scale_stride;
    int shift;
};

enum class Grouping { kNone, kRows, kContraction };

struct ScaledGemm {
    ScaledOperand a, b;
    void* c;
    int64_t ldc, stride_c;
    int m, n, k;
    int c_type, accumulate;
    const int32_t* offsets;
    int groups;
    Grouping grouping;
    bool a_e5m2, e8m0;
    bool wide;            // the caller's C is float32: operands are widened for 32-bit sums
    int parts;            // k is cut into so many; C is then a float32 plane of m x n for each
};

struct QuantizeCall {
    const void* x;
    int64_t ldx, stride_x;
    int x_type, rows, cols, batch;
    const int32_t* order;
    int order_div, x_rows;
    const int32_t* offsets;
    int groups;
    ScaledOperand out_rows, out_cols;      // data == nullptr: not asked for
    bool rows_e5m2, cols_e5m2, rows_e8m0, cols_e8m0;
    bool tiles;                            // 128 rows share a scale
};

void launch_scaled_gemm(hipStream_t st, const ScaledGemm& g, int num_cu, float* planes);
void launch_scaled_gemm_big(hipStream_t st, const ScaledGemm& g, bool square);     // tiles of 256 x 256, else 256 x 128
void launch_scaled_gemm_big_f32(hipStream_t st, const ScaledGemm& g);
bool prepare_scaled_gemm_f32();
void launch_scaled_gemm_few(hipStream_t st, const ScaledGemm& g, int rows, int waves);
bool prepare_scaled_gemm();            // once per process, before the first launch
size_t scaled_gemm_part_bytes(int64_t m, int64_t n, int64_t k, int num_cu);      // of the planes of a product without groups
void launch_quantize(hipStream_t st, const QuantizeCall& q);

void launch_sort_tokens(hipStream_t st, int choices, int experts, const void* chosen, bool wide, int32_t* offsets, int32_t* order,
                        int32_t* place, int32_t* ws);
size_t sort_tokens_bytes(int64_t choices, int64_t experts);
void launch_gather_rows(hipStream_t st, int tokens, int topk, int cols, int elem_bytes, const void* x, int64_t ldx, const int32_t* order,
                        const int32_t* place, void* y, int64_t ldy);
void launch_combine_rows(hipStream_t st, int tokens, int topk, int cols, int type, const void* x, int64_t ldx, int slots, const int32_t* place,
                         const float* weights, void* y, int64_t ldy);
void launch_combine_grad(hipStream_t st, int tokens, int topk, int cols, int type, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                         int slots, const int32_t* order, const int32_t* place, const float* weights, void* dx, int64_t lddx, float* dweights);

// Whether the calling thread's current device is the handle's; its compute units.
bool handle_on_device(oz_handle_t h);
int handle_compute_units(oz_handle_t h);

// Pieces of `size` that groups of `total` rows can be cut into at most, each group for itself (a group of its own for rows behind the last).
inline int64_t group_pieces(int64_t total, int64_t groups, int64_t size) {
    const int64_t g = groups + 1 < total ? groups + 1 : total;
    return (total + (size - 1) * g) / size;
}

// Columns, in blocks, that oz_quantize's grouped transpose can take.
inline int64_t grouped_blocks(int64_t rows, int64_t groups) {
    const int64_t g = groups < rows ? groups : rows;
    return (rows + (kScaleBlock - 1) * g) / kScaleBlock;
}

}  // namespace oz
