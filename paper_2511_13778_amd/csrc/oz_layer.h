// What stands around a layer's products: the router's choice of experts, weights in 4 bits, orthogonal weight updates.  Shared by their kernels and
// the C ABI.
#pragma once

#include "oz_scaled.h"

namespace oz {

// ---- choice of experts
struct ChooseCall {
    const void* scores;
    int64_t ld;
    int type, tokens, experts, topk, normalize;
    const uint8_t* live;                 // nullptr: every token
    int32_t* ids;
    float* weights;
    int32_t *counts, *counted;           // [experts] choices of each, [1] tokens that have one; nullptr: neither these nor shares and loss
    float *shares, *loss;
    void* ws;
};
struct ChooseGradCall {
    const void* scores;
    int64_t ld;
    int type, tokens, experts, topk, normalize;
    const uint8_t* live;
    const int32_t* ids;
    const float *weights, *dweights;     // dweights nullptr: 0
    const int32_t *counts, *counted;     // nullptr: no gradient of the loss
    const float* dloss;                  // nullptr: 1
    float factor;
    void* dscores;
    int64_t ldd;
};
size_t choose_bytes(int64_t tokens, int64_t experts, int num_cu);
void launch_choose(hipStream_t st, const ChooseCall& c, int num_cu);
void launch_choose_grad(hipStream_t st, const ChooseGradCall& c, int num_cu);

// ---- weights in 4 bits
struct PackedOperand {
    uint8_t* data;                       // (row, column 2i and 2i + 1) at row * ld + i, the even one in the low half
    void *scale, *zero;                  // (group, row) at group * scale_ld + row; zero nullptr: 8
    int64_t ld, scale_ld, stride, scale_stride;
    int shift, type;                     // log2 of the columns of a group; of scale and zero
};
struct PackCall {
    const void* x;
    int64_t ldx, stride_x;
    int x_type, rows, cols, batch;
    PackedOperand w;
};
struct PackedGemm {
    const void* x;
    int64_t ldx;
    int x_type;
    PackedOperand w;
    void* y;
    int64_t ldy;
    int y_type, m, n, k;
    const int32_t* offsets;              // nullptr: one group
    int groups;
};
void launch_pack(hipStream_t st, const PackCall& c);
void launch_unpack(hipStream_t st, const PackCall& c);         // x is written
void launch_packed_gemm(hipStream_t st, const PackedGemm& g, int num_cu);
void launch_packed_gemm_f32(hipStream_t st, const PackedGemm& g, int num_cu);
void launch_packed_gemm_bf16(hipStream_t st, const PackedGemm& g, int num_cu);
void launch_packed_gemm_f16(hipStream_t st, const PackedGemm& g, int num_cu);

// ---- orthogonal updates
struct OrthoCall {
    const void* x;
    void* y;
    int64_t ldx, stride_x, ldy, stride_y;
    int type, batch, rows, cols, steps;
    float a, b, c, eps;
    void* ws;
};
size_t ortho_bytes(int64_t batch, int64_t rows, int64_t cols, int type, int num_cu);
void launch_ortho(hipStream_t st, const OrthoCall& c, int num_cu);
// once per process, before the first launch
bool prepare_ortho();
bool prepare_packed_gemm_f32();
bool prepare_packed_gemm_bf16();
bool prepare_packed_gemm_f16();

}  // namespace oz
