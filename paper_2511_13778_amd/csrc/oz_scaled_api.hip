// C ABI of the 8-bit block-scaled operators and of rows sorted by group: argument checks, then launches on the caller's stream.
#include "oz_scaled.h"

namespace {

using namespace oz;

constexpr int64_t kMaxRows = int64_t(1) << 24, kMaxLd = int64_t(1) << 23, kMaxGroups = 1024, kMaxChoices = int64_t(1) << 30;
constexpr int64_t kMaxGrid = (int64_t(1) << 24) - 1;      // workgroups of 256 threads: a launch holds less than 2^32 threads
constexpr size_t kWorkspaceAlign = 256;

int elem_bytes(int32_t type) { return type == OZ_F32 ? 4 : type == OZ_BF16 || type == OZ_F16 ? 2 : 0; }
bool is_aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// `rows` x `cols` with scales; need_ld: columns that are written or read
bool check_scaled(const oz_scaled_t* s, int64_t rows, int64_t cols, int64_t need_blocks, bool batched) {
    if (!s || s->reserved_ != 0) return false;
    if (s->type != OZ_E4M3 && s->type != OZ_E5M2) return false;
    if (s->scale_type != OZ_E8M0 && s->scale_type != OZ_F32) return false;
    if (s->block_rows != 1 && s->block_rows != 128) return false;
    if (rows > 0 && cols > 0) {
        if (!s->data || !s->scale || !is_aligned(s->data, 16) || !is_aligned(s->scale, 4)) return false;
    }
    if (s->ld < cols || s->ld % 16 != 0 || s->ld >= kMaxLd) return false;
    if (s->scale_ld < need_blocks || s->scale_ld >= kMaxLd / 64) return false;
    if (s->scale_type == OZ_E8M0 && s->scale_ld % 4 != 0) return false;
    if (batched) {
        if (s->stride < 0 || s->stride % 16 != 0 || s->scale_stride < 0) return false;
        if (s->scale_type == OZ_E8M0 && s->scale_stride % 4 != 0) return false;
    }
    return true;
}

ScaledOperand operand_of(const oz_scaled_t* s) {
    if (!s) return ScaledOperand{nullptr, nullptr, 0, 0, 0, 0, 0};
    return ScaledOperand{static_cast<uint8_t*>(s->data), static_cast<uint8_t*>(s->scale), s->ld, s->scale_ld, s->stride, s->scale_stride,
                         s->block_rows == 128 ? 7 : 0};
}

inline int64_t blocks_of(int64_t n) { return (n + kScaleBlock - 1) / kScaleBlock; }

bool sizes_ok(int64_t m, int64_t n, int64_t k) {
    return m >= 0 && n >= 0 && k >= 0 && m <= kMaxRows && n <= kMaxRows && k <= kMaxRows;
}

oz_status_t gemm(oz_handle_t h, void* stream, Grouping grouping, int64_t groups, const int32_t* offsets, int64_t m, int64_t n, int64_t k,
                 const oz_scaled_t* A, const oz_scaled_t* B, void* C, int64_t ldc, int64_t stride_c, int32_t c_type, int32_t accumulate,
                 void* ws, size_t ws_bytes) {
    if (!h || !sizes_ok(m, n, k)) return OZ_ERR_ARG;
    const bool by_k = grouping == Grouping::kContraction, by_rows = grouping == Grouping::kRows;
    if (grouping != Grouping::kNone && (groups < 1 || groups > kMaxGroups || !offsets)) return OZ_ERR_ARG;
    const int esize = elem_bytes(c_type);
    if (esize == 0 || ldc < n || ldc > (int64_t(1) << 32) || (accumulate != 0 && accumulate != 1)) return OZ_ERR_ARG;
    if (!check_scaled(A, m, k, blocks_of(k), false) || !check_scaled(B, n, k, blocks_of(k), by_rows)) return OZ_ERR_ARG;
    if (B->type != OZ_E4M3 || A->scale_type != B->scale_type) return OZ_ERR_ARG;
    if (by_k && groups > 1 && m > 0 && n > 0 && stride_c < (m - 1) * ldc + n) return OZ_ERR_ARG;      // the results overlap
    if (by_k && (k % kScaleBlock != 0 || A->block_rows != 1 || B->block_rows != 1)) return OZ_ERR_ARG;
    if (m == 0 || n == 0) return OZ_OK;
    if (!C || !is_aligned(C, uintptr_t(esize))) return OZ_ERR_ARG;
    // workgroups: of 1024 threads on 16 columns for few rows, else of 256 on at least 64 x 64
    const bool few = (by_rows ? (m + groups - 1) / groups : m) <= 64;
    const int64_t tile = few ? 16 : 64;
    if (((m + tile - 1) / tile + (by_rows ? groups + 1 : 0)) * ((n + tile - 1) / tile) > (few ? kMaxGrid / 4 : kMaxGrid)) return OZ_ERR_ARG;
    const size_t need = grouping == Grouping::kNone ? oz_scaled_gemm_workspace_bytes(h, m, n, k) : 0;
    if (need > 0 && (!ws || !is_aligned(ws, kWorkspaceAlign) || ws_bytes < need)) return OZ_ERR_WORKSPACE;
    if (!handle_on_device(h)) return OZ_ERR_DEVICE;
    ScaledGemm g;
    g.a = operand_of(A);
    g.b = operand_of(B);
    g.c = C;
    g.ldc = ldc;
    g.stride_c = stride_c;
    g.m = int(m);
    g.n = int(n);
    g.k = int(k);
    g.c_type = c_type;
    g.accumulate = accumulate;
    g.offsets = offsets;
    g.groups = int(groups);
    g.grouping = grouping;
    g.a_e5m2 = A->type == OZ_E5M2;
    g.e8m0 = A->scale_type == OZ_E8M0;
    g.wide = c_type == OZ_F32;
    g.parts = 1;
    launch_scaled_gemm(static_cast<hipStream_t>(stream), g, handle_compute_units(h), static_cast<float*>(ws));
    return hipGetLastError() == hipSuccess ? OZ_OK : OZ_ERR_HIP;
}

bool rows_ok(int64_t rows, int64_t cols, const void* p, int64_t ld, int esize) {
    if (rows < 0 || cols < 0 || rows > kMaxChoices || cols > kMaxRows || ld < cols || ld > (int64_t(1) << 32)) return false;
    return rows == 0 || cols == 0 || (p && is_aligned(p, uintptr_t(esize)));
}

}  // namespace

extern "C" {

oz_status_t oz_quantize(oz_handle_t h, void* stream, int64_t rows, int64_t cols, const void* X, int64_t ldx, int32_t x_type, int64_t batch,
                        int64_t stride_x, const int32_t* order, int64_t order_div, int64_t x_rows, const int32_t* offsets, int64_t groups,
                        const oz_scaled_t* by_rows, const oz_scaled_t* by_columns) {
    const int esize = elem_bytes(x_type);
    if (!h || esize == 0 || !sizes_ok(rows, cols, 0) || cols >= (int64_t(1) << 22) || batch < 0 || batch > 65535 || stride_x < 0) return OZ_ERR_ARG;
    if (!by_rows && !by_columns) return OZ_ERR_ARG;
    const bool tiles = (by_rows ? by_rows : by_columns)->block_rows == 128;
    if (by_rows && by_columns && by_rows->block_rows != by_columns->block_rows) return OZ_ERR_ARG;
    if ((order || offsets) && (tiles || batch > 1)) return OZ_ERR_ARG;
    if (offsets && (groups < 1 || groups > kMaxGroups)) return OZ_ERR_ARG;
    if (order && (order_div < 1 || order_div > kMaxRows || x_rows < 0 || x_rows > kMaxRows)) return OZ_ERR_ARG;
    if (ldx < cols || ldx > (int64_t(1) << 32)) return OZ_ERR_ARG;
    const int64_t wide = offsets ? grouped_blocks(rows, groups) * kScaleBlock : rows;
    if (by_rows && !check_scaled(by_rows, rows, cols, blocks_of(cols), batch > 1)) return OZ_ERR_ARG;
    if (by_columns && !check_scaled(by_columns, cols, wide, blocks_of(wide), batch > 1)) return OZ_ERR_ARG;
    if (rows == 0 || cols == 0 || batch == 0) return OZ_OK;
    if ((!X && (!order || x_rows > 0)) || !is_aligned(X, uintptr_t(esize))) return OZ_ERR_ARG;
    if (rows * blocks_of(cols) > (int64_t(1) << 27)) return OZ_ERR_ARG;
    if (!handle_on_device(h)) return OZ_ERR_DEVICE;
    QuantizeCall q;
    q.x = X;
    q.ldx = ldx;
    q.stride_x = stride_x;
    q.x_type = x_type;
    q.rows = int(rows);
    q.cols = int(cols);
    q.batch = int(batch);
    q.order = order;
    q.order_div = int(order_div);
    q.x_rows = int(x_rows);
    q.offsets = by_columns ? offsets : nullptr;       // the groups are cut along the columns of the transposed matrix only
    q.groups = int(groups);
    q.out_rows = operand_of(by_rows);
    q.out_cols = operand_of(by_columns);
    q.rows_e5m2 = by_rows && by_rows->type == OZ_E5M2;
    q.cols_e5m2 = by_columns && by_columns->type == OZ_E5M2;
    q.rows_e8m0 = by_rows && by_rows->scale_type == OZ_E8M0;
    q.cols_e8m0 = by_columns && by_columns->scale_type == OZ_E8M0;
    q.tiles = tiles;
    launch_quantize(static_cast<hipStream_t>(stream), q);
    return hipGetLastError() == hipSuccess ? OZ_OK : OZ_ERR_HIP;
}

size_t oz_scaled_gemm_workspace_bytes(oz_handle_t h, int64_t m, int64_t n, int64_t k) {
    if (!h || !sizes_ok(m, n, k)) return 0;
    return scaled_gemm_part_bytes(m, n, k, handle_compute_units(h));
}

oz_status_t oz_scaled_gemm(oz_handle_t h, void* stream, int64_t m, int64_t n, int64_t k, const oz_scaled_t* A, const oz_scaled_t* B, void* C,
                           int64_t ldc, int32_t c_type, int32_t accumulate, void* workspace, size_t workspace_bytes) {
    return gemm(h, stream, Grouping::kNone, 0, nullptr, m, n, k, A, B, C, ldc, 0, c_type, accumulate, workspace, workspace_bytes);
}

oz_status_t oz_scaled_gemm_grouped(oz_handle_t h, void* stream, int64_t groups, const int32_t* offsets, int64_t m, int64_t n, int64_t k,
                                   const oz_scaled_t* A, const oz_scaled_t* B, void* C, int64_t ldc, int32_t c_type) {
    return gemm(h, stream, Grouping::kRows, groups, offsets, m, n, k, A, B, C, ldc, 0, c_type, 0, nullptr, 0);
}

oz_status_t oz_scaled_gemm_grouped_k(oz_handle_t h, void* stream, int64_t groups, const int32_t* offsets, int64_t m, int64_t n, int64_t k,
                                     const oz_scaled_t* A, const oz_scaled_t* B, void* C, int64_t ldc, int64_t stride_c, int32_t c_type,
                                     int32_t accumulate) {
    return gemm(h, stream, Grouping::kContraction, groups, offsets, m, n, k, A, B, C, ldc, stride_c, c_type, accumulate, nullptr, 0);
}

size_t oz_sort_tokens_workspace_bytes(oz_handle_t h, int64_t tokens, int64_t topk, int64_t experts) {
    if (!h || tokens < 0 || topk < 0 || experts < 1 || experts > kMaxGroups || tokens > kMaxChoices || topk > kMaxChoices) return 0;
    if (tokens * topk >= kMaxChoices) return 0;
    return sort_tokens_bytes(tokens * topk, experts);
}

oz_status_t oz_sort_tokens(oz_handle_t h, void* stream, int64_t tokens, int64_t topk, int64_t experts, const void* chosen, int32_t id_bytes,
                           int32_t* offsets, int32_t* order, int32_t* place, void* workspace, size_t workspace_bytes) {
    if (!h || tokens < 0 || topk < 0 || experts < 1 || experts > kMaxGroups || tokens > kMaxChoices || topk > kMaxChoices) return OZ_ERR_ARG;
    const int64_t choices = tokens * topk;
    if (choices >= kMaxChoices || (id_bytes != 4 && id_bytes != 8) || !offsets || !is_aligned(offsets, 4)) return OZ_ERR_ARG;
    if (choices > 0 && (!chosen || !order || !place || !is_aligned(chosen, uintptr_t(id_bytes)) || !is_aligned(order, 4) || !is_aligned(place, 4)))
        return OZ_ERR_ARG;
    const size_t need = sort_tokens_bytes(choices, experts);
    if (need > 0 && (!workspace || !is_aligned(workspace, kWorkspaceAlign) || workspace_bytes < need)) return OZ_ERR_WORKSPACE;
    if (!handle_on_device(h)) return OZ_ERR_DEVICE;
    launch_sort_tokens(static_cast<hipStream_t>(stream), int(choices), int(experts), chosen, id_bytes == 8, offsets, order, place,
                       static_cast<int32_t*>(workspace));
    return hipGetLastError() == hipSuccess ? OZ_OK : OZ_ERR_HIP;
}

oz_status_t oz_gather_rows(oz_handle_t h, void* stream, int64_t tokens, int64_t topk, int64_t cols, int32_t type, const void* X, int64_t ldx,
                           const int32_t* order, const int32_t* place, void* Y, int64_t ldy) {
    const int esize = elem_bytes(type);
    if (!h || esize == 0 || topk < 0 || topk > 64 || !rows_ok(tokens, cols, X, ldx, esize) || tokens * topk >= kMaxChoices) return OZ_ERR_ARG;
    const int64_t slots = tokens * topk;
    if (!rows_ok(slots, cols, Y, ldy, esize) || (slots > 0 && (!order || !place))) return OZ_ERR_ARG;
    if (slots == 0 || cols == 0) return OZ_OK;
    if (tokens * ((cols * esize + 4095) / 4096) > 4 * kMaxGrid) return OZ_ERR_ARG;
    if (!handle_on_device(h)) return OZ_ERR_DEVICE;
    launch_gather_rows(static_cast<hipStream_t>(stream), int(tokens), int(topk), int(cols), esize, X, ldx, order, place, Y, ldy);
    return hipGetLastError() == hipSuccess ? OZ_OK : OZ_ERR_HIP;
}

oz_status_t oz_combine_rows(oz_handle_t h, void* stream, int64_t tokens, int64_t topk, int64_t cols, int32_t type, const void* X, int64_t ldx,
                            int64_t slots, const int32_t* place, const float* weights, void* Y, int64_t ldy) {
    const int esize = elem_bytes(type);
    if (!h || esize == 0 || topk < 0 || topk > 64 || !rows_ok(slots, cols, X, ldx, esize) || !rows_ok(tokens, cols, Y, ldy, esize)) return OZ_ERR_ARG;
    if (tokens * topk >= kMaxChoices || (tokens > 0 && topk > 0 && !place)) return OZ_ERR_ARG;
    if (tokens == 0 || cols == 0) return OZ_OK;
    if (tokens * ((cols + 511) / 512) > 4 * kMaxGrid) return OZ_ERR_ARG;
    if (!handle_on_device(h)) return OZ_ERR_DEVICE;
    launch_combine_rows(static_cast<hipStream_t>(stream), int(tokens), int(topk), int(cols), type, X, ldx, int(slots), place, weights, Y, ldy);
    return hipGetLastError() == hipSuccess ? OZ_OK : OZ_ERR_HIP;
}

oz_status_t oz_combine_rows_grad(oz_handle_t h, void* stream, int64_t tokens, int64_t topk, int64_t cols, int32_t type, const void* dY,
                                 int64_t lddy, const void* X, int64_t ldx, int64_t slots, const int32_t* order, const int32_t* place,
                                 const float* weights, void* dX, int64_t lddx, float* dweights) {
    const int esize = elem_bytes(type);
    if (!h || esize == 0 || topk < 0 || topk > 64 || !rows_ok(tokens, cols, dY, lddy, esize) || !rows_ok(slots, cols, dX, lddx, esize)) return OZ_ERR_ARG;
    if (dweights && !rows_ok(slots, cols, X, ldx, esize)) return OZ_ERR_ARG;
    if (tokens * topk >= kMaxChoices || slots != tokens * topk || (slots > 0 && (!place || !order))) return OZ_ERR_ARG;
    if (slots == 0 || (cols == 0 && !dweights)) return OZ_OK;       // rows without columns have products all the same: zeros
    if (slots > 4 * kMaxGrid) return OZ_ERR_ARG;
    if (!handle_on_device(h)) return OZ_ERR_DEVICE;
    launch_combine_grad(static_cast<hipStream_t>(stream), int(tokens), int(topk), int(cols), type, dY, lddy, X, ldx, int(slots), order, place,
                        weights, dX, lddx, dweights);
    return hipGetLastError() == hipSuccess ? OZ_OK : OZ_ERR_HIP;
}

}  // extern "C"
