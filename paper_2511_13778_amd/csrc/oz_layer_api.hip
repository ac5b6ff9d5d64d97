// C ABI of the router's choice, weights in 4 bits and orthogonal updates: argument checks, then launches on the caller's stream.
#include <cmath>

#include "oz_layer.h"

namespace {

using namespace oz;

constexpr int64_t kMaxRows = int64_t(1) << 24, kMaxBytes = int64_t(1) << 23, kMaxLd = int64_t(1) << 32, kMaxGroups = 1024, kMaxChoices = int64_t(1) << 30;
constexpr int64_t kMaxGrid = (int64_t(1) << 24) - 1;      // workgroups of 256 threads: a launch holds less than 2^32 threads
constexpr int64_t kMaxSide = 32768, kMaxMatrices = 65535;
constexpr size_t kWorkspaceAlign = 256;

int elem_bytes(int32_t type) { return type == OZ_F32 ? 4 : type == OZ_BF16 || type == OZ_F16 ? 2 : 0; }
bool is_aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool there(const void* p, uintptr_t a) { return p && is_aligned(p, a); }

oz_status_t launched() { return hipGetLastError() == hipSuccess ? OZ_OK : OZ_ERR_HIP; }

bool choice_ok(int64_t tokens, int64_t experts, int64_t topk, int64_t ld, int esize) {
    return esize != 0 && tokens >= 0 && experts >= 1 && experts <= kMaxGroups && topk >= 1 && topk <= 64 && topk <= experts && tokens < kMaxChoices / topk &&
           ld >= experts && ld <= kMaxLd;
}

bool check_packed(const oz_packed_t* w, int64_t rows, int64_t cols, bool batched) {
    if (!w || w->reserved_ != 0 || rows < 0 || cols < 0 || rows > kMaxRows || cols > kMaxRows) return false;
    if ((w->group != 32 && w->group != 64 && w->group != 128) || elem_bytes(w->scale_type) == 0) return false;
    const uintptr_t align = uintptr_t(elem_bytes(w->scale_type));
    if (rows > 0 && cols > 0 && (!there(w->data, 16) || !there(w->scale, align))) return false;
    if (w->zero && !is_aligned(w->zero, align)) return false;
    if (w->ld % 16 != 0 || w->ld < (cols + 31) / 32 * 16 || w->ld >= kMaxBytes || w->scale_ld < rows || w->scale_ld > kMaxLd) return false;
    return !batched || (w->stride >= 0 && w->stride % 16 == 0 && w->scale_stride >= 0);
}

PackedOperand operand_of(const oz_packed_t* w) {
    return PackedOperand{static_cast<uint8_t*>(w->data), w->scale, w->zero, w->ld, w->scale_ld, w->stride, w->scale_stride,
                         w->group == 32 ? 5 : w->group == 64 ? 6 : 7, w->scale_type};
}

oz_status_t pack_call(oz_handle_t h, void* stream, int64_t rows, int64_t cols, const void* X, int64_t ldx, int32_t x_type, int64_t batch, int64_t stride_x,
                      const oz_packed_t* W, bool pack) {
    const int esize = elem_bytes(x_type);
    if (!h || esize == 0 || batch < 0 || batch > kMaxMatrices || stride_x < 0 || !check_packed(W, rows, cols, batch > 1)) return OZ_ERR_ARG;
    if (ldx < cols || ldx > kMaxLd) return OZ_ERR_ARG;
    if (batch > 1 && rows > 0 && cols > 0) {
        // what is written must not overlap
        const int64_t need = (rows - 1) * (pack ? W->ld : ldx) + (pack ? (cols + 31) / 32 * 16 : cols);
        if ((pack ? W->stride : stride_x) < need) return OZ_ERR_ARG;
        if (pack && W->scale_stride < ((cols + W->group - 1) / W->group - 1) * W->scale_ld + rows) return OZ_ERR_ARG;
    }
    if (rows == 0 || cols == 0 || batch == 0) return OZ_OK;
    if (!there(X, uintptr_t(esize)) || rows * ((cols + 511) / 512) > 4 * kMaxGrid) return OZ_ERR_ARG;
    if (!handle_on_device(h)) return OZ_ERR_DEVICE;
    PackCall c;
    c.x = X;
    c.ldx = ldx;
    c.stride_x = stride_x;
    c.x_type = x_type;
    c.rows = int(rows);
    c.cols = int(cols);
    c.batch = int(batch);
    c.w = operand_of(W);
    if (pack) launch_pack(static_cast<hipStream_t>(stream), c);
    else launch_unpack(static_cast<hipStream_t>(stream), c);
    return launched();
}

bool ortho_ok(int64_t batch, int64_t rows, int64_t cols, int32_t type) {
    return elem_bytes(type) != 0 && batch >= 0 && batch <= kMaxMatrices && rows >= 0 && cols >= 0 && rows <= kMaxSide && cols <= kMaxSide;
}

}  // namespace

extern "C" {

size_t oz_choose_experts_workspace_bytes(oz_handle_t h, int64_t tokens, int64_t experts) {
    if (!h || tokens < 0 || tokens >= kMaxChoices || experts < 1 || experts > kMaxGroups) return 0;
    return choose_bytes(tokens, experts, handle_compute_units(h));
}

oz_status_t oz_choose_experts(oz_handle_t h, void* stream, int64_t tokens, int64_t experts, int64_t topk, const void* scores, int64_t ld, int32_t type,
                              const uint8_t* live, int32_t normalize, int32_t* ids, float* weights, int32_t* counts, int32_t* counted, float* shares,
                              float* loss, void* workspace, size_t workspace_bytes) {
    const int esize = elem_bytes(type);
    if (!h || !choice_ok(tokens, experts, topk, ld, esize) || (normalize != 0 && normalize != 1)) return OZ_ERR_ARG;
    if (tokens > 0 && (!there(scores, uintptr_t(esize)) || !there(ids, 4) || !there(weights, 4))) return OZ_ERR_ARG;
    const bool any = counts || counted || shares || loss;
    if (any && (!there(counts, 4) || !there(counted, 4) || !there(shares, 4) || !there(loss, 4))) return OZ_ERR_ARG;
    if (any) {
        const size_t need = choose_bytes(tokens, experts, handle_compute_units(h));
        if (!workspace || !is_aligned(workspace, kWorkspaceAlign) || workspace_bytes < need) return OZ_ERR_WORKSPACE;
    } else if (tokens == 0) {
        return OZ_OK;
    }
    if (!handle_on_device(h)) return OZ_ERR_DEVICE;
    launch_choose(static_cast<hipStream_t>(stream),
                  ChooseCall{scores, ld, type, int(tokens), int(experts), int(topk), normalize, live, ids, weights, counts, counted, shares, loss, workspace},
                  handle_compute_units(h));
    return launched();
}

oz_status_t oz_choose_experts_grad(oz_handle_t h, void* stream, int64_t tokens, int64_t experts, int64_t topk, const void* scores, int64_t ld, int32_t type,
                                   const uint8_t* live, int32_t normalize, const int32_t* ids, const float* weights, const float* dweights,
                                   const int32_t* counts, const int32_t* counted, const float* dloss, float factor, void* dscores, int64_t ldd) {
    const int esize = elem_bytes(type);
    if (!h || !choice_ok(tokens, experts, topk, ld, esize) || (normalize != 0 && normalize != 1) || ldd < experts || ldd > kMaxLd) return OZ_ERR_ARG;
    if ((counts == nullptr) != (counted == nullptr) || !is_aligned(counts, 4) || !is_aligned(counted, 4) || !is_aligned(dloss, 4)) return OZ_ERR_ARG;
    if (tokens > 0 && (!there(scores, uintptr_t(esize)) || !there(dscores, uintptr_t(esize)))) return OZ_ERR_ARG;
    if (tokens > 0 && dweights && (!there(ids, 4) || !there(weights, 4) || !is_aligned(dweights, 4))) return OZ_ERR_ARG;
    if (tokens == 0) return OZ_OK;
    if (!handle_on_device(h)) return OZ_ERR_DEVICE;
    launch_choose_grad(static_cast<hipStream_t>(stream),
                       ChooseGradCall{scores, ld, type, int(tokens), int(experts), int(topk), normalize, live, ids, weights, dweights, counts, counted, dloss,
                                      factor, dscores, ldd},
                       handle_compute_units(h));
    return launched();
}

oz_status_t oz_pack4(oz_handle_t h, void* stream, int64_t rows, int64_t cols, const void* X, int64_t ldx, int32_t x_type, int64_t batch, int64_t stride_x,
                     const oz_packed_t* W) {
    return pack_call(h, stream, rows, cols, X, ldx, x_type, batch, stride_x, W, true);
}

oz_status_t oz_unpack4(oz_handle_t h, void* stream, int64_t rows, int64_t cols, void* X, int64_t ldx, int32_t x_type, int64_t batch, int64_t stride_x,
                       const oz_packed_t* W) {
    return pack_call(h, stream, rows, cols, X, ldx, x_type, batch, stride_x, W, false);
}

oz_status_t oz_packed_gemm(oz_handle_t h, void* stream, int64_t groups, const int32_t* offsets, int64_t m, int64_t n, int64_t k, const void* X, int64_t ldx,
                           int32_t x_type, const oz_packed_t* W, void* Y, int64_t ldy, int32_t y_type) {
    const int xsize = elem_bytes(x_type), ysize = elem_bytes(y_type);
    if (!h || xsize == 0 || ysize == 0 || m < 0 || m > kMaxRows || k < 0 || k > kMaxRows) return OZ_ERR_ARG;
    if (offsets ? groups < 1 || groups > kMaxGroups : groups != 0) return OZ_ERR_ARG;
    if (!check_packed(W, n, k, groups > 1) || ldx < k || ldx > kMaxLd || ldy < n || ldy > kMaxLd) return OZ_ERR_ARG;
    if (m == 0 || n == 0) return OZ_OK;
    if (!there(Y, uintptr_t(ysize)) || (k > 0 && !there(X, uintptr_t(xsize))) || !is_aligned(offsets, 4)) return OZ_ERR_ARG;
    if (((m + 15) / 16 + groups + 1) * ((n + 15) / 16) > kMaxGrid / 4) return OZ_ERR_ARG;
    if (!handle_on_device(h)) return OZ_ERR_DEVICE;
    PackedGemm g;
    g.x = X;
    g.ldx = ldx;
    g.x_type = x_type;
    g.w = operand_of(W);
    g.y = Y;
    g.ldy = ldy;
    g.y_type = y_type;
    g.m = int(m);
    g.n = int(n);
    g.k = int(k);
    g.offsets = offsets;
    g.groups = int(groups);
    launch_packed_gemm(static_cast<hipStream_t>(stream), g, handle_compute_units(h));
    return launched();
}

size_t oz_orthogonalize_workspace_bytes(oz_handle_t h, int64_t batch, int64_t rows, int64_t cols, int32_t type) {
    if (!h || !ortho_ok(batch, rows, cols, type)) return 0;
    return ortho_bytes(batch, rows, cols, type, handle_compute_units(h));
}

oz_status_t oz_orthogonalize(oz_handle_t h, void* stream, int64_t batch, int64_t rows, int64_t cols, int32_t type, const void* X, int64_t ldx,
                             int64_t stride_x, void* Y, int64_t ldy, int64_t stride_y, int32_t steps, float a, float b, float c, float eps, void* workspace,
                             size_t workspace_bytes) {
    if (!h || !ortho_ok(batch, rows, cols, type) || ldx < cols || ldx > kMaxLd || ldy < cols || ldy > kMaxLd || stride_x < 0) return OZ_ERR_ARG;
    if (steps < 1 || steps > 64 || !std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c) || !(eps >= 0.0f) || !std::isfinite(eps)) return OZ_ERR_ARG;
    if (batch > 1 && rows > 0 && cols > 0 && stride_y < (rows - 1) * ldy + cols) return OZ_ERR_ARG;       // the results overlap
    if (batch == 0 || rows == 0 || cols == 0) return OZ_OK;
    const uintptr_t esize = uintptr_t(elem_bytes(type));
    if (!there(X, esize) || !there(Y, esize)) return OZ_ERR_ARG;
    const size_t need = ortho_bytes(batch, rows, cols, type, handle_compute_units(h));
    if (!workspace || !is_aligned(workspace, kWorkspaceAlign) || workspace_bytes < need) return OZ_ERR_WORKSPACE;
    if (!handle_on_device(h)) return OZ_ERR_DEVICE;
    launch_ortho(static_cast<hipStream_t>(stream),
                 OrthoCall{X, Y, ldx, stride_x, ldy, stride_y, type, int(batch), int(rows), int(cols), steps, a, b, c, eps, workspace}, handle_compute_units(h));
    return launched();
}

}  // extern "C"
