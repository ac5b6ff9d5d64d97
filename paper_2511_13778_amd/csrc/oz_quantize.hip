// Quantiser: float32 / bfloat16 / float16 matrices to 8-bit floats with a power-of-two scale per block of 128.
//
//   a = max |x| over the block,  e = least integer >= -126 with a <= M 2^e  (M = 448 = 1.75 2^8, 57344 = 1.75 2^15),
//   value = RNE8(x 2^-e),  scale = 2^e
//
// The scale is a power of two because a floating-point value keeps its relative precision under one: x 2^-e is exact, so the
// conversion to 8 bits is the only rounding, and the matrix unit can apply the scale itself.  e comes from a's exponent field
// and one comparison of its fraction with 0.75.  What bounds it: memory; each input is read once, also where rows and columns of it
// are wanted.
#include "oz_scaled_device.h"

namespace oz {

namespace {

// e of a block whose largest |x| has the bits `top` (an infinity or NaN: any value, the caller looks)
template <bool E5M2>
__device__ __forceinline__ int block_exponent(uint32_t top) {
    if (top == 0) return 0;
    const int e = int(top >> 23) - 127 - (E5M2 ? 15 : 8) + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return max(e, -126);
}

__device__ __forceinline__ bool is_wild(uint32_t top) { return top >= 0x7F800000u; }

// four values in one word; `mul` scales exactly (a power of two, or NaN for a block that has none)
template <bool E5M2>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    int w = 0;
    if constexpr (E5M2) {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
    } else {
        w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    }
    return uint32_t(w);
}

struct Scale {
    float mul;        // 2^-e, or NaN
    uint8_t e8m0;
    float value;
};
template <bool E5M2>
__device__ __forceinline__ Scale scale_of(uint32_t top) {
    Scale s;
    const int e = block_exponent<E5M2>(top);      // -126 .. 120
    s.mul = __uint_as_float(uint32_t(127 - e) << 23);
    s.e8m0 = uint8_t(e + 127);
    s.value = __uint_as_float(uint32_t(e + 127) << 23);
    if (is_wild(top)) {
        s.mul = s.value = __uint_as_float(0x7FC00000u);
        s.e8m0 = 255;
    }
    return s;
}

__device__ __forceinline__ void put_scale(uint8_t* base, int64_t at, bool e8m0, const Scale& s) {
    if (e8m0) base[at] = s.e8m0;
    else reinterpret_cast<float*>(base)[at] = s.value;
}

__device__ __forceinline__ int64_t source_row(const int32_t* __restrict__ order, int div, int x_rows, int r) {
    if (!order) return r;
    const int o = order[r];
    const int s = o < 0 ? -1 : o / div;
    return s < x_rows ? s : -1;
}

struct RowArgs {
    const void* x;
    int64_t ldx, stride_x;
    ScaledOperand out;
    const int32_t* order;
    int order_div, x_rows, rows, cols, nblk;
    bool e8m0;
};

// A block of 128 per 16 lanes, 8 values a lane: maximum by shuffles, no LDS.  grid (blocks of the matrix / 16, batch)
template <typename T, bool E5M2>
__global__ __launch_bounds__(256) void quantize_rows_kernel(RowArgs p) {
    const uint32_t id = blockIdx.x * 16 + (threadIdx.x >> 4);        // less than 2^31: the caller bounds rows * nblk
    const int r = int(id / uint32_t(p.nblk)), blk = int(id - uint32_t(r) * uint32_t(p.nblk)), l = threadIdx.x & 15;
    if (r >= p.rows) return;               // whole groups of 16 lanes
    const int col = blk * kScaleBlock + l * 8;
    const int64_t src = source_row(p.order, p.order_div, p.x_rows, r);
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (src >= 0)
        load_row<8>(static_cast<const T*>(p.x) + int64_t(blockIdx.y) * p.stride_x + src * p.ldx + col, p.cols - col, p.cols, x);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) top = max(top, uint32_t(__shfl_xor(int(top), d)));
    const Scale s = scale_of<E5M2>(top);
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = pack4<E5M2>(x[4 * i] * s.mul, x[4 * i + 1] * s.mul, x[4 * i + 2] * s.mul, x[4 * i + 3] * s.mul);
    uint8_t* out = p.out.data + int64_t(blockIdx.y) * p.out.stride + int64_t(r) * p.out.ld;
    if (col < ((p.cols + 15) & ~15)) *reinterpret_cast<uint2*>(out + col) = make_uint2(w[0], w[1]);
    const int64_t esize = p.e8m0 ? 1 : 4;
    if (l == 0) put_scale(p.out.scale + int64_t(blockIdx.y) * p.out.scale_stride * esize, int64_t(r) * p.out.scale_ld + blk, p.e8m0, s);
}

struct TileArgs {
    const void* x;
    int64_t ldx, stride_x;
    ScaledOperand by_rows, by_cols;
    const int32_t* order;
    int order_div, x_rows, rows, cols;
    const int32_t* offsets;
    int groups;
    bool rows_e8m0, cols_e8m0;
};

// A tile of 128 x 128: rows, columns or the whole share a scale; written as it is and transposed from one read.
// Thread (g, l): rows 8g .. 8g+7, columns 8l .. 8l+7, in registers throughout; the transposed bytes change places through LDS.
// grid (row tiles, column tiles, batch)
// There the eight bytes of thread (g, l) lie at place g ^ l of their row: the 16 rows that lanes write at a time meet different banks.
template <typename T, bool ROWS_E5M2, bool COLS_E5M2, bool SHARED>
__global__ __launch_bounds__(256) void quantize_tiles_kernel(TileArgs p) {
    __shared__ __align__(16) uint32_t col_top[16][kScaleBlock];
    __shared__ __align__(16) uint8_t turned[kScaleBlock * kScaleBlock];
    const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
    int row0 = int(blockIdx.x) * kScaleBlock, end = p.rows, out_col = row0;
    bool cols_too = p.by_cols.data != nullptr;
    if (p.offsets) {
        const GroupPiece piece = find_piece<kScaleBlock>(p.offsets, p.groups, p.rows, int(blockIdx.x));
        if (piece.group < 0) return;
        row0 = piece.row;
        end = piece.end;
        if (piece.group == p.groups) cols_too = false;
        // the block's column in the transposed matrix: group g's first is blocks_before, and this is its (piece number)th
        const int lo = clamp_offset(p.offsets, piece.group, p.rows);
        out_col = (piece.blocks_before + (row0 - lo) / kScaleBlock) * kScaleBlock;
        cols_too = cols_too && out_col + kScaleBlock <= p.by_cols.ld;
        if (!cols_too && !p.by_rows.data) return;
    }
    const int col = int(blockIdx.y) * kScaleBlock + l * 8;
    const T* x0 = static_cast<const T*>(p.x) + int64_t(blockIdx.z) * p.stride_x;
    // the rows' places first, then all rows on their way together, then their values
    int from[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) from[i] = p.order ? p.order[min(row0 + g * 8 + i, p.rows - 1)] : row0 + g * 8 + i;
    RowPiece<8, T> piece[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        int src = from[i];
        if (p.order) src = src < 0 || src / p.order_div >= p.x_rows ? -1 : src / p.order_div;
        if (row0 + g * 8 + i >= end) src = -1;
        fetch_row<8>(x0 + int64_t(max(src, 0)) * p.ldx + col, src < 0 ? 0 : p.cols - col, p.cols, piece[i]);
    }
    float x[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) as_floats(piece[i], p.cols - col, p.cols, x[i]);
    auto mag = [](float v) -> uint32_t { return __float_as_uint(v) & 0x7FFFFFFFu; };
    const int64_t rsize = p.rows_e8m0 ? 1 : 4, csize = p.cols_e8m0 ? 1 : 4;
    uint8_t* rscale = p.by_rows.scale + int64_t(blockIdx.z) * p.by_rows.scale_stride * rsize;
    uint8_t* cscale = p.by_cols.scale + int64_t(blockIdx.z) * p.by_cols.scale_stride * csize;
    uint32_t shared_top = 0;
    if constexpr (SHARED) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) shared_top = max(shared_top, mag(x[i][j]));
        for (int d = 1; d < 64; d <<= 1) shared_top = max(shared_top, uint32_t(__shfl_xor(int(shared_top), d)));
        if ((threadIdx.x & 63) == 0) col_top[0][threadIdx.x >> 6] = shared_top;
        __syncthreads();
        shared_top = max(max(col_top[0][0], col_top[0][1]), max(col_top[0][2], col_top[0][3]));
        if (threadIdx.x == 0) {
            if (p.by_rows.data)
                put_scale(rscale, int64_t(blockIdx.x) * p.by_rows.scale_ld + blockIdx.y, p.rows_e8m0, scale_of<ROWS_E5M2>(shared_top));
            if (cols_too)
                put_scale(cscale, int64_t(blockIdx.y) * p.by_cols.scale_ld + blockIdx.x, p.cols_e8m0, scale_of<COLS_E5M2>(shared_top));
        }
    }
    if (p.by_rows.data) {
        uint8_t* out = p.by_rows.data + int64_t(blockIdx.z) * p.by_rows.stride;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = row0 + g * 8 + i;
            uint32_t top = shared_top;
            if constexpr (!SHARED) {
#pragma unroll
                for (int j = 0; j < 8; ++j) top = max(top, mag(x[i][j]));
#pragma unroll
                for (int d = 1; d < 16; d <<= 1) top = max(top, uint32_t(__shfl_xor(int(top), d)));
            }
            const Scale s = scale_of<ROWS_E5M2>(top);
            if (r < end && col < ((p.cols + 15) & ~15)) {
                uint32_t w[2];
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    w[j] = pack4<ROWS_E5M2>(x[i][4 * j] * s.mul, x[i][4 * j + 1] * s.mul, x[i][4 * j + 2] * s.mul, x[i][4 * j + 3] * s.mul);
                *reinterpret_cast<uint2*>(out + int64_t(r) * p.by_rows.ld + col) = make_uint2(w[0], w[1]);
            }
            if constexpr (!SHARED)
                if (l == 0 && r < end) put_scale(rscale, int64_t(r) * p.by_rows.scale_ld + blockIdx.y, p.rows_e8m0, s);
        }
    }
    if (!cols_too) return;                       // the same for all of a workgroup
    if constexpr (!SHARED) {
        uint32_t tops[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            tops[j] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) tops[j] = max(tops[j], mag(x[i][j]));
        }
#pragma unroll
        for (int j = 0; j < 8; j += 4) *reinterpret_cast<uint4*>(&col_top[g][l * 8 + j]) = make_uint4(tops[j], tops[j + 1], tops[j + 2], tops[j + 3]);
        __syncthreads();
        if (threadIdx.x < kScaleBlock) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) top = max(top, col_top[i][threadIdx.x]);
            col_top[0][threadIdx.x] = top;       // this thread alone reads its column
            const int c = int(blockIdx.y) * kScaleBlock + threadIdx.x;
            if (c < p.cols)
                put_scale(cscale, int64_t(c) * p.by_cols.scale_ld + out_col / kScaleBlock, p.cols_e8m0, scale_of<COLS_E5M2>(top));
        }
        __syncthreads();
    }
    uint32_t tops[8];
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
        const uint4 v = SHARED ? make_uint4(shared_top, shared_top, shared_top, shared_top) : *reinterpret_cast<const uint4*>(&col_top[0][l * 8 + j]);
        tops[j] = v.x; tops[j + 1] = v.y; tops[j + 2] = v.z; tops[j + 3] = v.w;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const Scale s = scale_of<COLS_E5M2>(tops[j]);
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            w[i] = pack4<COLS_E5M2>(x[4 * i][j] * s.mul, x[4 * i + 1][j] * s.mul, x[4 * i + 2][j] * s.mul, x[4 * i + 3][j] * s.mul);
        *reinterpret_cast<uint2*>(turned + (l * 8 + j) * kScaleBlock + (g ^ l) * 8) = make_uint2(w[0], w[1]);
    }
    __syncthreads();
    // columns to write: all 128 of a group's block, else what is there, up to a multiple of 16
    const int wide = p.offsets ? kScaleBlock : min(kScaleBlock, ((p.rows + 15) & ~15) - row0);
    uint8_t* out = p.by_cols.data + int64_t(blockIdx.z) * p.by_cols.stride;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int q = i * 256 + threadIdx.x, tr = q >> 3, piece = (q & 7) * 16;
        const int c = int(blockIdx.y) * kScaleBlock + tr;
        // eight bytes 2p at place 2p ^ l, 2p+1 beside it: in turned order where l is odd
        const int tl = tr >> 3;
        const v4i32 v = *reinterpret_cast<const v4i32*>(turned + tr * kScaleBlock + (((q & 7) * 2) ^ (tl & 14)) * 8);
        if (c < p.cols && piece < wide)
            *reinterpret_cast<v4i32*>(out + int64_t(c) * p.by_cols.ld + out_col + piece) = (tl & 1) ? v4i32{v[2], v[3], v[0], v[1]} : v;
    }
}

template <typename T>
void quantize_typed(hipStream_t st, const QuantizeCall& q) {
    const int nblk = (q.cols + kScaleBlock - 1) / kScaleBlock;
    if (!q.tiles && !q.out_cols.data) {
        const RowArgs p{q.x, q.ldx, q.stride_x, q.out_rows, q.order, q.order_div, q.x_rows, q.rows, q.cols, nblk, q.rows_e8m0};
        const dim3 grid(unsigned((int64_t(q.rows) * nblk + 15) / 16), unsigned(q.batch));
        if (q.rows_e5m2) hipLaunchKernelGGL((quantize_rows_kernel<T, true>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((quantize_rows_kernel<T, false>), grid, dim3(256), 0, st, p);
        return;
    }
    const TileArgs p{q.x, q.ldx, q.stride_x, q.out_rows, q.out_cols, q.order, q.order_div, q.x_rows, q.rows, q.cols, q.offsets, q.groups,
                     q.rows_e8m0, q.cols_e8m0};
    const int64_t tiles = q.offsets ? group_pieces(q.rows, q.groups, kScaleBlock) : (q.rows + kScaleBlock - 1) / kScaleBlock;
    const dim3 grid{unsigned(tiles), unsigned(nblk), unsigned(q.batch)};
    const int kind = (q.tiles ? 4 : 0) + (q.rows_e5m2 ? 2 : 0) + (q.cols_e5m2 ? 1 : 0);
    switch (kind) {
        case 0: hipLaunchKernelGGL((quantize_tiles_kernel<T, false, false, false>), grid, dim3(256), 0, st, p); break;
        case 1: hipLaunchKernelGGL((quantize_tiles_kernel<T, false, true, false>), grid, dim3(256), 0, st, p); break;
        case 2: hipLaunchKernelGGL((quantize_tiles_kernel<T, true, false, false>), grid, dim3(256), 0, st, p); break;
        case 3: hipLaunchKernelGGL((quantize_tiles_kernel<T, true, true, false>), grid, dim3(256), 0, st, p); break;
        case 4: hipLaunchKernelGGL((quantize_tiles_kernel<T, false, false, true>), grid, dim3(256), 0, st, p); break;
        case 5: hipLaunchKernelGGL((quantize_tiles_kernel<T, false, true, true>), grid, dim3(256), 0, st, p); break;
        case 6: hipLaunchKernelGGL((quantize_tiles_kernel<T, true, false, true>), grid, dim3(256), 0, st, p); break;
        default: hipLaunchKernelGGL((quantize_tiles_kernel<T, true, true, true>), grid, dim3(256), 0, st, p); break;
    }
}

}  // namespace

void launch_quantize(hipStream_t st, const QuantizeCall& q) {
    if (q.x_type == OZ_F32) quantize_typed<float>(st, q);
    else if (q.x_type == OZ_BF16) quantize_typed<bf16_t>(st, q);
    else quantize_typed<f16_t>(st, q);
}

}  // namespace oz
