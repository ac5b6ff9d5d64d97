// Quantiser: float32 / bfloat16 / float16 matrices to 8-bit floats with a power-of-two scale per block of 128.
//
//   a = max |x| over the block,  e = least integer >= -126 with a <= M 2^e  (M = 448 = 1.75 2^8, 57344 = 1.75 2^15),
//   value = RNE8(x 2^-e),  scale = 2^e
//
// The scale is a power of two because a floating-point value keeps its relative precision under one: x 2^-e is exact, so the
// conversion to 8 bits is the only rounding, and the matrix unit can apply the scale itself.  e comes from a's exponent field
// and whether its fraction is above 0.75.  What bounds it: memory; each input is read once, also where rows and columns of it
// are wanted.  4100 x 8192 of bfloat16: its rows 18.9 us (5.3 TB/s), both ways 28 us with operands in the last-level cache (4.9 TB/s), 38
// from memory: 2112 tiles of one load and one store phase each are little more than a round of the chip, which ends unevenly.
// 16 x 4096: 2.4 us, the launch.
#include "oz_scaled_device.h"

namespace oz {

namespace {

// ---- magnitudes: an element without its sign, one of 32 bits or two of 16 in a word, whose order is that of the values; an infinity or NaN
// is above all others
typedef uint16_t v2u16 __attribute__((ext_vector_type(2)));
template <typename T>
__device__ __forceinline__ uint32_t magnitudes(uint32_t w) { return w & (sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu); }
template <typename T>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    if constexpr (sizeof(T) == 4) return max(a, b);
    else return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2u16, a), __builtin_bit_cast(v2u16, b)));
}
// the largest of a word, as the bits of a float32
template <typename T>
__device__ __forceinline__ uint32_t float_bits(uint32_t w) {
    if constexpr (sizeof(T) == 4) return w;
    else return __float_as_uint(to_float(__builtin_bit_cast(T, uint16_t(max(w & 0xFFFFu, w >> 16)))));
}
// over the 16 lanes of a group: each lane meets the one 8, 4, 2 and 1 further round
template <int R>
__device__ __forceinline__ uint32_t turned_by(uint32_t w) { return uint32_t(__builtin_amdgcn_mov_dpp(int(w), 0x120 + R, 0xF, 0xF, false)); }
template <typename T>
__device__ __forceinline__ uint32_t largest_of_16(uint32_t w) {
    w = larger<T>(w, turned_by<8>(w));
    w = larger<T>(w, turned_by<4>(w));
    w = larger<T>(w, turned_by<2>(w));
    return larger<T>(w, turned_by<1>(w));
}
template <typename T>
__device__ __forceinline__ uint32_t largest_of_piece(const RowPiece<8, T>& r) {
    uint32_t top = magnitudes<T>(r.w[0]);
#pragma unroll
    for (int i = 1; i < r.kWords; ++i) top = larger<T>(top, magnitudes<T>(r.w[i]));
    return top;
}

// ---- scales, from the bits `top` of a block's largest |x| -----------------------------------------
// e + 127: the sum carries into the exponent where the fraction is above 0.75
template <bool E5M2>
__device__ __forceinline__ uint32_t biased_exponent(uint32_t top) { return uint32_t(max(int((top + 0x1FFFFFu) >> 23) - (E5M2 ? 15 : 8), 1)); }
__device__ __forceinline__ bool is_wild(uint32_t top) { return top >= 0x7F800000u; }
// 2^-e, or NaN (0 only meets zeros)
template <bool E5M2>
__device__ __forceinline__ float multiplier(uint32_t top) {
    return __uint_as_float(is_wild(top) ? 0x7FC00000u : (254u - biased_exponent<E5M2>(top)) << 23);
}
template <bool E5M2>
__device__ __forceinline__ void put_scale(uint8_t* base, int64_t at, bool e8m0, uint32_t top) {
    const uint32_t b = top == 0 ? 127u : biased_exponent<E5M2>(top);
    if (e8m0) base[at] = is_wild(top) ? uint8_t(255) : uint8_t(b);
    else reinterpret_cast<uint32_t*>(base)[at] = is_wild(top) ? 0x7FC00000u : b << 23;
}

// four values in one word; `mul` scales exactly (a power of two, or NaN for a block that has none)
template <bool E5M2>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    int w = __float_as_int(a);             // both halves are written
    if constexpr (E5M2) {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
    } else {
        w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    }
    return uint32_t(w);
}

// The lowest `have` bytes of word w of a run: what lies behind a row's end is zero also where the multiplier is NaN.
__device__ __forceinline__ uint32_t bytes_there(int have, int w) {
    const int n = min(max(have - 4 * w, 0), 4);
    return n == 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1;
}

__device__ __forceinline__ int source_row(const int32_t* __restrict__ order, int div, int x_rows, int r) {
    if (!order) return r;
    const int o = order[r];
    const int s = o < 0 ? -1 : int(uint32_t(o) / uint32_t(div));
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

// A block of 128 per 16 lanes, 8 values a lane: maximum by lane rotations, no LDS.  Loads are cached: with an order a token's row is read
// for each of its choices.  grid (blocks of the matrix / 16, batch)
template <typename T, bool E5M2>
__global__ __launch_bounds__(256) void quantize_rows_kernel(RowArgs p) {
    const uint32_t id = blockIdx.x * 16 + (threadIdx.x >> 4);        // less than 2^31: the caller bounds rows * nblk
    const int r = int(id / uint32_t(p.nblk)), blk = int(id - uint32_t(r) * uint32_t(p.nblk)), l = threadIdx.x & 15;
    if (r >= p.rows) return;               // whole groups of 16 lanes
    const int col = blk * kScaleBlock + l * 8, src = source_row(p.order, p.order_div, p.x_rows, r), have = src < 0 ? 0 : p.cols - col;
    RowPiece<8, T> x;
    fetch_row<8>(static_cast<const T*>(p.x) + int64_t(blockIdx.y) * p.stride_x + int64_t(max(src, 0)) * p.ldx + col, have, p.cols, x);
    settle_row(x, have, p.cols);
    const uint32_t top = float_bits<T>(largest_of_16<T>(largest_of_piece(x)));
    const float mul = multiplier<E5M2>(top);
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = pack4<E5M2>(to_float(x.e[4 * i]) * mul, to_float(x.e[4 * i + 1]) * mul, to_float(x.e[4 * i + 2]) * mul, to_float(x.e[4 * i + 3]) * mul);
    if (is_wild(top)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] &= bytes_there(have, i);
    }
    uint8_t* out = p.out.data + int64_t(blockIdx.y) * p.out.stride + int64_t(r) * p.out.ld;
    if (col < ((p.cols + 15) & ~15)) *reinterpret_cast<uint2*>(out + col) = make_uint2(w[0], w[1]);
    const int64_t esize = p.e8m0 ? 1 : 4;
    if (l == 0) put_scale<E5M2>(p.out.scale + int64_t(blockIdx.y) * p.out.scale_stride * esize, int64_t(r) * p.out.scale_ld + blk, p.e8m0, top);
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
// Thread (g, l): rows R g .. R g + R-1, columns 8l .. 8l+7, in registers throughout; the transposed bytes change places through LDS.
// grid (row tiles, column tiles, batch)
// There eight bytes' place is turned by l: the 16 rows that lanes write at a time meet different banks.
// R: 8, or 4 for calls of up to 1024 tiles, where a thread's own chain of loads and instructions is what takes the time (rows and columns of
// 128 x 128 bfloat16 6.0 -> 4.8 us, 4096 x 1024 7.4 -> 6.4, but 5155 x 3470 20.0 -> 20.4, 4100 x 8192 of float32 38 -> 41).
// Loads are cached: streamed ones are 4 % faster from memory (37.1 -> 35.7 us) but lose a quarter where a kernel before left x in the cache.
// A call of few tiles takes as long as its instructions take to come from memory: maxima are of the elements' own bits, two of 16
// in a word, and what ragged ends need is behind one branch.
template <int R, typename T, bool ROWS_E5M2, bool COLS_E5M2, bool SHARED>
__global__ __launch_bounds__(2048 / R) void quantize_tiles_kernel(TileArgs p) {
    constexpr int kWords = RowPiece<8, T>::kWords, kThreads = 2048 / R;
    __shared__ __align__(16) uint32_t col_words[kScaleBlock / R][16 * kWords];       // thread (g, l)'s column maxima
    __shared__ __align__(16) uint32_t col_top[kScaleBlock];
    __shared__ __align__(16) uint8_t turned[kScaleBlock * kScaleBlock];
    const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
    // dealt to the XCDs in turn: each gets a run of tiles one below the other, so that pieces of transposed rows meet in its L2
    const uint32_t tiles = gridDim.x * gridDim.y, dealt = blockIdx.y * gridDim.x + blockIdx.x, xcd = dealt & 7;
    const uint32_t id = xcd * (tiles >> 3) + min(xcd, tiles & 7) + (dealt >> 3);
    const int tile_c = int(id / gridDim.x), tile_r = int(id - uint32_t(tile_c) * gridDim.x);
    int row0 = tile_r * kScaleBlock, end = p.rows, out_col = row0;
    bool cols_too = p.by_cols.data != nullptr;
    if (p.offsets) {
        const GroupPiece piece = GroupPieces<kScaleBlock>(p.offsets, p.groups, p.rows).template find<true>(tile_r);
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
    const int col = tile_c * kScaleBlock + l * 8, have = p.cols - col;
    const T* x0 = static_cast<const T*>(p.x) + int64_t(blockIdx.z) * p.stride_x + col;
    // a wave's lanes find the sources of its 4 R rows; then all rows are on their way together
    const int found = source_row(p.order, p.order_div, p.x_rows, min(row0 + int(threadIdx.x >> 6) * (4 * R) + int(threadIdx.x & (4 * R - 1)), p.rows - 1));
    RowPiece<8, T> x[R];
    auto fetch = [&](auto&& load) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int row = __shfl(found, (g & 3) * R + i);        // by all lanes
            const int src = row0 + g * R + i < end ? row : -1;
            load(x0 + int64_t(max(src, 0)) * p.ldx, src < 0 ? 0 : have, x[i]);
        }
    };
    if (p.cols >= 8) {
        fetch([](const T* at, int n, RowPiece<8, T>& r) { fetch_long_row<8>(at, n, r); });
        if (have > 0 && have < 8)
#pragma unroll
            for (int i = 0; i < R; ++i) move_down(x[i], have);
    } else {
        fetch([](const T* at, int n, RowPiece<8, T>& r) { fetch_short_row(at, n, r); });
    }
    const int64_t rsize = p.rows_e8m0 ? 1 : 4, csize = p.cols_e8m0 ? 1 : 4;
    uint8_t* rscale = p.by_rows.scale + int64_t(blockIdx.z) * p.by_rows.scale_stride * rsize;
    uint8_t* cscale = p.by_cols.scale + int64_t(blockIdx.z) * p.by_cols.scale_stride * csize;
    uint32_t shared_top = 0;
    if constexpr (SHARED) {
        uint32_t top = largest_of_piece(x[0]);
#pragma unroll
        for (int i = 1; i < R; ++i) top = larger<T>(top, largest_of_piece(x[i]));
        top = largest_of_16<T>(top);
        top = larger<T>(top, uint32_t(__shfl_xor(int(top), 16)));
        top = larger<T>(top, uint32_t(__shfl_xor(int(top), 32)));
        if ((threadIdx.x & 63) == 0) col_top[threadIdx.x >> 6] = top;
        __syncthreads();
        top = col_top[0];
#pragma unroll
        for (int w = 1; w < kThreads / 64; ++w) top = larger<T>(top, col_top[w]);
        shared_top = float_bits<T>(top);
        if (threadIdx.x == 0) {
            if (p.by_rows.data) put_scale<ROWS_E5M2>(rscale, int64_t(tile_r) * p.by_rows.scale_ld + tile_c, p.rows_e8m0, shared_top);
            if (cols_too) put_scale<COLS_E5M2>(cscale, int64_t(tile_c) * p.by_cols.scale_ld + tile_r, p.cols_e8m0, shared_top);
        }
    }
    if (p.by_rows.data) {
        const int r0 = row0 + g * R;
        uint8_t* out = p.by_rows.data + int64_t(blockIdx.z) * p.by_rows.stride + int64_t(r0) * p.by_rows.ld + col;
        const int last = col < ((p.cols + 15) & ~15) ? end - r0 : 0;
        const uint32_t keep[2] = {bytes_there(have, 0), bytes_there(have, 1)};
        uint32_t mine = 0;                       // lane l < R: row l's
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const uint32_t top = SHARED ? shared_top : float_bits<T>(largest_of_16<T>(largest_of_piece(x[i])));
            if (l == i) mine = top;
            const float mul = multiplier<ROWS_E5M2>(top);
            auto at = [&](int j) { return to_float(x[i].e[j]) * mul; };
            const uint2 w = make_uint2(pack4<ROWS_E5M2>(at(0), at(1), at(2), at(3)) & keep[0], pack4<ROWS_E5M2>(at(4), at(5), at(6), at(7)) & keep[1]);
            if (i < last) *reinterpret_cast<uint2*>(out + int64_t(i) * p.by_rows.ld) = w;
        }
        if (!SHARED && l < R && r0 + l < end) put_scale<ROWS_E5M2>(rscale, int64_t(r0 + l) * p.by_rows.scale_ld + tile_c, p.rows_e8m0, mine);
    }
    if (!cols_too) return;                       // the same for all of a workgroup
    if constexpr (!SHARED) {
        uint32_t tops[kWords];
#pragma unroll
        for (int j = 0; j < kWords; ++j) {
            tops[j] = magnitudes<T>(x[0].w[j]);
#pragma unroll
            for (int i = 1; i < R; ++i) tops[j] = larger<T>(tops[j], magnitudes<T>(x[i].w[j]));
        }
#pragma unroll
        for (int j = 0; j < kWords; j += 4) *reinterpret_cast<uint4*>(&col_words[g][l * kWords + j]) = make_uint4(tops[j], tops[j + 1], tops[j + 2], tops[j + 3]);
        __syncthreads();
        if (threadIdx.x < kScaleBlock) {
            constexpr int kPer = 4 / int(sizeof(T));
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < kScaleBlock / R; ++i) top = larger<T>(top, col_words[i][threadIdx.x / kPer]);
            if (kPer == 2) top = (threadIdx.x & 1) ? top >> 16 : top & 0xFFFFu;
            top = float_bits<T>(top);
            col_top[threadIdx.x] = top;
            const int c = tile_c * kScaleBlock + threadIdx.x;
            if (c < p.cols) put_scale<COLS_E5M2>(cscale, int64_t(c) * p.by_cols.scale_ld + out_col / kScaleBlock, p.cols_e8m0, top);
        }
        __syncthreads();
    }
    uint32_t tops[8];
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
        const uint4 v = SHARED ? make_uint4(shared_top, shared_top, shared_top, shared_top) : *reinterpret_cast<const uint4*>(&col_top[l * 8 + j]);
        tops[j] = v.x; tops[j + 1] = v.y; tops[j + 2] = v.z; tops[j + 3] = v.w;
    }
    const int there = end - (row0 + g * R);
    const uint32_t keep[2] = {bytes_there(there, 0), bytes_there(there, 1)};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float mul = multiplier<COLS_E5M2>(tops[j]);
        auto at = [&](int i) { return to_float(x[i].e[j]) * mul; };
        uint8_t* to = turned + (l * 8 + j) * kScaleBlock;
        if constexpr (R == 8)
            *reinterpret_cast<uint2*>(to + (g ^ l) * 8) = make_uint2(pack4<COLS_E5M2>(at(0), at(1), at(2), at(3)) & keep[0], pack4<COLS_E5M2>(at(R - 4), at(R - 3), at(R - 2), at(R - 1)) & keep[1]);
        else
            *reinterpret_cast<uint32_t*>(to + ((g >> 1) ^ l) * 8 + (g & 1) * 4) = pack4<COLS_E5M2>(at(0), at(1), at(2), at(3)) & keep[0];
    }
    __syncthreads();
    // columns to write: all 128 of a group's block, else what is there, up to a multiple of 16
    const int wide = p.offsets ? kScaleBlock : min(kScaleBlock, ((p.rows + 15) & ~15) - row0);
    uint8_t* out = p.by_cols.data + int64_t(blockIdx.z) * p.by_cols.stride;
#pragma unroll
    for (int i = 0; i < 1024 / kThreads; ++i) {
        const int q = i * kThreads + threadIdx.x, tr = q >> 3, piece = (q & 7) * 16;
        const int c = tile_c * kScaleBlock + tr;
        // eight bytes 2p at place 2p ^ l, 2p+1 beside it: in turned order where l is odd
        const int tl = tr >> 3;
        const v4i32 v = *reinterpret_cast<const v4i32*>(turned + tr * kScaleBlock + (((q & 7) * 2) ^ (tl & 14)) * 8);
        if (c < p.cols && piece < wide)
            *reinterpret_cast<v4i32*>(out + int64_t(c) * p.by_cols.ld + out_col + piece) = (tl & 1) ? v4i32{v[2], v[3], v[0], v[1]} : v;
    }
}

template <int R, typename T>
void launch_tiles(hipStream_t st, const QuantizeCall& q, const TileArgs& p, const dim3& grid) {
    const dim3 threads(2048 / R);
    const int kind = (q.tiles ? 4 : 0) + (q.rows_e5m2 ? 2 : 0) + (q.cols_e5m2 ? 1 : 0);
    switch (kind) {
        case 0: hipLaunchKernelGGL((quantize_tiles_kernel<R, T, false, false, false>), grid, threads, 0, st, p); break;
        case 1: hipLaunchKernelGGL((quantize_tiles_kernel<R, T, false, true, false>), grid, threads, 0, st, p); break;
        case 2: hipLaunchKernelGGL((quantize_tiles_kernel<R, T, true, false, false>), grid, threads, 0, st, p); break;
        case 3: hipLaunchKernelGGL((quantize_tiles_kernel<R, T, true, true, false>), grid, threads, 0, st, p); break;
        case 4: hipLaunchKernelGGL((quantize_tiles_kernel<R, T, false, false, true>), grid, threads, 0, st, p); break;
        case 5: hipLaunchKernelGGL((quantize_tiles_kernel<R, T, false, true, true>), grid, threads, 0, st, p); break;
        case 6: hipLaunchKernelGGL((quantize_tiles_kernel<R, T, true, false, true>), grid, threads, 0, st, p); break;
        default: hipLaunchKernelGGL((quantize_tiles_kernel<R, T, true, true, true>), grid, threads, 0, st, p); break;
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
    if (tiles * nblk * q.batch <= 1024) launch_tiles<4, T>(st, q, p, grid);
    else launch_tiles<8, T>(st, q, p, grid);
}

}  // namespace

void launch_quantize(hipStream_t st, const QuantizeCall& q) {
    if (q.x_type == OZ_F32) quantize_typed<float>(st, q);
    else if (q.x_type == OZ_BF16) quantize_typed<bf16_t>(st, q);
    else quantize_typed<f16_t>(st, q);
}

}  // namespace oz
