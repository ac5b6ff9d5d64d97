// A matrix made orthogonal by Newton-Schulz steps: X0 = G / (|G| + eps), X <- a X + (b A + c A^2) X with A = X X^T.  X is m x n, m <= n (a tall G is
// taken transposed).
//
// A step is three products on v_mfma_f32_16x16x32_f16.  X, in 32 bits, goes into them in 16; what makes that exact enough is that everything large and
// regular stays in 32 bits: with A = diag(d) + O (O without a diagonal) and P = a I + b A + c A^2
//     P_ij = b O_ij + c ((d_i + d_j) O_ij + (O O)_ij),   P_ii = a + b d_i + c (d_i^2 + (O O)_ii),   X <- diag(P_ii) X + offdiag(P) X
// only O, off-diagonals of P and X are rounded to 16 bits as operands, in a power of two's scale.  A step multiplies an error in X by up to a, so
// after five a single rounding to 16 bits in one of these places is 2e-4 to 1e-3 of the result (A's diagonal left in O: 2e-3): bfloat16 results, whose
// own rounding is 1.7e-3, take one 16-bit part of each operand; float32 and float16 results take two, x = hi + lo with 22 bits, and the
// products hi hi + hi lo + lo hi.
//
// O, offdiag(P) and X are kept with their rows padded by zeros to whole tiles, so no product has edges.  A and A^2 are symmetric: their tiles below the
// diagonal are computed and written to both sides.
#include <algorithm>

#include "oz_layer.h"
#include "oz_scaled_gemm_device.h"

namespace oz {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// Scales of the operands: singular values stay below 1.3 (coefficients up to these: include/ozdgemm.h), so entries of X are below 1.3, of O below 0.9,
// off-diagonals of P below a; small ones reach down to 2^-24 below.
constexpr float kScaleX = 4096.0f, kScaleO = 16384.0f, kScaleP = 4096.0f;
constexpr int kStep = 64;                 // of k: 128 bytes of a row
constexpr int kNormParts = 64;

// What a matrix of the batch has in the workspace; everything is padded to tiles.
struct Ortho {
    const void* g;
    void* y;
    int64_t ldg, stride_g, ldy, stride_y;
    int rows, cols, m, n, mp, np, batch, tiles_m, tiles_n;
    bool tall, last;
    float a, b, c, eps;
    double* norm;                         // [batch][parts]
    float* x;                             // [batch][mp][np]
    float* gram;                          // [batch][mp][mp], at and below the diagonal
    float *diag, *scale;                  // [batch][mp]: of A; of P
    f16_t *xh, *xt, *xt_new, *o, *p;      // [batch][parts] of [mp][np], [np][mp], [np][mp], [mp][mp], [mp][mp]
};

__device__ __forceinline__ void split(float v, f16_t& hi, f16_t& lo) {
    hi = static_cast<f16_t>(v);
    lo = static_cast<f16_t>(v - static_cast<float>(hi));
}

// ---- |G|^2, in 64 bits: neither large nor small gradients leave their range
template <typename T>
__global__ __launch_bounds__(256) void ortho_norm_kernel(Ortho o) {
    __shared__ double part[4];
    const int b = blockIdx.y, pieces = (o.cols + 511) / 512;
    const T* g = static_cast<const T*>(o.g) + b * o.stride_g;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double sum = 0.0;
    for (int64_t id = int64_t(blockIdx.x) * 4 + wave; id < int64_t(o.rows) * pieces; id += int64_t(gridDim.x) * 4) {
        const int64_t row = id / pieces;
        const int col = int(id - row * pieces) * 512 + lane * 8;
        float x[8];
        load_row<8>(g + row * o.ldg + col, o.cols - col, o.cols, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fma(double(x[i]), double(x[i]), sum);
    }
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) o.norm[b * kNormParts + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// ---- X0 in 32 bits, and as operands along both of its sides.  64 x 64 of X.
template <typename T, int PARTS>
__global__ __launch_bounds__(256) void ortho_start_kernel(Ortho o) {
    __shared__ float tile[64][65];
    const int b = blockIdx.z, i0 = int(blockIdx.y) * 64, j0 = int(blockIdx.x) * 64;
    const T* g = static_cast<const T*>(o.g) + b * o.stride_g;
    const int x = threadIdx.x & 63, y0 = threadIdx.x >> 6;
    double sum = 0.0;
    for (int p = 0; p < kNormParts; ++p) sum += o.norm[b * kNormParts + p];
    const double inverse = 1.0 / (sqrt(sum) + double(o.eps));
    for (int y = y0; y < 64; y += 4) {
        // (y, x) along G's own rows
        const int r = o.tall ? j0 + y : i0 + y, c = o.tall ? i0 + x : j0 + x;
        const float v = r < o.rows && c < o.cols ? float(double(to_float(g[r * o.ldg + c])) * inverse) : 0.0f;
        if (o.tall) tile[x][y] = v;
        else tile[y][x] = v;
    }
    __syncthreads();
    const int64_t size = int64_t(o.mp) * o.np;
    for (int y = y0; y < 64; y += 4) {
        const float v = tile[y][x], w = tile[x][y];
        const int64_t at = int64_t(i0 + y) * o.np + j0 + x, turned = int64_t(j0 + y) * o.mp + i0 + x;
        o.x[b * size + at] = v;
        f16_t hi, lo;
        split(v * kScaleX, hi, lo);
        o.xh[b * PARTS * size + at] = hi;
        if (PARTS == 2) o.xh[(b * PARTS + 1) * size + at] = lo;
        split(w * kScaleX, hi, lo);
        o.xt[b * PARTS * size + turned] = hi;
        if (PARTS == 2) o.xt[(b * PARTS + 1) * size + turned] = lo;
    }
}

enum class Product { kGram, kSquare, kApply };

// One tile of a product L R^T, L and R in rows of `k`: T x T by four waves.  acc[j][i][r]: row 16 i + lane % 16 of L, row 16 j + 4 (lane / 16) + r of R,
// from the wave's corner on.  Two LDS stages: the transfers of a step lie beside the products of the one before.
template <int T>
struct Tile {
    static constexpr int kWave = T / 2, kF = kWave / 16;          // rows of a wave, fragments of 16
    static constexpr int kStage = 2 * T * 128, kLds = 2 * kStage;
};

template <int T, int PARTS>
__device__ __forceinline__ void multiply(uint8_t* lds, const f16_t* l, const f16_t* r, int64_t l_part, int64_t r_part, int k, v4f (&acc)[Tile<T>::kF][Tile<T>::kF]) {
    using S = Tile<T>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lds0 = lds_address(lds), ld = uint32_t(k) * 2;
    const uint32_t piece = uint32_t((lane & 7) ^ (lane >> 4)) * 16, off[2] = {uint32_t(lane >> 3) * ld + piece, uint32_t(lane >> 3) * ld + (piece ^ 64)};
    const int steps = k / kStep, total = steps * (PARTS == 2 ? 3 : 1);
    // eight rows a transfer; the four waves take them in turn
    auto copy = [&](int s) {
        // hi lo, lo hi, hi hi: the small sums first, so that only a third of the additions are rounded at the size of the result
        const int pass = PARTS == 2 ? s / steps : 2;
        const uint32_t at = uint32_t(PARTS == 2 ? s - pass * steps : s) * 128, to = lds0 + uint32_t(s & 1) * S::kStage;
        const v4i32 src_l = tile_buffer(reinterpret_cast<const uint8_t*>(l + (pass == 1 ? l_part : 0)), uint32_t(T) * ld);
        const v4i32 src_r = tile_buffer(reinterpret_cast<const uint8_t*>(r + (pass == 0 ? r_part : 0)), uint32_t(T) * ld);
#pragma unroll
        for (int x = 0; x < T / 32; ++x) {
            const uint32_t row = uint32_t(x * 4 + wave) * 8;
            copy16_to_lds(src_l, off[wave & 1], row * ld + at, to + row * 128);
            copy16_to_lds(src_r, off[wave & 1], row * ld + at, to + (T + row) * 128);
        }
    };
    const int q = lane >> 4, x16 = lane & 15;
    const uint32_t sw = uint32_t(x16 >> 1) & 7;
    typedef __attribute__((address_space(3))) const v4i32* lds16_t;
    uint32_t at[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) at[u] = uint32_t(x16) * 128 + ((uint32_t(u * 4 + q) ^ sw) * 16);
    const uint32_t wl = uint32_t(wave & 1) * S::kWave * 128, wr = uint32_t(T + (wave >> 1) * S::kWave) * 128;
    copy(0);
    for (int s = 0; s < total; ++s) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s + 1 < total) copy(s + 1);
        const uint32_t from = lds0 + uint32_t(s & 1) * S::kStage;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f16x8 fl[S::kF], fr[S::kF];
#pragma unroll
            for (int i = 0; i < S::kF; ++i) {
                fl[i] = __builtin_bit_cast(f16x8, *reinterpret_cast<lds16_t>(from + wl + uint32_t(i * 16) * 128 + at[u]));
                fr[i] = __builtin_bit_cast(f16x8, *reinterpret_cast<lds16_t>(from + wr + uint32_t(i * 16) * 128 + at[u]));
            }
#pragma unroll
            for (int j = 0; j < S::kF; ++j)
#pragma unroll
                for (int i = 0; i < S::kF; ++i) acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fr[j], fl[i], acc[j][i], 0, 0, 0);
        }
    }
}

// four consecutive elements of an operand, whole and what is left of them
template <int PARTS>
__device__ __forceinline__ void put_operand(f16_t* to, int64_t part, const float (&v)[4]) {
    f16x4 hi, lo;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        f16_t h, l;
        split(v[r], h, l);
        hi[r] = h;
        lo[r] = l;
    }
    *reinterpret_cast<f16x4*>(to) = hi;
    if (PARTS == 2) *reinterpret_cast<f16x4*>(to + part) = lo;
}
template <int PARTS>
__device__ __forceinline__ void put_turned(f16_t* to, int64_t part, int64_t ld, const float (&v)[4]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        f16_t h, l;
        split(v[r], h, l);
        to[r * ld] = h;
        if (PARTS == 2) to[r * ld + part] = l;
    }
}

// Y: the caller's matrix type, where the last step leaves the result
template <Product WHAT, int T, int PARTS, typename Y>
__global__ __launch_bounds__(256) void ortho_product_kernel(Ortho o) {
    using S = Tile<T>;
    extern __shared__ __align__(16) uint8_t lds[];
    const int64_t b = blockIdx.y, mm = int64_t(o.mp) * o.mp, mn = int64_t(o.mp) * o.np;
    int ti, tj;
    if constexpr (WHAT == Product::kApply) {
        ti = int(blockIdx.x) % o.tiles_m;
        tj = int(blockIdx.x) / o.tiles_m;
    } else {
        // tiles at and below the diagonal, row by row
        ti = int((sqrtf(8.0f * float(blockIdx.x) + 1.0f) - 1.0f) * 0.5f);
        while ((ti + 1) * (ti + 2) / 2 <= int(blockIdx.x)) ++ti;
        while (ti * (ti + 1) / 2 > int(blockIdx.x)) --ti;
        tj = int(blockIdx.x) - ti * (ti + 1) / 2;
    }
    v4f acc[S::kF][S::kF];
#pragma unroll
    for (int j = 0; j < S::kF; ++j)
#pragma unroll
        for (int i = 0; i < S::kF; ++i) acc[j][i] = v4f{0, 0, 0, 0};
    if constexpr (WHAT == Product::kGram) {
        const f16_t* x = o.xh + b * PARTS * mn;
        multiply<T, PARTS>(lds, x + int64_t(ti) * T * o.np, x + int64_t(tj) * T * o.np, mn, mn, o.np, acc);
    } else if constexpr (WHAT == Product::kSquare) {
        const f16_t* x = o.o + b * PARTS * mm;
        multiply<T, PARTS>(lds, x + int64_t(ti) * T * o.mp, x + int64_t(tj) * T * o.mp, mm, mm, o.mp, acc);
    } else {
        multiply<T, PARTS>(lds, o.p + b * PARTS * mm + int64_t(ti) * T * o.mp, o.xt + b * PARTS * mn + int64_t(tj) * T * o.mp, mm, mn, o.mp, acc);
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row0 = ti * T + (wave & 1) * S::kWave + (lane & 15), col0 = tj * T + (wave >> 1) * S::kWave + (lane >> 4) * 4;
    const float* diag = o.diag + b * o.mp;
#pragma unroll
    for (int i = 0; i < S::kF; ++i) {
        const int row = row0 + i * 16;
        float of_row = 0.0f;
        if constexpr (WHAT == Product::kSquare) of_row = diag[row];
        if constexpr (WHAT == Product::kApply) of_row = o.scale[b * o.mp + row];
#pragma unroll
        for (int j = 0; j < S::kF; ++j) {
            const int col = col0 + j * 16;
            float v[4];
            if constexpr (WHAT == Product::kApply) {
                float* x = o.x + b * mn + int64_t(row) * o.np + col;
                const v4f old = *reinterpret_cast<const v4f*>(x);
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = fmaf(of_row, old[r], acc[j][i][r] * (1.0f / (kScaleP * kScaleX)));
                if (o.last) {
                    Y* y = static_cast<Y*>(o.y) + b * o.stride_y;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (row < o.m && col + r < o.n) put(o.tall ? y + (col + r) * o.ldy + row : y + row * o.ldy + col + r, v[r]);
                } else {
                    *reinterpret_cast<v4f*>(x) = v4f{v[0], v[1], v[2], v[3]};
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] *= kScaleX;
                    put_operand<PARTS>(o.xh + b * PARTS * mn + int64_t(row) * o.np + col, mn, v);
                    put_turned<PARTS>(o.xt_new + b * PARTS * mn + int64_t(col) * o.mp + row, mn, o.mp, v);
                }
            } else {
                float* a = o.gram + b * mm + int64_t(row) * o.mp + col;
                f16_t* to = (WHAT == Product::kGram ? o.o : o.p) + b * PARTS * mm;
                if constexpr (WHAT == Product::kGram) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        v[r] = acc[j][i][r] * (1.0f / (kScaleX * kScaleX));
                        if (row == col + r) o.diag[b * o.mp + row] = v[r];
                    }
                    *reinterpret_cast<v4f*>(a) = v4f{v[0], v[1], v[2], v[3]};
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = row == col + r ? 0.0f : v[r] * kScaleO;
                } else {
                    const v4f old = *reinterpret_cast<const v4f*>(a), of_col = *reinterpret_cast<const v4f*>(diag + col);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float square = acc[j][i][r] * (1.0f / (kScaleO * kScaleO));
                        if (row == col + r) {
                            o.scale[b * o.mp + row] = fmaf(of_row, fmaf(o.c, of_row, o.b), o.a) + o.c * square;
                            v[r] = 0.0f;
                        } else {
                            v[r] = fmaf(old[r], fmaf(o.c, of_row + of_col[r], o.b), o.c * square) * kScaleP;
                        }
                    }
                }
                put_operand<PARTS>(to + int64_t(row) * o.mp + col, mm, v);
                if (ti != tj) put_turned<PARTS>(to + int64_t(col) * o.mp + row, mm, o.mp, v);
            }
        }
    }
}

int tile_of(int64_t, int64_t m, int64_t) { return m <= 256 ? 64 : 128; }

struct Plan {
    int64_t m, n, mp, np, chunk;
    int tile, parts;
    size_t norm, x, gram, vec, xh, o, total;      // bytes of each piece, for a chunk
};
Plan plan_of(int64_t batch, int64_t rows, int64_t cols, int type) {
    Plan p{};
    p.m = std::min(rows, cols);
    p.n = std::max(rows, cols);
    p.tile = tile_of(batch, p.m, p.n);
    p.mp = (p.m + p.tile - 1) / p.tile * p.tile;
    p.np = (p.n + p.tile - 1) / p.tile * p.tile;
    p.parts = type == OZ_BF16 ? 1 : 2;
    // as many matrices at a time as make 4096 tiles: more would only take more memory
    const int64_t tiles = (p.mp / p.tile) * (p.np / p.tile);
    p.chunk = std::min(batch, std::max<int64_t>(1, (4096 + tiles - 1) / tiles));
    auto piece = [&](int64_t elems, int64_t bytes) { return size_t((p.chunk * elems * bytes + 255) / 256 * 256); };
    p.norm = piece(kNormParts, 8);
    p.x = piece(p.mp * p.np, 4);
    p.gram = piece(p.mp * p.mp, 4);
    p.vec = piece(p.mp, 4);
    p.xh = piece(p.mp * p.np, 2 * p.parts);
    p.o = piece(p.mp * p.mp, 2 * p.parts);
    p.total = p.norm + p.x + p.gram + 2 * p.vec + 3 * p.xh + 2 * p.o;
    return p;
}

template <int T, int PARTS, typename Y>
void products(hipStream_t st, Ortho& o, int steps) {
    const dim3 half(unsigned(o.tiles_m * (o.tiles_m + 1) / 2), unsigned(o.batch)), all(unsigned(o.tiles_m * o.tiles_n), unsigned(o.batch));
    constexpr int lds = Tile<T>::kLds;
    for (int s = 0; s < steps; ++s) {
        o.last = s == steps - 1;
        hipLaunchKernelGGL((ortho_product_kernel<Product::kGram, T, PARTS, f16_t>), half, dim3(256), lds, st, o);
        hipLaunchKernelGGL((ortho_product_kernel<Product::kSquare, T, PARTS, f16_t>), half, dim3(256), lds, st, o);
        hipLaunchKernelGGL((ortho_product_kernel<Product::kApply, T, PARTS, Y>), all, dim3(256), lds, st, o);
        std::swap(o.xt, o.xt_new);
    }
}

template <typename Y, int PARTS>
void run(hipStream_t st, Ortho o, const Plan& p, int steps) {
    hipLaunchKernelGGL(ortho_norm_kernel<Y>, dim3(kNormParts, unsigned(o.batch)), dim3(256), 0, st, o);
    hipLaunchKernelGGL((ortho_start_kernel<Y, PARTS>), dim3(unsigned(o.np / 64), unsigned(o.mp / 64), unsigned(o.batch)), dim3(256), 0, st, o);
    if (p.tile == 64) products<64, PARTS, Y>(st, o, steps);
    else products<128, PARTS, Y>(st, o, steps);
}

template <Product WHAT, int T, int PARTS, typename Y>
bool allow_lds() {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(ortho_product_kernel<WHAT, T, PARTS, Y>), hipFuncAttributeMaxDynamicSharedMemorySize, Tile<T>::kLds) == hipSuccess;
}
template <int T, int PARTS>
bool allow_tile() {
    return allow_lds<Product::kGram, T, PARTS, f16_t>() && allow_lds<Product::kSquare, T, PARTS, f16_t>();
}

}  // namespace

bool prepare_ortho() {
    return allow_tile<128, 1>() && allow_tile<128, 2>() && allow_lds<Product::kApply, 128, 1, bf16_t>() && allow_lds<Product::kApply, 128, 2, f16_t>() &&
           allow_lds<Product::kApply, 128, 2, float>();
}

size_t ortho_bytes(int64_t batch, int64_t rows, int64_t cols, int type) {
    return batch > 0 && rows > 0 && cols > 0 ? plan_of(batch, rows, cols, type).total : 0;
}

void launch_ortho(hipStream_t st, const OrthoCall& c, int) {
    const Plan p = plan_of(c.batch, c.rows, c.cols, c.type);
    Ortho o{};
    o.ldg = c.ldx; o.stride_g = c.stride_x; o.ldy = c.ldy; o.stride_y = c.stride_y;
    o.rows = c.rows; o.cols = c.cols; o.m = int(p.m); o.n = int(p.n); o.mp = int(p.mp); o.np = int(p.np);
    o.tiles_m = o.mp / p.tile; o.tiles_n = o.np / p.tile;
    o.tall = c.rows > c.cols;
    o.a = c.a; o.b = c.b; o.c = c.c; o.eps = c.eps;
    uint8_t* at = static_cast<uint8_t*>(c.ws);
    auto take = [&](size_t bytes) { uint8_t* q = at; at += bytes; return q; };
    o.norm = reinterpret_cast<double*>(take(p.norm));
    o.x = reinterpret_cast<float*>(take(p.x));
    o.gram = reinterpret_cast<float*>(take(p.gram));
    o.diag = reinterpret_cast<float*>(take(p.vec));
    o.scale = reinterpret_cast<float*>(take(p.vec));
    o.xh = reinterpret_cast<f16_t*>(take(p.xh));
    o.xt = reinterpret_cast<f16_t*>(take(p.xh));
    o.xt_new = reinterpret_cast<f16_t*>(take(p.xh));
    o.o = reinterpret_cast<f16_t*>(take(p.o));
    o.p = reinterpret_cast<f16_t*>(take(p.o));
    const int64_t size = c.type == OZ_F32 ? 4 : 2;
    for (int64_t b = 0; b < c.batch; b += p.chunk) {
        o.batch = int(std::min<int64_t>(p.chunk, c.batch - b));
        o.g = static_cast<const uint8_t*>(c.x) + b * c.stride_x * size;
        o.y = static_cast<uint8_t*>(c.y) + b * c.stride_y * size;
        if (c.type == OZ_F32) run<float, 2>(st, o, p, c.steps);
        else if (c.type == OZ_BF16) run<bf16_t, 1>(st, o, p, c.steps);
        else run<f16_t, 2>(st, o, p, c.steps);
    }
}

}  // namespace oz
