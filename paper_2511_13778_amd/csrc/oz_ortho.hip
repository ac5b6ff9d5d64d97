// A matrix made orthogonal by Newton-Schulz steps: X0 = G / (|G| + eps), X <- a X + (b A + c A^2) X with A = X X^T.  X is m x n, m <= n (a tall G is
// taken transposed).
//
// A step is three products on v_mfma_f32_16x16x32_f16.  X goes into them in 16 bits; what makes that exact enough is that everything large and
// regular keeps more: with A = diag(d) + O (O without a diagonal) and P = a I + b A + c A^2
//     P_ij = b O_ij + c ((d_i + d_j) O_ij + (O O)_ij),   P_ii = a + b d_i + c (d_i^2 + (O O)_ii),   X <- diag(P_ii) X + offdiag(P) X
// only O, off-diagonals of P and X are rounded to 16 bits as operands, in a power of two's scale; diagonals and sums have 32.  A step multiplies an error in X by up
// to a, so after five a single rounding to 16 bits in one of these places is 2e-4 to 1e-3 of the result (A's diagonal left in O: 2e-3).
//   bfloat16 results, whose own rounding is 1.7e-3, take one 16-bit part of each operand.  O is held in that part alone, so its linear terms in P have 11 bits as well:
//   512 x 1024, before the result's rounding, 5.6e-4 instead of the 5.3e-4 that its rest would leave, for four bytes more of each element written and read.  X
//   keeps its rest, 22 bits in all, since X <- diag(P_ii) X carries it on; 32 instead would leave the same 5.6e-4 for two bytes more.
//   float32 and float16 results take two parts, x = hi + lo with 22 bits, and the products hi hi + hi lo + lo hi; X has 32 bits, O in its linear terms 22.
//
// O, offdiag(P) and X are kept with their rows padded by zeros to whole tiles, so no product has edges.  A and A^2 are symmetric: their tiles below the
// diagonal are computed and written to both sides.
//
// What bounds it is the matrix units for large matrices (4096 x 4096 bfloat16, five steps: 1250 us, 1070 at the rate of the library's product of that size), memory at
// the ends of the tiles for middling ones (16 of 1024 x 2048: 1040 us, of which P X takes 580 where its products alone would be 270: ten bytes for each element of
// X), and the number of launches for small ones (4 of 200 x 300 float32: 108 us in 17).
#include <algorithm>

#include "oz_layer.h"
#include "oz_ortho_plan.h"
#include "oz_scaled_gemm_device.h"

namespace oz {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Scales of the operands: singular values stay below 1.3 (coefficients up to these: include/ozdgemm.h), so entries of X are below 1.3, of O below 0.9,
// off-diagonals of P below a; small ones reach down to 2^-24 below.
constexpr float kScaleX = 4096.0f, kScaleO = 16384.0f, kScaleP = 4096.0f;
constexpr int kStep = 64;                 // of k: 128 bytes of a row
constexpr int kNormParts = 256;

// What a matrix of the batch has in the workspace.  Rows and columns are there up to whole tiles of each product, with zeros behind m and n as far as
// another product reads them: sums run to the next multiple of 64.
struct Ortho {
    const void* g;
    void* y;
    int64_t ldg, stride_g, ldy, stride_y;
    int rows, cols, m, n, ldm, ldn, batch;
    bool tall;
    float a, b, c, eps;
    double* norm;                         // [batch][parts]
    float* x;                             // [batch][ldm][ldn], times kScaleX: with operands of two parts
    f16_t* x_rest;                        // [batch][ldm][ldn], times kScaleX: what xh leaves of X, with operands of one
    float *diag, *scale;                  // [batch][ldm]: of A; of P
    f16_t *xh, *xt, *xt_new, *o, *p;      // [batch][parts] of [ldm][ldn], [ldn][ldm], [ldn][ldm], [ldm][ldm], [ldm][ldm]
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
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    double sum = 0.0;
    // four pieces on their way together (one: 4096 x 4096 bfloat16 25 us)
    constexpr int kAhead = 4;
    const uint32_t all = uint32_t(o.rows) * pieces, step = gridDim.x * 4;           // at most 32768 x 64
    for (uint32_t id = blockIdx.x * 4 + wave; id < all; id += kAhead * step) {
        RowPiece<8, T> raw[kAhead];
        int have[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t at = id + u * step, row = at / uint32_t(pieces);
            const int col = int(at - row * pieces) * 512 + lane * 8;
            have[u] = at < all ? o.cols - col : 0;
            fetch_row<8>(g + int64_t(row) * o.ldg + col, have[u], o.cols, raw[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (u > 0 && id + u * step >= all) break;
            float x[8];
            as_floats(raw[u], have[u], o.cols, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fma(double(x[i]), double(x[i]), sum);
        }
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
    // all of a lane's elements are on their way before the first is used
    T raw[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int y = y0 + 4 * i, r = min(o.tall ? j0 + y : i0 + y, o.rows - 1), c = min(o.tall ? i0 + x : j0 + x, o.cols - 1);
        raw[i] = g[r * o.ldg + c];
    }
    // the parts in one order, by every wave for itself
    double part[kNormParts / 64], sum = 0.0;
#pragma unroll
    for (int p = 0; p < kNormParts / 64; ++p) part[p] = o.norm[b * kNormParts + p * 64 + (threadIdx.x & 63)];
#pragma unroll
    for (int p = 0; p < kNormParts / 64; ++p) sum += part[p];
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    const double inverse = 1.0 / (sqrt(sum) + double(o.eps));
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        // (y, x) along G's own rows
        const int y = y0 + 4 * i, r = o.tall ? j0 + y : i0 + y, c = o.tall ? i0 + x : j0 + x;
        const float v = r < o.rows && c < o.cols ? float(double(to_float(raw[i])) * inverse) : 0.0f;
        if (o.tall) tile[x][y] = v;
        else tile[y][x] = v;
    }
    __syncthreads();
    const int64_t size = int64_t(o.ldm) * o.ldn;
#pragma unroll
    for (int y = y0; y < 64; y += 4) {
        const float v = tile[y][x] * kScaleX, w = tile[x][y] * kScaleX;
        const int64_t at = int64_t(i0 + y) * o.ldn + j0 + x, turned = int64_t(j0 + y) * o.ldm + i0 + x;
        f16_t hi, lo;
        split(v, hi, lo);
        o.xh[b * PARTS * size + at] = hi;
        if (PARTS == 2) {
            o.x[b * size + at] = v;
            o.xh[(b * PARTS + 1) * size + at] = lo;
        } else {
            o.x_rest[b * size + at] = lo;
        }
        split(w, hi, lo);
        o.xt[b * PARTS * size + turned] = hi;
        if (PARTS == 2) o.xt[(b * PARTS + 1) * size + turned] = lo;
    }
}

enum class Product { kGram, kSquare, kApply, kLast };        // kLast: the last step's kApply, which leaves the result

// One tile of a product L R^T, L and R in rows of `k`: T = 32 F rows of each by four waves, (T/2) x (T/2) each, in LDS stages of 64 of k, whose pieces
// of 16 bytes are turned by the row so that reads of 16 rows lie in different banks.  Rows lie in LDS so that a lane's results of two fragments are
// neighbours: 32 rows of a wave are two fragments of 16, of which one has the first four of each eight and the other the last four.  With H = F / 2, acc[s H + j][h H + i][r]
// is row 32 i + 8 (lane % 16 / 4) + 4 h + lane % 4 of L and row 32 j + 8 (lane / 16) + 4 s + r of R, from the wave's corner on.
template <int F>
struct Tile {
    static constexpr int kT = 32 * F, kWave = 16 * F, kH = F / 2;      // rows; of a wave; fragments of half of them
    static constexpr int kStage = 2 * kT * 128, kLds = 2 * kStage;
};
typedef __attribute__((address_space(3))) const v4i32* lds16_t;

template <int N>
struct Int { static constexpr int v = N; };

__device__ __forceinline__ v4f multiply_add(const v4i32& r, const v4i32& l, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, r), __builtin_bit_cast(f16x8, l), c, 0, 0, 0);
}

// Small tiles: a ring of stages, of which all but one are on their way.  Two parts: hi lo and lo hi are summed apart from hi hi and added last.
template <int F, int PARTS>
struct Ring {
    static constexpr int kPlane = Tile<F>::kT * 128, kStage = 2 * PARTS * kPlane, kStages = PARTS == 1 ? 4 : 3, kLds = kStages * kStage;
    static constexpr int kCopies = 2 * PARTS * Tile<F>::kT / 32;          // a wave's, of a stage
};
template <int F, int PARTS>
__device__ __forceinline__ void multiply_small(uint8_t* lds, const f16_t* l, const f16_t* r, int64_t l_part, int64_t r_part, int k, int64_t l_ld, int64_t r_ld, v4f (&acc)[F][F]) {
    using S = Tile<F>;
    using G = Ring<F, PARTS>;
    constexpr int T = S::kT;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lds0 = lds_address(lds), ld_l = uint32_t(l_ld) * 2, ld_r = uint32_t(r_ld) * 2;
    const uint32_t piece = (uint32_t((lane & 7) ^ (lane >> 4)) * 16) ^ ((wave & 1) ? 64u : 0u);
    const uint32_t row8 = uint32_t(lane >> 5) * 8 + uint32_t(lane >> 3 & 3);       // of a transfer's eight
    const uint32_t off_l = row8 * ld_l + piece, off_r = row8 * ld_r + piece;
    const int steps = k / kStep;
    static_assert(F == 2, "two fragments of a wave");
    v4i32 src_l[PARTS], src_r[PARTS];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        src_l[p] = tile_buffer(reinterpret_cast<const uint8_t*>(l + p * l_part), uint32_t(T - 1) * ld_l + uint32_t(k) * 2);
        src_r[p] = tile_buffer(reinterpret_cast<const uint8_t*>(r + p * r_part), uint32_t(T - 1) * ld_r + uint32_t(k) * 2);
    }
    // eight rows a transfer; the four waves take them in turn.  Behind the last step its transfers once more, into a stage that nobody reads: so
    // that as many are always on their way
    auto copy = [&](int s, int stage) {
        const uint32_t at = uint32_t(min(s, steps - 1)) * 128, to = lds0 + uint32_t(stage) * G::kStage;
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int x = 0; x < T / 32; ++x) {
                const uint32_t place = uint32_t(x * 4 + wave) * 8, row = uint32_t(x * 32 + (wave & 1) * 16 + (wave >> 1) * 4);
                copy16_to_lds(src_l[p], off_l, row * ld_l + at, to + uint32_t(2 * p) * G::kPlane + place * 128);
                copy16_to_lds(src_r[p], off_r, row * ld_r + at, to + uint32_t(2 * p + 1) * G::kPlane + place * 128);
            }
    };
    const int q = lane >> 4, x16 = lane & 15;
    const uint32_t sw = uint32_t(x16 >> 1) & 7;
    uint32_t at[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) at[u] = uint32_t(x16) * 128 + ((uint32_t(2 * q + u) ^ sw) * 16);
    const uint32_t wl = uint32_t(wave & 1) * S::kWave * 128, wr = uint32_t(G::kPlane + (wave >> 1) * S::kWave * 128);
    v4f few[F][F];
#pragma unroll
    for (int j = 0; j < F; ++j)
#pragma unroll
        for (int i = 0; i < F; ++i) acc[j][i] = few[j][i] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < G::kStages - 1; ++s) copy(s, s);
    int stage = 0;
    for (int s = 0; s < steps; ++s) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"((G::kStages - 2) * G::kCopies) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        copy(s + G::kStages - 1, stage == 0 ? G::kStages - 1 : stage - 1);
        const uint32_t from = lds0 + uint32_t(stage) * G::kStage;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            v4i32 fl[PARTS][F], fr[PARTS][F];
#pragma unroll
            for (int p = 0; p < PARTS; ++p)
#pragma unroll
                for (int i = 0; i < F; ++i) {
                    fl[p][i] = *reinterpret_cast<lds16_t>(from + uint32_t(2 * p) * G::kPlane + wl + uint32_t(i * 16) * 128 + at[u]);
                    fr[p][i] = *reinterpret_cast<lds16_t>(from + uint32_t(2 * p) * G::kPlane + wr + uint32_t(i * 16) * 128 + at[u]);
                }
#pragma unroll
            for (int j = 0; j < F; ++j)
#pragma unroll
                for (int i = 0; i < F; ++i) {
                    acc[j][i] = multiply_add(fr[0][j], fl[0][i], acc[j][i]);
                    if (PARTS == 2) {
                        few[j][i] = multiply_add(fr[PARTS - 1][j], fl[0][i], few[j][i]);
                        few[j][i] = multiply_add(fr[0][j], fl[PARTS - 1][i], few[j][i]);
                    }
                }
        }
        stage = stage + 1 == G::kStages ? 0 : stage + 1;
    }
    if (PARTS == 2) {
#pragma unroll
        for (int j = 0; j < F; ++j)
#pragma unroll
            for (int i = 0; i < F; ++i) acc[j][i] += few[j][i];
    }
    // what is still on its way lands in stages that nobody reads; the workgroup's LDS is not given back before
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
}

// Large tiles, one wave per SIMD: nothing hides an instruction that delays the next matrix instruction, so reads and transfers lie between them at fixed
// places.  A step goes in four quarters, (L0,R0) (L0,R1) (L1,R1) (L1,R0), of which each needs one new half of an operand, read before it; the next step
// starts with the half of R that this one ended with, hence two forms of a step that take turns, one per LDS stage.  A stage's halves are
// given up as they have been read: X, what a step's first quarter needs, when that step begins, Y, the rest, in its middle.  At both points the waves
// meet, and the transfers of the same half two steps on start: they have one and a half steps to arrive.
template <int F, int PARTS>
__device__ __forceinline__ void multiply_large(uint8_t* lds, const f16_t* l, const f16_t* r, int64_t l_part, int64_t r_part, int k, int64_t l_ld, int64_t r_ld, v4f (&acc)[F][F]) {
    using S = Tile<F>;
    constexpr int T = S::kT, H = S::kH, kPlaces = 2 * H * H, kQuarter = H * H, kReads = 4 * H, kCopies = F;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lds0 = lds_address(lds), ld_l = uint32_t(l_ld) * 2, ld_r = uint32_t(r_ld) * 2;
    const uint32_t bytes_l = uint32_t(T - 1) * ld_l + uint32_t(k) * 2, bytes_r = uint32_t(T - 1) * ld_r + uint32_t(k) * 2;
    const int per = k / kStep, steps = per * (PARTS == 2 ? 3 : 1);
    const v4i32 src_l[2] = {tile_buffer(reinterpret_cast<const uint8_t*>(l), bytes_l),
                            tile_buffer(reinterpret_cast<const uint8_t*>(l + (PARTS == 2 ? l_part : 0)), bytes_l)};
    const v4i32 src_r[2] = {tile_buffer(reinterpret_cast<const uint8_t*>(r), bytes_r),
                            tile_buffer(reinterpret_cast<const uint8_t*>(r + (PARTS == 2 ? r_part : 0)), bytes_r)};
    // a wave's transfers: T/8 rows of half of L and of half of R, eight at a time.  Lane: row lane / 8, piece (lane % 8) turned by the row, which differs by four
    // pieces between even and odd eights.
    const uint32_t mine = uint32_t((wave & 1) * (T / 2) + (wave >> 1) * (T / 8)), odd = (mine >> 3) & 1;            // in LDS
    const uint32_t mine_row = uint32_t((wave & 1) * (T / 2) + (wave >> 1) * (T / 4));                             // of the matrix
    const uint32_t piece = uint32_t((lane & 7) ^ (lane >> 4)) * 16;
    const uint32_t even_piece = odd ? piece ^ 64 : piece, row8 = uint32_t(lane >> 5) * 8 + uint32_t(lane >> 3 & 3);
    const uint32_t off_l[2] = {row8 * ld_l + even_piece, row8 * ld_l + (even_piece ^ 64)}, off_r[2] = {row8 * ld_r + even_piece, row8 * ld_r + (even_piece ^ 64)};
    // transfer x of half hl of L (x < H) or hr of R, of step s, into stage ST
    auto copy1 = [&](auto ST, int s, int hl, int hr, int x) {
        const int pass = PARTS == 2 ? (s >= per) + (s >= 2 * per) : 0;        // hi lo, lo hi, hi hi: the small sums first
        const uint32_t at = uint32_t(s - pass * per) * 128, to = lds0 + decltype(ST)::v * S::kStage;
        if (x < H) {
            const uint32_t place = mine + uint32_t(hl * (T / 4) + x * 8), row = mine_row + uint32_t(x * 16 + hl * 4);
            copy16_to_lds(PARTS == 2 && pass == 1 ? src_l[1] : src_l[0], off_l[x & 1], row * ld_l + at, to + place * 128);
        } else {
            const uint32_t place = mine + uint32_t(hr * (T / 4) + (x - H) * 8), row = mine_row + uint32_t((x - H) * 16 + hr * 4);
            copy16_to_lds(PARTS == 2 && pass == 0 ? src_r[1] : src_r[0], off_r[(x - H) & 1], row * ld_r + at, to + (T + place) * 128);
        }
    };
    const int q = lane >> 4, x16 = lane & 15;
    const uint32_t sw = uint32_t(x16 >> 1) & 7;
    uint32_t rd_l[2][2], rd_r[2][2];          // [stage][half of the fragment's 64 of k]
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t at = lds0 + uint32_t(st) * S::kStage + uint32_t(x16) * 128 + ((uint32_t(2 * q + u) ^ sw) * 16);
            rd_l[st][u] = at + uint32_t(wave & 1) * S::kWave * 128;
            rd_r[st][u] = at + uint32_t(T + (wave >> 1) * S::kWave) * 128;
        }
    v4i32 fl[2][H][2], fr[2][H][2];
    auto read_l = [&](auto ST, int half, int x) {
        fl[half][x >> 1][x & 1] = *reinterpret_cast<lds16_t>(rd_l[decltype(ST)::v][x & 1] + uint32_t(half * (T / 4) + (x >> 1) * 16) * 128);
    };
    auto read_r = [&](auto ST, int half, int x) {
        fr[half][x >> 1][x & 1] = *reinterpret_cast<lds16_t>(rd_r[decltype(ST)::v][x & 1] + uint32_t(half * (T / 4) + (x >> 1) * 16) * 128);
    };
    // where the matrix instructions of place y of a quarter lie; after a new half of L its fragments one after the other
    auto jf = [](bool new_l, int y) constexpr -> int { return new_l ? ((y / H) & 1 ? H - 1 - y % H : y % H) : y / H; };
    auto fi = [](bool new_l, int y) constexpr -> int { return new_l ? y / H : ((y / H) & 1 ? H - 1 - y % H : y % H); };
    auto half_step = [&](auto HH, auto BB, auto&& read, auto&& copy) {
        constexpr int h = decltype(HH)::v, b0 = decltype(BB)::v, b1 = 1 - b0;
#pragma unroll
        for (int x = 0; x < kPlaces; ++x) {
            const int y = x % kQuarter;
            const bool first = x < kQuarter, new_l = h == 1 && first;
            const int hr = (h == 0) == first ? b0 : b1, j = jf(new_l, y), i = fi(new_l, y);
            v4f& s = acc[hr * H + j][h * H + i];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                s = multiply_add(fr[hr][j][u], fl[h][i][u], s);
                // holds the instruction here and its sums in the accumulation registers
                asm volatile("" : "+a"(s));
            }
            __builtin_amdgcn_sched_barrier(0);
            // first half: the other half of R, then L1; second: L0, then, its registers being free, the half of R that is next
#pragma unroll
            for (int z = 0; z < kReads; ++z)
                if ((h == 0 ? z * (kPlaces - kPlaces / 8) / kReads : z < 2 * H ? z * kQuarter / (2 * H) : kQuarter + (z - 2 * H) * (kQuarter * 3 / 4) / (2 * H)) == x) read(z);
#pragma unroll
            for (int c = 0; c < kCopies; ++c)
                if ((2 * c + 1) * kPlaces / (2 * kCopies) == x) copy(c);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto meet = [&]() {
        // two halves may still be on their way
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(2 * kCopies) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // FIRST: the step's LDS stage, and the half of R that it starts with
    auto step = [&](auto FIRST, int s) {
        constexpr int b0 = decltype(FIRST)::v, b1 = 1 - b0;
        // behind the last step its transfers once more, into a stage that nobody reads: no branches
        const int ahead = min(s + 2, steps - 1);
        meet();
        half_step(Int<0>{}, Int<b0>{}, [&](int z) { if (z < 2 * H) read_r(Int<b0>{}, b1, z); else read_l(Int<b0>{}, 1, z - 2 * H); },
                  [&](int c) { copy1(Int<b0>{}, ahead, 0, b0, c); });
        meet();
        half_step(Int<1>{}, Int<b0>{}, [&](int z) { if (z < 2 * H) read_l(Int<b1>{}, 0, z); else read_r(Int<b1>{}, b1, z - 2 * H); },
                  [&](int c) { copy1(Int<b0>{}, ahead, 1, b1, c); });
    };
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int x = 0; x < kCopies; ++x) copy1(Int<0>{}, 0, half, half, x);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int x = 0; x < kCopies; ++x) copy1(Int<1>{}, min(1, steps - 1), half, 1 - half, x);
    // Cleared while the first tiles are on their way, by matrix instructions with zero operands: what the vector ALU writes the register allocator keeps in
    // ordinary registers, and moves over and back in every step.
    const v4i32 zero = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < F; ++j)
#pragma unroll
        for (int i = 0; i < F; ++i) {
            acc[j][i] = multiply_add(zero, zero, v4f{0, 0, 0, 0});
            asm volatile("" : "+a"(acc[j][i]));
        }
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(3 * kCopies) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int x = 0; x < 2 * H; ++x) read_l(Int<0>{}, 0, x);
#pragma unroll
    for (int x = 0; x < 2 * H; ++x) read_r(Int<0>{}, 0, x);
    for (int s = 0;;) {
        step(Int<0>{}, s);
        if (++s == steps) break;
        step(Int<1>{}, s);
        if (++s == steps) break;
    }
    // what is still on its way lands in stages that nobody reads; the workgroup's LDS is not given back before
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
}

typedef uint32_t v2u32 __attribute__((ext_vector_type(2)));
typedef uint32_t v4u32 __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
template <int CTRL>
__device__ __forceinline__ uint32_t from_lane(uint32_t x) { return uint32_t(__builtin_amdgcn_update_dpp(0, int(x), CTRL, 0xF, 0xF, false)); }

// Four 16-bit values of consecutive columns c .. c + 3, as two words, and those of the three other lanes of its four, which have the rows beside: lane
// k gets column c + k of the four rows.
__device__ __forceinline__ v2u32 turn(v2u32 w) {
    const uint32_t lane = threadIdx.x, pick = (lane & 1) ? 0x03020706u : 0x05040100u;
    const uint32_t low = __builtin_amdgcn_perm(from_lane<0xB1>(w[0]), w[0], pick), high = __builtin_amdgcn_perm(from_lane<0xB1>(w[1]), w[1], pick);
    const uint32_t other = from_lane<0x4E>((lane & 2) ? low : high);
    return (lane & 2) ? v2u32{other, high} : v2u32{low, other};
}
// A tile of a matrix that a kernel reads or writes: one offset per lane, one for the wave, no vector arithmetic in between.
struct Region {
    __amdgpu_buffer_rsrc_t buffer;
    uint32_t lane;                        // bytes
    __device__ __forceinline__ Region(void* base, int64_t rows, int64_t ld, int64_t cols, int bytes, uint32_t lane_row, uint32_t lane_col)
        : buffer(__builtin_amdgcn_make_buffer_rsrc(base, 0, int(uint32_t(((rows - 1) * ld + cols) * bytes)), 0x00020000)),
          lane((lane_row * uint32_t(ld) + lane_col) * uint32_t(bytes)) {}
    __device__ __forceinline__ v4u32 load(uint32_t at) const { return __builtin_bit_cast(v4u32, __builtin_amdgcn_raw_buffer_load_b128(buffer, lane, at, 0)); }
    __device__ __forceinline__ void store(uint32_t at, v4u32 w) const { __builtin_amdgcn_raw_buffer_store_b128(w, buffer, lane, at, 0); }
};

// Eight values as 16-bit numbers, two to a word, and what is left of them.
__device__ __forceinline__ float half_of(v4u32 w, int i) { return to_float(__builtin_bit_cast(f16_t, uint16_t(w[i / 2] >> (16 * (i & 1))))); }
__device__ __forceinline__ v4u32 halves(const float (&v)[8]) {
    v4u32 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{v[2 * i], v[2 * i + 1]}), f16x2));
    return w;
}
__device__ __forceinline__ v4u32 rest(const float (&v)[8], v4u32 w) {
    float left[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) left[i] = fmaf(half_of(w, i), -1.0f, v[i]);
    return halves(left);
}
// Rows 0 and 4 on of a lane's eight columns to eight rows of its own column of the first (s 0) or last four.
__device__ __forceinline__ v4u32 turn8(const v4u32 (&w)[2], int s) {
    const v2u32 a = turn(v2u32{w[0][2 * s], w[0][2 * s + 1]}), b = turn(v2u32{w[1][2 * s], w[1][2 * s + 1]});
    return v4u32{a[0], a[1], b[0], b[1]};
}

// 2 x 8 results at (row and row + 4, col .. col + 7) of the caller's matrix, which may end before them unless the tile is `whole`.
template <typename Y>
__device__ __forceinline__ void put_result(const Ortho& o, Y* y, int row, int col, bool whole, const float (&v)[2][8]) {
    Y t[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 8; ++i) put(&t[h][i], v[h][i]);
    auto along = [&](Y* to, const Y (&u)[8], int have) {
        if (whole || have >= 8) {
            __builtin_memcpy(to, u, sizeof(u));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) to[i] = u[i];
        }
    };
    if (!o.tall) {
#pragma unroll
        for (int h = 0; h < 2; ++h) along(y + int64_t(row + 4 * h) * o.ldy + col, t[h], row + 4 * h < o.m ? o.n - col : 0);
    } else if constexpr (sizeof(Y) == 2) {
        v4u32 w[2];
        __builtin_memcpy(w, t, sizeof(w));
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const v4u32 turned = turn8(w, s);
            const int c = col + 4 * s + (threadIdx.x & 3), r0 = row & ~7;
            Y u[8];
            __builtin_memcpy(u, &turned, sizeof(u));
            along(y + int64_t(c) * o.ldy + r0, u, c < o.n ? o.m - r0 : 0);
        }
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (whole || (row + 4 * h < o.m && col + i < o.n)) y[int64_t(col + i) * o.ldy + row + 4 * h] = t[h][i];
    }
}

// Y: the caller's matrix type, where the last step leaves the result
template <Product WHAT, int F, int PARTS, typename Y>
__global__ __launch_bounds__(256, F == 4 ? 2 : 1) void ortho_product_kernel(Ortho o, int tiles_m, int tiles_n) {
    using S = Tile<F>;
    constexpr int T = S::kT;
    extern __shared__ __align__(16) uint8_t lds[];
    const int64_t mm = int64_t(o.ldm) * o.ldm, mn = int64_t(o.ldm) * o.ldn;
    // workgroups are dealt to the 8 XCDs in turn: each gets a run of the batch's tiles, which share operands
    const int xcd = int(blockIdx.x & 7), run = int(gridDim.x >> 3), more = int(gridDim.x & 7);
    const int id = xcd * run + min(xcd, more) + int(blockIdx.x >> 3);
    constexpr bool kApplies = WHAT == Product::kApply || WHAT == Product::kLast;
    const int of = kApplies ? tiles_m * tiles_n : tiles_m * (tiles_m + 1) / 2;
    const int64_t b = id / of;
    const int tile = id - int(b) * of;
    int ti, tj;
    if constexpr (kApplies) {
        // bands of four rows of tiles
        const int band = tile / (4 * tiles_n), high = min(tiles_m - band * 4, 4), in = tile - band * 4 * tiles_n;
        ti = band * 4 + in % high;
        tj = in / high;
    } else {
        // tiles at and below the diagonal, row by row
        ti = int((sqrtf(8.0f * float(tile) + 1.0f) - 1.0f) * 0.5f);
        while ((ti + 1) * (ti + 2) / 2 <= tile) ++ti;
        while (ti * (ti + 1) / 2 > tile) --ti;
        tj = tile - ti * (ti + 1) / 2;
    }
    // ---- what becomes of the sums: a lane has 2 x 8 of each 32 x 32 of its wave, rows 4 apart and columns beside each other
    constexpr int H = S::kH;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lane_row = uint32_t((wave & 1) * S::kWave + (lane & 12) * 2 + (lane & 3)), lane_col = uint32_t((wave >> 1) * S::kWave + (lane >> 4) * 8);
    const uint32_t back_row = lane_col + uint32_t(lane & 3), back_col = lane_row & ~7u;                     // turned
    const int row0 = ti * T + int(lane_row), col0 = tj * T + int(lane_col);
    // read, before the product and then 32 rows ahead: O (times kScaleO) or X (times kScaleX), X of two-part operands in 32 bits, the others in two 16-bit parts
    constexpr bool kReads = WHAT != Product::kGram, kWide = kApplies && PARTS == 2, kTwo = kReads && !kWide && (kApplies || PARTS == 2);
    const int64_t ld = kApplies ? o.ldn : o.ldm, corner = int64_t(ti) * T * ld + tj * T, part = kApplies ? mn : mm;
    f16_t* const to = WHAT == Product::kGram ? o.o + b * PARTS * mm : WHAT == Product::kSquare ? o.p + b * PARTS * mm : o.xh + b * PARTS * mn;
    f16_t* const back = (kApplies ? o.xt_new + b * PARTS * mn : to) + int64_t(tj) * T * o.ldm + ti * T;
    const Region whole_to(to + corner, T, ld, T, 2, lane_row, lane_col), rest_to(to + corner + (PARTS - 1) * part, T, ld, T, 2, lane_row, lane_col);
    const Region whole_back(back, T, o.ldm, T, 2, back_row, back_col), rest_back(back + (PARTS - 1) * part, T, o.ldm, T, 2, back_row, back_col);
    f16_t* const first = WHAT == Product::kSquare ? o.o + b * PARTS * mm + corner : to + corner;
    f16_t* const second = kApplies && PARTS == 1 ? o.x_rest + b * mn + corner : first + (PARTS - 1) * part;
    const Region wide(kWide ? static_cast<void*>(o.x + b * mn + corner) : nullptr, T, ld, T, 4, lane_row, lane_col);
    const Region high(first, T, ld, T, 2, lane_row, lane_col), low(second, T, ld, T, 2, lane_row, lane_col);
    auto place = [&](int i, int h, int j) { return uint32_t(i * 32 + h * 4) * uint32_t(ld) + uint32_t(j * 32); };
    struct Old { v4u32 a[2], b[2]; };          // of the two rows: high and low parts, or the first and last four in 32 bits
    auto fetch = [&](int i, int j) {
        Old x{};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t at = place(i, h, j);
            if constexpr (kWide) {
                x.a[h] = wide.load(at * 4);
                x.b[h] = wide.load(at * 4 + 16);
            } else if constexpr (kReads) {
                x.a[h] = high.load(at * 2);
                if constexpr (kTwo) x.b[h] = low.load(at * 2);
            }
        }
        return x;
    };
    // factor * what was there + add
    auto times_old = [&](const Old& x, int h, int c, float factor, float add) {
        if constexpr (kWide) return fmaf(factor, __uint_as_float(c < 4 ? x.a[h][c & 3] : x.b[h][c & 3]), add);
        if constexpr (kTwo) add = fmaf(factor, half_of(x.b[h], c), add);
        return fmaf(factor, half_of(x.a[h], c), add);
    };
    constexpr int kAhead = H < 2 ? 1 : 2, kEarly = F == 8 ? 1 : kAhead;          // beside 256 sums of a lane there is room for fewer
    Old old[kReads ? H : 1][kReads ? H : 1];
    if constexpr (kReads) {
#pragma unroll
        for (int i = 0; i < kEarly; ++i)
#pragma unroll
            for (int j = 0; j < H; ++j) old[i][j] = fetch(i, j);
    }
    asm volatile("" ::: "memory");
    v4f acc[F][F];
    const f16_t *left, *right;
    int64_t left_part = mm, right_part = mm, left_ld = o.ldm, right_ld = o.ldm;
    int k = (o.m + kStep - 1) / kStep * kStep;
    if constexpr (WHAT == Product::kGram) {
        k = (o.n + kStep - 1) / kStep * kStep;
        left = right = o.xh + b * PARTS * mn;
        left_part = right_part = mn;
        left_ld = right_ld = o.ldn;
    } else if constexpr (WHAT == Product::kSquare) {
        left = right = o.o + b * PARTS * mm;
    } else {
        left = o.p + b * PARTS * mm;
        right = o.xt + b * PARTS * mn;
        right_part = mn;
    }
    left += int64_t(ti) * T * left_ld;
    right += int64_t(tj) * T * right_ld;
    if constexpr (F < 4) multiply_small<F, PARTS>(lds, left, right, left_part, right_part, k, left_ld, right_ld, acc);
    else multiply_large<F, PARTS>(lds, left, right, left_part, right_part, k, left_ld, right_ld, acc);
    float of_col[WHAT == Product::kSquare ? H : 1][8], of_row[kReads ? H : 1][2];
    if constexpr (kReads) {
#pragma unroll
        for (int i = 0; i < H; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) of_row[i][h] = (kApplies ? o.scale : o.diag)[b * o.ldm + row0 + i * 32 + h * 4];
#pragma unroll
        for (int j = 0; j < H; ++j) {
            if constexpr (WHAT == Product::kSquare) __builtin_memcpy(of_col[j], o.diag + b * o.ldm + col0 + j * 32, sizeof(of_col[j]));
        }
    }
    if constexpr (kReads) {
#pragma unroll
        for (int i = kEarly; i < kAhead; ++i)
#pragma unroll
            for (int j = 0; j < H; ++j) old[i][j] = fetch(i, j);
    }
    const bool on_diagonal = !kApplies && ti == tj && (wave & 1) == (wave >> 1);
    const bool whole = WHAT == Product::kLast && (ti + 1) * T <= o.m && (tj + 1) * T <= o.n;
#pragma unroll
    for (int i = 0; i < H; ++i) {
        if constexpr (kReads) {
            if (i + kAhead < H) {
#pragma unroll
                for (int j = 0; j < H; ++j) old[i + kAhead][j] = fetch(i + kAhead, j);
            }
        }
#pragma unroll
        for (int j = 0; j < H; ++j) {
            float v[2][8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float row_part = WHAT == Product::kSquare ? fmaf(o.c, of_row[i][h], o.b) * (kScaleP / kScaleO) : 0.0f;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const float sum = acc[(c >> 2) * H + j][h * H + i][c & 3];
                    if constexpr (kApplies) {
                        v[h][c] = times_old(old[i][j], h, c, of_row[i][h], sum * (1.0f / kScaleP));
                        if constexpr (WHAT == Product::kLast) v[h][c] *= 1.0f / kScaleX;
                    } else if constexpr (WHAT == Product::kGram) {
                        v[h][c] = sum * (kScaleO / (kScaleX * kScaleX));
                    } else {
                        v[h][c] = times_old(old[i][j], h, c, fmaf(o.c * (kScaleP / kScaleO), of_col[j][c], row_part), sum * (o.c * (kScaleP / (kScaleO * kScaleO))));
                    }
                }
            }
            if constexpr (WHAT == Product::kLast) {
                put_result(o, static_cast<Y*>(o.y) + b * o.stride_y, row0 + i * 32, col0 + j * 32, whole, v);
                continue;
            }
            if (!kApplies && i == j && on_diagonal) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if ((lane & 15) == (lane >> 4) * 4 + r) {
                            const int64_t d = b * o.ldm + row0 + i * 32 + h * 4;
                            float& x = v[h][h * 4 + r];
                            if constexpr (WHAT == Product::kGram) o.diag[d] = x * (1.0f / kScaleO);
                            if constexpr (WHAT == Product::kSquare)
                                o.scale[d] = fmaf(of_row[i][h], fmaf(o.c, of_row[i][h], o.b), o.a) + o.c * (acc[h * H + j][h * H + i][r] * (1.0f / (kScaleO * kScaleO)));
                            x = 0.0f;
                        }
            }
            const v4u32 w[2] = {halves(v[0]), halves(v[1])};
            const v4u32 l[2] = {rest(v[0], w[0]), rest(v[1], w[1])};
            const bool both = kApplies || ti != tj;                    // a tile on the diagonal has both of its sides itself
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t at = place(i, h, j), at_back = uint32_t(j * 32 + h * 4) * uint32_t(o.ldm) + uint32_t(i * 32);
                whole_to.store(at * 2, w[h]);
                if (both) whole_back.store(at_back * 2, turn8(w, h));
                if constexpr (kWide) {
                    wide.store(at * 4, v4u32{__float_as_uint(v[h][0]), __float_as_uint(v[h][1]), __float_as_uint(v[h][2]), __float_as_uint(v[h][3])});
                    wide.store(at * 4 + 16, v4u32{__float_as_uint(v[h][4]), __float_as_uint(v[h][5]), __float_as_uint(v[h][6]), __float_as_uint(v[h][7])});
                } else if constexpr (kApplies) {
                    low.store(at * 2, l[h]);
                }
                if constexpr (PARTS == 2) {
                    rest_to.store(at * 2, l[h]);
                    if (both) rest_back.store(at_back * 2, turn8(l, h));
                }
            }
        }
    }
}

struct Plan {
    int64_t m, n, ldm, ldn, chunk;
    OrthoTiles tiles;
    int parts;
    size_t norm, x, vec, xh, o, total;      // bytes of each piece, for a chunk
};
Plan plan_of(int64_t batch, int64_t rows, int64_t cols, int type, int num_cu) {
    Plan p{};
    p.m = std::min(rows, cols);
    p.n = std::max(rows, cols);
    p.parts = type == OZ_BF16 ? 1 : 2;
    p.tiles = ortho_tiles(batch, p.m, p.n, p.parts, num_cu);
    auto up = [](int64_t v, int64_t to) { return (v + to - 1) / to * to; };
    p.ldm = std::max(up(p.m, p.tiles.square), up(p.m, p.tiles.apply));
    p.ldn = up(p.n, p.tiles.apply);
    // as many matrices at a time as make 4096 tiles: more would only take more memory
    const int64_t tiles = up(p.m, p.tiles.apply) / p.tiles.apply * (p.ldn / p.tiles.apply);
    p.chunk = std::min(batch, std::max<int64_t>(1, (4096 + tiles - 1) / tiles));
    auto piece = [&](int64_t elems, int64_t bytes) { return size_t((p.chunk * elems * bytes + 255) / 256 * 256); };
    p.norm = piece(kNormParts, 8);
    p.x = piece(p.ldm * p.ldn, p.parts == 2 ? 4 : 2);
    p.vec = piece(p.ldm, 4);
    p.xh = piece(p.ldm * p.ldn, 2 * p.parts);
    p.o = piece(p.ldm * p.ldm, 2 * p.parts);
    p.total = p.norm + p.x + 2 * p.vec + 3 * p.xh + 2 * p.o;
    return p;
}

template <int F, int PARTS>
constexpr int kLdsOf = F < 4 ? Ring<F, PARTS>::kLds : Tile<F>::kLds;

template <Product WHAT, int F, int PARTS, typename Y>
void launch_product(hipStream_t st, const Ortho& o) {
    constexpr int T = Tile<F>::kT;
    const int tiles_m = (o.m + T - 1) / T, tiles_n = (o.n + T - 1) / T;
    const bool half = WHAT == Product::kGram || WHAT == Product::kSquare;
    const unsigned tiles = unsigned((half ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n) * o.batch);
    constexpr int lds = kLdsOf<F, PARTS>;
    hipLaunchKernelGGL((ortho_product_kernel<WHAT, F, PARTS, Y>), dim3(tiles), dim3(256), lds, st, o, tiles_m, tiles_n);
}
template <Product WHAT, int PARTS, typename Y>
void product(hipStream_t st, const Ortho& o, int tile) {
    if (tile == 64) launch_product<WHAT, 2, PARTS, Y>(st, o);
    else if (tile == 128) launch_product<WHAT, 4, PARTS, Y>(st, o);
    else if (tile == 192) launch_product<WHAT, 6, PARTS, Y>(st, o);
    else launch_product<WHAT, 8, PARTS, Y>(st, o);
}

template <typename Y, int PARTS>
void run(hipStream_t st, Ortho o, const Plan& p, int steps) {
    hipLaunchKernelGGL(ortho_norm_kernel<Y>, dim3(kNormParts, unsigned(o.batch)), dim3(256), 0, st, o);
    hipLaunchKernelGGL((ortho_start_kernel<Y, PARTS>), dim3(unsigned(o.ldn / 64), unsigned(o.ldm / 64), unsigned(o.batch)), dim3(256), 0, st, o);
    for (int s = 0; s < steps; ++s) {
        product<Product::kGram, PARTS, f16_t>(st, o, p.tiles.square);
        product<Product::kSquare, PARTS, f16_t>(st, o, p.tiles.square);
        if (s + 1 < steps) product<Product::kApply, PARTS, f16_t>(st, o, p.tiles.apply);
        else product<Product::kLast, PARTS, Y>(st, o, p.tiles.apply);
        std::swap(o.xt, o.xt_new);
    }
}

template <Product WHAT, int F, int PARTS, typename Y>
bool allow_lds() {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(ortho_product_kernel<WHAT, F, PARTS, Y>), hipFuncAttributeMaxDynamicSharedMemorySize,
                               kLdsOf<F, PARTS>) == hipSuccess;
}
template <int F>
bool allow_tile() {
    return allow_lds<Product::kGram, F, 1, f16_t>() && allow_lds<Product::kGram, F, 2, f16_t>() && allow_lds<Product::kSquare, F, 1, f16_t>() &&
           allow_lds<Product::kSquare, F, 2, f16_t>() && allow_lds<Product::kApply, F, 1, f16_t>() && allow_lds<Product::kApply, F, 2, f16_t>() &&
           allow_lds<Product::kLast, F, 1, bf16_t>() && allow_lds<Product::kLast, F, 2, f16_t>() && allow_lds<Product::kLast, F, 2, float>();
}

}  // namespace

bool prepare_ortho() { return allow_tile<2>() && allow_tile<4>() && allow_tile<6>() && allow_tile<8>(); }

size_t ortho_bytes(int64_t batch, int64_t rows, int64_t cols, int type, int num_cu) {
    return batch > 0 && rows > 0 && cols > 0 ? plan_of(batch, rows, cols, type, num_cu).total : 0;
}

void launch_ortho(hipStream_t st, const OrthoCall& c, int num_cu) {
    const Plan p = plan_of(c.batch, c.rows, c.cols, c.type, num_cu);
    Ortho o{};
    o.ldg = c.ldx; o.stride_g = c.stride_x; o.ldy = c.ldy; o.stride_y = c.stride_y;
    o.rows = c.rows; o.cols = c.cols; o.m = int(p.m); o.n = int(p.n); o.ldm = int(p.ldm); o.ldn = int(p.ldn);
    o.tall = c.rows > c.cols;
    o.a = c.a; o.b = c.b; o.c = c.c; o.eps = c.eps;
    uint8_t* at = static_cast<uint8_t*>(c.ws);
    auto take = [&](size_t bytes) { uint8_t* q = at; at += bytes; return q; };
    o.norm = reinterpret_cast<double*>(take(p.norm));
    uint8_t* const x = take(p.x);
    o.x = reinterpret_cast<float*>(x);
    o.x_rest = reinterpret_cast<f16_t*>(x);
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
