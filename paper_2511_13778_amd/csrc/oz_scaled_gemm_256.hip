// Product of 8-bit block-scaled matrices with E8M0 scales on 256 x 256 tiles of C: large calls.
//
// Four waves, one per SIMD, each 128 x 128 of C in 256 accumulator registers.  A step is a block of 128 of k: 64 matrix
// instructions in four quarters of 64 x 64, (A0,B0) (A0,B1) (A1,B1) (A1,B0), so that each quarter needs one new half of an operand, which
// the quarter before reads from LDS.  The next step starts with the half of B that this one ended with, hence two forms of
// a step that take turns.  In the middle of a step the registers hold all that its second half needs: there the waves meet, the
// step's LDS stage is given up, and the transfers of the step after next start into it; they have a whole step to arrive.
#include "oz_scaled_gemm_device.h"

namespace oz {

namespace {

constexpr int kT = 256;                                 // tile
constexpr int kRows = 2 * kT;                           // rows of A and B of a stage
constexpr int kStageBytes = kRows * kScaleBlock;        // 64 KB
constexpr int kScaleBytes = kRows * 4;                  // E8M0: a dword, four blocks of k, per row
static_assert((kStageBytes & (kStageBytes - 1)) == 0, "stages are told apart by one bit of the address");
constexpr int kLds = 2 * kStageBytes + 2 * kScaleBytes;
constexpr int kCopies = kRows / 8 / 4;                  // transfers of 1 KB per wave and step

template <int N>
struct Int { static constexpr int v = N; };

template <bool A_E5M2>
__global__ __launch_bounds__(256, 1) void scaled_gemm_256_kernel(ScaledGemm g, int tiles_m, int tiles_n) {
    extern __shared__ __align__(16) uint8_t lds[];
    // Workgroups are dealt to the XCDs in turn: an XCD gets a contiguous run of tiles, in blocks of 8 rows of tiles by 4 columns
    int id = int(blockIdx.x);
    const int total = tiles_m * tiles_n;
    {
        const int per = total / 8, extra = total % 8, xcd = id & 7, slot = id >> 3;
        id = xcd * per + min(xcd, extra) + slot;
    }
    constexpr int kBand = 8;
    const int band = id / (kBand * tiles_n), in_band = id - band * kBand * tiles_n;
    const int high = min(kBand, tiles_m - band * kBand);
    const int tile_m = band * kBand + in_band % high, tile_n = in_band / high;

    const GemmTile t = locate<kT, kT>(g, tile_m, tile_n, int(blockIdx.y));
    if (t.none) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave & 1) * 128, wn = (wave >> 1) * 128;
    const int steps = (t.k + kScaleBlock - 1) / kScaleBlock, tail = t.k & (kScaleBlock - 1);
    const int q = lane >> 4, x16 = lane & 15;

    // Cleared by matrix instructions with zero operands: what the vector ALU writes the register allocator keeps in ordinary
    // registers, and moves to the accumulation registers and back in every step.
    v4f acc[8][8];
    const v8i32 zero = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[j][i] = mfma_plain<false>(zero, zero);

    if (steps > 0) {
        const uint32_t lds0 = lds_address(lds);
        const uint32_t piece = uint32_t((lane & 7) ^ (lane >> 3)) * 16;
        // waves 0, 1 bring A, 2, 3 bring B: 16 transfers of eight rows each
        const bool mine_a = wave < 2;
        const uint8_t* src = mine_a ? t.a : t.b;
        const uint32_t ld = uint32_t(mine_a ? g.a.ld : g.b.ld);
        const uint32_t last_row = uint32_t((mine_a ? t.rows : t.cols) - 1);
        uint32_t row0 = uint32_t((wave & 1) * 128 + (lane >> 3));
        const uint32_t back = tail && int(piece) >= tail ? piece : 0;      // nothing may be read behind a row's end
        const uint32_t to0 = lds0 + uint32_t(wave) * (kCopies * 1024);
        // scales: 64 rows per transfer, two per wave
        auto copy_scales = [&](int s) {
            const int four = (t.block0 + s) & ~3;
            const uint32_t to = lds0 + 2 * kStageBytes + uint32_t((four >> 2) & 1) * kScaleBytes + uint32_t(wave) * 512;
            const int tile0 = mine_a ? t.row : t.col, shift = mine_a ? g.a.shift : g.b.shift;
            const int64_t sld = mine_a ? g.a.scale_ld : g.b.scale_ld;
            const uint8_t* base = (mine_a ? t.sa : t.sb) + int64_t(tile0 >> shift) * sld + four;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint32_t r = min(uint32_t((wave & 1) * 128 + x * 64 + lane), last_row);
                copy4_to_lds(base, uint32_t(((tile0 + int(r)) >> shift) - (tile0 >> shift)) * uint32_t(sld), to + x * 256);
            }
        };
        // Eight rows: the addresses are made anew for every transfer, in the matrix instructions' shadow, because registers are short.
        auto copy1 = [&](int s, int x, uint32_t less, int stage) {
            asm volatile("" : "+v"(row0));
            const uint32_t off = __umul24(min(row0 + uint32_t(x) * 8, last_row), ld) + (piece - less);
            copy16_to_lds(src + int64_t(s) * kScaleBlock, off, to0 + uint32_t(stage & 1) * kStageBytes + uint32_t(x) * 1024);
        };
        // bytes behind the end of k in a stage that has landed become zero
        auto clear_tail = [&](int s) {
            for (int x = threadIdx.x; x < kRows * 8; x += 256) {
                const int r = x >> 3, keep = tail - (x & 7) * 16;         // bytes of this piece that stay
                if (keep >= 16) continue;
                uint32_t* w = reinterpret_cast<uint32_t*>(lds + (s & 1) * kStageBytes + r * kScaleBlock + (((x ^ r) & 7) << 4));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int have = min(max(keep - 4 * i, 0), 4);
                    w[i] &= have == 4 ? 0xFFFFFFFFu : (1u << (8 * have)) - 1;
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };

        const uint32_t sw = uint32_t(lane & 7);
        const uint32_t p0 = uint32_t(x16) * kScaleBlock + ((uint32_t(2 * q) ^ sw) * 16), p1 = uint32_t(x16) * kScaleBlock + ((uint32_t(2 * q + 1) ^ sw) * 16);
        typedef __attribute__((address_space(3))) const v4i32* lds16_t;
        typedef __attribute__((address_space(3))) const uint32_t* lds4_t;
        // where this lane reads pieces 2q and 2q+1 of row x16 of a fragment of A and of B, in the stage that is read
        uint32_t rdA[2] = {lds0 + uint32_t(wm) * kScaleBlock + p0, lds0 + uint32_t(wm) * kScaleBlock + p1};
        uint32_t rdB[2] = {lds0 + uint32_t(kT + wn) * kScaleBlock + p0, lds0 + uint32_t(kT + wn) * kScaleBlock + p1};
        union Frag { v8i32 f; v4i32 h[2]; };
        Frag fa[2][4], fb[2][4];
        uint32_t sa[8], sb[8];
        // half h of fragment f of half `which` of an operand
        auto read = [&](Frag& to, const uint32_t (&rd)[2], int which, int f, int h) {
            to.h[h] = *reinterpret_cast<lds16_t>(rd[h] + uint32_t(which * 64 + f * 16) * kScaleBlock);
        };
        auto flip = [&]() {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                rdA[h] ^= kStageBytes;
                rdB[h] ^= kStageBytes;
            }
        };
        auto read_scales = [&](int s) {
            uint32_t at = lds0 + 2 * kStageBytes + uint32_t(((t.block0 + s) >> 2) & 1) * kScaleBytes + uint32_t(x16) * 4 + uint32_t(wm) * 4;
            uint32_t bt = at + uint32_t(kT + wn - wm) * 4;
            asm volatile("" : "+v"(at), "+v"(bt));         // else sixteen addresses are kept for the whole loop
            const int shift = ((t.block0 + s) & 3) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sa[i] = *reinterpret_cast<lds4_t>(at + uint32_t(i) * 64) >> shift;
                sb[i] = *reinterpret_cast<lds4_t>(bt + uint32_t(i) * 64) >> shift;
            }
        };

        // quarter (half AH of A, half BH of B): 16 matrix instructions, `more(x)` after the x-th
        auto quarter = [&](auto AH, auto BH, auto&& more) {
            constexpr int ah = decltype(AH)::v, bh = decltype(BH)::v;
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const int j = x >> 2, i = (j & 1) ? 3 - (x & 3) : (x & 3);
                acc[bh * 4 + j][ah * 4 + i] = mfma_e8m0<A_E5M2>(fb[bh][j].f, fa[ah][i].f, acc[bh * 4 + j][ah * 4 + i], sb[bh * 4 + j], sa[ah * 4 + i]);
                // holds the instruction here and its sums in the accumulation registers: nothing else in this block reads them
                asm volatile("" : "+a"(acc[bh * 4 + j][ah * 4 + i]));
                __builtin_amdgcn_sched_barrier(0);
                more(x);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // One step; FIRST: the half of B that it starts with.
        auto step = [&](auto FIRST, int s) {
            constexpr int b0 = decltype(FIRST)::v, b1 = 1 - b0;
            quarter(Int<0>{}, Int<b0>{}, [&](int x) { if (x < 8) read(fb[b1][x >> 1], rdB, b1, x >> 1, x & 1); });
            quarter(Int<0>{}, Int<b1>{}, [&](int x) { if (x < 8) read(fa[1][x >> 1], rdA, 1, x >> 1, x & 1); });
            // every wave has its operands of this step, and the next step's tiles are there
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (tail && s + 2 == steps) clear_tail(s + 1);
            flip();
            // behind the last step its transfers once more, into a stage that nobody reads: no branches
            const int ahead = min(s + 2, steps - 1);
            const uint32_t less = ahead == steps - 1 ? back : 0;
            if (((t.block0 + s + 2) & 3) == 0) copy_scales(ahead);
            quarter(Int<1>{}, Int<b1>{}, [&](int x) {
                if (x < 8) read(fa[0][x >> 1], rdA, 0, x >> 1, x & 1);
                else copy1(ahead, x - 8, less, s);
            });
            quarter(Int<1>{}, Int<b0>{}, [&](int x) {
                if (x < 8) read(fb[b1][x >> 1], rdB, b1, x >> 1, x & 1);
                else copy1(ahead, x, less, s);
            });
            if (((t.block0 + s + 1) & 3) == 0) read_scales(s + 1);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) { sa[i] >>= 8; sb[i] >>= 8; }
        };

        copy_scales(0);
#pragma unroll
        for (int x = 0; x < kCopies; ++x) copy1(0, x, steps == 1 ? back : 0, 0);
        wait_copies<0>();
        {
            const int ahead = min(1, steps - 1);
            if (((t.block0 + 1) & 3) == 0) copy_scales(ahead);
#pragma unroll
            for (int x = 0; x < kCopies; ++x) copy1(ahead, x, steps <= 2 ? back : 0, 1);
        }
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (tail && steps == 1) clear_tail(0);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            read(fa[0][x >> 1], rdA, 0, x >> 1, x & 1);
            read(fb[0][x >> 1], rdB, 0, x >> 1, x & 1);
        }
        read_scales(0);
        for (int s = 0;;) {
            step(Int<0>{}, s);
            if (++s == steps) break;
            step(Int<1>{}, s);
            if (++s == steps) break;
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    }

    if (steps == 0 && g.accumulate) return;
    __builtin_amdgcn_s_barrier();        // the other waves have read the last tiles
    store_results<2, 1, 8, 8>(g, acc, lds + wave * 32768, t.c + int64_t(t.row + wm) * g.ldc + t.col + wn, t.rows - wm, t.cols - wn);
}

}  // namespace

bool prepare_scaled_gemm() {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(scaled_gemm_256_kernel<false>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds) == hipSuccess &&
           hipFuncSetAttribute(reinterpret_cast<const void*>(scaled_gemm_256_kernel<true>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds) == hipSuccess;
}

void launch_scaled_gemm_256(hipStream_t st, const ScaledGemm& g) {
    const int tiles_n = (g.n + kT - 1) / kT;
    const int64_t tiles_m = g.grouping == Grouping::kRows ? group_pieces(g.m, g.groups, kT) : (g.m + kT - 1) / kT;
    const dim3 grid(unsigned(tiles_m * tiles_n), g.grouping == Grouping::kContraction ? unsigned(g.groups) : 1u);
    if (g.a_e5m2) hipLaunchKernelGGL(scaled_gemm_256_kernel<true>, grid, dim3(256), kLds, st, g, int(tiles_m), tiles_n);
    else hipLaunchKernelGGL(scaled_gemm_256_kernel<false>, grid, dim3(256), kLds, st, g, int(tiles_m), tiles_n);
}

}  // namespace oz
