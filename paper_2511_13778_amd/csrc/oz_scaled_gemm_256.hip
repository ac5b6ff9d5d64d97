// Product of 8-bit block-scaled matrices with E8M0 scales on 256 x 256 tiles of C: large calls.
//
// Four waves, one per SIMD, each 128 x 128 of C in 256 accumulator registers.  A step is a block of 128 of k: 64 matrix
// instructions in four quarters of 64 x 64, (A0,B0) (A0,B1) (A1,B1) (A1,B0), so that each quarter needs one new half of an operand, which
// the quarter before reads from LDS.  The next step starts with the half of B that this one ended with, hence two forms of
// a step that take turns.
// LDS holds two steps.  Its halves are given up as they have been read: X, what a step's first quarter needs (A0 and one half of
// B), when that step begins, Y, the rest, in its middle.  At both points the waves meet, and the transfers of the same half two steps
// on start: they have one and a half steps to arrive.
#include "oz_scaled_gemm_device.h"

namespace oz {

namespace {

constexpr int kT = 256;                                 // tile
constexpr int kRows = 2 * kT;                           // rows of A and B of a stage
constexpr int kStageBytes = kRows * kScaleBlock;        // 64 KB
constexpr int kScaleBytes = kRows * 4;                  // E8M0: a dword, four blocks of k, per row
static_assert((kStageBytes & (kStageBytes - 1)) == 0, "stages are told apart by one bit of the address");
constexpr int kLds = 2 * kStageBytes + 2 * kScaleBytes;

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
    if (t.k == 0) {
        store_nothing(g, t);
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave & 1) * 128, wn = (wave >> 1) * 128;
    const int steps = (t.k + kScaleBlock - 1) / kScaleBlock, tail = t.k & (kScaleBlock - 1);
    const int q = lane >> 4, x16 = lane & 15;

    const uint32_t lds0 = lds_address(lds);
    // waves 0, 1 bring A, 2, 3 bring B; eight transfers of eight rows per half.  Lane: row lane/8, piece (lane%8) ^ swizzle(row)
    const bool mine_a = wave < 2;
    const uint32_t ld = uint32_t(mine_a ? g.a.ld : g.b.ld);
    const uint32_t last_row = uint32_t((mine_a ? t.rows : t.cols) - 1);
    const v4i32 src = tile_buffer(mine_a ? t.a : t.b, last_row * ld + uint32_t((t.k + 3) & ~3));
    // offset of this lane in an even transfer, and in an odd one
    const uint32_t lane_row = uint32_t(lane >> 3) * ld, piece = uint32_t((lane & 7) ^ (lane >> 4)) * 16;
    const uint32_t lane_off[2] = {lane_row + piece, lane_row + (piece ^ 64)};
    const uint32_t my_rows = uint32_t(wave & 1) * 128 * ld;
    const uint32_t to0 = lds0 + uint32_t(wave) * (128 * kScaleBlock);
    // scales: 64 rows per transfer, two per wave; lane 4 x + f brings row 16 f + x, so that a lane reads four fragments' at once
    auto copy_scales = [&](int s) {
        const int four = (t.block0 + s) & ~3;
        const uint32_t to = lds0 + 2 * kStageBytes + uint32_t((four >> 2) & 1) * kScaleBytes + uint32_t(wave) * 512;
        const int tile0 = mine_a ? t.row : t.col, shift = mine_a ? g.a.shift : g.b.shift;
        const int64_t sld = mine_a ? g.a.scale_ld : g.b.scale_ld;
        const uint8_t* base = (mine_a ? t.sa : t.sb) + int64_t(tile0 >> shift) * sld + four;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint32_t r = min(uint32_t((wave & 1) * 128 + x * 64 + (lane & 3) * 16 + (lane >> 2)), last_row);
            copy4_to_lds(base, uint32_t(((tile0 + int(r)) >> shift) - (tile0 >> shift)) * uint32_t(sld), to + x * 256);
        }
    };
    // transfer x of half `half` of this wave's rows, of step `s`, into stage `stage`
    auto copy1 = [&](int s, int half, int x, int stage) {
        copy16_to_lds(src, lane_off[x & 1], my_rows + uint32_t(half * 64 + x * 8) * ld + uint32_t(s) * kScaleBlock,
                      to0 + uint32_t(stage & 1) * kStageBytes + uint32_t(half * 8 + x) * 1024);
    };
    // bytes behind the end of k in a half that has landed become zero
    auto clear_tail = [&](int s, int half_a, int half_b) {
        for (int x = threadIdx.x; x < kT * 8; x += 256) {
            const int i = x >> 3, keep = tail - (x & 7) * 16;         // row of the half; bytes of this piece that stay
            if (keep >= 16) continue;
            const int r = (i >> 6) * 128 + (i >> 7 ? half_b : half_a) * 64 + (i & 63);
            uint32_t* w = reinterpret_cast<uint32_t*>(lds + (s & 1) * kStageBytes + r * kScaleBlock + (((x ^ (r >> 1)) & 7) << 4));
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int have = min(max(keep - 4 * b, 0), 4);
                w[b] &= have == 4 ? 0xFFFFFFFFu : (1u << (8 * have)) - 1;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    const uint32_t sw = uint32_t(x16 >> 1) & 7;
    const uint32_t p0 = uint32_t(x16) * kScaleBlock + ((uint32_t(2 * q) ^ sw) * 16), p1 = uint32_t(x16) * kScaleBlock + ((uint32_t(2 * q + 1) ^ sw) * 16);
    typedef __attribute__((address_space(3))) const v4i32* lds16_t;
    // where this lane reads pieces 2q and 2q+1 of row x16 of a fragment of A and of B, in the stage that is read
    uint32_t rdA[2] = {lds0 + uint32_t(wm) * kScaleBlock + p0, lds0 + uint32_t(wm) * kScaleBlock + p1};
    uint32_t rdB[2] = {lds0 + uint32_t(kT + wn) * kScaleBlock + p0, lds0 + uint32_t(kT + wn) * kScaleBlock + p1};
    union Frag { v8i32 f; v4i32 h[2]; };
    Frag fa[2][4], fb[2][4];
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
    // scales of the four fragments of a half of A or B: E8M0 bytes of four blocks of k, this step's to be shifted down
    const uint32_t sc_at = lds0 + 2 * kStageBytes + uint32_t(x16 * 16 + wm * 4), sc_bt = lds0 + 2 * kStageBytes + uint32_t(x16 * 16 + (kT + wn) * 4);
    uint32_t sc_buffer = 0;
    int sc_shift = 0;
    auto scales_of = [&](int s) {
        sc_buffer = uint32_t(((t.block0 + s) >> 2) & 1) * kScaleBytes;
        sc_shift = ((t.block0 + s) & 3) * 8;
    };
    typedef uint32_t v4u __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) const v4u* lds4_t;
    v4u sa[2], sb[2], sa_new, sb_new;
    auto read_scales = [&](v4u& to, uint32_t at, int half) { to = *reinterpret_cast<lds4_t>(at + sc_buffer + uint32_t(half) * 256); };

    v4f acc[8][8];
    // quarter (half AH of A, half BH of B): 16 matrix instructions, A's fragments one after the other if NEW_A, else B's: those that
    // the quarter before has read.  Between them eight reads, read8(x), four transfers, copy4(x), and two reads of scales: spread so
    // that neither LDS nor the transfers' path is asked for more than it gives, and the last are back before the waves meet.
    auto quarter = [&](auto AH, auto BH, auto NEW_A, auto&& read8, auto&& copy4, auto&& scales2) {
        constexpr int ah = decltype(AH)::v, bh = decltype(BH)::v;
        constexpr bool new_a = decltype(NEW_A)::v != 0;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const int outer = x >> 2, inner = (outer & 1) ? 3 - (x & 3) : (x & 3);
            const int j = new_a ? inner : outer, i = new_a ? outer : inner;
            acc[bh * 4 + j][ah * 4 + i] = mfma_e8m0<A_E5M2>(fb[bh][j].f, fa[ah][i].f, acc[bh * 4 + j][ah * 4 + i], sb[bh][j], sa[ah][i]);
            // holds the instruction here and its sums in the accumulation registers: nothing else in this block reads them
            asm volatile("" : "+a"(acc[bh * 4 + j][ah * 4 + i]));
            __builtin_amdgcn_sched_barrier(0);
            // 0 .. 7: reads, 8, 9: scales, 10 .. 13: transfers
            constexpr int kOrder[16] = {0, 1, 10, 2, 8, 3, 11, 4, 9, 5, 12, 6, 7, -1, 13, -1};
            const int what = kOrder[x];
            if (what >= 10) copy4(what - 10);
            else if (what >= 8) scales2(what - 8);
            else if (what >= 0) read8(what);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto meet = [&]() {
        // two halves may still be on their way (scales make it a few transfers less)
        asm volatile("s_waitcnt vmcnt(16) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // One step; FIRST: the half of B that it starts with.
    auto step = [&](auto FIRST, int s) {
        constexpr int b0 = decltype(FIRST)::v, b1 = 1 - b0;
        // behind the last step its transfers once more, into a stage that nobody reads: no branches
        const int ahead = min(s + 2, steps - 1);
        meet();
        if (tail && s + 1 == steps) clear_tail(s, 1, b1);
        if (((t.block0 + s + 2) & 3) == 0) copy_scales(ahead);
        auto none = [](int) {};
        quarter(Int<0>{}, Int<b0>{}, Int<0>{}, [&](int x) { read(fb[b1][x >> 1], rdB, b1, x >> 1, x & 1); },
                [&](int x) { copy1(ahead, mine_a ? 0 : b0, x, s); },
                [&](int x) { if (x == 0) read_scales(sb_new, sc_bt, b1); else read_scales(sa_new, sc_at, 1); });
        sa[1] = sa_new >> sc_shift;
        sb[b1] = sb_new >> sc_shift;
        quarter(Int<0>{}, Int<b1>{}, Int<0>{}, [&](int x) { read(fa[1][x >> 1], rdA, 1, x >> 1, x & 1); },
                [&](int x) { copy1(ahead, mine_a ? 0 : b0, 4 + x, s); }, none);
        flip();
        meet();
        if (tail && s + 2 == steps) clear_tail(s + 1, 0, b1);
        scales_of(s + 1);
        quarter(Int<1>{}, Int<b1>{}, Int<1>{}, [&](int x) { read(fa[0][x >> 1], rdA, 0, x >> 1, x & 1); },
                [&](int x) { copy1(ahead, mine_a ? 1 : b1, x, s); }, none);
        quarter(Int<1>{}, Int<b0>{}, Int<0>{}, [&](int x) { read(fb[b1][x >> 1], rdB, b1, x >> 1, x & 1); },
                [&](int x) { copy1(ahead, mine_a ? 1 : b1, 4 + x, s); },
                [&](int x) { if (x == 0) read_scales(sb_new, sc_bt, b1); else read_scales(sa_new, sc_at, 0); });
        sa[0] = sa_new >> sc_shift;
        sb[b1] = sb_new >> sc_shift;
    };

    copy_scales(0);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int x = 0; x < 8; ++x) copy1(0, half, x, 0);
    if (((t.block0 + 1) & 3) == 0) copy_scales(min(1, steps - 1));
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int x = 0; x < 8; ++x)
            copy1(min(1, steps - 1), mine_a ? half : 1 - half, x, 1);
    // Cleared, while the first tiles are on their way, by matrix instructions with zero operands: what the vector ALU writes the register
    // allocator keeps in ordinary registers, and moves to the accumulation registers and back in every step.
    const v8i32 zero = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            acc[j][i] = mfma_plain<false>(zero, zero);
            asm volatile("" : "+a"(acc[j][i]));
        }
    asm volatile("s_waitcnt vmcnt(24)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (tail && steps == 1) clear_tail(0, 0, 0);
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        read(fa[0][x >> 1], rdA, 0, x >> 1, x & 1);
        read(fb[0][x >> 1], rdB, 0, x >> 1, x & 1);
    }
    scales_of(0);
    read_scales(sa[0], sc_at, 0);
    read_scales(sb[0], sc_bt, 0);
    sa[0] = sa[0] >> sc_shift;
    sb[0] = sb[0] >> sc_shift;
    for (int s = 0;;) {
        step(Int<0>{}, s);
        if (++s == steps) break;
        step(Int<1>{}, s);
        if (++s == steps) break;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();        // the other waves have read the last tiles
    store_results<false, 1>(g, acc, lds + wave * 32768, t.c + int64_t(t.row + wm) * g.ldc + t.col + wn, t.rows - wm, t.cols - wn);
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
