// Product of 8-bit block-scaled matrices on tiles of 256 x 64 NB of C (NB 4: 256 x 256, 2: 256 x 128): large calls.
//
// Four waves, one per SIMD, each 128 x 32 NB of C.  A step is a block of 128 of k, in four quarters of 64 x 16 NB, (A0,B0) (A0,B1) (A1,B1)
// (A1,B0), so that each quarter needs one new half of an operand, which is read from LDS before.  The next step starts with the
// half of B that this one ended with, hence two forms of a step that take turns, one per LDS stage.
// LDS holds two steps.  Its halves are given up as they have been read: X, what a step's first quarter needs (A0 and one half of
// B), when that step begins, Y, the rest, in its middle.  At both points the waves meet, and the transfers of the same half two steps
// on start: they have one and a half steps to arrive.  Reads, transfers and what little else there is lie in the matrix instructions'
// shadow, at places that are fixed here: one wave per SIMD, so nothing hides an instruction that delays the next one.
//
// E8M0 scales go into the matrix instruction, sums stay in the accumulation registers.  float32 scales are applied to a
// block's sums three matrix instructions after the one that made them, in ordinary registers: four multiply-adds where 128 rows of B
// share a scale (one factor per row of A then), eight where each has its own.
//
// What bounds it: at 8192^3 (E8M0, 256 x 256) 367 to 407 us, 2.7 to 3.0 PFLOP/s, 1.03 to 1.15 of the library's product with one scale
// for all, the power limit: the matrix unit is busy 72 % of the cycles at 2.0 to 2.1 GHz.  A tile's first loads and its results cost 9 us of about
// 95, and nothing hides them: a workgroup that went on to its next tile's loads while it stored took 389 where this took 390 (float32
// scales 645 against 620): its registers for two tiles' places slow the walk over k by as much.  float32 scales 609 to 651 us with one
// per 128 rows of B (3 to 4 % less with both scales multiplied first, which loses range), 684 to 774 with one per row.  There the matrix unit is busy 39 and
// 34 % of the cycles, vector instructions (matrix ones among them) are issued in 34 and 46 %, and waves wait in 23 and 21 %: with one wave
// per SIMD these add up, which of the waits could go is not known.  LDS is active 40 % (E8M0) and 30 to 32 %.
#pragma once

#include "oz_scaled_gemm_device.h"

namespace oz {

namespace {

enum class Scales { kE8M0, kBlocks, kRows };

template <int N>
struct Int { static constexpr int v = N; };

constexpr int kTM = 256;

template <int NB, Scales SC>
struct Big {
    static constexpr int kTN = 64 * NB, kRows = kTM + kTN;
    static constexpr int kStageBytes = kRows * kScaleBlock;
    static constexpr int kGroups = kRows / 64;                            // of rows, whose scales one transfer brings
    static constexpr int kScaleBytes = kRows * (SC == Scales::kE8M0 ? 4 : 16);      // four blocks of k
    static constexpr int kScaleCopies = kGroups * (SC == Scales::kE8M0 ? 1 : 4);
    static constexpr int kLds = 2 * kStageBytes + 2 * kScaleBytes;
    static constexpr int kHalfMfma = 8 * NB;                              // matrix instructions of half a step
    static constexpr int kReads = 8 + 2 * NB, kCopies = 4 + NB;           // a wave's reads and transfers in half a step
};

template <int NB, Scales SC, bool A_E5M2>
__global__ __launch_bounds__(256, 1) void scaled_gemm_big_kernel(ScaledGemm g, int tiles_m, int tiles_n) {
    using P = Big<NB, SC>;
    constexpr bool kVector = SC != Scales::kE8M0;                         // sums are the vector ALU's
    extern __shared__ __align__(16) uint8_t lds[];
    const GemmTile t = locate<kTM, P::kTN, true>(g, tiles_m, tiles_n);
    if (t.none) return;
    if (t.k == 0) {
        store_nothing(g, t);
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave & 1) * 128, wn = (wave >> 1) * (32 * NB);
    const int steps = (t.k + kScaleBlock - 1) / kScaleBlock;
    const int q = lane >> 4, x16 = lane & 15;
    const uint32_t lds0 = lds_address(lds), sc0 = lds0 + 2 * P::kStageBytes;

    // ---- transfers: eight rows each; of half a step a wave brings four of A and NB of B.  Lane: row lane/8, piece (lane%8) ^ swizzle(row),
    // which differs by four pieces between the even and the odd ones.
    const uint32_t lda = uint32_t(g.a.ld), ldb = uint32_t(g.b.ld), bytes = uint32_t((t.k + 3) & ~3);
    const v4i32 src_a = tile_buffer(t.a, uint32_t(t.rows - 1) * lda + bytes), src_b = tile_buffer(t.b, uint32_t(t.cols - 1) * ldb + bytes);
    const uint32_t piece = uint32_t((lane & 7) ^ (lane >> 4)) * 16;
    const uint32_t off_a[2] = {uint32_t(lane >> 3) * lda + piece, uint32_t(lane >> 3) * lda + (piece ^ 64)};
    const uint32_t off_b[2] = {uint32_t(lane >> 3) * ldb + piece, uint32_t(lane >> 3) * ldb + (piece ^ 64)};
    const uint32_t my_a = uint32_t((wave & 1) * 128 + (wave >> 1) * 32), my_b = uint32_t((wave & 1) * (32 * NB) + (wave >> 1) * (8 * NB));
    // transfer x of half ha of A (x < 4) or hb of B, of step `s`, into stage ST
    auto copy1 = [&](auto ST, int s, int ha, int hb, int x) {
        const uint32_t k = uint32_t(s) * kScaleBlock, to = lds0 + decltype(ST)::v * P::kStageBytes;
        if (x < 4) {
            const uint32_t r = my_a + uint32_t(ha * 64 + x * 8);
            copy16_to_lds(src_a, off_a[x & 1], r * lda + k, to + r * kScaleBlock);
        } else {
            const uint32_t r = my_b + uint32_t(hb * 16 * NB + (x - 4) * 8);
            copy16_to_lds(src_b, off_b[x & 1], r * ldb + k, to + (kTM + r) * kScaleBlock);
        }
    };
    // The scales of the four blocks of k around step s, 64 rows per transfer.  A's (E8M0: B's too) so that a lane reads four fragments'
    // at once: lane 4 x + f brings row 16 f + x; float32 scales of B in the rows' order.
    auto copy_scales = [&](int s) {
        const int four = (t.block0 + s) & ~3;
        const uint32_t to = sc0 + uint32_t((four >> 2) & 1) * P::kScaleBytes;
#pragma unroll
        for (int z = 0; z < (P::kScaleCopies + 3) / 4; ++z) {
            const int y = z * 4 + wave;
            if (y >= P::kScaleCopies) break;
            const int group = y % P::kGroups;
            const bool is_a = group < kTM / 64;
            const int in_group = kVector && !is_a ? lane : (lane & 3) * 16 + (lane >> 2);
            const int tile0 = is_a ? t.row : t.col, shift = is_a ? g.a.shift : g.b.shift, last = (is_a ? t.rows : t.cols) - 1;
            const int r = tile0 + min((is_a ? group : group - kTM / 64) * 64 + in_group, last);
            const int64_t ld = is_a ? g.a.scale_ld : g.b.scale_ld;
            const int blk = kVector ? min(max(four + y / P::kGroups, t.block0), t.block0 + steps - 1) : four;
            const int esize = kVector ? 4 : 1;
            copy4_to_lds((is_a ? t.sa : t.sb) + (int64_t(tile0 >> shift) * ld + blk) * esize, uint32_t((r >> shift) - (tile0 >> shift)) * uint32_t(ld) * uint32_t(esize),
                         to + uint32_t(y) * 256);
        }
    };
    // bytes from `from` on in a half that has landed become zero
    auto clear_tail = [&](int from, int stage, int ha, int hb) {
        for (int x = threadIdx.x; x < P::kRows / 2 * 8; x += 256) {
            const int i = x >> 3, keep = from - (x & 7) * 16;             // row of the half; bytes of this piece that stay
            if (keep >= 16) continue;
            const int ib = i - kTM / 2;
            const int r = ib < 0 ? (i >> 6) * 128 + ha * 64 + (i & 63) : kTM + (ib / (16 * NB)) * (32 * NB) + hb * 16 * NB + ib % (16 * NB);
            uint32_t* w = reinterpret_cast<uint32_t*>(lds + stage * P::kStageBytes + r * kScaleBlock + (((x ^ (r >> 1)) & 7) << 4));
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

    // ---- fragments: 16 rows, a lane has pieces 2q and 2q+1 of row x16
    const uint32_t sw = uint32_t(x16 >> 1) & 7;
    const uint32_t at16[2] = {uint32_t(x16) * kScaleBlock + ((uint32_t(2 * q) ^ sw) * 16), uint32_t(x16) * kScaleBlock + ((uint32_t(2 * q + 1) ^ sw) * 16)};
    typedef __attribute__((address_space(3))) const v4i32* lds16_t;
    uint32_t rd_a[2][2], rd_b[2][2];          // [stage][half of the fragment]
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            rd_a[st][h] = lds0 + uint32_t(st * P::kStageBytes + wm * kScaleBlock) + at16[h];
            rd_b[st][h] = lds0 + uint32_t(st * P::kStageBytes + (kTM + wn) * kScaleBlock) + at16[h];
        }
    union Frag { v8i32 f; v4i32 h[2]; };
    Frag fa[2][4], fb[2][NB];
    // read x of half ha of A (x < 8) or of half hb of B
    auto read_a = [&](auto ST, int ha, int x) {
        fa[ha][x >> 1].h[x & 1] = *reinterpret_cast<lds16_t>(rd_a[decltype(ST)::v][x & 1] + uint32_t(ha * 64 + (x >> 1) * 16) * kScaleBlock);
    };
    auto read_b = [&](auto ST, int hb, int x) {
        fb[hb][x >> 1].h[x & 1] = *reinterpret_cast<lds16_t>(rd_b[decltype(ST)::v][x & 1] + uint32_t(hb * 16 * NB + (x >> 1) * 16) * kScaleBlock);
    };

    // ---- scales of the halves.  E8M0: four blocks' bytes, this step's in the low one.  float32: a row's, per fragment of A; of B
    // one for all (kBlocks: in A's factors and in the matrix instruction), or a lane's four rows' per fragment.
    typedef uint32_t v4u __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) const v4u* lds4_t;
    typedef __attribute__((address_space(3))) const uint32_t* lds1_t;
    typedef __attribute__((address_space(3))) const uint64_t* lds2_t;
    v4u ea[2], eb[2], ea_new, eb_new;                          // E8M0; float32: A's (with kBlocks times B's fraction), bit patterns
    uint32_t eb_all[2] = {127, 127};                           // kBlocks: B's exponent, as a byte
    v4f sb[2][NB], sb_new[NB];                                 // kRows
    uint32_t b_new = 0;                                        // kBlocks
    uint32_t sc_at = 0;                                        // this step's part of LDS
    int sc_shift = 0;
    const uint32_t sc_a = uint32_t(x16 * 16 + wm * 4), sc_b = uint32_t(kTM * 4 + wn * 4 + (kVector ? q * 16 : x16 * 16));
    auto scales_of = [&](int s) {
        const int blk = t.block0 + s;
        sc_at = sc0 + uint32_t((blk >> 2) & 1) * P::kScaleBytes + (kVector ? uint32_t(blk & 3) * (P::kRows * 4) : 0);
        sc_shift = (blk & 3) * 8;
    };
    auto read_scale_a = [&](int ha) { ea_new = *reinterpret_cast<lds4_t>(sc_at + sc_a + uint32_t(ha) * 256); };
    // x-th read of half hb of B's scales: one, or NB of them (kRows)
    constexpr int kScaleReads = SC == Scales::kRows ? NB : 1;
    auto read_scale_b = [&](int hb, int x) {
        if constexpr (SC == Scales::kRows) {
            union { v4u u; v4f f; } v;
            v.u = *reinterpret_cast<lds4_t>(sc_at + sc_b + uint32_t(hb * 16 * NB + x * 16) * 4);
            sb_new[x] = v.f;
        } else if constexpr (SC == Scales::kBlocks) {
            b_new = *reinterpret_cast<lds1_t>(sc_at + uint32_t(kTM * 4));
        } else if constexpr (NB == 4) {
            eb_new = *reinterpret_cast<lds4_t>(sc_at + sc_b + uint32_t(hb) * 256);
        } else {
            const uint64_t two = *reinterpret_cast<lds2_t>(sc_at + sc_b + uint32_t(hb) * 8);
            eb_new[0] = uint32_t(two);
            eb_new[1] = uint32_t(two >> 32);
        }
    };
    // live: not the step of zeros behind the last one, whose scales are zeros too
    auto take_scales = [&](int ha, int hb, bool live) {
        if constexpr (SC == Scales::kE8M0) {
            ea[ha] = ea_new >> sc_shift;
            eb[hb] = eb_new >> sc_shift;
        } else if constexpr (SC == Scales::kBlocks) {
            // The product of the two scales may leave float32's range where the result does not: B's power of two goes into the matrix instruction,
            // its fraction, below 1, to A's scale.
            const float b = __uint_as_float(b_new);
            const int e = min(max(__builtin_amdgcn_frexp_expf(b), -126), 127);
            const float fraction = __builtin_amdgcn_ldexpf(b, -e);
            eb_all[ha] = uint32_t(e + 127);
#pragma unroll
            for (int i = 0; i < 4; ++i) ea[ha][i] = live ? __float_as_uint(__uint_as_float(ea_new[i]) * fraction) : 0;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) ea[ha][i] = live ? ea_new[i] : 0;
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) sb[hb][j][r] = live ? sb_new[j][r] : 0.0f;
        }
    };

    // ---- sums
    v4f acc[2 * NB][8];
    float each[2 * NB][8][4];          // float32 scales: one by one, four registers in a row are hard to come by then
    constexpr int kLag = 3;            // float32 scales: matrix instructions from the one that makes a result to its use
    v4f made[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) made[i] = v4f{0, 0, 0, 0};
    // where matrix instruction y of a quarter lies: fragment j of the half of B, i of A.  NEW_A: A's fragments one after the other
    auto jf = [](bool new_a, int y) constexpr -> int { return new_a ? ((y / NB) & 1 ? NB - 1 - y % NB : y % NB) : y / 4; };
    auto fi = [](bool new_a, int y) constexpr -> int { return new_a ? y / NB : ((y / 4) & 1 ? 3 - y % 4 : y % 4); };
    // applies the scales to results `m` of fragments (hb, j) and (ha, i)
    auto finish = [&](int ha, int i, int hb, int j, const v4f& m) {
        float (&s)[4] = each[hb * NB + j][ha * 4 + i];
        const float f = __uint_as_float(ea[ha][i]);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] = fmaf(SC == Scales::kRows ? m[r] * sb[hb][j][r] : m[r], f, s[r]);
        asm volatile("" : "+v"(s[0]), "+v"(s[1]), "+v"(s[2]), "+v"(s[3]));        // here, not where the block ends
    };
    // Half H of a step that starts with half B0 of B, its 8 NB matrix instructions with read(x), copy(x) and scale(x) between them.
    auto half_step = [&](auto HH, auto BB, auto&& read, auto&& copy, auto&& scale, auto&& middle) {
        constexpr int h = decltype(HH)::v, b0 = decltype(BB)::v, b1 = 1 - b0, M = P::kHalfMfma, kQ = M / 2;
#pragma unroll
        for (int x = 0; x < M; ++x) {
            if (x == kQ) middle();
            const int y = x % kQ;
            const bool first = x < kQ, new_a = h == 1 && first;
            const int ha = h, hb = (h == 0) == first ? b0 : b1, j = jf(new_a, y), i = fi(new_a, y);
            if constexpr (!kVector) {
                v4f& s = acc[hb * NB + j][ha * 4 + i];
                s = mfma_e8m0<A_E5M2>(fb[hb][j].f, fa[ha][i].f, s, eb[hb][j], ea[ha][i]);
                // holds the instruction here and its sums in the accumulation registers: nothing else in this block reads them
                asm volatile("" : "+a"(s));
            } else {
                const int px = x - kLag;
                const int ph = px < 0 ? 1 - h : h, py = (px + M) % M;
                const bool pfirst = py < kQ, pnew = ph == 1 && pfirst;
                // before the first of a step lies the step that started with the other half
                const int pb0 = px < 0 && h == 0 ? b1 : b0, phb = (ph == 0) == pfirst ? pb0 : 1 - pb0;
                finish(ph, fi(pnew, py % kQ), phb, jf(pnew, py % kQ), made[(x - kLag) & 3]);
                if constexpr (SC == Scales::kBlocks) made[x & 3] = mfma_e8m0<A_E5M2>(fb[hb][j].f, fa[ha][i].f, v4f{0, 0, 0, 0}, eb_all[ha], 127);
                else made[x & 3] = mfma_plain<A_E5M2>(fb[hb][j].f, fa[ha][i].f);
                asm volatile("" : "+v"(made[x & 3]));
            }
            __builtin_amdgcn_sched_barrier(0);
            // first half: the other half of B, then A1; second: A0, then, its registers being free, the half of B that is next
#pragma unroll
            for (int r = 0; r < P::kReads; ++r)
                if ((h == 0 ? r * (M - 4) / P::kReads : r < 8 ? r * kQ / 8 : kQ + (r - 8) * (kQ * 3 / 4) / (2 * NB)) == x) read(r);
#pragma unroll
            for (int c = 0; c < P::kCopies; ++c)
                if ((2 * c + 1) * M / (2 * P::kCopies) == x) copy(c);
            if (x >= 1 && x <= 1 + kScaleReads) scale(x - 1);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto meet = [&]() {
        // two halves may still be on their way (scales make it a few transfers less)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(2 * P::kCopies) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // One step; FIRST: its LDS stage, and the half of B that it starts with.
    // bytes of k of step s that there are
    auto valid = [&](int s) { return min(max(t.k - s * kScaleBlock, 0), kScaleBlock); };
    auto step = [&](auto FIRST, int s) {
        constexpr int b0 = decltype(FIRST)::v, b1 = 1 - b0;
        // behind the last step its transfers once more, into a stage that nobody reads: no branches
        const int ahead = min(s + 2, steps - 1);
        meet();
        if (s + 1 >= steps && valid(s) < kScaleBlock) clear_tail(valid(s), b0, 1, b1);
        if (((t.block0 + s + 2) & 3) == 0) copy_scales(ahead);
        half_step(Int<0>{}, Int<b0>{},
                  [&](int r) { if (r < 2 * NB) read_b(Int<b0>{}, b1, r); else read_a(Int<b0>{}, 1, r - 2 * NB); },
                  [&](int c) { copy1(Int<b0>{}, ahead, 0, b0, c); },
                  [&](int x) { if (x == 0) read_scale_a(1); else read_scale_b(b1, x - 1); },
                  [&]() { take_scales(1, b1, s < steps); });
        meet();
        if (s + 2 >= steps && valid(s + 1) < kScaleBlock) clear_tail(valid(s + 1), b1, 0, b1);
        scales_of(s + 1);
        half_step(Int<1>{}, Int<b0>{},
                  [&](int r) { if (r < 8) read_a(Int<b1>{}, 0, r); else read_b(Int<b1>{}, b1, r - 8); },
                  [&](int c) { copy1(Int<b0>{}, ahead, 1, b1, c); },
                  [&](int x) { if (x == 0) read_scale_a(0); else read_scale_b(b1, x - 1); },
                  []() {});
        take_scales(0, b1, s + 1 < steps);
    };
    // the last results of a step that started with half B0
    auto finish_step = [&](auto BB) {
        constexpr int b0 = decltype(BB)::v, kQ = P::kHalfMfma / 2;
        if constexpr (kVector) {
#pragma unroll
            for (int y = kQ - kLag; y < kQ; ++y) finish(1, fi(false, y), b0, jf(false, y), made[(y + kQ) & 3]);
        }
    };

    copy_scales(0);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int x = 0; x < P::kCopies; ++x) copy1(Int<0>{}, 0, half, half, x);
    if (((t.block0 + 1) & 3) == 0) copy_scales(min(1, steps - 1));
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int x = 0; x < P::kCopies; ++x) copy1(Int<1>{}, min(1, steps - 1), half, 1 - half, x);
    // Cleared while the first tiles are on their way; the accumulation registers by matrix instructions with zero operands: what the vector ALU
    // writes the register allocator keeps in ordinary registers, and moves over and back in every step.
    const v8i32 zero = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 2 * NB; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (kVector) {
                each[j][i][0] = each[j][i][1] = each[j][i][2] = each[j][i][3] = 0.0f;
            } else {
                acc[j][i] = mfma_plain<false>(zero, zero);
                asm volatile("" : "+a"(acc[j][i]));
            }
        }
    // what the first step finishes, and before it there is none: nothing times nothing
    ea[1] = v4u{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < NB; ++j) sb[1][j] = v4f{0, 0, 0, 0};
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(3 * P::kCopies) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (valid(0) < kScaleBlock) clear_tail(valid(0), 0, 0, 0);
    scales_of(0);
    read_scale_a(0);
#pragma unroll
    for (int x = 0; x < kScaleReads; ++x) read_scale_b(0, x);
#pragma unroll
    for (int x = 0; x < 8; ++x) read_a(Int<0>{}, 0, x);
#pragma unroll
    for (int x = 0; x < 2 * NB; ++x) read_b(Int<0>{}, 0, x);
    take_scales(0, 0, true);
    if constexpr (kVector) {
        // An odd number of steps is followed by one of zeros: with one way out of the loop the sums stay where they are, with two the register
        // allocator moves all of them in every step.
        for (int s = 0; s < steps; s += 2) {
            step(Int<0>{}, s);
            step(Int<1>{}, s + 1);
        }
        finish_step(Int<1>{});
    } else {
        for (int s = 0;;) {
            step(Int<0>{}, s);
            if (++s == steps) break;
            step(Int<1>{}, s);
            if (++s == steps) break;
        }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();        // the other waves have read the last tiles
    if constexpr (kVector) {
#pragma unroll
        for (int j = 0; j < 2 * NB; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[j][i] = v4f{each[j][i][0], each[j][i][1], each[j][i][2], each[j][i][3]};
    }
    store_results<false, false, 128 * 32 * NB * 2>(g, acc, lds + wave * (128 * 32 * NB * 2), t.c + int64_t(t.row + wm) * g.ldc + t.col + wn, t.rows - wm, t.cols - wn);
}

template <int NB, Scales SC>
void launch(hipStream_t st, const ScaledGemm& g) {
    const int tiles_n = (g.n + Big<NB, SC>::kTN - 1) / Big<NB, SC>::kTN;
    const int64_t tiles_m = g.grouping == Grouping::kRows ? group_pieces(g.m, g.groups, kTM) : (g.m + kTM - 1) / kTM;
    const dim3 grid(unsigned(tiles_m * tiles_n), g.grouping == Grouping::kContraction ? unsigned(g.groups) : 1u);
    constexpr int lds = Big<NB, SC>::kLds;
    if (g.a_e5m2) hipLaunchKernelGGL((scaled_gemm_big_kernel<NB, SC, true>), grid, dim3(256), lds, st, g, int(tiles_m), tiles_n);
    else hipLaunchKernelGGL((scaled_gemm_big_kernel<NB, SC, false>), grid, dim3(256), lds, st, g, int(tiles_m), tiles_n);
}

template <int NB, Scales SC>
bool prepare() {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(scaled_gemm_big_kernel<NB, SC, false>), hipFuncAttributeMaxDynamicSharedMemorySize,
                               Big<NB, SC>::kLds) == hipSuccess &&
           hipFuncSetAttribute(reinterpret_cast<const void*>(scaled_gemm_big_kernel<NB, SC, true>), hipFuncAttributeMaxDynamicSharedMemorySize,
                               Big<NB, SC>::kLds) == hipSuccess;
}

}  // namespace

}  // namespace oz
