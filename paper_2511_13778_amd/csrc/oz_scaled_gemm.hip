// Product of 8-bit block-scaled matrices on tiles of C, tiles of the operands through LDS.
//
// A step is a block of 128 of k.  Its rows of A and B (128 bytes each) go from L2 straight into LDS, STAGES - 1 steps ahead;
// one barrier per step.  A row's eight 16-byte pieces are stored at piece ^ (row & 7), which spreads the lanes that read the same piece of
// 16 rows over the banks; 43 to 47 % of LDS' active cycles are counted as conflicts all the same, here and in the other kernels.  The scales come in the same way, four blocks at a time, into two buffers of their own.
//
// 128 x 128 tiles: two workgroups to a CU, each hides the other's first loads and results; a step of one costs 0.54 us a CU (E8M0).
// Counters at 8192 x 8192 x 512: matrix unit busy 23 % of a CU's cycles, LDS active 32 %, waves waiting 40 % of theirs: neither unit is the
// bound by itself, their turns in a step hardly overlap.  64 x 64: four to a CU,
// for outputs that would leave CUs idle.  1024^3 6.4 us, 2048^3 18 us (935 TFLOP/s), 16 groups of about 1024 rows, 4096 x 2048, float32
// scales 206 to 223 us (1.23 to 1.33 PFLOP/s).  float32 results on widened operands: 8192^3 880 to 970 us (1.13 to 1.25 PFLOP/s; the
// library's bfloat16 product of that size 690 to 740), bound by matrix and conversion instructions: matrix unit busy 58 % of the cycles,
// vector instructions issued in 53 %.
#include <type_traits>

#include "oz_scaled_gemm_device.h"
#include "oz_scaled_plan.h"

namespace oz {

namespace {

template <int BM, int BN, int WM, int WN, int STAGES, bool A_E5M2, bool E8M0, bool WIDE>
__global__ __launch_bounds__(64 * (BM / WM) * (BN / WN)) void scaled_gemm_kernel(ScaledGemm g, int tiles_m, int tiles_n) {
    constexpr int WAVES = (BM / WM) * (BN / WN), ROWS = BM + BN;
    constexpr int COPIES = (ROWS / 8 + WAVES - 1) / WAVES;        // 1 KB each, per wave and step
    static_assert(ROWS / 8 % WAVES == 0 && BM % 64 == 0 && BN % 64 == 0, "whole transfers");
    constexpr int STAGE_BYTES = ROWS * kScaleBlock;
    constexpr int SCALE_BYTES = ROWS * (E8M0 ? 4 : 16);           // four blocks of k
    constexpr int SCALE_COPIES = ROWS / 64 * (E8M0 ? 1 : 4);
    constexpr int MT = WM / 16, NT = WN / 16;
    __shared__ __align__(16) uint8_t lds[STAGES * STAGE_BYTES + 2 * SCALE_BYTES];
    constexpr bool kE8M0Wide = E8M0 && WIDE;
    __shared__ int wild_waves[kE8M0Wide ? WAVES : 1];

    const GemmTile t = locate<BM, BN, true>(g, tiles_m, tiles_n);
    if (t.none) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % (BM / WM) * WM, wn = wave / (BM / WM) * WN;
    const int steps = (t.k + kScaleBlock - 1) / kScaleBlock;
    const int tail = t.k & (kScaleBlock - 1);                     // bytes of the last step if it is not whole

    v4f acc[NT][MT];
    auto clear = [&]() {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[j][i] = v4f{0, 0, 0, 0};
    };
    clear();

    if (steps > 0) {
        const uint32_t lds0 = lds_address(lds);
        // transfer x of this wave: rows 8y .. 8y+7 of the stage, y = wave + x * WAVES; lane: row lane/8, piece (lane%8) ^ (row%8)
        const uint32_t piece = uint32_t((lane & 7) ^ (lane >> 3)) * 16, lda = uint32_t(g.a.ld), ldb = uint32_t(g.b.ld);
        const v4i32 src_a = tile_buffer(t.a, uint32_t(t.rows - 1) * lda + uint32_t((t.k + 3) & ~3));
        const v4i32 src_b = tile_buffer(t.b, uint32_t(t.cols - 1) * ldb + uint32_t((t.k + 3) & ~3));
        const uint32_t off_a = uint32_t(lane >> 3) * lda + piece, off_b = uint32_t(lane >> 3) * ldb + piece;
        auto copy_step = [&](int s) {
            const uint32_t to = lds0 + uint32_t(s % STAGES) * STAGE_BYTES;
#pragma unroll
            for (int x = 0; x < COPIES; ++x) {
                const int y = wave + x * WAVES;
                if (y < BM / 8) copy16_to_lds(src_a, off_a, uint32_t(y * 8) * lda + uint32_t(s) * kScaleBlock, to + uint32_t(y) * 1024);
                else copy16_to_lds(src_b, off_b, uint32_t(y * 8 - BM) * ldb + uint32_t(s) * kScaleBlock, to + uint32_t(y) * 1024);
            }
        };
        // the four blocks of k around block0 + s: dword [row] (E8M0: four bytes), or [block][row]
        auto copy_scales = [&](int s) {
            const int four = (t.block0 + s) & ~3;
            const uint32_t to = lds0 + STAGES * STAGE_BYTES + uint32_t((four >> 2) & 1) * SCALE_BYTES;
            for (int y = wave; y < SCALE_COPIES; y += WAVES) {
                const int r0 = (E8M0 ? y : y % (ROWS / 64)) * 64;
                const bool is_a = r0 < BM;
                const int r = is_a ? min(t.row + r0 + lane, t.row + t.rows - 1) >> g.a.shift
                                   : min(t.col + r0 - BM + lane, t.col + t.cols - 1) >> g.b.shift;
                const int first = is_a ? t.row >> g.a.shift : t.col >> g.b.shift;
                const int64_t ld = is_a ? g.a.scale_ld : g.b.scale_ld;
                const int blk = E8M0 ? four : min(max(four + y / (ROWS / 64), t.block0), t.block0 + steps - 1);
                copy4_to_lds((is_a ? t.sa : t.sb) + (int64_t(first) * ld + blk) * (E8M0 ? 1 : 4),
                             uint32_t(r - first) * uint32_t(ld) * (E8M0 ? 1u : 4u), to + uint32_t(y) * 256);
            }
        };
        auto copy = [&](int s) {
            if (s >= steps) return;
            if (s == 0 || ((t.block0 + s) & 3) == 0) copy_scales(s);
            copy_step(s);
        };
        const uint32_t sw = uint32_t(lane & 7);
        const int q = lane >> 4, x16 = lane & 15;
        // this lane's pieces 2q and 2q+1 of row x16 of a fragment
        const uint32_t p0 = uint32_t(x16) * kScaleBlock + ((uint32_t(2 * q) ^ sw) * 16), p1 = uint32_t(x16) * kScaleBlock + ((uint32_t(2 * q + 1) ^ sw) * 16);
        // The walk over k.  Widened operands with E8M0 scales: the first walk folds these into the operands and notes the least and the largest
        // (as float32's exponent field); if a wave met one that does not allow it, the tile is computed once more, APART: scales applied to the
        // sums.  A branch in the step instead costs every call 5 to 13 % (8192^3 886 -> 980 us, so 905).
        uint32_t least = 0x7F800000u, most = 0;
        auto walk = [&](auto APART) {
            constexpr bool apart = decltype(APART)::value;
#pragma unroll
            for (int s = 0; s < STAGES - 1; ++s) copy(s);
            for (int s = 0; s < steps; ++s) {
                if (s + STAGES - 1 <= steps) wait_copies<COPIES * (STAGES - 2)>();
                else wait_copies<0>();
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                copy(s + STAGES - 1);
                const int blk = t.block0 + s;
                const uint8_t* sc = lds + STAGES * STAGE_BYTES + ((blk >> 2) & 1) * SCALE_BYTES;
                const uint8_t* st = lds + (s % STAGES) * STAGE_BYTES;
                auto fragment = [&](int row0) -> v8i32 {
                    union { v8i32 f; v4i32 h[2]; } u;
                    u.h[0] = *reinterpret_cast<const v4i32*>(st + row0 * kScaleBlock + p0);
                    u.h[1] = *reinterpret_cast<const v4i32*>(st + row0 * kScaleBlock + p1);
                    return u.f;
                };
                v8i32 fa[MT], fb[NT];
#pragma unroll
                for (int i = 0; i < MT; ++i) fa[i] = fragment(wm + i * 16);
#pragma unroll
                for (int j = 0; j < NT; ++j) fb[j] = fragment(BM + wn + j * 16);
                if (tail && s == steps - 1) {
#pragma unroll
                    for (int w = 0; w < 8; ++w) {
                        const int have = min(max(tail - (q * 32 + w * 4), 0), 4);
                        const int keep = have == 4 ? -1 : (1 << (8 * have)) - 1;
#pragma unroll
                        for (int i = 0; i < MT; ++i) fa[i][w] &= keep;
#pragma unroll
                        for (int j = 0; j < NT; ++j) fb[j][w] &= keep;
                    }
                }
                if constexpr (E8M0) {
                    uint32_t sa[MT], sb[NT];
                    const int shift = (blk & 3) * 8;
#pragma unroll
                    for (int i = 0; i < MT; ++i) sa[i] = *reinterpret_cast<const uint32_t*>(sc + (wm + i * 16 + x16) * 4) >> shift;
#pragma unroll
                    for (int j = 0; j < NT; ++j) sb[j] = *reinterpret_cast<const uint32_t*>(sc + (BM + wn + j * 16 + x16) * 4) >> shift;
                    if constexpr (apart) {
                        // one product after the other, widened anew for each, in no more registers than the usual step has: they decide how
                        // many workgroups a CU holds
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            const uint4 four = *reinterpret_cast<const uint4*>(sc + (BM + wn + j * 16 + q * 4) * 4);      // of this lane's results
                            const uint32_t each[4] = {four.x >> shift, four.y >> shift, four.z >> shift, four.w >> shift};
#pragma unroll
                            for (int i = 0; i < MT; ++i) {
                                float one = 1.0f;
                                asm volatile("" : "+v"(one));
                                const v4f p = mfma_wide(widen<false>(fb[j], one), widen<A_E5M2>(fa[i], one), v4f{0, 0, 0, 0});
#pragma unroll
                                for (int r = 0; r < 4; ++r) acc[j][i][r] = add_scaled(acc[j][i][r], p[r], sa[i], each[r]);
                                __builtin_amdgcn_sched_barrier(0);
                            }
                        }
                    } else if constexpr (WIDE) {
                        Wide wa[MT], wb[NT];
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            const float scale = scale_float(sa[i]);
                            least = min(least, __float_as_uint(scale));
                            most = max(most, __float_as_uint(scale));
                            wa[i] = widen<A_E5M2>(fa[i], scale);
                        }
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            const float scale = scale_float(sb[j]);
                            least = min(least, __float_as_uint(scale));
                            most = max(most, __float_as_uint(scale));
                            wb[j] = widen<false>(fb[j], scale);
                        }
                        // a tile's four instructions apart from each other: each waits for the one before it
#pragma unroll
                        for (int w = 0; w < 4; ++w)
#pragma unroll
                            for (int j = 0; j < NT; ++j)
#pragma unroll
                                for (int i = 0; i < MT; ++i)
                                    acc[j][i] = mfma_bf16(wb[j].part[w], wa[i].part[w], acc[j][i]);
                    } else {
#pragma unroll
                        for (int j = 0; j < NT; ++j)
#pragma unroll
                            for (int i = 0; i < MT; ++i) acc[j][i] = mfma_e8m0<A_E5M2>(fb[j], fa[i], acc[j][i], sb[j], sa[i]);
                    }
                } else {
                    const float* fs = reinterpret_cast<const float*>(sc) + (blk & 3) * ROWS;
                    float sa[MT];
                    v4f sb[NT];
#pragma unroll
                    for (int i = 0; i < MT; ++i) sa[i] = fs[wm + i * 16 + x16];
#pragma unroll
                    for (int j = 0; j < NT; ++j) sb[j] = *reinterpret_cast<const v4f*>(fs + BM + wn + j * 16 + q * 4);
                    Wide wa[MT], wb[NT];
                    if constexpr (WIDE) {
#pragma unroll
                        for (int i = 0; i < MT; ++i) wa[i] = widen<A_E5M2>(fa[i], 1.0f);
#pragma unroll
                        for (int j = 0; j < NT; ++j) wb[j] = widen<false>(fb[j], 1.0f);
                    }
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        v4f p[MT];
                        if constexpr (WIDE) {
#pragma unroll
                            for (int w = 0; w < 4; ++w)
#pragma unroll
                                for (int i = 0; i < MT; ++i)
                                    p[i] = mfma_bf16(wb[j].part[w], wa[i].part[w], w == 0 ? v4f{0, 0, 0, 0} : p[i]);
                        } else {
#pragma unroll
                            for (int i = 0; i < MT; ++i) p[i] = mfma_plain<A_E5M2>(fb[j], fa[i]);
                        }
#pragma unroll
                        for (int i = 0; i < MT; ++i)
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc[j][i][r] = fmaf(p[i][r] * sb[j][r], sa[i], acc[j][i][r]);
                    }
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
        };
        walk(std::false_type{});
        if constexpr (kE8M0Wide) {
            const bool wild = __ballot(least < kWidenLeast << 23 || most > kWidenMost << 23) != 0;
            if (lane == 0) wild_waves[wave] = wild;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            int any = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) any |= wild_waves[w];
            if (__builtin_amdgcn_readfirstlane(any)) {                  // all of the workgroup: they bring the tiles together
                clear();
                walk(std::true_type{});
            }
        }
    }

    if (steps == 0 && g.accumulate) return;
    __builtin_amdgcn_s_barrier();        // the other waves have read the last tiles
    constexpr int kWaveBytes = int(sizeof(lds)) / WAVES / 1024 * 1024;
    store_results<WIDE, BM == 64, kWaveBytes>(g, acc, lds + wave * kWaveBytes, t.c + int64_t(t.row + wm) * g.ldc + t.col + wn, t.rows - wm,
                                              t.cols - wn);
}

// C = the parts' planes, in their order (+ C).  Four results a thread.
__global__ __launch_bounds__(256) void add_planes_kernel(ScaledGemm g, const float* __restrict__ planes, int parts, int quads) {
    const uint32_t x = blockIdx.x * 256 + threadIdx.x;
    const int r = int(x / uint32_t(quads)), c = int(x % uint32_t(quads)) * 4;
    if (r >= g.m) return;
    const int have = min(4, g.n - c);
    const int64_t at = int64_t(r) * g.n + c, plane = int64_t(g.m) * g.n;
    v4f s = {0, 0, 0, 0};
    typedef v4f __attribute__((aligned(4), may_alias)) v4f_any;
    if (have == 4) {
#pragma unroll 8
        for (int p = 0; p < parts; ++p) s += *reinterpret_cast<const v4f_any*>(planes + p * plane + at);
    } else {
        for (int p = 0; p < parts; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < have) s[i] += planes[p * plane + at + i];
    }
    put4(g, int64_t(r) * g.ldc + c, have, s);
}

template <int BM, int BN, int WM, int WN, int STAGES>
void launch_tiles(hipStream_t st, const ScaledGemm& g) {
    const int tiles_n = (g.n + BN - 1) / BN;
    const int64_t tiles_m = g.grouping == Grouping::kRows ? group_pieces(g.m, g.groups, BM) : (g.m + BM - 1) / BM;
    const dim3 grid(unsigned(tiles_m * tiles_n), g.grouping == Grouping::kContraction ? unsigned(g.groups) : unsigned(g.parts));
    const dim3 block(64 * (BM / WM) * (BN / WN));
    const int kind = (g.a_e5m2 ? 4 : 0) + (g.e8m0 ? 2 : 0) + (g.wide ? 1 : 0);
#define OZ_KIND(K) case K: hipLaunchKernelGGL((scaled_gemm_kernel<BM, BN, WM, WN, STAGES, (K & 4) != 0, (K & 2) != 0, (K & 1) != 0>), grid, block, 0, st, g, int(tiles_m), tiles_n); break;
    switch (kind) { OZ_KIND(0) OZ_KIND(1) OZ_KIND(2) OZ_KIND(3) OZ_KIND(4) OZ_KIND(5) OZ_KIND(6) OZ_KIND(7) }
#undef OZ_KIND
}


}  // namespace

size_t scaled_gemm_part_bytes(int64_t m, int64_t n, int64_t k, int num_cu) {
    if (m == 0 || n == 0 || k == 0) return 0;
    const ScaledPlan p = cut_plan(m, n, k, num_cu);
    return p.parts > 1 ? size_t(p.parts) * size_t(m) * size_t(n) * 4 : 0;
}

void launch_scaled_gemm(hipStream_t st, const ScaledGemm& call, int num_cu, float* planes) {
    ScaledGemm g = call;
    const bool by_rows = g.grouping == Grouping::kRows, by_k = g.grouping == Grouping::kContraction;
    const ScaledPlan p = scaled_plan((g.wide ? 2 : 0) + (g.e8m0 ? 0 : 1), g.m, g.n, g.k, g.groups, by_rows, by_k, num_cu);
    if (p.parts > 1) {
        g.parts = p.parts;
        g.c = planes;
        g.ldc = g.n;
        g.c_type = OZ_F32;
        g.accumulate = 0;
    }
    switch (p.route) {
        case ScaledRoute::kFew: launch_scaled_gemm_few(st, g, by_rows ? int(div_up(g.m, g.groups)) : g.m, p.waves); break;
        case ScaledRoute::kTiles64:
            // parts of a cut k are few to a CU: four stages, from memory (128 x 4096 x 4096 17.1 -> 16.0 us), but not for widened operands (17.6 -> 18.1)
            if (p.parts > 1 && !g.wide) launch_tiles<64, 64, 32, 32, 4>(st, g);
            else launch_tiles<64, 64, 32, 32, 2>(st, g);
            break;
        case ScaledRoute::kTiles64Deep: launch_tiles<64, 64, 32, 32, 4>(st, g); break;
        case ScaledRoute::kTiles128: launch_tiles<128, 128, 64, 64, 2>(st, g); break;
        case ScaledRoute::kTall: launch_scaled_gemm_big(st, g, false); break;
        case ScaledRoute::kBig: launch_scaled_gemm_big(st, g, true); break;
    }
    if (p.parts > 1) {
        const int quads = int(div_up(g.n, 4));
        hipLaunchKernelGGL(add_planes_kernel, dim3(unsigned(div_up(int64_t(g.m) * quads, 256))), dim3(256), 0, st, call, planes, p.parts, quads);
    }
}

}  // namespace oz
