// Product of 8-bit block-scaled matrices for few rows of A (a token, a few in flight, the few tokens of an expert): B is read once, and
// that is what bounds it.
//
// A workgroup has 16 rows of B and up to 64 rows of A; its waves share k, four blocks of 128 at a time, and add up their sums through
// LDS in the waves' order.  Operands go from memory into the registers that the matrix instruction reads: a lane's 32 bytes of a row
// are two of its loads, two loads of a wave are the whole cache lines of 16 rows, and a wave has all loads of four blocks (two for 64
// rows of A) on their way at once, 16 KB for 16 rows.
// One token, 4096 x 4096: 5.1 us (3.3 TB/s, of which the launch is 2.4); 24 tokens with four of 32 experts each, 2048 x 2048: 23 us (5.8 TB/s);
// 32 rows 8.5 to 8.8 us.
#include "oz_scaled_gemm_device.h"

namespace oz {

namespace {

// blocks of k that a wave takes at a time: as many as its registers hold
template <int MT>
constexpr int kFew = MT == 4 ? 2 : 4;

template <int MT, bool A_E5M2, bool E8M0, bool WIDE>
__global__ __launch_bounds__(MT == 1 ? 1024 : 512) void scaled_gemm_few_kernel(ScaledGemm g, int strips) {
    extern __shared__ __align__(16) float sums[];                 // [wave][row][16]
    constexpr int kB = kFew<MT>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = int(blockDim.x) >> 6;
    const GemmTile t = locate<MT * 16, 16, false>(g, 0, strips);
    if (t.none) return;
    const int q = lane >> 4, x16 = lane & 15;
    const int blocks = (t.k + kScaleBlock - 1) / kScaleBlock, tail = t.k & (kScaleBlock - 1);
    v4f acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = v4f{0, 0, 0, 0};

    const uint32_t lda = uint32_t(g.a.ld), ldb = uint32_t(g.b.ld), bytes = uint32_t((t.k + 3) & ~3);
    const __amdgpu_buffer_rsrc_t buf_a = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(t.a), 0, int(uint32_t(t.rows - 1) * lda + bytes), 0x00020000);
    const __amdgpu_buffer_rsrc_t buf_b = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(t.b), 0, int(uint32_t(t.cols - 1) * ldb + bytes), 0x00020000);
    const uint32_t lane_a = uint32_t(x16) * lda + uint32_t(q) * 32, lane_b = uint32_t(x16) * ldb + uint32_t(q) * 32;
    // rows of scales: a lane's own row of each fragment
    const uint8_t* row_sb = t.sb + (int64_t((t.col + min(x16, t.cols - 1)) >> g.b.shift) * g.b.scale_ld + t.block0) * (E8M0 ? 1 : 4);
    const uint8_t* row_sa[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) row_sa[i] = t.sa + (int64_t((t.row + min(i * 16 + x16, t.rows - 1)) >> g.a.shift) * g.a.scale_ld + t.block0) * (E8M0 ? 1 : 4);

    for (int b0 = wave * kB; b0 < blocks; b0 += waves * kB) {
        union Frag { v8i32 f; v4i32 h[2]; };
        Frag fb[kB], fa[kB][MT];
        uint32_t eb = 0, ea[MT];
        float sb[kB], sa[kB][MT];
#pragma unroll
        for (int u = 0; u < kB; ++u) {
            // a block behind the end: the last one again, not used
            const uint32_t at = uint32_t(min(b0 + u, blocks - 1)) * kScaleBlock;
#pragma unroll
            for (int h = 0; h < 2; ++h) fb[u].h[h] = __builtin_amdgcn_raw_buffer_load_b128(buf_b, lane_b + h * 16, at, 0);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) fa[u][i].h[h] = __builtin_amdgcn_raw_buffer_load_b128(buf_a, lane_a + h * 16, at + uint32_t(i * 16) * lda, 0);
        }
        if constexpr (E8M0) {
            eb = *reinterpret_cast<const uint32_t*>(row_sb + (b0 & ~3)) >> (8 * (b0 & 3));
#pragma unroll
            for (int i = 0; i < MT; ++i) ea[i] = *reinterpret_cast<const uint32_t*>(row_sa[i] + (b0 & ~3)) >> (8 * (b0 & 3));
        } else {
#pragma unroll
            for (int u = 0; u < kB; ++u) {
                const int blk = min(b0 + u, blocks - 1);
                sb[u] = reinterpret_cast<const float*>(row_sb)[blk];
#pragma unroll
                for (int i = 0; i < MT; ++i) sa[u][i] = reinterpret_cast<const float*>(row_sa[i])[blk];
            }
        }
        bool ordinary = true;                     // E8M0, widened
        if constexpr (E8M0 && WIDE) {
            const uint32_t of_b[1] = {eb};
            ordinary = widens_exactly(ea, of_b, min(blocks - b0, kB));
        }
#pragma unroll
        for (int u = 0; u < kB; ++u) {
            if (b0 + u >= blocks) break;
            if (tail && b0 + u == blocks - 1) {
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    const int have = min(max(tail - (q * 32 + w * 4), 0), 4);
                    const int keep = have == 4 ? -1 : (1 << (8 * have)) - 1;
                    fb[u].f[w] &= keep;
#pragma unroll
                    for (int i = 0; i < MT; ++i) fa[u][i].f[w] &= keep;
                }
            }
            if constexpr (E8M0 && !WIDE) {
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[i] = mfma_e8m0<A_E5M2>(fb[u].f, fa[u][i].f, acc[i], eb >> (8 * u), ea[i] >> (8 * u));
            } else if constexpr (E8M0) {
                if (__builtin_expect(ordinary, 1)) {
                    const Wide wb = widen<false>(fb[u].f, scale_float(eb >> (8 * u)));
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[i] = mfma_wide(wb, widen<A_E5M2>(fa[u][i].f, scale_float(ea[i] >> (8 * u))), acc[i]);
                } else {
                    uint32_t each[4];             // B's scales of this lane's four results
#pragma unroll
                    for (int r = 0; r < 4; ++r) each[r] = uint32_t(__shfl(int(eb >> (8 * u)), q * 4 + r));
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        float one = 1.0f;
                        asm volatile("" : "+v"(one));
                        const v4f p = mfma_wide(widen<false>(fb[u].f, one), widen<A_E5M2>(fa[u][i].f, one), v4f{0, 0, 0, 0});
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[i][r] = add_scaled(acc[i][r], p[r], ea[i] >> (8 * u), each[r]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            } else {
                v4f each;                     // B's scales of this lane's four results
#pragma unroll
                for (int r = 0; r < 4; ++r) each[r] = __shfl(sb[u], q * 4 + r);
                Wide wb;
                if constexpr (WIDE) wb = widen<false>(fb[u].f, 1.0f);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    v4f p;
                    if constexpr (WIDE) p = mfma_wide(wb, widen<A_E5M2>(fa[u][i].f, 1.0f), v4f{0, 0, 0, 0});
                    else p = mfma_plain<A_E5M2>(fb[u].f, fa[u][i].f);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][r] = fmaf(p[r] * each[r], sa[u][i], acc[i][r]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) *reinterpret_cast<v4f*>(sums + ((wave * MT + i) * 16 + x16) * 16 + q * 4) = acc[i];
    __syncthreads();
    for (int x = threadIdx.x; x < MT * 64; x += blockDim.x) {
        const int r = x >> 2, c = (x & 3) * 4;
        v4f s = {0, 0, 0, 0};
        for (int w = 0; w < waves; ++w) s += *reinterpret_cast<const v4f*>(sums + (w * MT * 16 + r) * 16 + c);
        if (r < t.rows && c < t.cols && (t.k > 0 || !g.accumulate)) put4(g, t.c + int64_t(t.row + r) * g.ldc + t.col + c, t.cols - c, s);
    }
}

template <int MT>
void launch_rows(hipStream_t st, const ScaledGemm& g, int waves) {
    const int strips = (g.n + 15) / 16;
    const int64_t tiles_m = g.grouping == Grouping::kRows ? group_pieces(g.m, g.groups, MT * 16) : (g.m + MT * 16 - 1) / (MT * 16);
    waves = MT == 1 || waves < 8 ? waves : 8;
    const dim3 grid(unsigned(tiles_m * strips), unsigned(g.parts)), block(64 * waves);
    const size_t lds = size_t(waves) * MT * 16 * 16 * 4;
    const int kind = (g.a_e5m2 ? 4 : 0) + (g.e8m0 ? 2 : 0) + (g.wide ? 1 : 0);
#define OZ_KIND(K) case K: hipLaunchKernelGGL((scaled_gemm_few_kernel<MT, (K & 4) != 0, (K & 2) != 0, (K & 1) != 0>), grid, block, lds, st, g, strips); break;
    switch (kind) { OZ_KIND(0) OZ_KIND(1) OZ_KIND(2) OZ_KIND(3) OZ_KIND(4) OZ_KIND(5) OZ_KIND(6) OZ_KIND(7) }
#undef OZ_KIND
}

}  // namespace

// rows: of A that share a read of B, at most 64 (more are other workgroups, which read B again)
void launch_scaled_gemm_few(hipStream_t st, const ScaledGemm& g, int rows, int waves) {
    if (rows <= 16) launch_rows<1>(st, g, waves);
    else if (rows <= 32) launch_rows<2>(st, g, waves);
    else launch_rows<4>(st, g, waves);
}

}  // namespace oz
