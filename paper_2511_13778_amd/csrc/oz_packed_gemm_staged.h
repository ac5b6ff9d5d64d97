// Product with weights in 4 bits for more than a few rows of x.
//
// A matrix instruction's lanes want 16 bytes of x from 16 different rows; loaded that way, straight into registers, a load's lanes share no line, the first
// cache takes 14 bytes an access, and x bounds the product (64 x 8192 x 8192, bfloat16: 41 us, 6 of them for W).  Here four to eight lanes load a row's
// consecutive bytes, a stage of 32 columns at a time and two to four stages ahead, and lay them into LDS, as each wave's own pair of stages, from which
// the lanes take their 16 bytes: 27 us, 33 x 1300 x 777 5.0 for 6.8, 64 x 4095 x 4001 with its rows at odd addresses 15 for 45.  What bounds it then is the
// latency of those loads and LDS, close to the vector instructions that widen the codes and, of float32, cut x into parts.  (Transfers straight
// into LDS are as fast and need rows at multiples of 16 bytes.)
#pragma once

namespace oz {

namespace {

template <typename X, int MT, int R, int PER, bool ZEROS>
struct Staged {
    static constexpr int kRow = 32 * int(sizeof(X)), kStage = MT * 16 * kRow, kCopies = kStage / 1024;        // bytes of a row and of a stage; 16 of each lane
    static constexpr int kDeep = kCopies > 2 ? 2 : 4;                                // stages on their way
    static constexpr int kCodes = R * 1024;                                          // a block's
    static constexpr int kAhead = 8 / PER, kScales = 8 * 16 * R, kLoads = kScales / 64;   // blocks whose scales are loaded together; of them
    static constexpr int kWaveBytes = std::max(2 * kStage + kCodes + kScales * 4 * (ZEROS ? 2 : 1), MT * 16 * 16 * R * 4);
};

// A row's 16-byte pieces change places in LDS by the row, so that 16 rows' same piece lies in different banks.
template <int ROW>
__device__ __forceinline__ int place_of(int row, int piece) { return ROW == 64 ? piece ^ ((row >> 2) & 3) : piece ^ ((row >> 1) & 7); }

// As packed_gemm_kernel, with 16 MT rows of x.
template <typename X, int MT, int R, int PER, bool ZEROS, bool EXACT>
__global__ __launch_bounds__(512) void packed_gemm_staged_kernel(PackedGemm g, int strips) {
    using E = Eight<X>;
    using W = typename E::W;
    using S = Staged<X, MT, R, PER, ZEROS>;
    constexpr int kEach = 4 / PER, kSize = sizeof(X);
    constexpr bool kSums = ZEROS || !EXACT;                           // sums of x are needed
    extern __shared__ __align__(16) float lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = int(blockDim.x) >> 6;
    const int q = lane >> 4, x16 = lane & 15;
    const int strip = int(blockIdx.x % unsigned(strips)), piece = int(blockIdx.x / unsigned(strips)), col0 = strip * 16 * R, cols = min(g.n - col0, 16 * R);
    int row0 = piece * MT * 16, rows = min(g.m - row0, MT * 16), of = 0;
    if (g.offsets) {
        GroupPieces<MT * 16> pieces(g.offsets, g.groups, g.m);
        const GroupPiece p = pieces.template find<false>(piece);
        if (p.group < 0) return;
        of = p.group;
        row0 = p.row;
        rows = min(p.end - p.row, MT * 16);
    }
    const bool none = g.offsets && of >= g.groups;                    // rows behind the last group: zeros
    uint8_t* const mine = reinterpret_cast<uint8_t*>(lds) + wave * S::kWaveBytes;
    float* const scale_at = reinterpret_cast<float*>(mine + 2 * S::kStage + S::kCodes);
    v4f acc[MT][R];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int s = 0; s < R; ++s) acc[i][s] = v4f{0, 0, 0, 0};
    const int blocks = (g.k + kBlock - 1) / kBlock, per = (blocks + waves - 1) / waves, begin = wave * per, end = min(begin + per, blocks);
    if (!none && begin < end) {
        const int bytes = (g.k + 31) / 32 * 16;
        // lane's place in a stage -> row and piece
        constexpr int kPieces = S::kRow / 16, kRows = 64 / kPieces, kOf = 16 / kSize;
        const X* x_row[S::kCopies];
        int x_col[kSize == 4 ? 2 : 1];
#pragma unroll
        for (int d = 0; d < S::kCopies; ++d) {
            const int row = d * kRows + lane / kPieces;
            x_row[d] = static_cast<const X*>(g.x) + int64_t(row0 + min(row, rows - 1)) * g.ldx;
            if (d < (kSize == 4 ? 2 : 1)) x_col[d] = place_of<S::kRow>(row, lane % kPieces) * kOf;
        }
        const uint8_t* w_row[R];
        const int w_col = place_of<64>(lane / 4, lane % 4) * 16;
#pragma unroll
        for (int s = 0; s < R; ++s) w_row[s] = g.w.data + of * g.w.stride + int64_t(col0 + min(s * 16 + lane / 4, cols - 1)) * g.w.ld;
        // without a branch, which would wait: columns behind the last are those before it, and are moved into place or out of it when they are there
        struct Piece { uint32_t e[4]; };
        Piece way[S::kDeep][S::kCopies];
        v4u32 codes[R];
        const int last = g.k - kOf, end_stage = end * 4;
        auto fetch = [&](int stage, Piece (&to)[S::kCopies]) {
            const int col = min(stage, end_stage - 1) * 32;
#pragma unroll
            for (int d = 0; d < S::kCopies; ++d) __builtin_memcpy(to[d].e, x_row[d] + min(col + x_col[kSize == 4 ? d & 1 : 0], last), 16);
        };
        auto fetch_codes = [&](int b) {
#pragma unroll
            for (int s = 0; s < R; ++s) codes[s] = *reinterpret_cast<const v4u32*>(w_row[s] + min(min(b, end - 1) * 64 + w_col, bytes - 16));
        };
        auto lay = [&](int stage, Piece (&of_stage)[S::kCopies]) {
            const int col = stage * 32;
            if (col + 32 > g.k) {
#pragma unroll
                for (int d = 0; d < S::kCopies; ++d) {
                    const int down = min(max(col + x_col[kSize == 4 ? d & 1 : 0] - last, 0), kOf);
#pragma unroll
                    for (int by = 2; by > 0; by /= 2)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t now = of_stage[d].e[i], far = i + by < 4 ? of_stage[d].e[i + by] : 0u;
                            of_stage[d].e[i] = down * kSize / 4 & by ? far : now;
                        }
                    if constexpr (kSize == 2) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t now = of_stage[d].e[i], odd = now >> 16 | (i < 3 ? of_stage[d].e[i + 1] << 16 : 0u);
                            of_stage[d].e[i] = down & 1 ? odd : now;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) of_stage[d].e[i] = down >= kOf ? 0u : of_stage[d].e[i];
                }
            }
#pragma unroll
            for (int d = 0; d < S::kCopies; ++d)
                *reinterpret_cast<v4u32*>(mine + (stage & 1) * S::kStage + d * 1024 + lane * 16) =
                    v4u32{of_stage[d].e[0], of_stage[d].e[1], of_stage[d].e[2], of_stage[d].e[3]};
        };
        fetch_codes(begin);
#pragma unroll
        for (int y = 0; y < S::kDeep; ++y) fetch(begin * 4 + y, way[y]);
        lay(begin * 4, way[0]);
        fetch(begin * 4 + S::kDeep, way[0]);
        const ScaleLoad scales(g.w.scale, g.w.type), zeros(g.w.zero, g.w.type);
        uint32_t ones[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) ones[i] = uint32_t(__builtin_bit_cast(uint16_t, static_cast<W>(1.0f))) * 0x10001u;
        for (int b = begin; b < end; ++b) {
            // lanes read what others of their wave wrote: LDS is in order, and what the compiler moves is held here and at each stage
            __builtin_amdgcn_wave_barrier();
            const int in = (b - begin) % S::kAhead;
            if (in == 0) {
                // the next blocks' scales, [block, group][row]
                typename ScaleLoad::Halves scale_bits[S::kLoads], zero_bits[ZEROS ? S::kLoads : 1];
#pragma unroll
                for (int y = 0; y < S::kLoads; ++y) {
                    const int z = y * 64 + lane, row = z % (16 * R), p = z / (16 * R);
                    const int64_t group = min(((b * PER + p) * (kBlock / PER)) >> g.w.shift, (g.k - 1) >> g.w.shift);
                    const int64_t at = of * g.w.scale_stride + group * g.w.scale_ld + col0 + min(row, cols - 1);
                    scale_bits[y] = scales.fetch(at);
                    if constexpr (ZEROS) zero_bits[y] = zeros.fetch(at);
                }
#pragma unroll
                for (int y = 0; y < S::kLoads; ++y) {
                    scale_at[y * 64 + lane] = scales.value(scale_bits[y]);
                    if constexpr (ZEROS) scale_at[S::kScales + y * 64 + lane] = (EXACT ? 8.0f : -128.0f) - zeros.value(zero_bits[y]);
                }
                __builtin_amdgcn_s_waitcnt(0x0F70);                   // vmcnt(0), which the compiler takes note of: it waits for these loads at every block else
                __builtin_amdgcn_wave_barrier();
            }
#pragma unroll
            for (int s = 0; s < R; ++s) *reinterpret_cast<v4u32*>(mine + 2 * S::kStage + s * 1024 + lane * 16) = codes[s];
            fetch_codes(b + 1);
            v4f sum[MT][R], here[MT];
            auto of_stage = [&](auto V) {
                constexpr int v = decltype(V)::value;
                __builtin_amdgcn_wave_barrier();
                E x[MT];
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const uint8_t* row = mine + (v & 1) * S::kStage + (i * 16 + x16) * S::kRow;
#pragma unroll
                    for (int z = 0; z < kSize / 2; ++z) {
                        const v4u32 e = *reinterpret_cast<const v4u32*>(row + place_of<S::kRow>(x16, q * (kSize / 2) + z) * 16);
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[i].e[z * 4 + r] = e[r];
                    }
                }
                uint32_t word[R];
#pragma unroll
                for (int s = 0; s < R; ++s)
                    word[s] = *reinterpret_cast<const uint32_t*>(mine + 2 * S::kStage + s * 1024 + x16 * 64 + place_of<64>(x16, v) * 16 + q * 4);
                const int next = b * 4 + v + 1;
                lay(next, way[(v + 1) % S::kDeep]);
                fetch(next + S::kDeep, way[(v + 1) % S::kDeep]);
                if constexpr (v % kEach == 0) {
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        here[i] = v4f{0, 0, 0, 0};
#pragma unroll
                        for (int s = 0; s < R; ++s) sum[i][s] = v4f{0, 0, 0, 0};
                    }
                }
                uint32_t w[R][4];
#pragma unroll
                for (int s = 0; s < R; ++s) widen_codes<W, EXACT>(word[s], w[s]);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if (i > 0 && i * 16 >= rows) break;
                    uint32_t part[E::kParts][4];
                    x[i].parts(part);
#pragma unroll
                    for (int y = E::kParts - 1; y >= 0; --y) {
#pragma unroll
                        for (int s = 0; s < R; ++s) sum[i][s] = mfma16(w[s], part[y], sum[i][s], W{});
                        if constexpr (kSums) here[i] = mfma16(ones, part[y], here[i], W{});
                    }
                }
                if constexpr (v % kEach == kEach - 1) {
#pragma unroll
                    for (int s = 0; s < R; ++s) {
                        const float* of_group = scale_at + (in * PER + v / kEach) * (16 * R) + s * 16 + q * 4;
                        const v4f scale = *reinterpret_cast<const v4f*>(of_group);
                        v4f less = {-136.0f, -136.0f, -136.0f, -136.0f};
                        if constexpr (ZEROS) less = *reinterpret_cast<const v4f*>(of_group + S::kScales);
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            if (i > 0 && i * 16 >= rows) break;
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                float e = sum[i][s][r];
                                if constexpr (kSums) e = fmaf(less[r], here[i][r], e);
                                acc[i][s][r] = fmaf(scale[r], e, acc[i][s][r]);
                            }
                        }
                    }
                }
            };
            of_stage(std::integral_constant<int, 0>{});
            of_stage(std::integral_constant<int, 1>{});
            of_stage(std::integral_constant<int, 2>{});
            of_stage(std::integral_constant<int, 3>{});
        }
    }
    // the wave's sums take the place of all that
    float* const sums = reinterpret_cast<float*>(mine);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int s = 0; s < R; ++s) *reinterpret_cast<v4f*>(sums + (i * 16 + x16) * (16 * R) + s * 16 + q * 4) = acc[i][s];
    __syncthreads();
    for (int x = threadIdx.x; x < MT * 64 * R; x += blockDim.x) {
        const int r = x / (4 * R), c = (x % (4 * R)) * 4;
        const bool in = r < rows && c < cols;
        v4f s = {0, 0, 0, 0};
        for (int w = 0; w < waves; ++w) s += *reinterpret_cast<const v4f*>(lds + w * (S::kWaveBytes / 4) + r * (16 * R) + c);
        mend_results<X>(g, of, in, row0 + r, col0 + c, s);
        if (in) store_results(g, int64_t(row0 + r) * g.ldy + col0 + c, cols - c, s);
    }
}

}  // namespace

}  // namespace oz
