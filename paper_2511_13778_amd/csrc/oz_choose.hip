// The router's choice: a token's scores s over the experts -> its topk experts and their weights, with the balance loss and the gradient of both.
//
//   p = softmax(s), chosen by falling score (ties: the lowest expert), w_j = p_j / sum of the chosen ones' (or p_j)
//   f_e = choices of e / all choices, P_e = mean over the tokens of p_e, loss = experts * sum_e f_e P_e
//   ds_i = w_i (dw_i - sum_j w_j dw_j) for the chosen (or p_i (dw_i - sum_j w_j dw_j), dw = 0 for the others) + dloss experts / tokens * p_i (f_i - sum_e f_e p_e)
//
// A token is a group of 16 lanes (64 beyond 256 experts), each with consecutive experts in registers: four tokens to a wave, so that maxima and sums over
// the experts are four rotations of 16 lanes.  65000 tokens of 256 bfloat16 scores, 8 chosen: 23 us forward, 6 for the batch's sums, 19 for the gradient, where a
// copy of as many bytes takes 16 in all; 16384 tokens of 64 float32 scores: 6, 6 and 5; 24 tokens: a launch.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "oz_layer.h"
#include "oz_scaled_device.h"

namespace oz {

namespace {

constexpr int kThreads = 512, kSumThreads = 1024;

template <int L, typename F>
__device__ __forceinline__ uint32_t fold(uint32_t x, F&& f) {
    x = f(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x128, 0xF, 0xF, false)));
    x = f(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x124, 0xF, 0xF, false)));
    x = f(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x122, 0xF, 0xF, false)));
    x = f(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x121, 0xF, 0xF, false)));
    if constexpr (L == 64) {
        x = f(x, uint32_t(__shfl_xor(int(x), 16)));
        x = f(x, uint32_t(__shfl_xor(int(x), 32)));
    }
    return x;
}
// over a group's lanes; every lane gets the same bits
template <int L>
__device__ __forceinline__ float group_sum(float x) {
    return __uint_as_float(fold<L>(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
template <int L>
__device__ __forceinline__ int group_count(int x) {
    return int(fold<L>(uint32_t(x), [](uint32_t a, uint32_t b) { return a + b; }));
}
template <int L>
__device__ __forceinline__ float group_largest(float x) {
    return __uint_as_float(fold<L>(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
template <int L>
__device__ __forceinline__ int32_t fold_max(int32_t x) {
    return int32_t(fold<L>(uint32_t(x), [](uint32_t a, uint32_t b) { return uint32_t(max(int32_t(a), int32_t(b))); }));
}
template <int L>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
    return fold<L>(x, [](uint32_t a, uint32_t b) { return max(a, b); });
}
// whether it holds for any of the group's lanes
template <int L>
__device__ __forceinline__ bool in_group(bool x) {
    uint64_t has = __ballot(x) >> (int(threadIdx.x & 63) / L * L);
    if (L < 64) has &= (uint64_t(1) << (L & 63)) - 1;
    return has != 0;
}

// Scores as whole numbers that rise with them, the expert in the low bits (lower ones above higher ones), so that no two are equal.  16-bit scores
// leave room for the expert in the same word; float32 takes two.  -0 counts as +0, a NaN is above all; what is not above `kNone` is an expert that
// is not to be had (score -infinity, or no such expert).
template <typename T>
struct Key {
    static constexpr bool kNamed = sizeof(T) == 2;
    using Head = std::conditional_t<kNamed, int32_t, uint32_t>;          // what is compared first
    using type = std::conditional_t<kNamed, int32_t, uint64_t>;
    static constexpr uint32_t kInf = kNamed ? (std::is_same_v<T, f16_t> ? 0x7C00u : 0x7F80u) : 0x7F800000u;
    static constexpr Head kNone = kNamed ? Head(0xFFFFu - (kInf << 16)) : Head(0x007FFFFFu);
    static __device__ __forceinline__ Head head(type key) { return kNamed ? Head(key) : Head(uint64_t(key) >> 32); }
    static __device__ __forceinline__ int expert(type key) { return kNamed ? 0xFFFF - int(uint32_t(key) & 0xFFFFu) : int(~uint32_t(key)); }
    static __device__ __forceinline__ float score(Head h) {
        if constexpr (kNamed) {
            const int up = h >> 16;
            return to_float(__builtin_bit_cast(T, uint16_t(up < 0 ? 0x8000 - up : up)));
        } else {
            return __uint_as_float((h & 0x80000000u) ? h ^ 0x80000000u : ~h);
        }
    }
};

// A lane's part of a token's scores: V consecutive elements, -infinity behind the last expert.  They are sent for before they are used, without a
// branch, which would wait for what is on its way: behind the last token its own scores again, behind the last expert the last V, moved into place
// by `settle`.  There are at least V experts and one token.
template <int V, typename T>
struct Scores {
    using K = Key<T>;
    static constexpr int kWords = V * int(sizeof(T)) / 4;
    union { T e[V]; uint32_t w[kWords + (V == 1)]; };
    uint8_t alive;
    __device__ __forceinline__ Scores() {}
    __device__ __forceinline__ void fetch(const T* scores, int64_t ld, int experts, const uint8_t* live, int64_t t, int64_t tokens, int first) {
        t = min(t, tokens - 1);
        const T* p = scores + t * ld + min(first, experts - V);
        __builtin_memcpy(e, p, sizeof(e));
        alive = *(live ? live + t : reinterpret_cast<const uint8_t*>(p));
    }
    __device__ __forceinline__ void settle(int experts, int all, int first) {
        if (experts == all) return;
        const int d = min(first - min(first, experts - V), V);
        constexpr uint32_t kLow = sizeof(T) == 4 ? 0xFF800000u : uint32_t(uint16_t(0x8000u | K::kInf)) * 0x10001u;
        if constexpr (V == 1) {
            if (d) e[0] = T(-INFINITY);
        } else {
            if constexpr (sizeof(T) == 2) {
                if (experts & 1) {
#pragma unroll
                    for (int i = 0; i < kWords; ++i) w[i] = d & 1 ? w[i] >> 16 | (i + 1 < kWords ? w[i + 1] : kLow) << 16 : w[i];
                }
            }
#pragma unroll
            for (int by = 1; by <= kWords; by *= 2) {
                const bool move = d & (by * 4 / int(sizeof(T)));
#pragma unroll
                for (int i = 0; i < kWords; ++i) w[i] = move ? i + by < kWords ? w[i + by] : kLow : w[i];
            }
        }
    }
    __device__ __forceinline__ void keys(int first, typename K::type (&key)[V]) {
        if constexpr (K::kNamed && V >= 2) {
            typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
            typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
            u16x2 top = {0, 0};
#pragma unroll
            for (int i = 0; i < V / 2; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu));
            if (__any(max(top[0], top[1]) > K::kInf)) {
                // whatever a NaN's sign and other bits are
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if ((__builtin_bit_cast(uint16_t, e[v]) & 0x7FFFu) > K::kInf) e[v] = __builtin_bit_cast(T, uint16_t(0x7FFF));
            }
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                // magnitude and sign to two's complement, two at a time
                const i16x2 sign = __builtin_bit_cast(i16x2, w[i]) >> i16x2{15, 15}, size = __builtin_bit_cast(i16x2, w[i] & 0x7FFF7FFFu);
                const uint32_t up = __builtin_bit_cast(uint32_t, i16x2((size ^ sign) - sign));
                key[2 * i] = int32_t(up << 16 | uint32_t(0xFFFF - (first + 2 * i)));
                key[2 * i + 1] = int32_t((up & 0xFFFF0000u) | uint32_t(0xFFFF - (first + 2 * i + 1)));
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float f = to_float(e[v]);
                if constexpr (K::kNamed) {
                    const uint32_t u = f != f ? 0x7FFFu : uint32_t(__builtin_bit_cast(uint16_t, e[v]));
                    const int size = int(u & 0x7FFFu), up = (u & 0x8000u) ? -size : size;
                    key[v] = int32_t(uint32_t(up) << 16 | uint32_t(0xFFFF - (first + v)));
                } else {
                    const uint32_t u = f != f ? 0x7FFFFFFFu : __float_as_uint(f + 0.0f);
                    key[v] = uint64_t(u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u)) << 32 | uint32_t(~(first + v));
                }
            }
        }
    }
};

// exp(s - m) to a step of the result and 2^-23 |s - m|; zero below 2^-126.  (As 2^(s log2 e - m log2 e) it would be an instruction less, and infinite where
// m log2 e is: bfloat16 and float32 have such m.)
__device__ __forceinline__ float exp_of(float s, float m) { return __builtin_amdgcn_exp2f((s - m) * 1.44269504f); }

// those of a lane's experts, and their sum over the group
template <int L, int V, typename T>
__device__ __forceinline__ float exponentials(const T (&e)[V], float m, float (&ex)[V]) {
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        ex[v] = exp_of(to_float(e[v]), m);
        sum += ex[v];
    }
    return group_sum<L>(sum);
}

// Falling order, by odd-even merges: 5 exchanges for four, 19 for eight, 63 for sixteen.
template <int V>
struct Merges {
    int count = 0, a[64] = {}, b[64] = {};
    constexpr Merges() {
        for (int p = 1; p < V; p *= 2)
            for (int d = p; d >= 1; d /= 2)
                for (int j = d % p; j <= V - 1 - d; j += 2 * d)
                    for (int i = 0; i < d; ++i)
                        if (i + j + d < V && (i + j) / (2 * p) == (i + j + d) / (2 * p)) {
                            a[count] = i + j;
                            b[count] = i + j + d;
                            ++count;
                        }
    }
};
template <int V, typename K, int... I>
__device__ __forceinline__ void exchange(K (&k)[V], std::integer_sequence<int, I...>) {
    constexpr Merges<V> net;
    auto one = [&](auto at) {
        constexpr int a = net.a[decltype(at)::value], b = net.b[decltype(at)::value];
        const K x = k[a], y = k[b];
        const bool less = x < y;
        k[a] = less ? y : x;
        k[b] = less ? x : y;
    };
    (one(std::integral_constant<int, I>{}), ...);
}
template <int V, typename K>
__device__ __forceinline__ void sort_falling(K (&k)[V]) {
    exchange(k, std::make_integer_sequence<int, Merges<V>().count>{});
}

// The largest KEEP of V in falling order, the first of `k`; KEEP is V or its half: halves sorted, the larger of the first and the last, the second and
// the last but one, ..., which rise and fall once, sorted.
template <int KEEP, int V, typename K>
__device__ __forceinline__ void sort_first(K (&k)[V]) {
    if constexpr (KEEP == V) {
        sort_falling(k);
    } else {
        static_assert(2 * KEEP == V, "half of them");
        K a[KEEP], b[KEEP];
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            a[i] = k[i];
            b[i] = k[KEEP + i];
        }
        sort_falling(a);
        sort_falling(b);
#pragma unroll
        for (int i = 0; i < KEEP; ++i) a[i] = a[i] < b[KEEP - 1 - i] ? b[KEEP - 1 - i] : a[i];
        auto halve = [&](auto D) {
            constexpr int d = decltype(D)::value;
#pragma unroll
            for (int i = 0; i < KEEP; ++i)
                if ((i & d) == 0 && i + d < KEEP) {
                    const K x = a[i], y = a[i + d];
                    const bool less = x < y;
                    a[i] = less ? y : x;
                    a[i + d] = less ? x : y;
                }
        };
        static_assert(KEEP == 8, "steps of 4, 2 and 1");
        halve(std::integral_constant<int, 4>{});
        halve(std::integral_constant<int, 2>{});
        halve(std::integral_constant<int, 1>{});
#pragma unroll
        for (int i = 0; i < KEEP; ++i) k[i] = a[i];
    }
}

struct Partials {                 // in the workspace, for each of `blocks` workgroups
    float* p;                     // [blocks][experts] sums of the probabilities
    int32_t* count;               // [blocks][experts] choices
    int32_t* tokens;              // [blocks] tokens that have an expert
    double* loss;                 // [pieces] of the last step
    int32_t *choices, *arrived;   // [pieces], [1]
    int blocks;
};
constexpr int kPiece = 16;        // experts of a workgroup of the last step

int choose_blocks(int64_t tokens, int64_t experts, int num_cu) {
    const int64_t per = kThreads / (experts <= 256 ? 16 : 64);
    return int(std::max<int64_t>(std::min<int64_t>((tokens + per - 1) / per, 2 * num_cu), 1));
}
Partials partials_of(void* ws, int blocks, int experts) {
    Partials q{};
    uint8_t* at = static_cast<uint8_t*>(ws);
    const int pieces = (experts + kPiece - 1) / kPiece;
    q.loss = reinterpret_cast<double*>(at);
    q.p = reinterpret_cast<float*>(q.loss + pieces);
    q.count = reinterpret_cast<int32_t*>(q.p + int64_t(blocks) * experts);
    q.tokens = q.count + int64_t(blocks) * experts;
    q.choices = q.tokens + blocks;
    q.arrived = q.choices + pieces;
    q.blocks = blocks;
    return q;
}

// A lane sorts its experts, or the KEEP that can be chosen at all; the largest of the lanes' first ones is the next choice, and its lane moves up.
// What bounds it is the vector instructions: with 256 bfloat16 scores and 8 chosen, six hundred for four tokens (eight hundred with a sort of all 16 of a
// lane, keys of 16-bit scores made one at a time and weights in the loop over the choices).
template <typename T, int L, int V, int KEEP, bool BALANCE>
__global__ __launch_bounds__(kThreads) void choose_kernel(ChooseCall c, Partials q) {
    constexpr int kGroups = kThreads / L, kWaves = kThreads / 64;
    using K = Key<T>;
    __shared__ float part[BALANCE ? kWaves : 1][BALANCE ? L * V : 1];
    __shared__ int32_t count[BALANCE ? L * V : 1], some[BALANCE ? kGroups : 1];
    const int lane = threadIdx.x % L, group = threadIdx.x / L, first = lane * V, shift = int(threadIdx.x & 63) / L * L;
    const T* scores = static_cast<const T*>(c.scores);
    float psum[V];
    int mine = 0;
    if constexpr (BALANCE) {
        for (int e = threadIdx.x; e < L * V; e += kThreads) count[e] = 0;
        if (blockIdx.x == 0 && threadIdx.x == 0) *q.arrived = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) psum[v] = 0.0f;
        __syncthreads();
    }
    const int64_t step = int64_t(gridDim.x) * kGroups;
    int64_t t = int64_t(blockIdx.x) * kGroups + group;
    Scores<V, T> next;
    if (c.tokens > 0) next.fetch(scores, c.ld, c.experts, c.live, t, c.tokens, first);
    // every group of a wave comes along to the end: lanes ask each other
    for (; t - group < c.tokens; t += step) {
        Scores<V, T> now = next;
        const bool in = t < c.tokens, on = in && (!c.live || now.alive);
        next.fetch(scores, c.ld, c.experts, c.live, t + step, c.tokens, first);
        now.settle(c.experts, L * V, first);
        typename K::type key[V];
        now.keys(first, key);
        sort_first<KEEP>(key);
        auto largest = [&]() {
            const typename K::Head h = K::head(key[0]);
            if constexpr (K::kNamed) return fold_max<L>(h);
            else return group_max<L>(h);
        };
        typename K::Head top = largest();
        const bool any = on && top > K::kNone;
        const float m = any ? K::score(top) : 0.0f;
        float inverse = 0.0f;                        // of the probabilities' sum
        if (BALANCE || !c.normalize) {
            float ex[V];
            const float sum = exponentials<L>(now.e, m, ex);
            inverse = any ? 1.0f / sum : 0.0f;
            if constexpr (BALANCE) {
                if (any) {
                    mine += 1;
#pragma unroll
                    for (int v = 0; v < V; ++v) psum[v] = fmaf(ex[v], inverse, psum[v]);
                }
            }
        }
        int32_t* ids = c.ids + t * c.topk;
        float* weights = c.weights + t * c.topk;
        typename K::Head held[64 / L];               // lane j % L has the j-th choice
#pragma unroll
        for (int j0 = 0; j0 < 64 / L; ++j0) {
            held[j0] = K::kNone;
            if (j0 * L >= c.topk) continue;
            for (int j = j0 * L; j < min(j0 * L + L, c.topk); ++j) {
                if (j > 0) top = largest();
                bool won = K::head(key[0]) == top;
                if (lane == j - j0 * L) held[j0] = top;
                if constexpr (!K::kNamed) {
                    // of lanes with equal scores the lowest, which has the lower experts
                    uint64_t has = __ballot(won) >> shift;
                    if (L < 64) has &= (uint64_t(1) << (L & 63)) - 1;
                    won = won && (has & ((uint64_t(1) << lane) - 1)) == 0;
                    if (won && any && top > K::kNone) {
                        const int id = K::expert(key[0]);
                        if constexpr (BALANCE) atomicAdd(&count[id], 1);
                        ids[j] = id;
                    }
                }
#pragma unroll
                for (int v = 0; v < KEEP; ++v) {
                    const typename K::type now = key[v], next = v + 1 < KEEP ? key[v + 1] : typename K::type(K::kNamed ? INT32_MIN : 0);
                    key[v] = won ? next : now;
                }
            }
        }
        float w[64 / L], total = 0.0f;
#pragma unroll
        for (int j0 = 0; j0 < 64 / L; ++j0) {
            w[j0] = any && held[j0] > K::kNone ? exp_of(K::score(held[j0]), m) : 0.0f;
            total += w[j0];
        }
        const float scale = !c.normalize ? inverse : any ? 1.0f / group_sum<L>(total) : 0.0f;
#pragma unroll
        for (int j0 = 0; j0 < 64 / L; ++j0) {
            const int j = j0 * L + lane;
            if (j < c.topk && in) {
                const bool have = any && held[j0] > K::kNone;
                weights[j] = have ? w[j0] * scale : 0.0f;
                if constexpr (K::kNamed) {
                    const int id = have ? K::expert(held[j0]) : -1;
                    ids[j] = id;
                    if (BALANCE && have) atomicAdd(&count[id], 1);
                } else if (!have) {
                    ids[j] = -1;
                }
            }
        }
    }
    if constexpr (BALANCE) {
        // the wave's groups, then the waves, in one order
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if constexpr (L == 16) {
                psum[v] += __shfl_xor(psum[v], 16);
                psum[v] += __shfl_xor(psum[v], 32);
            }
            if ((threadIdx.x & 63) < L) part[threadIdx.x / 64][first + v] = psum[v];
        }
        if (lane == 0) some[group] = mine;
        __syncthreads();
        const int64_t at = int64_t(blockIdx.x) * c.experts;
        for (int e = threadIdx.x; e < c.experts; e += kThreads) {
            float sum = 0.0f;
            for (int g = 0; g < kWaves; ++g) sum += part[g][e];
            q.p[at + e] = sum;
            q.count[at + e] = count[e];
        }
        if (threadIdx.x == 0) {
            int n = 0;
            for (int g = 0; g < kGroups; ++g) n += some[g];
            q.tokens[blockIdx.x] = n;
        }
    }
}

// The workgroups' partial sums, added in their order: 16 experts to a workgroup; the one that is through last has the loss.  What bounds its 6 us is latency: a read
// of the partial sums, one more of the parts of the loss.
__global__ __launch_bounds__(kSumThreads) void balance_kernel(Partials q, int experts, int32_t* counts, int32_t* of_tokens, float* shares, float* loss) {
    constexpr int kRows = kSumThreads / kPiece, kWaves = kSumThreads / 64;
    __shared__ double p[kWaves][kPiece];
    __shared__ int32_t n[kWaves][kPiece], some[kWaves];
    __shared__ bool last;
    const int col = threadIdx.x % kPiece, row = threadIdx.x / kPiece, e = int(blockIdx.x) * kPiece + col, wave = threadIdx.x / 64;
    double sum = 0.0;
    int many = 0, tokens = 0;
    if (e < experts) {
#pragma unroll 8
        for (int b = row; b < q.blocks; b += kRows) {
            sum += double(q.p[int64_t(b) * experts + e]);
            many += q.count[int64_t(b) * experts + e];
        }
    }
    for (int b = threadIdx.x; b < q.blocks; b += kSumThreads) tokens += q.tokens[b];
    // four rows of a wave, then the waves
    for (int d = 16; d < 64; d *= 2) {
        sum += __shfl_xor(sum, d);
        many += __shfl_xor(many, d);
    }
    tokens = __builtin_amdgcn_readlane(sum_up_to(tokens), 63);
    if ((threadIdx.x & 63) < kPiece) {
        p[wave][col] = sum;
        n[wave][col] = many;
    }
    if ((threadIdx.x & 63) == 0) some[wave] = tokens;
    __syncthreads();
    sum = 0.0;
    many = tokens = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        sum += p[w][col];
        many += n[w][col];
        tokens += some[w];
    }
    const double inverse = tokens > 0 ? 1.0 / double(tokens) : 0.0;
    __syncthreads();
    if (threadIdx.x < kPiece) {
        if (e < experts) {
            shares[e] = float(sum * inverse);
            counts[e] = many;
        }
        // the sixteen, by one wave
        double l = sum * inverse * double(many);
        for (int d = 1; d < kPiece; d *= 2) {
            l += __shfl_xor(l, d);
            many += __shfl_xor(many, d);
        }
        p[0][col] = l;
        n[0][col] = many;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        if (blockIdx.x == 0) *of_tokens = tokens;
        const double l = p[0][0];
        const int all = n[0][0];
        // relaxed stores at the device's scope, then an arrival that is ordered behind them
        __hip_atomic_store(&q.loss[blockIdx.x], l, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(&q.choices[blockIdx.x], all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = __hip_atomic_fetch_add(q.arrived, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == int(gridDim.x) - 1;
    }
    __syncthreads();
    if (last && threadIdx.x < 64) {
        // at most 64 workgroups
        const bool there = threadIdx.x < gridDim.x;
        double l = there ? __hip_atomic_load(&q.loss[threadIdx.x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
        int64_t all = there ? __hip_atomic_load(&q.choices[threadIdx.x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
        for (int d = 1; d < 64; d *= 2) {
            l += __shfl_xor(l, d);
            all += __shfl_xor(all, d);
        }
        if (threadIdx.x == 0) *loss = all > 0 ? float(l * double(experts) / double(all)) : 0.0f;
    }
}

// The scores' gradient: p once more from the scores, and what the chosen experts get put into a row of LDS that is read as the scores are and cleared by
// those who wrote.  What bounds it is half the vector instructions, four hundred for four tokens of 256 scores, and half memory; loads with a branch around
// them, which made each wait for the one before, and instructions of cases that are not asked for took 28 us instead of 24; counts loaded by each lane 24
// instead of 19.
enum Parts { kAny, kNormalized, kPlain };
template <typename T, int L, int V, Parts P>
__global__ __launch_bounds__(kThreads, 4) void choose_grad_kernel(ChooseGradCall c) {
    // training has the weights' gradient and the loss's: those without the others' instructions
    const bool of_weights = P != kAny || c.dweights, normalize = P == kAny ? c.normalize != 0 : P == kNormalized, of_loss = P != kAny || c.counts;
    constexpr int kGroups = kThreads / L;
    // what a token's chosen experts get: a lane's part starts four words further on every 16, so that the lanes' 16 bytes lie in different banks
    constexpr int kPad = V >= 8 ? 4 : 0;
    __shared__ __align__(16) float spread[kGroups][L * (V + kPad)];
    const int lane = threadIdx.x % L, group = threadIdx.x / L, first = lane * V;
    float* part = spread[group] + lane * (V + kPad);
    auto at = [&](int id) { return &spread[group][id + id / V * kPad]; };
    const T* scores = static_cast<const T*>(c.scores);
    if (of_weights) {
#pragma unroll
        for (int v = 0; v < V; ++v) part[v] = 0.0f;
        __builtin_amdgcn_wave_barrier();
    }
    // a lane's choice of the first L: more are loaded when they are needed
    struct Chosen { int id; float w, dw; };
    auto chosen = [&](int64_t t, int j) {
        Chosen x{-1, 0.0f, 0.0f};
        if (of_weights) {
            const int64_t at = min(t, int64_t(c.tokens) - 1) * c.topk + min(j, c.topk - 1);
            x = Chosen{c.ids[at], c.weights[at], c.dweights[at]};
        }
        return x;
    };
    auto counts = [&](const Chosen& x, bool on) { return on && uint32_t(x.id) < uint32_t(c.experts); };
    const int64_t stride = int64_t(gridDim.x) * kGroups;
    int64_t t = int64_t(blockIdx.x) * kGroups + group;
    Scores<V, T> next;
    next.fetch(scores, c.ld, c.experts, c.live, t, c.tokens, first);
    Chosen next_chosen = chosen(t, lane);
    float f[V], scale = 0.0f;                 // f_e, times the loss's gradient
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = 0.0f;
    if (of_loss) {
        // through LDS: a lane's own are V apart from the next lane's, so that loads of them would share no line
        __shared__ __align__(16) int32_t of_all[L * V];
        for (int e = threadIdx.x; e < L * V; e += kThreads) of_all[e] = e < c.experts ? c.counts[e] : 0;
        const int tokens = *c.counted;
        const float dloss = c.dloss ? *c.dloss : 1.0f;
        __syncthreads();
        int n = 0, of[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            of[v] = of_all[first + v];
            n += of[v];
        }
        n = group_count<L>(n);
        const float inverse = n > 0 ? 1.0f / float(n) : 0.0f;
        if (tokens > 0) scale = c.factor * dloss * float(c.experts) / float(tokens);
#pragma unroll
        for (int v = 0; v < V; ++v) f[v] = scale * (float(of[v]) * inverse);
    }
    for (; t - group < c.tokens; t += stride) {
        Scores<V, T> now = next;
        const bool in = t < c.tokens, on = in && (!c.live || now.alive);
        Chosen mine = next_chosen;
        if (lane >= c.topk) mine.id = -1;
        float p[V];
        next.fetch(scores, c.ld, c.experts, c.live, t + stride, c.tokens, first);
        next_chosen = chosen(t + stride, lane);
        now.settle(c.experts, L * V, first);
        float m = -INFINITY;
#pragma unroll
        for (int v = 0; v < V; ++v) m = fmaxf(m, to_float(now.e[v]));
        m = group_largest<L>(m);
        // The maximum sees no NaN.  A token of NaN and -infinity alone has an expert all the same, so scores are looked at again where it found none
        bool any = m != -INFINITY, odd = false;
        const bool softmax = of_loss || !normalize;
        if (!softmax || __any(!any)) {
#pragma unroll
            for (int v = 0; v < V; ++v) odd = odd || to_float(now.e[v]) != to_float(now.e[v]);
            odd = in_group<L>(odd);
            any = any || odd;
        }
        any = any && on;
        if (softmax) {
            // a NaN, which the maximum does not see, is in the sum
            const float sum = exponentials<L>(now.e, m, p), inverse = 1.0f / sum;
#pragma unroll
            for (int v = 0; v < V; ++v) p[v] *= inverse;
        } else {
            // not needed, but for what NaN and +infinity make of all of them
#pragma unroll
            for (int v = 0; v < V; ++v) p[v] = odd || m == INFINITY ? NAN : 0.0f;
        }
        float s[V];
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = 0.0f;
        if (of_weights) {
            float dot = 0.0f;
            if (normalize) {
                dot = counts(mine, on) ? mine.w * mine.dw : 0.0f;
                for (int j = lane + L; j < c.topk; j += L) {
                    const Chosen x = chosen(t, j);
                    if (counts(x, on)) dot += x.w * x.dw;
                }
                dot = group_sum<L>(dot);
            }
            // each expert once: the order does not matter
            auto spend = [&](const Chosen& x) {
                if (counts(x, on)) atomicAdd(at(x.id), normalize ? x.w * (x.dw - dot) : x.dw);
            };
            spend(mine);
            for (int j = lane + L; j < c.topk; j += L) spend(chosen(t, j));
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int v = 0; v < V; ++v) s[v] = part[v];
            __builtin_amdgcn_wave_barrier();
            // and nothing for the next token
            if (counts(mine, on)) *at(mine.id) = 0.0f;
            for (int j = lane + L; j < c.topk; j += L) {
                const Chosen x = chosen(t, j);
                if (counts(x, on)) *at(x.id) = 0.0f;
            }
            __builtin_amdgcn_wave_barrier();
        }
        // through the softmax: of the loss's f, and without normalisation of the weights'
        const bool through = of_weights && !normalize;
        float dot = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) dot = fmaf(through ? f[v] + s[v] : f[v], p[v], dot);
        dot = group_sum<L>(dot);
        union { T r[V]; uint32_t w[V * sizeof(T) / 4 + (V == 1)]; } g;
#pragma unroll
        for (int v = 0; v < V; ++v) put(&g.r[v], through ? p[v] * (f[v] + s[v] - dot) : fmaf(p[v], f[v] - dot, s[v]));
        // a token that does not count, or has no expert: zero, whatever its scores are
#pragma unroll
        for (int i = 0; i < int(V * sizeof(T) + 3) / 4; ++i) g.w[i] = any ? g.w[i] : 0;
        T* out = static_cast<T*>(c.dscores) + t * c.ldd + first;
        const int have = in ? c.experts - first : 0;
        if (have >= V) {
            __builtin_memcpy(out, g.r, sizeof(g.r));
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (v < have) out[v] = g.r[v];
        }
    }
}

template <typename T, typename F>
void by_size(int experts, F&& f) {
    // lanes of a token, and experts of a lane
    if (experts <= 16) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    else if (experts <= 32) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
    else if (experts <= 64) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 4>{});
    else if (experts <= 128) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 8>{});
    else if (experts <= 256) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 16>{});
    else if (experts <= 512) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 8>{});
    else f(std::integral_constant<int, 64>{}, std::integral_constant<int, 16>{});
}

template <typename T>
void choose_typed(hipStream_t st, const ChooseCall& c, int num_cu) {
    by_size<T>(c.experts, [&](auto L, auto V) {
        constexpr int kL = decltype(L)::value, kV = decltype(V)::value;
        if (c.counts) {
            const Partials q = partials_of(c.ws, choose_blocks(c.tokens, c.experts, num_cu), c.experts);
            if (kV == 16 && c.topk <= 8) hipLaunchKernelGGL((choose_kernel<T, kL, kV, kV == 16 ? 8 : kV, true>), dim3(unsigned(q.blocks)), dim3(kThreads), 0, st, c, q);
            else hipLaunchKernelGGL((choose_kernel<T, kL, kV, kV, true>), dim3(unsigned(q.blocks)), dim3(kThreads), 0, st, c, q);
            hipLaunchKernelGGL(balance_kernel, dim3(unsigned((c.experts + kPiece - 1) / kPiece)), dim3(kSumThreads), 0, st, q, c.experts, c.counts, c.counted, c.shares, c.loss);
        } else {
            const int64_t blocks = (int64_t(c.tokens) * kL + kThreads - 1) / kThreads;
            const dim3 grid(unsigned(std::min<int64_t>(blocks, 8 * num_cu)));
            if (kV == 16 && c.topk <= 8) hipLaunchKernelGGL((choose_kernel<T, kL, kV, kV == 16 ? 8 : kV, false>), grid, dim3(kThreads), 0, st, c, Partials{});
            else hipLaunchKernelGGL((choose_kernel<T, kL, kV, kV, false>), grid, dim3(kThreads), 0, st, c, Partials{});
        }
    });
}

template <typename T>
void choose_grad_typed(hipStream_t st, const ChooseGradCall& c, int num_cu) {
    by_size<T>(c.experts, [&](auto L, auto V) {
        constexpr int kL = decltype(L)::value, kV = decltype(V)::value;
        const int64_t blocks = (int64_t(c.tokens) * kL + kThreads - 1) / kThreads;
        const dim3 grid(unsigned(std::min<int64_t>(blocks, 2 * num_cu)));
        auto launch = [&](auto P) { hipLaunchKernelGGL((choose_grad_kernel<T, kL, kV, decltype(P)::value>), grid, dim3(kThreads), 0, st, c); };
        if (!c.dweights || !c.counts) launch(std::integral_constant<Parts, kAny>{});
        else if (c.normalize) launch(std::integral_constant<Parts, kNormalized>{});
        else launch(std::integral_constant<Parts, kPlain>{});
    });
}

}  // namespace

size_t choose_bytes(int64_t tokens, int64_t experts, int num_cu) {
    const int64_t blocks = choose_blocks(tokens, experts, num_cu), pieces = (experts + kPiece - 1) / kPiece;
    return size_t(pieces * 12 + blocks * (experts * 8 + 4) + 4);
}

void launch_choose(hipStream_t st, const ChooseCall& c, int num_cu) {
    if (c.type == OZ_F32) choose_typed<float>(st, c, num_cu);
    else if (c.type == OZ_BF16) choose_typed<bf16_t>(st, c, num_cu);
    else choose_typed<f16_t>(st, c, num_cu);
}

void launch_choose_grad(hipStream_t st, const ChooseGradCall& c, int num_cu) {
    if (c.type == OZ_F32) choose_grad_typed<float>(st, c, num_cu);
    else if (c.type == OZ_BF16) choose_grad_typed<bf16_t>(st, c, num_cu);
    else choose_grad_typed<f16_t>(st, c, num_cu);
}

}  // namespace oz
