// The router's choice: a token's scores s over the experts -> its topk experts and their weights, with the balance loss and the gradient of both.
//
//   p = softmax(s), chosen by falling score (ties: the lowest expert), w_j = p_j / sum of the chosen ones' (or p_j)
//   f_e = choices of e / all choices, P_e = mean over the tokens of p_e, loss = experts * sum_e f_e P_e
//   ds_i = w_i (dw_i - sum_j w_j dw_j) for the chosen (or p_i (dw_i - sum_j w_j dw_j), dw = 0 for the others) + dloss experts / tokens * p_i (f_i - sum_e f_e p_e)
//
// A token is a group of 16 lanes (64 beyond 256 experts), each with consecutive experts in registers: four tokens to a wave, so that maxima and sums over
// the experts are four rotations of 16 lanes.
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
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
    return fold<L>(x, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// Scores as whole numbers that rise with them, the expert in the low bits (lower ones above higher ones), so that no two are equal.  16-bit scores
// are 19 bits of a float32 at most and leave room for the expert in the same word; float32 takes two.  -0 counts as +0, a NaN is above all; what is
// not above `kNone` is an expert that is not to be had (score -infinity, or no such expert).
template <typename T>
struct Key {
    static constexpr bool kNamed = sizeof(T) == 2;
    using type = std::conditional_t<kNamed, uint32_t, uint64_t>;
    static constexpr uint32_t kLow = 0x1FFF, kNone = 0x007FFFFF;
    static __device__ __forceinline__ uint32_t rising(float f) {
        f = f != f ? __uint_as_float(0x7FFFFFFFu) : f + 0.0f;
        return __float_as_uint(f) ^ (uint32_t(int32_t(__float_as_uint(f)) >> 31) | 0x80000000u);
    }
    static __device__ __forceinline__ type of(float f, int expert) {
        if constexpr (kNamed) return (rising(f) & ~kLow) | (kLow - uint32_t(expert));
        else return uint64_t(rising(f)) << 32 | uint32_t(~expert);
    }
    static __device__ __forceinline__ uint32_t head(type key) {
        if constexpr (kNamed) return key;
        else return uint32_t(key >> 32);
    }
    // of a key, or of a float32's upper word
    static __device__ __forceinline__ float score(uint32_t head) {
        const uint32_t up = kNamed ? head | kLow : head;
        const uint32_t u = (head & 0x80000000u) ? (kNamed ? head & ~kLow : head) ^ 0x80000000u : ~up;
        return __uint_as_float(u);
    }
};

// A lane's part of a token's scores, sent for before it is used: V consecutive elements, `have` of which are there, and whether the token counts.
template <int V, typename T>
struct Scores {
    T e[V];
    int have;
    bool in, on;
    __device__ __forceinline__ void fetch(const T* scores, int64_t ld, int experts, const uint8_t* live, int64_t t, int64_t tokens, int first) {
        in = t < tokens;
        have = in ? experts - first : 0;
        const T* p = scores + (in ? t : 0) * ld + first;
        if (have >= V) {
            __builtin_memcpy(e, p, sizeof(e));
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) e[v] = v < have ? p[v] : T(0.0f);
        }
        on = in && (!live || live[t]);
    }
    // -infinity: not to be had
    __device__ __forceinline__ void settle(float (&s)[V]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = on && v < have ? to_float(e[v]) : -INFINITY;
    }
};

// exp(x), x <= 0: 2^(x log2 e), relatively off by a step of the result and by 2^-24 |x|; zero below 2^-126
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// exp(s - m) and their sum over the group
template <int L, int V>
__device__ __forceinline__ float exponentials(const float (&s)[V], float m, float (&ex)[V]) {
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        ex[v] = exp_of(s[v] - m);
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

// A lane sorts its experts; the largest of the lanes' first ones is the next choice, and its lane moves up.
template <typename T, int L, int V, bool BALANCE>
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
    next.fetch(scores, c.ld, c.experts, c.live, t, c.tokens, first);
    // every group of a wave comes along to the end: lanes ask each other
    for (; t - group < c.tokens; t += step) {
        const bool in = next.in;
        float s[V];
        typename K::type key[V];
        next.settle(s);
        if (t - group + step < c.tokens) next.fetch(scores, c.ld, c.experts, c.live, t + step, c.tokens, first);
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = K::of(s[v], first + v);
        sort_falling(key);
        uint32_t top = group_max<L>(K::head(key[0]));
        const bool any = top > K::kNone;
        const float m = any ? K::score(top) : 0.0f;
        float inverse = 0.0f;                        // of the probabilities' sum
        if (BALANCE || !c.normalize) {
            float ex[V];
            const float sum = exponentials<L>(s, m, ex);
            inverse = any ? 1.0f / sum : 0.0f;
            if constexpr (BALANCE) {
#pragma unroll
                for (int v = 0; v < V; ++v) psum[v] = any ? fmaf(ex[v], inverse, psum[v]) : psum[v];
                mine += any ? 1 : 0;
            }
        }
        int32_t* ids = c.ids + t * c.topk;
        float* weights = c.weights + t * c.topk;
        float held[64 / L], total = 0.0f;            // lane j % L has the j-th choice
        int32_t held_id[64 / L];
#pragma unroll
        for (int j0 = 0; j0 < 64 / L; ++j0) {
            held[j0] = 0.0f;
            held_id[j0] = -1;
            if (j0 * L >= c.topk) continue;
            for (int j = j0 * L; j < min(j0 * L + L, c.topk); ++j) {
                if (j > 0) top = group_max<L>(K::head(key[0]));
                const bool have = top > K::kNone;
                bool won = have && K::head(key[0]) == top;
                if constexpr (K::kNamed) {
                    if (lane == j - j0 * L && have) held_id[j0] = int32_t(K::kLow - (top & K::kLow));
                } else {
                    // of lanes with equal scores the lowest, which has the lower experts
                    uint64_t has = __ballot(won) >> shift;
                    if (L < 64) has &= (uint64_t(1) << (L & 63)) - 1;
                    won = won && (has & ((uint64_t(1) << lane) - 1)) == 0;
                    if (won) {
                        const int id = int(~uint32_t(key[0]));
                        if constexpr (BALANCE) atomicAdd(&count[id], 1);
                        ids[j] = id;
                    }
                    if (!have && lane == 0 && in) ids[j] = -1;
                }
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const typename K::type now = key[v], next = v + 1 < V ? key[v + 1] : 0;
                    key[v] = won ? next : now;
                }
                const float w = have ? exp_of(K::score(top) - m) : 0.0f;
                total += w;
                if (lane == j - j0 * L) held[j0] = w;
            }
        }
        const float scale = c.normalize ? (any ? 1.0f / total : 0.0f) : inverse;
#pragma unroll
        for (int j0 = 0; j0 < 64 / L; ++j0) {
            const int j = j0 * L + lane;
            if (j < c.topk && in) {
                weights[j] = held[j0] * scale;
                if constexpr (K::kNamed) {
                    ids[j] = held_id[j0];
                    if (BALANCE && held_id[j0] >= 0) atomicAdd(&count[held_id[j0]], 1);
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

// The workgroups' partial sums, added in their order: 16 experts to a workgroup; the one that is through last has the loss.
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
    if (last && threadIdx.x == 0) {
        double l = 0.0;
        int64_t all = 0;
        for (int i = 0; i < int(gridDim.x); ++i) {
            l += __hip_atomic_load(&q.loss[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            all += __hip_atomic_load(&q.choices[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        *loss = all > 0 ? float(l * double(experts) / double(all)) : 0.0f;
    }
}

template <typename T, int L, int V>
__global__ __launch_bounds__(kThreads) void choose_grad_kernel(ChooseGradCall c) {
    constexpr int kGroups = kThreads / L;
    // what a token's chosen experts get: a lane's part starts four words further on every 16, so that the lanes' 16 bytes lie in different banks
    constexpr int kPad = V >= 8 ? 4 : 0;
    __shared__ __align__(16) float spread[kGroups][L * (V + kPad)];
    const int lane = threadIdx.x % L, group = threadIdx.x / L, first = lane * V;
    float* part = spread[group] + lane * (V + kPad);
    const T* scores = static_cast<const T*>(c.scores);
    float f[V], scale = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = 0.0f;
    if (c.counts) {
        int n = 0, of[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            of[v] = first + v < c.experts ? c.counts[first + v] : 0;
            n += of[v];
        }
        n = group_count<L>(n);
        const int tokens = *c.counted;
        const float inverse = n > 0 ? 1.0f / float(n) : 0.0f;
        if (tokens > 0) scale = c.factor * (c.dloss ? *c.dloss : 1.0f) * float(c.experts) / float(tokens);
#pragma unroll
        for (int v = 0; v < V; ++v) f[v] = float(of[v]) * inverse;
    }
    // a lane's choice of the first L: more are loaded when they are needed
    struct Chosen { int id; float w, dw; };
    auto chosen = [&](int64_t t, int j, bool in) {
        Chosen x{-1, 0.0f, 0.0f};
        if (in && j < c.topk && c.dweights) {
            const int64_t at = t * c.topk + j;
            x = Chosen{c.ids[at], c.weights[at], c.dweights[at]};
        }
        return x;
    };
    auto counts = [&](const Chosen& x, bool on) { return on && uint32_t(x.id) < uint32_t(c.experts); };
    const int64_t stride = int64_t(gridDim.x) * kGroups;
    int64_t t = int64_t(blockIdx.x) * kGroups + group;
    Scores<V, T> next;
    next.fetch(scores, c.ld, c.experts, c.live, t, c.tokens, first);
    Chosen next_chosen = chosen(t, lane, next.in);
    for (; t - group < c.tokens; t += stride) {
        const bool in = next.in, on = next.on;
        const Chosen mine = next_chosen;
        float s[V], p[V], g[V];
        next.settle(s);
        if (t - group + stride < c.tokens) {
            next.fetch(scores, c.ld, c.experts, c.live, t + stride, c.tokens, first);
            next_chosen = chosen(t + stride, lane, next.in);
        }
        float m = -INFINITY;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            m = fmaxf(m, s[v]);
            g[v] = scale * f[v];
        }
        m = group_largest<L>(m);
        const bool any = m != -INFINITY;
        if (c.counts || !c.normalize) {
            // a NaN is not seen by the maximum, but in the sum
            const float sum = exponentials<L>(s, any ? m : 0.0f, p), inverse = any ? 1.0f / sum : 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) p[v] *= inverse;
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) p[v] = 0.0f;
        }
        if (c.dweights) {
            float dot = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) part[v] = 0.0f;
            if (c.normalize) {
                dot = counts(mine, on) ? mine.w * mine.dw : 0.0f;
                for (int j = lane + L; j < c.topk; j += L) {
                    const Chosen x = chosen(t, j, in);
                    if (counts(x, on)) dot += x.w * x.dw;
                }
                dot = group_sum<L>(dot);
            }
            __builtin_amdgcn_wave_barrier();
            // each expert once: the order does not matter
            auto spend = [&](const Chosen& x) {
                if (counts(x, on)) atomicAdd(&spread[group][x.id + x.id / V * kPad], c.normalize ? x.w * (x.dw - dot) : x.dw);
            };
            spend(mine);
            for (int j = lane + L; j < c.topk; j += L) spend(chosen(t, j, in));
            __builtin_amdgcn_wave_barrier();
        }
        // through the softmax: of the loss's f, and without normalisation of the weights'
        if (c.dweights && !c.normalize) {
#pragma unroll
            for (int v = 0; v < V; ++v) g[v] += part[v];
        }
        float dot = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) dot = fmaf(g[v], p[v], dot);
        dot = group_sum<L>(dot);
        T r[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float d = p[v] * (g[v] - dot);
            if (c.dweights && c.normalize) d += part[v];
            put(&r[v], s[v] != -INFINITY ? d : 0.0f);
        }
        __builtin_amdgcn_wave_barrier();
        T* out = static_cast<T*>(c.dscores) + t * c.ldd + first;
        const int have = in ? c.experts - first : 0;
        if (have >= V) {
            __builtin_memcpy(out, r, sizeof(r));
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (v < have) out[v] = r[v];
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
            hipLaunchKernelGGL((choose_kernel<T, kL, kV, true>), dim3(unsigned(q.blocks)), dim3(kThreads), 0, st, c, q);
            hipLaunchKernelGGL(balance_kernel, dim3(unsigned((c.experts + kPiece - 1) / kPiece)), dim3(kSumThreads), 0, st, q, c.experts, c.counts, c.counted, c.shares, c.loss);
        } else {
            const int64_t blocks = (int64_t(c.tokens) * kL + kThreads - 1) / kThreads;
            hipLaunchKernelGGL((choose_kernel<T, kL, kV, false>), dim3(unsigned(std::min<int64_t>(blocks, 8 * num_cu))), dim3(kThreads), 0, st, c, Partials{});
        }
    });
}

template <typename T>
void choose_grad_typed(hipStream_t st, const ChooseGradCall& c, int num_cu) {
    by_size<T>(c.experts, [&](auto L, auto V) {
        constexpr int kL = decltype(L)::value, kV = decltype(V)::value;
        const int64_t blocks = (int64_t(c.tokens) * kL + kThreads - 1) / kThreads;
        hipLaunchKernelGGL((choose_grad_kernel<T, kL, kV>), dim3(unsigned(std::min<int64_t>(blocks, 2 * num_cu))), dim3(kThreads), 0, st, c);
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
