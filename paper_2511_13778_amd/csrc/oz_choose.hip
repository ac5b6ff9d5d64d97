// The router's choice: a token's scores s over the experts -> its topk experts and their weights, with the balance loss and the gradient of both.
//
//   p = softmax(s), chosen by falling score (ties: the lowest expert), w_j = p_j / sum of the chosen ones' (or p_j)
//   f_e = choices of e / all choices, P_e = mean over the tokens of p_e, loss = experts * sum_e f_e P_e
//   ds_i = w_i (dw_i - sum_j w_j dw_j) for the chosen (or p_i (dw_i - sum_j w_j dw_j), dw = 0 for the others) + dloss experts / tokens * p_i (f_i - sum_e f_e p_e)
//
// A token is a group of 16 lanes (64 beyond 256 experts), each with consecutive experts in registers: four tokens to a wave, so that maxima and sums over
// the experts are four rotations of 16 lanes.  Scores are compared as whole numbers that rise with them; 16-bit scores have their expert in the
// same word, whose maximum is then the choice itself.
#include <algorithm>

#include "oz_layer.h"
#include "oz_scaled_device.h"

namespace oz {

namespace {

constexpr int kThreads = 256;

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
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
    return fold<L>(x, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// Whole numbers that rise with the score: 0 where the expert is not to be had (score -infinity, or no such expert), a NaN above all, -0 as +0.
template <typename T>
struct Key {
    static constexpr bool kNamed = sizeof(T) == 2;       // the expert is in the low half, lower ones above higher ones
    static __device__ __forceinline__ uint32_t of(T x, int expert) {
        const float f = to_float(x) + 0.0f;
        if constexpr (kNamed) {
            const uint32_t u = f == 0.0f ? 0u : uint32_t(__builtin_bit_cast(uint16_t, x));
            const uint32_t up = (u & 0x8000u) ? 0xFFFFu - u : u + 0x8000u;
            const uint32_t key = (f != f ? 0xFFFFu : up) << 16 | uint32_t(0xFFFF - expert);
            return f == -INFINITY ? 0u : key;
        } else {
            const uint32_t u = __float_as_uint(f);
            const uint32_t up = u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
            return f == -INFINITY ? 0u : f != f ? 0xFFFFFFFFu : up;
        }
    }
    static __device__ __forceinline__ float score(uint32_t key) {
        if constexpr (kNamed) {
            const uint32_t up = key >> 16, u = (up & 0x8000u) ? up - 0x8000u : 0xFFFFu - up;
            return up == 0xFFFFu ? NAN : to_float(__builtin_bit_cast(T, uint16_t(u)));
        } else {
            return key == 0xFFFFFFFFu ? NAN : __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key);
        }
    }
};

// V consecutive elements, `have` of which are there.
template <int V, typename T>
__device__ __forceinline__ void load_scores(const T* p, int have, T (&e)[V]) {
    if (have >= V) {
        __builtin_memcpy(e, p, sizeof(e));
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) e[v] = v < have ? p[v] : T(0.0f);
    }
}

// exp(s - m) of a lane's experts (0 for those not to be had) and their sum over the group
template <int L, int V, typename T>
__device__ __forceinline__ float exponentials(const T (&e)[V], const uint32_t (&key)[V], float m, float (&ex)[V]) {
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        ex[v] = key[v] ? expf(to_float(e[v]) - m) : 0.0f;
        sum += ex[v];
    }
    return group_sum<L>(sum);
}

template <int V>
__device__ __forceinline__ uint32_t largest(const uint32_t (&key)[V]) {
    uint32_t top = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) top = max(top, key[v]);
    return top;
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

template <typename T, int L, int V, bool BALANCE>
__global__ __launch_bounds__(kThreads) void choose_kernel(ChooseCall c, Partials q) {
    constexpr int kGroups = kThreads / L;
    constexpr bool kNamed = Key<T>::kNamed;
    __shared__ float part[BALANCE ? kGroups : 1][BALANCE ? L * V : 1];
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
    // every group of a wave comes along to the end: lanes ask each other
    for (int64_t t0 = int64_t(blockIdx.x) * kGroups; t0 < c.tokens; t0 += int64_t(gridDim.x) * kGroups) {
        const int64_t t = t0 + group;
        const bool in = t < c.tokens, on = in && (!c.live || c.live[t]);
        T e[V];
        uint32_t key[V];
        load_scores(scores + (on ? t : 0) * c.ld + first, on ? c.experts - first : 0, e);
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = on && first + v < c.experts ? Key<T>::of(e[v], first + v) : 0u;
        uint32_t top = group_max<L>(largest(key));
        const float m = Key<T>::score(top);
        float inverse = 0.0f;                        // of the probabilities' sum
        if (BALANCE || !c.normalize) {
            float ex[V];
            const float sum = exponentials<L>(e, key, m, ex);
            inverse = top ? 1.0f / sum : 0.0f;
            if constexpr (BALANCE) {
#pragma unroll
                for (int v = 0; v < V; ++v) psum[v] += top ? ex[v] * inverse : 0.0f;
                mine += top ? 1 : 0;
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
                if (j > 0) top = group_max<L>(largest(key));
                if constexpr (kNamed) {
#pragma unroll
                    for (int v = 0; v < V; ++v) key[v] = key[v] == top ? 0u : key[v];
                    if (lane == j - j0 * L && top) held_id[j0] = int32_t(0xFFFFu - (top & 0xFFFFu));
                } else {
                    // the lowest lane that has it, and there the lowest expert
                    uint64_t has = __ballot(top != 0 && largest(key) == top) >> shift;
                    if (L < 64) has &= (uint64_t(1) << (L & 63)) - 1;
                    int32_t id = -1;
                    if (has && lane == int(__builtin_ctzll(has))) {
#pragma unroll
                        for (int v = V - 1; v >= 0; --v) id = key[v] == top ? first + v : id;
#pragma unroll
                        for (int v = 0; v < V; ++v) key[v] = first + v == id ? 0u : key[v];
                        if constexpr (BALANCE) atomicAdd(&count[id], 1);
                        ids[j] = id;
                    }
                    if (!has && lane == 0 && in) ids[j] = -1;
                }
                const float w = top ? expf(Key<T>::score(top) - m) : 0.0f;
                total += w;
                if (lane == j - j0 * L) held[j0] = w;
            }
        }
        const float scale = c.normalize ? (total != 0.0f ? 1.0f / total : 0.0f) : inverse;
#pragma unroll
        for (int j0 = 0; j0 < 64 / L; ++j0) {
            const int j = j0 * L + lane;
            if (j < c.topk && in) {
                weights[j] = held[j0] * scale;
                if constexpr (kNamed) {
                    ids[j] = held_id[j0];
                    if (BALANCE && held_id[j0] >= 0) atomicAdd(&count[held_id[j0]], 1);
                }
            }
        }
    }
    if constexpr (BALANCE) {
#pragma unroll
        for (int v = 0; v < V; ++v) part[group][first + v] = psum[v];
        if (lane == 0) some[group] = mine;
        __syncthreads();
        const int64_t at = int64_t(blockIdx.x) * c.experts;
        for (int e = threadIdx.x; e < c.experts; e += kThreads) {
            float sum = 0.0f;
            for (int g = 0; g < kGroups; ++g) sum += part[g][e];
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
__global__ __launch_bounds__(kThreads) void balance_kernel(Partials q, int experts, int32_t* counts, int32_t* of_tokens, float* shares, float* loss) {
    constexpr int kRows = kThreads / kPiece;
    __shared__ double p[kRows][kPiece];
    __shared__ int32_t n[kRows][kPiece], some[kThreads];
    __shared__ bool last;
    const int col = threadIdx.x % kPiece, row = threadIdx.x / kPiece, e = int(blockIdx.x) * kPiece + col;
    double sum = 0.0;
    int many = 0, tokens = 0;
    if (e < experts) {
#pragma unroll 4
        for (int b = row; b < q.blocks; b += kRows) {
            sum += double(q.p[int64_t(b) * experts + e]);
            many += q.count[int64_t(b) * experts + e];
        }
    }
    for (int b = threadIdx.x; b < q.blocks; b += kThreads) tokens += q.tokens[b];
    p[row][col] = sum;
    n[row][col] = many;
    some[threadIdx.x] = tokens;
    __syncthreads();
    for (int d = kThreads / 2; d > 0; d >>= 1) {
        if (int(threadIdx.x) < d) some[threadIdx.x] += some[threadIdx.x + d];
        __syncthreads();
    }
    const double inverse = some[0] > 0 ? 1.0 / double(some[0]) : 0.0;
    if (row == 0) {
        sum = 0.0;
        many = 0;
        for (int r = 0; r < kRows; ++r) {
            sum += p[r][col];
            many += n[r][col];
        }
        if (e < experts) {
            shares[e] = float(sum * inverse);
            counts[e] = many;
        }
        p[0][col] = sum * inverse * double(many);
        n[0][col] = many;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        if (blockIdx.x == 0) *of_tokens = some[0];
        double l = 0.0;
        int all = 0;
        for (int i = 0; i < kPiece; ++i) {
            l += p[0][i];
            all += n[0][i];
        }
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
    __shared__ __align__(16) float spread[kGroups][L * V];            // what a token's chosen experts get
    const int lane = threadIdx.x % L, group = threadIdx.x / L, first = lane * V;
    const T* scores = static_cast<const T*>(c.scores);
    float f[V], scale = 0.0f;
    if (c.counts) {
        int n = 0, of[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            of[v] = first + v < c.experts ? c.counts[first + v] : 0;
            n += of[v];
        }
        n = group_count<L>(n);
        const int tokens = *c.counted;
        if (tokens > 0) scale = c.factor * (c.dloss ? *c.dloss : 1.0f) * float(c.experts) / float(tokens);
#pragma unroll
        for (int v = 0; v < V; ++v) f[v] = n > 0 ? float(of[v]) / float(n) : 0.0f;
    }
    for (int64_t t0 = int64_t(blockIdx.x) * kGroups; t0 < c.tokens; t0 += int64_t(gridDim.x) * kGroups) {
        const int64_t t = t0 + group;
        const bool in = t < c.tokens, on = in && (!c.live || c.live[t]);
        T e[V];
        uint32_t key[V];
        float p[V], d[V];
        load_scores(scores + (on ? t : 0) * c.ld + first, on ? c.experts - first : 0, e);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            key[v] = on && first + v < c.experts ? Key<T>::of(e[v], first + v) : 0u;
            p[v] = d[v] = 0.0f;
        }
        const uint32_t top = group_max<L>(largest(key));
        if (c.counts || !c.normalize) {
            const float sum = exponentials<L>(e, key, Key<T>::score(top), p), inverse = top ? 1.0f / sum : 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) p[v] *= inverse;
        }
        if (c.dweights) {
            const int64_t at = t * c.topk;
            float dot = 0.0f;
            for (int j = lane; j < c.topk; j += L)
                if (on && uint32_t(c.ids[at + j]) < uint32_t(c.experts)) dot += c.weights[at + j] * c.dweights[at + j];
            dot = group_sum<L>(dot);
#pragma unroll
            for (int v = 0; v < V; ++v) spread[group][first + v] = 0.0f;
            __builtin_amdgcn_wave_barrier();
            for (int j = lane; j < c.topk; j += L) {
                const int id = on ? c.ids[at + j] : -1;
                if (uint32_t(id) < uint32_t(c.experts)) {
                    const float dw = c.dweights[at + j];
                    atomicAdd(&spread[group][id], c.normalize ? c.weights[at + j] * (dw - dot) : dw);      // each expert once: the order does not matter
                }
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int v = 0; v < V; ++v) d[v] = c.normalize ? spread[group][first + v] : p[v] * (spread[group][first + v] - dot);
            __builtin_amdgcn_wave_barrier();
        }
        if (c.counts) {
            float dot = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) dot = fmaf(f[v], p[v], dot);
            dot = group_sum<L>(dot);
#pragma unroll
            for (int v = 0; v < V; ++v) d[v] = fmaf(scale * p[v], f[v] - dot, d[v]);
        }
        T* out = static_cast<T*>(c.dscores) + t * c.ldd + first;
        const int have = in ? c.experts - first : 0;
        T r[V];
#pragma unroll
        for (int v = 0; v < V; ++v) put(&r[v], key[v] ? d[v] : 0.0f);
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
            hipLaunchKernelGGL(balance_kernel, dim3(unsigned((c.experts + kPiece - 1) / kPiece)), dim3(kThreads), 0, st, q, c.experts, c.counts, c.counted, c.shares, c.loss);
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
        hipLaunchKernelGGL((choose_grad_kernel<T, kL, kV>), dim3(unsigned(std::min<int64_t>(blocks, 8 * num_cu))), dim3(kThreads), 0, st, c);
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
