// Top-k gate, forward and backward: scores (softmax or sigmoid of given logits), a bias for the selection alone, groups of
// experts, the k largest keys, renormalised weights.  Its outputs are those of the DTS gate, so that dispatch, expert FFNs
// and combine follow in the same way.
//
// LPT lanes work on one token, lane g on the experts 4 g .. 4 g + 3 (LPT a power of two, 4 LPT >= E), 256 / LPT tokens to a
// block; a token's lanes lie in one wave.
#include <type_traits>

#include "kernels.h"

namespace evomoe {

namespace {

struct TopkArgs {
    const float* logits;      // [T,E]
    const float* bias;        // [E] or null
    float* scores;            // [T,E] or null
    float* gate_w;            // [T,E]
    uint64_t* mask_bits;      // [T]
    int32_t* counts;          // [E], cleared
    int32_t* k_per_token;     // [T] or null
    int32_t* block_hist;      // [ceil(T/256), E], cleared, or null
    int T, E;
    evomoe_topk o;
};

// sums, maxima and unions over a token's lanes, in the same order for every lane
template <int LPT, typename V> __device__ __forceinline__ V lanes_sum(V v) {
#pragma unroll
    for (int o = LPT >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
template <int LPT> __device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
    for (int o = LPT >> 1; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// A token's four logits of this lane; -inf for experts and tokens that do not exist.
__device__ __forceinline__ void load_logits(const float* logits, int t, int T, int e0, int E, float (&z)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] = t < T && e0 + j < E ? logits[(size_t)t * E + e0 + j] : -INFINITY;
}

// The weights without `scale`: w^_i = s_i / sum of the selected s, or s_i.  A ratio of scores is taken between values that
// the largest of them has been divided out of -- of a softmax exp(z_i - z_max), of a sigmoid exp(z_i - z_max) / (1 + exp(z_i))
// where all are negative -- so that it is right where the scores themselves are below what float32 holds.
template <int LPT>
__device__ __forceinline__ void shares(const float (&z)[4], const float (&s)[4], const bool (&sel)[4], bool softmax,
                                       bool renormalise, float (&w)[4]) {
    if (!renormalise) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = sel[j] ? s[j] : 0.f;
        return;
    }
    float zm = -INFINITY, sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) zm = sel[j] ? fmaxf(zm, z[j]) : zm;
    zm = lanes_max<LPT>(zm);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float up = softmax ? zm : fminf(zm, 0.f);
        float v = expf(softmax ? z[j] - up : fminf(z[j], 0.f) - up);
        if (!softmax) v /= 1.f + expf(-fabsf(z[j]));
        w[j] = sel[j] ? v : 0.f;
        sum += w[j];
    }
    sum = lanes_sum<LPT>(sum);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = sel[j] ? w[j] / sum : 0.f;
}

template <int LPT>
__global__ __launch_bounds__(256) void topk_gate_kernel(TopkArgs a)
{
    constexpr int TPB = 256 / LPT, EP = 4 * LPT;
    __shared__ double keys[TPB][EP + 1], worth[TPB][EP + 1];
    __shared__ int cnt[64];
    const int g = threadIdx.x % LPT, tl = threadIdx.x / LPT, e0 = 4 * g;
    const int t = blockIdx.x * TPB + tl, E = a.E;
    const bool softmax = a.o.score == EVOMOE_SOFTMAX;
    if (threadIdx.x < 64) cnt[threadIdx.x] = 0;

    float z[4];
    double s[4], key[4];
    load_logits(a.logits, t, a.T, e0, E, z);
    if (softmax) {
        float m = lanes_max<LPT>(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])));
        if (m == -INFINITY) m = 0.f;                        // no expert left: every score is 0
        double sum = 0.;
#pragma unroll
        for (int j = 0; j < 4; ++j) { s[j] = exp((double)z[j] - (double)m); sum += s[j]; }
        sum = lanes_sum<LPT>(sum);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = sum == 0. ? 0. : s[j] / sum;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = 1. / (1. + exp(-(double)z[j]));
    }
    const bool by_logit = !a.bias && a.o.groups == 1;       // scores rise with the logits
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float b = a.bias && e0 + j < E ? a.bias[e0 + j] : 0.f;
        key[j] = by_logit ? (double)z[j] : s[j] + (double)b;
        if (key[j] != key[j]) key[j] = INFINITY;
        if (z[j] == -INFINITY || b == -INFINITY) key[j] = -INFINITY;
        keys[tl][e0 + j] = key[j];
    }
    __syncthreads();

    if (a.o.groups > 1) {
        const int size = E / a.o.groups;
        for (int n = g; n < a.o.groups; n += LPT) {
            double first = -INFINITY, second = -INFINITY;
            for (int i = 0; i < size; ++i) {
                const double v = keys[tl][n * size + i];
                second = v > first ? first : v > second ? v : second;
                first = v > first ? v : first;
            }
            worth[tl][n] = a.o.group_keys == 2 && second > -INFINITY ? first + second : first;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int own = (e0 + j) / size;
            if (e0 + j >= E) continue;
            const double v = worth[tl][own];
            int rank = 0;
            for (int n = 0; n < a.o.groups; ++n) rank += worth[tl][n] > v || (worth[tl][n] == v && n < own);
            if (rank >= a.o.top_groups) key[j] = -INFINITY;
            keys[tl][e0 + j] = key[j];
        }
        __syncthreads();
    }

    bool sel[4];
    uint64_t bits = 0;
    int rank[4] = {0, 0, 0, 0};
    for (int i = 0; i < E; ++i) {
        const double v = keys[tl][i];
#pragma unroll
        for (int j = 0; j < 4; ++j) rank[j] += v > key[j] || (v == key[j] && i < e0 + j);
    }
    float sf[4], w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        sel[j] = key[j] > -INFINITY && rank[j] < a.o.k;
        if (sel[j]) bits |= 1ull << (e0 + j);
        sf[j] = (float)s[j];
    }
#pragma unroll
    for (int o = LPT >> 1; o > 0; o >>= 1) bits |= __shfl_xor((unsigned long long)bits, o, 64);
    shares<LPT>(z, sf, sel, softmax, a.o.renormalise, w);

    if (t < a.T) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (e0 + j < E) {
                if (a.scores) a.scores[(size_t)t * E + e0 + j] = sf[j];
                a.gate_w[(size_t)t * E + e0 + j] = sel[j] ? a.o.scale * w[j] : 0.f;
                if (sel[j]) atomicAdd(&cnt[e0 + j], 1);
            }
        if (g == 0) {
            a.mask_bits[t] = bits;
            if (a.k_per_token) a.k_per_token[t] = __popcll(bits);
        }
    }
    __syncthreads();
    if ((int)threadIdx.x < E && cnt[threadIdx.x]) {
        atomicAdd(&a.counts[threadIdx.x], cnt[threadIdx.x]);
        if (a.block_hist) atomicAdd(&a.block_hist[(size_t)(blockIdx.x * TPB / kDispatchTokens) * E + threadIdx.x], cnt[threadIdx.x]);
    }
}

struct TopkBwdArgs {
    const float* dG_pairs;    // [P_cap]
    const int32_t* tok_off;   // [T+1]
    const int32_t* tok_rows;  // [P_cap]
    const float* logits;      // [T,E]
    const uint64_t* mask_bits;
    const float* coef;        // [E] or null
    float coef_scale;
    float* dlogits;           // [T,E]
    int T, E;
    int64_t P_cap;
    evomoe_topk o;
};

// The row of the pair (t, e) is tok_rows[tok_off[t] + number of selected experts below e].
template <int LPT>
__global__ __launch_bounds__(256) void topk_gate_bwd_kernel(TopkBwdArgs a)
{
    constexpr int TPB = 256 / LPT;
    const int g = threadIdx.x % LPT, tl = threadIdx.x / LPT, e0 = 4 * g;
    const int t = blockIdx.x * TPB + tl, E = a.E;
    const bool softmax = a.o.score == EVOMOE_SOFTMAX;
    float z[4], s[4], rest[4], w[4], dw[4], v[4];          // rest = 1 - s of a sigmoid
    bool sel[4];
    load_logits(a.logits, t, a.T, e0, E, z);
    const uint64_t bits = t < a.T ? a.mask_bits[t] : 0;
    const int64_t first = t < a.T ? a.tok_off[t] : 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int e = e0 + j;
        sel[j] = e < E && (bits >> e) & 1;
        dw[j] = 0.f;
        if (sel[j]) {
            const int64_t slot = first + __popcll(bits & ((1ull << e) - 1));
            if (slot < a.P_cap) dw[j] = a.dG_pairs[a.tok_rows[slot]];
        }
    }
    if (softmax) {
        float m = lanes_max<LPT>(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]))), sum = 0.f;
        if (m == -INFINITY) m = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) { s[j] = expf(z[j] - m); sum += s[j]; }
        sum = lanes_sum<LPT>(sum);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = sum == 0.f ? 0.f : s[j] / sum;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float e = expf(-fabsf(z[j])), big = 1.f / (1.f + e), small = e / (1.f + e);
            s[j] = z[j] >= 0.f ? big : z[j] < 0.f ? small : z[j];           // (a NaN stays one)
            rest[j] = z[j] >= 0.f ? small : z[j] < 0.f ? big : z[j];
        }
    }
    shares<LPT>(z, s, sel, softmax, a.o.renormalise, w);
    float inner = 0.f;
    if (a.o.renormalise) {
#pragma unroll
        for (int j = 0; j < 4; ++j) inner += w[j] * dw[j];
        inner = lanes_sum<LPT>(inner);
    }
    float vsum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = sel[j] ? a.o.scale * w[j] * (dw[j] - inner) : 0.f;
        if (a.coef && e0 + j < E) v[j] += s[j] * (a.coef_scale * a.coef[e0 + j]);
        vsum += v[j];
    }
    if (softmax) vsum = lanes_sum<LPT>(vsum);
    if (t >= a.T) return;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (e0 + j < E) a.dlogits[(size_t)t * E + e0 + j] = softmax ? v[j] - s[j] * vsum : v[j] * rest[j];
}

// calls f with the lanes per token as a constant
template <class F> hipError_t with_lanes(int E, F&& f) {
    if (E <= 4) return f(std::integral_constant<int, 1>{});
    if (E <= 8) return f(std::integral_constant<int, 2>{});
    if (E <= 16) return f(std::integral_constant<int, 4>{});
    if (E <= 32) return f(std::integral_constant<int, 8>{});
    return f(std::integral_constant<int, 16>{});
}

}  // namespace

hipError_t launch_topk_gate(const Ctx& c, const evomoe_shape& s, const evomoe_topk& o, const float* logits,
                            const float* balance_bias, float* scores, float* gate_w, uint64_t* mask_bits,
                            int32_t* counts, int32_t* k_per_token, int32_t* block_hist) {
    const TopkArgs a{logits, balance_bias, scores, gate_w, mask_bits, counts, k_per_token, block_hist, s.T, s.E, o};
    ProfScope ps(c, EVOMOE_K_TOPK_GATE);
    hipError_t err = launch_clear_counts(c, s, counts, block_hist);
    if (err != hipSuccess) return err;
    return with_lanes(s.E, [&](auto lanes) {
        constexpr int LPT = decltype(lanes)::value, TPB = 256 / LPT;
        hipLaunchKernelGGL(topk_gate_kernel<LPT>, dim3((s.T + TPB - 1) / TPB), dim3(256), 0, c.stream, a);
        return hipGetLastError();
    });
}

hipError_t launch_topk_gate_bwd(const Ctx& c, const evomoe_shape& s, const evomoe_topk& o, const float* dG_pairs,
                                const int32_t* tok_off, const int32_t* tok_rows, const float* logits,
                                const uint64_t* mask_bits, const float* dscore_coef, float loss_scale, float* dlogits) {
    const TopkBwdArgs a{dG_pairs, tok_off, tok_rows, logits, mask_bits, dscore_coef, loss_scale, dlogits, s.T, s.E,
                        s.P_cap, o};
    ProfScope ps(c, EVOMOE_K_TOPK_GATE_BWD);
    return with_lanes(s.E, [&](auto lanes) {
        constexpr int LPT = decltype(lanes)::value, TPB = 256 / LPT;
        hipLaunchKernelGGL(topk_gate_bwd_kernel<LPT>, dim3((s.T + TPB - 1) / TPB), dim3(256), 0, c.stream, a);
        return hipGetLastError();
    });
}

}  // namespace evomoe
