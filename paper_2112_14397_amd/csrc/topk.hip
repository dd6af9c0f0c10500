// Top-k gate, forward and backward: scores (softmax or sigmoid of given logits), a bias for the selection alone, groups of
// experts, the k largest keys, renormalised weights.  Its outputs are those of the DTS gate, so that dispatch, expert FFNs
// and combine follow in the same way.
//
// LPT lanes work on one token, lane g on the experts 4 g .. 4 g + 3 (LPT a power of two, 4 LPT >= E), and lie in one wave.  32768 tokens,
// 64 experts, k 8 of the 4 best of 8 groups, sigmoid with a bias: 22 us, of which two small launches are 4; 25 MB of logits, scores and
// weights are 5 us.  What bounds it is the number of instructions, 8 exchanges over the lanes in a row among them.  softmax, no groups: 16.
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
    int32_t* counts;          // [E]; added to (cleared before) where there are several blocks and no block_hist, else not
    int32_t* k_per_token;     // [T] or null
    int32_t* block_hist;      // [ceil(T/256), E] or null; added to (cleared before) where span < 256, else written
    int T, E, span;           // a block's tokens: 256, 128, 64 ...
    evomoe_topk o;
};

// Sums, maxima and unions over a token's 1, 2, 4, 8 or 16 lanes, in the same order for every lane: exchanges inside a row of 16 lanes
// cost one instruction, with the operation.
template <int CTRL> __device__ __forceinline__ uint32_t exchange(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int LPT, class F> __device__ __forceinline__ uint32_t over_lanes(uint32_t v, F&& f) {
    if (LPT >= 2) v = f(v, exchange<0xb1>(v));         // lanes 1, 0, 3, 2
    if (LPT >= 4) v = f(v, exchange<0x4e>(v));         // 2, 3, 0, 1
    if (LPT >= 8) v = f(v, exchange<0x141>(v));        // 7 .. 0
    if (LPT >= 16) v = f(v, exchange<0x140>(v));       // 15 .. 0
    return v;
}
template <int LPT> __device__ __forceinline__ float lanes_max(float v) {
    return __uint_as_float(over_lanes<LPT>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
}
template <int LPT> __device__ __forceinline__ float lanes_sum(float v) {
    return __uint_as_float(over_lanes<LPT>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}
template <int LPT> __device__ __forceinline__ int lanes_max(int v) {
    return (int)over_lanes<LPT>((uint32_t)v, [](uint32_t a, uint32_t b) { return (uint32_t)max((int)a, (int)b); });
}
template <int LPT> __device__ __forceinline__ uint32_t lanes_or(uint32_t v) {
    return over_lanes<LPT>(v, [](uint32_t a, uint32_t b) { return a | b; });
}
template <int CTRL> __device__ __forceinline__ double exchange(double v) {
    return __hiloint2double((int)exchange<CTRL>((uint32_t)__double2hiint(v)), (int)exchange<CTRL>((uint32_t)__double2loint(v)));
}
template <int LPT, class F> __device__ __forceinline__ double over_lanes(double v, F&& f) {
    if (LPT >= 2) v = f(v, exchange<0xb1>(v));
    if (LPT >= 4) v = f(v, exchange<0x4e>(v));
    if (LPT >= 8) v = f(v, exchange<0x141>(v));
    if (LPT >= 16) v = f(v, exchange<0x140>(v));
    return v;
}
template <int LPT> __device__ __forceinline__ double lanes_max(double v) {
    return over_lanes<LPT>(v, [](double a, double b) { return fmax(a, b); });
}
template <int LPT> __device__ __forceinline__ double lanes_sum(double v) {
    return over_lanes<LPT>(v, [](double a, double b) { return a + b; });
}

// A token's four logits of this lane; -inf for experts and tokens that do not exist.
__device__ __forceinline__ void load4(const float* from, bool there, size_t at, int e0, int E, float other, float (&z)[4]) {
    if (E % 4 == 0) {
        const f32x4 v = there && e0 < E ? *reinterpret_cast<const f32x4*>(from + at + e0) : f32x4{other, other, other, other};
        z[0] = v.x; z[1] = v.y; z[2] = v.z; z[3] = v.w;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = there && e0 + j < E ? from[at + e0 + j] : other;
    }
}
__device__ __forceinline__ void store4(float* to, bool there, size_t at, int e0, int E, const float (&z)[4]) {
    if (!there) return;
    if (E % 4 == 0) {
        if (e0 < E) *reinterpret_cast<f32x4*>(to + at + e0) = f32x4{z[0], z[1], z[2], z[3]};
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (e0 + j < E) to[at + e0 + j] = z[j];
    }
}

// Scores in float32; rest = 1 - s of a sigmoid.  The reciprocals, here and of the weights, are the instruction's, within one step of float32
// where a division is within half of one; key_margin counts it, and no output is narrower than that.
template <int LPT> __device__ __forceinline__ void scores_of(const float (&z)[4], bool softmax, float (&s)[4], float (&rest)[4]) {
    if (softmax) {
        float m = lanes_max<LPT>(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]))), sum = 0.f;
        if (m == -INFINITY) m = 0.f;                        // no expert left: every score is 0
#pragma unroll
        for (int j = 0; j < 4; ++j) { s[j] = expf(z[j] - m); sum += s[j]; }
        sum = lanes_sum<LPT>(sum);
        const float scale = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum);     // (of 1 .. 64; a NaN stays one)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] *= scale;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float e = expf(-fabsf(z[j])), big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
            s[j] = z[j] < 0.f ? small : big;                // (of a NaN both are one)
            rest[j] = z[j] < 0.f ? big : small;
        }
    }
}

// The weights without `scale`: w^_i = s_i / sum of the selected s, or s_i.  Where even the largest selected score is below 2^-100, a
// ratio is taken between values that the largest has been divided out of -- of a softmax exp(z_i - z_max), of a sigmoid exp(z_i -
// z_max) / (1 + exp(z_i)), as all are negative then -- so that it is right where the scores are below what float32 holds.
template <int LPT>
__device__ __forceinline__ void shares(const float (&z)[4], const float (&s)[4], const bool (&sel)[4], bool softmax,
                                       bool renormalise, float (&w)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = sel[j] ? s[j] : 0.f;
    if (!renormalise) return;
    float sum = lanes_sum<LPT>((w[0] + w[1]) + (w[2] + w[3]));
    if (!(sum >= 0x1p-100f)) {                           // (also where an expert that was not selected made the softmax a NaN)
        float zm = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) zm = sel[j] ? fmaxf(zm, z[j]) : zm;
        zm = lanes_max<LPT>(zm);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float v = expf(z[j] - zm);
            w[j] = sel[j] ? softmax ? v : v / (1.f + expf(z[j])) : 0.f;
        }
        sum = lanes_sum<LPT>((w[0] + w[1]) + (w[2] + w[3]));
    }
    const float inv = __builtin_amdgcn_rcpf(sum);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = sel[j] ? w[j] * inv : 0.f;
}

// The groups that are kept, as bits.  Lane g works on groups g, g + LPT, ...: the sum of the group's largest keys, then its place among
// all groups.  row: the token's keys (EP of them) in the LDS, and room for as many sums; sure: whether the kept groups are further from the
// others than margin(keys, their magnitudes).  A token's lanes lie in one wave, whose LDS accesses are made in order.
template <int LPT, class V, class M>
__device__ __forceinline__ uint64_t keep_groups(const evomoe_topk& o, int E, const V* keys, V* sums, int g, M&& margin, bool& sure) {
    const int size = E / o.groups;
    V worth[4], off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = g + LPT * i;
        V first = -INFINITY, second = -INFINITY;
        if (n < o.groups)
            for (int k = 0; k < size; ++k) {
                const V v = keys[n * size + k];
                second = v > first ? first : v > second ? v : second;
                first = v > first ? v : first;
            }
        const bool two = o.group_keys == 2 && second > (V)-INFINITY;
        worth[i] = two ? first + second : first;
        off[i] = margin(1 + two, fabs(first) + (two ? fabs(second) : (V)0));
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (g + LPT * i < o.groups) sums[g + LPT * i] = worth[i];
    __builtin_amdgcn_wave_barrier();
    uint64_t kept = 0;
    float last = INFINITY, next = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = g + LPT * i;
        bool keep = false;
        if (n < o.groups) {
            int rank = 0;
            for (int k = 0; k < o.groups; ++k) {
                const V w = sums[k];
                rank += w > worth[i] || (w == worth[i] && k < n);
            }
            keep = rank < o.top_groups;
            // (an infinity less or more an infinity is a NaN, which is passed over)
            if (keep) last = fminf(last, (float)(worth[i] - off[i])); else next = fmaxf(next, (float)(worth[i] + off[i]));
        }
        if (LPT * i < o.groups)
            kept |= (__ballot(keep) >> ((threadIdx.x & 63) & ~(LPT - 1)) & ((1ull << LPT) - 1)) << (LPT * i);
    }
    __builtin_amdgcn_wave_barrier();
    last = -lanes_max<LPT>(-last);
    next = lanes_max<LPT>(next);
    sure = !(next > -INFINITY) || last > next;
    return kept;
}
__device__ __forceinline__ bool in_group(uint64_t kept, int e, float inv_size) { return (kept >> (int)((e + 0.5f) * inv_size)) & 1; }

// The selection of the definition: keys in 64 bits, ties by index, one expert at a time.  For tokens whose float32 keys are too
// near to each other to decide.  How many those are depends on the logits (32768 tokens, 64 experts, k 8 of the 4 best of 8 groups): sigmoid
// with a bias of std 0.05 about one in ten thousand, for logits of std 1 as of std 8; softmax one in a thousand at std 1, 5 % at std 5, 39 % at
// std 8, as the keys at the border become small beside the margin, which is not relative; the call then takes 25.5, 32.4 and 35.9 us (two
// events).  row: room for EP doubles in the LDS.
template <int LPT>
__device__ __forceinline__ uint32_t select_exactly(const TopkArgs& a, const float (&z)[4], int e0, double* row) {
    const int E = a.E, g = e0 / 4;
    double key[4];
    if (a.o.score == EVOMOE_SOFTMAX) {
        float m = lanes_max<LPT>(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])));
        if (m == -INFINITY) m = 0.f;
        double sum = 0.;
#pragma unroll
        for (int j = 0; j < 4; ++j) { key[j] = exp((double)z[j] - (double)m); sum += key[j]; }
        sum = lanes_sum<LPT>(sum);
#pragma unroll
        for (int j = 0; j < 4; ++j) key[j] = sum == 0. ? 0. : key[j] / sum;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) key[j] = 1. / (1. + exp(-(double)z[j]));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float b = a.bias && e0 + j < E ? a.bias[e0 + j] : 0.f;
        if (a.bias) key[j] += (double)b;
        if (key[j] != key[j]) key[j] = INFINITY;
        if (z[j] == -INFINITY || b == -INFINITY) key[j] = -INFINITY;
    }
    if (a.o.groups > 1) {
        bool sure;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < 4; ++j) row[e0 + j] = key[j];
        __builtin_amdgcn_wave_barrier();
        const uint64_t kept = keep_groups<LPT>(a.o, E, row, row, g, [](int, double) { return 0.; }, sure);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (!in_group(kept, e0 + j, (float)a.o.groups / E)) key[j] = -INFINITY;
    }
    uint32_t sel = 0;
    for (int i = 0; i < a.o.k; ++i) {
        const double m = lanes_max<LPT>(fmax(fmax(key[0], key[1]), fmax(key[2], key[3])));
        if (!(m > -INFINITY)) break;
        uint32_t lowest = 64;                        // the lowest expert that has it
#pragma unroll
        for (int j = 3; j >= 0; --j) lowest = key[j] == m ? (uint32_t)(e0 + j) : lowest;
        lowest = over_lanes<LPT>(lowest, [](uint32_t p, uint32_t q) { return p < q ? p : q; });
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (lowest == (uint32_t)(e0 + j)) { sel |= 1u << j; key[j] = -INFINITY; }
    }
    return sel;
}

// How far the sum of n float32 keys may be from the exact one.  An exponential and a reciprocal are within 2 half steps, an operation
// within one: a sigmoid is off by 6 of its own size, a softmax by 15 (7 of them the sum over the experts) and 0.4 of 1 (the exponential's
// argument); the bias and the sum of two keys round by half a step of their own size, and so does the comparison.  size: of what has been
// added, the magnitudes.
__device__ __forceinline__ float key_margin(int n, float size, bool softmax) {
    return (n * (softmax ? 18.f : 8.f) + 4.f * size) * 0x1p-24f;
}

// float32 keys as integers of the same order (-0 as 0), and the one that is never taken, -inf
constexpr int kNoKey = (int)0x807fffffu;
__device__ __forceinline__ int in_order(float key) {
    const int b = __float_as_int(key + 0.f);
    return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float from_order(int key) { return __int_as_float(key ^ ((key >> 31) & 0x7fffffff)); }
__device__ __forceinline__ void sort_pair(int& high, int& low) {
    const int h = max(high, low);
    low = min(high, low);
    high = h;
}

// A block works on `span` tokens in passes of NT / LPT; the next pass's logits arrive under the present one's arithmetic.
// Selection: every lane sorts its four keys; k times the largest head of all lanes is taken off, and the last one taken is the border.
// Where it gives more than k experts, as several have its key, once more, one expert at a time.  Where the last key taken and the first
// one left (or two groups at the border) are within the margin, the token is decided in 64 bits.
template <int LPT> constexpr int kTopkThreads = LPT >= 4 ? 1024 : 256 * LPT;
template <int LPT>
__global__ __launch_bounds__(kTopkThreads<LPT>) void topk_gate_kernel(TopkArgs a)
{
    constexpr int NT = kTopkThreads<LPT>, TPB = NT / LPT, EP = 4 * LPT;
    __shared__ double rows[TPB][EP + 1];
    __shared__ int cnt[64];
    const int g = threadIdx.x % LPT, tl = threadIdx.x / LPT, e0 = 4 * g, E = a.E;
    const bool softmax = a.o.score == EVOMOE_SOFTMAX, by_logit = !a.bias && a.o.groups == 1;       // (scores rise with the logits)
    const int t0 = blockIdx.x * a.span, t1 = min(a.T, t0 + a.span);
    auto margin = [&](int n, float size) { return key_margin(n, size, softmax); };
    if (threadIdx.x < 64) cnt[threadIdx.x] = 0;
    __syncthreads();
    float bias[4], z_next[4];
    load4(a.bias, a.bias != nullptr, 0, e0, E, 0.f, bias);
    load4(a.logits, t0 + tl < t1, (size_t)(t0 + tl) * E, e0, E, -INFINITY, z_next);
    // (a wave ends with its own last token)
    for (int t = t0 + tl, first = __builtin_amdgcn_readfirstlane(t); first < t1; t += TPB, first += TPB) {
        const bool there = t < t1;
        const size_t at = (size_t)t * E;
        float z[4], s[4], rest[4], key[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = z_next[j];
        load4(a.logits, t + TPB < t1, at + (size_t)TPB * E, e0, E, -INFINITY, z_next);
        scores_of<LPT>(z, softmax, s, rest);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            key[j] = by_logit ? z[j] : s[j] + bias[j];
            if (key[j] != key[j]) key[j] = INFINITY;
            if (z[j] == -INFINITY || bias[j] == -INFINITY) key[j] = -INFINITY;
        }
        bool sure = true;
        if (a.o.groups > 1) {
            float* row = reinterpret_cast<float*>(rows[tl]);
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int j = 0; j < 4; ++j) row[e0 + j] = key[j];
            __builtin_amdgcn_wave_barrier();
            const uint64_t kept = keep_groups<LPT>(a.o, E, row, row + EP, g, margin, sure);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (!in_group(kept, e0 + j, (float)a.o.groups / E)) key[j] = -INFINITY;
        }
        int left[4], head[4];                                // in falling order
#pragma unroll
        for (int j = 0; j < 4; ++j) left[j] = head[j] = in_order(key[j]);
        sort_pair(head[0], head[1]); sort_pair(head[2], head[3]);
        sort_pair(head[0], head[2]); sort_pair(head[1], head[3]);
        sort_pair(head[1], head[2]);
        int last = kNoKey;
        for (int i = 0; i < a.o.k; ++i) {
            last = lanes_max<LPT>(head[0]);
            const bool hit = head[0] == last;
            head[0] = hit ? head[1] : head[0];
            head[1] = hit ? head[2] : head[1];
            head[2] = hit ? head[3] : head[2];
            head[3] = hit ? kNoKey : head[3];
        }
        int next = lanes_max<LPT>(head[0]);
        last = max(last, kNoKey + 1);
        uint32_t mine = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) mine |= (uint32_t)(left[j] >= last) << j;
        if (lanes_sum<LPT>((float)__popc(mine)) > (float)a.o.k) {
            mine = 0;
            for (int i = 0; i < a.o.k; ++i) {
                last = lanes_max<LPT>(max(max(left[0], left[1]), max(left[2], left[3])));
                uint32_t lowest = 64;                // the lowest expert that has it
#pragma unroll
                for (int j = 3; j >= 0; --j) lowest = left[j] == last ? (uint32_t)(e0 + j) : lowest;
                lowest = over_lanes<LPT>(lowest, [](uint32_t p, uint32_t q) { return p < q ? p : q; });
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (lowest == (uint32_t)(e0 + j)) { mine |= 1u << j; left[j] = kNoKey; }
            }
            next = last;                             // (more keys than k reach to it)
        }
        const float in = from_order(last), out = from_order(next);
        // (of two infinities the difference is a NaN: a tie)
        sure = sure && (by_logit || next == kNoKey || in - out > margin(1, fabsf(in)) + margin(1, fabsf(out)));
        if (!sure) mine = select_exactly<LPT>(a, z, e0, rows[tl]);

        bool sel[4];
        float w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) sel[j] = (mine >> j) & 1;
        shares<LPT>(z, s, sel, softmax, a.o.renormalise, w);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] *= a.o.scale;
        const uint32_t lo = lanes_or<LPT>(g < 8 ? mine << (4 * g & 31) : 0u), hi = LPT > 8 ? lanes_or<LPT>(g < 8 ? 0u : mine << (4 * g & 31)) : 0u;
        if (a.scores) store4(a.scores, there, at, e0, E, s);
        store4(a.gate_w, there, at, e0, E, w);
        if (there) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (sel[j]) atomicAdd(&cnt[e0 + j], 1);
            if (g == 0) {
                a.mask_bits[t] = (uint64_t)hi << 32 | lo;
                if (a.k_per_token) a.k_per_token[t] = __popc(lo) + __popc(hi);
            }
        }
    }
    __syncthreads();
    if ((int)threadIdx.x >= E) return;
    const int n = cnt[threadIdx.x];
    if (a.block_hist) {
        int32_t* h = a.block_hist + (size_t)(t0 / kDispatchTokens) * E + threadIdx.x;
        if (a.span == kDispatchTokens) *h = n; else if (n) atomicAdd(h, n);
    }
    if (gridDim.x == 1) a.counts[threadIdx.x] = n;
    else if (!a.block_hist && n) atomicAdd(&a.counts[threadIdx.x], n);
}

// counts = the column sums of block_hist.  (Integer additions of every block to the same E words took 30 us at 32768 tokens in blocks of
// 16.)  One block: EP columns by 1024 / EP row lanes.
template <int LPT>
__global__ __launch_bounds__(1024) void topk_counts_kernel(const int32_t* __restrict__ block_hist, int rows, int E, int32_t* __restrict__ counts)
{
    constexpr int EP = 4 * LPT, RL = 1024 / EP;
    __shared__ int sums[64];
    const int e = threadIdx.x % EP, rl = threadIdx.x / EP;
    if (threadIdx.x < 64) sums[threadIdx.x] = 0;
    __syncthreads();
    int n = 0;
    if (e < E)
#pragma unroll 8
        for (int r = rl; r < rows; r += RL) n += block_hist[(size_t)r * E + e];
    if (n) atomicAdd(&sums[e], n);
    __syncthreads();
    if ((int)threadIdx.x < E) counts[threadIdx.x] = sums[threadIdx.x];
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
    const bool softmax = a.o.score == EVOMOE_SOFTMAX, there = t < a.T;
    const size_t at = (size_t)t * E;
    float z[4], s[4], rest[4], w[4], dw[4], v[4], coef[4];
    bool sel[4];
    load4(a.logits, there, at, e0, E, -INFINITY, z);
#pragma unroll
    for (int j = 0; j < 4; ++j) coef[j] = a.coef && e0 + j < E ? a.coef_scale * a.coef[e0 + j] : 0.f;      // (aligned to 4 bytes only)
    const uint64_t bits = there ? a.mask_bits[t] : 0;
    int64_t slot = there ? (int64_t)a.tok_off[t] + __popcll(bits & ((1ull << e0) - 1)) : 0;
    int row[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        sel[j] = e0 + j < E && (bits >> (e0 + j)) & 1;
        row[j] = sel[j] && slot < a.P_cap ? a.tok_rows[slot] : -1;
        slot += sel[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) dw[j] = row[j] >= 0 ? a.dG_pairs[row[j]] : 0.f;
    scores_of<LPT>(z, softmax, s, rest);
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
        if (a.coef) v[j] += s[j] * coef[j];
        vsum += v[j];
    }
    if (softmax) vsum = lanes_sum<LPT>(vsum);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = softmax ? v[j] - s[j] * vsum : v[j] * rest[j];
    store4(a.dlogits, there, at, e0, E, v);
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
    const TopkArgs a{logits, balance_bias, scores, gate_w, mask_bits, counts, k_per_token, block_hist, s.T, s.E, kDispatchTokens, o};
    ProfScope ps(c, EVOMOE_K_TOPK_GATE);
    return with_lanes(s.E, [&](auto lanes) {
        constexpr int LPT = decltype(lanes)::value;
        // Blocks of 256 tokens, dispatch's unit, write their rows of block_hist outright; where they would leave CUs idle, smaller ones add
        // to cleared rows, or without them to the counts (32768 tokens, 64 experts, k 8, in groups: 39 us in 256 blocks, 43 in 128).
        TopkArgs b = a;
        while (s.T > b.span && b.span > kTopkThreads<LPT> / LPT && (s.T - 1) / b.span + 1 <= c.num_cu / 2) b.span /= 2;
        const int blocks = (s.T - 1) / b.span + 1;
        if (b.span < kDispatchTokens || (blocks > 1 && !block_hist)) {
            hipError_t err = launch_clear_counts(c, s, counts, block_hist);
            if (err != hipSuccess) return err;
        }
        hipLaunchKernelGGL(topk_gate_kernel<LPT>, dim3(blocks), dim3(kTopkThreads<LPT>), 0, c.stream, b);
        if (blocks > 1 && block_hist)
            hipLaunchKernelGGL(topk_counts_kernel<LPT>, dim3(1), dim3(1024), 0, c.stream, block_hist, dispatch_blocks(s), s.E, counts);
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
