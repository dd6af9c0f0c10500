// Expert FFNs forward in 8 bits (e4m3 elements, a power of two scale for 32 of them along the contraction), on the scaled
// matrix instructions:
//   A = act(X W1^T + b1), to 8 bits again;     O = A W2^T + b2, bf16.
//
// Both products are computed transposed, C^T[n,r] = sum_k W[n,k] X[r,k]: the weights' rows are the matrix instruction's rows,
// and a lane of the result holds consecutive columns n of ONE row r, so that a group of 32 columns of A lies in a few
// lanes' registers and is converted without a detour through the LDS.
#include <type_traits>

#include "kernels.h"
#include "mx8.h"

namespace evomoe {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Mx8Args {
    const uint8_t* X;  const uint8_t* Xs;     // [*,K], [*,K/32]
    const uint8_t* W;  const uint8_t* Ws;     // [E,N,K], [E,N,K/32]
    const int32_t* rows;                      // gather of X's rows, or null
    const int32_t* expert_offsets;
    const float* bias;                        // [E,N] or null
    uint8_t* Aq;  uint8_t* As;                // first product: [P,N], [P,N/32]
    bf16_t* O;                                // second product: [P,N]
    int E, N, K, act;
    int64_t P_cap;
};

// v_mfma_scale_f32_16x16x128_f8f6f4: lane (q = lane / 16, i = lane % 16) brings the k's 16 q .. 16 q + 15 and 64 + 16 q .. of row i
// of either operand, and the scale of that row's k's 32 q .. 32 q + 31; it receives rows 4 q .. 4 q + 3 of column i.
__device__ __forceinline__ f32x4 mfma16(i32x8 a, i32x8 b, f32x4 c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}

// One wave: 16 rows x 32 columns.
template <bool FIRST>
__global__ __launch_bounds__(64) void mx8_gemm_kernel(Mx8Args p)
{
    const int lane = threadIdx.x, i16 = lane & 15, q = lane >> 4;
    int tile = blockIdx.x, g = 0, row0 = 0, rows = 0;
    for (; g < p.E; ++g) {
        row0 = clamp_pairs(p.expert_offsets[g], p.P_cap);
        rows = clamp_pairs(p.expert_offsets[g + 1], p.P_cap) - row0;
        const int n = (rows + 15) / 16;
        if (tile < n) break;
        tile -= n;
    }
    if (g == p.E) return;
    row0 += tile * 16;
    rows = min(16, rows - tile * 16);
    const int r = row0 + min(i16, rows - 1), n0 = blockIdx.y * 32, kg = p.K / kMxGroup;
    const int64_t xr = p.rows ? p.rows[r] : r;
    const uint8_t* x = p.X + xr * p.K;
    const uint8_t* xs = p.Xs + xr * kg;
    const int64_t wr = (int64_t)g * p.N + n0 + i16;
    f32x4 acc[2] = {};
    const u32x4 zero = {};
    for (int k = 0; k < p.K; k += 128) {
        auto load = [&](const uint8_t* row) {
            const int c0 = k + 16 * q, c1 = c0 + 64;
            const u32x4 lo = c0 < p.K ? *reinterpret_cast<const u32x4*>(row + c0) : zero;
            const u32x4 hi = c1 < p.K ? *reinterpret_cast<const u32x4*>(row + c1) : zero;
            return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        };
        auto scale = [&](const uint8_t* row) { return k / kMxGroup + q < kg ? (int)row[k / kMxGroup + q] : 127; };
        const i32x8 b = load(x);
        const int sb = scale(xs);
#pragma unroll
        for (int j = 0; j < 2; ++j)
            acc[j] = mfma16(load(p.W + (wr + 16 * j) * p.K), b, acc[j], scale(p.Ws + (wr + 16 * j) * kg), sb);
    }
    // (the compiler may move a matrix instruction under the branch that uses its result, where lanes without a row would
    // not bring their operands)
    asm volatile("" : "+v"(acc[0]), "+v"(acc[1]));
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[j] = acc[j / 4][j % 4];
        if (p.bias) v[j] += p.bias[(int64_t)g * p.N + n0 + 16 * (j / 4) + 4 * q + j % 4];
        if (FIRST) v[j] = act_fwd(v[j], p.act);
    }
    if constexpr (FIRST) {
        float m = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, mx_magnitude(v[j]));
        m = fmaxf(m, __shfl_xor(m, 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        const uint32_t b = mx_scale_byte(m);
        const float inv = mx_inverse(b);
        if (i16 < rows) {
            uint8_t* out = p.Aq + (int64_t)(row0 + i16) * p.N + n0 + 4 * q;
            *reinterpret_cast<uint32_t*>(out) = mx_pack4(v[0], v[1], v[2], v[3], inv);
            *reinterpret_cast<uint32_t*>(out + 16) = mx_pack4(v[4], v[5], v[6], v[7], inv);
            if (q == 0) p.As[(int64_t)(row0 + i16) * (p.N / kMxGroup) + n0 / kMxGroup] = (uint8_t)b;
        }
    } else if (i16 < rows) {
        bf16_t* out = p.O + (int64_t)(row0 + i16) * p.N + n0 + 4 * q;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            *reinterpret_cast<u32x2*>(out + 16 * j) = u32x2{pack_bf16x2(v[4 * j], v[4 * j + 1]), pack_bf16x2(v[4 * j + 2], v[4 * j + 3])};
    }
}

template <bool FIRST> hipError_t launch(const Ctx& c, const evomoe_shape& s, const Mx8Args& a) {
    const dim3 grid((unsigned)((s.P_cap + 15) / 16 + s.E), (unsigned)(a.N / 32));
    hipLaunchKernelGGL(mx8_gemm_kernel<FIRST>, grid, dim3(64), 0, c.stream, a);
    return hipGetLastError();
}

size_t aq_bytes(const evomoe_shape& s) { return ((size_t)s.P_cap * s.F + 255) & ~(size_t)255; }

}  // namespace

// [A : P_cap x F bytes, rounded up to 256][its scales]
size_t ffn_mx8_workspace_bytes(const evomoe_shape& s) {
    return aq_bytes(s) + (((size_t)s.P_cap * (s.F / kMxGroup) + 255) & ~(size_t)255);
}

hipError_t launch_expert_ffn_mx8(const Ctx& c, const evomoe_shape& s, const void* x_q, const uint8_t* x_scale,
                                 const int32_t* pair_token, const int32_t* expert_offsets, const void* W1_q,
                                 const uint8_t* W1_scale, const float* b1, const void* W2_q, const uint8_t* W2_scale,
                                 const float* b2, void* O, void* workspace) {
    uint8_t* Aq = (uint8_t*)workspace;
    uint8_t* As = Aq + aq_bytes(s);
    Mx8Args a{(const uint8_t*)x_q, x_scale, (const uint8_t*)W1_q, W1_scale, pair_token, expert_offsets, b1, Aq, As, nullptr,
              s.E, s.F, s.d, s.act, s.P_cap};
    hipError_t err;
    {
        ProfScope ps(c, EVOMOE_K_FFN_MX8_GEMM1);
        err = launch<true>(c, s, a);
    }
    if (err != hipSuccess) return err;
    a.X = Aq; a.Xs = As; a.W = (const uint8_t*)W2_q; a.Ws = W2_scale; a.rows = nullptr; a.bias = b2; a.O = (bf16_t*)O;
    a.N = s.d; a.K = s.F;
    ProfScope ps(c, EVOMOE_K_FFN_MX8_GEMM2);
    return launch<false>(c, s, a);
}

}  // namespace evomoe
