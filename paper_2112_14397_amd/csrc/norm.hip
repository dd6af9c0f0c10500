// Residual addition with the root-mean-square norm, forward (to the layer's type and to 8 bits) and backward, and the conversion of
// a matrix to 8 bits.  All of it is reading and writing rows.
#include "kernels.h"
#include "mx8.h"

namespace evomoe {

namespace {

template <typename TX> struct NormArgs {
    const TX* x;
    const TX* residual;       // or null
    const float* gamma;
    TX* h;                    // or null
    TX* y;                    // or null
    float* rstd;              // or null
    uint8_t* q;               // or null
    uint8_t* q_scale;
    float eps;
    int T, d;
};

// sum over the block's 256 threads, the same in all of them; fixed order
__device__ __forceinline__ float block_sum(float v, float* red) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return ((red[0] + red[1]) + red[2]) + red[3];
}

// One vector of a row, in 8 bits: the 32 / KV lanes of a group lie next to each other, and all of them or none are here.
template <int KV>
__device__ __forceinline__ void store_mx8(const float (&v)[KV], uint8_t* q, uint8_t* scale, int64_t at) {
    float m = mx_largest(v);
#pragma unroll
    for (int o = 1; o < kMxGroup / KV; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    const uint32_t b = mx_scale_byte(m);
#pragma unroll
    for (int j = 0; j < KV; j += 4)
        *reinterpret_cast<uint32_t*>(q + at + j) = mx_pack4(v[j], v[j + 1], v[j + 2], v[j + 3], b);
    if (at % kMxGroup == 0) scale[at / kMxGroup] = (uint8_t)b;
}

// One block per row.  (Outputs may be inputs: a vector is written after the same thread has read it.)
template <typename TX>
__global__ __launch_bounds__(256) void add_rmsnorm_kernel(NormArgs<TX> a)
{
    constexpr int KV = Elem<TX>::kVec;
    __shared__ float red[4];
    const int64_t row = (int64_t)blockIdx.x * a.d;
    auto sum_of = [&](int i, float (&v)[KV]) {              // h, as it is stored
        Elem<TX>::load_vec(a.x + row + i, v);
        if (!a.residual) return;
        float r[KV];
        Elem<TX>::load_vec(a.residual + row + i, r);
#pragma unroll
        for (int j = 0; j < KV; ++j) v[j] = (float)(TX)(v[j] + r[j]);
    };
    float ss = 0.f;
    for (int i = threadIdx.x * KV; i < a.d; i += 256 * KV) {
        float v[KV];
        sum_of(i, v);
        if (a.h) Elem<TX>::store_vec(a.h + row + i, v);
#pragma unroll
        for (int j = 0; j < KV; ++j) ss += v[j] * v[j];
    }
    const float rstd = 1.f / sqrtf(block_sum(ss, red) / a.d + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[blockIdx.x] = rstd;
    if (!a.y && !a.q) return;
    for (int i = threadIdx.x * KV; i < a.d; i += 256 * KV) {
        float v[KV];
        if (a.h) Elem<TX>::load_vec(a.h + row + i, v); else sum_of(i, v);
#pragma unroll
        for (int j = 0; j < KV; ++j) v[j] = v[j] * rstd * a.gamma[i + j];
        if (a.y) Elem<TX>::store_vec(a.y + row + i, v);
        if (a.q) store_mx8<KV>(v, a.q, a.q_scale, row + i);
    }
}

template <typename TX> struct NormBwdArgs {
    const TX* dy;
    const TX* dh;             // or null
    const TX* h;
    const float* gamma;
    const float* rstd;
    TX* dx;
    float* part;              // [parts][d], or null
    int T, d, parts;
};

// dgamma, a range of rows for each blockIdx.y: part[range][j] = sum of dy_tj h_tj rstd_t.  Before dx, which may overwrite dy.
template <typename TX>
__global__ __launch_bounds__(256) void rmsnorm_dgamma_kernel(NormBwdArgs<TX> a)
{
    constexpr int KV = Elem<TX>::kVec;
    const int i = (blockIdx.x * 256 + threadIdx.x) * KV;
    if (i >= a.d) return;
    const int per = (a.T + a.parts - 1) / a.parts, t0 = blockIdx.y * per, t1 = min(a.T, t0 + per);
    float acc[KV] = {};
    for (int t = t0; t < t1; ++t) {
        float dy[KV], h[KV];
        Elem<TX>::load_vec(a.dy + (int64_t)t * a.d + i, dy);
        Elem<TX>::load_vec(a.h + (int64_t)t * a.d + i, h);
#pragma unroll
        for (int j = 0; j < KV; ++j) acc[j] += dy[j] * (h[j] * a.rstd[t]);
    }
#pragma unroll
    for (int j = 0; j < KV; ++j) a.part[(size_t)blockIdx.y * a.d + i + j] = acc[j];
}

// One block per row.
template <typename TX>
__global__ __launch_bounds__(256) void rmsnorm_dx_kernel(NormBwdArgs<TX> a)
{
    constexpr int KV = Elem<TX>::kVec;
    __shared__ float red[4];
    const int64_t row = (int64_t)blockIdx.x * a.d;
    const float rstd = a.rstd[blockIdx.x];
    float inner = 0.f;
    for (int i = threadIdx.x * KV; i < a.d; i += 256 * KV) {
        float dy[KV], h[KV];
        Elem<TX>::load_vec(a.dy + row + i, dy);
        Elem<TX>::load_vec(a.h + row + i, h);
#pragma unroll
        for (int j = 0; j < KV; ++j) inner += a.gamma[i + j] * dy[j] * (h[j] * rstd);
    }
    inner = block_sum(inner, red) / a.d;
    for (int i = threadIdx.x * KV; i < a.d; i += 256 * KV) {
        float dy[KV], h[KV], dh[KV] = {};
        Elem<TX>::load_vec(a.dy + row + i, dy);
        Elem<TX>::load_vec(a.h + row + i, h);
        if (a.dh) Elem<TX>::load_vec(a.dh + row + i, dh);
#pragma unroll
        for (int j = 0; j < KV; ++j) dh[j] += rstd * (a.gamma[i + j] * dy[j] - h[j] * rstd * inner);
        Elem<TX>::store_vec(a.dx + row + i, dh);
    }
}

int dgamma_parts(const evomoe_shape& s) { const int n = (s.T + 15) / 16; return n < 256 ? n : 256; }

// A matrix as one run of vectors: rows are whole groups, so that a group never crosses one.
template <typename TX>
__global__ __launch_bounds__(256) void quantize_mx8_kernel(const TX* __restrict__ src, int64_t n, uint8_t* __restrict__ q,
                                                           uint8_t* __restrict__ scale)
{
    constexpr int KV = Elem<TX>::kVec;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * KV; i < n; i += (int64_t)gridDim.x * 256 * KV) {
        float v[KV];
        Elem<TX>::load_vec(src + i, v);
        store_mx8<KV>(v, q, scale, i);
    }
}

template <typename TX>
hipError_t add_rmsnorm_t(const Ctx& c, const evomoe_shape& s, const void* x, const void* residual, const float* gamma,
                         float eps, void* h, void* y, float* rstd, void* q, uint8_t* q_scale) {
    const NormArgs<TX> a{(const TX*)x, (const TX*)residual, gamma, (TX*)h, (TX*)y, rstd, (uint8_t*)q, q_scale, eps, s.T, s.d};
    hipLaunchKernelGGL(add_rmsnorm_kernel<TX>, dim3(s.T), dim3(256), 0, c.stream, a);
    return hipGetLastError();
}

template <typename TX>
hipError_t add_rmsnorm_bwd_t(const Ctx& c, const evomoe_shape& s, const void* dy, const void* dh, const void* h,
                             const float* gamma, const float* rstd, void* dx, float* dgamma, void* workspace) {
    const NormBwdArgs<TX> a{(const TX*)dy, (const TX*)dh, (const TX*)h, gamma, rstd, (TX*)dx, (float*)workspace, s.T, s.d,
                            dgamma_parts(s)};
    if (dgamma) {
        const int cols = 256 * Elem<TX>::kVec;
        hipLaunchKernelGGL(rmsnorm_dgamma_kernel<TX>, dim3((s.d + cols - 1) / cols, a.parts), dim3(256), 0, c.stream, a);
        hipError_t err = hipGetLastError();
        if (err == hipSuccess) err = launch_sum_rows(c, a.part, a.parts, s.d, dgamma);
        if (err != hipSuccess) return err;
    }
    hipLaunchKernelGGL(rmsnorm_dx_kernel<TX>, dim3(s.T), dim3(256), 0, c.stream, a);
    return hipGetLastError();
}

}  // namespace

size_t rmsnorm_bwd_workspace_bytes(const evomoe_shape& s) { return (size_t)dgamma_parts(s) * s.d * sizeof(float); }

hipError_t launch_add_rmsnorm(const Ctx& c, const evomoe_shape& s, const void* x, const void* residual,
                              const float* gamma, float eps, void* h, void* y, float* rstd, void* q, uint8_t* q_scale) {
    ProfScope ps(c, EVOMOE_K_ADD_RMSNORM);
    return s.dtype == EVOMOE_BF16 ? add_rmsnorm_t<bf16_t>(c, s, x, residual, gamma, eps, h, y, rstd, q, q_scale)
                                  : add_rmsnorm_t<float>(c, s, x, residual, gamma, eps, h, y, rstd, q, q_scale);
}

hipError_t launch_add_rmsnorm_bwd(const Ctx& c, const evomoe_shape& s, const void* dy, const void* dh, const void* h,
                                  const float* gamma, const float* rstd, void* dx, float* dgamma, void* workspace) {
    ProfScope ps(c, EVOMOE_K_ADD_RMSNORM_BWD);
    return s.dtype == EVOMOE_BF16 ? add_rmsnorm_bwd_t<bf16_t>(c, s, dy, dh, h, gamma, rstd, dx, dgamma, workspace)
                                  : add_rmsnorm_bwd_t<float>(c, s, dy, dh, h, gamma, rstd, dx, dgamma, workspace);
}

hipError_t launch_quantize_mx8(const Ctx& c, int64_t rows, int64_t cols, int dtype, const void* src, void* q,
                               uint8_t* q_scale) {
    ProfScope ps(c, EVOMOE_K_QUANTIZE_MX8);
    const int64_t n = rows * cols, want = (n / (dtype == EVOMOE_BF16 ? 8 : 4) + 255) / 256, cap = (int64_t)c.num_cu * 16;
    const dim3 grid((unsigned)(want < cap ? want : cap));
    if (dtype == EVOMOE_BF16)
        hipLaunchKernelGGL(quantize_mx8_kernel<bf16_t>, grid, dim3(256), 0, c.stream, (const bf16_t*)src, n, (uint8_t*)q, q_scale);
    else
        hipLaunchKernelGGL(quantize_mx8_kernel<float>, grid, dim3(256), 0, c.stream, (const float*)src, n, (uint8_t*)q, q_scale);
    return hipGetLastError();
}

}  // namespace evomoe
