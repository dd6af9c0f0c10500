// Residual addition with the root-mean-square norm, forward (to the layer's type and to 8 bits) and backward, and the conversion of
// a matrix to 8 bits.  All of it is reading and writing rows.
#include <algorithm>
#include <type_traits>

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

// gamma's KV values from column i on, 0 beyond d
template <int KV> __device__ __forceinline__ void load_gamma(const float* gamma, int i, int d, float (&out)[KV]) {
#pragma unroll
    for (int j = 0; j < KV; j += 4) {
        const f32x4 v = i < d ? *reinterpret_cast<const f32x4*>(gamma + i + j) : f32x4{0.f, 0.f, 0.f, 0.f};
        out[j] = v.x; out[j + 1] = v.y; out[j + 2] = v.z; out[j + 3] = v.w;
    }
}

// One wave per row, the row in registers: NV vectors a lane, lane l's k-th at 64 k + l.  Every byte is moved once, and no wave
// waits for another.  (Outputs may be inputs: a row is written after the same wave has read it.)
template <typename TX, int NV>
__global__ __launch_bounds__(256) void add_rmsnorm_wave_kernel(NormArgs<TX> a)
{
    constexpr int KV = Elem<TX>::kVec;
    constexpr bool KEEP = NV * KV <= 32;                    // gamma stays in registers over a wave's rows
    const int lane = threadIdx.x & 63;
    float gamma[KEEP ? NV : 1][KV];
    if (KEEP) {
#pragma unroll
        for (int k = 0; k < NV; ++k) load_gamma(a.gamma, (64 * k + lane) * KV, a.d, gamma[KEEP ? k : 0]);
    }
    for (int t = blockIdx.x * 4 + (threadIdx.x >> 6); t < a.T; t += gridDim.x * 4) {
        const int64_t row = (int64_t)t * a.d;
        float v[NV][KV], r[NV][KV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int i = (64 * k + lane) * KV;
#pragma unroll
            for (int j = 0; j < KV; ++j) v[k][j] = r[k][j] = 0.f;
            if (i < a.d) {
                Elem<TX>::load_vec(a.x + row + i, v[k]);
                if (a.residual) Elem<TX>::load_vec(a.residual + row + i, r[k]);
            }
        }
        float ss = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int i = (64 * k + lane) * KV;
            if (a.residual) {
#pragma unroll
                for (int j = 0; j < KV; ++j) v[k][j] = (float)(TX)(v[k][j] + r[k][j]);      // h, as it is stored
            }
            if (a.h && i < a.d) Elem<TX>::store_vec(a.h + row + i, v[k]);
#pragma unroll
            for (int j = 0; j < KV; ++j) ss += v[k][j] * v[k][j];
        }
        const float rstd = 1.f / sqrtf(wave_sum(ss) / a.d + a.eps);
        if (a.rstd && lane == 0) a.rstd[t] = rstd;
        if (!a.y && !a.q) continue;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int i = (64 * k + lane) * KV;
            if (i >= a.d) continue;
            if (!KEEP) load_gamma(a.gamma, i, a.d, gamma[0]);
#pragma unroll
            for (int j = 0; j < KV; ++j) v[k][j] = v[k][j] * rstd * gamma[KEEP ? k : 0][j];
            if (a.y) Elem<TX>::store_vec(a.y + row + i, v[k]);
            if (a.q) store_mx8<KV>(v[k], a.q, a.q_scale, row + i);
        }
    }
}

// Rows that do not fit a wave's registers: one block per row at a time, which reads h (or x and the residual) a second time.
template <typename TX>
__global__ __launch_bounds__(256) void add_rmsnorm_block_kernel(NormArgs<TX> a)
{
    constexpr int KV = Elem<TX>::kVec;
    __shared__ float red[4];
    for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
        const int64_t row = (int64_t)t * a.d;
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
        if (a.rstd && threadIdx.x == 0) a.rstd[t] = rstd;
        if (!a.y && !a.q) continue;
        for (int i = threadIdx.x * KV; i < a.d; i += 256 * KV) {
            float v[KV];
            if (a.h) Elem<TX>::load_vec(a.h + row + i, v); else sum_of(i, v);
#pragma unroll
            for (int j = 0; j < KV; ++j) v[j] = v[j] * rstd * a.gamma[i + j];
            if (a.y) Elem<TX>::store_vec(a.y + row + i, v);
            if (a.q) store_mx8<KV>(v, a.q, a.q_scale, row + i);
        }
    }
}

// A vector of 16 bytes -> its elements
template <typename TX> __device__ __forceinline__ void unpack(u32x4 v, float (&out)[Elem<TX>::kVec]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (std::is_same<TX, bf16_t>::value) { out[2 * j] = lo_bf16(v[j]); out[2 * j + 1] = hi_bf16(v[j]); }
        else out[j] = __uint_as_float(v[j]);
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

// dx and dgamma in one pass.  One wave per row as in the forward; a lane meets the same columns in every row, so that it adds up its share
// of dgamma in registers over all rows of its wave.  The block's NW waves meet in the LDS, in wave order, and leave one row of partial
// sums, which a second launch adds in block order.  (dx may be dy or dh: see the forward.)
template <typename TX, int NV, int NW>
__global__ __launch_bounds__(NW * 64) void rmsnorm_bwd_wave_kernel(NormBwdArgs<TX> a)
{
    constexpr int KV = Elem<TX>::kVec;
    constexpr bool KEEP = NV * KV <= 16;
    __shared__ float sums[NW / 2][64 * KV];                // (one vector of every lane at a time)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float acc[NV][KV] = {}, gamma[KEEP ? NV : 1][KV];
    if (KEEP) {
#pragma unroll
        for (int k = 0; k < NV; ++k) load_gamma(a.gamma, (64 * k + lane) * KV, a.d, gamma[KEEP ? k : 0]);
    }
    for (int t = blockIdx.x * NW + wave; t < a.T; t += gridDim.x * NW) {
        const int64_t row = (int64_t)t * a.d;
        const float rstd = a.rstd[t];
        u32x4 dy[NV], h[NV], dh[NV];                        // as they are stored
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int i = (64 * k + lane) * KV;
            dy[k] = h[k] = dh[k] = u32x4{0u, 0u, 0u, 0u};
            if (i < a.d) {
                dy[k] = *reinterpret_cast<const u32x4*>(a.dy + row + i);
                h[k] = *reinterpret_cast<const u32x4*>(a.h + row + i);
                if (a.dh) dh[k] = *reinterpret_cast<const u32x4*>(a.dh + row + i);
            }
        }
        auto of = [&](int k, float (&d)[KV], float (&n)[KV], float (&g)[KV]) {        // dy, n, gamma
            const int i = (64 * k + lane) * KV;
            unpack<TX>(dy[k], d);
            unpack<TX>(h[k], n);
            if (!KEEP) load_gamma(a.gamma, i, a.d, gamma[0]);
#pragma unroll
            for (int j = 0; j < KV; ++j) {
                n[j] *= rstd;
                g[j] = gamma[KEEP ? k : 0][j];
            }
        };
        float inner = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float d[KV], n[KV], g[KV];
            of(k, d, n, g);
#pragma unroll
            for (int j = 0; j < KV; ++j) {
                acc[k][j] += d[j] * n[j];
                inner += g[j] * d[j] * n[j];
            }
        }
        inner = wave_sum(inner) / a.d;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int i = (64 * k + lane) * KV;
            if (i >= a.d) continue;
            float d[KV], n[KV], g[KV], out[KV];
            of(k, d, n, g);
            unpack<TX>(dh[k], out);
#pragma unroll
            for (int j = 0; j < KV; ++j) out[j] += rstd * (g[j] * d[j] - n[j] * inner);
            Elem<TX>::store_vec(a.dx + row + i, out);
        }
    }
    if (!a.part) return;
    // the upper half of the waves hand over to the lower half, until one is left: a tree in a fixed order
#pragma unroll
    for (int k = 0; k < NV; ++k)
        for (int half = NW / 2; half >= 1; half >>= 1) {
            __syncthreads();
            if (wave >= half && wave < 2 * half) {
#pragma unroll
                for (int j = 0; j < KV; ++j) sums[wave - half][j * 64 + lane] = acc[k][j];
            }
            __syncthreads();
            if (wave < half) {
#pragma unroll
                for (int j = 0; j < KV; ++j) acc[k][j] += sums[wave][j * 64 + lane];
            }
        }
    if (wave > 0) return;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int i = (64 * k + lane) * KV;
        if (i >= a.d) continue;
#pragma unroll
        for (int j = 0; j < KV; ++j) a.part[(size_t)blockIdx.x * a.d + i + j] = acc[k][j];
    }
}

// Rows that do not fit a wave's registers.  dgamma, a range of rows for each blockIdx.y: part[range][j] = sum of dy_tj h_tj rstd_t; before
// dx, which may overwrite dy.
template <typename TX>
__global__ __launch_bounds__(256) void rmsnorm_dgamma_kernel(NormBwdArgs<TX> a)
{
    constexpr int KV = Elem<TX>::kVec;
    const int i = (blockIdx.x * 256 + threadIdx.x) * KV;
    if (i >= a.d) return;
    const int per = (a.T + a.parts - 1) / a.parts;
    const int64_t t0 = (int64_t)blockIdx.y * per, t1 = min((int64_t)a.T, t0 + per);
    float acc[KV] = {};
    for (int64_t t = t0; t < t1; ++t) {
        float dy[KV], h[KV];
        Elem<TX>::load_vec(a.dy + t * a.d + i, dy);
        Elem<TX>::load_vec(a.h + t * a.d + i, h);
#pragma unroll
        for (int j = 0; j < KV; ++j) acc[j] += dy[j] * (h[j] * a.rstd[t]);
    }
#pragma unroll
    for (int j = 0; j < KV; ++j) a.part[(size_t)blockIdx.y * a.d + i + j] = acc[j];
}
// ... and dx, one block per row at a time.
template <typename TX>
__global__ __launch_bounds__(256) void rmsnorm_dx_kernel(NormBwdArgs<TX> a)
{
    constexpr int KV = Elem<TX>::kVec;
    __shared__ float red[4];
    for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
        const int64_t row = (int64_t)t * a.d;
        const float rstd = a.rstd[t];
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
}

// dgamma = the partial rows' sum.  Sixteen threads to a column, sixteen rows each at most (kParts), whose loads are all on their way at once;
// their sums are added in order.  A block has 64 columns at a time: a block for every 64 up to kSumBlocks (a grid dimension holds fewer
// than 2^32 threads).
constexpr int kParts = 256, kSumBlocks = 1 << 20;
__global__ __launch_bounds__(1024) void dgamma_sum_kernel(const float* __restrict__ part, int parts, int d, float* __restrict__ dgamma)
{
    __shared__ float sums[16][64];
    const int o = threadIdx.x & 63, grp = threadIdx.x >> 6, per = (parts + 15) / 16;
    for (int i0 = blockIdx.x * 64; i0 < d; i0 += gridDim.x * 64) {       // (d up to 2^30, a step up to 2^26)
        const int i = i0 + o;
        float v[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const int r = grp * per + u;
            v[u] = u < per && r < parts && i < d ? part[(size_t)r * d + i] : 0.f;
        }
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < 16; ++u) s += v[u];
        sums[grp][o] = s;
        __syncthreads();
        if (grp == 0 && i < d) {
#pragma unroll
            for (int g = 1; g < 16; ++g) s += sums[g][o];
            dgamma[i] = s;
        }
        __syncthreads();                             // (the sums have been read)
    }
}

// Rows of partial sums of dgamma: blocks of the one-pass kernel (sixteen rows each at least), or ranges of rows.
int dgamma_parts(const evomoe_shape& s) { const int n = (s.T + 15) / 16; return n < kParts ? n : kParts; }

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

// calls f with the vectors per lane of a wave that holds a row, as a constant; false if a row does not fit MOST of them
template <typename TX, int MOST, class F> bool with_vectors(int d, F&& f) {
    const int n = (d / Elem<TX>::kVec + 63) / 64;
    bool done = false;
    auto with = [&](auto nv) {
        if constexpr (decltype(nv)::value <= MOST)
            if (!done && n <= decltype(nv)::value) { f(nv); done = true; }
    };
    with(std::integral_constant<int, 1>{});
    with(std::integral_constant<int, 2>{});
    with(std::integral_constant<int, 3>{});
    with(std::integral_constant<int, 4>{});
    with(std::integral_constant<int, 6>{});
    with(std::integral_constant<int, 8>{});
    with(std::integral_constant<int, 16>{});
    return done;
}

template <typename TX>
hipError_t add_rmsnorm_t(const Ctx& c, const evomoe_shape& s, const void* x, const void* residual, const float* gamma,
                         float eps, void* h, void* y, float* rstd, void* q, uint8_t* q_scale) {
    const NormArgs<TX> a{(const TX*)x, (const TX*)residual, gamma, (TX*)h, (TX*)y, rstd, (uint8_t*)q, q_scale, eps, s.T, s.d};
    const int blocks = std::min((s.T + 3) / 4, c.num_cu * 8);
    if (!with_vectors<TX, 64 / Elem<TX>::kVec>(s.d, [&](auto nv) {
            hipLaunchKernelGGL((add_rmsnorm_wave_kernel<TX, decltype(nv)::value>), dim3(blocks), dim3(256), 0, c.stream, a);
        }))
        hipLaunchKernelGGL(add_rmsnorm_block_kernel<TX>, dim3(std::min(s.T, c.num_cu * 8)), dim3(256), 0, c.stream, a);
    return hipGetLastError();
}

template <typename TX>
hipError_t add_rmsnorm_bwd_t(const Ctx& c, const evomoe_shape& s, const void* dy, const void* dh, const void* h,
                             const float* gamma, const float* rstd, void* dx, float* dgamma, void* workspace) {
    constexpr int KV = Elem<TX>::kVec;
    const NormBwdArgs<TX> a{(const TX*)dy, (const TX*)dh, (const TX*)h, gamma, rstd, (TX*)dx, dgamma ? (float*)workspace : nullptr,
                            s.T, s.d, dgamma_parts(s)};
    auto sum_up = [&] {
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess || !dgamma) return err;
        hipLaunchKernelGGL(dgamma_sum_kernel, dim3(std::min((s.d + 63) / 64, kSumBlocks)), dim3(1024), 0, c.stream, a.part, a.parts, s.d, dgamma);
        return hipGetLastError();
    };
    if (with_vectors<TX, 64 / KV>(s.d, [&](auto nv) {
            constexpr int NV = decltype(nv)::value, NW = NV * KV <= 16 ? 16 : NV * KV <= 32 ? 8 : 4;
            hipLaunchKernelGGL((rmsnorm_bwd_wave_kernel<TX, NV, NW>), dim3(a.parts), dim3(NW * 64), 0, c.stream, a);
        }))
        return sum_up();
    if (dgamma) {
        const int cols = 256 * KV;
        hipLaunchKernelGGL(rmsnorm_dgamma_kernel<TX>, dim3((s.d + cols - 1) / cols, a.parts), dim3(256), 0, c.stream, a);
        if (const hipError_t err = sum_up(); err != hipSuccess) return err;
    }
    hipLaunchKernelGGL(rmsnorm_dx_kernel<TX>, dim3(std::min(s.T, c.num_cu * 8)), dim3(256), 0, c.stream, a);
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
