// Expert FFNs forward in 8 bits (e4m3 elements, a power of two scale for 32 of them along the contraction), on the scaled
// matrix instructions:
//   A = act(X W1^T + b1), to 8 bits again;     O = A W2^T + b2, bf16.
//
// Both products are computed transposed, C^T[n,r] = sum_k W[n,k] X[r,k]: the weights' rows are the matrix instruction's rows,
// and a lane of the result holds consecutive columns n of ONE row r, so that a group of 32 columns of A lies in a few
// lanes' registers and is converted without a detour through the LDS.
//
// How exact the sums are is the matrix instructions' property, of the scaled one as of the plain ones for 8-bit values: the products of eight
// neighbouring k's, 8 i .. 8 i + 7, are cut off, towards zero, below 2^-13 of 2^(the largest sum of their two factors' exponents) and added
// exactly; only what comes of each eight enters sums with float32's roundings.  In 8-bit products that cut is chosen with the
// elements, whose own rounding is 2^-4: sums without it would need products in 16 bits, at half the rate.  An act(H) whose rounding to 8
// bits is close may so become the neighbouring value: over the experts of the GPT-shaped and the large layer O's error against
// 64 bits is 0.0018 to 0.0019 of its size, with float32 sums 0.0017, which is the rounding of O to bf16.
#include <type_traits>

#include "ffn_internal.h"
#include "mfma_tools.h"
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

// gelu(h) = max(h, 0) - x 2^p(x), x = |h|: 2^p is Phi(-x), p of degree five fitted for the least largest error of the product.  For every
// finite h (p falls to -inf) the value is within 4.7e-7 and half a float32 step of itself of the exact one, 6.4e-7 at most (near h = 4).
// Ten VALU instructions and an exponential.
__device__ __forceinline__ float gelu5(float h) {
    const float x = fabsf(h);
    float p = -0.000473309294f;
    p = fmaf(p, x, 0.00708455719f);
    p = fmaf(p, x, -0.0518273829f);
    p = fmaf(p, x, -0.459992439f);
    p = fmaf(p, x, -1.15078785f);
    p = fmaf(p, x, -1.00003762f);
    return fmaf(-x, __builtin_amdgcn_exp2f(p), fmaxf(h, 0.f));       // (of a NaN the exponential is one)
}

// v_mfma_scale_f32_32x32x64_f8f6f4: lane (h = lane / 32, i = lane % 32) brings the k's 16 h .. 16 h + 15 and 32 + 16 h .. of row i of
// either operand, and the scale of that row's k's 32 h .. 32 h + 31 in byte `OP` of sa, sb; it receives, of column i, the rows
// 8 (r / 4) + 4 h + r % 4, r = 0 .. 15.
template <int OP> __device__ __forceinline__ f32x16 mfma32(i32x8 a, i32x8 b, f32x16 c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, OP, sa, OP, sb);
}

// Exchanges the upper half of a with the lower half of b.
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
    const auto v = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = v[0];
    b = v[1];
}

// EPI: what becomes of the sums.
enum { TO_RELU = EVOMOE_RELU, TO_GELU = EVOMOE_GELU_ERF, TO_OUTPUT };

// Few rows for an expert: what counts is how fast its weights arrive.  A block takes 32 rows by 32 columns and its four waves deal the
// slabs of 128 k's among them, each straight from memory into the matrix instruction's registers, DEPTH slabs (8 loads of 1 KB each) in
// flight; the waves' sums meet in the LDS.  K may be any multiple of 32: what lies beyond it is 0.
template <int EPI, int DEPTH>
__global__ __launch_bounds__(256) void mx8_few_rows_kernel(Mx8Args p)
{
    constexpr int LD = 33;
    __shared__ float sums[4][32][LD];
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5, wave = threadIdx.x >> 6;
    // lane e: expert e's rows, and the row tiles up to it
    const int begin = clamp_pairs(p.expert_offsets[min(lane, p.E)], p.P_cap),
              end = clamp_pairs(p.expert_offsets[min(lane + 1, p.E)], p.P_cap);
    int upto = (end - begin + 31) / 32;
    const int mine = upto;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(upto, o, 64);
        if (lane >= o) upto += v;
    }
    const int kg = p.K / kMxGroup, nct = p.N / 32;
    const int64_t tiles = (int64_t)__builtin_amdgcn_readlane(upto, 63) * nct;
    for (int64_t at = blockIdx.x; at < tiles; at += gridDim.x) {
        const int tile = (int)(at / nct), n0 = (int)(at - (int64_t)tile * nct) * 32, g = __popcll(__ballot(upto <= tile));
        const int row0 = __builtin_amdgcn_readlane(begin, g) + (tile - __builtin_amdgcn_readlane(upto - mine, g)) * 32;
        const int rows = min(32, __builtin_amdgcn_readlane(end, g) - row0);
        const int xr = row0 + min(l32, rows - 1);
        const int64_t wrow = (int64_t)g * p.N + n0 + l32;
        const uint8_t *w = p.W + wrow * p.K, *ws = p.Ws + wrow * kg;
        const int token = p.rows ? p.rows[xr] : xr;
        __builtin_amdgcn_sched_barrier(0);       // (the first weights are on their way before anything waits for the row number)
        f32x16 acc = {};
        const u32x4 zero = {};
        for (int s0 = wave; s0 * 128 < p.K; s0 += 4 * DEPTH) {
            u32x4 wv[DEPTH][4], xv[DEPTH][4];
            int wsc[DEPTH][2], xsc[DEPTH][2];
            auto load = [&](const uint8_t* row, const uint8_t* scale, u32x4 (&v)[DEPTH][4], int (&sc)[DEPTH][2]) {
#pragma unroll
                for (int u = 0; u < DEPTH; ++u)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int k = (s0 + 4 * u) * 128 + c * 32 + half * 16;
                        v[u][c] = k < p.K ? *reinterpret_cast<const u32x4*>(row + k) : zero;
                    }
#pragma unroll
                for (int u = 0; u < DEPTH; ++u)
#pragma unroll
                    for (int ks = 0; ks < 2; ++ks) {
                        const int i = (s0 + 4 * u) * 4 + 2 * ks + half;
                        sc[u][ks] = i < kg ? scale[i] : 127;
                    }
                __builtin_amdgcn_sched_barrier(0);
            };
            load(w, ws, wv, wsc);
            load(p.X + (int64_t)token * p.K, p.Xs + (int64_t)token * kg, xv, xsc);
#pragma unroll
            for (int u = 0; u < DEPTH; ++u)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    auto eight = [](u32x4 lo, u32x4 hi) {
                        return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
                    };
                    acc = mfma32<0>(eight(wv[u][2 * ks], wv[u][2 * ks + 1]), eight(xv[u][2 * ks], xv[u][2 * ks + 1]), acc, wsc[u][ks], xsc[u][ks]);
                }
        }
        asm volatile("" : "+v"(acc));       // (not to be moved under a branch: see the tile kernel's epilogue)
#pragma unroll
        for (int r = 0; r < 16; ++r) sums[wave][8 * (r >> 2) + 4 * half + (r & 3)][l32] = acc[r];
        __syncthreads();
        // eight threads to a row, four columns each; the waves' sums in wave order
        const int row = threadIdx.x >> 3, n4 = (threadIdx.x & 7) * 4;
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = ((sums[0][n4 + j][row] + sums[1][n4 + j][row]) + sums[2][n4 + j][row]) + sums[3][n4 + j][row];
            if (p.bias) v[j] += p.bias[(int64_t)g * p.N + n0 + n4 + j];
            if (EPI == TO_RELU) v[j] = relu(v[j]);
            if (EPI == TO_GELU) v[j] = gelu5(v[j]);
        }
        if constexpr (EPI == TO_OUTPUT) {
            if (row < rows)
                *reinterpret_cast<u32x2*>(p.O + (int64_t)(row0 + row) * p.N + n0 + n4) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        } else {
            float m = mx_max(v);
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
            const uint32_t b = mx_scale_byte(m);
            if (row < rows) {
                *reinterpret_cast<uint32_t*>(p.Aq + (int64_t)(row0 + row) * p.N + n0 + n4) = mx_pack4(v[0], v[1], v[2], v[3], b);
                if (n4 == 0) p.As[(int64_t)(row0 + row) * (p.N / kMxGroup) + n0 / kMxGroup] = (uint8_t)b;
            }
        }
        __syncthreads();         // (the sums have been read)
    }
}

// Any multiples of 32 for K and N, many rows: tiles of 128x128, four waves of 64x64, through registers into the LDS, one slab of 128 k's
// ahead, two blocks to a CU.  What lies beyond K is 0 with a scale of 1; columns beyond N repeat the last ones and are not stored.  Scales are read
// byte by byte, as a row of them begins anywhere.  The LDS layout is the tile kernel's (below).
template <int EPI>
__global__ __launch_bounds__(256, 2) void mx8_any_size_kernel(Mx8Args p)
{
    constexpr bool FIRST = EPI != TO_OUTPUT;
    __shared__ __align__(16) unsigned char data[2][256 * 128];           // 128 rows of X, then 128 of W
    __shared__ uint32_t scales[2][256];
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wx = wave >> 1, ww = wave & 1;
    // lane e: expert e's rows, and the row tiles up to it
    const int begin = clamp_pairs(p.expert_offsets[min(lane, p.E)], p.P_cap),
              end = clamp_pairs(p.expert_offsets[min(lane + 1, p.E)], p.P_cap);
    int upto = (end - begin + 127) / 128;
    const int mine = upto;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(upto, o, 64);
        if (lane >= o) upto += v;
    }
    const int kg = p.K / kMxGroup, nct = (p.N + 127) / 128, nslab = (p.K + 127) / 128;
    const int64_t tiles = (int64_t)__builtin_amdgcn_readlane(upto, 63) * nct;
    for (int64_t at = blockIdx.x; at < tiles; at += gridDim.x) {
        const int tile = (int)(at / nct), n0 = (int)(at - (int64_t)tile * nct) * 128, g = __popcll(__ballot(upto <= tile));
        const int row0 = __builtin_amdgcn_readlane(begin, g) + (tile - __builtin_amdgcn_readlane(upto - mine, g)) * 128;
        const int rows = min(128, __builtin_amdgcn_readlane(end, g) - row0);
        auto x_row = [&](int r) {
            const int at_row = row0 + min(r, rows - 1);
            return (int64_t)(p.rows ? p.rows[at_row] : at_row);
        };
        auto w_row = [&](int r) { return (int64_t)g * p.N + min(n0 + r, p.N - 1); };
        // this thread's part of a slab: chunk c16 of the rows r8, r8 + 32, .. of X and of W, and the scales of one row
        const int r8 = threadIdx.x >> 3, c16 = threadIdx.x & 7, sr = threadIdx.x & 127;
        const uint8_t* from[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            from[i] = p.X + x_row(r8 + 32 * i) * p.K;
            from[4 + i] = p.W + w_row(r8 + 32 * i) * p.K;
        }
        const uint8_t* scale_from = threadIdx.x < 128 ? p.Xs + x_row(sr) * kg : p.Ws + w_row(sr) * kg;
        u32x4 next[8];
        uint32_t next_scale;
        auto load = [&](int s) {
            const int k = s * 128 + c16 * 16;
#pragma unroll
            for (int i = 0; i < 8; ++i) next[i] = k < p.K ? *reinterpret_cast<const u32x4*>(from[i] + k) : u32x4{0u, 0u, 0u, 0u};
            next_scale = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) next_scale |= (uint32_t)(s * 4 + j < kg ? scale_from[s * 4 + j] : 127) << (8 * j);
        };
        auto put = [&](int s) {
            unsigned char* to = data[s & 1];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = r8 + 32 * (i & 3);
                *reinterpret_cast<u32x4*>(to + ((i >> 2) * 128 + r) * 128 + ((c16 ^ (r >> 1 & 7)) << 4)) = next[i];
            }
            scales[s & 1][threadIdx.x] = next_scale;
        };
        f32x16 acc[2][2] = {};
        load(0);
        put(0);
        __syncthreads();
        for (int s = 0; s < nslab; ++s) {
            if (s + 1 < nslab) load(s + 1);
            const unsigned char* st = data[s & 1];
            const uint32_t* sc = scales[s & 1];
            const int key = l32 >> 1 & 7;
            auto fragment = [&](int row, int ks) {
                const u32x4 lo = *reinterpret_cast<const u32x4*>(st + row * 128 + (((ks * 4 + half) ^ key) << 4));
                const u32x4 hi = *reinterpret_cast<const u32x4*>(st + row * 128 + (((ks * 4 + 2 + half) ^ key) << 4));
                return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
            };
            int sx[2], sw[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                sx[i] = (int)(sc[(wx * 2 + i) * 32 + l32] >> (8 * half));
                sw[i] = (int)(sc[128 + (ww * 2 + i) * 32 + l32] >> (8 * half));
            }
            auto kstep = [&](auto op, int ks) {
                i32x8 x[2], w[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    x[i] = fragment((wx * 2 + i) * 32 + l32, ks);
                    w[i] = fragment(128 + (ww * 2 + i) * 32 + l32, ks);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = mfma32<decltype(op)::value>(w[i], x[j], acc[i][j], sw[i], sx[j]);
            };
            kstep(std::integral_constant<int, 0>{}, 0);
            kstep(std::integral_constant<int, 2>{}, 1);
            if (s + 1 < nslab) put(s + 1);           // (its last readers passed the barrier before this slab)
            __syncthreads();
        }
        // lane = row, registers = columns, as in the tile kernel
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int n = n0 + (ww * 2 + i) * 32;                    // N is a multiple of 32
            const uint32_t beyond = n < p.N ? 0u : 0x40000000u;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r0 = (wx * 2 + j) * 32, there = min(32, max(0, rows - r0));
                const int64_t first = (int64_t)(row0 + r0);
                asm volatile("" : "+v"(acc[i][j]));
                float v[16];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 b = p.bias && n < p.N ? *reinterpret_cast<const f32x4*>(p.bias + (int64_t)g * p.N + n + 8 * q + 4 * half) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[4 * q + r] = acc[i][j][4 * q + r] + b[r];
                }
                if constexpr (FIRST) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) v[r] = EPI == TO_RELU ? relu(v[r]) : gelu5(v[r]);
                    uint32_t ma = __float_as_uint(mx_max(v)), mb = ma;
                    swap_halves(ma, mb);
                    const uint32_t b = mx_scale_byte(fmaxf(__uint_as_float(ma), __uint_as_float(mb)));
                    uint32_t d[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) d[q] = mx_pack4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3], b);
                    swap_halves(d[0], d[2]);
                    swap_halves(d[1], d[3]);
                    __builtin_amdgcn_raw_buffer_store_b128(u32x4{d[0], d[2], d[1], d[3]}, rows_of(p.Aq + first * p.N, there * p.N),
                                                           (l32 * p.N + n + 16 * half) | beyond, 0, 0);
                    const int ng = p.N / kMxGroup;
                    __builtin_amdgcn_raw_buffer_store_b8((uint8_t)b, rows_of(p.As + first * ng, there * ng),
                                                         half ? 0x40000000 : (int)((l32 * ng + n / kMxGroup) | beyond), 0, 0);
                } else {
                    uint32_t d[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q) d[q] = pack_bf16x2(v[2 * q], v[2 * q + 1]);
                    swap_halves(d[0], d[4]); swap_halves(d[1], d[5]); swap_halves(d[2], d[6]); swap_halves(d[3], d[7]);
                    const auto to = rows_of(p.O + first * p.N, there * p.N * 2);
                    const uint32_t off = ((l32 * p.N + n + 16 * half) * 2) | beyond;
                    __builtin_amdgcn_raw_buffer_store_b128(u32x4{d[0], d[1], d[4], d[5]}, to, off, 0, 0);
                    __builtin_amdgcn_raw_buffer_store_b128(u32x4{d[2], d[3], d[6], d[7]}, to, off + 16, 0, 0);
                }
            }
        }
    }
}

// The tile kernel, for d and F that are multiples of 128.  A block of WX x WW waves computes BX rows of X by BW rows of W, a
// wave TX x TW matrix instructions of 32 x 32.  The contraction runs in slabs of 128 bytes (one line of every row), two LDS stages
// deep; a stage holds both operands' slabs, rows of 128 bytes with the 16-byte chunk c of row r at chunk c ^ (r >> 1 & 7), so that
// sixteen lanes' reads of one chunk column meet all banks.  Scales come for four slabs at a time, 16 bytes of a row (with the loads of
// the first of them), as every row lies in another line: slab by slab, 4 bytes of a row, they took as long as half of the data (65536 pairs, one
// expert, d = 1024, F = 4096: second product 290 us, without loading scales 253).  Loads go straight to the LDS.
// Slab s + 2 is fetched into slab s's stage as soon as its last fragments are in registers, and lands while one and a half
// slabs multiply.  Blocks are persistent and walk the tiles as the bf16 kernels do: expert by expert, column group by column
// group, row tile by row tile, every XCD on a run of its own.
template <int EPI, int BX, int BW, int WX, int WW, int NST, int WPE>
__global__ __launch_bounds__(WX * WW * 64, WPE) void mx8_tile_kernel(Mx8Args p, int col_group)
{
    constexpr bool FIRST = EPI != TO_OUTPUT;
    constexpr int NW = WX * WW, TX = BX / WX / 32, TW = BW / WW / 32;
    constexpr int XLD = BX / 8 / NW, WLD = BW / 8 / NW;         // 1 KB load instructions per wave and slab
    constexpr int ROWS = BX + BW, SLD = (ROWS / 64 + NW - 1) / NW;       // scale load instructions per wave (64 rows each)
    constexpr int STAGE = ROWS * 128, SCALES = ROWS * 16;
    static_assert(!FIRST || TW == 2 || TW == 4, "a row's scale bytes of a wave leave together");
    static_assert(XLD * 8 * NW == BX && WLD * 8 * NW == BW && BX % 64 == 0 && BW % 64 == 0, "whole instructions");
    static_assert(NST >= 2 && NST <= 4, "two sets of scales hold");
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int offs[65], tstart[65];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wx = wave / WW, ww = wave % WW;
    if (wave == 0) {          // lane e: expert e's rows, and the row tiles before it
        const int begin = clamp_pairs(p.expert_offsets[min(lane, p.E)], p.P_cap),
                  end = clamp_pairs(p.expert_offsets[min(lane + 1, p.E)], p.P_cap);
        if (lane == 0) offs[0] = begin;
        offs[lane + 1] = end;
        int upto = (end - begin + BX - 1) / BX;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o, 64);
            if (lane >= o) upto += v;
        }
        if (lane == 0) tstart[0] = 0;
        tstart[lane + 1] = upto;
    }
    __syncthreads();
    const int nct = (p.N + BW - 1) / BW, total = tstart[p.E] * nct, nslab = p.K / 128, kg = p.K / kMxGroup;
    const bool xcds = (gridDim.x & 7) == 0;
    int seq, seq_end, step;
    if (xcds && col_group < nct) {
        const int x = blockIdx.x & 7;
        seq = (int)((int64_t)total * x / 8) + (blockIdx.x >> 3);
        seq_end = (int)((int64_t)total * (x + 1) / 8);
        step = gridDim.x >> 3;
    } else {
        seq = xcds ? (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3) : blockIdx.x;
        seq_end = total;
        step = gridDim.x;
    }

    // the 64 rows (X's, then W's) that scale load instruction i of this wave brings; instructions beyond the last repeat one
    auto scale_rows = [&](int i) { return (wave + NW * i) % (ROWS / 64) * 64; };
    // What depends on the lane is made again for every tile's parts from a copy of the lane number that the compiler cannot see through:
    // the values then do not occupy registers through the parts that do not use them.
    auto fresh_lane = [&] { int v = lane; asm volatile("" : "+v"(v)); return v; };
    // ---- a tile: where it lies, and its operands' addresses.  Rows beyond it repeat its last one, their products are not stored ----
    struct Tile { int g, row0, rows, n0; };
    auto locate = [&](int at) {
        const int e = fresh_lane(), first = tstart[e], next = tstart[e + 1], begin = offs[e], end = offs[e + 1];
        Tile t;
        t.g = __popcll(__ballot(at >= next * nct));
        const int t0 = __builtin_amdgcn_readlane(first, t.g), nrt = __builtin_amdgcn_readlane(next, t.g) - t0;
        const int r = at - t0 * nct, cg = r / (nrt * col_group), r2 = r - cg * nrt * col_group;
        const int gc = min(col_group, nct - cg * col_group), rt = r2 / gc;
        t.n0 = __builtin_amdgcn_readfirstlane((cg * col_group + (r2 - rt * gc)) * BW);
        t.row0 = __builtin_amdgcn_readfirstlane(__builtin_amdgcn_readlane(begin, t.g) + rt * BX);
        t.rows = __builtin_amdgcn_readfirstlane(min(BX, __builtin_amdgcn_readlane(end, t.g) - t.row0));
        t.g = __builtin_amdgcn_readfirstlane(t.g);
        return t;
    };
    // the rows of X that this lane brings: XLD for the data (row lane / 8 of an instruction's eight), then SLD for the scales
    auto x_rows = [&](const Tile& t, uint32_t (&xr)[XLD + SLD]) {
        const int lane = fresh_lane();
#pragma unroll
        for (int i = 0; i < XLD + SLD; ++i)
            xr[i] = (uint32_t)min(i < XLD ? (wave + NW * i) * 8 + (lane >> 3) : scale_rows(i - XLD) + lane, t.rows - 1);
        if (p.rows) {
            const int32_t* from = p.rows + t.row0;
#pragma unroll
            for (int i = 0; i < XLD + SLD; ++i) xr[i] = (uint32_t)from[xr[i]];
        }
    };
    const unsigned char *xb = nullptr, *xsb = nullptr, *wb = nullptr, *wsb = nullptr;
    uint32_t xo[XLD], wo[WLD], so[SLD];
    static_assert(NW % 2 == 0, "chunk");
    auto aim = [&](const Tile& t, const uint32_t (&xr)[XLD + SLD]) {
        const int lane = fresh_lane();
        // (an instruction's eight rows begin at a multiple of 8 and NW is even: the chunk that a lane brings is the same in all of them)
        const uint32_t chunk = (uint32_t)(((lane & 7) ^ ((wave * 8 + (lane >> 3)) >> 1 & 7)) << 4);
        xb = p.X + (p.rows ? (int64_t)0 : (int64_t)t.row0 * p.K);
        xsb = p.Xs + (p.rows ? (int64_t)0 : (int64_t)t.row0 * kg);
        wb = p.W + ((int64_t)t.g * p.N + t.n0) * p.K;
        wsb = p.Ws + ((int64_t)t.g * p.N + t.n0) * kg;
        const int last = p.N - 1 - t.n0;
#pragma unroll
        for (int i = 0; i < XLD; ++i) xo[i] = xr[i] * (uint32_t)p.K + chunk;
#pragma unroll
        for (int i = 0; i < WLD; ++i) wo[i] = (uint32_t)min((wave + NW * i) * 8 + (lane >> 3), last) * (uint32_t)p.K + chunk;
#pragma unroll
        for (int i = 0; i < SLD; ++i) {
            const int r = scale_rows(i);
            so[i] = (r < BX ? xr[XLD + i] : (uint32_t)min(r + lane - BX, last)) * (uint32_t)kg;
        }
    };
    // load instruction number x of a slab: X's rows, then W's
    constexpr int NLD = XLD + WLD;
    auto issue_one = [&](int x, int slab) {
        unsigned char* st = smem + slab % NST * STAGE;
        if (x < XLD) {
            load_to_lds(xb + slab * 128, xo[x], st + (wave + NW * x) * 1024);
        } else {
            const int i = x - XLD;
            load_to_lds(wb + slab * 128, wo[i], st + BX * 128 + (wave + NW * i) * 1024);
        }
    };
    // Scales, [2][ROWS][4 slabs' 4 bytes] by the parity of the four; the last four begin where they end with the row.  A contraction of
    // fewer than four slabs has them slab by slab, [slab][ROWS].
    unsigned char* const scales = smem + NST * STAGE;
    const bool by_four = nslab >= 4;
    auto first_of = [&](int slab) { return min(slab & ~3, nslab - 4); };
    auto issue_scales = [&](int slab) {
#pragma unroll
        for (int i = 0; i < SLD; ++i) {
            const int r = scale_rows(i);
            const unsigned char* from = r < BX ? xsb : wsb;
            if (by_four) load_to_lds(from + first_of(slab) * 4, so[i], scales + (slab >> 2 & 1) * SCALES + r * 16);
            else
                for (int u = 0; u < nslab; ++u)
                    load_dword_to_lds(reinterpret_cast<const int32_t*>(from + u * 4), so[i], reinterpret_cast<const int*>(scales + (u * ROWS + r) * 4));
        }
    };
    auto issue = [&](int slab) {
#pragma unroll
        for (int x = 0; x < NLD; ++x) issue_one(x, slab);
    };
    // a tile's bias (zeros, where there is none), its first scales and its first slabs
    float* const bias_lds = reinterpret_cast<float*>(scales + 2 * SCALES);    // [2][BW], by the tile's parity
    auto begin = [&](const Tile& t, int parity) {
        if (p.bias) {
            const int i = wave % (BW / 64) * 64;
            load_dword_to_lds(reinterpret_cast<const int32_t*>(p.bias + (int64_t)t.g * p.N), (uint32_t)min(t.n0 + i + lane, p.N - 1) * 4,
                              reinterpret_cast<const int*>(bias_lds + parity * BW + i));
        }
        issue_scales(0);
#pragma unroll
        for (int u = 0; u < NST; ++u)
            if (u < nslab) issue(u);
    };

    if (!p.bias)
        for (int i = threadIdx.x; i < 2 * BW; i += NW * 64) bias_lds[i] = 0.f;
    if (seq >= seq_end) return;
    Tile t = locate(seq);
    {
        uint32_t xr[XLD + SLD];
        x_rows(t, xr);
        aim(t, xr);
        __builtin_amdgcn_s_waitcnt(0x0f70);       // vmcnt(0): what the compiler itself has loaded is complete before the loads it does not count
        begin(t, 0);
    }
    // a wave's stores in an epilogue, at least: they follow the next tile's first loads, and are not waited for with them
    constexpr int STORES = TX * (FIRST ? TW + 1 : 2 * TW);
    static_assert((NST - 1) * NLD + STORES <= 63, "vmcnt");
    bool first = true;
    for (int parity = 0;; parity ^= 1) {
        const int lane_t = fresh_lane(), l32 = lane_t & 31, half = lane_t >> 5, key = l32 >> 1 & 7;
        auto fragment = [&](int row, int slab, int ks) {      // of k-step ks: this lane's 32 bytes of a row of the stage
            const unsigned char* at = smem + slab % NST * STAGE + row * 128;
            const u32x4 lo = *reinterpret_cast<const u32x4*>(at + (((ks * 4 + half) ^ key) << 4));
            const u32x4 hi = *reinterpret_cast<const u32x4*>(at + (((ks * 4 + 2 + half) ^ key) << 4));
            return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        };
        auto w_fragment = [&](int i, int slab, int ks) { return fragment(BX + (ww * TW + i) * 32 + l32, slab, ks); };
        auto x_fragment = [&](int j, int slab, int ks) { return fragment((wx * TX + j) * 32 + l32, slab, ks); };
        auto read_scales = [&](int slab, int (&sw)[TW], int (&sx)[TX]) {
            const int per_row = by_four ? 16 : 4;
            const unsigned char* st = scales + (by_four ? (slab >> 2 & 1) * SCALES + (slab - first_of(slab)) * 4 : slab * ROWS * 4) + l32 * per_row;
#pragma unroll
            for (int i = 0; i < TW; ++i) sw[i] = *reinterpret_cast<const int*>(st + (BX + (ww * TW + i) * 32) * per_row);
#pragma unroll
            for (int j = 0; j < TX; ++j) sx[j] = *reinterpret_cast<const int*>(st + (wx * TX + j) * 32 * per_row);
        };
        f32x16 acc[TW][TX];
        i32x8 w0[TW], w1[TW], x[TX];
        int sw[TW], sx[TX], sw_next[TW], sx_next[TX];
        // One k-step (64 k's) on w and x: its matrix instructions, and between them, pinned there, the reads of the next k-step's fragments
        // (next: there is one, k-step ks of slab `slab`), W's into the other set, X's into a fragment's own registers after its last use,
        // and what else is to go out.
        auto kstep = [&](auto op, auto begins, auto next, const i32x8 (&w)[TW], i32x8 (&w_next)[TW], int slab, int ks, auto&& also) {
#pragma unroll
            for (int j = 0; j < TX; ++j) {
#pragma unroll
                for (int i = 0; i < TW; ++i) {
                    const int m = j * TW + i;
                    acc[i][j] = mfma32<decltype(op)::value>(w[i], x[j], decltype(begins)::value ? f32x16{} : acc[i][j], sw[i], sx[j]);
                    also(m);
                    if (decltype(next)::value) {
                        if (m < TW) w_next[m] = w_fragment(m, slab, ks);
                        if (i == TW - 1) x[j] = x_fragment(j, slab, ks);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        auto use_scales = [&](const int (&w)[TW], const int (&x)[TX]) {       // this half's bytes: 0 (first k-step) and 2 (second)
#pragma unroll
            for (int i = 0; i < TW; ++i) sw[i] = (int)((uint32_t)w[i] >> (8 * half));
#pragma unroll
            for (int j = 0; j < TX; ++j) sx[j] = (int)((uint32_t)x[j] >> (8 * half));
        };
        if (nslab < NST) wait_vmcnt<0>();
        else if (first) wait_vmcnt<(NST - 1) * NLD>();
        else wait_vmcnt<(NST - 1) * NLD + STORES>();
        first = false;
        block_sync_lds();
#pragma unroll
        for (int i = 0; i < TW; ++i) w0[i] = w_fragment(i, 0, 0);
#pragma unroll
        for (int j = 0; j < TX; ++j) x[j] = x_fragment(j, 0, 0);
        read_scales(0, sw_next, sx_next);
        use_scales(sw_next, sx_next);
        constexpr auto OP0 = std::integral_constant<int, 0>{};
        constexpr auto OP2 = std::integral_constant<int, 2>{};
        constexpr auto YES = std::true_type{};
        constexpr auto NO = std::false_type{};
        auto first_half = [&](int s, auto begins) { kstep(OP0, begins, YES, w0, w1, s, 1, [](int) {}); };
        auto second_half = [&](int s, auto more) {            // of a slab that has a next; more: there is a slab s + NST
            // (of the loads that came after slab s + 1's, all may be on their way)
            if (decltype(more)::value || s + NST == nslab) wait_vmcnt<(NST - 2) * NLD>();
            else if (NST == 4 && s + 3 == nslab) wait_vmcnt<NLD>();
            else wait_vmcnt<0>();
            block_sync_lds();                                 // slab s + 1 is there, and everybody has slab s in registers
            kstep(OP2, NO, YES, w1, w0, s + 1, 0, [&](int m) {
                if (m == 0) read_scales(s + 1, sw_next, sx_next);
                if (decltype(more)::value) {
                    if (m == 0 && (s + NST) % 4 == 0) issue_scales(s + NST);
#pragma unroll
                    for (int u = NLD * m / (TX * TW); u < NLD * (m + 1) / (TX * TW); ++u) issue_one(u, s + NST);
                }
            });
            use_scales(sw_next, sx_next);
        };
        first_half(0, YES);
        int s = 0;
        for (; s + NST < nslab; ++s) {
            second_half(s, YES);
            first_half(s + 1, NO);
        }
        // the next tile's row numbers arrive under the last slabs
        const bool more_tiles = seq + step < seq_end;
        Tile next = t;
        if (more_tiles) next = locate(seq + step);
        for (; s + 1 < nslab; ++s) {
            second_half(s, NO);
            first_half(s + 1, NO);
        }
        uint32_t xr[XLD + SLD];
        x_rows(next, xr);
        kstep(OP2, NO, NO, w1, w0, 0, 0, [](int) {});
        // (the compiler would move these matrix instructions down to where their sums are read, and keep their operands until there)
        auto pin = [](f32x16& sums) {
            if constexpr (TW * TX * 16 > 128) asm volatile("" : "+a"(sums));
            else asm volatile("" : "+v"(sums));
        };
#pragma unroll
        for (int i = 0; i < TW; ++i)
#pragma unroll
            for (int j = 0; j < TX; ++j) pin(acc[i][j]);
        block_sync_lds();                                     // everybody is done with both stages
        if (more_tiles) {
            aim(next, xr);
            __builtin_amdgcn_s_waitcnt(0x0f70);               // vmcnt(0), as above
            begin(next, parity ^ 1);
        }

        // ---- epilogue: lane = row, registers = columns; stores end where the tile's rows do, and are made without a branch (a matrix
        // instruction whose result only some lanes use may be moved under their branch, where the others bring no operands) ----
        {
            const int lane_e = fresh_lane(), l32 = lane_e & 31, half = lane_e >> 5;
            uint32_t bytes[TX][TW];
#pragma unroll
            for (int i = 0; i < TW; ++i) {
                const int n = t.n0 + (ww * TW + i) * 32;      // N is a multiple of 32
                const uint32_t beyond = n < p.N ? 0u : 0x40000000u;
                f32x4 bias[4];
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    bias[q] = *reinterpret_cast<const f32x4*>(bias_lds + parity * BW + (ww * TW + i) * 32 + 8 * q + 4 * half);
#pragma unroll
                for (int j = 0; j < TX; ++j) {
                    const int r0 = (wx * TX + j) * 32, there = min(32, max(0, t.rows - r0));
                    const int64_t at = (int64_t)(t.row0 + r0);
                    pin(acc[i][j]);                           // (one unit's sums in vector registers at a time)
                    float v[16];
#pragma unroll
                    for (int r = 0; r < 16; ++r) v[r] = acc[i][j][r] + bias[r / 4][r % 4];
                    if constexpr (FIRST) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) v[r] = EPI == TO_RELU ? relu(v[r]) : gelu5(v[r]);
                        uint32_t ma = __float_as_uint(mx_max(v)), mb = ma;      // (of a group with an infinity any scale will do: O is NaN)
                        swap_halves(ma, mb);
                        const uint32_t b = mx_scale_byte(fmaxf(__uint_as_float(ma), __uint_as_float(mb)));
                        bytes[j][i] = b;
                        uint32_t d[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) d[q] = mx_pack4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3], b);
                        swap_halves(d[0], d[2]);              // the lower lanes get columns 0 .. 15, the upper ones 16 .. 31
                        swap_halves(d[1], d[3]);
                        __builtin_amdgcn_raw_buffer_store_b128(u32x4{d[0], d[2], d[1], d[3]}, rows_of(p.Aq + at * p.N, there * p.N),
                                                               (l32 * p.N + n + 16 * half) | beyond, 0, 0);
                    } else {
                        uint32_t d[8];
#pragma unroll
                        for (int q = 0; q < 8; ++q) d[q] = pack_bf16x2(v[2 * q], v[2 * q + 1]);
                        swap_halves(d[0], d[4]); swap_halves(d[1], d[5]); swap_halves(d[2], d[6]); swap_halves(d[3], d[7]);
                        const auto to = rows_of(p.O + at * p.N, there * p.N * 2);
                        const uint32_t off = ((l32 * p.N + n + 16 * half) * 2) | beyond;
                        __builtin_amdgcn_raw_buffer_store_b128(u32x4{d[0], d[1], d[4], d[5]}, to, off, 0, 0);
                        __builtin_amdgcn_raw_buffer_store_b128(u32x4{d[2], d[3], d[6], d[7]}, to, off + 16, 0, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if constexpr (FIRST) {
                const int ng = p.N / kMxGroup, n = (t.n0 + ww * TW * 32) / kMxGroup;
                const int off = half || n >= ng ? 0x40000000 : l32 * ng + n;           // (N is a multiple of a wave's columns)
#pragma unroll
                for (int j = 0; j < TX; ++j) {
                    const int r0 = (wx * TX + j) * 32, there = min(32, max(0, t.rows - r0));
                    const auto to = rows_of(p.As + (int64_t)(t.row0 + r0) * ng, there * ng);
                    if constexpr (TW == 4)
                        __builtin_amdgcn_raw_buffer_store_b32(bytes[j][0] | bytes[j][1] << 8 | bytes[j][2 % TW] << 16 | bytes[j][3 % TW] << 24, to, off, 0, 0);
                    else
                        __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(bytes[j][0] | bytes[j][1] << 8), to, off, 0, 0);
                }
            }
        }
        if (!more_tiles) break;
        t = next;
        seq += step;
    }
}

// Tiles.  BIG: one block per compute unit, four waves of 128x128; the least LDS traffic per product.  BIG8: the same tile by eight waves
// (128x64 each, two to a SIMD): they fill each other's stalls in an epilogue that gelu and conversion make as long as the main loop.
// MID: 128x128, two blocks per unit, one's epilogue under the other's products.  DEEP: 128x128 with four slabs on their way, for
// long contractions with few tiles.  TALL: 192x128, three slabs, where DEEP's tiles begin another round on the CUs and TALL's do not.
// SML: 64x128.  LOW: the same with four slabs, as long as its tiles are one round; SLIM: 64x64, where half as many places would be
// in use.  us, E = 16, d = 768, F = 3072 (but for the last row) / E = 64, d = 1024, F = 4096:
//   first product, pairs   48   512  2048  5998 16384 65536 /    96 65536    second product   48   512  2048  5998 16384 65536 / 65536
//     SML                 13.0  14.4  20.6  40.6  96.2   359 /  48.5   575                   20.4  21.0  22.9  44.6  79.1   315 /   542
//     MID                 14.8  16.2  21.9  37.0  79.9   281 /  52.6   467                   20.8  21.7  24.4  47.6  60.9   230 /   391
//     DEEP                20.0  20.3  27.7  44.2   104   381 /  66.9   561                   16.7  17.2  20.5  36.7  67.1   244 /   416
//     SLIM                  -     -     -     -     -     -     /    -     -                     12.2  17.4  18.3    -     -     -  /    -
//     LOW                   -     -     -     -     -     -     /    -     -                     15.1  15.7  17.6    -     -     -  /    -
//     TALL                  -     -     -     -     -     -     /    -     -                     20.5  20.5  23.1  27.6  68.2   227 /   392
//     BIG                   -   23.4  25.1  44.0  84.1   276 /    -    445                     -   36.2  38.1  42.8  49.6   207 /   325
//     BIG8                  -   21.8  23.9  40.8  77.2   256 /    -    420                     -   35.3  37.8  42.2  50.5   218 /   342
//     few rows            16.4  25.1  62.9   157     -     - /  74.5     -                   17.9  28.1  65.9   162     -     - /     -
// Few rows for up to eight pairs whose weights are little, and in the first product while its blocks of 32x32, each as long as the contraction,
// are few (us, first product, few rows / SML: 8 pairs of 16 experts, d = 768, F = 3072 9.3 / 12.0, 16 pairs 13.2 / 12.5; 452 pairs of
// one, d = 640, F = 768 8.7 / 10.6; 465 pairs of 40, d = 640, F = 640 11.7 / 9.3; 600 pairs of 4, d = 2048, F = 1024 22.4 / 15.8.
// Second, few rows / SLIM: 1 pair, d = 768, F = 3072 10.2 / 11.1, 8 pairs 11.2 / 11.4; 1911 pairs of 32, d = 128, F = 3840 23.4 / 13.2),
// and for sizes that the tile kernel does not take, until the kernel of any size is faster (us, few rows / any size, both products: 48 pairs
// of 16 experts, d = 800, F = 2400 24 / 53; 2000 pairs, d = 736, F = 2080 71 / 58; 8000 pairs, d = 992, F = 3104 423 / 208; 32768 pairs of
// 64, d = 352, F = 1376 337 / 156).  SLIM also while its tiles fill half of the CUs at most (the same 1911 pairs 13.2,
// LOW 17.2; 452 pairs of one, d = 640 7.2, LOW 8.5).
struct Big { static constexpr int BX = 256, BW = 256, WX = 2, WW = 2, NST = 2, WPE = 1, BLOCKS = 1; };
struct Big8 { static constexpr int BX = 256, BW = 256, WX = 2, WW = 4, NST = 2, WPE = 2, BLOCKS = 1; };
struct Mid { static constexpr int BX = 128, BW = 128, WX = 2, WW = 2, NST = 2, WPE = 2, BLOCKS = 2; };
struct Deep { static constexpr int BX = 128, BW = 128, WX = 2, WW = 2, NST = 4, WPE = 1, BLOCKS = 1; };
struct Sml { static constexpr int BX = 64, BW = 128, WX = 2, WW = 2, NST = 2, WPE = 2, BLOCKS = 2; };
struct Tall { static constexpr int BX = 192, BW = 128, WX = 2, WW = 2, NST = 3, WPE = 1, BLOCKS = 1; };
struct Slim { static constexpr int BX = 64, BW = 64, WX = 2, WW = 2, NST = 4, WPE = 2, BLOCKS = 2; };
struct Low { static constexpr int BX = 64, BW = 128, WX = 2, WW = 2, NST = 4, WPE = 1, BLOCKS = 1; };

enum class Pick { FewRows, AnySize, Sml, Mid, Slim, Low, Deep, Tall, Big, Big8 };
Pick pick(const Ctx& c, const evomoe_shape& s, bool first) {
    const int64_t pairs = c.pair_hint > 0 && c.pair_hint < s.P_cap ? c.pair_hint : s.P_cap, weights = (int64_t)s.d * s.F;
    const int n = first ? s.F : s.d;
    // tiles of few rows: an expert's last 32 rows are half full, and there are no more of them than pairs
    const int64_t panels = (pairs + 31) / 32 + s.E / 2, few = (panels < pairs ? panels : pairs) * (n / 32);
    if (s.d % 128 || s.F % 128) {     // a tile of any size costs as much as four of few rows, and eight of those per CU as much as a round of it
        const int64_t any = ((pairs + 127) / 128 + s.E / 2) * ((n + 127) / 128);
        return few <= 8 * c.num_cu || few <= 4 * any ? Pick::FewRows : Pick::AnySize;
    }
    if (pairs <= 8 && pairs * weights <= 20000000) return Pick::FewRows;
    if (first && few * s.d <= 400000) return Pick::FewRows;
    // 256x256 tiles: an expert fills two of them, and there are enough (short contractions need more, their epilogues being long)
    const int64_t tiles = ((pairs + 255) / 256 + s.E / 2) * ((n + 255) / 256);
    if (n >= 256 && pairs >= 512 * s.E && tiles >= (first ? 2 * c.num_cu : c.num_cu / 2)) return first ? Pick::Big8 : Pick::Big;
    if (!first) {     // (a DEEP tile takes two thirds of a TALL one's time)
        if (pairs <= 16 * s.E || ((pairs + 63) / 64 + s.E / 2) * (n / 64) <= c.num_cu / 2) return Pick::Slim;
        auto rounds = [&](int64_t rows) { return (((pairs + rows - 1) / rows + s.E / 2) * ((n + 127) / 128) + c.num_cu - 1) / c.num_cu; };
        if (rounds(Low::BX) == 1) return Pick::Low;
        return 3 * rounds(Tall::BX) < 2 * rounds(Deep::BX) ? Pick::Tall : Pick::Deep;
    }
    return pairs >= 256 * s.E ? Pick::Mid : Pick::Sml;
}

template <int EPI, class Cfg> hipError_t launch_tiles(const Ctx& c, const evomoe_shape& s, const Mx8Args& a) {
    auto kern = mx8_tile_kernel<EPI, Cfg::BX, Cfg::BW, Cfg::WX, Cfg::WW, Cfg::NST, Cfg::WPE>;
    constexpr int smem = (Cfg::BX + Cfg::BW) * (Cfg::NST * 128 + 2 * 16) + 2 * Cfg::BW * 4;
    static_assert((smem + 1024) * Cfg::BLOCKS <= 160 * 1024, "LDS");
    static bool configured[kMaxDevices];
    if (c.device < 0 || c.device >= kMaxDevices) return hipErrorInvalidDevice;
    if (!configured[c.device]) {
        hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != hipSuccess) return e;
        configured[c.device] = true;
    }
    const int nct = (a.N + Cfg::BW - 1) / Cfg::BW;
    const int64_t worst = ((s.P_cap + Cfg::BX - 1) / Cfg::BX + s.E) * nct, cap = (int64_t)c.num_cu * Cfg::BLOCKS;
    // column tiles whose weight panels stay in an XCD's L2 together, or all where a row panel is as large itself
    const int64_t fit = (int64_t)(2.4 * 1024 * 1024) / ((int64_t)Cfg::BW * a.K);
    const int col_group = (int64_t)Cfg::BX * a.K >= (1 << 20) ? nct : (int)(fit < 1 ? 1 : fit > nct ? nct : fit);
    hipLaunchKernelGGL(kern, dim3((unsigned)(worst < cap ? worst : cap)), dim3(Cfg::WX * Cfg::WW * 64), smem, c.stream, a, col_group);
    return hipGetLastError();
}

template <int EPI> hipError_t launch_few_rows(const Ctx& c, const evomoe_shape& s, const Mx8Args& a) {
    const int64_t worst = ((s.P_cap + 31) / 32 + s.E) * (a.N / 32), cap = (int64_t)c.num_cu * 16;
    const dim3 grid((unsigned)(worst < cap ? worst : cap));
    if (a.K <= 1024) hipLaunchKernelGGL((mx8_few_rows_kernel<EPI, 2>), grid, dim3(256), 0, c.stream, a);
    else hipLaunchKernelGGL((mx8_few_rows_kernel<EPI, 3>), grid, dim3(256), 0, c.stream, a);
    return hipGetLastError();
}

template <int EPI> hipError_t launch_any_size(const Ctx& c, const evomoe_shape& s, const Mx8Args& a) {
    const int64_t worst = ((s.P_cap + 127) / 128 + s.E) * ((a.N + 127) / 128), cap = (int64_t)c.num_cu * 2;
    hipLaunchKernelGGL(mx8_any_size_kernel<EPI>, dim3((unsigned)(worst < cap ? worst : cap)), dim3(256), 0, c.stream, a);
    return hipGetLastError();
}

template <int EPI> hipError_t launch_first(const Ctx& c, const evomoe_shape& s, const Mx8Args& a) {
    switch (pick(c, s, true)) {
        case Pick::FewRows: return launch_few_rows<EPI>(c, s, a);
        case Pick::AnySize: return launch_any_size<EPI>(c, s, a);
        case Pick::Sml: return launch_tiles<EPI, Sml>(c, s, a);
        case Pick::Mid: return launch_tiles<EPI, Mid>(c, s, a);
        default: return launch_tiles<EPI, Big8>(c, s, a);
    }
}
hipError_t launch_second(const Ctx& c, const evomoe_shape& s, const Mx8Args& a) {
    switch (pick(c, s, false)) {
        case Pick::FewRows: return launch_few_rows<TO_OUTPUT>(c, s, a);
        case Pick::AnySize: return launch_any_size<TO_OUTPUT>(c, s, a);
        case Pick::Deep: return launch_tiles<TO_OUTPUT, Deep>(c, s, a);
        case Pick::Slim: return launch_tiles<TO_OUTPUT, Slim>(c, s, a);
        case Pick::Low: return launch_tiles<TO_OUTPUT, Low>(c, s, a);
        case Pick::Tall: return launch_tiles<TO_OUTPUT, Tall>(c, s, a);
        default: return launch_tiles<TO_OUTPUT, Big>(c, s, a);
    }
}

size_t aq_bytes(const evomoe_shape& s) { return ((size_t)s.P_cap * s.F + 255) & ~(size_t)255; }

}  // namespace

FfnTile mx8_ffn_tile(const Ctx& c, const evomoe_shape& s, int kernel) {
    switch (pick(c, s, kernel == EVOMOE_K_FFN_MX8_GEMM1)) {
        case Pick::FewRows: return {32, 32, 4};
        case Pick::AnySize: return {128, 128, 4};
        case Pick::Sml: return {Sml::BX, Sml::BW, 4};
        case Pick::Mid: return {Mid::BX, Mid::BW, 4};
        case Pick::Deep: return {Deep::BX, Deep::BW, 4};
        case Pick::Slim: return {Slim::BX, Slim::BW, 4};
        case Pick::Low: return {Low::BX, Low::BW, 4};
        case Pick::Tall: return {Tall::BX, Tall::BW, 4};
        case Pick::Big: return {Big::BX, Big::BW, 4};
        case Pick::Big8: return {Big8::BX, Big8::BW, 8};
    }
    return {};
}

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
        err = s.act == EVOMOE_RELU ? launch_first<TO_RELU>(c, s, a) : launch_first<TO_GELU>(c, s, a);
    }
    if (err != hipSuccess) return err;
    a.X = Aq; a.Xs = As; a.W = (const uint8_t*)W2_q; a.Ws = W2_scale; a.rows = nullptr; a.bias = b2; a.O = (bf16_t*)O;
    a.N = s.d; a.K = s.F;
    ProfScope ps(c, EVOMOE_K_FFN_MX8_GEMM2);
    return launch_second(c, s, a);
}

}  // namespace evomoe
