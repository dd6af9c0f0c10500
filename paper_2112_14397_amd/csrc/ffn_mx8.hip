// Expert FFNs forward in 8 bits (e4m3 elements, a power of two scale for 32 of them along the contraction), on the scaled
// matrix instructions:
//   A = act(X W1^T + b1), to 8 bits again;     O = A W2^T + b2, bf16.
//
// Both products are computed transposed, C^T[n,r] = sum_k W[n,k] X[r,k]: the weights' rows are the matrix instruction's rows,
// and a lane of the result holds consecutive columns n of ONE row r, so that a group of 32 columns of A lies in a few
// lanes' registers and is converted without a detour through the LDS.
#include <type_traits>

#include "kernels.h"
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
        float m = mx_largest(v);
        m = fmaxf(m, __shfl_xor(m, 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        const uint32_t b = mx_scale_byte(m);
        if (i16 < rows) {
            uint8_t* out = p.Aq + (int64_t)(row0 + i16) * p.N + n0 + 4 * q;
            *reinterpret_cast<uint32_t*>(out) = mx_pack4(v[0], v[1], v[2], v[3], b);
            *reinterpret_cast<uint32_t*>(out + 16) = mx_pack4(v[4], v[5], v[6], v[7], b);
            if (q == 0) p.As[(int64_t)(row0 + i16) * (p.N / kMxGroup) + n0 / kMxGroup] = (uint8_t)b;
        }
    } else if (i16 < rows) {
        bf16_t* out = p.O + (int64_t)(row0 + i16) * p.N + n0 + 4 * q;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            *reinterpret_cast<u32x2*>(out + 16 * j) = u32x2{pack_bf16x2(v[4 * j], v[4 * j + 1]), pack_bf16x2(v[4 * j + 2], v[4 * j + 3])};
    }
}

// gelu(h) = max(h, 0) - x 2^p(x), x = |h|: 2^p is Phi(-x), p of degree five fitted for the least largest error of the product,
// 5e-7 with float32's own, for every finite h (p falls to -inf).  Ten VALU instructions and an exponential.
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

// The tile kernel, for d and F that are multiples of 128.  A block of WX x WW waves computes BX rows of X by BW rows of W, a
// wave TX x TW matrix instructions of 32 x 32.  The contraction runs in slabs of 128 bytes (one line of every row), two LDS stages
// deep; a stage holds both operands' slabs, rows of 128 bytes with the 16-byte chunk c of row r at chunk c ^ (r >> 1 & 7), so that
// sixteen lanes' reads of one chunk column meet all banks.  Scales come for four slabs at a time, 16 bytes of a row (with the loads of
// the first of them), as every row lies in another line: slab by slab, 4 bytes of a row, they took as long as half of the data (65536 pairs, one
// expert, d = 1024, F = 4096: second product 290 us, without loading scales 253).  Loads go straight to the LDS.
// Slab s + 2 is fetched into slab s's stage as soon as its last fragments are in registers, and lands while one and a half
// slabs multiply.  Blocks are persistent and walk the tiles as the bf16 kernels do: expert by expert, column group by column
// group, row tile by row tile, every XCD on a run of its own.
// EPI: what becomes of the sums.
enum { TO_RELU = EVOMOE_RELU, TO_GELU = EVOMOE_GELU_ERF, TO_OUTPUT };
template <int EPI, int BX, int BW, int WX, int WW, int WPE>
__global__ __launch_bounds__(WX * WW * 64, WPE) void mx8_tile_kernel(Mx8Args p, int col_group)
{
    constexpr bool FIRST = EPI != TO_OUTPUT;
    constexpr int NW = WX * WW, TX = BX / WX / 32, TW = BW / WW / 32;
    constexpr int XLD = BX / 8 / NW, WLD = BW / 8 / NW;         // 1 KB load instructions per wave and slab
    constexpr int ROWS = BX + BW, SLD = ROWS / 64 / NW;         // scale load instructions per wave (64 rows each)
    constexpr int STAGE = ROWS * 128, SCALES = ROWS * 16;
    static_assert(TW == 2 || TW == 4, "a row's scale bytes of a wave leave together");
    static_assert(XLD * 8 * NW == BX && WLD * 8 * NW == BW && SLD * 64 * NW == ROWS && BX % 64 == 0, "whole instructions");
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
            xr[i] = (uint32_t)min(i < XLD ? (wave + NW * i) * 8 + (lane >> 3) : (wave + NW * (i - XLD)) * 64 + lane, t.rows - 1);
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
            const int r = (wave + NW * i) * 64;               // X's rows, then W's; 64 of one operand, as BX is a multiple of 64
            so[i] = (r < BX ? xr[XLD + i] : (uint32_t)min(r + lane - BX, last)) * (uint32_t)kg;
        }
    };
    // load instruction number x of a slab: X's rows, then W's
    constexpr int NLD = XLD + WLD;
    auto issue_one = [&](int x, int slab) {
        unsigned char* st = smem + (slab & 1) * STAGE;
        if (x < XLD) {
            load_to_lds(xb + slab * 128, xo[x], st + (wave + NW * x) * 1024);
        } else {
            const int i = x - XLD;
            load_to_lds(wb + slab * 128, wo[i], st + BX * 128 + (wave + NW * i) * 1024);
        }
    };
    // Scales, [2][ROWS][4 slabs' 4 bytes] by the parity of the four; the last four begin where they end with the row.  A contraction of
    // fewer than four slabs has them slab by slab, [slab][ROWS].
    unsigned char* const scales = smem + 2 * STAGE;
    const bool by_four = nslab >= 4;
    auto first_of = [&](int slab) { return min(slab & ~3, nslab - 4); };
    auto issue_scales = [&](int slab) {
#pragma unroll
        for (int i = 0; i < SLD; ++i) {
            const int r = (wave + NW * i) * 64;
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
    // a tile's bias (zeros, where there is none), its first scales and its first two slabs
    float* const bias_lds = reinterpret_cast<float*>(scales + 2 * SCALES);    // [2][BW], by the tile's parity
    auto begin = [&](const Tile& t, int parity) {
        if (p.bias) {
            const int i = wave % (BW / 64) * 64;
            load_dword_to_lds(reinterpret_cast<const int32_t*>(p.bias + (int64_t)t.g * p.N), (uint32_t)min(t.n0 + i + lane, p.N - 1) * 4,
                              reinterpret_cast<const int*>(bias_lds + parity * BW + i));
        }
        issue_scales(0);
        issue(0);
        if (nslab > 1) issue(1);
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
    static_assert(NLD + STORES <= 63, "vmcnt");
    bool first = true;
    for (int parity = 0;; parity ^= 1) {
        const int lane_t = fresh_lane(), l32 = lane_t & 31, half = lane_t >> 5, key = l32 >> 1 & 7;
        // fragment number f (W's, then X's) of k-step ks
        auto read_one = [&](int f, int slab, int ks, i32x8 (&fw)[TW], i32x8 (&fx)[TX]) {
            const unsigned char* st = smem + (slab & 1) * STAGE;
            const unsigned char* row = st + (f < TW ? BX + (ww * TW + f) * 32 + l32 : (wx * TX + f - TW) * 32 + l32) * 128;
            const u32x4 lo = *reinterpret_cast<const u32x4*>(row + (((ks * 4 + half) ^ key) << 4));
            const u32x4 hi = *reinterpret_cast<const u32x4*>(row + (((ks * 4 + 2 + half) ^ key) << 4));
            (f < TW ? fw[f < TW ? f : 0] : fx[f < TW ? 0 : f - TW]) =
                i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        };
        auto read_scales = [&](int slab, int (&sw)[TW], int (&sx)[TX]) {
            const int per_row = by_four ? 16 : 4;
            const unsigned char* st = scales + (by_four ? (slab >> 2 & 1) * SCALES + (slab - first_of(slab)) * 4 : slab * ROWS * 4) + l32 * per_row;
#pragma unroll
            for (int i = 0; i < TW; ++i) sw[i] = *reinterpret_cast<const int*>(st + (BX + (ww * TW + i) * 32) * per_row);
#pragma unroll
            for (int j = 0; j < TX; ++j) sx[j] = *reinterpret_cast<const int*>(st + (wx * TX + j) * 32 * per_row);
        };
        f32x16 acc[TW][TX];
        i32x8 w0[TW], x0[TX], w1[TW], x1[TX];
        int sw[TW], sx[TX], sw_next[TW], sx_next[TX];
        // One k-step (64 k's): its matrix instructions, and between them, pinned there, the reads of the next k-step's fragments (the
        // first half of the instructions take them) and a later slab's loads.
        auto kstep = [&](auto op, auto begins, const i32x8 (&fw)[TW], const i32x8 (&fx)[TX], auto&& between) {
            constexpr int NMF = TW * TX;
#pragma unroll
            for (int m = 0; m < NMF; ++m) {
                const int j = m / TW, i = m % TW;
                acc[i][j] = mfma32<decltype(op)::value>(fw[i], fx[j], decltype(begins)::value ? f32x16{} : acc[i][j], sw[i], sx[j]);
                between(m, NMF);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        constexpr int NFR = TW + TX;
        auto read_share = [&](int m, int n, int slab, int ks, i32x8 (&fw)[TW], i32x8 (&fx)[TX]) {
            const int h = n / 2;
            if (m >= h) return;
#pragma unroll
            for (int f = NFR * m / h; f < NFR * (m + 1) / h; ++f) read_one(f, slab, ks, fw, fx);
        };
        auto use_scales = [&](const int (&w)[TW], const int (&x)[TX]) {       // this half's bytes: 0 (first k-step) and 2 (second)
#pragma unroll
            for (int i = 0; i < TW; ++i) sw[i] = (int)((uint32_t)w[i] >> (8 * half));
#pragma unroll
            for (int j = 0; j < TX; ++j) sx[j] = (int)((uint32_t)x[j] >> (8 * half));
        };
        if (nslab == 1) wait_vmcnt<0>();
        else if (first) wait_vmcnt<NLD>();
        else wait_vmcnt<NLD + STORES>();
        first = false;
        block_sync_lds();
#pragma unroll
        for (int f = 0; f < NFR; ++f) read_one(f, 0, 0, w0, x0);
        read_scales(0, sw_next, sx_next);
        use_scales(sw_next, sx_next);
        constexpr auto OP0 = std::integral_constant<int, 0>{};
        constexpr auto OP2 = std::integral_constant<int, 2>{};
        auto first_half = [&](int s, auto begins) {
            kstep(OP0, begins, w0, x0, [&](int m, int n) { read_share(m, n, s, 1, w1, x1); });
        };
        auto second_half = [&](int s, auto more) {            // of a slab that has a next; more: which has a next as well
            wait_vmcnt<0>();
            block_sync_lds();                                 // slab s + 1 is there, and everybody has slab s in registers
            kstep(OP2, std::false_type{}, w1, x1, [&](int m, int n) {
                if (m == 0) read_scales(s + 1, sw_next, sx_next);
                read_share(m, n, s + 1, 0, w0, x0);
                if (decltype(more)::value) {
                    if (m == 0 && (s + 2) % 4 == 0) issue_scales(s + 2);
#pragma unroll
                    for (int x = NLD * m / n; x < NLD * (m + 1) / n; ++x) issue_one(x, s + 2);
                }
            });
            use_scales(sw_next, sx_next);
        };
        first_half(0, std::true_type{});
        int s = 0;
        for (; s + 2 < nslab; ++s) {
            second_half(s, std::true_type{});
            first_half(s + 1, std::false_type{});
        }
        // the next tile's row numbers arrive under the last slabs
        const bool more_tiles = seq + step < seq_end;
        Tile next = t;
        if (more_tiles) next = locate(seq + step);
        if (s + 1 < nslab) {
            second_half(s, std::false_type{});
            first_half(s + 1, std::false_type{});
        }
        uint32_t xr[XLD + SLD];
        x_rows(next, xr);
        kstep(OP2, std::false_type{}, w1, x1, [&](int, int) {});
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
#pragma unroll
            for (int j = 0; j < TX; ++j) {
                const int r0 = (wx * TX + j) * 32, there = min(32, max(0, t.rows - r0));
                const int64_t at = (int64_t)(t.row0 + r0);
                uint32_t bytes[TW];
#pragma unroll
                for (int i = 0; i < TW; ++i) {
                    const int n = t.n0 + (ww * TW + i) * 32;  // N is a multiple of 32
                    const uint32_t beyond = n < p.N ? 0u : 0x40000000u;
                    pin(acc[i][j]);                           // (one unit's sums in vector registers at a time)
                    float v[16];
#pragma unroll
                    for (int r = 0; r < 16; ++r) v[r] = acc[i][j][r];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x4 b = *reinterpret_cast<const f32x4*>(bias_lds + parity * BW + (ww * TW + i) * 32 + 8 * q + 4 * half);
                        v[4 * q] += b.x; v[4 * q + 1] += b.y; v[4 * q + 2] += b.z; v[4 * q + 3] += b.w;
                    }
                    if constexpr (FIRST) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) v[r] = EPI == TO_RELU ? relu(v[r]) : gelu5(v[r]);
                        uint32_t ma = __float_as_uint(mx_max(v)), mb = ma;      // (of a group with an infinity any scale will do: O is NaN)
                        swap_halves(ma, mb);
                        const uint32_t b = mx_scale_byte(fmaxf(__uint_as_float(ma), __uint_as_float(mb)));
                        bytes[i] = b;
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
                if constexpr (FIRST) {
                    const int ng = p.N / kMxGroup, n = (t.n0 + ww * TW * 32) / kMxGroup;
                    const auto to = rows_of(p.As + at * ng, there * ng);
                    const int off = half || n >= ng ? 0x40000000 : l32 * ng + n;       // (N is a multiple of a wave's columns)
                    if constexpr (TW == 4)
                        __builtin_amdgcn_raw_buffer_store_b32(bytes[0] | bytes[1] << 8 | bytes[2 % TW] << 16 | bytes[3 % TW] << 24, to, off, 0, 0);
                    else
                        __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(bytes[0] | bytes[1] << 8), to, off, 0, 0);
                }
            }
        }
        if (!more_tiles) break;
        t = next;
        seq += step;
    }
}

template <bool FIRST> hipError_t launch_small(const Ctx& c, const evomoe_shape& s, const Mx8Args& a) {
    const dim3 grid((unsigned)((s.P_cap + 15) / 16 + s.E), (unsigned)(a.N / 32));
    hipLaunchKernelGGL(mx8_gemm_kernel<FIRST>, grid, dim3(64), 0, c.stream, a);
    return hipGetLastError();
}

struct Big { static constexpr int BX = 256, BW = 256, WX = 2, WW = 2, WPE = 1; };
struct Mid { static constexpr int BX = 128, BW = 128, WX = 2, WW = 2, WPE = 2; };

template <int EPI, class Cfg> hipError_t launch_tiles(const Ctx& c, const evomoe_shape& s, const Mx8Args& a) {
    auto kern = mx8_tile_kernel<EPI, Cfg::BX, Cfg::BW, Cfg::WX, Cfg::WW, Cfg::WPE>;
    constexpr int smem = 2 * (Cfg::BX + Cfg::BW) * (128 + 16) + 2 * Cfg::BW * 4;
    static bool configured[kMaxDevices];
    if (c.device < 0 || c.device >= kMaxDevices) return hipErrorInvalidDevice;
    if (!configured[c.device]) {
        hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != hipSuccess) return e;
        configured[c.device] = true;
    }
    const int nct = (a.N + Cfg::BW - 1) / Cfg::BW;
    const int64_t worst = ((s.P_cap + Cfg::BX - 1) / Cfg::BX + s.E) * nct, cap = (int64_t)c.num_cu * Cfg::WPE;
    const int64_t fit = (int64_t)(2.4 * 1024 * 1024) / ((int64_t)Cfg::BW * a.K);
    const int col_group = (int64_t)Cfg::BX * a.K >= (1 << 20) ? nct : (int)(fit < 1 ? 1 : fit > nct ? nct : fit);
    hipLaunchKernelGGL(kern, dim3((unsigned)(worst < cap ? worst : cap)), dim3(Cfg::WX * Cfg::WW * 64), smem, c.stream, a, col_group);
    return hipGetLastError();
}

template <bool FIRST> hipError_t launch(const Ctx& c, const evomoe_shape& s, const Mx8Args& a) {
    const int64_t pairs = c.pair_hint > 0 && c.pair_hint < s.P_cap ? c.pair_hint : s.P_cap;
    if (s.d % 128 || s.F % 128 || pairs < 32 * s.E) return launch_small<FIRST>(c, s, a);
    const int64_t tiles = ((pairs + 255) / 256 + s.E / 2) * ((a.N + 255) / 256);
    auto run = [&](auto epi) {
        constexpr int EPI = decltype(epi)::value;
        return tiles >= 2 * c.num_cu ? launch_tiles<EPI, Big>(c, s, a) : launch_tiles<EPI, Mid>(c, s, a);
    };
    if (!FIRST) return run(std::integral_constant<int, TO_OUTPUT>{});
    return a.act == EVOMOE_RELU ? run(std::integral_constant<int, TO_RELU>{}) : run(std::integral_constant<int, TO_GELU>{});
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
