// The whole MoE layer for up to 16 tokens in two launches (three where the gate matrix or x is large), on bf16 or MXFP4 weights.
//
//   few_up_kernel    routes, and leaves h[t, j] = w_tj * silu(x_t W1_e) * (x_t W3_e) for each pick e of token t, and of each shared expert
//   few_down_kernel  out[t] = sum over the picks and the shared experts of h W2_e
// The weight of a pick is part of h, so that the sum over experts is one chain of matrix instructions along a contraction of (experts x F),
// and no launch has to combine.  What a few tokens cost is reading the weights of the experts that they pick, so activations stay as
// they are: x is bf16, and h is kept as two bf16 (16 bits of it), each multiplied with the weights.  4-bit weights become bf16, which
// holds their values exactly, in registers.
//
// A wavefront takes 16 columns: W is the row operand straight from memory, the tokens are the 16 columns of the other one, whether they picked
// the expert or not; what they did not pick is not stored (gate and up) or left out of the sum (down).
//
// Bound by reading the weights where they are large and bf16 (8 experts, H = 4096, F = 14336, 16 tokens 418 us, 6.7 TB/s).  The same layer in MXFP4 takes 148 (5.1 TB/s) and 160 + 2
// experts, H = 5120, F = 1536 178 to 188 (5.2): there a piece of 1 KiB is 16 conversions and four to eight matrix instructions, which share the time with its load.  Gate/up and
// down launch of the former: 103 and 54 us, without conversions 87 and 48, without loads of weights 59 and 31.  By the chain of launches, routing and first loads where
// they are small (64 + 2 experts, H = 2048, one token 23.5 us: logits 3.5, gate/up 12, down 8.5; 8 experts, H = 512, F = 1024, bf16, 16 tokens 15.8 us, where the
// layer for any batch takes 17.7).
#include <algorithm>

#include "few.h"
#include "fp4.h"
#include "topk.h"

namespace moe {
namespace {

// Said to be global memory: after loads through a generic pointer the compiler waits for every load in flight.
typedef const __attribute__((address_space(1))) u32x4* gpiece_t;
typedef const __attribute__((address_space(1))) uint32_t* gword_t;
template <bool NT = false>
__device__ __forceinline__ u32x4 load_piece(const char* at) {
    return NT ? __builtin_nontemporal_load((gpiece_t)(uintptr_t)at) : *(gpiece_t)(uintptr_t)at;
}
__device__ __forceinline__ uint32_t load_word(const char* at) { return *(gword_t)(uintptr_t)at; }

constexpr int WAVES = 8;
constexpr int LOGIT_STRIDE = 256;

__device__ __forceinline__ f32x4 mfma(const bf16x8 a, const bf16x8 b, const f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Part f of a lane's piece of a block of 16 rows: 8 values along the contraction as bf16.  bf16: the piece is 8 values.  MXFP4: it is 32.
template <bool FP4>
__device__ __forceinline__ bf16x8 weight_part(const u32x4 piece, const float scale, const int f) {
    if constexpr (!FP4) {
        return __builtin_bit_cast(bf16x8, piece);
    } else {
        u32x4 v = {0u, 0u, 0u, 0u};
#if defined(__gfx950__)
        const uint32_t c = piece[f];
        v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
        v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
        v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
        v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
#endif
        return __builtin_bit_cast(bf16x8, v);
    }
}
// The scale of sub-tile t from the four sub-tiles' bytes; one of 255 is NaN, whatever the codes are.
__device__ __forceinline__ float scale_of(const uint32_t four, const int t) {
    const uint32_t byte = four >> (8 * (t & 3)) & 255u;
    return __uint_as_float(byte == 255u ? 0x7fc00000u : byte << 23);
}

// A pointer that is the same for the wavefront, to global memory.
__device__ __forceinline__ const char* uniform(const char* ptr) {
    const uint64_t v = (uint64_t)ptr;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (const char*)(((uint64_t)hi << 32) | lo);
}

// By a whole workgroup of at least 256 threads, from idx [T][k] in LDS.
__device__ __forceinline__ void gather_picks(Picks& s, const int32_t* idx, const int T, const int k, const int E) {
    __shared__ int wave_count[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int e = tid; e < E; e += blockDim.x) *reinterpret_cast<u32x4*>(s.pick[e]) = u32x4{~0u, ~0u, ~0u, ~0u};
    __syncthreads();
    for (int p = tid; p < T * k; p += blockDim.x) s.pick[idx[p]][p / k] = (int8_t)(p - p / k * k);
    __syncthreads();
    bool any = false;
    if (tid < E) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(s.pick[tid]);
        any = (v[0] & v[1] & v[2] & v[3]) != ~0u;
    }
    const uint64_t b = __ballot(any);
    if (wave < 4 && lane == 0) wave_count[wave] = __popcll(b);
    __syncthreads();
    int at = __popcll(b & ((1ull << lane) - 1));
    for (int w = 0; w < 4; ++w) at += w < wave ? wave_count[w] : 0;
    if (any) s.active[at] = (int16_t)tid;
    if (tid == 0) s.n = wave_count[0] + wave_count[1] + wave_count[2] + wave_count[3];
    __syncthreads();
}

// x in LDS or as a copy in memory, so that what one load of a wavefront takes is consecutive: pieces of 8 values in the order [step][part][row][g], where
// piece (step, part, g) of a row is what lane group g multiplies in that part of that step (MXFP4: values 128 step + 32 g + 8 part on, bf16:
// 32 step + 8 g on).  `row_pieces`: rows that it holds.
template <bool FP4>
__device__ __forceinline__ int x_place(const int piece, const int row, const int rows) {   // piece: of the row, in its own order
    const int step_part = FP4 ? (piece >> 4) * 4 + (piece & 3) : piece >> 2, g = FP4 ? piece >> 2 & 3 : piece & 3;
    return ((step_part * rows + row) * 4 + g) * 16;
}

// Logits of 16 experts (block nb) by one wavefront over the blocks of 32 first, first + step, ..: lane (rl, g) gets tokens 4g .. 4g+3 of expert rl.
// x_of(s): the lane's piece of block s.
template <class X>
__device__ __forceinline__ f32x4 logits_of(const FewArgs& p, const int nb, const int first, const int step, const X x_of) {
    const int lane = threadIdx.x & 63, rl = lane & 15, g = lane >> 4;
    const char* const wb = p.wg + (size_t)nb * (p.H >> 5) * 1024 + rl * 64 + ((g ^ block_swizzle(rl)) << 4);
    const int KS = p.H >> 5;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    constexpr int AHEAD = 16;
    for (int s0 = first; s0 < KS; s0 += step * AHEAD) {
        u32x4 b[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (s0 + u * step < KS) b[u] = load_piece(wb + (size_t)(s0 + u * step) * 1024);   // wave-uniform
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (s0 + u * step < KS) acc = mfma(__builtin_bit_cast(bf16x8, x_of(s0 + u * step)), __builtin_bit_cast(bf16x8, b[u]), acc);
    }
    return acc;
}

// A large gate matrix, or more x than LDS holds: K cut over the wavefronts of few_logit_shares workgroups to 16 experts, sums in wave order, and over the workgroups
// where the logits are read; the workgroups behind them copy x.
constexpr int LOGIT_WAVES = 16;   // (whole layer, us, with 8: 160 + 2 experts, H = 5120, 16 tokens 180.9, 178.8; 64 + 2 experts, one token 24.5, 24.2)
template <bool FP4>
__global__ __launch_bounds__(LOGIT_WAVES * 64) void few_logits_kernel(const FewArgs p) {
    __shared__ float part[LOGIT_WAVES][256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int blocks = (p.E + 15) >> 4, share = blockIdx.x / blocks, nb = blockIdx.x - share * blocks;
    if (share >= p.logit_shares) {
        const int pieces = p.H >> 3, i = (blockIdx.x - blocks * p.logit_shares) * LOGIT_WAVES * 64 + tid, row = i / pieces, piece = i - row * pieces;
        if (row < p.T) *reinterpret_cast<u32x4*>(p.x_copy + x_place<FP4>(piece, row, p.T)) = load_piece(p.x + (size_t)i * 16);
        return;
    }
    const char* const xa = p.x + (size_t)min(lane & 15, p.T - 1) * p.H * 2 + (lane >> 4) * 16;
    const f32x4 acc = logits_of(p, nb, share * LOGIT_WAVES + wave, p.logit_shares * LOGIT_WAVES, [&](const int s) __attribute__((always_inline)) { return load_piece(xa + (size_t)s * 64); });
#pragma unroll
    for (int r = 0; r < 4; ++r) part[wave][(4 * (lane >> 4) + r) * 16 + (lane & 15)] = acc[r];
    __syncthreads();
    const int t = tid >> 4;
    if (t >= p.T) return;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < LOGIT_WAVES; ++w) v += part[w][tid];
    p.logits_out[(share * p.T + t) * p.ep + nb * 16 + (tid & 15)] = v;
}

// Softmax and top-k of all tokens, by four wavefronts, into idx and w [16][16] in LDS.  logits: `shares` matrices that are added in order.
template <int NV>
__device__ __forceinline__ void select(const FewArgs& p, const float* logits, const int stride, const int shares, int32_t* idx, float* w) {
    const int lane = threadIdx.x & 63, row = lane & 15, t = (threadIdx.x >> 6) * 4 + (lane >> 4);
    float v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = row + 16 * i;
        v[i] = e < p.E ? logits[min(t, p.T - 1) * stride + e] : 0.f;
    }
    for (int q = 1; q < shares; ++q)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = row + 16 * i;
            if (e < p.E) v[i] += logits[(q * p.T + min(t, p.T - 1)) * stride + e];
        }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = row + 16 * i;
        v[i] = e < p.E ? v[i] + (p.bias ? p.bias[e] : 0.f) : -INFINITY;
    }
    int e;
    float we;
    route_select_row16<NV>(v, row, p.E, p.k, p.renorm, p.scale, e, we);
    if (t < p.T && row < p.k) {
        idx[t * p.k + row] = e;
        w[t * p.k + row] = we;
    }
}

// h: row [step][part][hi, lo][g] of pieces of 8, as x above.
template <bool FP4>
__device__ __forceinline__ int h_place(const int f) {   // byte of the high half of value f; the low half 64 bytes on
    return FP4 ? (f >> 7) * 512 + (f >> 3 & 3) * 128 + (f >> 5 & 3) * 16 + (f & 7) * 2 : (f >> 5) * 128 + (f >> 3 & 3) * 16 + (f & 7) * 2;
}

// A contraction is cut into tasks of four steps (MXFP4: 512, one dword of scales to a lane; bf16: 128).
constexpr int TASK = 4;

// Gate and up, and the router before them.  An item is 32 columns (64 where x does not fit LDS: each load of it then
// meets twice the weights) of both matrices of a picked or shared expert; the tasks of a workgroup's items, one
// after the other, go to its wavefronts in turn, and after each round the sums of eight tasks meet in LDS, where every thread adds up one
// column of a token in the order of the tasks.  Loads run a task ahead.  XLDS: x is in LDS.
template <bool FP4, bool NT, bool XLDS>
__global__ __launch_bounds__(WAVES * 64) void few_up_kernel(const FewArgs p) {
    extern __shared__ __attribute__((aligned(16))) char x_lds[];
    // the logits and their parts, then the wavefronts' sums (in two places in turn one barrier a round is enough)
    constexpr int NB = XLDS ? 2 : 4, PLACES = XLDS ? 2 : 1, DEPTH = FP4 && !XLDS ? 2 : TASK;
    __shared__ __attribute__((aligned(16))) float room[PLACES][WAVES][2][NB][256];
    __shared__ Picks picks;
    __shared__ int32_t idx[FEW_TOKENS * FEW_TOP_K];
    __shared__ float w[FEW_TOKENS * FEW_TOP_K];
    __shared__ const char* matrix[2][256];   // of every expert
    float* const logits = &room[0][0][0][0][0];
    float(*const part)[256] = room[0][WAVES / 2][0];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), rl = lane & 15, g = lane >> 4;
    const int experts = p.E + p.Ns, x_row = min(rl, p.T - 1);
    if (tid < 256)
#pragma unroll
        for (int m = 0; m < 2; ++m) matrix[m][tid] = (const char*)p.weights[m * experts + min(tid, experts - 1)];
    if (XLDS) {
        const int pieces = p.H >> 3;
        for (int i = tid; i < p.T * pieces; i += WAVES * 64) {
            const int row = i / pieces, piece = i - row * pieces;
            *reinterpret_cast<u32x4*>(x_lds + x_place<FP4>(piece, row, p.T)) = load_piece(p.x + (size_t)i * 16);
        }
        __syncthreads();
    }
    if (!p.logits) {
        // up to 8 blocks of 16 experts side by side; what wavefronts are left share the contraction, and are added in order
        const int blocks = (p.E + 15) >> 4;
        int per = WAVES;
        while (per > 1 && WAVES / per < blocks) per >>= 1;
        const int beside = WAVES / per, share = wave / beside;
        for (int nb = wave - share * beside; nb < blocks; nb += beside) {
            const f32x4 acc = logits_of(p, nb, share, per, [&](const int s) __attribute__((always_inline)) {
                return *reinterpret_cast<const u32x4*>(x_lds + x_place<FP4>(s * 4 + g, x_row, p.T));
            });
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (per == 1) logits[(4 * g + r) * LOGIT_STRIDE + nb * 16 + rl] = acc[r];
                else part[wave][(4 * g + r) * 16 + rl] = acc[r];
            }
        }
        __syncthreads();
        if (per > 1) {
            for (int i = tid; i < blocks * 256; i += WAVES * 64) {
                const int nb = i >> 8;
                float v = 0.f;
                for (int q = 0; q < per; ++q) v += part[q * beside + nb][i & 255];
                logits[(i >> 4 & 15) * LOGIT_STRIDE + nb * 16 + (i & 15)] = v;
            }
            __syncthreads();
        }
    }
    const float* const l = p.logits ? p.logits : logits;
    const int stride = p.logits ? p.ep : LOGIT_STRIDE, shares = p.logits ? p.logit_shares : 1;
    if (wave * 4 < p.T) {
        if (p.E <= 16) select<1>(p, l, stride, shares, idx, w);
        else if (p.E <= 64) select<4>(p, l, stride, shares, idx, w);
        else if (p.E <= 160) select<10>(p, l, stride, shares, idx, w);
        else select<16>(p, l, stride, shares, idx, w);
    }
    __syncthreads();
    gather_picks(picks, idx, p.T, p.k, p.E);
    if (blockIdx.x == 0) {
        const uint32_t* const from = reinterpret_cast<const uint32_t*>(&picks);
        for (int i = tid; i < (int)sizeof(Picks) / 4; i += WAVES * 64) reinterpret_cast<uint32_t*>(p.picks)[i] = from[i];
        for (int i = tid; i < p.H >> 4; i += WAVES * 64) p.arrived[i] = 0;
    }

    const int units = p.F / (NB * 16), n_active = __builtin_amdgcn_readfirstlane(picks.n);
    const int KT = FP4 ? (p.H + 127) >> 7 : p.H >> 5, groups = (p.H + 511) >> 9, G = (KT + TASK - 1) / TASK;
    const int items = (n_active + p.Ns) * units, mine = items > (int)blockIdx.x ? (items - 1 - blockIdx.x) / gridDim.x + 1 : 0;
    const int tasks = mine * G;
    const uint32_t lane_w = (uint32_t)(rl * 64 + ((g ^ block_swizzle(rl)) << 4)), lane_s = (uint32_t)(rl * 16 + g * 4);
    constexpr int PARTS = FP4 ? 4 : 1;
    u32x4 a[DEPTH][2][NB], x[XLDS ? 1 : DEPTH][PARTS];
    uint32_t sc[2][NB], sc_next[2][NB];
    const uint32_t lane_x = (uint32_t)(x_row * 64 + g * 16);
    // asked for next: step `ls` of task group lg of the li-th item
    int lq = wave, li = wave / G, lg = wave - li * G, ls = 0;
    const char *lw[2] = {nullptr, nullptr};
    int block = 0;
    auto load = [&](const int slot) __attribute__((always_inline)) {
        if (lq >= tasks) return;
        if (ls == 0) {
            const int item = blockIdx.x + li * gridDim.x, at = item / units, e = at < n_active ? picks.active[at] : p.E + at - n_active;
            block = (item - at * units) * NB;
            lw[0] = uniform(matrix[0][e]);
            lw[1] = uniform(matrix[1][e]);
            if (FP4)
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int c = 0; c < NB; ++c) sc_next[m][c] = load_word(lw[m] + p.up_scales_at + ((size_t)(block + c) * groups + lg) * 256 + lane_s);
        }
        const int t = lg * TASK + ls;
        if (t < KT) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int c = 0; c < NB; ++c) a[slot][m][c] = load_piece<NT>(lw[m] + ((size_t)(block + c) * KT + t) * 1024 + lane_w);
            if (!XLDS)
#pragma unroll
                for (int f = 0; f < PARTS; ++f) x[XLDS ? 0 : slot][f] = load_piece(p.x_copy + (size_t)(t * PARTS + f) * p.T * 64 + lane_x);
        }
        if (++ls == TASK) {
            ls = 0;
            lq += WAVES;
            for (lg += WAVES; lg >= G; lg -= G) ++li;
        }
    };
#pragma unroll
    for (int u = 0; u < DEPTH; ++u) load(u);
    // of token tid / 32, columns tid % 32 (and 32 further) of the item that is being added up
    float gate[NB / 2] = {}, up[NB / 2] = {};
    int item = 0, group = 0, my_group = wave % G;
    for (int q0 = 0; q0 < tasks; q0 += WAVES) {
        f32x4 acc[2][NB] = {};
        if (q0 + wave < tasks) {
#pragma unroll
            for (int u = 0; u < TASK; ++u) {
                if (u == 0)
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int c = 0; c < NB; ++c) sc[m][c] = sc_next[m][c];
                const int t = my_group * TASK + u;
                if (t < KT) {
                    if (XLDS)
#pragma unroll
                        for (int f = 0; f < PARTS; ++f) x[0][f] = *reinterpret_cast<const u32x4*>(x_lds + (t * PARTS + f) * p.T * 64 + lane_x);
#pragma unroll
                    for (int f = 0; f < PARTS; ++f) {
                        // past H (a multiple of 64) the weights are zero and x is not there
                        u32x4 v = x[XLDS ? 0 : u % DEPTH][f];
                        if (FP4 && t * 128 + g * 32 >= p.H) v = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
                        for (int m = 0; m < 2; ++m)
#pragma unroll
                            for (int c = 0; c < NB; ++c)
                                acc[m][c] = mfma(weight_part<FP4>(a[u % DEPTH][m][c], FP4 ? scale_of(sc[m][c], u) : 0.f, f), __builtin_bit_cast(bf16x8, v), acc[m][c]);
                    }
                }
                load(u % DEPTH);
            }
            for (my_group += WAVES; my_group >= G;) my_group -= G;
        }
        // lane (rl, g) has columns 4 g + r of 16 of token rl
        float(*const sums)[2][NB][256] = room[q0 / WAVES % PLACES];
        if (PLACES == 1 && q0 > 0) __syncthreads();
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int c = 0; c < NB; ++c) *reinterpret_cast<f32x4*>(&sums[wave][m][c][rl * 16 + 4 * g]) = acc[m][c];
        __syncthreads();
        const int t = tid >> 5, c = tid >> 4 & 1, n = tid & 15;
#pragma unroll
        for (int q = 0; q < WAVES; ++q) {
            if (q0 + q >= tasks) break;
#pragma unroll
            for (int j = 0; j < NB / 2; ++j) {
                gate[j] += sums[q][0][j * 2 + c][t * 16 + n];
                up[j] += sums[q][1][j * 2 + c][t * 16 + n];
            }
            if (++group < G) continue;
            const int it = blockIdx.x + item * gridDim.x, at = it / units, f0 = (it - at * units) * NB * 16 + c * 16 + n;
            int row = -1;
            float weight = 1.f;
            if (t < p.T) {
                if (at >= n_active) row = p.T * (p.k + at - n_active) + t;
                else if (const int j = picks.pick[picks.active[at]][t]; j >= 0) {
                    row = t * p.k + j;
                    weight = w[row];
                }
            }
#pragma unroll
            for (int j = 0; j < NB / 2; ++j) {
                if (row >= 0) {
                    const float v = weight * (gate[j] / (1.0f + __expf(-gate[j])) * up[j]);
                    // what is finite in fp32 stays finite: above the largest bf16 that one is the high half; an infinity or NaN has no low half
                    const __bf16 hi = __builtin_isfinite(v) ? (__bf16)fminf(fmaxf(v, -0x1.fep127f), 0x1.fep127f) : (__bf16)v;
                    char* const to = p.h + (size_t)row * p.h_row + h_place<FP4>(f0 + j * 32);
                    *reinterpret_cast<__bf16*>(to) = hi;
                    *reinterpret_cast<__bf16*>(to + 64) = __builtin_isfinite(v) ? (__bf16)(v - (float)hi) : (__bf16)0.0f;
                }
                gate[j] = up[j] = 0.f;
            }
            group = 0;
            ++item;
        }
    }
}

// Down: NB * 16 columns to a workgroup, and a share of the tasks of all picked and shared experts, one after the other; its wavefronts take them in turn.
// The shares' sums meet in the workgroup that comes last, which adds them in order: no workgroup waits for another.  Sums and counter
// pass by the L2s, each of which only its own XCD sees.
template <bool FP4, bool NT, int NB>
__global__ __launch_bounds__(WAVES * 64) void few_down_kernel(const FewArgs p) {
    __shared__ Picks picks;
    __shared__ __attribute__((aligned(16))) float sums[WAVES][NB][256];
    __shared__ const char* matrix[256];   // of every expert
    __shared__ int last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), rl = lane & 15, g = lane >> 4;
    const int experts = p.E + p.Ns, x_row = min(rl, p.T - 1);
    if (tid < 256) matrix[tid] = (const char*)p.weights[2 * experts + min(tid, experts - 1)];
    const u32x4* const from_up = reinterpret_cast<const u32x4*>(p.picks);
    for (int i = tid; i < (int)sizeof(Picks) / 16; i += WAVES * 64) reinterpret_cast<u32x4*>(&picks)[i] = from_up[i];
    __syncthreads();
    const int n_active = __builtin_amdgcn_readfirstlane(picks.n);
    const int share = blockIdx.x % p.shares, columns = blockIdx.x / p.shares;
    const int KT = FP4 ? (p.F + 127) >> 7 : p.F >> 5, groups = (p.F + 511) >> 9, G = (KT + TASK - 1) / TASK;
    constexpr int DEPTH = FP4 && NB > 1 ? 2 : TASK, PARTS = FP4 ? 4 : 1, HSTEP = FP4 ? 512 : 128;
    const uint32_t lane_w = (uint32_t)(rl * 64 + ((g ^ block_swizzle(rl)) << 4)), lane_s = (uint32_t)(rl * 16 + g * 4);
    const int total = (n_active + p.Ns) * G;
    const int from = (int)((int64_t)total * share / p.shares), to = (int)((int64_t)total * (share + 1) / p.shares);
    u32x4 a[DEPTH][NB], hi[DEPTH][PARTS], lo[DEPTH][PARTS];
    uint32_t sc[NB], sc_next[NB];
    // asked for next: step `ls` of group lg of the le-th expert
    int lq = from + wave, le = lq / G, lg = lq - le * G, ls = 0;
    const char *w2 = nullptr, *h_at = nullptr;
    auto load = [&](const int slot) __attribute__((always_inline)) {
        if (lq >= to) return;
        if (ls == 0) {
            const int e = __builtin_amdgcn_readfirstlane(le < n_active ? picks.active[le] : p.E + le - n_active);
            w2 = uniform(matrix[e]);
            // a token that did not pick the expert multiplies another row: its column of the product is not used
            const int j = picks.pick[min(e, p.E - 1)][x_row], row = le >= n_active ? p.T * (p.k + le - n_active) + x_row : (j >= 0 ? x_row * p.k + j : 0);
            h_at = p.h + (size_t)row * p.h_row + g * 16;
            if (FP4)
#pragma unroll
                for (int c = 0; c < NB; ++c) sc_next[c] = load_word(w2 + p.down_scales_at + ((size_t)(columns * NB + c) * groups + lg) * 256 + lane_s);
        }
        const int t = lg * TASK + ls;
        if (t < KT) {
#pragma unroll
            for (int c = 0; c < NB; ++c) a[slot][c] = load_piece<NT>(w2 + ((size_t)(columns * NB + c) * KT + t) * 1024 + lane_w);
            const char* const from_h = h_at + (uint32_t)(t * HSTEP);
#pragma unroll
            for (int f = 0; f < PARTS; ++f) {
                hi[slot][f] = load_piece(from_h + f * 128);
                lo[slot][f] = load_piece(from_h + f * 128 + 64);
            }
        }
        if (++ls == TASK) {
            ls = 0;
            lq += WAVES;
            for (lg += WAVES; lg >= G; lg -= G) ++le;
        }
    };
#pragma unroll
    for (int u = 0; u < DEPTH; ++u) load(u);
    f32x4 sum[NB] = {};
    for (int q = from + wave; q < to; q += WAVES) {
        const int at = q / G, group = q - at * G;
        f32x4 acc[NB] = {};
#pragma unroll
        for (int u = 0; u < TASK; ++u) {
            if (u == 0)
#pragma unroll
                for (int c = 0; c < NB; ++c) sc[c] = sc_next[c];
            const int t = group * TASK + u;
            if (t < KT) {
                if (FP4 && t * 128 + 128 > p.F) {   // past F (a multiple of 64) the weights are zero and nothing was written
#pragma unroll
                    for (int f = 0; f < PARTS; ++f)
                        if (t * 128 + g * 32 >= p.F) hi[u % DEPTH][f] = lo[u % DEPTH][f] = u32x4{0u, 0u, 0u, 0u};
                }
#pragma unroll
                for (int c = 0; c < NB; ++c) {
                    const float scale = FP4 ? scale_of(sc[c], u) : 0.f;
#pragma unroll
                    for (int f = 0; f < PARTS; ++f) {
                        const bf16x8 v = weight_part<FP4>(a[u % DEPTH][c], scale, f);
                        acc[c] = mfma(v, __builtin_bit_cast(bf16x8, hi[u % DEPTH][f]), acc[c]);
                        acc[c] = mfma(v, __builtin_bit_cast(bf16x8, lo[u % DEPTH][f]), acc[c]);
                    }
                }
            }
            load(u % DEPTH);
        }
        // a token that did not pick the expert takes nothing from it, not even what is not a number
        bool picked = rl < p.T;
        if (at < n_active && picked) picked = picks.pick[picks.active[at]][rl] >= 0;
#pragma unroll
        for (int c = 0; c < NB; ++c)
            if (picked) sum[c] += acc[c];
    }
#pragma unroll
    for (int c = 0; c < NB; ++c) *reinterpret_cast<f32x4*>(&sums[wave][c][rl * 16 + 4 * g]) = sum[c];
    __syncthreads();
    // thread: columns n, n + 32, .. of a token, or one of 16 columns (NB = 1)
    constexpr int WIDE = NB > 1 ? 32 : 16, EACH = NB > 1 ? NB / 2 : 1, COLUMNS = NB * 16;
    const int t = tid / WIDE, n = tid % WIDE;
    float v[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        v[j] = 0.f;
        const int col = j * 32 + n;
        if (t < FEW_TOKENS)
#pragma unroll
            for (int q = 0; q < WAVES; ++q) v[j] += sums[q][col >> 4][t * 16 + (col & 15)];
    }
    if (p.shares > 1) {
        float* const all = p.partial + (size_t)columns * p.shares * (FEW_TOKENS * COLUMNS);
        if (t < FEW_TOKENS)
#pragma unroll
            for (int j = 0; j < EACH; ++j)
                __hip_atomic_store(&all[(size_t)share * (FEW_TOKENS * COLUMNS) + t * COLUMNS + j * 32 + n], v[j], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): they have arrived
        __syncthreads();
        if (tid == 0) last = __hip_atomic_fetch_add(&p.arrived[columns], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == p.shares - 1;
        __syncthreads();
        if (!last || t >= p.T) return;
#pragma unroll
        for (int j = 0; j < EACH; ++j) v[j] = 0.f;
        constexpr int AHEAD = 8;   // loads on their way
        for (int q0 = 0; q0 < p.shares; q0 += AHEAD) {
            float u[AHEAD][EACH];
#pragma unroll
            for (int q = 0; q < AHEAD; ++q)
#pragma unroll
                for (int j = 0; j < EACH; ++j)
                    u[q][j] = __hip_atomic_load(&all[(size_t)min(q0 + q, p.shares - 1) * (FEW_TOKENS * COLUMNS) + t * COLUMNS + j * 32 + n],
                                                __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
            for (int q = 0; q < AHEAD; ++q)
#pragma unroll
                for (int j = 0; j < EACH; ++j) v[j] += q0 + q < p.shares ? u[q][j] : 0.f;
        }
    }
    if (t >= p.T) return;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        const size_t o = (size_t)t * p.H + columns * COLUMNS + j * 32 + n;
        if (p.out_fp32) *reinterpret_cast<float*>(p.out + o * 4) = v[j];
        else *reinterpret_cast<__bf16*>(p.out + o * 2) = (__bf16)v[j];
    }
}

// Tasks of the down launch.
int64_t down_tasks(const moe_shape& s, const bool fp4) {
    const int64_t active = std::min<int64_t>(s.E, (int64_t)s.T * s.top_k) + s.num_shared;
    return active * ((s.F + (fp4 ? 511 : 127)) / (fp4 ? 512 : 128));
}

}  // namespace

size_t few_x_bytes(const moe_shape& s) { return (size_t)s.T * ((s.H + 127) / 128 * 128) * 2; }
int few_h_row(const moe_shape& s) { return (s.F + 127) / 128 * 512; }   // bytes
size_t few_h_bytes(const moe_shape& s) { return (size_t)s.T * (s.top_k + s.num_shared) * few_h_row(s); }
size_t few_partial_bytes(const moe_shape& s) { return (size_t)s.H * FEW_SHARES * FEW_TOKENS * 4; }

// x in LDS (whole layers, us, with and without: 8 experts, H = 512, one token 12.9, 15.6; 8 experts, H = 4096, 7 tokens 132, 143; 64 + 2 experts, H = 2048, 16 tokens
// 68.4, 69.9), and then a gate matrix of up to 128 KiB with it, which every workgroup reads (inside and in a launch of its own: 64 KiB 51.3, 54.6; 256 KiB,
// 64 experts, one token 29.6, 25.0; 1.6 MiB 107, 48).
bool few_x_in_lds(const moe_shape& s) { return few_x_bytes(s) <= FEW_X_LDS; }
bool few_routes_inside(const moe_shape& s) { return few_x_in_lds(s) && (int64_t)((s.E + 15) / 16) * s.H * 32 <= 128 << 10; }

// Workgroups to the logits of 16 experts: one to 1024 of H where there is more x than LDS holds (whole layers, us, one and H / 1024: 160 + 2 experts, H = 5120, 16 tokens
// 206, 202.5; 8 experts, H = 4096, 16 tokens 153.4, 151.1; with less x the sums cost more: 64 + 2 experts, one token 24.4, 25.0).
int few_logit_shares(const moe_shape& s) { return few_x_in_lds(s) ? 1 : std::max(1, std::min(s.H / 1024, 8)); }

// Columns of a down workgroup.  Few tasks: 16, so that there are workgroups enough and each has little to do one after the other; else 64, where a load of h
// meets four of weights, and 128 in the longest launches on MXFP4.  Whole layers, us; tasks x columns / 64:
//   16 and 64: 8 experts, H = 512, one token 12.6, 14.3 (128), 16 tokens bf16 16.2, 17.6 (512); 64 + 2 experts, H = 2048, one token 24.7, 26.3 (768), bf16 43.8, 39.2
//     (2816); H = 2048, 16 tokens 33.4, 31.1 (2048); 8 experts, H = 4096, one token 59.7, 51.1 (3584)
//   64 and 128: 160 + 2 experts, H = 5120, 7 tokens 115, 113 (10560), 16 tokens 207, 201 (23520); 8 experts, H = 4096, 16 tokens 159, 154 (14336), but bf16 432, 437;
//     64 + 2 experts, 16 tokens, bf16 154, 159
int few_down_columns(const moe_shape& s, bool fp4) {
    const int64_t work = down_tasks(s, fp4) * (s.H / 64);
    return work <= 1024 ? 16 : (fp4 && work >= 8192 && s.H % 128 == 0 ? 128 : 64);
}
// Workgroups that share columns: as many as fill the chip (a CU holds one), but one to up to eight tasks, and more to four of MXFP4, which are four times as long, or
// eight of bf16 (64 + 2 experts, 16 tokens, bf16, at most 8 and 32 shares: 171, 159 us; 8 experts, H = 512, 16 tokens, 16 tasks of MXFP4 by eight and by four 17.2, 15.5; 8
// tasks, bf16, in one and two shares 16.4, 17.4; 64 + 2 experts, one token, in 256 and 384 workgroups 24.8, 29.1).
int few_shares(const moe_shape& s, bool fp4) {
    const int64_t tasks = down_tasks(s, fp4), each = fp4 ? WAVES / 2 : WAVES;
    if (tasks <= WAVES) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)FEW_SHARES, 256 / (s.H / few_down_columns(s, fp4)), (tasks + each - 1) / each}));
}

hipError_t few_init() {
    const auto to = hipFuncAttributeMaxDynamicSharedMemorySize;
    for (const void* k : {reinterpret_cast<const void*>(&few_up_kernel<true, true, true>), reinterpret_cast<const void*>(&few_up_kernel<true, false, true>),
                          reinterpret_cast<const void*>(&few_up_kernel<false, true, true>), reinterpret_cast<const void*>(&few_up_kernel<false, false, true>)})
        if (const hipError_t e = hipFuncSetAttribute(k, to, FEW_X_LDS)) return e;
    return hipSuccess;
}

namespace {

template <bool FP4, bool NT>
hipError_t launch(const FewArgs& a, hipStream_t st) {
    const dim3 block(WAVES * 64);
    if (a.logits) {
        const int blocks = (a.E + 15) / 16, copies = a.x_in_lds ? 0 : (a.T * (a.H / 8) + LOGIT_WAVES * 64 - 1) / (LOGIT_WAVES * 64);
        hipLaunchKernelGGL(few_logits_kernel<FP4>, dim3((unsigned)(blocks * a.logit_shares + copies)), dim3(LOGIT_WAVES * 64), 0, st, a);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    // Gate/up: a workgroup to an item where all are on the chip at once, two to a CU (64 + 2 experts, one token, 352 items, whole layer 25.0 us; 256 workgroups
    // 25.5), else 256 that take several, whose loads then run on into the next one (160 + 2 experts, one token, 384 items, of which a CU holds one at a
    // time, 48.0 and 42.3 us; 64 + 2 experts, 7 tokens, 1936 items 77, 48).
    const int64_t active = std::min<int64_t>(a.E, (int64_t)a.T * a.k) + a.Ns, items = active * (a.F / (a.x_in_lds ? 32 : 64));
    const bool two = !a.x_in_lds || a.x_bytes <= FEW_X_TWO;
    const dim3 up((unsigned)(two && items <= 512 ? items : std::min<int64_t>(items, 256))), down((unsigned)(a.H / a.down_columns * a.shares));
    if (a.x_in_lds) hipLaunchKernelGGL((few_up_kernel<FP4, NT, true>), up, block, (unsigned)a.x_bytes, st, a);
    else hipLaunchKernelGGL((few_up_kernel<FP4, NT, false>), up, block, 0, st, a);
    if (const hipError_t e = hipGetLastError()) return e;
    if (a.down_columns == 16) hipLaunchKernelGGL((few_down_kernel<FP4, NT, 1>), down, block, 0, st, a);
    else if (a.down_columns == 64) hipLaunchKernelGGL((few_down_kernel<FP4, NT, 4>), down, block, 0, st, a);
    else hipLaunchKernelGGL((few_down_kernel<FP4, NT, 8>), down, block, 0, st, a);
    return hipGetLastError();
}

}  // namespace

// nt: lists above 256 MB, which no cache holds from one call to the next (us, without and with: 64 + 2 experts, one token, bf16 43.3, 39.3; 8 experts, H = 4096, 7
// tokens 143, 131; a list of 7 MB 12.9, 13.9).
hipError_t launch_few(const FewArgs& a, bool fp4, hipStream_t st) {
    if (fp4) return a.nt ? launch<true, true>(a, st) : launch<true, false>(a, st);
    return a.nt ? launch<false, true>(a, st) : launch<false, false>(a, st);
}

}  // namespace moe
