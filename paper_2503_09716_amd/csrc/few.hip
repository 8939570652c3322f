// The whole MoE layer for up to 16 tokens in two launches (three where the gate matrix is large), on bf16 or MXFP4 weights.
//
//   few_up_kernel    routes, and leaves h[t, j] = w_tj * silu(x_t W1_e) * (x_t W3_e) for each pick e of token t, and of each shared expert
//   few_down_kernel  out[t] = sum over the picks and the shared experts of h W2_e
// The weight of a pick is part of h, so that the sum over experts is one chain of matrix instructions along a contraction of (experts x F),
// and no launch has to combine.  What a few tokens cost is reading the weights of the experts that they pick, so activations stay as
// they are: x is bf16, and h is kept as two bf16 (16 bits of it), each multiplied with the weights.  4-bit weights become bf16, which
// holds their values exactly, in registers.
//
// A wavefront takes 16 columns: W is the row operand straight from memory, the tokens are the 16 columns of the other one, whether they picked
// the expert or not; what they did not pick is not stored (gate and up) or zero (down).
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

// Logits of 16 experts (block nb) by one wavefront over the sub-tiles first, first + step, ..: lane (rl, g) gets tokens 4g .. 4g+3 of expert rl.
__device__ __forceinline__ f32x4 logits_of(const FewArgs& p, const int nb, const int first, const int step) {
    const int lane = threadIdx.x & 63, rl = lane & 15, g = lane >> 4;
    const char* const xa = p.x + (size_t)min(rl, p.T - 1) * p.H * 2 + g * 16;
    const char* const wb = p.wg + (size_t)nb * (p.H >> 5) * 1024 + rl * 64 + ((g ^ block_swizzle(rl)) << 4);
    const int KS = p.H >> 5;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    constexpr int AHEAD = 8;
    for (int s0 = first; s0 < KS; s0 += step * AHEAD) {
        bf16x8 a[AHEAD], b[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int s = s0 + u * step;
            if (s < KS) {   // wave-uniform
                a[u] = *reinterpret_cast<const bf16x8*>(xa + (size_t)s * 64);
                b[u] = *reinterpret_cast<const bf16x8*>(wb + (size_t)s * 1024);
            } else {
                a[u] = b[u] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) acc = mfma(a[u], b[u], acc);
    }
    return acc;
}

// A large gate matrix: one workgroup to 16 experts, K cut over its wavefronts, sums in wave order.
__global__ __launch_bounds__(WAVES * 64) void few_logits_kernel(const FewArgs p) {
    __shared__ float part[WAVES][256];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const f32x4 acc = logits_of(p, blockIdx.x, wave, WAVES);
#pragma unroll
    for (int r = 0; r < 4; ++r) part[wave][(4 * (lane >> 4) + r) * 16 + (lane & 15)] = acc[r];
    __syncthreads();
    const int t = tid >> 4;
    if (t >= p.T) return;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += part[w][tid];
    p.logits_out[t * p.ep + blockIdx.x * 16 + (tid & 15)] = v;
}

// Softmax and top-k of all tokens, by four wavefronts, into idx and w [16][16] in LDS.
template <int NV>
__device__ __forceinline__ void select(const FewArgs& p, const float* logits, const int stride, int32_t* idx, float* w) {
    const int lane = threadIdx.x & 63, row = lane & 15, t = (threadIdx.x >> 6) * 4 + (lane >> 4);
    float v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = row + 16 * i;
        v[i] = e < p.E ? logits[min(t, p.T - 1) * stride + e] + (p.bias ? p.bias[e] : 0.f) : -INFINITY;
    }
    int e;
    float we;
    route_select_row16<NV>(v, row, p.E, p.k, p.renorm, p.scale, e, we);
    if (t < p.T && row < p.k) {
        idx[t * p.k + row] = e;
        w[t * p.k + row] = we;
    }
}

// Gate and up, and the router before them.  A workgroup takes 32 columns of both matrices of a picked or shared expert at a time, its wavefronts every
// eighth sub-tile of the contraction (eight together read consecutive blocks), and their sums meet in LDS.  The loads of the next steps, the
// next columns' among them, are on their way while one is multiplied.
template <bool FP4, bool NT>
__global__ __launch_bounds__(WAVES * 64) void few_up_kernel(const FewArgs p) {
    // the logits and their parts, then the wavefronts' sums (two places in turn: one barrier each)
    __shared__ __attribute__((aligned(16))) float room[2][WAVES][2][2][256];
    __shared__ __attribute__((aligned(16))) Picks picks;
    __shared__ int32_t idx[FEW_TOKENS * FEW_TOP_K];
    __shared__ float w[FEW_TOKENS * FEW_TOP_K];
    __shared__ const char* matrix[2][256];   // of every expert
    float* const logits = &room[0][0][0][0][0];
    float(*const part)[256] = room[1][0][0];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), rl = lane & 15, g = lane >> 4;
    const int experts = p.E + p.Ns;
    if (tid < 256)
#pragma unroll
        for (int m = 0; m < 2; ++m) matrix[m][tid] = (const char*)p.weights[m * experts + min(tid, experts - 1)];
    if (!p.logits) {
        // up to 8 blocks of 16 experts side by side; what wavefronts are left share the contraction, and are added in order
        const int blocks = (p.E + 15) >> 4;
        int per = WAVES;
        while (per > 1 && WAVES / per < blocks) per >>= 1;
        const int beside = WAVES / per, share = wave / beside;
        for (int nb = wave - share * beside; nb < blocks; nb += beside) {
            const f32x4 acc = logits_of(p, nb, share, per);
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
    const int stride = p.logits ? p.ep : LOGIT_STRIDE;
    if (wave < 4) {
        if (p.E <= 16) select<1>(p, l, stride, idx, w);
        else if (p.E <= 64) select<4>(p, l, stride, idx, w);
        else if (p.E <= 160) select<10>(p, l, stride, idx, w);
        else select<16>(p, l, stride, idx, w);
    }
    __syncthreads();
    gather_picks(picks, idx, p.T, p.k, p.E);
    if (blockIdx.x == 0) {
        const uint32_t* const from = reinterpret_cast<const uint32_t*>(&picks);
        for (int i = tid; i < (int)sizeof(Picks) / 4; i += WAVES * 64) reinterpret_cast<uint32_t*>(p.picks)[i] = from[i];
        for (int i = tid; i < p.H / DOWN_COLUMNS; i += WAVES * 64) p.arrived[i] = 0;
    }

    const int units = p.F >> 5, n_active = __builtin_amdgcn_readfirstlane(picks.n);
    const int KT = FP4 ? (p.H + 127) >> 7 : p.H >> 5, groups = (p.H + 511) >> 9, steps = (KT + WAVES - 1) / WAVES;
    const int items = (n_active + p.Ns) * units, mine = items > (int)blockIdx.x ? (items - 1 - blockIdx.x) / gridDim.x + 1 : 0;
    const char* const xa = p.x + (size_t)min(rl, p.T - 1) * p.H * 2 + g * (FP4 ? 64 : 16);
    const uint32_t lane_w = (uint32_t)(rl * 64 + ((g ^ block_swizzle(rl)) << 4)), lane_s = (uint32_t)(rl * 16 + g * 4);
    constexpr int DEPTH = FP4 ? 2 : 4, PARTS = FP4 ? 4 : 1, XSTEP = FP4 ? 256 : 64;
    u32x4 a[DEPTH][2][2], x[DEPTH][PARTS];
    uint32_t sc[DEPTH][2][2];
    // what is asked for next: step `ls` of item blockIdx.x + li * gridDim.x, its expert's matrices and columns
    int li = 0, ls = 0;
    const char *lw[2] = {nullptr, nullptr};
    auto load = [&](const int slot) __attribute__((always_inline)) {
        if (li >= mine) return;
        const int item = blockIdx.x + li * gridDim.x, at = item / units, unit = item - at * units;
        if (ls == 0) {
            const int e = at < n_active ? picks.active[at] : p.E + at - n_active;
            lw[0] = uniform(matrix[0][e]);
            lw[1] = uniform(matrix[1][e]);
        }
        const int t = wave + ls * WAVES;
        if (t < KT) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int block = unit * 2 + c;
                    a[slot][m][c] = load_piece<NT>(lw[m] + ((size_t)block * KT + t) * 1024 + lane_w);
                    if (FP4) sc[slot][m][c] = load_word(lw[m] + p.up_scales_at + ((size_t)block * groups + (t >> 2)) * 256 + lane_s);
                }
#pragma unroll
            for (int f = 0; f < PARTS; ++f) {
                // past H (a multiple of 64) the weights are zero; x there is not read
                const bool in = !FP4 || t * 128 + g * 32 < p.H;
                x[slot][f] = in ? load_piece(xa + (size_t)t * XSTEP + f * 16) : u32x4{0u, 0u, 0u, 0u};
            }
        }
        if (++ls == steps) { ls = 0; ++li; }
    };
#pragma unroll
    for (int u = 0; u < DEPTH; ++u) load(u);
    f32x4 acc[2][2] = {};
    int i = 0, s = 0;   // item and step that are multiplied next
    while (i < mine) {
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            if (i >= mine) break;
            if (wave + s * WAVES < KT) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float scale = FP4 ? scale_of(sc[u][m][c], wave) : 0.f;
#pragma unroll
                        for (int f = 0; f < PARTS; ++f) acc[m][c] = mfma(weight_part<FP4>(a[u][m][c], scale, f), __builtin_bit_cast(bf16x8, x[u][f]), acc[m][c]);
                    }
            }
            load(u);
            if (++s < steps) continue;
            // the item's last step: lane (rl, g) has columns 4 g + r of 16 of token rl
            float(*const sums)[2][2][256] = room[i & 1];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    *reinterpret_cast<f32x4*>(&sums[wave][m][c][rl * 16 + 4 * g]) = acc[m][c];
                    acc[m][c] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
            __syncthreads();
            {
                const int item = blockIdx.x + i * gridDim.x, at = item / units, unit = item - at * units;
                const int e = at < n_active ? picks.active[at] : p.E + at - n_active;
                const int t = tid >> 5, c = tid >> 4 & 1, n = tid & 15;   // token, half and column of the unit
                int row = -1;
                float weight = 1.f;
                if (t < p.T) {
                    if (at >= n_active) row = p.T * (p.k + at - n_active) + t;
                    else if (picks.pick[e][t] >= 0) {
                        row = t * p.k + picks.pick[e][t];
                        weight = w[row];
                    }
                }
                if (row >= 0) {
                    float gate = 0.f, up = 0.f;
#pragma unroll
                    for (int q = 0; q < WAVES; ++q) {
                        gate += sums[q][0][c][t * 16 + n];
                        up += sums[q][1][c][t * 16 + n];
                    }
                    const float v = weight * (gate / (1.0f + __expf(-gate)) * up);
                    const __bf16 hi = (__bf16)v;
                    char* const to = p.h + ((size_t)row * (p.F >> 3) + unit * 4 + c * 2 + (n >> 3)) * 32 + (n & 7) * 2;
                    *reinterpret_cast<__bf16*>(to) = hi;
                    *reinterpret_cast<__bf16*>(to + 16) = __builtin_isfinite((float)hi) ? (__bf16)(v - (float)hi) : (__bf16)0.0f;
                }
            }
            s = 0;
            ++i;
        }
    }
}

// Down: 64 columns to a workgroup, and a share of all sub-tiles of all picked and shared experts, one after the other; its wavefronts take every eighth of
// them.  The shares' sums meet in the workgroup that comes last, which adds them in order: no workgroup waits for another.  Sums and
// counter pass by the L2s, each of which only its own XCD sees.
template <bool FP4, bool NT>
__global__ __launch_bounds__(WAVES * 64) void few_down_kernel(const FewArgs p) {
    __shared__ __attribute__((aligned(16))) Picks picks;
    __shared__ __attribute__((aligned(16))) float sums[WAVES][4][256];
    __shared__ const char* matrix[256];   // of every expert
    __shared__ int last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), rl = lane & 15, g = lane >> 4;
    const int experts = p.E + p.Ns;
    if (tid < 256) matrix[tid] = (const char*)p.weights[2 * experts + min(tid, experts - 1)];
    const u32x4* const from_up = reinterpret_cast<const u32x4*>(p.picks);
    for (int i = tid; i < (int)sizeof(Picks) / 16; i += WAVES * 64) reinterpret_cast<u32x4*>(&picks)[i] = from_up[i];
    __syncthreads();
    const int n_active = __builtin_amdgcn_readfirstlane(picks.n);
    const int share = blockIdx.x % p.shares, columns = blockIdx.x / p.shares;
    const int KT = FP4 ? (p.F + 127) >> 7 : p.F >> 5, groups = (p.F + 511) >> 9;
    constexpr int DEPTH = FP4 ? 2 : 4, PARTS = FP4 ? 4 : 1, HSTEP = FP4 ? 512 : 128, NB = DOWN_COLUMNS / 16;
    const uint32_t lane_w = (uint32_t)(rl * 64 + ((g ^ block_swizzle(rl)) << 4)), lane_s = (uint32_t)(rl * 16 + g * 4);
    const int total = (n_active + p.Ns) * KT;
    const int from = (int)((int64_t)total * share / p.shares), to = (int)((int64_t)total * (share + 1) / p.shares);
    u32x4 a[DEPTH][NB], hi[DEPTH][PARTS], lo[DEPTH][PARTS];
    uint32_t sc[DEPTH][NB];
    int expert[DEPTH];       // which in the list; -1: none
    bool picked[DEPTH];
    int lc = from + wave, le = lc / KT, lt = lc - le * KT;   // sub-tile lt of the le-th expert is asked for next
    auto load = [&](const int slot) __attribute__((always_inline)) {
        expert[slot] = -1;
        picked[slot] = false;
        if (lc >= to) return;
        expert[slot] = le;
        const int e = __builtin_amdgcn_readfirstlane(le < n_active ? picks.active[le] : p.E + le - n_active);
        const char* const w2 = uniform(matrix[e]);
#pragma unroll
        for (int c = 0; c < NB; ++c) {
            const int block = columns * NB + c;
            a[slot][c] = load_piece<NT>(w2 + ((size_t)block * KT + lt) * 1024 + lane_w);
            if (FP4) sc[slot][c] = load_word(w2 + p.down_scales_at + ((size_t)block * groups + (lt >> 2)) * 256 + lane_s) >> (8 * (lt & 3));
        }
        int row = -1;
        if (rl < p.T) {
            if (le >= n_active) row = p.T * (p.k + le - n_active) + rl;
            else if (const int j = picks.pick[e][rl]; j >= 0) row = rl * p.k + j;
        }
        picked[slot] = row >= 0;
        const bool in = row >= 0 && (!FP4 || lt * 128 + g * 32 < p.F);
        const char* const from_h = p.h + (size_t)max(row, 0) * p.F * 4 + (size_t)lt * HSTEP + g * (FP4 ? 128 : 32);
#pragma unroll
        for (int f = 0; f < PARTS; ++f) {
            hi[slot][f] = in ? load_piece(from_h + f * 32) : u32x4{0u, 0u, 0u, 0u};
            lo[slot][f] = in ? load_piece(from_h + f * 32 + 16) : u32x4{0u, 0u, 0u, 0u};
        }
        lc += WAVES;
        for (lt += WAVES; lt >= KT; lt -= KT) ++le;
    };
#pragma unroll
    for (int u = 0; u < DEPTH; ++u) load(u);
    // each expert's sum by itself: a token that did not pick it takes nothing from it, not even what is not a number
    f32x4 acc[NB] = {}, sum[NB] = {};
    int now = expert[0];
    bool now_picked = picked[0];
    auto flush = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < NB; ++c) {
            if (now_picked) sum[c] += acc[c];
            acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    for (bool more = expert[0] >= 0; more;) {
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            if (expert[u] < 0) { more = false; break; }
            if (expert[u] != now) {
                flush();
                now = expert[u];
                now_picked = picked[u];
            }
#pragma unroll
            for (int c = 0; c < NB; ++c) {
                const float scale = FP4 ? scale_of(sc[u][c], 0) : 0.f;
#pragma unroll
                for (int f = 0; f < PARTS; ++f) {
                    const bf16x8 v = weight_part<FP4>(a[u][c], scale, f);
                    acc[c] = mfma(v, __builtin_bit_cast(bf16x8, hi[u][f]), acc[c]);
                    acc[c] = mfma(v, __builtin_bit_cast(bf16x8, lo[u][f]), acc[c]);
                }
            }
            load(u);
        }
    }
    flush();
#pragma unroll
    for (int c = 0; c < NB; ++c) *reinterpret_cast<f32x4*>(&sums[wave][c][rl * 16 + 4 * g]) = sum[c];
    __syncthreads();
    // thread: columns n and n + 32 of a token
    const int t = tid >> 5, n = tid & 31;
    float v[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int q = 0; q < WAVES; ++q) v[j] += sums[q][j * 2 + (n >> 4)][t * 16 + (n & 15)];
    if (p.shares > 1) {
        float* const mine = p.partial + ((size_t)columns * p.shares + share) * (FEW_TOKENS * DOWN_COLUMNS);
#pragma unroll
        for (int j = 0; j < 2; ++j) __hip_atomic_store(&mine[t * DOWN_COLUMNS + j * 32 + n], v[j], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): they have arrived
        __syncthreads();
        if (tid == 0) last = __hip_atomic_fetch_add(&p.arrived[columns], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == p.shares - 1;
        __syncthreads();
        if (!last) return;
        const float* const all = p.partial + (size_t)columns * p.shares * (FEW_TOKENS * DOWN_COLUMNS);
        v[0] = v[1] = 0.f;
        constexpr int AHEAD = 8;   // loads on their way
        for (int q0 = 0; q0 < p.shares; q0 += AHEAD) {
            float u[AHEAD][2];
#pragma unroll
            for (int q = 0; q < AHEAD; ++q)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    u[q][j] = __hip_atomic_load(&all[(size_t)min(q0 + q, p.shares - 1) * (FEW_TOKENS * DOWN_COLUMNS) + t * DOWN_COLUMNS + j * 32 + n],
                                                __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
            for (int q = 0; q < AHEAD; ++q)
#pragma unroll
                for (int j = 0; j < 2; ++j) v[j] += q0 + q < p.shares ? u[q][j] : 0.f;
        }
    }
    if (t >= p.T) return;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const size_t o = (size_t)t * p.H + columns * DOWN_COLUMNS + j * 32 + n;
        if (p.out_fp32) *reinterpret_cast<float*>(p.out + o * 4) = v[j];
        else *reinterpret_cast<__bf16*>(p.out + o * 2) = (__bf16)v[j];
    }
}

}  // namespace

int few_shares(const moe_shape& s, bool fp4) {
    const int64_t active = std::min<int64_t>(s.E, (int64_t)s.T * s.top_k) + s.num_shared, sub_tiles = active * ((s.F + (fp4 ? 127 : 31)) / (fp4 ? 128 : 32));
    return (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)FEW_SHARES, 256 / (s.H / DOWN_COLUMNS), (sub_tiles + WAVES - 1) / WAVES}));
}

size_t few_h_bytes(const moe_shape& s) { return (size_t)s.T * (s.top_k + s.num_shared) * s.F * 4; }
size_t few_partial_bytes(const moe_shape& s) { return (size_t)(s.H / DOWN_COLUMNS) * FEW_SHARES * FEW_TOKENS * DOWN_COLUMNS * 4; }

bool few_routes_inside(const moe_shape& s) { return (int64_t)((s.E + 15) / 16) * s.H * 32 <= 128 << 10; }

hipError_t launch_few(const FewArgs& a, bool fp4, hipStream_t st) {
    if (a.logits) {
        hipLaunchKernelGGL(few_logits_kernel, dim3((unsigned)((a.E + 15) / 16)), dim3(WAVES * 64), 0, st, a);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    const int64_t active = std::min<int64_t>(a.E, (int64_t)a.T * a.k) + a.Ns, items = active * (a.F / 32);
    const dim3 up((unsigned)std::min<int64_t>(512, items)), down((unsigned)(a.H / DOWN_COLUMNS * a.shares)), block(WAVES * 64);
#define FEW(FP4_, NT_)                                                                      \
    do {                                                                                    \
        hipLaunchKernelGGL((few_up_kernel<FP4_, NT_>), up, block, 0, st, a);                \
        if (const hipError_t e = hipGetLastError()) return e;                               \
        hipLaunchKernelGGL((few_down_kernel<FP4_, NT_>), down, block, 0, st, a);            \
    } while (0)
    if (fp4 && a.nt) FEW(true, true);
    else if (fp4) FEW(true, false);
    else if (a.nt) FEW(false, true);
    else FEW(false, false);
#undef FEW
    return hipGetLastError();
}

}  // namespace moe
