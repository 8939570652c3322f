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

// Where the picks of the tokens sit: pick[e][t] = j of token t's pick e, or -1; the experts that have any, ascending.
struct Picks {
    int8_t pick[256][FEW_TOKENS];
    int16_t active[256];
    int32_t n;
};

// By a whole workgroup of at least 256 threads, from idx [T][k] in LDS or global memory.
template <class Idx>
__device__ __forceinline__ void gather_picks(Picks& s, const Idx idx, const int T, const int k, const int E) {
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

template <bool FP4>
__global__ __launch_bounds__(WAVES * 64) void few_up_kernel(const FewArgs p) {
    __shared__ float logits[FEW_TOKENS * LOGIT_STRIDE];
    __shared__ __attribute__((aligned(16))) Picks picks;
    __shared__ int32_t idx[FEW_TOKENS * FEW_TOP_K];
    __shared__ float w[FEW_TOKENS * FEW_TOP_K];
    __shared__ float part[WAVES][256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), rl = lane & 15, g = lane >> 4;
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
    if (blockIdx.x == 0)
        for (int i = tid; i < p.T * p.k; i += WAVES * 64) p.idx[i] = idx[i];

    const int units = p.F >> 4, experts = p.E + p.Ns;
    const int KT = FP4 ? (p.H + 127) >> 7 : p.H >> 5, groups = (p.H + 511) >> 9;
    const char* const xa = p.x + (size_t)min(rl, p.T - 1) * p.H * 2 + g * (FP4 ? 64 : 16);
    constexpr int DEPTH = FP4 ? 4 : 8, PARTS = FP4 ? 4 : 1, XSTEP = FP4 ? 256 : 64;
    for (int item = blockIdx.x * WAVES + wave; item < (picks.n + p.Ns) * units; item += gridDim.x * WAVES) {
        const int a = item / units, unit = item - a * units;
        const int e = a < picks.n ? picks.active[a] : p.E + a - picks.n;
        const char* const w1 = (const char*)p.weights[e];
        const char* const w3 = (const char*)p.weights[experts + e];
        const size_t at = (size_t)unit * KT * 1024 + rl * 64 + ((g ^ block_swizzle(rl)) << 4);
        const size_t sat = (size_t)p.up_scales_at + (size_t)unit * groups * 256 + rl * 16 + g * 4;
        f32x4 ag = {0.f, 0.f, 0.f, 0.f}, au = {0.f, 0.f, 0.f, 0.f};
        for (int t0 = 0; t0 < KT; t0 += DEPTH) {
            u32x4 a1[DEPTH], a3[DEPTH], b[DEPTH][PARTS];
            uint32_t s1 = 0, s3 = 0;
            if (FP4) {
                s1 = *reinterpret_cast<const uint32_t*>(w1 + sat + (t0 >> 2) * 256);
                s3 = *reinterpret_cast<const uint32_t*>(w3 + sat + (t0 >> 2) * 256);
            }
#pragma unroll
            for (int u = 0; u < DEPTH; ++u) {
                const int t = min(t0 + u, KT - 1);
                a1[u] = *reinterpret_cast<const u32x4*>(w1 + at + (size_t)t * 1024);
                a3[u] = *reinterpret_cast<const u32x4*>(w3 + at + (size_t)t * 1024);
#pragma unroll
                for (int f = 0; f < PARTS; ++f) {
                    // past H (a multiple of 64) the weights are zero; x there is not read
                    const bool in = t0 + u < KT && (!FP4 || t * 128 + g * 32 < p.H);
                    b[u][f] = in ? *reinterpret_cast<const u32x4*>(xa + (size_t)t * XSTEP + f * 16) : u32x4{0u, 0u, 0u, 0u};
                }
            }
#pragma unroll
            for (int u = 0; u < DEPTH; ++u) {
                if (t0 + u >= KT) break;
                const float c1 = FP4 ? scale_of(s1, u) : 0.f, c3 = FP4 ? scale_of(s3, u) : 0.f;
#pragma unroll
                for (int f = 0; f < PARTS; ++f) {
                    ag = mfma(weight_part<FP4>(a1[u], c1, f), __builtin_bit_cast(bf16x8, b[u][f]), ag);
                    au = mfma(weight_part<FP4>(a3[u], c3, f), __builtin_bit_cast(bf16x8, b[u][f]), au);
                }
            }
        }
        // columns 16 unit + 4 g + r of token rl
        int row = -1;
        float weight = 1.f;
        if (rl < p.T) {
            if (a >= picks.n) row = p.T * (p.k + a - picks.n) + rl;
            else if (picks.pick[e][rl] >= 0) {
                row = rl * p.k + picks.pick[e][rl];
                weight = w[row];
            }
        }
        if (row < 0) continue;
        bf16x4 hi, lo;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float v = weight * (ag[r] / (1.0f + __expf(-ag[r])) * au[r]);
            hi[r] = (__bf16)v;
            lo[r] = __builtin_isfinite((float)hi[r]) ? (__bf16)(v - (float)hi[r]) : (__bf16)0.0f;
        }
        char* const to = p.h + ((size_t)row * (p.F >> 3) + unit * 2 + (g >> 1)) * 32 + (g & 1) * 8;
        *reinterpret_cast<bf16x4*>(to) = hi;
        *reinterpret_cast<bf16x4*>(to + 16) = lo;
    }
}

template <bool FP4>
__global__ __launch_bounds__(WAVES * 64) void few_down_kernel(const FewArgs p) {
    __shared__ __attribute__((aligned(16))) Picks picks;
    __shared__ float part[WAVES][256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), rl = lane & 15, g = lane >> 4;
    gather_picks(picks, p.idx, p.T, p.k, p.E);
    const int unit = blockIdx.x, experts = p.E + p.Ns;
    const int KT = FP4 ? (p.F + 127) >> 7 : p.F >> 5, groups = (p.F + 511) >> 9;
    const size_t at = (size_t)unit * KT * 1024 + rl * 64 + ((g ^ block_swizzle(rl)) << 4);
    const size_t sat = (size_t)p.down_scales_at + (size_t)unit * groups * 256 + rl * 16 + g * 4;
    constexpr int DEPTH = FP4 ? 2 : 8, PARTS = FP4 ? 4 : 1, HSTEP = FP4 ? 512 : 128;
    // all experts' sub-tiles one after the other, cut evenly over the wavefronts
    const int total = (picks.n + p.Ns) * KT;
    const int from = (int)((int64_t)total * wave / WAVES), to = (int)((int64_t)total * (wave + 1) / WAVES);
    // each expert's sum by itself: a token that did not pick it takes nothing from it, not even what is not a number
    f32x4 acc = {0.f, 0.f, 0.f, 0.f}, sum = {0.f, 0.f, 0.f, 0.f};
    for (int c0 = from; c0 < to; c0 += DEPTH) {
        u32x4 a[DEPTH], hi[DEPTH][PARTS], lo[DEPTH][PARTS];
        uint32_t s[DEPTH];
        bool picked[DEPTH];
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            const int c = min(c0 + u, to - 1), i = c / KT, t = c - i * KT;
            const int e = i < picks.n ? picks.active[i] : p.E + i - picks.n;
            const char* const w2 = (const char*)p.weights[2 * experts + e];
            a[u] = *reinterpret_cast<const u32x4*>(w2 + at + (size_t)t * 1024);
            s[u] = FP4 ? *reinterpret_cast<const uint32_t*>(w2 + sat + (t >> 2) * 256) >> (8 * (t & 3)) : 0u;
            int row = -1;
            if (rl < p.T && c0 + u < to) {
                if (i >= picks.n) row = p.T * (p.k + i - picks.n) + rl;
                else if (picks.pick[e][rl] >= 0) row = rl * p.k + picks.pick[e][rl];
            }
            picked[u] = row >= 0;
            if (FP4 && t * 128 + g * 32 >= p.F) row = -1;
            const char* const from_h = p.h + (size_t)max(row, 0) * p.F * 4 + (size_t)t * HSTEP + g * (FP4 ? 128 : 32);
#pragma unroll
            for (int f = 0; f < PARTS; ++f) {
                hi[u][f] = row >= 0 ? *reinterpret_cast<const u32x4*>(from_h + f * 32) : u32x4{0u, 0u, 0u, 0u};
                lo[u][f] = row >= 0 ? *reinterpret_cast<const u32x4*>(from_h + f * 32 + 16) : u32x4{0u, 0u, 0u, 0u};
            }
        }
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            if (c0 + u >= to) break;
            const float scale = FP4 ? scale_of(s[u], 0) : 0.f;
#pragma unroll
            for (int f = 0; f < PARTS; ++f) {
                const bf16x8 v = weight_part<FP4>(a[u], scale, f);
                acc = mfma(v, __builtin_bit_cast(bf16x8, hi[u][f]), acc);
                acc = mfma(v, __builtin_bit_cast(bf16x8, lo[u][f]), acc);
            }
            if (c0 + u == to - 1 || (c0 + u + 1) % KT == 0) {
                if (picked[u]) sum += acc;
                acc = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) part[wave][rl * 16 + 4 * g + r] = sum[r];
    __syncthreads();
    const int t = tid >> 4;
    if (t >= p.T) return;
    float v = 0.f;
#pragma unroll
    for (int q = 0; q < WAVES; ++q) v += part[q][tid];
    const size_t o = (size_t)t * p.H + unit * 16 + (tid & 15);
    if (p.out_fp32) *reinterpret_cast<float*>(p.out + o * 4) = v;
    else *reinterpret_cast<__bf16*>(p.out + o * 2) = (__bf16)v;
}

}  // namespace

size_t few_h_bytes(const moe_shape& s) { return (size_t)s.T * (s.top_k + s.num_shared) * s.F * 4; }

bool few_routes_inside(const moe_shape& s) { return (int64_t)s.E * s.H * 2 <= 256 << 10; }

hipError_t launch_few(const FewArgs& a, bool fp4, hipStream_t st) {
    if (a.logits) {
        hipLaunchKernelGGL(few_logits_kernel, dim3((unsigned)((a.E + 15) / 16)), dim3(WAVES * 64), 0, st, a);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    const int64_t active = std::min<int64_t>(a.E, (int64_t)a.T * a.k) + a.Ns, items = active * (a.F / 16);
    const dim3 up((unsigned)std::min<int64_t>(512, (items + WAVES - 1) / WAVES)), down((unsigned)(a.H / 16)), block(WAVES * 64);
    if (fp4) hipLaunchKernelGGL(few_up_kernel<true>, up, block, 0, st, a);
    else hipLaunchKernelGGL(few_up_kernel<false>, up, block, 0, st, a);
    if (const hipError_t e = hipGetLastError()) return e;
    if (fp4) hipLaunchKernelGGL(few_down_kernel<true>, down, block, 0, st, a);
    else hipLaunchKernelGGL(few_down_kernel<false>, down, block, 0, st, a);
    return hipGetLastError();
}

}  // namespace moe
