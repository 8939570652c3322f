// Balance loss of the router with its per-expert counts and its gradient.
//
// n kept tokens, c_e picks of expert e among them, p_te the softmax of a token's logits, lse_t the logarithm of their sum of
// exponentials:   loss_0 = E sum_e c_e / (k n) mean_t p_te,   loss_1 = mean_t lse_t^2.
// With off_e = E c_e / (k n) - 1 and sum_e p_te = 1:   loss_0 = 1 + mean_t s_t,   s_t = sum_e p_te off_e,
// so a token adds one number to the loss, no sums of p over tokens are kept for each expert, and the gradient hangs on the same s_t:
//   dlogits_te = p_te ((off_e - s_t) balance_coef / n + 2 z_coef / n lse_t)     (the counts have no gradient).
// off is what the gradient of nearly even counts consists of: its numerator E c_e - k n is formed in whole numbers.
//
// Two launches: the counts (integer sums in LDS, one partial histogram to a workgroup: no atomics on global memory but the one
// that finds the last workgroup), then one pass over the logits with a token in a row of 16 lanes.  The last workgroup of the second
// launch adds the workgroups' partial losses in order, in 64 bits.  Few tokens: one workgroup does it all.
// Bound by latency: each launch is a chain of two or three memory round trips, and the gradient waits for all counts.  us (of which
// counts, loss): 256 tokens of 8 experts 6.4 (alone), 5003 of 64 11.1 (5.0, 6.4), 32768 of 160 17.7 (3.9, 14: 42 MB at 3 TB/s, half of it spent on
// 350 vector instructions for every four tokens); without the gradient 6.1, 10.8, 15.1.  A workgroup to
// a CU: with two the last one's wait for all partial losses outgrows what the second saves (20.8).
#include "common.h"
#include "router_rows.h"
#include "train.h"

namespace moe {
namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int MAX_E = 256;

// Picks of the kept tokens in [t0, t1) into hist (LDS, zeroed here); the kept tokens among them.  Ids outside [0, E) are not counted.
// A thread takes a pick at a time, eight loads in flight (a thread that goes through a token's picks one after the other: 5.8 us
// instead of 4.8 for 5003 tokens of 6 picks).
__device__ __forceinline__ int count_picks(int* hist, int* kept, const int32_t* __restrict__ idx, const uint8_t* __restrict__ keep, const int t0, const int t1,
                                           const int E, const int k) {
    for (int e = threadIdx.x; e < MAX_E; e += blockDim.x) hist[e] = 0;
    if (threadIdx.x == 0) *kept = 0;
    __syncthreads();
    const int32_t* const p = idx + (size_t)t0 * k;
    const int n = (t1 - t0) * k;
    const int step = blockDim.x;
    constexpr int AHEAD = 8;
    auto count = [&]<bool KEEP>() {
        for (int i0 = threadIdx.x; i0 < n; i0 += AHEAD * step) {
            uint32_t e[AHEAD];
            uint8_t on[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int i = min(i0 + u * step, n - 1);
                e[u] = p[i];
                on[u] = KEEP ? keep[t0 + i / k] : 1;
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (i0 + u * step < n && on[u] && e[u] < (uint32_t)E) atomicAdd(&hist[e[u]], 1);
        }
    };
    if (keep) count.template operator()<true>();
    else count.template operator()<false>();
    if (keep) {
        int mine = 0;
        for (int t = t0 + threadIdx.x; t < t1; t += step) mine += keep[t] != 0;
        if (mine) atomicAdd(kept, mine);
    } else if (threadIdx.x == 0) {
        *kept = t1 - t0;
    }
    __syncthreads();
    return *kept;
}

__global__ __launch_bounds__(THREADS) void balance_count_kernel(const BalanceArgs a) {
    __shared__ int hist[MAX_E], kept;
    const int t0 = blockIdx.x * a.count_tokens, t1 = min(t0 + a.count_tokens, a.T);
    const int n = count_picks(hist, &kept, a.idx, a.keep, t0, t1, a.E, a.k);
    int32_t* const out = a.partial_counts + (size_t)blockIdx.x * (a.E + 1);
    for (int e = threadIdx.x; e < a.E; e += THREADS) out[e] = hist[e];
    if (threadIdx.x == 0) {
        out[a.E] = n;
        if (blockIdx.x == 0) *a.done = 0;
    }
}

// ALONE: one workgroup, which counts for itself.
template <int NV, bool WIDE, bool ALONE>
__global__ __launch_bounds__(THREADS) void balance_loss_kernel(const BalanceArgs a) {
    __shared__ int hist[MAX_E + 1], kept;
    __shared__ float off[MAX_E];
    __shared__ double sums[2][WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15;
    const int E = a.E;
    const int q0 = blockIdx.x * WAVES + wave, stride = gridDim.x * WAVES;
    float ahead[NV];
    bool kept_here = true;
    auto fetch = [&](const int q) {
        const size_t t = min((int64_t)q * 4 + (lane >> 4), (int64_t)a.T - 1);
        load_row16<NV, WIDE>(ahead, a.logits, t, E, row, -INFINITY);
        if (a.keep) kept_here = a.keep[t];
    };
    fetch(q0);
    if (ALONE) {
        count_picks(hist, &kept, a.idx, a.keep, 0, a.T, E, a.k);
        if (threadIdx.x == 0) hist[E] = kept;
    } else {
        // all threads read the partial histograms: one thread an expert, however many loads it has in flight, costs 3 us more
        for (int e = threadIdx.x; e <= E; e += THREADS) hist[e] = 0;
        __syncthreads();
        const int total = a.count_blocks * (E + 1);
        for (int i0 = threadIdx.x; i0 < total; i0 += 6 * THREADS) {
            int c[6];
#pragma unroll
            for (int u = 0; u < 6; ++u) c[u] = a.partial_counts[min(i0 + u * THREADS, total - 1)];
#pragma unroll
            for (int u = 0; u < 6; ++u)
                if (i0 + u * THREADS < total && c[u]) atomicAdd(&hist[(i0 + u * THREADS) % (E + 1)], c[u]);
        }
    }
    __syncthreads();
    const int n = hist[E];
    const double kn = (double)a.k * n;
    for (int e = threadIdx.x; e < E; e += blockDim.x) {
        off[e] = n ? (float)(((double)hist[e] * E - kn) / kn) : 0.f;
        if (blockIdx.x == 0) a.counts[e] = hist[e];
    }
    __syncthreads();
    float o[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = row16_expert<WIDE>(row, i);
        o[i] = e < E ? off[e] : 0.f;
    }
    const float bal = n ? (float)(a.balance_coef / n) : 0.f, zc = n ? (float)(2.0 * a.z_coef / n) : 0.f;
    double sum_s = 0, sum_z = 0;
    // The first rows are asked for before the counts are known, and each pass asks for the next one's.
    for (int q = q0; q * 4 < a.T; q += stride) {
        const int tok = q * 4 + (lane >> 4), t = min(tok, a.T - 1);
        const bool on = tok < a.T && kept_here;
        float v[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = ahead[i];
        fetch(q + stride);
        float z, s = 0.f;
        const float top = exps_row16<NV>(v, z), rz = 1.0f / z, lse = top + logf(z);
#pragma unroll
        for (int i = 0; i < NV; ++i) s = fmaf(v[i], o[i], s);
        s = row16_sum(s) * rz;
        if (on && row == 0) {
            sum_s += s;
            sum_z += (double)lse * lse;
        }
        const float slope = rz * bal, at = rz * lse * zc;
        if (a.dlogits && tok < a.T) {
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = on ? v[i] * fmaf(o[i] - s, slope, at) : 0.f;
            store_row16<NV, WIDE>(v, a.dlogits, t, E, row);
        }
    }
#pragma unroll
    for (int m = 16; m < 64; m *= 2) {   // the sums sit in lanes 0, 16, 32, 48
        sum_s += __shfl_xor(sum_s, m, 64);
        sum_z += __shfl_xor(sum_z, m, 64);
    }
    if (lane == 0) { sums[0][wave] = sum_s; sums[1][wave] = sum_z; }
    __syncthreads();
    if (threadIdx.x < 2) {
        double v = 0;
        for (int w = 0; w < WAVES; ++w) v += sums[threadIdx.x][w];
        if (ALONE) {
            a.loss[threadIdx.x] = n ? (float)(threadIdx.x ? v / n : 1.0 + v / n) : 0.f;
        } else {
            __hip_atomic_store(&a.partial_loss[2 * blockIdx.x + threadIdx.x], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (ALONE || wave != 0) return;
    // The last workgroup to get here adds up what all have written.  The partial losses are atomic stores past the L2, complete when the
    // count goes up, and atomic loads past it read them: no fence at agent scope, which would write this XCD's L2 back with all of dlogits in
    // it (32768 tokens, 160 experts: 18.6 us instead of 17.6).
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    int before = 0;
    if (lane == 0) before = __hip_atomic_fetch_add(a.done, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__builtin_amdgcn_readfirstlane(before) != (int)gridDim.x - 1) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    double v = 0;
#pragma unroll
    for (int u = 0; u < (2 * BALANCE_LOSS_BLOCKS + 63) / 64; ++u) {   // all in flight
        const int b = lane + 64 * u, n = 2 * (int)gridDim.x;
        const double x = __hip_atomic_load(&a.partial_loss[min(b, n - 1)], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        v += b < n ? x : 0;
    }
#pragma unroll
    for (int m = 2; m < 64; m *= 2) v += __shfl_xor(v, m, 64);   // even lanes the balance terms, odd lanes the z terms
    if (lane < 2) a.loss[lane] = n ? (float)(lane ? v / n : 1.0 + v / n) : 0.f;
}

__global__ void balance_empty_kernel(int E, int32_t* counts, float* loss) {
    for (int e = threadIdx.x; e < E; e += blockDim.x) counts[e] = 0;
    if (threadIdx.x < 2) loss[threadIdx.x] = 0.f;
}

}  // namespace

hipError_t launch_balance_loss(const BalanceArgs& a, hipStream_t st) {
    if (a.T == 0) {
        hipLaunchKernelGGL(balance_empty_kernel, dim3(1), dim3(256), 0, st, a.E, a.counts, a.loss);
        return hipGetLastError();
    }
    const bool wide = wide_rows(a.E, {a.logits, a.dlogits ? a.dlogits : a.logits});
    const int row = (a.E + 63) & ~63;
    const bool alone = a.T <= BALANCE_ALONE_TOKENS && a.T * row <= BALANCE_ALONE_LOGITS && a.T * (row + a.k) <= BALANCE_ALONE;
    if (!alone) hipLaunchKernelGGL(balance_count_kernel, dim3(a.count_blocks), dim3(THREADS), 0, st, a);
    return for_row16(a.E, wide, [&]<int NV, bool WIDE>() {
        if (alone) hipLaunchKernelGGL((balance_loss_kernel<NV, WIDE, true>), dim3(1), dim3(THREADS), 0, st, a);
        else hipLaunchKernelGGL((balance_loss_kernel<NV, WIDE, false>), dim3(a.loss_blocks), dim3(THREADS), 0, st, a);
        return hipGetLastError();
    });
}

}  // namespace moe
