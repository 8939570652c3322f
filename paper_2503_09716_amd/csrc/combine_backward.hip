// Backward pass of the weighted combine: out_t = sum_j w_tj y_row(t,j) (+ y_shared_t) gives
//   dw_tj = <y_row(t,j), dout_t>,   dy_row(t,j) = w_tj dout_t   (and dout_t itself for the shared experts).
// HBM-bound: every row of y is read and, with dy_perm, written once.  W wavefronts take a pair's row; those of a token's pairs are one
// workgroup, so that dout's row comes from memory once.  A row's product is added up in fp32 along each lane, in as many sums as a load has
// elements (memory bounds the kernel either way, and a single sum of H / 64 terms was off by up to that many times more), and then across the
// lanes, once to a row: a thread that took a piece of all of a token's rows would end on a sum across lanes for every 8 elements of each.
// us: 3001 tokens x 2048, k = 6, fp32, weights alone 27.0 (172 MB at 6.4 TB/s), 4096 x 4096, k = 2, fp32 54.6 (302 MB at 5.5), 32768 x 5120,
// k = 6, bf16 795 to 868 by box (4.4 GB at 5.5 to 5.0; a 1 GiB copy 5.1).
#include "common.h"
#include "topk.h"
#include "train.h"

namespace moe {
namespace {

// N consecutive elements of a row.
template <bool F32, int N>
struct Row {
    typedef uint32_t words __attribute__((ext_vector_type(N * (F32 ? 4 : 2) / 4)));
    words v;
    template <bool NT>
    __device__ __forceinline__ void load(const char* row, const int c) {
        const words* const p = reinterpret_cast<const words*>(row) + c;
        v = NT ? __builtin_nontemporal_load(p) : *p;
    }
    __device__ __forceinline__ float operator[](const int i) const {
        return __uint_as_float(F32 ? v[i] : ((i & 1) ? v[i / 2] & 0xffff0000u : v[i / 2] << 16));
    }
};

// LD, ST: y is read, dy written past the caches.
template <bool YF32, bool DF32, bool DY, int W, bool LD, bool ST>
__global__ __launch_bounds__(1024) void combine_backward_kernel(const char* __restrict__ dout, const char* __restrict__ y_perm,
                                                                const int32_t* __restrict__ inv_perm, const float* __restrict__ w, const int k, const int H,
                                                                float* __restrict__ dw, char* __restrict__ dy_perm) {
    constexpr int N = YF32 || DF32 ? 4 : 8;
    __shared__ float part[16];
    const int t = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rows = (blockDim.x >> 6) / W, r = wave / W, sub = wave % W;
    const int n = H / N;
    const char* const d = dout + (size_t)t * H * (DF32 ? 4 : 2);
    for (int j0 = 0; j0 < k; j0 += rows) {
        const int j = j0 + r;
        float sum = 0.f;
        if (j < k) {
            float sums[N] = {};
            const size_t p = (size_t)t * k + j, at = (size_t)inv_perm[p] * H * (YF32 ? 4 : 2);
            const float wj = DY ? w[p] : 0.f;
            // A pieces of the row, all in flight before the first is used: the compiler would move each load behind the branch that needs it
            // (3001 x 2048, k = 6, fp32, weights alone 28.9 us).  As many as the row has, for short ones (20000 x 192, k = 6 with four at a time
            // 66.7 us, one by one 60.7, so 47.6).
            auto pieces = [&]<int A>(const int c0) {
                Row<YF32, N> y[A];
                Row<DF32, N> g[A];
#pragma unroll
                for (int u = 0; u < A; ++u) {
                    const int c = min(c0 + u * W * 64, n - 1);
                    y[u].template load<LD>(y_perm + at, c);
                    g[u].template load<false>(d, c);
                }
                if constexpr (A > 1)
#pragma unroll
                    for (int u = 0; u < A; ++u) asm volatile("" : "+v"(y[u].v), "+v"(g[u].v));
#pragma unroll
                for (int u = 0; u < A; ++u) {
                    const int c = c0 + u * W * 64;
                    if (c >= n) break;
#pragma unroll
                    for (int i = 0; i < N; ++i) sums[i] = fmaf(y[u][i], g[u][i], sums[i]);
                    if (DY) {
                        if (YF32) {
                            f32x4 o;
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[i] = wj * g[u][i];
                            if (ST) __builtin_nontemporal_store(o, reinterpret_cast<f32x4*>(dy_perm + at) + c); else reinterpret_cast<f32x4*>(dy_perm + at)[c] = o;
                        } else {
                            typedef __bf16 bf16_n __attribute__((ext_vector_type(N)));
                            bf16_n o;
#pragma unroll
                            for (int i = 0; i < N; ++i) o[i] = (__bf16)(wj * g[u][i]);
                            if (ST) __builtin_nontemporal_store(o, reinterpret_cast<bf16_n*>(dy_perm + at) + c); else reinterpret_cast<bf16_n*>(dy_perm + at)[c] = o;
                        }
                    }
                }
            };
            int c0 = sub * 64;   // of the wavefront's first lane
            for (; c0 + 3 * W * 64 < n; c0 += 4 * W * 64) pieces.template operator()<4>(c0 + lane);
            if (c0 + W * 64 < n) {
                pieces.template operator()<2>(c0 + lane);
                c0 += 2 * W * 64;
            }
            if (c0 < n) pieces.template operator()<1>(c0 + lane);
#pragma unroll
            for (int m = N / 2; m > 0; m /= 2)
#pragma unroll
                for (int i = 0; i < m; ++i) sums[i] += sums[i + m];
            sum = row16_sum(sums[0]);
            sum += pair_f<16>(sum);
            sum += pair_f<32>(sum);
            if (W == 1 && lane == 0) dw[p] = sum;
        }
        if (W > 1) {
            if (lane == 0) part[wave] = sum;
            __syncthreads();
            if (threadIdx.x < (unsigned)rows && j0 + (int)threadIdx.x < k) {
                float v = 0.f;
#pragma unroll
                for (int q = 0; q < W; ++q) v += part[threadIdx.x * W + q];
                dw[(size_t)t * k + j0 + threadIdx.x] = v;
            }
            __syncthreads();
        }
    }
}

}  // namespace

hipError_t launch_combine_backward(const moe_shape& s, const void* dout, const void* y_perm, const int32_t* inv_perm, const float* w, float* dw,
                                   void* dy_perm, bool y_fp32, bool dout_fp32, hipStream_t st) {
    const int64_t pairs = (int64_t)s.T * s.top_k, bytes = pairs * s.H * (y_fp32 ? 4 : 2);
    const bool split = pairs <= 2048 && s.H >= 1024;
    // Past the caches, us without, loads, stores, both: 4096 tokens x 4096, k = 2, fp32 (134 MB) 61.7, 58.9, 59.4, 54.1; 32768 x 5120, k = 6, bf16
    // (2 GB) 801, 811, 797, 795, without dy_perm 376, 359; 3001 x 2048, k = 6, fp32 (147 MB) without dy_perm 32.8, 28.4; 2000 x 2048, k = 6, bf16
    // (49 MB) 22.1, 21.1, 17.6, 21.7.
    const bool ld = !split && bytes > (int64_t)64 << 20, st_past = !split && dy_perm && bytes > (int64_t)16 << 20;
    auto run = [&]<bool Y, bool D, bool DY, int W, bool LD, bool ST>() {
        const int rows = s.top_k < 16 / W ? s.top_k : 16 / W;
        hipLaunchKernelGGL((combine_backward_kernel<Y, D, DY, W, LD, ST>), dim3(s.T), dim3(rows * W * 64), 0, st, (const char*)dout, (const char*)y_perm, inv_perm,
                           w, s.top_k, s.H, dw, (char*)dy_perm);
        return hipGetLastError();
    };
    auto with_policy = [&]<bool Y, bool D, bool DY>() {
        if (split) return run.template operator()<Y, D, DY, 4, false, false>();
        if constexpr (DY) {
            if (ld) return run.template operator()<Y, D, true, 1, true, true>();
            if (st_past) return run.template operator()<Y, D, true, 1, false, true>();
        }
        if constexpr (!DY)
            if (ld) return run.template operator()<Y, D, false, 1, true, false>();
        return run.template operator()<Y, D, DY, 1, false, false>();
    };
    auto with_dy = [&]<bool Y, bool D>() {
        return dy_perm ? with_policy.template operator()<Y, D, true>() : with_policy.template operator()<Y, D, false>();
    };
    if (y_fp32) return dout_fp32 ? with_dy.operator()<true, true>() : with_dy.operator()<true, false>();
    return dout_fp32 ? with_dy.operator()<false, true>() : with_dy.operator()<false, false>();
}

}  // namespace moe
