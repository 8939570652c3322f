// Norm of all gradients of a list, and the gradients scaled down to a norm: out = g min(1, max_norm / sqrt(sum g^2)).
// HBM-bound: one pass for the norm, one to read and write.  Chunks of at most 32 KiB of one tensor (the list's table) are dealt to the
// workgroups; squares are formed and added up in 64 bits, so that no gradient in the range of its type overflows or vanishes (in fp32 the
// pass takes as long), and added up in a fixed order.  Small lists are two launches of 3 us each.
// The second pass goes through the chunks from the last to the first: the last 245 MB that the first read are still in the memory-side
// cache.  All else goes past the caches, the outputs too, and so does not displace them (1.16 GB, us: 635 with ordinary loads and stores,
// 611 with the stores past the caches, 551 with everything past them, 540 as it is; 360 MB 198, 172, 172, 161).
#include "common.h"
#include "train.h"

namespace moe {
namespace {

constexpr int THREADS = 256;
constexpr int KEPT_CHUNKS = 7500;
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));   // tensors are as aligned as their elements
// The table's pointers are to device memory (the compiler would take a pointer from memory for one that may be to LDS).
#define GLOBAL __attribute__((address_space(1)))

__device__ __forceinline__ float element(const u32x4& v, const bool f32, const int i) {
    return __uint_as_float(f32 ? v[i] : ((i & 1) ? v[i / 2] & 0xffff0000u : v[i / 2] << 16));
}

template <bool F32>
__device__ __forceinline__ double square_sum(const u32x4 v) {
    double s = 0;
#pragma unroll
    for (int i = 0; i < (F32 ? 4 : 8); ++i) {
        const double g = element(v, F32, i);
        s = fma(g, g, s);
    }
    return s;
}

// A piece, past the caches (STREAM) or not.
template <bool STREAM>
__device__ __forceinline__ u32x4 load_piece(const GLOBAL u32x4_any* p) {
    return STREAM ? __builtin_nontemporal_load(p) : *p;
}

template <bool F32, bool STREAM>
__device__ __forceinline__ double chunk_squares(const ClipChunk& c) {
    constexpr int N = F32 ? 4 : 8;
    const int pieces = c.elements / N;
    const GLOBAL u32x4_any* const p = (const GLOBAL u32x4_any*)c.src;
    double s = 0;
    if (pieces == CLIP_CHUNK / 16) {
        u32x4 v[CLIP_CHUNK / 16 / THREADS];
#pragma unroll
        for (int u = 0; u < CLIP_CHUNK / 16 / THREADS; ++u) v[u] = load_piece<STREAM>(p + u * THREADS + threadIdx.x);
#pragma unroll
        for (int u = 0; u < CLIP_CHUNK / 16 / THREADS; ++u) s += square_sum<F32>(v[u]);
    } else {
        for (int i = threadIdx.x; i < pieces; i += THREADS) s += square_sum<F32>(p[i]);
    }
    const int rest = c.elements - pieces * N;
    if ((int)threadIdx.x < rest) {
        const int i = pieces * N + threadIdx.x;
        const double g = F32 ? ((const GLOBAL float*)c.src)[i] : bf16_bits_to_float(((const GLOBAL uint16_t*)c.src)[i]);
        s = fma(g, g, s);
    }
    return s;
}

template <bool F32>
__device__ __forceinline__ u32x4 scaled(const u32x4 v, const float scale) {
    if (F32) {
        u32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __float_as_uint(element(v, true, i) * scale);
        return o;
    }
    bf16x8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)(element(v, false, i) * scale);
    return __builtin_bit_cast(u32x4, o);
}

template <bool F32, bool STREAM>
__device__ __forceinline__ void scale_chunk(const ClipChunk& c, const float scale) {
    constexpr int N = F32 ? 4 : 8;
    const int pieces = c.elements / N;
    const GLOBAL u32x4_any* const p = (const GLOBAL u32x4_any*)c.src;
    GLOBAL u32x4_any* const q = (GLOBAL u32x4_any*)c.dst;
    if (pieces == CLIP_CHUNK / 16) {
        u32x4 v[CLIP_CHUNK / 16 / THREADS];
#pragma unroll
        for (int u = 0; u < CLIP_CHUNK / 16 / THREADS; ++u) v[u] = load_piece<STREAM>(p + u * THREADS + threadIdx.x);
#pragma unroll
        for (int u = 0; u < CLIP_CHUNK / 16 / THREADS; ++u) {
            const u32x4_any o = scaled<F32>(v[u], scale);
            __builtin_nontemporal_store(o, q + u * THREADS + threadIdx.x);
        }
    } else {
        for (int i = threadIdx.x; i < pieces; i += THREADS) q[i] = scaled<F32>(p[i], scale);
    }
    const int rest = c.elements - pieces * N;
    if ((int)threadIdx.x < rest) {
        const int i = pieces * N + threadIdx.x;
        if (F32) ((GLOBAL float*)c.dst)[i] = ((const GLOBAL float*)c.src)[i] * scale;
        else ((GLOBAL __bf16*)c.dst)[i] = (__bf16)(bf16_bits_to_float(((const GLOBAL uint16_t*)c.src)[i]) * scale);
    }
}

// Sum over the workgroup, to every thread, in a fixed order.
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double part[THREADS / 64];
#pragma unroll
    for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) s += part[w];
    return s;
}

__global__ __launch_bounds__(THREADS) void clip_norm_kernel(const ClipArgs a) {
    double s = 0;
    for (int i = blockIdx.x; i < a.n_chunks; i += gridDim.x) {
        const ClipChunk c = a.chunks[i];
        if (i < a.n_chunks - KEPT_CHUNKS) s += c.fp32 ? chunk_squares<true, true>(c) : chunk_squares<false, true>(c);
        else s += c.fp32 ? chunk_squares<true, false>(c) : chunk_squares<false, false>(c);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = s;
}

__global__ __launch_bounds__(THREADS) void clip_scale_kernel(const ClipArgs a, const int parts) {
    double s = 0;
    for (int i = threadIdx.x; i < parts; i += THREADS) s += a.partial[i];
    const double norm = sqrt(block_sum(s));
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
    const float scale = norm > a.max_norm ? (float)(a.max_norm / norm) : 1.0f;   // a norm that is no number scales nothing
    for (int i = a.n_chunks - 1 - (int)blockIdx.x; i >= 0; i -= gridDim.x) {
        const ClipChunk c = a.chunks[i];
        if (scale == 1.0f && c.src == c.dst) continue;
        if (i < a.n_chunks - KEPT_CHUNKS) {
            if (c.fp32) scale_chunk<true, true>(c, scale);
            else scale_chunk<false, true>(c, scale);
        } else {
            if (c.fp32) scale_chunk<true, false>(c, scale);
            else scale_chunk<false, false>(c, scale);
        }
    }
}

}  // namespace

hipError_t launch_clip(const ClipArgs& a, hipStream_t st) {
    const int blocks = a.n_chunks < CLIP_BLOCKS ? (a.n_chunks > 0 ? a.n_chunks : 1) : CLIP_BLOCKS;
    hipLaunchKernelGGL(clip_norm_kernel, dim3(blocks), dim3(THREADS), 0, st, a);
    hipLaunchKernelGGL(clip_scale_kernel, dim3(blocks), dim3(THREADS), 0, st, a, blocks);
    return hipGetLastError();
}

}  // namespace moe
