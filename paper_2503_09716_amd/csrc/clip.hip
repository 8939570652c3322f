// Norm of all gradients of a list, and the gradients scaled down to a norm: out = g min(1, max_norm / sqrt(sum g^2)).
// HBM-bound: one pass for the norm, one to read and write.  Chunks of at most 32 KiB of one tensor (the list's table) are dealt to the
// workgroups; squares are formed and added up in 64 bits, so that no gradient in the range of its type overflows or vanishes (in fp32 the
// pass takes as long), and added up in a fixed order.  Small lists are one launch, unless an output is in place (32 to 512 KB out of place 4.5 to
// 7.6 us, in place 7.7).
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

// The squares of a chunk that thread `me` of N adds up, eight pieces in flight.
template <bool F32, bool STREAM, int N>
__device__ __forceinline__ double chunk_squares(const ClipChunk& c, const int me) {
    constexpr int PER = F32 ? 4 : 8, AHEAD = 8;
    const int pieces = c.elements / PER;
    const GLOBAL u32x4_any* const p = (const GLOBAL u32x4_any*)c.src;
    double s = 0;
    for (int i0 = me; i0 < pieces; i0 += AHEAD * N) {
        u32x4 v[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) v[u] = load_piece<STREAM>(p + min(i0 + u * N, pieces - 1));
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) s += i0 + u * N < pieces ? square_sum<F32>(v[u]) : 0;
    }
    const int rest = c.elements - pieces * PER;
    if (me < rest) {
        const int i = pieces * PER + me;
        const double g = F32 ? ((const GLOBAL float*)c.src)[i] : bf16_bits_to_float(((const GLOBAL uint16_t*)c.src)[i]);
        s = fma(g, g, s);
    }
    return s;
}

// min(1, max_norm / norm) as a product: where the norm passes the range of fp32 the factor can fall below it, though no gradient's product
// with it does.  `rest` is 1, or 2^-126 where the factor would not be a normal number.
struct Factor {
    float first, rest;
    __device__ __forceinline__ float operator()(const float g) const { return g * first * rest; }
    __device__ __forceinline__ bool one() const { return first == 1.0f && rest == 1.0f; }
};

template <bool F32>
__device__ __forceinline__ u32x4 scaled(const u32x4 v, const Factor scale) {
    if (F32) {
        u32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __float_as_uint(scale(element(v, true, i)));
        return o;
    }
    bf16x8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)scale(element(v, false, i));
    return __builtin_bit_cast(u32x4, o);
}

template <bool F32, bool STREAM, int N>
__device__ __forceinline__ void scale_chunk(const ClipChunk& c, const Factor scale) {
    constexpr int PER = F32 ? 4 : 8, AHEAD = CLIP_CHUNK / 16 / N < 8 ? CLIP_CHUNK / 16 / N : 8;
    const int pieces = c.elements / PER;
    const GLOBAL u32x4_any* const p = (const GLOBAL u32x4_any*)c.src;
    GLOBAL u32x4_any* const q = (GLOBAL u32x4_any*)c.dst;
    for (int i0 = threadIdx.x; i0 < pieces; i0 += AHEAD * N) {
        u32x4 v[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) v[u] = load_piece<STREAM>(p + min(i0 + u * N, pieces - 1));
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const u32x4_any o = scaled<F32>(v[u], scale);
            if (i0 + u * N < pieces) __builtin_nontemporal_store(o, q + i0 + u * N);
        }
    }
    const int rest = c.elements - pieces * PER;
    if ((int)threadIdx.x < rest) {
        const int i = pieces * PER + threadIdx.x;
        if (F32) ((GLOBAL float*)c.dst)[i] = scale(((const GLOBAL float*)c.src)[i]);
        else ((GLOBAL __bf16*)c.dst)[i] = (__bf16)scale(bf16_bits_to_float(((const GLOBAL uint16_t*)c.src)[i]));
    }
}

// Sum over the workgroup's N threads, to every thread, in a fixed order.
template <int N>
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double part[N / 64];
#pragma unroll
    for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0;
#pragma unroll
    for (int w = 0; w < N / 64; ++w) s += part[w];
    return s;
}

__device__ __forceinline__ Factor factor(const ClipArgs& a, const double norm) {
    const double f = norm > a.max_norm ? a.max_norm / norm : 1.0;   // a norm that is no number scales nothing
    const bool small = f < 0x1p-126;
    return Factor{(float)(small ? f * 0x1p126 : f), small ? 0x1p-126f : 1.0f};
}

__global__ __launch_bounds__(THREADS) void clip_norm_kernel(const ClipArgs a) {
    double s = 0;
    for (int i = blockIdx.x; i < a.n_chunks; i += gridDim.x) {
        const ClipChunk c = a.chunks[i];
        if (i < a.n_chunks - KEPT_CHUNKS) s += c.fp32 ? chunk_squares<true, true, THREADS>(c, threadIdx.x) : chunk_squares<false, true, THREADS>(c, threadIdx.x);
        else s += c.fp32 ? chunk_squares<true, false, THREADS>(c, threadIdx.x) : chunk_squares<false, false, THREADS>(c, threadIdx.x);
    }
    s = block_sum<THREADS>(s);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = s;
}

__global__ __launch_bounds__(THREADS) void clip_scale_kernel(const ClipArgs a, const int parts) {
    double s = 0;
    for (int i = threadIdx.x; i < parts; i += THREADS) s += a.partial[i];
    const double norm = sqrt(block_sum<THREADS>(s));
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
    const Factor scale = factor(a, norm);
    for (int i = a.n_chunks - 1 - (int)blockIdx.x; i >= 0; i -= gridDim.x) {
        const ClipChunk c = a.chunks[i];
        if (scale.one() && c.src == c.dst) continue;
        if (i < a.n_chunks - KEPT_CHUNKS) {
            if (c.fp32) scale_chunk<true, true, THREADS>(c, scale);
            else scale_chunk<false, true, THREADS>(c, scale);
        } else {
            if (c.fp32) scale_chunk<true, false, THREADS>(c, scale);
            else scale_chunk<false, false, THREADS>(c, scale);
        }
    }
}

// Few chunks, no output in place of its gradient: every workgroup forms the norm, a wavefront to a chunk, and scales one chunk (us in two
// launches, in one: 8 tensors of 66 KB in all 6.3, 4.0; 262 KB 7.0, 5.3; 524 KB 6.8, 7.3).
constexpr int FEW_THREADS = 1024;
static_assert(CLIP_FEW_CHUNKS == FEW_THREADS / 64);
__global__ __launch_bounds__(FEW_THREADS) void clip_few_kernel(const ClipArgs a) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const ClipChunk mine = a.chunks[blockIdx.x];
    double s = 0;
    if (wave < a.n_chunks) {
        const ClipChunk c = a.chunks[wave];
        s = c.fp32 ? chunk_squares<true, false, 64>(c, lane) : chunk_squares<false, false, 64>(c, lane);
    }
    const double norm = sqrt(block_sum<FEW_THREADS>(s));
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
    const Factor scale = factor(a, norm);
    if (mine.fp32) scale_chunk<true, false, FEW_THREADS>(mine, scale);
    else scale_chunk<false, false, FEW_THREADS>(mine, scale);
}

}  // namespace

hipError_t launch_clip(const ClipArgs& a, hipStream_t st) {
    if (a.one_launch && a.n_chunks > 0) {
        hipLaunchKernelGGL(clip_few_kernel, dim3(a.n_chunks), dim3(FEW_THREADS), 0, st, a);
        return hipGetLastError();
    }
    const int blocks = a.n_chunks < CLIP_BLOCKS ? (a.n_chunks > 0 ? a.n_chunks : 1) : CLIP_BLOCKS;
    hipLaunchKernelGGL(clip_norm_kernel, dim3(blocks), dim3(THREADS), 0, st, a);
    hipLaunchKernelGGL(clip_scale_kernel, dim3(blocks), dim3(THREADS), 0, st, a, blocks);
    return hipGetLastError();
}

}  // namespace moe
