// MXFP4 quantisation of rows and of weight matrices, and the values back.
//
// A block of 32 neighbours along the contraction shares the scale 2^s, s = floor(log2 amax) - 2, at least -127: the largest
// magnitude lands in [4, 8) and the grid {0, 0.5, 1, 1.5, 2, 3, 4, 6} ends at 6.  From the exponent field e of amax the scale's
// byte is max(e - 2, 0).  A value is rounded to the nearest code, ties to the even one, by the conversion instructions, which
// saturate.  A block that holds an infinity or NaN has the scale 255 and reads back as 32 NaN.
//
// All four kernels are bound by memory: one pass, each element in one lane's registers.  Rows to MXFP4: 5.4 to 5.8 TB/s from 18006 x 1408 bf16 (12 us) on; what is
// read goes through the caches (past them 14), where the kernel before has left it.
#include "fp4.h"

namespace moe {
namespace {

__device__ __forceinline__ uint32_t max_over_quad(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));   // quad_perm [1,0,3,2]
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));  // quad_perm [2,3,0,1]
}

// The scale's byte from the largest magnitude's exponent field.
__device__ __forceinline__ uint32_t scale_byte(const uint32_t e) { return e == 255u ? 255u : (e < 2u ? 0u : e - 2u); }

__device__ __forceinline__ bf16x2 pair_of(const uint32_t v) { return __builtin_bit_cast(bf16x2, v); }   // (of a vector's element it takes element 0)

// Eight codes of values that the conversion divides by the scale 2^(byte - 127), given as a float's exponent field.
__device__ __forceinline__ uint32_t codes_of_bf16(const u32x4 v, const uint32_t byte) {
    uint32_t c = 0;
#if defined(__gfx950__)
    const float scale = __uint_as_float(byte << 23);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair_of(v[0]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair_of(v[1]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair_of(v[2]), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair_of(v[3]), scale, 3);
#endif
    return c;
}
__device__ __forceinline__ uint32_t codes_of_fp32(const f32x4 a, const f32x4 b, const uint32_t byte) {
    uint32_t c = 0;
#if defined(__gfx950__)
    const float scale = __uint_as_float(byte << 23);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, a[0], a[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, a[2], a[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, b[0], b[1], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, b[2], b[3], scale, 3);
#endif
    return c;
}

// The values of eight codes: exact in bf16, whose exponents reach as far down as 2^-133.  A scale of 255 is NaN.
__device__ __forceinline__ u32x4 values_of(const uint32_t c, const uint32_t byte) {
    u32x4 v = {0u, 0u, 0u, 0u};
#if defined(__gfx950__)
    const float scale = __uint_as_float(byte << 23);
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
#endif
    if (byte == 255u) v = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
    return v;
}

// A wavefront takes groups of 512 of a row: 8 neighbours to a lane, a block to four lanes, the group's 16 scale bytes together.
constexpr int QUANTIZE_WAVES = 4;

template <bool FP32>
__global__ __launch_bounds__(QUANTIZE_WAVES * 64) void fp4_quantize_kernel(const char* __restrict__ x, const uint32_t units, const int groups,
                                                                          const int K, const int sub_tiles, char* __restrict__ codes,
                                                                          char* __restrict__ scales) {
    const int lane = threadIdx.x & 63;
    const uint32_t unit = blockIdx.x * QUANTIZE_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= units) return;
    const size_t row = unit / (uint32_t)groups;   // below 2^26 units: each takes 80 bytes of 4 GiB or more
    const int q = (int)(unit - (uint32_t)row * (uint32_t)groups), k = q * FP4_GROUP + lane * 8;
    uint32_t code = 0, byte = 127;
    if (k < K) {   // K is a multiple of 32: the four lanes of a block agree
        if (FP32) {
            const f32x4* const at = reinterpret_cast<const f32x4*>(x + (row * K + k) * 4);
            const f32x4 a = at[0], b = at[1];
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) m = max(m, max(__float_as_uint(a[i]) & 0x7fffffffu, __float_as_uint(b[i]) & 0x7fffffffu));
            byte = scale_byte(max_over_quad(m) >> 23);
            code = codes_of_fp32(a, b, byte);
        } else {
            const u32x4 v = *reinterpret_cast<const u32x4*>(x + (row * K + k) * 2);
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) m = max(m, max(v[i] & 0x7fffu, v[i] >> 16 & 0x7fffu));
            byte = scale_byte(max_over_quad(m) >> 7);
            code = codes_of_bf16(v, byte);
        }
        if (byte == 255u) code = 0;
    }
    if (k < sub_tiles * FP4_SUB) *reinterpret_cast<uint32_t*>(codes + row * sub_tiles * 64 + (k >> 1)) = code;
    const int b = lane >> 2;   // block of the group
    if ((lane & 3) == 0) scales[(row * groups + q) * 16 + (b & 3) * 4 + (b >> 2)] = (char)byte;
}

// The way back: bf16 as above; fp32 in two halves of the group of four neighbours to a lane, so that each store is 1 KiB in one piece.  Stores past the caches
// (98304 x 1408 to bf16 75 -> 50 us, 7.0 TB/s, and with a kernel that reads it 172 -> 162; 18006 x 1408 11.5 -> 10.7, 26.5 -> 27.5; 5003 x 2048 to fp32 10.5 -> 7.7, which
// past the caches without the halves are 13.4).
template <bool FP32>
__global__ __launch_bounds__(QUANTIZE_WAVES * 64) void fp4_dequantize_kernel(const char* __restrict__ codes, const char* __restrict__ scales,
                                                                            const uint32_t units, const int groups, const int K,
                                                                            const int sub_tiles, char* __restrict__ out) {
    const int lane = threadIdx.x & 63;
    const uint32_t unit = blockIdx.x * QUANTIZE_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= units) return;
    const size_t row = unit / (uint32_t)groups;
    const int q = (int)(unit - (uint32_t)row * (uint32_t)groups);
    const char* const row_codes = codes + row * sub_tiles * 64;
    const char* const row_scales = scales + (row * groups + q) * 16;
    auto byte_of = [&](const int b) __attribute__((always_inline)) { return (uint32_t)(uint8_t)row_scales[(b & 3) * 4 + (b >> 2)]; };   // block b of the group
    if constexpr (FP32) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int at = j * 256 + lane * 4, k = q * FP4_GROUP + at;
            if (k >= K) continue;
            const u32x4 v = values_of(*reinterpret_cast<const uint16_t*>(row_codes + (k >> 1)), byte_of(at >> 5));
            __builtin_nontemporal_store(u32x4{v[0] << 16, v[0] & 0xffff0000u, v[1] << 16, v[1] & 0xffff0000u}, reinterpret_cast<u32x4*>(out + (row * K + k) * 4));
        }
    } else {
        const int k = q * FP4_GROUP + lane * 8;
        if (k >= K) return;
        const u32x4 v = values_of(*reinterpret_cast<const uint32_t*>(row_codes + (k >> 1)), byte_of(lane >> 2));
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(out + (row * K + k) * 2));
    }
}

// Weights [K, N] row-major to blocks of their transpose: a lane holds 32 k of two neighbouring columns, so a block's largest
// magnitude needs no other lane, and each of a wavefront's loads is 256 consecutive bytes of a row.  A workgroup has a sub-tile of 128 columns, whose
// 1 KiB blocks pass through LDS and are stored whole (K = 4096, N = 14336: 33.3 us; 16 bytes a lane straight to memory 39.8).  The way back loads them
// piece by piece (30.5 us, through LDS 32.8).  The matrix itself passes the caches by, where it would displace what is used again: 33.3 -> 29.4 us (5.0 TB/s), 30.5 -> 24
// (6.1).
constexpr int PACK_WAVES = 4;   // as many neighbouring blocks along K: a sub-tile
constexpr int PACK_COLUMNS = 128, PACK_BLOCKS = PACK_COLUMNS / 16;

__device__ __forceinline__ int tile_piece(const int n, const int kb) {   // of a sub-tile's blocks: column n, block kb of 32 k
    const int r = n & 15;
    return (n >> 4) * 64 + r * 4 + ((kb & 3) ^ block_swizzle(r));
}
__device__ __forceinline__ size_t weight_scale(const int n, const int kb, const int groups) {
    return ((size_t)(n >> 4) * groups + (kb >> 4)) * 256 + (n & 15) * 16 + (kb & 3) * 4 + (kb >> 2 & 3);
}

__global__ __launch_bounds__(PACK_WAVES * 64) void fp4_pack_kernel(const uint32_t* __restrict__ w, const int K, const int N, const int sub_tiles,
                                                                  const int groups, char* __restrict__ codes, char* __restrict__ scales) {
    __shared__ u32x4 tile[PACK_BLOCKS * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n0 = blockIdx.y * PACK_COLUMNS, n = n0 + lane * 2;
    const int kb = blockIdx.x * PACK_WAVES + wave;   // up to groups * 16: past K come zeros
    u32x4 code[2] = {{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
    uint32_t byte[2] = {127u, 127u};
    if (n < N && kb * 32 < K) {
        uint32_t v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = __builtin_nontemporal_load(&w[((size_t)(kb * 32 + i) * N + n) >> 1]);
        uint32_t m0 = 0, m1 = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) { m0 = max(m0, v[i] & 0x7fffu); m1 = max(m1, v[i] >> 16 & 0x7fffu); }
        byte[0] = scale_byte(m0 >> 7);
        byte[1] = scale_byte(m1 >> 7);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            u32x4 a, b;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = v[p * 8 + 2 * i], hi = v[p * 8 + 2 * i + 1];
                a[i] = (lo & 0xffffu) | hi << 16;
                b[i] = lo >> 16 | (hi & 0xffff0000u);
            }
            code[0][p] = byte[0] == 255u ? 0u : codes_of_bf16(a, byte[0]);
            code[1][p] = byte[1] == 255u ? 0u : codes_of_bf16(b, byte[1]);
        }
    }
    if (n < N)
#pragma unroll
        for (int j = 0; j < 2; ++j) scales[weight_scale(n + j, kb, groups)] = (char)byte[j];
    if ((int)blockIdx.x >= sub_tiles) return;
#pragma unroll
    for (int j = 0; j < 2; ++j) tile[tile_piece(lane * 2 + j, wave)] = code[j];
    __syncthreads();
    for (int b = wave; b < PACK_BLOCKS && n0 + b * 16 < N; b += PACK_WAVES)
        *reinterpret_cast<u32x4*>(codes + ((size_t)((n0 >> 4) + b) * sub_tiles + blockIdx.x) * 1024 + lane * 16) = tile[b * 64 + lane];
}

__global__ __launch_bounds__(PACK_WAVES * 64) void fp4_unpack_kernel(const char* __restrict__ codes, const char* __restrict__ scales, const int K,
                                                                    const int N, const int sub_tiles, const int groups, uint32_t* __restrict__ w) {
    const int n = blockIdx.y * PACK_COLUMNS + (threadIdx.x & 63) * 2;
    const int kb = blockIdx.x * PACK_WAVES + (threadIdx.x >> 6);
    if (n >= N || kb * 32 >= K) return;
    u32x4 code[2];
    uint32_t byte[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        code[j] = *reinterpret_cast<const u32x4*>(codes + ((size_t)((n + j) >> 4) * sub_tiles + (kb >> 2)) * 1024 + tile_piece((n + j) & 15, kb) * 16);
        byte[j] = (uint8_t)scales[weight_scale(n + j, kb, groups)];
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const u32x4 a = values_of(code[0][p], byte[0]), b = values_of(code[1][p], byte[1]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t at = ((size_t)(kb * 32 + p * 8 + 2 * i) * N + n) >> 1;
            __builtin_nontemporal_store((a[i] & 0xffffu) | b[i] << 16, &w[at]);
            __builtin_nontemporal_store(a[i] >> 16 | (b[i] & 0xffff0000u), &w[at + (N >> 1)]);
        }
    }
}

}  // namespace

hipError_t launch_fp4_quantize(const void* x, bool fp32, int64_t rows, int K, void* q, hipStream_t st) {
    const int sub_tiles = (int)fp4_sub_tiles(K), groups = (int)fp4_groups(K);
    const uint32_t units = (uint32_t)(rows * groups);
    const dim3 grid((unsigned)((units + QUANTIZE_WAVES - 1) / QUANTIZE_WAVES)), block(QUANTIZE_WAVES * 64);
    char* const codes = (char*)q;
    char* const scales = codes + fp4_scales_at(rows, K);
    if (fp32) hipLaunchKernelGGL(fp4_quantize_kernel<true>, grid, block, 0, st, (const char*)x, units, groups, K, sub_tiles, codes, scales);
    else hipLaunchKernelGGL(fp4_quantize_kernel<false>, grid, block, 0, st, (const char*)x, units, groups, K, sub_tiles, codes, scales);
    return hipGetLastError();
}

hipError_t launch_fp4_dequantize(const void* q, int64_t rows, int K, void* out, bool fp32, hipStream_t st) {
    const int sub_tiles = (int)fp4_sub_tiles(K), groups = (int)fp4_groups(K);
    const uint32_t units = (uint32_t)(rows * groups);
    const dim3 grid((unsigned)((units + QUANTIZE_WAVES - 1) / QUANTIZE_WAVES)), block(QUANTIZE_WAVES * 64);
    const char* const codes = (const char*)q;
    const char* const scales = codes + fp4_scales_at(rows, K);
    if (fp32) hipLaunchKernelGGL(fp4_dequantize_kernel<true>, grid, block, 0, st, codes, scales, units, groups, K, sub_tiles, (char*)out);
    else hipLaunchKernelGGL(fp4_dequantize_kernel<false>, grid, block, 0, st, codes, scales, units, groups, K, sub_tiles, (char*)out);
    return hipGetLastError();
}

hipError_t launch_fp4_pack(const void* w, int K, int N, void* q, hipStream_t st) {
    const int sub_tiles = (int)fp4_sub_tiles(K), groups = (int)fp4_groups(K);
    const dim3 grid((unsigned)(groups * 16 / PACK_WAVES), (unsigned)((N + PACK_COLUMNS - 1) / PACK_COLUMNS));
    hipLaunchKernelGGL(fp4_pack_kernel, grid, dim3(PACK_WAVES * 64), 0, st, (const uint32_t*)w, K, N, sub_tiles, groups, (char*)q,
                       (char*)q + fp4_scales_at(N, K));
    return hipGetLastError();
}

hipError_t launch_fp4_unpack(const void* q, int K, int N, void* w, hipStream_t st) {
    const int sub_tiles = (int)fp4_sub_tiles(K), groups = (int)fp4_groups(K);
    const dim3 grid((unsigned)((K / 32 + PACK_WAVES - 1) / PACK_WAVES), (unsigned)((N + PACK_COLUMNS - 1) / PACK_COLUMNS));
    hipLaunchKernelGGL(fp4_unpack_kernel, grid, dim3(PACK_WAVES * 64), 0, st, (const char*)q, (const char*)q + fp4_scales_at(N, K), K, N, sub_tiles,
                       groups, (uint32_t*)w);
    return hipGetLastError();
}

}  // namespace moe
