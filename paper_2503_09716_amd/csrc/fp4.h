// MXFP4 (4-bit floating point, e2m1, 32 neighbours along the contraction under one power of two): layouts and launchers.
//
// Both operands of a product are cut along K in sub-tiles of 128 (what one matrix instruction takes) and the scales in groups of
// 512: a row's 16 scale bytes of a group are ordered [k / 32 % 4][k / 128 % 4], so that the four lanes that hold a row in the
// matrix instruction each find the scales of their 32 values of four sub-tiles in one dword.
#pragma once
#include "common.h"

namespace moe {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int FP4_BLOCK = 32, FP4_SUB = 128, FP4_GROUP = 512;

// Rows: codes [rows][sub_tiles * 64 bytes] in the order of k (low nibble first), zero past K; then, 256-byte aligned, scales
// [rows][groups * 16], 127 past K.  Weights: codes [N/16][sub_tiles] blocks of 16 rows x 64 bytes, piece c of row r at slot
// c ^ block_swizzle(r), as the bf16 blocks have it; then, 256-byte aligned, scales [N/16][groups][16 rows][16].
inline int64_t fp4_sub_tiles(const int64_t K) { return (K + FP4_SUB - 1) / FP4_SUB; }
inline int64_t fp4_groups(const int64_t K) { return (K + FP4_GROUP - 1) / FP4_GROUP; }
inline int64_t fp4_scales_at(const int64_t rows, const int64_t K) { return (rows * fp4_sub_tiles(K) * 64 + 255) & ~(int64_t)255; }
inline int64_t fp4_bytes(const int64_t rows, const int64_t K) { return fp4_scales_at(rows, K) + rows * fp4_groups(K) * 16; }

hipError_t launch_fp4_quantize(const void* x, bool fp32, int64_t rows, int K, void* q, hipStream_t st);
hipError_t launch_fp4_dequantize(const void* q, int64_t rows, int K, void* out, bool fp32, hipStream_t st);
hipError_t launch_fp4_pack(const void* w, int K, int N, void* q, hipStream_t st);
hipError_t launch_fp4_unpack(const void* q, int K, int N, void* w, hipStream_t st);

// out[r, n] = x[r] . Wa_e[n] of the rows r of group e; gated: silu(x Wa) * (x Wb).
struct Fp4Product {
    const char *codes, *scales;   // quantised rows
    const int32_t* row_index;     // row r of a product is row row_index[r] of x, or row r (nullptr)
    const void* const* wa;        // device tables of packed matrices
    const void* const* wb;        // gated
    char* out;
    const int32_t* offsets;
    PlanHeader* plan;
    TileDesc* descs;
    int32_t rows, E, K, N, sub_tiles, groups;
    int32_t out_fp32;
    uint32_t scales_at;           // of a weight matrix: its scales, from its start
    int32_t n_tiles, max_mtiles, group_m;
    int32_t inside, rounds;       // 1: no list of m-tiles in memory, workgroups find theirs, of which each has at most that many (rounded up)
};
struct Fp4Layout {
    size_t plan, descs, total;
};
Fp4Layout fp4_layout(int64_t rows, int E);
int64_t fp4_tiles(int64_t rows, int E, int64_t N, bool gated);   // workgroups at most
hipError_t fp4_product_init();
hipError_t launch_fp4_product(const Fp4Product& p, bool gated, hipStream_t st);

}  // namespace moe
