// Arguments and launchers of the kernels that train a router: balance loss, gradients of the router and of the combine, clipping.
#pragma once
#include <initializer_list>

#include "common.h"

namespace moe {

struct BalanceArgs {
    const float* logits;
    const int32_t* idx;
    const uint8_t* keep;       // or nullptr: every token counts
    double balance_coef, z_coef;
    int32_t* counts;
    float *loss, *dlogits;     // dlogits: or nullptr
    int32_t T, E, k;
    int32_t count_blocks, count_tokens, loss_blocks;   // workgroups of the two launches; tokens to one of the first
    int32_t* partial_counts;   // [count_blocks][E + 1]: histograms, kept tokens
    double* partial_loss;      // [loss_blocks][2]
    int32_t* done;
};
constexpr int BALANCE_COUNT_BLOCKS = 32, BALANCE_LOSS_BLOCKS = 256;
// One workgroup does all up to this many tokens, logits (in rows as wide as the kernel takes them), and logits and picks together.  us in one
// workgroup, in two launches: 256 tokens of 8 experts, k = 2 6.5, 9.4; 384 of 8 7.1, 9.3; 448 of 64, k = 8 10.0, 9.4; 384 of 64, k = 8 9.0, 9.5;
// k = 64 10.3, 9.5; 320, k = 64 9.4, 9.6; 384 of 48, k = 48 10.2, 9.5; 256 of 128, k = 8 9.1, 9.3; k = 64 9.8, 9.4; 320 of 85, k = 8 10.8, 9.5;
// 128 of 256, k = 64 8.7, 10.4.
constexpr int BALANCE_ALONE_TOKENS = 384, BALANCE_ALONE_LOGITS = 32768, BALANCE_ALONE = 40960;
hipError_t launch_balance_loss(const BalanceArgs& a, hipStream_t st);

// The gradient of the logits travels in pieces of bf16 (hi + mid + lo = its 24 bits) in the order in which the matrix instructions
// take operands: 1 KiB blocks of 16 rows x 32 contraction steps, lane l's 16 bytes at 16 l (row l % 16, steps 8 (l / 16) .. + 7).
struct RouteBackwardArgs {
    const char *x, *wg;
    const float* logits;
    const int32_t* idx;
    const float* dw;           // gradient of the weights
    const float* dlogits;      // or nullptr
    const uint8_t* keep;       // or nullptr
    char* dx;                  // or nullptr
    float *dwg, *dbias;        // dbias: or nullptr
    int32_t T, H, E, k, renorm, accumulate;
    float scale;
    int32_t nb, kb;            // blocks of 16 experts (as many as the kernel's variant takes), of 32 experts
    int32_t steps;             // blocks of 32 tokens
    int32_t tiles, splits, split_steps;   // tiles of H, parts of the tokens that dWg is summed over apart, blocks of 32 tokens to one
    int32_t own_dl;            // 1: no launch for dl, the products' workgroups compute their tokens'
    int32_t narrow;            // 1: tiles of 128 columns (nb > 2, own_dl)
    int32_t direct;            // 1: the products write dWg and dbias themselves (one part), 2: dWg 16 bytes at a time
    int32_t wg_wide;           // 1: the gate matrix can be read 16 bytes at a time
    char* zeros;               // 1 KiB that the first launch clears
    uint32_t* masks;           // [T / 32]: the tokens that count
    char* dl_blocks;           // [T / 32][hi, mid, lo][nb] blocks: rows are experts (dl_row), steps tokens
    char* wg_blocks;           // [H / 32][2][kb] blocks: row i of block b is h = 8 (i / 4) + 4 b + i % 4 of 32, steps are experts
    float* partial;            // [splits][H + 1][16 nb]: row H the sum of dl
};
int route_backward_blocks(int E);   // nb
// nb up to which own_dl is taken, with narrow tiles (12: 1000 x 2048, 180 experts 27.7 -> 29.9 us; 16 does not fit the registers) and without (they
// would not fit)
constexpr int ROUTE_BACKWARD_OWN_NARROW = 10, ROUTE_BACKWARD_OWN_WIDE = 6;
int route_backward_columns(int nb, bool narrow);   // columns of x to a workgroup
hipError_t launch_route_backward(const RouteBackwardArgs& a, hipStream_t st);
hipError_t launch_route_backward_empty(const moe_shape& s, float* dwg, float* dbias, hipStream_t st);
hipError_t route_backward_init();

hipError_t launch_combine_backward(const moe_shape& s, const void* dout, const void* y_perm, const int32_t* inv_perm, const float* w, float* dw,
                                   void* dy_perm, bool y_fp32, bool dout_fp32, hipStream_t st);

// A piece of a tensor: at most CLIP_CHUNK bytes.
struct ClipChunk {
    const char* src;
    char* dst;
    uint32_t elements, fp32;
};
constexpr int CLIP_CHUNK = 32768;
struct ClipArgs {
    const ClipChunk* chunks;
    double* partial;           // [CLIP_BLOCKS]
    float* norm;
    double max_norm;
    int32_t n_chunks, one_launch;
};
constexpr int CLIP_BLOCKS = 1024;
// Lists that one launch takes: up to that many chunks and bytes, no output in place of its gradient.
constexpr int CLIP_FEW_CHUNKS = 16, CLIP_FEW_BYTES = 384 << 10;
hipError_t launch_clip(const ClipArgs& a, hipStream_t st);

}  // namespace moe
