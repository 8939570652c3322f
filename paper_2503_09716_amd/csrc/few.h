// The whole layer for up to 16 tokens (few.hip): arguments and launchers.
#pragma once
#include "common.h"

namespace moe {

constexpr int FEW_TOKENS = 16, FEW_TOP_K = 16;
constexpr int FEW_SHARES = 32;        // workgroups to the same columns of the down launch at most
constexpr size_t FEW_X_LDS = 80 << 10;     // beside the gate/up launch's own 75 KiB
constexpr int FEW_X_TWO = 5 << 10;         // and with that much a CU holds two of its workgroups

// Where the picks of the tokens sit: pick[e][t] = j of token t's pick e, or -1; the experts that have any, ascending.
struct alignas(16) Picks {
    int8_t pick[256][FEW_TOKENS];
    int16_t active[256];
    int32_t n;
};

struct FewArgs {
    const char *x, *wg;                  // tokens; packed gate matrix
    const float *bias, *logits;          // bias: or nullptr; logits [logit_shares][T][ep]: computed by a launch before, or nullptr
    float* logits_out;                   // that launch's
    const void* const* weights;          // device table of packed matrices [3][E + Ns]
    Picks* picks;                        // from the first launch to the second
    char* h;                             // [T * k + Ns * T] rows: values as bf16, and what that leaves of them as bf16
    char* x_copy;                        // x as the gate/up launch takes it
    float* partial;                      // [columns of the down launch][shares][16][columns]
    int32_t* arrived;                    // workgroups that have left theirs; cleared by the launch before
    char* out;
    int32_t shares;                      // workgroups to the same columns
    int32_t logit_shares;                // of the logits
    int32_t down_columns;                // columns of a workgroup of the down launch: 16, 64 or 128
    int32_t h_row, x_bytes, x_in_lds;
    int32_t nt;                          // 1: weights past the caches
    int32_t T, H, F, E, k, Ns, ep, renorm, out_fp32;
    float scale;
    uint32_t up_scales_at, down_scales_at;   // MXFP4: of a matrix, its scales
};
size_t few_x_bytes(const moe_shape& s);
int few_h_row(const moe_shape& s);
size_t few_h_bytes(const moe_shape& s);
size_t few_partial_bytes(const moe_shape& s);
bool few_x_in_lds(const moe_shape& s);
bool few_routes_inside(const moe_shape& s);   // no launch for the logits
int few_logit_shares(const moe_shape& s);
int few_down_columns(const moe_shape& s, bool fp4);
int few_shares(const moe_shape& s, bool fp4);
hipError_t few_init();
hipError_t launch_few(const FewArgs& a, bool fp4, hipStream_t st);

}  // namespace moe
