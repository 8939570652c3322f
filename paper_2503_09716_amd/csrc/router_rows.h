// A token's row of logits in 16 lanes, for the kernels that train the router (balance.hip, route_backward.hip).
#pragma once
#include "topk.h"

namespace moe {
namespace {

// Lane c of a row of 16 holds NV values.  WIDE: experts 4c..4c+3 of every 64, 16 bytes to a load (E % 4 == 0 and 16-byte aligned
// matrices); else experts c, c + 16, ..., so that matrices of any alignment and odd E are read 64 bytes to a row.
template <int NV, bool WIDE>
__device__ __forceinline__ void load_row16(float (&v)[NV], const float* __restrict__ m, const size_t t, const int E, const int row, const float pad) {
    const float* const p = m + t * E;
    if constexpr (WIDE) {
#pragma unroll
        for (int b = 0; b < NV / 4; ++b) {
            const int e = row * 4 + 64 * b;
            f32x4 q = {pad, pad, pad, pad};
            if (e < E) q = *reinterpret_cast<const f32x4*>(p + e);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * b + i] = q[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = row + 16 * i < E ? p[row + 16 * i] : pad;
    }
}

template <int NV, bool WIDE>
__device__ __forceinline__ void store_row16(const float (&v)[NV], float* __restrict__ m, const size_t t, const int E, const int row) {
    float* const p = m + t * E;
    if constexpr (WIDE) {
#pragma unroll
        for (int b = 0; b < NV / 4; ++b) {
            const int e = row * 4 + 64 * b;
            if (e < E) *reinterpret_cast<f32x4*>(p + e) = f32x4{v[4 * b], v[4 * b + 1], v[4 * b + 2], v[4 * b + 3]};
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (row + 16 * i < E) p[row + 16 * i] = v[i];
    }
}

// e^x for x <= 0 as 2^(x log2 e): the product's rounding and the constant's go into a linear factor, so that the result is off by two steps
// of fp32 at most however large x is (below 2^-126 it is 0).  Half as many instructions as expf, whose care for other x the softmax of 5
// million logits paid for (balance loss, 32768 x 160: 18.5 us with expf, 17.3).
__device__ __forceinline__ float exp_nonpositive(float x) {
    constexpr float L = 1.44269504088896341f, REST = (float)(1.44269504088896341 - (double)L), LN2 = 0.693147180559945309f;
    x = x < -200.f ? -200.f : x;   // infinities; a NaN stays
    const float hi = x * L, lo = fmaf(x, REST, fmaf(x, L, -hi));
#if defined(__AMDGCN__)
    const float e = __builtin_amdgcn_exp2f(hi);
#else
    const float e = exp2f(hi);
#endif
    return fmaf(e, lo * LN2, e);
}

// Logits to e^(logit - the largest); the sum of those in z.  The largest.  Values of -inf give 0.
template <int NV>
__device__ __forceinline__ float exps_row16(float (&v)[NV], float& z) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i) m = fmaxf(m, v[i]);
    m = row16_max(m);
    z = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) { v[i] = exp_nonpositive(v[i] - m); z += v[i]; }
    z = row16_sum(z);
    return m;
}

}  // namespace

// Runs f.template operator()<NV, WIDE>() for the narrowest row that holds E experts.
template <class F>
hipError_t for_row16(const int E, const bool wide, F&& f) {
    if (wide) {
        if (E <= 64) return f.template operator()<4, true>();
        if (E <= 128) return f.template operator()<8, true>();
        if (E <= 192) return f.template operator()<12, true>();
        return f.template operator()<16, true>();
    }
    if (E <= 16) return f.template operator()<1, false>();
    if (E <= 32) return f.template operator()<2, false>();
    if (E <= 64) return f.template operator()<4, false>();
    if (E <= 128) return f.template operator()<8, false>();
    if (E <= 192) return f.template operator()<12, false>();
    return f.template operator()<16, false>();
}

inline bool wide_rows(const int E, std::initializer_list<const void*> matrices) {
    bool ok = E % 4 == 0 && E > 16;   // up to 16 experts a lane has one of them
    for (const void* m : matrices) ok = ok && ((uintptr_t)m & 15) == 0;
    return ok;
}

}  // namespace moe
