// Grouped products of MXFP4 rows and MXFP4 matrices on the scaled matrix instruction, fp32 accumulation.
//
//   plain: out[r, n] = sum_k x[r, k] W_e[k, n]        gated: out[r, n] = silu(x[r] . Wa_e[n]) * (x[r] . Wb_e[n])
// for the rows r of group e.  v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 values in 16 cycles, four times what
// the bf16 form does, and takes one scale for 32 values of a row.
#include "fp4.h"
#include "plan.h"

namespace moe {
namespace {

constexpr int DIRECT_ROWS = 64;

__device__ __forceinline__ f32x4 mfma_fp4(const i32x4 a, const i32x4 b, const f32x4 c, const uint32_t sa, const uint32_t sb) {
#if defined(__gfx950__)
    typedef int i32x8 __attribute__((ext_vector_type(8)));
    const i32x8 x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, (int)sa, 0, (int)sb);
#else
    return c;
#endif
}

__device__ __forceinline__ float silu_times(const float g, const float u) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u; }

__global__ __launch_bounds__(256) void fp4_plan_kernel(const PlanArgs p) { plan_list(p, 0, p.offsets); }

// One wavefront: 16 columns of up to 64 rows of one group over the whole of K, straight from memory.  W is the row operand: a
// lane has four neighbouring columns of one row.
template <bool GATED>
__global__ __launch_bounds__(256) void fp4_direct_kernel(const Fp4Product p) {
    constexpr int XB = DIRECT_ROWS / 16, WM = GATED ? 2 : 1;
    const int lane = threadIdx.x & 63, rl = lane & 15, g = lane >> 4;
    const int mt = blockIdx.x / p.n_tiles;
    const int n16 = (blockIdx.x - mt * p.n_tiles) * 4 + (threadIdx.x >> 6);
    if (mt >= p.plan->n_gate_up || n16 * 16 >= p.N) return;
    TileDesc d = p.descs[mt];
    d.nrows &= TILE_ROWS_MASK;
    const char* w[2];
    const char* ws[2];
#pragma unroll
    for (int m = 0; m < WM; ++m) {
        const char* const base = (const char*)(m == 0 ? p.wa : p.wb)[d.group];
        w[m] = base + (size_t)n16 * p.sub_tiles * 1024 + rl * 64 + ((g ^ block_swizzle(rl)) << 4);
        ws[m] = base + p.scales_at + (size_t)n16 * p.groups * 256 + rl * 16 + g * 4;
    }
    const char *x[XB], *xs[XB];
#pragma unroll
    for (int i = 0; i < XB; ++i) {
        const int r = d.row0 + min(i * 16 + rl, d.nrows - 1);
        const size_t at = p.row_index ? p.row_index[r] : r;
        x[i] = p.codes + at * p.sub_tiles * 64 + g * 16;
        xs[i] = p.scales + at * p.groups * 16 + g * 4;
    }
    f32x4 acc[WM][XB];
#pragma unroll
    for (int m = 0; m < WM; ++m)
#pragma unroll
        for (int i = 0; i < XB; ++i) acc[m][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    uint32_t sw[WM], sx[XB];
    for (int t = 0; t < p.sub_tiles; ++t) {
        if ((t & 3) == 0) {
#pragma unroll
            for (int m = 0; m < WM; ++m) sw[m] = *reinterpret_cast<const uint32_t*>(ws[m] + (t >> 2) * 256);
#pragma unroll
            for (int i = 0; i < XB; ++i) sx[i] = *reinterpret_cast<const uint32_t*>(xs[i] + (t >> 2) * 16);
        }
        i32x4 a[WM], b[XB];
#pragma unroll
        for (int m = 0; m < WM; ++m) a[m] = *reinterpret_cast<const i32x4*>(w[m] + (size_t)t * 1024);
#pragma unroll
        for (int i = 0; i < XB; ++i) b[i] = *reinterpret_cast<const i32x4*>(x[i] + t * 64);
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int i = 0; i < XB; ++i) acc[m][i] = mfma_fp4(a[m], b[i], acc[m][i], sw[m], sx[i]);
#pragma unroll
        for (int m = 0; m < WM; ++m) sw[m] >>= 8;
#pragma unroll
        for (int i = 0; i < XB; ++i) sx[i] >>= 8;
    }
    const int esz = p.out_fp32 ? 4 : 2;
#pragma unroll
    for (int i = 0; i < XB; ++i) {
        if (i * 16 + rl >= d.nrows) continue;
        char* const at = p.out + ((size_t)(d.row0 + i * 16 + rl) * p.N + n16 * 16 + g * 4) * esz;
        f32x4 v = acc[0][i];
        if (GATED)
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = silu_times(v[q], acc[WM - 1][i][q]);
        if (p.out_fp32) {
            *reinterpret_cast<f32x4*>(at) = v;
        } else {
            bf16x4 o;
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = (__bf16)v[q];
            *reinterpret_cast<bf16x4*>(at) = o;
        }
    }
}

}  // namespace

Fp4Layout fp4_layout(int64_t rows, int E) {
    Fp4Layout L;
    L.plan = 0;
    L.descs = 256;
    L.total = L.descs + (((size_t)(rows / DIRECT_ROWS + E) * sizeof(TileDesc) + 255) & ~(size_t)255);
    return L;
}

hipError_t launch_fp4_product(const Fp4Product& args, bool gated, hipStream_t st) {
    Fp4Product p = args;
    PlanArgs a = {};
    a.offsets = p.offsets;
    a.E = p.E;
    a.tm_up = DIRECT_ROWS;
    a.nt_up = p.n_tiles = (p.N + 63) / 64;
    a.e_hi = p.E;
    a.plan = p.plan;
    a.descs_up = p.descs;
    p.max_mtiles = p.rows / DIRECT_ROWS + p.E;
    hipLaunchKernelGGL(fp4_plan_kernel, dim3(1), dim3(256), 0, st, a);
    if (const hipError_t e = hipGetLastError()) return e;
    const dim3 grid((unsigned)(p.max_mtiles * p.n_tiles));
    if (gated) hipLaunchKernelGGL(fp4_direct_kernel<true>, grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL(fp4_direct_kernel<false>, grid, dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace moe
