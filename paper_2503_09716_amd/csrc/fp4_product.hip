// Grouped products of MXFP4 rows and MXFP4 matrices on the scaled matrix instruction, fp32 accumulation.
//
//   plain: out[r, n] = sum_k x[r, k] W_e[k, n]        gated: out[r, n] = silu(x[r] . Wa_e[n]) * (x[r] . Wb_e[n])
// for the rows r of group e.  v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 values in 16 cycles, four times what
// the bf16 form does, and takes one scale for 32 values of a row.
#include <initializer_list>
#include <type_traits>

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

// ---- tiles ---------------------------------------------------------------------------------
// A workgroup of four wavefronts (one to a SIMD) multiplies up to 256 rows of x with 256 rows of W (gated: 128 of each matrix, so that the
// gate meets its up value in registers) in sub-tiles of 128 along K.  Codes go from memory straight into a ring of four LDS stages of
// 64-byte rows, three sub-tiles ahead; a row's 16 scale bytes of a group of four sub-tiles into a ring of two.  Each wavefront has all rows
// of x and 64 of W: 256 accumulators.  A fragment is read from the next stage right after its last use, and one barrier a sub-tile hands the ring over.
constexpr int ROWB = 64, NS = 4, TILE_ROWS = 256, WROWS = 256;
constexpr int SCALE_X = TILE_ROWS * 16, SCALE_STAGE = SCALE_X + WROWS * 16;
constexpr int TILE_LDS = NS * (TILE_ROWS + WROWS) * ROWB + 2 * SCALE_STAGE;

typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;
typedef __attribute__((address_space(3))) char* lds_t;
typedef const __attribute__((address_space(3))) i32x4* lfrag_t;
typedef const __attribute__((address_space(3))) uint32_t* lword_t;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void* ptr, const uint32_t bytes = 0xFFFFFFFF) {
    const uint64_t v = (uint64_t)ptr;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void*)(((uint64_t)hi << 32) | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
// 64 lanes x 16 bytes to LDS at l + 16 lane
__device__ __forceinline__ void load_lds(const __amdgpu_buffer_rsrc_t rsrc, lptr_t l, const uint32_t voff, const int soff) {
#if defined(__gfx950__)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, l, 16, voff, soff, 0, 0);
#endif
}
__device__ __forceinline__ void store_b128(const __amdgpu_buffer_rsrc_t rsrc, const uint32_t voff, const u32x4 v) {
#if defined(__gfx950__)
    __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, voff, 0, 0);
#endif
}
__device__ __forceinline__ void store_b32(const __amdgpu_buffer_rsrc_t rsrc, const uint32_t voff, const float v) {
#if defined(__gfx950__)
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), rsrc, voff, 0, 0);
#endif
}
__device__ __forceinline__ void store_bf16(const __amdgpu_buffer_rsrc_t rsrc, const uint32_t voff, const float v) {
#if defined(__gfx950__)
    const __bf16 b = (__bf16)v;
    __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, b), rsrc, voff, 0, 0);
#endif
}
// Lanes 16..31 and 48..63 of a and lanes 0..15 and 32..47 of b change places; both halves as one piece.
__device__ __forceinline__ u32x4 swap_rows16(const u32x2 a, const u32x2 b) {
    u32x4 o = {0u, 0u, 0u, 0u};
#if defined(__gfx950__)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(a[i], b[i], false, false));
        o[i] = r[0];
        o[2 + i] = r[1];
    }
#endif
    return o;
}
// The accumulator is tied to AGPRs (all 256 hold accumulators; left alone the register allocator copies).  The hazards that the compiler does not see
// here: operands come from LDS reads that it waits for, scales from vector instructions fenced off below, an accumulator is used again a
// sub-tile later, and the epilogue waits (mfma_drain).
__device__ __forceinline__ void mfma_tile(f32x4& c, const i32x4& a, const i32x4& b, const uint32_t sa, const uint32_t sb) {
#if defined(__gfx950__)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                 : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
#endif
}
__device__ __forceinline__ void mfma_drain() {
#if defined(__gfx950__)
    asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");
#endif
}
// Hand-over of the ring: at most N of this wavefront's loads are still on their way and its LDS reads have returned; then meet the others.
template <int N>
__device__ __forceinline__ void ring_sync() {
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | 0x0070);   // vmcnt(N) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <int TI, bool GATED>
__device__ __forceinline__ void tile_product(const Fp4Product& p, const TileDesc d, const int n_tile, char* lds) {
    constexpr int NW = 4, BM = TI * 32, XB = 2 * TI, WB = 4, WBH = 2;
    constexpr int NLX = (BM / 16 + NW - 1) / NW, XBYTES = NLX * NW * 1024, NL = NLX + WROWS / 16 / NW, STAGE = NL * NW * 1024;
    constexpr int BN = GATED ? 128 : WROWS;
    constexpr int NL0 = XB * NL / (2 * XB);   // loads of a sub-tile issued before its hand-over
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rl = lane & 15, g = lane >> 4;
    const int N = p.N, n0 = n_tile * BN, KT = p.sub_tiles;
    lds_t const ring = (lds_t)lds, scale_ring = ring + NS * STAGE;

    // loads: rows of x, then blocks of W, each wave every fourth
    const int lrow = lane >> 2, lpiece = (lane & 3) ^ block_swizzle(lrow);
    uint32_t loff[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int q = i * NW + wave;
        if (i < NLX) {
            const int r = d.row0 + min(q * 16 + lrow, d.nrows - 1);   // rows past the end are the last one again
            const uint32_t at = p.row_index ? p.row_index[r] : r;
            loff[i] = at * (uint32_t)(KT * 64) + (uint32_t)(lpiece * 16);
        } else {
            const int qw = q - NLX * NW, grp = min((n0 >> 4) + (GATED ? (qw & 7) : qw), (N >> 4) - 1);
            loff[i] = (uint32_t)grp * (uint32_t)(KT * 1024) + (uint32_t)(lane * 16);
        }
    }
    uint32_t xs_off, ws_off;
    {
        const int r = d.row0 + min(wave * 64 + lane, d.nrows - 1);
        xs_off = (uint32_t)(p.row_index ? p.row_index[r] : r) * (uint32_t)(p.groups * 16);
        const int wr = wave * 64 + lane, n = min(n0 + (GATED ? (wr & 127) : wr), N - 1);
        ws_off = p.scales_at + (uint32_t)(n >> 4) * (uint32_t)(p.groups * 256) + (uint32_t)((n & 15) * 16);
    }
    const __amdgpu_buffer_rsrc_t rs_x = rsrc_of(p.codes), rs_xs = rsrc_of(p.scales), rs_w = rsrc_of(p.wa[d.group]), rs_u = rsrc_of((GATED ? p.wb : p.wa)[d.group]);
    const __amdgpu_buffer_rsrc_t rs_ws = GATED && wave >= 2 ? rs_u : rs_w;
    int koff_x = 0, koff_w = 0;
    auto issue_one = [&](const int i, const int stage) __attribute__((always_inline)) {
        lptr_t dst = (lptr_t)(ring + stage * STAGE + (i * NW + wave) * 1024);
        if (i < NLX) load_lds(rs_x, dst, loff[i], koff_x);
        else if (GATED && (i - NLX) * NW >= 8) load_lds(rs_u, dst, loff[i], koff_w);
        else load_lds(rs_w, dst, loff[i], koff_w);
    };
    auto issue_scales = [&](const int q) __attribute__((always_inline)) {
        lds_t const dst = scale_ring + (q & 1) * SCALE_STAGE + wave * 1024;
        load_lds(rs_xs, (lptr_t)dst, xs_off, q * 16);
        load_lds(rs_ws, (lptr_t)(dst + SCALE_X), ws_off, q * 256);
    };

    const uint32_t offX = (uint32_t)(rl * ROWB + ((g ^ block_swizzle(rl)) << 4));
    const uint32_t offW = offX + (uint32_t)(XBYTES + wave * (GATED ? 32 : 64) * ROWB);
    const uint32_t offSX = (uint32_t)(rl * 16 + g * 4), offSW = offSX + (uint32_t)(SCALE_X + wave * (GATED ? 32 : 64) * 16);
    auto w_row = [](const int hf, const int jj) __attribute__((always_inline)) { return GATED ? hf * 128 + jj * 16 : (hf * WBH + jj) * 16; };

    f32x4 acc[WB][XB];
#pragma unroll
    for (int j = 0; j < WB; ++j)
#pragma unroll
        for (int i = 0; i < XB; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[j][i][r] = 0.f;
    i32x4 xf[XB], wA[WBH], wB[WBH];
    uint32_t sx[XB], sw[WB], sx_next[XB], sw_next[WB];
    auto read_x = [&](const int stage, const int i) __attribute__((always_inline)) { xf[i] = *(lfrag_t)(ring + stage * STAGE + offX + i * 16 * ROWB); };
    auto read_w = [&](const int stage, const int hf, const int jj) __attribute__((always_inline)) {
        const i32x4 v = *(lfrag_t)(ring + stage * STAGE + offW + w_row(hf, jj) * ROWB);
        if (hf == 0) wA[jj] = v;
        else wB[jj] = v;
    };
    auto read_scales = [&](const int q) __attribute__((always_inline)) {
        lds_t const from = scale_ring + (q & 1) * SCALE_STAGE;
#pragma unroll
        for (int i = 0; i < XB; ++i) sx_next[i] = *(lword_t)(from + offSX + i * 256);
#pragma unroll
        for (int j = 0; j < WB; ++j) sw_next[j] = *(lword_t)(from + offSW + w_row(j / WBH, j % WBH) * 16);
    };

    // Half HF of a sub-tile: XB groups of two matrix instructions with one block of x.
    auto part = [&](auto hf_tag, auto rd_tag, auto ld_tag, const int cur, const int nxt, const int ld_stage) __attribute__((always_inline)) {
        constexpr int HF = decltype(hf_tag)::value;
        constexpr bool RD = decltype(rd_tag)::value, LD = decltype(ld_tag)::value;
#pragma unroll
        for (int i = 0; i < XB; ++i) {
#pragma unroll
            for (int jj = 0; jj < WBH; ++jj) {
                const int j = HF * WBH + jj;
                const i32x4 w = HF == 0 ? wA[jj] : wB[jj];
                if (GATED) mfma_tile(acc[j][i], w, xf[i], sw[j], sx[i]);
                else mfma_tile(acc[j][i], xf[i], w, sx[i], sw[j]);
            }
            if (HF == 1 && RD) read_x(nxt, i);
            if (i < WBH && (HF == 0 || RD)) read_w(HF == 0 ? cur : nxt, HF == 0 ? 1 : 0, i);
            if (LD) {
                constexpr int G = 2 * XB;
                const int q = HF * XB + i;
#pragma unroll
                for (int l = (q * NL) / G; l < ((q + 1) * NL) / G; ++l) issue_one(l, ld_stage);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    using T_ = std::true_type;
    using F_ = std::false_type;
    using H0 = std::integral_constant<int, 0>;
    using H1 = std::integral_constant<int, 1>;
    // Sub-tile t; its scales are byte 0 of sx and sw.
    auto sub_tile = [&](auto rd_tag, auto ld_tag, const int t, auto sync) __attribute__((always_inline)) {
        if ((t & 3) == 0) {
#pragma unroll
            for (int i = 0; i < XB; ++i) sx[i] = sx_next[i];
#pragma unroll
            for (int j = 0; j < WB; ++j) sw[j] = sw_next[j];
            if (t + 4 < KT) issue_scales((t >> 2) + 1);
        } else {
#pragma unroll
            for (int i = 0; i < XB; ++i) sx[i] >>= 8;
#pragma unroll
            for (int j = 0; j < WB; ++j) sw[j] >>= 8;
        }
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_nop 3" ::: "memory");   // between those and the first matrix instruction
        const int cur = t % NS, nxt = (t + 1) % NS, ld = (t + NS - 1) % NS;
        part(H0{}, rd_tag, ld_tag, cur, nxt, ld);
        sync();
        // the scales of the next group came in during this one's first sub-tile
        if ((t & 3) == 3 && t + 1 < KT) read_scales((t >> 2) + 1);
        part(H1{}, rd_tag, ld_tag, cur, nxt, ld);
    };

    issue_scales(0);
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) {
        if (s < KT) {
#pragma unroll
            for (int i = 0; i < NL; ++i) issue_one(i, s);
            koff_x += 64;
            koff_w += 1024;
        }
    }
    if (KT >= NS - 1) ring_sync<(NS - 2) * NL>();
    else ring_sync<0>();
    read_scales(0);
#pragma unroll
    for (int i = 0; i < XB; ++i) {
        read_x(0, i);
        if (i < WBH) read_w(0, 0, i);
        __builtin_amdgcn_sched_barrier(0);
    }
    int t = 0;
    for (; t + NS - 1 < KT; ++t) {
        // Scales may be among the loads that are younger than sub-tile t + 1, which then waits for a few more than it has to.
        sub_tile(T_{}, T_{}, t, [] __attribute__((always_inline)) { ring_sync<(NS - 3) * NL + NL0>(); });
        koff_x += 64;
        koff_w += 1024;
    }
    auto drain = [] __attribute__((always_inline)) { ring_sync<0>(); };
    for (; t < KT - 1; ++t) sub_tile(T_{}, F_{}, t, drain);
    sub_tile(F_{}, F_{}, t, drain);

    mfma_drain();
    __builtin_amdgcn_sched_barrier(0);
    if (GATED) {
        // W is the row operand: a lane has the four columns 4g .. 4g+3 of row rl of a block; lanes 16 apart swap halves of two blocks, so that each has
        // 16 bytes of a row and a store covers 16 rows x 64 bytes.
        const uint32_t rowbytes = (uint32_t)N * (p.out_fp32 ? 4u : 2u);
        const __amdgpu_buffer_rsrc_t rs_o = rsrc_of(p.out + (size_t)d.row0 * rowbytes, (uint32_t)d.nrows * rowbytes);
        const int col = n0 + wave * 32;
        if (col >= N) return;   // N is a multiple of 32
#pragma unroll
        for (int i = 0; i < XB; ++i) {
            float v[2][4];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) v[j][q] = silu_times(acc[j][i][q], acc[WBH + j][i][q]);
            const int row = i * 16 + rl;
            const bool ok = row < d.nrows;
            if (p.out_fp32) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    store_b128(rs_o, ok ? (uint32_t)row * rowbytes + (uint32_t)(col + j * 16 + g * 4) * 4u : 0xFFFFFFF0u,
                               u32x4{__float_as_uint(v[j][0]), __float_as_uint(v[j][1]), __float_as_uint(v[j][2]), __float_as_uint(v[j][3])});
            } else {
                u32x2 o[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bf16x4 b = {(__bf16)v[j][0], (__bf16)v[j][1], (__bf16)v[j][2], (__bf16)v[j][3]};
                    o[j] = __builtin_bit_cast(u32x2, b);
                }
                // lane g: block g & 1, columns 8 (g >> 1) .. + 7 of it
                store_b128(rs_o, ok ? (uint32_t)row * rowbytes + (uint32_t)(col + (g & 1) * 16 + (g >> 1) * 8) * 2u : 0xFFFFFFF0u, swap_rows16(o[0], o[1]));
            }
            if (i % 2) __builtin_amdgcn_sched_barrier(0);
        }
    } else {
        // x is the row operand: a lane has column rl of a block and rows 4g .. 4g+3; a store covers 4 rows x 64 bytes (fp32)
        auto store_tile = [&](auto f32_tag) __attribute__((always_inline)) {
            constexpr bool F32 = decltype(f32_tag)::value;
            constexpr int esz = F32 ? 4 : 2;
            const uint32_t rowbytes = (uint32_t)N * (uint32_t)esz;
            uint32_t vcol[WB][4];
#pragma unroll
            for (int j = 0; j < WB; ++j) {
                const int col = n0 + wave * 64 + j * 16 + rl;
                const uint32_t base = col < N ? (uint32_t)(g * 4) * rowbytes + (uint32_t)col * esz : 0x80000000u;
#pragma unroll
                for (int r = 0; r < 4; ++r) vcol[j][r] = base + (uint32_t)r * rowbytes;
            }
#pragma unroll
            for (int i = 0; i < XB; ++i) {
                const int left = min(max(d.nrows - i * 16, 0), 16);
                const __amdgpu_buffer_rsrc_t rs_o = rsrc_of(p.out + (size_t)(d.row0 + i * 16) * rowbytes, (uint32_t)left * rowbytes);
#pragma unroll
                for (int j = 0; j < WB; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float v;   // read here, not earlier: left alone all accumulators are copied ahead of the first store
                        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(acc[j][i][r]) : "memory");
                        if (F32) store_b32(rs_o, vcol[j][r], v);
                        else store_bf16(rs_o, vcol[j][r], v);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        if (p.out_fp32) store_tile(T_{});
        else store_tile(F_{});
    }
}

// Workgroup id -> position in the order of the tiles: ids are dealt to the 8 XCDs in turn; inside each whole round of 256 tiles an XCD gets a run of 32.
__device__ __forceinline__ int tile_order(const int wg, const int total) {
    if (wg >= (total & ~255)) return wg;
    const int r = wg & 255;
    return (wg - r) + (r & 7) * 32 + (r >> 3);
}

template <bool GATED>
__global__ __launch_bounds__(256, 1) void fp4_tile_kernel(const Fp4Product p) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int count = p.plan->n_gate_up, n_run = p.plan->n_run_up;
    const int L = tile_order(blockIdx.x, count * p.n_tiles);
    int mt, n_tile;
    if (L < n_run * p.n_tiles) {   // group_m m-tiles side by side along n: they share panels of W, and those along n panels of x
        const int per = p.group_m * p.n_tiles, sr = L / per, rem = L - sr * per;
        const int mt0 = sr * p.group_m, gm = min(p.group_m, n_run - mt0);
        n_tile = rem / gm;
        mt = mt0 + (rem - n_tile * gm);
    } else {
        const int rem = L - n_run * p.n_tiles;
        mt = n_run + rem / p.n_tiles;
        n_tile = rem - (mt - n_run) * p.n_tiles;
    }
    if (mt >= count) return;
    TileDesc d = p.descs[mt];
    d.nrows &= TILE_ROWS_MASK;
    const int blocks = (d.nrows + 31) >> 5;
    if (blocks > 7) tile_product<8, GATED>(p, d, n_tile, lds);
    else if (blocks > 6) tile_product<7, GATED>(p, d, n_tile, lds);
    else if (blocks > 5) tile_product<6, GATED>(p, d, n_tile, lds);
    else if (blocks > 4) tile_product<5, GATED>(p, d, n_tile, lds);
    else if (blocks > 3) tile_product<4, GATED>(p, d, n_tile, lds);
    else if (blocks > 2) tile_product<3, GATED>(p, d, n_tile, lds);
    else if (blocks > 1) tile_product<2, GATED>(p, d, n_tile, lds);
    else tile_product<1, GATED>(p, d, n_tile, lds);
}

}  // namespace

hipError_t fp4_product_init() {
    for (const void* k : {reinterpret_cast<const void*>(&fp4_tile_kernel<true>), reinterpret_cast<const void*>(&fp4_tile_kernel<false>)})
        if (const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, TILE_LDS)) return e;
    return hipSuccess;
}

Fp4Layout fp4_layout(int64_t rows, int E) {
    Fp4Layout L;
    L.plan = 0;
    L.descs = 256;
    L.total = L.descs + (((size_t)(rows / DIRECT_ROWS + E) * sizeof(TileDesc) + 255) & ~(size_t)255);
    return L;
}

hipError_t launch_fp4_product(const Fp4Product& args, bool gated, hipStream_t st) {
    Fp4Product p = args;
    const bool tiles = p.rows > 2 * DIRECT_ROWS;
    const int tm = tiles ? TILE_ROWS : DIRECT_ROWS, bn = tiles ? (gated ? 128 : WROWS) : 64;
    PlanArgs a = {};
    a.offsets = p.offsets;
    a.E = p.E;
    a.tm_up = tm;
    a.nt_up = p.n_tiles = (p.N + bn - 1) / bn;
    a.tails_last_up = tiles;
    a.small_tiles = 1;
    a.e_hi = p.E;
    a.plan = p.plan;
    a.descs_up = p.descs;
    p.group_m = 8;
    p.max_mtiles = p.rows / tm + p.E;
    hipLaunchKernelGGL(fp4_plan_kernel, dim3(1), dim3(256), 0, st, a);
    if (const hipError_t e = hipGetLastError()) return e;
    const dim3 grid((unsigned)(p.max_mtiles * p.n_tiles));
    if (tiles && gated) hipLaunchKernelGGL(fp4_tile_kernel<true>, grid, dim3(256), TILE_LDS, st, p);
    else if (tiles) hipLaunchKernelGGL(fp4_tile_kernel<false>, grid, dim3(256), TILE_LDS, st, p);
    else if (gated) hipLaunchKernelGGL(fp4_direct_kernel<true>, grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL(fp4_direct_kernel<false>, grid, dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace moe
