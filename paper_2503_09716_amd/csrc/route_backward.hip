// Backward pass of the router: from the gradients of the routing weights and of the logits to those of x, gate matrix and bias.
//
// Weights w are scale times the softmax p over all experts, or over a token's picks (renormalize): either way
//   dl_te = scale p_te (g_te - sum_i p_ti g_ti) + dlogits_te,   g the gradient of the weights at the picks, 0 elsewhere,
// and without renormalisation p runs over all experts, so that every logit has a gradient.  Then
//   dx = dl Wg^T,   dWg = x^T dl,   dbias = sum_t dl_t.
// x and Wg are bf16, so a matrix instruction multiplies them exactly; dl is fp32 and goes in as a sum of bf16 pieces: hi + mid + lo
// hold its 24 bits, and three products give dWg and dx what products in fp32 would.  (Those run at a sixteenth of the rate.)  dx takes the
// third piece, too, although it is rounded to bf16 afterwards: where the experts' terms cancel, what is left hangs on dl's last bits
// (with hi + mid alone, 2^-17 of dl, 32768 x 5120, 160 experts took 260 us instead of 291).
//
// Three launches: dl and the gate matrix in operand order; both products; the sum of dWg's parts.  Short batches do without the first; up to
// 128 tokens (96 from 65 experts on) do without the last, too, unless their rows of dWg can only be written 4 bytes at a time and are longer than
// 48 experts.  us (of which products): 128 tokens x 4096, 8 experts 8.9 (one launch), 256 x 512, 8 experts 10.8 (4.7; two), 256 x 5120,
// 160 experts 21.5 (two), 3001 x 2048, 64 experts 20 (16.7; two), 16384 x 6144, 8 experts 91 (82: 403 MB at 4.9 TB/s, a copy of x takes 74), 32768 x
// 5120, 64 experts 162 (matrix units 47 % busy; a copy of x takes 124), 160 experts 286 to 298 by box (267: matrix units 64 % busy with 322 GFLOP of
// bf16 products, 1.2 PFLOP/s); without dx 16384 x 6144, 8 experts 48, 32768 x 5120, 160 experts 165.  What keeps them from more there is that both
// wavefronts of a SIMD wait at the same time, after the step's barrier and for operands from LDS (30 % of their cycles).  While dx took two
// pieces of dl (262): two workgroups of four wavefronts to a CU, other priorities, one of the two starting with the other product: no gain; two
// tiles of their own for the products, one after the other or in turn, 262 to 310.
#include <utility>

#include "common.h"
#include "router_rows.h"
#include "train.h"

namespace moe {
namespace {

typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;
typedef __attribute__((address_space(3))) char* lds_t;
typedef __attribute__((address_space(3))) const bf16x8* frag_ptr_t;

__device__ __forceinline__ f32x4 mfma(const bf16x8 a, const bf16x8 b, const f32x4 c) {
#if defined(__gfx950__)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
#else
    return c;
#endif
}

// 64 lanes x 16 bytes from each lane's own address to LDS at l + 16 * lane.
__device__ __forceinline__ void load16_to_lds(const char* p, lds_t l) {
#if defined(__gfx950__)
    __builtin_amdgcn_global_load_lds((gptr_t)p, (lptr_t)l, 16, 0, 0);
#endif
}

// Columns of rows of bf16 in LDS as matrix operands.  ds_read_b64_tr_b16 takes four rows of 16 to a group of 16 lanes: lane i gives the
// address of elements 4 (i % 4) .. + 3 of row i / 4 and gets column i.  Two of them make a lane's 8 steps.  Assembly with its own wait:
// before the builtin the compiler waits for every direct load in flight.
// Two operands, from p0 and p1, the second half of each NEXT bytes behind its first.
template <int NEXT>
__device__ __forceinline__ void read_transposed(bf16x8 (&f)[2], const lds_t p0, const lds_t p1) {
#if defined(__gfx950__)
    u32x2 a, b, c, d;
    asm volatile("ds_read_b64_tr_b16 %0, %4\n\t"
                 "ds_read_b64_tr_b16 %1, %4 offset:%6\n\t"
                 "ds_read_b64_tr_b16 %2, %5\n\t"
                 "ds_read_b64_tr_b16 %3, %5 offset:%6\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d) : "v"((uint32_t)(uintptr_t)p0), "v"((uint32_t)(uintptr_t)p1), "n"(NEXT) : "memory");
    f[0] = __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
    f[1] = __builtin_bit_cast(bf16x8, u32x4{c[0], c[1], d[0], d[1]});
#endif
}
// Four operands, the second half of each NEXT bytes behind its first.
template <int NEXT>
__device__ __forceinline__ void read_transposed(bf16x8 (&f)[4], const lds_t p0, const lds_t p1, const lds_t p2, const lds_t p3) {
#if defined(__gfx950__)
    u32x2 a, b, c, d, e, g, h, i;
    asm volatile("ds_read_b64_tr_b16 %0, %8\n\t"
                 "ds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %2, %9\n\t"
                 "ds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %4, %10\n\t"
                 "ds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %6, %11\n\t"
                 "ds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d), "=&v"(e), "=&v"(g), "=&v"(h), "=&v"(i)
                 : "v"((uint32_t)(uintptr_t)p0), "v"((uint32_t)(uintptr_t)p1), "v"((uint32_t)(uintptr_t)p2), "v"((uint32_t)(uintptr_t)p3), "n"(NEXT) : "memory");
    f[0] = __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
    f[1] = __builtin_bit_cast(bf16x8, u32x4{c[0], c[1], d[0], d[1]});
    f[2] = __builtin_bit_cast(bf16x8, u32x4{e[0], e[1], g[0], g[1]});
    f[3] = __builtin_bit_cast(bf16x8, u32x4{h[0], h[1], i[0], i[1]});
#endif
}
// Three operands, from p + A and q + A to p + C and q + C.
template <int A, int B, int C>
__device__ __forceinline__ void read_transposed(bf16x8 (&f)[3], const lds_t p, const lds_t q) {
#if defined(__gfx950__)
    u32x2 a, b, c, d, e, g;
    asm volatile("ds_read_b64_tr_b16 %0, %6 offset:%8\n\t"
                 "ds_read_b64_tr_b16 %1, %7 offset:%8\n\t"
                 "ds_read_b64_tr_b16 %2, %6 offset:%9\n\t"
                 "ds_read_b64_tr_b16 %3, %7 offset:%9\n\t"
                 "ds_read_b64_tr_b16 %4, %6 offset:%10\n\t"
                 "ds_read_b64_tr_b16 %5, %7 offset:%10\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d), "=&v"(e), "=&v"(g)
                 : "v"((uint32_t)(uintptr_t)p), "v"((uint32_t)(uintptr_t)q), "n"(A), "n"(B), "n"(C) : "memory");
    f[0] = __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
    f[1] = __builtin_bit_cast(bf16x8, u32x4{c[0], c[1], d[0], d[1]});
    f[2] = __builtin_bit_cast(bf16x8, u32x4{e[0], e[1], g[0], g[1]});
#endif
}

// ---- gradient of the logits -----------------------------------------------------------------
// A workgroup takes 32 tokens, a token in a row of 16 lanes; they meet in LDS and leave as operand blocks.  Workgroups past those of
// the tokens lay the gate matrix out.
constexpr int PREP_TOKENS = 32;

// The expert (of 16) that lies e-th among those of tokens 8 g .. + 7 in a block of dl, and the other way round: neither what the
// transposing read takes at a time of two neighbouring g (experts 0 .. 3 and 8 .. 11, or the others) nor what a 16-byte operand read does
// (0 .. 3 and 12 .. 15 of the one, 4 .. 11 of the other) meets in a bank.
__device__ __forceinline__ int dl_row(const int e, const int g) { return e ^ ((g & 1) * 12); }

// v as bf16 pieces.  hi is cut off: rounded, it could pass the type's range next to the end of fp32's.
__device__ __forceinline__ void split3(const float v, __bf16& hi, __bf16& mid, __bf16& lo) {
    hi = __builtin_bit_cast(__bf16, (uint16_t)(__float_as_uint(v) >> 16));
    const float r = v - (float)hi;
    mid = (__bf16)r;
    lo = (__bf16)(r - (float)mid);
}

// The lane's 16 bytes of block b of 16 columns and kb of 32 experts, of the 32 columns from h on.
__device__ __forceinline__ u32x4 gate_piece(const RouteBackwardArgs& a, const int h, const int b, const int kb, const int lane) {
    const int i = lane & 15, e0 = kb * 32 + 8 * (lane >> 4);
    const uint16_t* const src = reinterpret_cast<const uint16_t*>(a.wg) + (size_t)(h + 8 * (i >> 2) + 4 * b + (i & 3)) * a.E;
    if (a.wg_wide) return e0 < a.E ? *reinterpret_cast<const u32x4*>(src + e0) : u32x4{0u, 0u, 0u, 0u};
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = src[min(e0 + j, a.E - 1)];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = e0 + j < a.E ? v[j] : 0u;
    return u32x4{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16};
}

// LDS accesses of a wavefront's lanes on either side keep their order.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// What a lane of a token's row reads: its logits and their gradients, one pick, whether the token counts.
template <int NV>
struct TokenRow {
    float v[NV], add[NV], dw;
    int token, pick;
    uint8_t kept;
    template <bool WIDE>
    __device__ __forceinline__ void load(const RouteBackwardArgs& a, const int tok, const int row) {
        token = tok;
        const size_t t = min(tok, a.T - 1), at = t * a.k + min(row, a.k - 1);
        pick = a.idx[at];
        dw = a.dw[at];
        load_row16<NV, WIDE>(v, a.logits, t, a.E, row, -INFINITY);
        if (a.dlogits) load_row16<NV, WIDE>(add, a.dlogits, t, a.E, row, 0.f);
        kept = a.keep ? a.keep[t] : 1;
    }
    __device__ __forceinline__ bool on(const RouteBackwardArgs& a) const { return token < a.T && kept; }
    // The next 16 picks of the row.
    __device__ __forceinline__ void next_picks(const RouteBackwardArgs& a, const int j0, const int row) {
        const size_t at = (size_t)min(token, a.T - 1) * a.k + min(j0 + row, a.k - 1);
        pick = a.idx[at];
        dw = a.dw[at];
    }
    // Gradients of the weights at the lane's experts, 0 where they are not picked, and which are: by way of the token's row of LDS (to
    // compare every pick with every expert takes five times the instructions).
    template <bool WIDE>
    __device__ __forceinline__ uint32_t picks(const RouteBackwardArgs& a, const int row, float (&g)[NV], float* const at) {
        constexpr uint32_t NONE = 0xffffffffu, NOT_A_NUMBER = 0x7fc00000u;
#pragma unroll
        for (int i = 0; i < NV; ++i) at[row16_expert<WIDE>(row, i)] = __uint_as_float(NONE);
        wave_sync();
        for (int j0 = 0; j0 < a.k; j0 += 16) {   // one round unless k > 16
            if (j0 > 0) next_picks(a, j0, row);
            const uint32_t d = __float_as_uint(dw * a.scale);
            if (j0 + row < a.k && (uint32_t)pick < (uint32_t)a.E) at[pick] = __uint_as_float(d == NONE ? NOT_A_NUMBER : d);
        }
        wave_sync();
        uint32_t picked = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t d = __float_as_uint(at[row16_expert<WIDE>(row, i)]);
            g[i] = d == NONE ? 0.f : __uint_as_float(d);
            picked |= d == NONE ? 0u : 1u << i;
        }
        return picked;
    }
    // v becomes dl, zero where the token does not count and past the experts
    template <bool WIDE>
    __device__ __forceinline__ void gradient(const RouteBackwardArgs& a, const int row, const float (&g)[NV], const uint32_t picked) {
        if (a.renorm) {
            // A row none of whose ids names an expert has no weights: any softmax will do, its gradients g are zero.
            const float others = row16_max(picked) ? -INFINITY : 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = picked >> i & 1 ? v[i] : others;
        }
        float z, s = 0.f;
        exps_row16<NV>(v, z);
        const float rz = 1.0f / z;
#pragma unroll
        for (int i = 0; i < NV; ++i) { v[i] *= rz; s = fmaf(v[i], g[i], s); }
        s = row16_sum(s);
        const bool counts = on(a);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const float d = v[i] * (g[i] - s) + (a.dlogits ? add[i] : 0.f);
            v[i] = counts && row16_expert<WIDE>(row, i) < a.E ? d : 0.f;
        }
    }
};

template <int NV, bool WIDE>
__global__ __launch_bounds__(256) void route_backward_prep_kernel(const RouteBackwardArgs a, const int token_blocks) {
    constexpr int LDS_E = 16 * NV + 1;
    __shared__ float dl[PREP_TOKENS][LDS_E];
    __shared__ uint32_t mask;
    if ((int)blockIdx.x >= token_blocks) {
        // a block of the gate matrix to a wavefront
        const uint32_t blk = (blockIdx.x - token_blocks) * 4 + (threadIdx.x >> 6), kb = blk % a.kb, hb = blk / a.kb;
        if (hb < (uint32_t)a.H / 16) reinterpret_cast<u32x4*>(a.wg_blocks)[(size_t)blk * 64 + (threadIdx.x & 63)] = gate_piece(a, hb / 2 * 32, hb & 1, kb, threadIdx.x & 63);
        return;
    }
    if (threadIdx.x == 0) mask = 0;
    __syncthreads();
    if (blockIdx.x == 0 && threadIdx.x < 64) reinterpret_cast<u32x4*>(a.zeros)[threadIdx.x] = u32x4{0u, 0u, 0u, 0u};
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15;
    TokenRow<NV> rows[2];   // both asked for before either is computed with
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) rows[pass].template load<WIDE>(a, blockIdx.x * PREP_TOKENS + pass * 16 + wave * 4 + (lane >> 4), row);
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        const int lt = pass * 16 + wave * 4 + (lane >> 4);
        float g[NV];
        const uint32_t picked = rows[pass].template picks<WIDE>(a, row, g, dl[lt]);
        rows[pass].template gradient<WIDE>(a, row, g, picked);
#pragma unroll
        for (int i = 0; i < NV; ++i) dl[lt][row16_expert<WIDE>(row, i)] = rows[pass].v[i];
        if (rows[pass].on(a) && row == 0) atomicOr(&mask, 1u << lt);
    }
    __syncthreads();
    if (threadIdx.x == 0) a.masks[blockIdx.x] = mask;
    // Blocks of 16 experts, steps are the 32 tokens.
    char* const out = a.dl_blocks + (size_t)blockIdx.x * 3 * a.nb * 1024;
    for (int p = threadIdx.x; p < a.nb * 64; p += 256) {
        const int at = p & 63, g = at >> 4, e = (p >> 6) * 16 + dl_row(at & 15, g);
        bf16x8 hi, mid, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __bf16 h, m, w;
            split3(e < 16 * NV ? dl[8 * g + i][e] : 0.f, h, m, w);
            hi[i] = h; mid[i] = m; lo[i] = w;
        }
        bf16x8* const o = reinterpret_cast<bf16x8*>(out) + p;
        o[0] = hi;
        o[a.nb * 64] = mid;
        o[2 * a.nb * 64] = lo;
    }
}

// Hand-over point of an LDS ring: at most N of this wave's loads and stores are in flight and its LDS reads have returned; then it
// meets the others.
template <int N>
__device__ __forceinline__ void ring_wait() {
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | 0x0070);  // vmcnt(N) lgkmcnt(0), gfx9 encoding
    asm volatile("" ::: "memory");
}
// ... at most the loads of `stages` stages, N or, where not `all`, FEW to a stage: a case for each number of stages up to MOST.
template <int MOST, int N, int FEW>
__device__ __forceinline__ void wait_stages(const int stages, const bool all) {
    if constexpr (MOST >= 0) {
        if (stages >= MOST) {
            if (all) ring_wait<MOST * N>();
            else ring_wait<MOST * FEW>();
        } else {
            wait_stages<MOST - 1, N, FEW>(stages, all);
        }
    }
}
__device__ __forceinline__ void ring_meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Consecutive places of an XCD's run of workgroups (ids are dealt over the 8 XCDs in turn) in [0, n): neighbours share an L2.
__device__ __forceinline__ int xcd_place(const int id, const int n) {
    const int x = id & 7;
    return x * (n >> 3) + min(x, n & 7) + (id >> 3);
}

// ---- dWg = x^T dl and dx = dl Wg^T ------------------------------------------------------------
// A workgroup of 8 wavefronts takes HT columns of x, all experts and a part of the tokens, 32 tokens at a time through a ring of LDS
// stages filled by direct loads: x as it lies (32-byte chunks swizzled by row) and dl in operand blocks.  Both products use the stage:
//   dWg: the tokens are the contraction, so x comes out of LDS by the transposing read.  Experts are the row operand: a lane ends up
//        with four consecutive experts of a column.  The accumulators stay for all tokens.
//   dx:  the experts are the contraction, so dl comes out by the transposing read.  A wavefront takes a quarter of the columns, whose
//        part of the gate matrix stays in its registers as the row operand, and 16 of the tokens: a lane ends up with 8 consecutive
//        columns of a token, two blocks whose rows are interleaved by fours.
// So x is read and dx written side by side, dl is read once for both.  Rows of x past the end and of tokens that do not count come from
// a page of zeros: their dl is zero, but what x holds there may be no number.
// More than 160 experts take half the columns, or the accumulators and the gate matrix would not fit the registers; so (NARROW) do short
// batches of more than 32, for twice the workgroups to as many parts, as long as a part has up to 5 blocks of tokens.  us with 256, 128
// columns: 64 experts 256 x 5120 15.9, 12.4, 1000 x 2048 17.0, 15.0; 96 experts 1000 x 2048 21.0, 17.9.  At 6 blocks two ways to measure disagree,
// with and without padding: 3001 x 2048, 64 experts, inputs that change from call to call 19.9, 20.2, with padding 20.2, 21.3; the same buffers
// again and again, from a graph, 24.3, 23.3 and 25.1, 24.2.  The former is taken for what programs do.
template <int NB, bool NARROW>
struct Tile {
    static constexpr int HT = NB <= 10 && !NARROW ? 256 : 128;
    static constexpr int KB = (NB + 1) / 2;            // blocks of 32 experts
    static constexpr int WE = NB <= 2 ? 1 : NB <= 10 ? 2 : 4;   // wavefronts along the experts
    static constexpr int WH = 8 / WE;                  // and along the columns
    static constexpr int HB = HT / 16 / WH;            // blocks of 16 columns to a wavefront
    static constexpr int EB = NB / WE;                 // blocks of 16 experts to a wavefront
    static constexpr int DB = HT / 64;                 // dx: blocks of 16 columns to a wavefront
    static constexpr int ROW = HT * 2;                 // bytes of a row of x
    static constexpr int XL = HT / 128;                // wave-loads of 1 KiB of x to a wavefront
    static constexpr int LOADS = 8 * XL + 3 * NB;      // to a stage
    static constexpr int NL = (LOADS + 7) / 8;         // to a wavefront
    static constexpr int MORE = LOADS % 8;             // wavefronts with NL of them, where not all have as many
    static constexpr int STAGE = LOADS * 1024;
    static constexpr int NS = (NB <= 2 ? 80 : 160) * 1024 / STAGE;
    static constexpr int LDS = NS * STAGE;
    static constexpr int STORES = DB / 2;              // of dx, of a wavefront in a stage
    static_assert(HB * WH * 16 == HT && EB * WE == NB && NS >= 2);
};

// Rows 0..3 and 8..11 (16..19 and 24..27, ...), which a transposing read takes at a time, in different 32-byte chunks of 256 bytes.
__device__ __forceinline__ int swizzle(const int r) { return (r & 3) | ((r >> 1) & 4); }

// A page of zeros where no launch before could clear one.
__device__ __align__(1024) const unsigned char zeros_page[1024] = {};

// dl of token t (of 32) into the blocks of a stage: expert e's is lane e % 16's value e / 16.
template <int NB>
__device__ __forceinline__ void put_dl(const float (&v)[NB], const lds_t ds, const int t, const int row) {
    typedef __attribute__((address_space(3))) __bf16* put_ptr_t;
    const int g = t >> 3, at = (g * 16 + dl_row(row, g)) * 16 + (t & 7) * 2;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        __bf16 hi, mid, lo;
        split3(v[i], hi, mid, lo);
        *(put_ptr_t)(ds + i * 1024 + at) = hi;
        *(put_ptr_t)(ds + (NB + i) * 1024 + at) = mid;
        *(put_ptr_t)(ds + (2 * NB + i) * 1024 + at) = lo;
    }
}

// PAST: past the caches, for long batches (16384 x 6144, 8 experts 94.9 -> 91.7 us, 32768 x 5120, 64 experts 164 -> 160; loads of x past them,
// too, gain nothing more).
template <bool PAST>
__device__ __forceinline__ void store_dx(char* p, const u32x4 v) {
    if (PAST) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
    else *reinterpret_cast<u32x4*>(p) = v;
}

// OWN: the workgroup computes the dl of its tokens and lays out its part of the gate matrix by itself, so that the launch before is
// saved; each of the tiles of H does it again.
template <int NB, bool DX, bool OWN, bool NARROW>
__global__ __launch_bounds__(512) void route_backward_products_kernel(const RouteBackwardArgs a) {
    typedef Tile<NB, NARROW> L;
    extern __shared__ char lds_raw[];
    const lds_t lds = (lds_t)lds_raw;
    constexpr int PICK_ROW = 16 * NB + 1;
    float* const scratch = reinterpret_cast<float*>(lds_raw + 2 * L::STAGE);   // OWN: a row for each of the 32 tokens' picks
    const lds_t counted = lds + 2 * L::STAGE + 32 * PICK_ROW * 4;   // OWN: [2 stages][8]: a bit for each of a wavefront's four tokens that counts
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int id = xcd_place(blockIdx.x, a.tiles * a.splits);
    const int ht = id % a.tiles, split = id / a.tiles;
    const int h0 = ht * L::HT;
    const int s0 = split * a.split_steps, s1 = min(s0 + a.split_steps, a.steps);
    const int we = wave % L::WE, wh = wave / L::WE;

    // Which of a step's tokens count, read one step ahead.
    typedef const __attribute__((address_space(4))) uint32_t* masks_t;
    const masks_t masks = (masks_t)a.masks;
    // wave-load i of this wave is load q = wave + 8 i of the stage: those of x, then dl's blocks
    uint32_t x_at[L::XL];    // of this lane's piece from the step's first row on
    int x_row[L::XL];
    bool x_in[L::XL];
#pragma unroll
    for (int i = 0; i < L::XL; ++i) {
        constexpr int PER = L::ROW / 16;   // lanes to a row
        x_row[i] = (wave + 8 * i) * (64 / PER) + lane / PER;
        const int c = (lane % PER) ^ (swizzle(x_row[i]) << 1);   // source chunk of 16 bytes
        x_in[i] = h0 + c * 8 < a.H;
        x_at[i] = (uint32_t)x_row[i] * (uint32_t)a.H * 2 + (uint32_t)(h0 + c * 8) * 2;
    }
    const bool inside = h0 + L::HT <= a.H;
    // OWN: no masks, whether the rows count is read one step ahead
    uint8_t x_kept[L::XL];
    auto ask_kept = [&](const int step) {
#pragma unroll
        for (int i = 0; i < L::XL; ++i) x_kept[i] = a.keep ? a.keep[min(step * 32 + x_row[i], a.T - 1)] : 1;
    };
    auto issue_x = [&](const int step, const int stage) {
        const char* const xs = a.x + (size_t)step * 64 * a.H;
#pragma unroll
        for (int i = 0; i < L::XL; ++i) {
            const bool on = x_in[i] && step * 32 + x_row[i] < a.T && x_kept[i];
            load16_to_lds(on ? xs + x_at[i] : reinterpret_cast<const char*>(zeros_page) + lane * 16, lds + stage * L::STAGE + (wave + 8 * i) * 1024);
        }
    };
    auto issue = [&](const int step, const uint32_t mask, const int stage) {
        const lds_t base = lds + stage * L::STAGE + wave * 1024;
        const char* const xs = a.x + (size_t)step * 64 * a.H;
        if (inside && mask == ~0u) {   // addresses without a vector operation
#pragma unroll
            for (int i = 0; i < L::XL; ++i) load16_to_lds(xs + x_at[i], base + i * 8192);
        } else {
#pragma unroll
            for (int i = 0; i < L::XL; ++i) {
                const char* const p = x_in[i] && (mask >> x_row[i] & 1) ? xs + x_at[i] : a.zeros + lane * 16;
                load16_to_lds(p, base + i * 8192);
            }
        }
        const char* const ds = a.dl_blocks + ((size_t)step * 3 * NB + wave) * 1024;
#pragma unroll
        for (int i = L::XL; i < L::NL; ++i) {
            if (wave + 8 * i >= L::LOADS) break;   // the last of some wavefronts
            load16_to_lds(ds + (i - L::XL) * 8192 + (uint32_t)lane * 16, base + i * 8192);
        }
    };

    // dx: this wavefront's columns and tokens
    const int dh = h0 + (wave & 3) * (L::DB * 16), th = wave >> 2;
    // dl as the column operand: tokens 8 g .. + 7 of two g, four experts from e on and four more
    const int g = 2 * th + ((lane & 3) >> 1), e = 8 * ((lane >> 4) & 1) + ((lane & 15) >> 2);
    const int dl_lane = g * 256 + (lane & 1) * 8 + (NB > 1 ? (lane >> 5) * 1024 : 0);   // one block: its rows again, times zeros of the gate matrix
    const int dl_first = dl_lane + dl_row(e, g) * 16, dl_next = dl_lane + dl_row(e + 4, g) * 16;
    TokenRow<NB> rows;   // OWN: this wavefront's four tokens of the step
    if (OWN) {
        rows.template load<false>(a, s0 * 32 + wave * 4 + (lane >> 4), lane & 15);
        ask_kept(s0);
    }
    bf16x8 wg[L::DB][L::KB];
    auto load_gate = [&] {
#pragma unroll
        for (int b = 0; b < L::DB; ++b)
#pragma unroll
            for (int kb = 0; kb < L::KB; ++kb) {
                const int h = min(dh + b / 2 * 32, a.H - 32);
                wg[b][kb] = OWN ? __builtin_bit_cast(bf16x8, gate_piece(a, h, b % 2, kb, lane))
                                : reinterpret_cast<const bf16x8*>(a.wg_blocks)[((size_t)(h / 16 + b % 2) * L::KB + kb) * 64 + lane];
            }
    };
    // Rows that do not start on 16 bytes: the tile's part of the gate matrix, which is one piece of memory, by way of LDS that is not in use
    // yet (from memory 2 bytes at a time a tile of 63 experts took 5 us more).
    auto stage_gate = [&] {
        const lds_t area = lds + 32 * L::ROW;
        static_assert(!OWN || 2 * L::STAGE - 32 * L::ROW >= L::HT * 16 * NB * 2);
        const char* const src = a.wg + (size_t)h0 * a.E * 2;
        const uint32_t bytes = (uint32_t)min(L::HT, a.H - h0) * a.E * 2;
        for (uint32_t at = wave * 1024; at < bytes; at += 8192) {
            const uint32_t here = at + lane * 16;
            load16_to_lds(here < bytes ? src + here : reinterpret_cast<const char*>(zeros_page) + lane * 16, area + at);
        }
        ring_wait<0>();
        ring_meet();
        typedef __attribute__((address_space(3))) const uint16_t* element_t;
#pragma unroll
        for (int b = 0; b < L::DB; ++b)
#pragma unroll
            for (int kb = 0; kb < L::KB; ++kb) {
                const int i = lane & 15, e0 = kb * 32 + 8 * (lane >> 4);
                const element_t p = (element_t)area + (min(dh + b / 2 * 32, a.H - 32) - h0 + 8 * (i >> 2) + 4 * (b % 2) + (i & 3)) * a.E;
                uint32_t v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = e0 + j < a.E ? p[min(e0 + j, a.E - 1)] : 0u;
                wg[b][kb] = __builtin_bit_cast(bf16x8, u32x4{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16});
            }
        ring_wait<0>();
        ring_meet();   // read before dl comes there
    };
    if constexpr (DX) {
        if (OWN && !a.wg_wide) stage_gate();
        else load_gate();
    }

    f32x4 acc[L::EB][L::HB] = {};
    f32x4 bias[L::EB] = {};
    if (OWN) {
        issue_x(s0, 0);
        ask_kept(s0 + 1);
    } else {
        for (int s = s0; s < min(s0 + L::NS - 1, s1); ++s) issue(s, masks[s], s - s0);
    }
    // SUMS: dl's blocks are added up for dbias, too.
    auto steps = [&]<bool SUMS>() {
        bf16x8 ones;
#pragma unroll
        for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
        int stage = 0;
        uint32_t mask = OWN ? 0u : masks[min(s0 + L::NS - 1, s1 - 1)];
        for (int s = s0; s < s1; ++s) {
            const uint32_t count = OWN ? 0u : masks[s];   // the step's tokens that count
            if constexpr (OWN) {
                float g[NB];
                const uint32_t picked = rows.template picks<false>(a, lane & 15, g, scratch + (wave * 4 + (lane >> 4)) * PICK_ROW);
                rows.template gradient<false>(a, lane & 15, g, picked);
                put_dl<NB>(rows.v, lds + stage * L::STAGE + 32 * L::ROW, wave * 4 + (lane >> 4), lane & 15);
                if (DX && a.keep) {
                    const uint64_t on = __ballot(rows.on(a));
                    counted[stage * 8 + wave] = (char)((on & 1) | (on >> 15 & 2) | (on >> 30 & 4) | (on >> 45 & 8));
                }
                ring_wait<0>();
                ring_meet();
                if (s + 1 < s1) {
                    rows.template load<false>(a, (s + 1) * 32 + wave * 4 + (lane >> 4), lane & 15);
                    issue_x(s + 1, 1 - stage);
                    ask_kept(s + 2);
                }
            } else {
                // Loads and stores retire in the order they were issued.  Behind this stage's loads there are those of the stages that have
                // been asked for since, NS - 2 or what is left, and, from the ring's second round on, NS - 1 steps' stores (all tokens exist in
                // every step but the last, and all columns or none).
                const int later = s1 - 1 - s;
                if (later < L::NS - 2) wait_stages<L::NS - 3, L::NL, L::NL - 1>(later, L::MORE == 0 || wave < L::MORE);
                else if (DX && s - s0 >= L::NS - 1 && dh + L::DB * 16 <= a.H) {
                    if (L::MORE == 0 || wave < L::MORE) ring_wait<(L::NS - 2) * L::NL + (L::NS - 1) * L::STORES>();
                    else ring_wait<(L::NS - 2) * (L::NL - 1) + (L::NS - 1) * L::STORES>();
                } else {
                    if (L::MORE == 0 || wave < L::MORE) ring_wait<(L::NS - 2) * L::NL>();
                    else ring_wait<(L::NS - 2) * (L::NL - 1)>();
                }
                ring_meet();
                if (s + L::NS - 1 < s1) {
                    int next = stage + L::NS - 1;
                    if (next >= L::NS) next -= L::NS;
                    issue(s + L::NS - 1, mask, next);
                }
                mask = masks[min(s + L::NS, s1 - 1)];
            }
            const lds_t xs = lds + stage * L::STAGE, ds = xs + 32 * L::ROW;
            {
                // dl's blocks are read some ahead of the products that need them, the first of them before x's
                constexpr int N = 3 * L::EB, AHEAD = N < 6 ? N : 6;
                const lds_t dp = ds + we * L::EB * 1024 + ((lane & 48) + dl_row(lane & 15, lane >> 4)) * 16;
                auto read = [&](const int i) { return *(frag_ptr_t)(dp + ((2 - i % 3) * NB + i / 3) * 1024); };
                bf16x8 df[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) df[i] = read(i);
                bf16x8 xf[L::HB];
                {
                    const int r = 8 * (lane >> 4) + ((lane & 15) >> 2);
                    const lds_t p = xs + r * L::ROW + (lane & 3) * 8;
                    const int f = swizzle(r);   // that of row r + 4, too
                    const int c = wh * L::HB;
                    auto at = [&](const int hb) { return p + (((c + hb) ^ f) << 5); };
                    if constexpr (L::HB == 2) read_transposed<4 * L::ROW>(xf, at(0), at(1));
                    else read_transposed<4 * L::ROW>(xf, at(0), at(1), at(2), at(3));
                }
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int eb = i / 3;
                    const bf16x8 d = df[i % AHEAD];
                    if (i + AHEAD < N) df[i % AHEAD] = read(i + AHEAD);
#pragma unroll
                    for (int hb = 0; hb < L::HB; ++hb) acc[eb][hb] = mfma(d, xf[hb], acc[eb][hb]);
                    if (SUMS) bias[eb] = mfma(d, ones, bias[eb]);
                    __builtin_amdgcn_sched_barrier(0);   // a read and the products of an earlier one in turn
                }
            }
            if (DX) {
                f32x4 out[L::DB] = {};
                const lds_t p = ds + dl_first, q4 = ds + dl_next;
                auto block = [&]<int K>() {   // of 32 experts: lo, mid, hi
                    bf16x8 d[3];
                    read_transposed<2 * NB * 1024 + K * 2048, NB * 1024 + K * 2048, K * 2048>(d, p, q4);
#pragma unroll
                    for (int q = 0; q < 3; ++q)
#pragma unroll
                        for (int b = 0; b < L::DB; ++b) out[b] = mfma(wg[b][K], d[q], out[b]);
                };
                [&]<int... K>(std::integer_sequence<int, K...>) { (block.template operator()<K>(), ...); }(std::make_integer_sequence<int, L::KB>{});
                u32x4 o[L::DB / 2];   // 8 columns of token lane % 16 in each group of 32
#pragma unroll
                for (int g = 0; g < L::DB / 2; ++g) {
                    bf16x8 v;
#pragma unroll
                    for (int r = 0; r < 4; ++r) { v[r] = (__bf16)out[2 * g][r]; v[4 + r] = (__bf16)out[2 * g + 1][r]; }
                    o[g] = __builtin_bit_cast(u32x4, v);
                }
                // A token that does not count has zeros for dl, but what the gate matrix holds may be no number.
                if (OWN ? a.keep != nullptr : count != ~0u) {
                    typedef __attribute__((address_space(3))) const uint32_t* word_ptr_t;
                    const uint32_t four = OWN ? __builtin_amdgcn_readfirstlane(*(word_ptr_t)(counted + stage * 8 + th * 4)) : 0u;
                    const bool on = (OWN ? four >> (2 * (lane & 12) + (lane & 3)) : count >> (th * 16 + (lane & 15))) & 1;
#pragma unroll
                    for (int g = 0; g < L::DB / 2; ++g) o[g] = on ? o[g] : u32x4{0u, 0u, 0u, 0u};
                }
                const int t0 = s * 32 + th * 16;
                if constexpr (L::DB == 4) {
                    // Lanes of tokens i and i + 8 exchange a group, so that a store writes whole lines: 128 bytes of 8 tokens.
                    const bool upper = lane & 8;
                    u32x4 first, second;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint32_t got = dpp_move<0x128>(upper ? o[0][r] : o[1][r]);   // row_ror:8
                        first[r] = upper ? got : o[0][r];
                        second[r] = upper ? o[1][r] : got;
                    }
                    const int t = t0 + (lane & 7);
                    char* const at = a.dx + ((size_t)t * a.H + dh) * 2 + (lane & 8) * 8 + (lane >> 4) * 16;
                    if (dh + 64 <= a.H) {
                        if (t < a.T) store_dx<!OWN>(at, first);
                        if (t + 8 < a.T) store_dx<!OWN>(at + (size_t)a.H * 16, second);
                    }
                } else {
                    const int t = t0 + (lane & 15);
                    if (dh + 32 <= a.H && t < a.T) *reinterpret_cast<u32x4*>(a.dx + ((size_t)t * a.H + dh) * 2 + (lane >> 4) * 16) = o[0];
                }
            }
            if (++stage == (OWN ? 2 : L::NS)) stage = 0;
        }
    };
    const bool sums = ht == 0 && wh == 0;
    if (sums) steps.template operator()<true>();
    else steps.template operator()<false>();
    // A single part is the sum: dWg and dbias at once.  Of several each goes to its place among the parts, in rows of 16 NB.
    auto put = [&](const int h, const int e, f32x4 v) {
        if (!a.direct) {
            *reinterpret_cast<f32x4*>(a.partial + ((size_t)split * (a.H + 1) + h) * (16 * NB) + e) = v;
            return;
        }
        float* const o = h < a.H ? a.dwg + (size_t)h * a.E + e : a.dbias ? a.dbias + e : nullptr;
        if (!o || e >= a.E) return;
        if (a.direct == 2 && h < a.H) {
            if (a.accumulate) v += *reinterpret_cast<const f32x4*>(o);
            *reinterpret_cast<f32x4*>(o) = v;
            return;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (e + j < a.E) o[j] = a.accumulate ? v[j] + o[j] : v[j];
    };
#pragma unroll
    for (int hb = 0; hb < L::HB; ++hb) {
        const int h = h0 + (wh * L::HB + hb) * 16 + (lane & 15);
        if (h < a.H)
#pragma unroll
            for (int eb = 0; eb < L::EB; ++eb) put(h, (we * L::EB + eb) * 16 + 4 * (lane >> 4), acc[eb][hb]);
    }
    if (sums && (lane & 15) == 0)
#pragma unroll
        for (int eb = 0; eb < L::EB; ++eb) put(a.H, (we * L::EB + eb) * 16 + 4 * (lane >> 4), bias[eb]);
}

// dWg and dbias: the parts of the tokens added in order, four experts to a thread.  Workgroups of one wavefront: short batches have few
// threads here, and they are to be spread over all CUs.
__global__ __launch_bounds__(64) void route_backward_sum_kernel(const RouteBackwardArgs a) {
    const uint32_t per = 4 * a.nb, i = blockIdx.x * 64 + threadIdx.x;   // (H + 1) E < 2^30
    const uint32_t h = i / per, e = (i - h * per) * 4;
    if (h > (uint32_t)a.H || e >= (uint32_t)a.E) return;
    float* const out = h < (uint32_t)a.H ? a.dwg + (size_t)h * a.E + e : a.dbias ? a.dbias + e : nullptr;
    if (!out) return;
    const float* p = a.partial + (size_t)h * (16 * a.nb) + e;
    const size_t stride = (size_t)(a.H + 1) * 16 * a.nb;
    const int n = min(4, a.E - (int)e);
    f32x4 old = {0.f, 0.f, 0.f, 0.f};
    if (a.accumulate)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) old[j] = out[j];
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < a.splits; s0 += 8) {   // eight in flight
        f32x4 q[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) q[u] = *reinterpret_cast<const f32x4*>(p + min(s0 + u, a.splits - 1) * stride);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (s0 + u < a.splits) v += q[u];
    }
    v += old;
    if (n == 4 && ((uintptr_t)out & 15) == 0) {
        *reinterpret_cast<f32x4*>(out) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) out[j] = v[j];
    }
}

__global__ void route_backward_empty_kernel(const size_t n, const int E, float* dwg, float* dbias) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) dwg[i] = 0.f;
    if (dbias && i < (size_t)E) dbias[i] = 0.f;
}

template <class F>
hipError_t for_blocks(const int nb, F&& f) {
    switch (nb) {
        case 1: return f.template operator()<1>();
        case 2: return f.template operator()<2>();
        case 4: return f.template operator()<4>();
        case 6: return f.template operator()<6>();
        case 8: return f.template operator()<8>();
        case 10: return f.template operator()<10>();
        case 12: return f.template operator()<12>();
        default: return f.template operator()<16>();
    }
}

}  // namespace

int route_backward_blocks(const int E) {
    const int nb = (E + 15) / 16;
    if (nb <= 2) return nb;
    if (nb <= 12) return (nb + 1) & ~1;
    return 16;
}

int route_backward_columns(const int nb, const bool narrow) {
    int columns = 0;
    (void)for_blocks(nb, [&]<int NB>() { columns = narrow && NB > 2 ? Tile<NB, true>::HT : Tile<NB, false>::HT; return hipSuccess; });
    return columns;
}

template <int NB, bool OWN, bool NARROW>
constexpr int products_lds() {
    typedef Tile<NB, NARROW> L;
    return OWN ? 2 * L::STAGE + 32 * (16 * NB + 1) * 4 + 16 : L::NS * L::STAGE;
}

template <class F>
hipError_t for_products(const int nb, const bool dx, const bool own, const bool narrow, F&& f) {
    return for_blocks(nb, [&]<int NB>() {
        if constexpr (NB > 2 && NB <= ROUTE_BACKWARD_OWN_NARROW)
            if (own && narrow) return dx ? f.template operator()<NB, true, true, true>() : f.template operator()<NB, false, true, true>();
        if constexpr (NB <= ROUTE_BACKWARD_OWN_WIDE)
            if (own) return dx ? f.template operator()<NB, true, true, false>() : f.template operator()<NB, false, true, false>();
        return dx ? f.template operator()<NB, true, false, false>() : f.template operator()<NB, false, false, false>();
    });
}

hipError_t route_backward_init() {
    hipError_t e = hipSuccess;
    auto set = [&](const int nb, const bool own, const bool narrow) {
        for (const bool dx : {false, true})
            if (e == hipSuccess)
                e = for_products(nb, dx, own, narrow, []<int NB, bool DX, bool OWN, bool NARROW>() {
                    return hipFuncSetAttribute((const void*)route_backward_products_kernel<NB, DX, OWN, NARROW>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                               products_lds<NB, OWN, NARROW>());
                });
    };
    for (int nb : {1, 2, 4, 6, 8, 10, 12, 16}) {
        set(nb, false, false);
        if (nb <= ROUTE_BACKWARD_OWN_WIDE) set(nb, true, false);
        if (nb > 2 && nb <= ROUTE_BACKWARD_OWN_NARROW) set(nb, true, true);
    }
    return e;
}

hipError_t launch_route_backward(const RouteBackwardArgs& a, hipStream_t st) {
    hipError_t e;
    if (!a.own_dl) {
        const bool wide = wide_rows(a.E, {a.logits, a.dlogits ? a.dlogits : a.logits});
        const unsigned pack = a.dx ? ((unsigned)a.H / 16 * a.kb + 3) / 4 : 0u;
        e = for_row16(a.E, wide, [&]<int NV, bool WIDE>() {
            hipLaunchKernelGGL((route_backward_prep_kernel<NV, WIDE>), dim3(a.steps + pack), dim3(256), 0, st, a, a.steps);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    e = for_products(a.nb, a.dx != nullptr, a.own_dl, a.narrow, [&]<int NB, bool DX, bool OWN, bool NARROW>() {
        hipLaunchKernelGGL((route_backward_products_kernel<NB, DX, OWN, NARROW>), dim3(a.tiles * a.splits), dim3(512), (products_lds<NB, OWN, NARROW>()),
                           st, a);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    if (a.direct) return hipSuccess;
    hipLaunchKernelGGL(route_backward_sum_kernel, dim3((unsigned)(((size_t)(a.H + 1) * 4 * a.nb + 63) / 64)), dim3(64), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_route_backward_empty(const moe_shape& s, float* dwg, float* dbias, hipStream_t st) {
    const size_t n = (size_t)s.H * s.E;
    hipLaunchKernelGGL(route_backward_empty_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, n, s.E, dwg, dbias);
    return hipGetLastError();
}

}  // namespace moe
