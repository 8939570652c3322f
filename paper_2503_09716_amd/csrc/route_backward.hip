// Backward pass of the router: from the gradients of the routing weights and of the logits to those of x, gate matrix and bias.
//
// Weights w are scale times the softmax p over all experts, or over a token's picks (renormalize): either way
//   dl_te = scale p_te (g_te - sum_i p_ti g_ti) + dlogits_te,   g the gradient of the weights at the picks, 0 elsewhere,
// and without renormalisation p runs over all experts, so that every logit has a gradient.  Then
//   dx = dl Wg^T,   dWg = x^T dl,   dbias = sum_t dl_t.
// x and Wg are bf16, so a matrix instruction multiplies them exactly; dl is fp32 and goes in as a sum of bf16 pieces: hi + mid + lo
// hold its 24 bits, and three products give dWg what products in fp32 would; dx is rounded to bf16 (8 bits), and the two pieces it
// takes hold dl to 2^-17.
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

// Column blocks of x as matrix operands, from rows of 512 bytes in LDS.  ds_read_b64_tr_b16 takes four rows of 16 bf16 to a group of 16
// lanes: lane i gives the address of elements 4 (i % 4) .. + 3 of row i / 4 and gets column i.  Two of them, four rows apart, make a
// lane's 8 steps.  Assembly with its own wait: before the builtin the compiler waits for every direct load in flight.
__device__ __forceinline__ void read_transposed(bf16x8 (&f)[2], const lds_t p0, const lds_t p1) {
#if defined(__gfx950__)
    u32x2 a, b, c, d;
    asm volatile("ds_read_b64_tr_b16 %0, %4\n\t"
                 "ds_read_b64_tr_b16 %1, %4 offset:2048\n\t"
                 "ds_read_b64_tr_b16 %2, %5\n\t"
                 "ds_read_b64_tr_b16 %3, %5 offset:2048\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d) : "v"((uint32_t)(uintptr_t)p0), "v"((uint32_t)(uintptr_t)p1) : "memory");
    f[0] = __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
    f[1] = __builtin_bit_cast(bf16x8, u32x4{c[0], c[1], d[0], d[1]});
#endif
}
__device__ __forceinline__ void read_transposed(bf16x8 (&f)[4], const lds_t p0, const lds_t p1, const lds_t p2, const lds_t p3) {
#if defined(__gfx950__)
    u32x2 a, b, c, d, e, g, h, i;
    asm volatile("ds_read_b64_tr_b16 %0, %8\n\t"
                 "ds_read_b64_tr_b16 %1, %8 offset:2048\n\t"
                 "ds_read_b64_tr_b16 %2, %9\n\t"
                 "ds_read_b64_tr_b16 %3, %9 offset:2048\n\t"
                 "ds_read_b64_tr_b16 %4, %10\n\t"
                 "ds_read_b64_tr_b16 %5, %10 offset:2048\n\t"
                 "ds_read_b64_tr_b16 %6, %11\n\t"
                 "ds_read_b64_tr_b16 %7, %11 offset:2048\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d), "=&v"(e), "=&v"(g), "=&v"(h), "=&v"(i)
                 : "v"((uint32_t)(uintptr_t)p0), "v"((uint32_t)(uintptr_t)p1), "v"((uint32_t)(uintptr_t)p2), "v"((uint32_t)(uintptr_t)p3) : "memory");
    f[0] = __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
    f[1] = __builtin_bit_cast(bf16x8, u32x4{c[0], c[1], d[0], d[1]});
    f[2] = __builtin_bit_cast(bf16x8, u32x4{e[0], e[1], g[0], g[1]});
    f[3] = __builtin_bit_cast(bf16x8, u32x4{h[0], h[1], i[0], i[1]});
#endif
}

// ---- gradient of the logits -----------------------------------------------------------------
// A workgroup takes 32 tokens, a token in a row of 16 lanes; they meet in LDS and leave as operand blocks.  Workgroups past those of
// the tokens lay the gate matrix out.
constexpr int PREP_TOKENS = 32;

// v as bf16 pieces.
__device__ __forceinline__ void split3(const float v, __bf16& hi, __bf16& mid, __bf16& lo) {
    hi = (__bf16)v;
    const float r = v - (float)hi;
    mid = (__bf16)r;
    lo = (__bf16)(r - (float)mid);
}

// 16-byte piece p of wg_blocks.
__device__ __forceinline__ void pack_gate_piece(const RouteBackwardArgs& a, const size_t p) {
    const int lane = p & 63, i = lane & 15;
    const size_t blk = p >> 6;
    const int kb = (int)(blk % a.kb), b = (int)(blk / a.kb) & 1;
    const size_t h = blk / a.kb / 2 * 32 + 8 * (i >> 2) + 4 * b + (i & 3);
    const int e0 = kb * 32 + 8 * (lane >> 4);
    const uint16_t* const src = reinterpret_cast<const uint16_t*>(a.wg) + h * a.E;
    uint32_t q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int e = e0 + 2 * j;
        q[j] = (e < a.E ? src[e] : 0u) | (e + 1 < a.E ? (uint32_t)src[e + 1] << 16 : 0u);
    }
    reinterpret_cast<u32x4*>(a.wg_blocks)[p] = u32x4{q[0], q[1], q[2], q[3]};
}

template <int NV, bool WIDE>
__global__ __launch_bounds__(256) void route_backward_prep_kernel(const RouteBackwardArgs a, const int token_blocks) {
    constexpr int LDS_E = 16 * NV + 1;
    __shared__ float dl[PREP_TOKENS][LDS_E];
    __shared__ uint32_t mask;
    if ((int)blockIdx.x >= token_blocks) {
        const size_t pieces = (size_t)a.H / 16 * a.kb * 64;
        const size_t p = (size_t)(blockIdx.x - token_blocks) * 256 + threadIdx.x;
        if (p < pieces) pack_gate_piece(a, p);
        return;
    }
    if (threadIdx.x == 0) mask = 0;
    __syncthreads();
    if (blockIdx.x == 0 && threadIdx.x < 64) reinterpret_cast<u32x4*>(a.zeros)[threadIdx.x] = u32x4{0u, 0u, 0u, 0u};
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15;
    const int E = a.E, k = a.k;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        const int lt = pass * 16 + wave * 4 + (lane >> 4), tok = blockIdx.x * PREP_TOKENS + lt, t = min(tok, a.T - 1);
        const bool on = tok < a.T && (!a.keep || a.keep[t]);
        float v[NV], g[NV];
        load_row16<NV, WIDE>(v, a.logits, t, E, row, -INFINITY);
        uint32_t picked = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) g[i] = 0.f;
        for (int j = 0; j < k; ++j) {
            const int e = a.idx[(size_t)t * k + j];
            const float d = a.dw[(size_t)t * k + j] * a.scale;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (row16_expert<WIDE>(row, i) == e) { g[i] = d; picked |= 1u << i; }
        }
        if (a.renorm)
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = picked >> i & 1 ? v[i] : -INFINITY;
        softmax_row16<NV>(v);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) s = fmaf(v[i], g[i], s);
        s = row16_sum(s);
        float add[NV];
        if (a.dlogits) load_row16<NV, WIDE>(add, a.dlogits, t, E, row, 0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const float d = v[i] * (g[i] - s) + (a.dlogits ? add[i] : 0.f);
            const int e = row16_expert<WIDE>(row, i);
            dl[lt][e] = on && e < E ? d : 0.f;
        }
        if (on && row == 0) atomicOr(&mask, 1u << lt);
    }
    __syncthreads();
    if (threadIdx.x == 0) a.masks[blockIdx.x] = mask;
    // For dWg: blocks of 16 experts, steps are the 32 tokens.
    char* const out = a.dl_dw + (size_t)blockIdx.x * 3 * a.nb * 1024;
    for (int p = threadIdx.x; p < a.nb * 64; p += 256) {
        const int l = p & 63, e = (p >> 6) * 16 + (l & 15), t0 = 8 * (l >> 4);
        bf16x8 hi, mid, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __bf16 h, m, w;
            split3(e < 16 * NV ? dl[t0 + i][e] : 0.f, h, m, w);
            hi[i] = h; mid[i] = m; lo[i] = w;
        }
        bf16x8* const o = reinterpret_cast<bf16x8*>(out) + p;
        o[0] = hi;
        o[a.nb * 64] = mid;
        o[2 * a.nb * 64] = lo;
    }
    if (!a.dx) return;
    // For dx: blocks of 16 tokens, steps are experts.
    char* const out2 = a.dl_dx + (size_t)blockIdx.x * 4 * a.kb * 1024;
    for (int p = threadIdx.x; p < 2 * a.kb * 64; p += 256) {
        const int l = p & 63, half = (p >> 6) / a.kb, kb = (p >> 6) % a.kb, t = 16 * half + (l & 15), e0 = kb * 32 + 8 * (l >> 4);
        bf16x8 hi, mid;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __bf16 h, m, w;
            split3(e0 + i < 16 * NV ? dl[t][e0 + i] : 0.f, h, m, w);
            hi[i] = h; mid[i] = m;
        }
        bf16x8* const o = reinterpret_cast<bf16x8*>(out2) + (size_t)half * 2 * a.kb * 64 + kb * 64 + l;
        o[0] = hi;
        o[a.kb * 64] = mid;
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

// ---- dx = dl Wg^T ---------------------------------------------------------------------------
// A workgroup of 8 wavefronts takes 256 tokens and a part of H.  A wavefront keeps the dl of 32 tokens in registers; the gate matrix
// comes 128 columns at a time through a ring of LDS stages.  The gate matrix is the row operand, so that a lane ends up with 8
// consecutive columns of a token (two blocks whose rows are interleaved by fours) and stores 16 bytes.
template <int KB>
struct DxTile {
    static constexpr int GROUPS = 4;                  // groups of 32 columns to a stage
    static constexpr int STAGE = GROUPS * 2 * KB * 1024;   // KB wave-loads of 1 KiB to a wavefront
    static constexpr int NS = KB <= 4 ? 4 : KB <= 6 ? 3 : 2;
    static constexpr int LDS = NS * STAGE;
    static constexpr int STORES = GROUPS * 2;         // of a wavefront, to a stage
};

template <int KB>
__device__ __forceinline__ void dx_tile(const RouteBackwardArgs& a, const int id, const lds_t lds) {
    typedef DxTile<KB> L;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = id % a.dx_tiles, part = id / a.dx_tiles;
    const int t32 = tile * 8 + wave, here = min(t32, a.steps - 1);
    const bool full = t32 * 32 + 32 <= a.T;
    const int g0 = part * a.dx_groups, g1 = min(g0 + a.dx_groups, a.H / 32);
    const int n = (g1 - g0 + L::GROUPS - 1) / L::GROUPS;
    const int last_block = g1 * 2 * KB - 1;
    auto issue = [&](const int i, const int stage) {
#pragma unroll
        for (int u = 0; u < KB; ++u) {
            const int q = wave * KB + u;
            const int blk = min((g0 + min(i, n - 1) * L::GROUPS) * 2 * KB + q, last_block);
            load16_to_lds(a.wg_blocks + (size_t)blk * 1024 + lane * 16, lds + stage * L::STAGE + q * 1024);
        }
    };
    bf16x8 d[2][2][KB];   // [half][piece]
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                d[half][q][kb] = reinterpret_cast<const bf16x8*>(a.dl_dx)[((size_t)(here * 2 + half) * 2 * KB + q * KB + kb) * 64 + lane];
#pragma unroll
    for (int i = 0; i < L::NS - 1; ++i) issue(i, i);
    const int t = t32 * 32 + (lane & 15);
    int stage = 0;
    for (int i = 0; i < n; ++i) {
        // Loads and stores retire in the order they were issued.  A wavefront whose tokens all exist stores the same number of times in
        // every stage but the last, so it can leave those behind the stage's loads in flight; others wait for all but loads.
        if (full) ring_wait<(L::NS - 2) * KB + (L::NS - 1) * L::STORES>();
        else ring_wait<(L::NS - 2) * KB>();
        ring_meet();
        int next = stage + L::NS - 1;
        if (next >= L::NS) next -= L::NS;
        issue(i + L::NS - 1, next);
        const lds_t w = lds + stage * L::STAGE + lane * 16;
#pragma unroll
        for (int u = 0; u < L::GROUPS; ++u) {
            const int g = g0 + i * L::GROUPS + u;
            if (g >= g1) break;
            f32x4 acc[2][2] = {};
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int q = 1; q >= 0; --q)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const bf16x8 m = *(frag_ptr_t)(w + ((u * 2 + b) * KB + kb) * 1024);
#pragma unroll
                        for (int half = 0; half < 2; ++half) acc[half][b] = mfma(m, d[half][q][kb], acc[half][b]);
                    }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                bf16x8 o;
#pragma unroll
                for (int j = 0; j < 4; ++j) { o[j] = (__bf16)acc[half][0][j]; o[4 + j] = (__bf16)acc[half][1][j]; }
                if (full || t + 16 * half < a.T)
                    *reinterpret_cast<bf16x8*>(a.dx + ((size_t)(t + 16 * half) * a.H + g * 32 + 8 * (lane >> 4)) * 2) = o;
            }
        }
        if (++stage == L::NS) stage = 0;
    }
    ring_wait<0>();   // no load may land in LDS that belongs to another workgroup
}

// ---- dWg = x^T dl ---------------------------------------------------------------------------
// A workgroup of 8 wavefronts takes 256 columns of x, all experts and a part of the tokens, 32 tokens at a time through a ring of LDS
// stages filled by direct loads: x as it lies (rows of 512 bytes, 32-byte chunks swizzled by row), dl in operand blocks.  The tokens
// are the contraction, so x is read from LDS by the transposing read.  Rows of x past the end and of tokens that do not count come
// from a page of zeros: their dl is zero, but what x holds there may be no number.
// Experts are the row operand: a lane ends up with four consecutive experts of a column.
template <int NB>
struct DwTile {
    static constexpr int WE = NB >= 4 ? 2 : 1;        // wavefronts along the experts
    static constexpr int WH = 8 / WE;                 // and along the columns
    static constexpr int HB = 16 / WH;                // blocks of 16 columns to a wavefront
    static constexpr int EB = NB / WE;                // blocks of 16 experts to a wavefront
    static constexpr int XBYTES = 32 * ROUTE_BACKWARD_TILE * 2;
    static constexpr int NL = (16 + 3 * NB + 7) / 8;  // wave-loads of 1 KiB to a wavefront and stage
    static constexpr int MORE = (16 + 3 * NB) % 8;    // wavefronts with NL wave-loads, where not all have as many
    static constexpr int STAGE = (16 + 3 * NB) * 1024;
    static constexpr int NS = 4 * STAGE <= 80 * 1024 ? 4 : 3 * STAGE <= 160 * 1024 ? 3 : 2;
    static constexpr int LDS = NS * STAGE;
};

// Rows 0..3 and 8..11 (16..19 and 24..27, ...), which a transposing read takes at a time, in different 32-byte chunks of 256 bytes.
__device__ __forceinline__ int swizzle(const int r) { return (r & 3) | ((r >> 1) & 4); }

template <int NB>
__device__ __forceinline__ void dw_tile(const RouteBackwardArgs& a, const int id, const lds_t lds) {
    typedef DwTile<NB> L;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ht = id % a.dw_tiles, split = id / a.dw_tiles;
    const int h0 = ht * ROUTE_BACKWARD_TILE;
    const int s0 = split * a.split_steps, s1 = min(s0 + a.split_steps, a.steps);
    const int we = wave % L::WE, wh = wave / L::WE;

    // Which of a step's tokens count, read one step ahead.
    typedef const __attribute__((address_space(4))) uint32_t* masks_t;
    const masks_t masks = (masks_t)a.masks;
    // wave-load i of this wave is load q = wave + 8 i of the stage: 16 of x (two rows each), then dl's blocks
    auto issue = [&](const int step, const uint32_t mask, const int stage) {
        const lds_t base = lds + stage * L::STAGE;
#pragma unroll
        for (int i = 0; i < L::NL; ++i) {
            const int q = wave + 8 * i;
            if (q >= 16 + 3 * NB) break;   // the last of some wavefronts
            const char* p = a.zeros + lane * 16;
            if (i < 2) {
                const int r = 2 * q + (lane >> 5);
                const int c = (lane & 31) ^ (swizzle(r) << 1);      // source chunk of 16 bytes
                const int h = h0 + c * 8;
                if ((mask >> r & 1) && h < a.H) p = a.x + ((size_t)(step * 32 + r) * a.H + h) * 2;
            } else {
                p = a.dl_dw + ((size_t)step * 3 * NB + (q - 16)) * 1024 + lane * 16;
            }
            load16_to_lds(p, base + q * 1024);
        }
    };

    f32x4 acc[L::EB][L::HB] = {};
    f32x4 bias[L::EB] = {};
    const bool sums = ht == 0 && wh == 0;   // whose dl blocks are added up for dbias, too

    for (int i = 0; i < L::NS - 1; ++i) {
        const int s = min(s0 + i, s1 - 1);
        issue(s, masks[s], i);
    }
    auto steps = [&]<bool SUMS>() {
        bf16x8 ones;
#pragma unroll
        for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
        int stage = 0;
        uint32_t mask = masks[min(s0 + L::NS - 1, s1 - 1)];
        for (int s = s0; s < s1; ++s) {
            if (L::MORE == 0 || wave < L::MORE) ring_wait<(L::NS - 2) * L::NL>();
            else ring_wait<(L::NS - 2) * (L::NL - 1)>();
            ring_meet();
            int next = stage + L::NS - 1;
            if (next >= L::NS) next -= L::NS;
            issue(min(s + L::NS - 1, s1 - 1), mask, next);
            mask = masks[min(s + L::NS, s1 - 1)];
            const lds_t xs = lds + stage * L::STAGE, ds = xs + L::XBYTES;
            bf16x8 xf[L::HB];
            {
                const int r = 8 * (lane >> 4) + ((lane & 15) >> 2);
                const lds_t p = xs + r * 512 + (lane & 3) * 8;
                const int f = swizzle(r);   // that of row r + 4, too
                const int c = wh * L::HB;
                if constexpr (L::HB == 2) read_transposed(xf, p + ((c ^ f) << 5), p + (((c + 1) ^ f) << 5));
                else read_transposed(xf, p + ((c ^ f) << 5), p + (((c + 1) ^ f) << 5), p + (((c + 2) ^ f) << 5), p + (((c + 3) ^ f) << 5));
            }
#pragma unroll
            for (int eb = 0; eb < L::EB; ++eb)
#pragma unroll
                for (int q = 2; q >= 0; --q) {
                    const bf16x8 d = *(frag_ptr_t)(ds + (q * NB + we * L::EB + eb) * 1024 + lane * 16);
#pragma unroll
                    for (int hb = 0; hb < L::HB; ++hb) acc[eb][hb] = mfma(d, xf[hb], acc[eb][hb]);
                    if (SUMS) bias[eb] = mfma(d, ones, bias[eb]);
                }
            if (++stage == L::NS) stage = 0;
        }
    };
    if (sums) steps.template operator()<true>();
    else steps.template operator()<false>();
    ring_wait<0>();   // no load may land in LDS that belongs to another workgroup
    float* const out = a.partial + (size_t)split * (a.H + 1) * (16 * NB);
#pragma unroll
    for (int hb = 0; hb < L::HB; ++hb) {
        const int h = h0 + (wh * L::HB + hb) * 16 + (lane & 15);
        if (h < a.H)
#pragma unroll
            for (int eb = 0; eb < L::EB; ++eb)
                *reinterpret_cast<f32x4*>(out + (size_t)h * (16 * NB) + (we * L::EB + eb) * 16 + 4 * (lane >> 4)) = acc[eb][hb];
    }
    if (sums && (lane & 15) == 0)
#pragma unroll
        for (int eb = 0; eb < L::EB; ++eb)
            *reinterpret_cast<f32x4*>(out + (size_t)a.H * (16 * NB) + (we * L::EB + eb) * 16 + 4 * (lane >> 4)) = bias[eb];
}

// Both products in one launch: the workgroups of dWg, then those of dx.
template <int NB>
__global__ __launch_bounds__(512) void route_backward_products_kernel(const RouteBackwardArgs a) {
    extern __shared__ char lds_raw[];
    const lds_t lds = (lds_t)lds_raw;
    const int n = a.dw_tiles * a.splits;
    if ((int)blockIdx.x < n) dw_tile<NB>(a, xcd_place(blockIdx.x, n), lds);
    else dx_tile<(NB + 1) / 2>(a, blockIdx.x - n, lds);
}
template <int NB>
constexpr int products_lds() {
    return DwTile<NB>::LDS > DxTile<(NB + 1) / 2>::LDS ? DwTile<NB>::LDS : DxTile<(NB + 1) / 2>::LDS;
}

// dWg and dbias: the parts of the tokens added in order.
__global__ __launch_bounds__(256) void route_backward_sum_kernel(const RouteBackwardArgs a) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, n = (size_t)(a.H + 1) * a.E;
    if (i >= n) return;
    const size_t h = i / a.E, e = i - h * a.E, ld = 16 * a.nb;
    float* const out = h < (size_t)a.H ? a.dwg + i : a.dbias ? a.dbias + e : nullptr;
    if (!out) return;
    const float* p = a.partial + h * ld + e;
    float v = 0.f;
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) v += p[(size_t)s * (a.H + 1) * ld];
    *out = a.accumulate ? *out + v : v;
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

hipError_t route_backward_init() {
    hipError_t e = hipSuccess;
    for (int nb : {1, 2, 4, 6, 8, 10, 12, 16}) {
        const hipError_t r = for_blocks(nb, []<int NB>() {
            return hipFuncSetAttribute((const void*)route_backward_products_kernel<NB>, hipFuncAttributeMaxDynamicSharedMemorySize, products_lds<NB>());
        });
        if (e == hipSuccess) e = r;
    }
    return e;
}

hipError_t launch_route_backward(const RouteBackwardArgs& a, hipStream_t st) {
    const bool wide = wide_rows(a.E, {a.logits, a.dlogits ? a.dlogits : a.logits});
    const unsigned pack = a.dx ? (unsigned)(((size_t)a.H / 16 * a.kb * 64 + 255) / 256) : 0u;
    hipError_t e = for_row16(a.E, wide, [&]<int NV, bool WIDE>() {
        hipLaunchKernelGGL((route_backward_prep_kernel<NV, WIDE>), dim3(a.steps + pack), dim3(256), 0, st, a, a.steps);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    e = for_blocks(a.nb, [&]<int NB>() {
        const unsigned grid = (unsigned)(a.dw_tiles * a.splits + (a.dx ? a.dx_tiles * a.dx_parts : 0));
        hipLaunchKernelGGL(route_backward_products_kernel<NB>, dim3(grid), dim3(512), products_lds<NB>(), st, a);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(route_backward_sum_kernel, dim3((unsigned)(((size_t)(a.H + 1) * a.E + 255) / 256)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_route_backward_empty(const moe_shape& s, float* dwg, float* dbias, hipStream_t st) {
    const size_t n = (size_t)s.H * s.E;
    hipLaunchKernelGGL(route_backward_empty_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, n, s.E, dwg, dbias);
    return hipGetLastError();
}

}  // namespace moe
