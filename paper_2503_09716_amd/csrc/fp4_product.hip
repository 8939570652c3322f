// Grouped products of MXFP4 rows and MXFP4 matrices on the scaled matrix instruction, fp32 accumulation.
//
//   plain: out[r, n] = sum_k x[r, k] W_e[k, n]        gated: out[r, n] = silu(x[r] . Wa_e[n]) * (x[r] . Wb_e[n])
// for the rows r of group e.  v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 values in 16 cycles, four times what
// the bf16 form does, and takes one scale for 32 values of a row.
//
// What bounds it: at low heights reading the matrices once.  Above some hundred rows a group no single thing.  A sub-tile of 256 x 256 takes 0.90 us, 0.74 without its loads and
// 0.79 without its matrix instructions, which the power limit holds at 23 for 16 cycles on real data (6.2 to 6.7 PFLOP/s in a loop of registers alone, 8.0 to 8.4 on
// zeros).  A tile's epilogue comes behind its K loop, not beside one: the next tile's first hand-overs wait for the stores, which are older than the loads that
// they may leave on their way.  Measured, and in a copy without the epilogues: gate/up of 8 experts, K = 4096, N = 14336, 8192 rows 503 us (3.8 PFLOP/s; 14 tiles
// to a workgroup of 29 us of K loop, 3 of waits at its ends, 4 of epilogue), 443; of 64 experts, K = 2048, N = 1408, 18006 rows 98, 80; down, K = 1408, N = 2048,
// 98304 rows to fp32 254 (12 tiles of 10 us of K loop, 1.6 of waits, 10 of stores at 6.9 TB/s), 138, to bf16 203, 138; K = 1536, N = 5120, 160 experts, 12000 rows
// 143 (5.6 TB/s), 116.
#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "fp4.h"
#include "plan.h"

namespace moe {
namespace {

__device__ __forceinline__ float silu_times(const float g, const float u) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u; }

__global__ __launch_bounds__(256) void fp4_plan_kernel(const PlanArgs p) { plan_list(p, 0, p.offsets); }

// ---- tiles ---------------------------------------------------------------------------------
// A workgroup multiplies up to ROWS rows of x with 256 rows of W (gated: 128 of each matrix, so that the gate meets its up value in registers) in
// sub-tiles of 128 along K.  Codes go from memory straight into a ring of NS LDS stages of 64-byte rows, NS - 1 sub-tiles ahead; a row's 16
// scale bytes of a group of four sub-tiles into places of their own.  A fragment is read from the next stage right after its last use, and one
// barrier a sub-tile hands the ring over.  Two forms:
struct Long {    // long batches: one workgroup of eight wavefronts to a CU, which takes every 256th tile and asks for the next one's first sub-tiles behind the
                 // last ones of its own
    static constexpr int NW = 8, NS = 4, ROWS = 256, MW = 2, SCALES = 2;   // MW: wavefronts side by side along x
    static constexpr bool NEXT = true;
};
struct Short {   // short and ragged ones: two workgroups of four wavefronts to a CU, one tile each
    static constexpr int NW = 4, NS = 3, ROWS = 128, MW = 1, SCALES = 1;
    static constexpr bool NEXT = false;
};
constexpr int ROWB = 64, WROWS = 256;
template <class C>
struct Ring {
    static constexpr int X = C::ROWS * ROWB, STAGE = X + WROWS * ROWB;
    static constexpr int SCALE_X = C::ROWS * 16, SCALE_STAGE = SCALE_X + WROWS * 16;
    static constexpr int BYTES = C::NS * STAGE + C::SCALES * SCALE_STAGE;
    static constexpr int XL = C::ROWS / 16 / C::NW, WL = WROWS / 16 / C::NW, SL = 8 / C::NW;   // loads of a sub-tile per wavefront, of a tile of full height
};
constexpr int ROUNDS = 64;   // tiles of a workgroup that it can list itself
template <class C>
constexpr int OWN = C::NEXT ? (ROUNDS + 1) * 16 : 0;
static_assert(Ring<Long>::BYTES + OWN<Long> <= 160 * 1024 && Ring<Short>::BYTES <= 80 * 1024, "LDS");

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
template <bool NT>
__device__ __forceinline__ void store_b128(const __amdgpu_buffer_rsrc_t rsrc, const uint32_t voff, const u32x4 v) {
#if defined(__gfx950__)
    __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, voff, 0, NT ? 2 : 0);
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
// The same on an accumulator of zeros.
__device__ __forceinline__ void mfma_tile_first(f32x4& c, const i32x4& a, const i32x4& b, const uint32_t sa, const uint32_t sb) {
#if defined(__gfx950__)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, 0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                 : "=a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
#endif
}
// Here, not earlier: left alone all accumulators are copied ahead of the first store.
__device__ __forceinline__ float read_acc(const float& a) {
    float v = 0.f;
#if defined(__gfx950__)
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(a) : "memory");
#endif
    return v;
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

// A tile: what its loads need, one tile ahead of its use.
template <class C>
struct TileLoads {
    const char *w_at, *u_at;                    // the matrix (gated: gate, up)
    uint32_t x[Ring<C>::XL], sc[Ring<C>::SL];   // offsets of this lane's pieces
    int w[Ring<C>::WL];                         // and of this wavefront's blocks of W
    int row0, nrows, n0;
    bool any;
};

// Through the scalar cache: what the launch before left, at an address that is the same for the wavefront.
template <class T>
__device__ __forceinline__ T scalar_load(const T* ptr) {
    return *(const __attribute__((address_space(4))) T*)(uintptr_t)ptr;
}

// The lane's number, anew: what is computed from it then stays where it is needed and does not take registers around the loop over the tiles.
__device__ __forceinline__ int fresh_lane() {
    int lane = threadIdx.x & 63;
#if defined(__gfx950__)
    asm volatile("" : "+v"(lane));
#endif
    return lane;
}

__device__ __forceinline__ int row_of(const Fp4Product& p, const int r) { return p.row_index ? p.row_index[r] : r; }

// Workgroup id -> position in the order of the tiles: ids are dealt to the 8 XCDs in turn; inside each whole round of 256 tiles an XCD gets a run of 32.
__device__ __forceinline__ int tile_order(const int wg, const int total) {
    if (wg >= (total & ~255)) return wg;
    const int r = wg & 255;
    return (wg - r) + (r & 7) * 32 + (r >> 3);
}

// m-tile and columns of the tile at place `at` of `count` m-tiles, the first n_run of which are in group order.
template <bool GATED>
__device__ __forceinline__ int place_of(const Fp4Product& p, const int count, const int n_run, const int at, int& n0) {
    const int L = tile_order(at, count * p.n_tiles);
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
    n0 = n_tile * (GATED ? 128 : WROWS);
    return mt;
}

// The list of m-tiles that plan_list would leave in memory, by one wavefront in its registers: group 64 q + lane is slot q of a lane.
constexpr int SLOTS = 4;
struct WaveList {
    int row0[SLOTS], rows[SLOTS], h[SLOTS], nfull[SLOTS], first[SLOTS], nrun[SLOTS];   // first: of its tiles in group order
    int blocks[SLOTS];                                                                // of 32 rows of its moved tail, or 0
    int n_run, count;
};
__device__ __forceinline__ int scan_wave(int v) {   // inclusive prefix sums over the lanes
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);   // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // lane 15 of a row to the next one
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // lane 31 to the upper half
    return v;
}
template <int TM>
__device__ __forceinline__ WaveList wave_list(const Fp4Product& p, const int lane) {
    WaveList l = {};
    int at[SLOTS] = {}, end[SLOTS] = {};
#pragma unroll
    for (int q = 0; q < SLOTS; ++q)
        if (q * 64 < p.E) {
            const int e = min(q * 64 + lane, p.E - 1);
            at[q] = p.offsets[e];
            end[q] = p.offsets[e + 1];
        }
    int moved = 0;
#pragma unroll
    for (int q = 0; q < SLOTS; ++q)
        if (q * 64 < p.E) {
            l.row0[q] = at[q];
            l.rows[q] = q * 64 + lane < p.E ? end[q] - at[q] : 0;
            const GroupCut cut = cut_group(l.rows[q], TM, false, true);
            const int blocks = (cut.tail + 31) >> 5;
            const bool last = blocks > 0 && !cut.even && blocks * 64 <= TM;
            l.h[q] = cut.h;
            l.nfull[q] = cut.nfull;
            l.nrun[q] = cut.nfull + (blocks > 0 && !last);
            l.blocks[q] = last ? blocks : 0;
            const int upto = scan_wave(l.nrun[q]);
            l.first[q] = l.n_run + upto - l.nrun[q];
            l.n_run += __builtin_amdgcn_readlane(upto, 63);
            moved += __popcll(__ballot(last));
        }
    l.count = l.n_run + moved;
    return l;
}
__device__ __forceinline__ TileDesc m_tile_at(const Fp4Product& p, const WaveList& l, const int mt, const int lane) {
    TileDesc d = {0, 0, 0, 0};
    if (mt < l.n_run) {
#pragma unroll
        for (int q = 0; q < SLOTS; ++q)
            if (q * 64 < p.E) {
                const int i = mt - l.first[q];
                const uint64_t hit = __ballot(i >= 0 && i < l.nrun[q]);
                if (hit == 0) continue;
                const int from = __ffsll((unsigned long long)hit) - 1, at = min(i, l.nfull[q]) * l.h[q];
                d = TileDesc{q * 64 + from, __builtin_amdgcn_readlane(l.row0[q] + at, from), __builtin_amdgcn_readlane(min(l.h[q], l.rows[q] - at), from), 0};
            }
        return d;
    }
    int rank = mt - l.n_run;   // of the tails: higher ones first, then in group order
    for (int b = 4; b > 0; --b)
#pragma unroll
        for (int q = 0; q < SLOTS; ++q)
            if (q * 64 < p.E) {
                const uint64_t tails = __ballot(l.blocks[q] == b);
                const int n = __popcll(tails);
                if (rank >= 0 && rank < n) {
                    const int from = __ffsll((unsigned long long)__ballot((tails >> lane & 1) && __popcll(tails & ((1ull << lane) - 1)) == rank)) - 1, at = l.nfull[q] * l.h[q];
                    d = TileDesc{q * 64 + from, __builtin_amdgcn_readlane(l.row0[q] + at, from), __builtin_amdgcn_readlane(l.rows[q] - at, from), 0};
                }
                rank -= n;
            }
    return d;
}
// The tile at place `at` of the launch (nrows = 0: there is none).
template <bool GATED>
__device__ __forceinline__ TileDesc tile_at(const Fp4Product& p, const WaveList& l, const int at, const int lane, int& n0) {
    n0 = 0;
    if (at >= l.count * p.n_tiles) return TileDesc{0, 0, 0, 0};
    return m_tile_at(p, l, place_of<GATED>(p, l.count, l.n_run, at, n0), lane);
}
// From the list in memory.
template <bool GATED>
__device__ __forceinline__ TileDesc tile_at(const Fp4Product& p, const int count, const int n_run, const int at, int& n0) {
    n0 = 0;
    if (at >= count * p.n_tiles) return TileDesc{0, 0, 0, 0};
    const i32x4 v = scalar_load((const i32x4*)p.descs + __builtin_amdgcn_readfirstlane(place_of<GATED>(p, count, n_run, at, n0)));
    return TileDesc{v[0], v[1], v[2] & TILE_ROWS_MASK, v[3]};
}

// Rows of x for the four pieces that this lane loads of a sub-tile, and for its scales; rows past the end are the last one again.
template <class C>
struct TileRows {
    int x[Ring<C>::XL], xs;
};
template <class C>
__device__ __forceinline__ TileRows<C> tile_rows(const Fp4Product& p, const TileDesc& d, const int lane, const int wave) {
    TileRows<C> r = {};
    if (d.nrows == 0) return r;
#pragma unroll
    for (int i = 0; i < Ring<C>::XL; ++i) r.x[i] = row_of(p, d.row0 + min((i * C::NW + wave) * 16 + (lane >> 2), d.nrows - 1));
    r.xs = row_of(p, d.row0 + min((wave & 3) * 64 + lane, d.nrows - 1));
    return r;
}

template <bool GATED>
__device__ __forceinline__ void tile_weights(const Fp4Product& p, const TileDesc& d, const char*& w_at, const char*& u_at) {
    const int group = __builtin_amdgcn_readfirstlane(d.group);
    w_at = scalar_load((const char* const*)p.wa + group);
    u_at = GATED ? scalar_load((const char* const*)p.wb + group) : w_at;
}

template <class C, bool GATED>
__device__ __forceinline__ TileLoads<C> tile_loads(const Fp4Product& p, const TileDesc& d, const int n0, const TileRows<C>& rows, const char* w_at,
                                                   const char* u_at, const int lane, const int wave) {
    TileLoads<C> t;
    t.row0 = d.row0;
    t.nrows = d.nrows;
    t.n0 = n0;
    t.any = d.nrows > 0;
    t.w_at = w_at;
    t.u_at = u_at;
    const int lrow = lane >> 2, lpiece = (lane & 3) ^ block_swizzle(lrow);
#pragma unroll
    for (int i = 0; i < Ring<C>::XL; ++i) t.x[i] = (uint32_t)rows.x[i] * (uint32_t)(p.sub_tiles * 64) + (uint32_t)(lpiece * 16);
#pragma unroll
    for (int i = 0; i < Ring<C>::WL; ++i) {
        const int qw = i * C::NW + wave, block = min((n0 >> 4) + (GATED ? (qw & 7) : qw), (p.N >> 4) - 1);
        t.w[i] = block * p.sub_tiles * 1024;
    }
    const int wr = (wave & 3) * 64 + lane, n = min(n0 + (GATED ? (wr & 127) : wr), p.N - 1);
    t.sc[Ring<C>::SL - 1] = p.scales_at + (uint32_t)(n >> 4) * (uint32_t)(p.groups * 256) + (uint32_t)((n & 15) * 16);
    if (Ring<C>::SL == 2 || wave < 4) t.sc[0] = (uint32_t)rows.xs * (uint32_t)(p.groups * 16);
    return t;
}

template <class C>
__device__ __forceinline__ void load_x(const TileLoads<C>& t, const __amdgpu_buffer_rsrc_t rs_x, lds_t stage, const int wave, const int i, const int sub) {
    load_lds(rs_x, (lptr_t)(stage + (i * C::NW + wave) * 1024), t.x[i], sub * 64);
}
template <class C, bool GATED>
__device__ __forceinline__ void load_w(const TileLoads<C>& t, lds_t stage, const int wave, const int i, const int sub) {
    load_lds(rsrc_of(GATED && i * 2 >= Ring<C>::WL ? t.u_at : t.w_at), (lptr_t)(stage + Ring<C>::X + (i * C::NW + wave) * 1024), (uint32_t)(threadIdx.x & 63) * 16u, t.w[i] + sub * 1024);
}
// 64 rows of x or W to a wavefront: with eight of them one of the two, with four up to both.
template <class C, bool GATED>
__device__ __forceinline__ void load_scales(const TileLoads<C>& t, const __amdgpu_buffer_rsrc_t rs_xs, lds_t stage, const int wave, const int q) {
    const int part = wave & 3;
    if (wave < 4 && part * 64 < C::ROWS) load_lds(rs_xs, (lptr_t)(stage + part * 1024), t.sc[0], q * 16);
    if (C::NW == 4 || wave >= 4)
        load_lds(rsrc_of(GATED && part >= 2 ? t.u_at : t.w_at), (lptr_t)(stage + Ring<C>::SCALE_X + part * 1024), t.sc[Ring<C>::SL - 1], q * 256);
}
// A whole sub-tile of a tile whose height the caller does not know.
template <class C, bool GATED>
__device__ __forceinline__ void load_sub_tile(const TileLoads<C>& t, const __amdgpu_buffer_rsrc_t rs_x, lds_t stage, const int wave, const int sub) {
#pragma unroll
    for (int i = 0; i < Ring<C>::XL; ++i)
        if (i == 0 || i * C::NW * 16 < t.nrows) load_x<C>(t, rs_x, stage, wave, i, sub);
#pragma unroll
    for (int i = 0; i < Ring<C>::WL; ++i) load_w<C, GATED>(t, stage, wave, i, sub);
}

// A tile of TI * 32 rows: MW x 4 wavefronts, each with XB blocks of 16 rows of x and four of W (gated: two of each matrix).
constexpr int WB = 4, WBH = 2;
template <class C, int TI>
struct Grid {
    static constexpr int XB = 2 * TI / C::MW;
    static __device__ __forceinline__ int x_row(const int wave) { return (wave >> 2) * XB * 16; }
    // of the first of its rows of W (gated: in the gate's half, and as far into the other one)
    static __device__ __forceinline__ int w_row(const int wave, const bool gated) { return (wave & 3) * (gated ? 32 : 64); }
};

// Multiplies tile t, whose first sub-tiles and scales are in the ring from stages `base` and `sbase` on.  NEXT: asks for the first ones of the next tile
// behind the last ones of its own; when it returns, those have landed for every wavefront.
template <class C, int TI, bool GATED>
__device__ __forceinline__ void multiply(const Fp4Product& p, const TileLoads<C>& t, const TileLoads<C>& next, const __amdgpu_buffer_rsrc_t rs_x,
                                         const __amdgpu_buffer_rsrc_t rs_xs, lds_t ring, const int base, const int sbase,
                                         f32x4 (&acc)[WB][Grid<C, TI>::XB]) {
    constexpr int XB = Grid<C, TI>::XB, NS = C::NS, STAGE = Ring<C>::STAGE;
    constexpr int NLX = (2 * TI + C::NW - 1) / C::NW, NL = NLX + Ring<C>::WL;   // loads of a sub-tile per wavefront
    constexpr int NL0 = XB * NL / (2 * XB);                                     // of them, those issued before the hand-over
    const int lane = fresh_lane(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rl = lane & 15, g = lane >> 4;
    const int KT = p.sub_tiles;
    lds_t const scale_ring = ring + NS * STAGE;
    const int x_row = Grid<C, TI>::x_row(wave), wn_row = Grid<C, TI>::w_row(wave, GATED);
    const uint32_t off = (uint32_t)(rl * ROWB + ((g ^ block_swizzle(rl)) << 4)), offS = (uint32_t)(rl * 16 + g * 4);
    const uint32_t offX = off + (uint32_t)(x_row * ROWB), offW = off + (uint32_t)(Ring<C>::X + wn_row * ROWB);
    const uint32_t offSX = offS + (uint32_t)(x_row * 16), offSW = offS + (uint32_t)(Ring<C>::SCALE_X + wn_row * 16);
    auto w_row = [](const int hf, const int jj) __attribute__((always_inline)) { return GATED ? hf * 128 + jj * 16 : (hf * WBH + jj) * 16; };
    auto stage_of = [&](const int s) __attribute__((always_inline)) { return ring + (int)((uint32_t)(base + s) % NS) * STAGE; };
    auto scales_of = [&](const int q) __attribute__((always_inline)) { return scale_ring + (int)((uint32_t)(sbase + q) % C::SCALES) * Ring<C>::SCALE_STAGE; };

    i32x4 xf[XB], wA[WBH], wB[WBH];
    uint32_t sx[XB], sw[WB], sx_next[XB], sw_next[WB];
    auto read_x = [&](lds_t stage, const int i) __attribute__((always_inline)) { xf[i] = *(lfrag_t)(stage + offX + i * 16 * ROWB); };
    auto read_w = [&](lds_t stage, const int hf, const int jj) __attribute__((always_inline)) {
        const i32x4 v = *(lfrag_t)(stage + offW + w_row(hf, jj) * ROWB);
        if (hf == 0) wA[jj] = v;
        else wB[jj] = v;
    };
    auto read_scales = [&](const int q) __attribute__((always_inline)) {
        lds_t const from = scales_of(q);
#pragma unroll
        for (int i = 0; i < XB; ++i) sx_next[i] = *(lword_t)(from + offSX + i * 256);
#pragma unroll
        for (int j = 0; j < WB; ++j) sw_next[j] = *(lword_t)(from + offSW + w_row(j / WBH, j % WBH) * 16);
    };

    // Half HF of sub-tile s: XB groups of two matrix instructions with one block of x.  RD: fragments of the next sub-tile are read, LD: sub-tile s + NS - 1 is
    // asked for, spread over the groups.
    auto part = [&](auto hf_tag, auto first_tag, auto rd_tag, auto ld_tag, const int s) __attribute__((always_inline)) {
        constexpr int HF = decltype(hf_tag)::value;
        constexpr bool FIRST = decltype(first_tag)::value, RD = decltype(rd_tag)::value, LD = decltype(ld_tag)::value;
        lds_t const cur = stage_of(s), nxt = stage_of(s + 1), ahead = stage_of(s + NS - 1);
#pragma unroll
        for (int i = 0; i < XB; ++i) {
#pragma unroll
            for (int jj = 0; jj < WBH; ++jj) {
                const int j = HF * WBH + jj;
                const i32x4 w = HF == 0 ? wA[jj] : wB[jj];
                if (FIRST) mfma_tile_first(acc[j][i], w, xf[i], sw[j], sx[i]);
                else mfma_tile(acc[j][i], w, xf[i], sw[j], sx[i]);
            }
            if (HF == 1 && RD) read_x(nxt, i);
            constexpr int PER = (WBH + XB - 1) / XB;
            if (HF == 0 || RD)
#pragma unroll
                for (int jj = i * PER; jj < (i + 1) * PER && jj < WBH; ++jj) read_w(HF == 0 ? cur : nxt, HF == 0 ? 1 : 0, jj);
            if (LD) {
                constexpr int G = 2 * XB;
                const int q = HF * XB + i;
#pragma unroll
                for (int l = (q * NL) / G; l < ((q + 1) * NL) / G; ++l) {
                    if (l < NLX) load_x<C>(t, rs_x, ahead, wave, l, s + NS - 1);
                    else load_w<C, GATED>(t, ahead, wave, l - NLX, s + NS - 1);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    using T_ = std::true_type;
    using F_ = std::false_type;
    using H0 = std::integral_constant<int, 0>;
    using H1 = std::integral_constant<int, 1>;
    // Sub-tile s; its scales are byte 0 of sx and sw.
    auto sub_tile = [&](auto first_tag, auto rd_tag, auto ld_tag, const int s, auto sync) __attribute__((always_inline)) {
        if (C::SCALES == 2 && (s & 3) == 0 && s + 4 < KT) load_scales<C, GATED>(t, rs_xs, scales_of((s >> 2) + 1), wave, (s >> 2) + 1);
        if (decltype(first_tag)::value || (s & 3) == 0) {
#pragma unroll
            for (int i = 0; i < XB; ++i) sx[i] = sx_next[i];
#pragma unroll
            for (int j = 0; j < WB; ++j) sw[j] = sw_next[j];
        } else {
#pragma unroll
            for (int i = 0; i < XB; ++i) sx[i] >>= 8;
#pragma unroll
            for (int j = 0; j < WB; ++j) sw[j] >>= 8;
        }
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_nop 3" ::: "memory");   // between those and the first matrix instruction
        part(H0{}, first_tag, rd_tag, ld_tag, s);
        sync();
        // one place for scales: free once every wavefront is here
        if (C::SCALES == 1 && (s & 3) == 0 && s + 4 < KT) load_scales<C, GATED>(t, rs_xs, scales_of(0), wave, (s >> 2) + 1);
        // the scales of the next group came in since this one's first sub-tile
        if ((s & 3) == 3 && s + 1 < KT) read_scales((s >> 2) + 1);
        part(H1{}, first_tag, rd_tag, ld_tag, s);
    };

    read_scales(0);
#pragma unroll
    for (int i = 0; i < XB; ++i) {
        constexpr int PER = (WBH + XB - 1) / XB;
        read_x(stage_of(0), i);
#pragma unroll
        for (int jj = i * PER; jj < (i + 1) * PER && jj < WBH; ++jj) read_w(stage_of(0), 0, jj);
        __builtin_amdgcn_sched_barrier(0);
    }
    // One of the two wavefronts of a SIMD goes first, so that the other's matrix instructions fill its gaps instead of both meeting at each hand-over (us,
    // without and with: 8 experts, K = 4096, 250 rows gate/up 172, 162, 1024 rows 531, 525; down, K = 14336 108, 100 and 253, 248; 160 experts, K = 5120, 300 rows
    // 523, 510); not in the epilogue, which should not hold up the next tile's start (64 experts, K = 1408, 1500 rows to fp32 247.7, 245.5).
    if (C::NEXT && wave >= C::NW / 2) __builtin_amdgcn_s_setprio(1);
    int s = 0;
    // Scales may be among the loads that are younger than sub-tile s + 1, which then waits for a few more than it has to.
    auto steady = [] __attribute__((always_inline)) { ring_sync<(NS - 3) * NL + NL0>(); };
    // The last NS - 1 sub-tiles.  NEXT: in the stages that come free, the next tile's first ones.  Behind sub-tile KT - 1 are at least the
    // AFTER loads of the next tile's first sub-tile that every height has, or nothing.
    constexpr int AFTER = Ring<C>::WL + 1;
    static_assert(!C::NEXT || NS == 4, "what is waited for below");
    auto ask_next = [&] __attribute__((always_inline)) {
        const int ahead = s + NS - 1 - KT;
        if (C::NEXT && next.any && ahead >= 0 && ahead < KT) {
            if (ahead == 0) load_scales<C, GATED>(next, rs_xs, scales_of(p.groups), wave, 0);
            load_sub_tile<C, GATED>(next, rs_x, stage_of(KT + ahead), wave, ahead);
        }
    };
    auto late = [&] __attribute__((always_inline)) {
        if (C::NEXT && s == KT - 3) ring_sync<NL>();
        else if (C::NEXT && next.any && KT >= NS) ring_sync<AFTER>();
        else ring_sync<0>();
    };
    if (KT >= NS) {
        sub_tile(T_{}, T_{}, T_{}, 0, steady);
        for (s = 1; s + NS - 1 < KT; ++s) sub_tile(F_{}, T_{}, T_{}, s, steady);
    } else {   // all of it is there
        ask_next();
        sub_tile(T_{}, T_{}, F_{}, 0, late);
        s = 1;
    }
    for (; s < KT - 1; ++s) {
        ask_next();
        sub_tile(F_{}, T_{}, F_{}, s, late);
    }
    if (s < KT) {
        ask_next();
        sub_tile(F_{}, F_{}, F_{}, s, [] __attribute__((always_inline)) {});
    }
    if (C::NEXT) {
        if (next.any && KT < NS - 1) {   // KT = 1, 2: the sub-tiles above never came to the next tile's first one
            load_scales<C, GATED>(next, rs_xs, scales_of(p.groups), wave, 0);
            load_sub_tile<C, GATED>(next, rs_x, stage_of(KT), wave, 0);
        }
    }
    if (C::NEXT || !GATED) ring_sync<0>();   // store_tile writes into the ring
}

template <class C, int TI, bool GATED, bool NT>
__device__ __forceinline__ void store_tile(const Fp4Product& p, const TileLoads<C>& t, lds_t spare, f32x4 (&acc)[WB][Grid<C, TI>::XB]) {
    constexpr int XB = Grid<C, TI>::XB;
    const int lane = fresh_lane(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rl = lane & 15, g = lane >> 4;
    const int N = p.N, x_row = Grid<C, TI>::x_row(wave), wn_row = Grid<C, TI>::w_row(wave, GATED);
    if (C::NEXT) __builtin_amdgcn_s_setprio(0);
    mfma_drain();
    __builtin_amdgcn_sched_barrier(0);
    // W is the row operand: a lane has the four columns 4g .. 4g+3 of row rl of a block.  Rows past the end get an offset that the descriptor drops.
    const uint32_t rowbytes = (uint32_t)N * (p.out_fp32 ? 4u : 2u);
    const __amdgpu_buffer_rsrc_t rs_o = rsrc_of(p.out + (size_t)t.row0 * rowbytes, (uint32_t)t.nrows * rowbytes);
    auto offset = [&](const int row, const int col, const bool ok) __attribute__((always_inline)) {
        return ok && row < t.nrows ? (uint32_t)row * rowbytes + (uint32_t)col * (p.out_fp32 ? 4u : 2u) : 0xFFFFFFF0u;
    };
    const int col0 = t.n0 + wn_row;
    if constexpr (GATED) {
        // fp32: 16 bytes of a row; bf16: lanes 16 apart swap halves of two blocks for that.  A store covers 16 rows x 64 bytes.
        if (col0 >= N) return;   // N is a multiple of 32
#pragma unroll
        for (int i = 0; i < XB; ++i) {
            f32x4 v[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) v[j][q] = silu_times(read_acc(acc[j][i][q]), read_acc(acc[WBH + j][i][q]));
            const int row = x_row + i * 16 + rl;
            if (p.out_fp32) {
#pragma unroll
                for (int j = 0; j < 2; ++j) store_b128<NT>(rs_o, offset(row, col0 + j * 16 + g * 4, true), __builtin_bit_cast(u32x4, v[j]));
            } else {
                u32x2 o[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bf16x4 w = {(__bf16)v[j][0], (__bf16)v[j][1], (__bf16)v[j][2], (__bf16)v[j][3]};
                    o[j] = __builtin_bit_cast(u32x2, w);
                }
                // lane g: block g & 1, columns 8 (g >> 1) .. + 7 of it
                store_b128<NT>(rs_o, offset(row, col0 + (g & 1) * 16 + (g >> 1) * 8, true), swap_rows16(o[0], o[1]));
            }
            if (i % 2) __builtin_amdgcn_sched_barrier(0);
        }
    } else {
        // Whole lines: 16 rows x 64 columns at a time through 4 KiB of LDS that only this wavefront's loads fill, as four pieces of four rows; 16-byte
        // pieces of a row at slot piece ^ row, so that neither way has bank conflicts.  A store covers 4 rows x 256 bytes (fp32) or 8 x 128.
        typedef __attribute__((address_space(3))) f32x4* lpiece_t;
        auto place = [&](const int row, const int piece) __attribute__((always_inline)) {
            return (lpiece_t)(spare + (row >> 2) * C::NW * 1024 + (row & 3) * 256 + ((piece ^ row) << 4));
        };
#pragma unroll
        for (int i = 0; i < XB; ++i) {
#pragma unroll
            for (int j = 0; j < WB; ++j) *place(rl, j * 4 + g) = f32x4{read_acc(acc[j][i][0]), read_acc(acc[j][i][1]), read_acc(acc[j][i][2]), read_acc(acc[j][i][3])};
            if (p.out_fp32) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int r = q * 4 + (lane >> 4), col = col0 + (lane & 15) * 4;
                    store_b128<NT>(rs_o, offset(x_row + i * 16 + r, col, col < N), __builtin_bit_cast(u32x4, *place(r, lane & 15)));
                }
            } else {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int r = q * 8 + (lane >> 3), piece = (lane & 7) * 2, col = col0 + piece * 4;
                    const f32x4 lo = *place(r, piece), hi = *place(r, piece + 1);
                    const bf16x8 w = {(__bf16)lo[0], (__bf16)lo[1], (__bf16)lo[2], (__bf16)lo[3], (__bf16)hi[0], (__bf16)hi[1], (__bf16)hi[2], (__bf16)hi[3]};
                    store_b128<NT>(rs_o, offset(x_row + i * 16 + r, col, col < N), __builtin_bit_cast(u32x4, w));
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// NEXT: the next tile's descriptor and offsets are there, and its first three sub-tiles on their way, when the present one ends.
template <class C, bool GATED, bool NT>
__global__ __launch_bounds__(C::NW * 64, 2) void fp4_tile_kernel(const Fp4Product p) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int KT = p.sub_tiles;
    lds_t const ring = (lds_t)lds, scale_ring = ring + C::NS * Ring<C>::STAGE;
    const __amdgpu_buffer_rsrc_t rs_x = rsrc_of(p.codes), rs_xs = rsrc_of(p.scales);
    typedef __attribute__((address_space(3))) i32x4* lentry_t;
    lentry_t const own = (lentry_t)(ring + Ring<C>::BYTES);   // this workgroup's tiles
    int count = 0, n_run = 0, round = 0;
    TileDesc d = {0, 0, 0, 0};
    int n0 = 0, n0_next = 0, n0_after = 0, n0_last = 0, base = 0, sbase = 0;
    if (p.inside) {
        const WaveList l = wave_list<C::ROWS>(p, lane);
        if (C::NEXT) {
            for (int i = wave; i <= p.rounds; i += C::NW) {   // the list ends with none
                const TileDesc t = tile_at<GATED>(p, l, blockIdx.x + i * gridDim.x, lane, n0);
                if (lane == 0) own[i] = i32x4{t.group, t.row0, i < p.rounds ? t.nrows : 0, n0};
            }
            __syncthreads();
        } else {
            d = tile_at<GATED>(p, l, blockIdx.x, lane, n0);
        }
    } else {
        count = scalar_load(&p.plan->n_gate_up);
        n_run = scalar_load(&p.plan->n_run_up);
    }
    auto following = [&](int& n0) __attribute__((always_inline)) {
        if (C::NEXT && p.inside) {
            const i32x4 v = own[round++];
            n0 = __builtin_amdgcn_readfirstlane(v[3]);
            return TileDesc{__builtin_amdgcn_readfirstlane(v[0]), __builtin_amdgcn_readfirstlane(v[1]), __builtin_amdgcn_readfirstlane(v[2]), 0};
        }
        return tile_at<GATED>(p, count, n_run, blockIdx.x + round++ * gridDim.x, n0);
    };
    if (C::NEXT || !p.inside) d = following(n0);
    if (d.nrows == 0) return;
    const char *w_at, *u_at;
    tile_weights<GATED>(p, d, w_at, u_at);
    TileLoads<C> t = tile_loads<C, GATED>(p, d, n0, tile_rows<C>(p, d, lane, wave), w_at, u_at, lane, wave), next;
    load_scales<C, GATED>(t, rs_xs, scale_ring, wave, 0);
    for (int s = 0; s < C::NS - 1 && s < KT; ++s) load_sub_tile<C, GATED>(t, rs_x, ring + s * Ring<C>::STAGE, wave, s);
    next.any = false;
    TileDesc after = {0, 0, 0, 0};   // two tiles on
    if (C::NEXT) {
        const TileDesc d_next = following(n0_next);
        tile_weights<GATED>(p, d_next, w_at, u_at);
        next = tile_loads<C, GATED>(p, d_next, n0_next, tile_rows<C>(p, d_next, lane, wave), w_at, u_at, lane, wave);
        after = following(n0_after);
    }
    ring_sync<0>();
    for (;;) {
        TileRows<C> rows;
        TileDesc last;
        auto run = [&](auto ti_tag) __attribute__((always_inline)) {
            constexpr int TI = decltype(ti_tag)::value;
            f32x4 acc[WB][Grid<C, TI>::XB];
            multiply<C, TI, GATED>(p, t, next, rs_x, rs_xs, ring, base, sbase, acc);
            if (C::NEXT) {   // on their way while this tile is stored
                tile_weights<GATED>(p, after, w_at, u_at);
                last = following(n0_last);
                rows = tile_rows<C>(p, after, fresh_lane(), wave);
                __builtin_amdgcn_sched_barrier(0);
            }
            // the stage that comes free last, at the places of this wavefront's own loads
            store_tile<C, TI, GATED, NT>(p, t, ring + (int)((uint32_t)(base + KT + C::NS - 1) % C::NS) * Ring<C>::STAGE + wave * 1024, acc);
        };
        const int blocks = (t.nrows + 31) >> 5;
        if constexpr (C::ROWS > 128) {
            if (blocks > 7) run(std::integral_constant<int, 8>{});
            else if (blocks > 6) run(std::integral_constant<int, 7>{});
            else if (blocks > 5) run(std::integral_constant<int, 6>{});
            else if (blocks > 4) run(std::integral_constant<int, 5>{});
        }
        if (blocks <= 4) {
            if (blocks > 3) run(std::integral_constant<int, 4>{});
            else if (blocks > 2) run(std::integral_constant<int, 3>{});
            else if (blocks > 1) run(std::integral_constant<int, 2>{});
            else run(std::integral_constant<int, 1>{});
        }
        if (!C::NEXT || !next.any) return;
        base += KT;
        sbase += p.groups;
        t = next;
        next = tile_loads<C, GATED>(p, after, n0_after, rows, w_at, u_at, fresh_lane(), wave);
        after = last;
        n0_after = n0_last;
    }
}

template <class C, bool NT>
void launch_tiles(const Fp4Product& p, const bool gated, const dim3 grid, hipStream_t st) {
    if (gated) hipLaunchKernelGGL((fp4_tile_kernel<C, true, NT>), grid, dim3(C::NW * 64), Ring<C>::BYTES + OWN<C>, st, p);
    else hipLaunchKernelGGL((fp4_tile_kernel<C, false, NT>), grid, dim3(C::NW * 64), Ring<C>::BYTES + OWN<C>, st, p);
}

template <class C, bool NT>
hipError_t set_lds() {
    const auto to = hipFuncAttributeMaxDynamicSharedMemorySize;
    if (const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&fp4_tile_kernel<C, true, NT>), to, Ring<C>::BYTES + OWN<C>)) return e;
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&fp4_tile_kernel<C, false, NT>), to, Ring<C>::BYTES + OWN<C>);
}

}  // namespace

hipError_t fp4_product_init() {
    for (const auto f : {set_lds<Long, false>, set_lds<Long, true>, set_lds<Short, false>, set_lds<Short, true>})
        if (const hipError_t e = f()) return e;
    return hipSuccess;
}

Fp4Layout fp4_layout(int64_t rows, int E) {
    Fp4Layout L;
    L.plan = 0;
    L.descs = 256;
    L.total = L.descs + (((size_t)(rows / Short::ROWS + E) * sizeof(TileDesc) + 255) & ~(size_t)255);
    return L;
}

int64_t fp4_tiles(int64_t rows, int E, int64_t N, bool gated) { return (rows / Short::ROWS + E) * ((N + (gated ? 127 : 255)) / (gated ? 128 : 256)); }

hipError_t launch_fp4_product(const Fp4Product& args, bool gated, hipStream_t st) {
    Fp4Product p = args;
    const int bn = gated ? 128 : WROWS;
    p.n_tiles = (p.N + bn - 1) / bn;
    // Which form, by the tiles that even groups would have (us, short and long; rows per group): 64 experts, K = 2048, gated 94 rows 54.8, 53.0, 141 64.8, 60.3, 281
    // 99.5, 97.9, 750 198, 176; K = 1408 94 26.0, 28.7, 112 36.0, 30.4, 281 57.9, 55.5, 750 125, 104; 160 experts, K = 1536 37 141.3, 141.6, 112 175.8, 175.5, 600
    // 616, 533; 8 experts, K = 4096, gated 25 86.6, 90.5, 100 105, 108, 250 183, 165, 750 406, 368.  Few tiles: a CU has one workgroup in either form, and a long
    // contraction is better off with the deeper ring (8 experts, K = 14336, 25 rows 92, 61, 100 98, 78), a short one with lower tiles (K = 512, gated 250 rows 8.8, 11.4, 750
    // 11.4, 13.5).
    // (64 bits: rows + E may pass 2^31.  A grid of the short form has fewer than 2^24 workgroups, above which its threads would pass 2^32: up to 100 rows
    // a group it is at most 456 m-tiles of 16384 columns' tiles.)
    const int64_t per = ((int64_t)p.rows + p.E - 1) / p.E, groups = std::min(p.E, p.rows);
    const int64_t long_tiles = groups * ((per + Long::ROWS - 1) / Long::ROWS) * p.n_tiles, short_tiles = groups * ((per + Short::ROWS - 1) / Short::ROWS) * p.n_tiles;
    const bool is_long = (per > 100 && long_tiles >= 256) || (short_tiles <= 256 && p.sub_tiles >= 32);
    // Outputs go past the L2s, where they would displace what tiles share (us, without and with: down of K = 1408, 64 experts, 16000 tokens, bf16 230, 195, fp32
    // 287, 249; K = 1536, 160 experts, 16000 593, 538; gate/up of K = 2048 339, 326, of K = 5120, 160 experts, 3000 tokens 306, 288), but for gated ones of a
    // long contraction and tall groups, which are few bytes for their time, in half lines (K = 4096, 8 experts, 16000 tokens 1828, 1852).
    const bool nt = !gated || p.sub_tiles <= 16 || per <= 128;
    p.group_m = 8;
    p.max_mtiles = p.rows / (is_long ? Long::ROWS : Short::ROWS) + p.E;
    const dim3 all((unsigned)(p.max_mtiles * p.n_tiles)), cus(std::min(all.x, 256u));
    // The list of m-tiles: a launch of its own is 3 to 5 us and a gap, finding tiles costs each workgroup a little under 1 us.  us, with the launch and without:
    // gate/up 8 experts, K = 512, 64 to 256 rows 10.7, 8.3; 64 experts, K = 2048, 94 rows (1400 workgroups) 56.4, 55.2; down K = 1408, 94 rows (1000) 28.5, 26.2,
    // 1500 rows (long) 204, 200; but 160 experts, K = 5120, 2 to 75 rows (2000 to 3800) 230, 233; K = 1536 (3300 to 6400) 133, 139.
    p.rounds = (int32_t)std::min<int64_t>((all.x + cus.x - 1) / cus.x + 3, ROUNDS + 1);
    p.inside = is_long ? p.rounds <= ROUNDS : all.x <= 3 * 512;
    if (!p.inside) {
        PlanArgs a = {};
        a.offsets = p.offsets;
        a.E = p.E;
        a.tm_up = is_long ? Long::ROWS : Short::ROWS;
        a.nt_up = p.n_tiles;
        a.tails_last_up = 1;
        a.small_tiles = 1;
        a.e_hi = p.E;
        a.plan = p.plan;
        a.descs_up = p.descs;
        hipLaunchKernelGGL(fp4_plan_kernel, dim3(1), dim3(256), 0, st, a);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    if (is_long && nt) launch_tiles<Long, true>(p, gated, cus, st);
    else if (is_long) launch_tiles<Long, false>(p, gated, cus, st);
    else if (nt) launch_tiles<Short, true>(p, gated, all, st);
    else launch_tiles<Short, false>(p, gated, all, st);
    return hipGetLastError();
}

}  // namespace moe
