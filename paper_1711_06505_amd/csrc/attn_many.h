// attn_many.h -- the attention kernels for samples of many rows in bf16, where
// the matrix products are the cost: 32 x 32 x 16 instructions, 32 rows (or
// keys) a wave, the streamed side in tiles of 64 through shared memory, read
// by all four waves of the block.
//
// As in attn_device.h a product's result is the next one's operand without
// leaving its lane: S^T = K Q^T has a query per lane (lane % 32) and, in its
// 16 registers, the keys 8 (r / 4) + 4 (lane / 32) + r % 4; registers 8 c .. 8 c + 7
// are the operand of the c-th contraction over 16 keys if V^T is read in that
// order, which is two transposed 8-byte reads (ds_read_b64_tr_b16: lane i of 16
// gets column i of four rows of 16 values).  Row reads and transposed reads
// use one layout: row-major, a row's 16-byte pieces permuted by the row so that
// eight consecutive rows fall on different banks either way.
//
// Weights and their gradients are rounded to bf16 once before the second
// product (relative 2^-8 at most, their sums are not rounded), but for dQ of
// heads up to 32 wide.  A pair as in attn_device.h everywhere takes the errors
// against 64 bits (by norm, normal inputs) from 2.2e-3 to 1.7e-3 for outputs and
// from 2.4e-3 to 1.7e-3 for gradients, where the rounding of the result alone is
// 1.7e-3, and the time of 8 samples of 1024..2048 queries and 2048..4096 keys, 16
// heads of 128, from 1.66 to 2.21 ms (forward 360 -> 489, dQ 517 -> 626, dK and dV
// 777 -> 1086 us).  dQ of narrow heads is off by more, 2.4e-3 at 32, 2.6e-3 at 16
// and 2.7e-3 at 8 wide: pairs there (1.7e-3, 1.8e-3, 1.9e-3; with heads of 32 the
// same samples' dQ takes 251 us instead of 195).
#pragma once

#include "attn_device.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

typedef __attribute__((address_space(3))) void lds_bytes;

// All of this wave's loads into shared memory and its reads of it done: before
// the barrier after which others read the one and overwrite the other.
__device__ __forceinline__ void staged()
{
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x7 << 4);             // vmcnt 0, lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
}

// Two waves share a SIMD, one of either block on the compute unit.  Treated
// alike they fall into step, both in their products and then both in their
// exponentials; with one of them (by its slot) always first, the other one
// fills in what it leaves free (364 and 512 us without, 353 and 495 with, forward
// and dQ of 8 samples of 1024..2048 queries and 2048..4096 keys, 16 heads of 128).
__device__ __forceinline__ void take_turns()
{
    if (__builtin_amdgcn_s_getreg((3 << 11) | 4) & 1) __builtin_amdgcn_s_setprio(1);
}

constexpr int kManyRows = 128;        // rows (keys) of a block, 32 a wave
constexpr int kManyShift = 7;
constexpr int kManyStep = 64;         // streamed entries of a tile

__device__ __forceinline__ f32x16 mma32(const Frag &a, const Frag &b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.b, b.b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 zero16()
{
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}
// registers 8 c .. 8 c + 7 of a result, rounded, as operand of the c-th contraction over 16
__device__ __forceinline__ Frag pack16(const f32x16 &x, int c)
{
    Frag f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.u[i] = pack_bf16(x[8 * c + 2 * i], x[8 * c + 2 * i + 1]);
    return f;
}
// what that rounding left, rounded
__device__ __forceinline__ Frag rest16(const f32x16 &x, int c, const Frag &h)
{
    Frag f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        f.u[i] = pack_bf16(x[8 * c + 2 * i] - __uint_as_float(h.u[i] << 16),
                           x[8 * c + 2 * i + 1] - __uint_as_float(h.u[i] & 0xffff0000u));
    return f;
}
// entry of register r in lane half hh
__device__ __forceinline__ int entry_of(int r, int hh) { return 8 * (r >> 2) + 4 * hh + (r & 3); }

// A tile of N rows of DH bf16 values in shared memory.
template <int DH, int N = kManyStep> struct Tile {
    static constexpr int kRows = N, kPieces = DH / 8, kRowBytes = DH * 2, kBytes = N * kRowBytes,
                         kPer = N * kPieces / kAttnThreads;              // pieces a thread stages
    // A row read takes one piece of 16 consecutive rows at a time, a transposed read four pieces of 4 rows:
    // with the row's low bits in the piece's high bits both fall on all 64 banks once.
    __device__ static __forceinline__ int swizzle(int row)
    {
        return DH == 128 ? (row & 3) << 2 | (row >> 2 & 3) : (DH == 64 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : row >> 2 & 3);
    }
    __device__ static __forceinline__ uint32_t at(int row, int piece)
    {
        return (uint32_t)(row * kRowBytes + ((piece ^ swizzle(row)) << 4));
    }
    // The permutation is an exclusive or on the piece's bits, so a lane keeps one offset for all its row reads and
    // one for its transposed reads; a piece further, or eight rows, is another bit.
    __device__ static __forceinline__ uint32_t row_base()
    {
        return at(ams_lane() & 31, ams_lane() >> 5);
    }
    __device__ static __forceinline__ uint32_t col_base()
    {
        const int lane = ams_lane(), i = lane & 15;
        return at(4 * (lane >> 5) + (i >> 2), 2 * ((lane >> 4) & 1) + ((i & 3) >> 1)) + (i & 1) * 8;
    }
    // rows `row0` + lane % 32 as operand of a contraction over the width, piece 2 c + lane / 32
    __device__ static __forceinline__ Frag row_frag(const char *t, uint32_t base, int row0, int c)
    {
        Frag f;
        *(uint4 *)f.u = *(const uint4 *)(t + (base ^ (uint32_t)(c << 5)) + row0 * kRowBytes);
        return f;
    }
    // operand of output columns 32 dt + lane % 32 for the contraction over rows row0 .. row0 + 15
    __device__ static __forceinline__ Frag col_frag(const char *t, uint32_t base, int row0, int dt)
    {
        const uint32_t at = base ^ (uint32_t)(dt << 6);
        Frag f;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(t + at + row0 * kRowBytes));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(t + (at ^ 32u) + (row0 + 8) * kRowBytes));
        *(s16x4 *)&f.u[0] = lo;
        *(s16x4 *)&f.u[2] = hi;
        return f;
    }
};

// Block of the work, so that neighbouring tiles (of one sample and key head,
// which read the same keys) run on one XCD and share its cache: hardware deals
// the blocks out to the 8 XCDs in turn.
__device__ __forceinline__ uint32_t xcd_block()
{
    const uint32_t b = blockIdx.x, per = gridDim.x / 8;
    return b < per * 8 ? (b % 8) * per + b / 8 : b;
}
__device__ __forceinline__ Work many_work(uint32_t b, const AttnArgs &a)
{
    const uint32_t tiles = (uint32_t)a.tiles;
    Work w;
    w.tile = b % tiles;
    b /= tiles;
    w.split = (int)(b % (uint32_t)a.nsplit);
    w.h = (int)(b / (uint32_t)a.nsplit);
    return w;
}

// A tile's way into shared memory: loads that put their 16 bytes there
// themselves, lane by lane, so the permutation is made on the source side.
// What lies behind D or behind the last row reads another piece of the tile:
// the first meets zeros of the other operand or results that nobody stores,
// the second weights of zero.  Rows that are not aligned to 16 bytes (PB < 16)
// come through registers, in loads of PB bytes.
template <int DH, int PB, int N = kManyStep> struct Dma {
    using TL = Tile<DH, N>;
    uint32_t off[TL::kPer];                            // of the row; with 16-byte pieces of the piece in it

    __device__ static __forceinline__ int slot(int i)
    {
        return (__builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE) * TL::kPer + i) * AMS_WAVE + ams_lane();
    }
    __device__ static __forceinline__ int row(int i) { return slot(i) / TL::kPieces; }
    __device__ static __forceinline__ int piece(int i) { return (slot(i) % TL::kPieces) ^ TL::swizzle(row(i)); }
    __device__ static __forceinline__ uint32_t col(int i, int D)
    {
        return PB == 16 && piece(i) * 8 < D ? piece(i) * 16 : 0;
    }
    __device__ __forceinline__ void rows(int last, uint32_t ld, int D)        // of a plain list
    {
#pragma unroll
        for (int i = 0; i < TL::kPer; ++i) off[i] = (uint32_t)min(row(i), last) * ld + col(i, D);
    }
    __device__ __forceinline__ void issue(const char *base, char *tile, int D) const
    {
        if constexpr (PB == 16) {
            char *t = tile + __builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE) * TL::kPer * 1024;
#pragma unroll
            for (int i = 0; i < TL::kPer; ++i)
                __builtin_amdgcn_global_load_lds(base + off[i], (lds_bytes *)(t + i * 1024), 16, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < TL::kPer; ++i) {
                uint4 v;
                Cols<uint16_t, 8, PB>(piece(i) * 8, D).load((uint32_t *)&v, base, off[i]);
                *(uint4 *)(tile + slot(i) * 16) = v;
            }
        }
    }
};

// A list's rows into a tile that stays, with zeros behind D; there after the next barrier.
template <int DH, int PB, int N>
__device__ __forceinline__ void stage_rows(const char *base, int last, uint32_t ld, int D, char *tile)
{
    Dma<DH, PB, N> dma;
    dma.rows(last, ld, D);
    dma.issue(base, tile, D);
    if (D == DH) return;
    staged();
    for (int i = threadIdx.x; i < N * DH / 2; i += kAttnThreads) {           // words
        const int r = i / (DH / 2), d = i % (DH / 2) * 2;
        uint32_t *w = (uint32_t *)(tile + Tile<DH, N>::at(r, d / 8)) + d % 8 / 2;
        if (d >= D) *w = 0;
        else if (d + 1 == D) *w &= 0xffffu;
    }
}

// The keys' side: 64 of K and V a step ahead.
template <int DH, int PB> struct KeyStage {
    Dma<DH, PB> k, v;
    uint32_t byte;                                     // the lane's key's mask byte

    __device__ __forceinline__ explicit KeyStage(const AttnArgs &a)
    {
        k.rows(kManyStep - 1, (uint32_t)(a.ld_k * 2), a.D);
        v.rows(kManyStep - 1, (uint32_t)(a.ld_v * 2), a.D);
    }
    __device__ __forceinline__ void issue(const AttnArgs &a, int h, int k0, int kb, int hi, char *kt, char *vt)
    {
        const int last = hi - 1 - kb;
        if (last < kManyStep - 1) {
            k.rows(last, (uint32_t)(a.ld_k * 2), a.D);
            v.rows(last, (uint32_t)(a.ld_v * 2), a.D);
        }
        byte = a.mask ? a.mask[k0 + kb + min(ams_lane(), last)] : 1;
        k.issue((const char *)a.k + ((int64_t)(k0 + kb) * a.ld_k + (int64_t)h * a.D) * 2, kt, a.D);
        v.issue((const char *)a.v + ((int64_t)(k0 + kb) * a.ld_v + (int64_t)h * a.D) * 2, vt, a.D);
    }
    // The tile of the keys from kb on is there: which of them take part.  Masked ones become zeros.
    __device__ __forceinline__ uint64_t arrive(const AttnArgs &a, int kb, int hi, char *kt, char *vt)
    {
        staged();
        const uint64_t kept = ams_ballot(byte != 0);
        if (a.mask && kept != ~0ull) {
            for (int i = threadIdx.x; i < kManyStep * Tile<DH>::kPieces; i += kAttnThreads) {
                if (kept >> (i / Tile<DH>::kPieces) & 1) continue;
                *(uint4 *)(kt + i * 16) = make_uint4(0, 0, 0, 0);
                *(uint4 *)(vt + i * 16) = make_uint4(0, 0, 0, 0);
            }
            __syncthreads();
        }
        return kept & ams_ballot(kb + ams_lane() < hi);
    }
};

// The same from 8-bit pages: codes a step ahead in registers, page numbers two;
// decoded on the way into shared memory, once for all four waves.  Tokens that
// take no part become zeros there.
template <int DH> struct PageStage {
    using TL = Tile<DH>;
    static constexpr int kUnits = kManyStep * DH / 16, kPer = (kUnits + kAttnThreads - 1) / kAttnThreads;
    uint4 k[kPer], v[kPer];
    float ks, vs, ks_next, vs_next;                    // of the lane's token
    int page;                                          // of the lane's token, a step ahead of the codes
    bool there, there_next;

    __device__ __forceinline__ explicit PageStage(const AttnArgs &) {}
    __device__ __forceinline__ void find(const AttnArgs &a, const int32_t *pages, int kb, int hi)
    {
        page = pages[min(kb + ams_lane(), hi - 1) >> a.page_shift];
    }
    __device__ __forceinline__ void issue(const AttnArgs &a, int h, int kb, int hi)
    {
        there_next = page >= 0 && page < a.n_pages;
        const int mine = there_next ? page : 0;
        const int64_t at = (int64_t)mine * a.Hk + h;
        ks_next = a.ks[at];
        vs_next = a.vs[at];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int u = min(i * kAttnThreads + (int)threadIdx.x, kUnits - 1), row = u / (DH / 16), piece = u % (DH / 16);
            const int tok = min(kb + row, hi - 1), p = __shfl(mine, min(row, hi - 1 - kb), AMS_WAVE);
            const int64_t first = ((((int64_t)p * a.Hk + h) << a.page_shift) + (tok & ((1 << a.page_shift) - 1))) * a.D +
                                  (piece * 16 < a.D ? piece * 16 : 0);
            k[i] = *(const uint4 *)(a.kc + first);
            v[i] = *(const uint4 *)(a.vc + first);
        }
    }
    __device__ __forceinline__ uint64_t arrive(int kb, int hi, char *kt, char *vt)
    {
        // a token without a page: zeros, whatever the scales that were read in its place
        there = there_next, ks = there ? ks_next : 1.f, vs = there ? vs_next : 0.f;
        const uint64_t live = ams_ballot(there && kb + ams_lane() < hi);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int u = i * kAttnThreads + threadIdx.x, row = u / (DH / 16), piece = u % (DH / 16);
            if (kUnits % kAttnThreads && u >= kUnits) break;
            if (!(live >> row & 1)) k[i] = v[i] = make_uint4(0, 0, 0, 0);
            uint32_t x[8];
            auto put = [&](const uint4 &c, char *tile) {
                decode4<uint16_t>(c.x, x), decode4<uint16_t>(c.y, x + 2), decode4<uint16_t>(c.z, x + 4), decode4<uint16_t>(c.w, x + 6);
                *(uint4 *)(tile + TL::at(row, 2 * piece)) = make_uint4(x[0], x[1], x[2], x[3]);
                *(uint4 *)(tile + TL::at(row, 2 * piece + 1)) = make_uint4(x[4], x[5], x[6], x[7]);
            };
            put(k[i], kt);
            put(v[i], vt);
        }
        staged();
        return live;
    }
    // scale of the 16 tokens from 16 g on (they share a page)
    __device__ __forceinline__ static float of(float x, int g)
    {
        return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), 16 * g));
    }
};

// The rows' side: N of Q and dO a step ahead, with their log-sum-exp and delta.
template <int DH, int PB, int N> struct RowStage {
    using DM = Dma<DH, PB, N>;
    DM q, d;
    float lse, delta;
    bool same = false;                                 // the offsets of a whole step hold for the next one

    __device__ __forceinline__ void issue(const AttnArgs &a, int h, int q0, int rb, int hi, char *qt, char *dt)
    {
        // the step's first query; a row lies at most N queries on
        const int qb = __builtin_amdgcn_readfirstlane(a.by_g.div(rb));
        const int64_t query = (int64_t)q0 + qb;
        const bool whole = rb + N <= hi;
        if (!same || !whole) {
#pragma unroll
            for (int i = 0; i < Tile<DH, N>::kPer; ++i) {
                const int r = min(rb + DM::row(i), hi - 1), n = a.by_g.div(r);
                const uint32_t col = (uint32_t)((r - n * a.G) * a.D * 2) + DM::col(i, a.D);
                q.off[i] = (uint32_t)(n - qb) * (uint32_t)(a.ld_q * 2) + col;
                d.off[i] = (uint32_t)(n - qb) * (uint32_t)(a.ld_dout * 2) + col;
            }
            same = whole && kKeyTile % a.G == 0;       // steps begin on whole queries
        }
        const int r = min(rb + (ams_lane() & (N - 1)), hi - 1), n = a.by_g.div(r);
        const int64_t at = ((int64_t)q0 + n) * a.H + h * a.G + (r - n * a.G);
        lse = a.lse[at];
        delta = a.delta[at];
        q.issue((const char *)a.q + (query * a.ld_q + (int64_t)h * a.G * a.D) * 2, qt, a.D);
        d.issue((const char *)a.dout + (query * a.ld_dout + (int64_t)h * a.G * a.D) * 2, dt, a.D);
    }
};

// The wave's 32 rows as operand, with zeros behind D.
template <int DH, int PB>
__device__ __forceinline__ void rows_frag(Frag *f, const void *x, int64_t ld, const Row &row, int D)
{
    const char *p = (const char *)x + (row.query * ld + (int64_t)row.head * D) * 2;
    const int hh = ams_lane() >> 5;
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) {
        const int d = 16 * c + 8 * hh;
        const Cols<uint16_t, 8, PB> cols(d, D);
        cols.load(f[c].u, p, 0);
        if (D < DH) cols.mask(f[c].u, d, D);
    }
}

// Four consecutive values of a result row.
template <int PB> __device__ __forceinline__ void store4(void *row, int d, int D, float a, float b, float c, float e)
{
    const float v[4] = {a, b, c, e};
    store_elems<uint16_t, 4, PB>((uint16_t *)row, d, D, v);
}

// ---------------------------------------------------------------- forward

// A factor of scores that is not zero, so that the -infinity of an entry that
// takes no part stays one under it.  The least float32 (2^-149) stands for
// zero: it moves no weight by more than 2^-21, whatever the product.
__device__ __forceinline__ float above_zero(float x) { return fmaxf(x, 1.4e-45f); }

template <int DH, int PB, bool PAGED> __global__ __launch_bounds__(kAttnThreads, 2) void attn_fwd_many_k(AttnArgs a)
{
    using TL = Tile<DH>;
    constexpr int NC = DH / 16, ND = DH / 32;
    // each buffer an array of its own, so that the compiler sees that a step's loads go elsewhere than its reads
    __shared__ __attribute__((aligned(16))) char s_k0[TL::kBytes], s_k1[TL::kBytes], s_v0[TL::kBytes], s_v1[TL::kBytes];
    const int lane = ams_lane(), hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE);
    const Work wk = many_work(xcd_block(), a);
    const int h = wk.h;
    const Span rows = span_of(a.q_off, a.B, a.n_q, a.G, kManyShift, wk.tile);
    const int64_t R = (int64_t)rows.count * a.G;
    if (rows.first < 0 || rows.first >= R) return;
    const int64_t r_mine = rows.first + wave * 32 + (lane & 31);
    const Row row = row_at(a, rows.begin, h, (int)(r_mine < R ? r_mine : R - 1));
    int k0 = 0, nk;
    const int32_t *pages = nullptr;
    if constexpr (PAGED) {
        nk = clamp_off(a.len[rows.i], (int64_t)a.max_pages << a.page_shift);
        pages = a.page_table + (int64_t)rows.i * a.max_pages;
    } else {
        k0 = clamp_off(a.k_off[rows.i], a.n_k);
        const int k1 = clamp_off(a.k_off[rows.i + 1], a.n_k);
        nk = k1 > k0 ? k1 - k0 : 0;
    }
    int lo, hi;
    split_range(nk, wk.split, a.nsplit, lo, hi);

    Frag qf[NC];
    rows_frag<DH, PB>(qf, a.q, a.ld_q, row, a.D);
    // a positive factor, so that the maximum can be taken before it: a negative scale goes onto Q's signs
    const float c = fabsf(a.scale) * kLog2e, c0 = above_zero(c);
    if (a.scale < 0.f) {
#pragma unroll
        for (int x = 0; x < NC; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) qf[x].u[i] ^= 0x80008000u;
    }
    f32x16 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) acc[d] = zero16();
    float mx = kNegInf, l = 0.f;
    take_turns();
    const uint32_t row_at_lane = TL::row_base(), col_at_lane = TL::col_base();
    typename std::conditional<PAGED, PageStage<DH>, KeyStage<DH, PB>>::type st(a);
    auto step = [&](int kb, char *kt, char *vt, char *kn, char *vn) {
        uint64_t live;
        float sk[4] = {c0, c0, c0, c0}, sv[4] = {1.f, 1.f, 1.f, 1.f};
        if constexpr (PAGED) {
            live = st.arrive(kb, hi, kt, vt);
#pragma unroll
            for (int g = 0; g < 4; ++g) sk[g] = above_zero(c * st.of(st.ks, g)), sv[g] = st.of(st.vs, g);
            if (kb + kManyStep < hi) {
                st.issue(a, h, kb + kManyStep, hi);
                if (kb + 2 * kManyStep < hi) st.find(a, pages, kb + 2 * kManyStep, hi);
            }
        } else {
            live = st.arrive(a, kb, hi, kt, vt);
            if (kb + kManyStep < hi) st.issue(a, h, k0, kb + kManyStep, hi, kn, vn);
        }
        f32x16 s[2] = {zero16(), zero16()};
#pragma unroll
        for (int x = 0; x < NC; ++x)
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = mma32(TL::row_frag(kt, row_at_lane, 32 * t, x), qf[x], s[t]);
        if (live != ~0ull) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(live >> (32 * t + entry_of(r, hh)) & 1)) s[t][r] = kNegInf;
        }
        // the running maximum may lag by 2^8: weights stay below 2^8, and the sums are rescaled that much less often
        float tm = kNegInf;                            // of each 16 keys, which have one positive factor
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float m = s[g >> 1][8 * (g & 1)];
#pragma unroll
            for (int r = 1; r < 8; ++r) m = fmaxf(m, s[g >> 1][8 * (g & 1) + r]);
            tm = fmaxf(tm, m * sk[g]);
        }
        tm = fmaxf(tm, __shfl_xor(tm, 32, AMS_WAVE));
        if (ams_ballot(tm > mx + 8.f)) {
            const float mn = fmaxf(mx, tm), alpha = __builtin_amdgcn_exp2f(mx - (mn == kNegInf ? 0.f : mn));
            mx = mn;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < ND; ++d) acc[d] *= alpha;
        }
        const float base = mx == kNegInf ? 0.f : mx;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[t][r] = __builtin_amdgcn_exp2f(s[t][r] * sk[2 * t + (r >> 3)] - base);
                l += s[t][r];
                if constexpr (PAGED) s[t][r] *= sv[2 * t + (r >> 3)];          // a power of two: exact
            }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const Frag p = pack16(s[t], x);
#pragma unroll
                for (int d = 0; d < ND; ++d) acc[d] = mma32(TL::col_frag(vt, col_at_lane, 32 * t + 16 * x, d), p, acc[d]);
            }
    };
    if (lo < hi) {
        if constexpr (PAGED) {
            st.find(a, pages, lo, hi);
            st.issue(a, h, lo, hi);
            if (lo + kManyStep < hi) st.find(a, pages, lo + kManyStep, hi);
        } else {
            st.issue(a, h, k0, lo, hi, s_k0, s_v0);
        }
    }
    for (int kb = lo; kb < hi; kb += 2 * kManyStep) {
        step(kb, s_k0, s_v0, s_k1, s_v1);
        if (kb + kManyStep < hi) step(kb + kManyStep, s_k1, s_v1, s_k0, s_v0);
    }
    l += __shfl_xor(l, 32, AMS_WAVE);
    if (c != c && l != 0.f) l = c;                     // a scale that is NaN, which above_zero took out
    if (r_mine >= R) return;
    const int64_t at = row.query * a.H + row.head;
    if (a.nsplit > 1) {
        const int64_t p = (int64_t)wk.split * a.n_q * a.H + at;
        if (hh == 0) {
            a.part_ml[2 * p] = mx;
            a.part_ml[2 * p + 1] = l;
        }
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (32 * d + entry_of(r, hh) < a.D) a.part_o[p * a.D + 32 * d + entry_of(r, hh)] = acc[d][r];
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    void *out = (uint16_t *)a.out + row.query * a.ld_out + (int64_t)row.head * a.D;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            store4<PB>(out, 32 * d + entry_of(r, hh), a.D, acc[d][r] * inv, acc[d][r + 1] * inv, acc[d][r + 2] * inv,
                   acc[d][r + 3] * inv);
    if (a.lse && hh == 0) a.lse[at] = l == 0.f ? kNegInf : (mx + __builtin_amdgcn_logf(l)) * kLn2;
}

// -------------------------------------------------------------- dQ, delta

template <int DH, int PB> __global__ __launch_bounds__(kAttnThreads, 2) void attn_dq_many_k(AttnArgs a)
{
    using TL = Tile<DH>;
    constexpr int NC = DH / 16, ND = DH / 32;
    // each buffer an array of its own, so that the compiler sees that a step's loads go elsewhere than its reads
    __shared__ __attribute__((aligned(16))) char s_k0[TL::kBytes], s_k1[TL::kBytes], s_v0[TL::kBytes], s_v1[TL::kBytes];
    const int lane = ams_lane(), hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE);
    const Work wk = many_work(xcd_block(), a);
    const int h = wk.h;
    const Span rows = span_of(a.q_off, a.B, a.n_q, a.G, kManyShift, wk.tile);
    const int64_t R = (int64_t)rows.count * a.G;
    if (rows.first < 0 || rows.first >= R) return;
    const int64_t r_mine = rows.first + wave * 32 + (lane & 31);
    const Row row = row_at(a, rows.begin, h, (int)(r_mine < R ? r_mine : R - 1));
    const int64_t at = row.query * a.H + row.head;
    const int k0 = clamp_off(a.k_off[rows.i], a.n_k), k1 = clamp_off(a.k_off[rows.i + 1], a.n_k);
    int lo, hi;
    split_range(k1 > k0 ? k1 - k0 : 0, wk.split, a.nsplit, lo, hi);

    Frag qf[NC], df[NC];
    rows_frag<DH, PB>(qf, a.q, a.ld_q, row, a.D);
    rows_frag<DH, PB>(df, a.dout, a.ld_dout, row, a.D);
    float delta = 0.f;
    {
        Frag of[NC];
        rows_frag<DH, PB>(of, a.o, a.ld_o, row, a.D);
#pragma unroll
        for (int x = 0; x < NC; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                delta += __uint_as_float(df[x].u[i] << 16) * __uint_as_float(of[x].u[i] << 16);
                delta += __uint_as_float(df[x].u[i] & 0xffff0000u) * __uint_as_float(of[x].u[i] & 0xffff0000u);
            }
        delta += __shfl_xor(delta, 32, AMS_WAVE);
    }
    const float lse = a.lse[at];
    const bool on = lse != kNegInf;                   // a row without keys: its upstream gradient goes nowhere
    delta = on ? delta : 0.f;
    if (wk.split == 0 && hh == 0 && r_mine < R) a.delta[at] = delta;
    const float c = a.scale * kLog2e, lse2 = on ? lse * kLog2e : 0.f;
    const uint64_t all_on = ams_ballot(on);
    f32x16 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) acc[d] = zero16();
    take_turns();
    const uint32_t row_at_lane = TL::row_base(), col_at_lane = TL::col_base();
    KeyStage<DH, PB> st(a);
    auto step = [&](int kb, char *kt, char *vt, char *kn, char *vn) {
        const uint64_t live = st.arrive(a, kb, hi, kt, vt);
        if (kb + kManyStep < hi) st.issue(a, h, k0, kb + kManyStep, hi, kn, vn);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x16 s = zero16(), dp = zero16();
#pragma unroll
            for (int x = 0; x < NC; ++x) {
                s = mma32(TL::row_frag(kt, row_at_lane, 32 * t, x), qf[x], s);
                dp = mma32(TL::row_frag(vt, row_at_lane, 32 * t, x), df[x], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(s[r] * c - lse2);
                s[r] = p * (dp[r] - delta);
            }
            if (live != ~0ull || all_on != ~0ull) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!on || !(live >> (32 * t + entry_of(r, hh)) & 1)) s[r] = 0.f;
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const Frag p = pack16(s, x);
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const Frag k = TL::col_frag(kt, col_at_lane, 32 * t + 16 * x, d);
                    acc[d] = mma32(k, p, acc[d]);
                    if constexpr (DH == 32) acc[d] = mma32(k, rest16(s, x, p), acc[d]);
                }
            }
        }
    };
    if (lo < hi) st.issue(a, h, k0, lo, hi, s_k0, s_v0);
    for (int kb = lo; kb < hi; kb += 2 * kManyStep) {
        step(kb, s_k0, s_v0, s_k1, s_v1);
        if (kb + kManyStep < hi) step(kb + kManyStep, s_k1, s_v1, s_k0, s_v0);
    }
#pragma unroll
    for (int d = 0; d < ND; ++d) acc[d] *= a.scale;
    if (r_mine >= R) return;
    if (a.nsplit > 1) {
        float *p = a.part_o + ((int64_t)wk.split * a.n_q * a.H + at) * a.D;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (32 * d + entry_of(r, hh) < a.D) p[32 * d + entry_of(r, hh)] = acc[d][r];
        return;
    }
    void *dq = (uint16_t *)a.dq + row.query * a.ld_dq + (int64_t)row.head * a.D;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            store4<PB>(dq, 32 * d + entry_of(r, hh), a.D, acc[d][r], acc[d][r + 1], acc[d][r + 2], acc[d][r + 3]);
}

// ----------------------------------------------------------------- dK, dV

// 128 keys a block, 32 a wave; rows in tiles with their log-sum-exp and delta.
// Both sums of a wave are 2 DH registers.  For two waves per SIMD at DH = 128
// the values stay in shared memory, read anew for each tile, and a tile is 32
// rows (8 samples of 1024..2048 queries and 2048..4096 keys, 16 heads: 745 us;
// one wave per SIMD with all in registers: 1125).
template <int DH, int PB> __global__ __launch_bounds__(kAttnThreads, 2) void attn_dkv_many_k(AttnArgs a)
{
    constexpr bool kShared = DH == 128;
    constexpr int N = kShared ? 32 : 64;
    using TL = Tile<DH, N>;
    using VT = Tile<DH, kManyRows>;
    constexpr int NC = DH / 16, ND = DH / 32;
    __shared__ __attribute__((aligned(16))) char s_q0[TL::kBytes], s_q1[TL::kBytes], s_d0[TL::kBytes], s_d1[TL::kBytes];
    __shared__ __attribute__((aligned(16))) char s_v[kShared ? VT::kBytes : 16];
    __shared__ __attribute__((aligned(16))) float s_lse[2][N], s_delta[2][N];
    const int lane = ams_lane(), hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE);
    const Work wk = many_work(xcd_block(), a);
    const int h = wk.h;
    const Span keys = span_of(a.k_off, a.B, a.n_k, 1, kManyShift, wk.tile);
    if (keys.first < 0 || keys.first >= keys.count) return;
    const int q0 = clamp_off(a.q_off[keys.i], a.n_q), q1 = clamp_off(a.q_off[keys.i + 1], a.n_q);
    int lo, hi;
    split_range((int)(q1 > q0 ? (int64_t)(q1 - q0) * a.G : 0), wk.split, a.nsplit, lo, hi);
    const int64_t mine = keys.first + wave * 32 + (lane & 31);
    const int64_t key = keys.begin + (mine < keys.count ? mine : keys.count - 1);
    const bool live_key = mine < keys.count && !(a.mask && a.mask[key] == 0);
    const uint64_t all_live = ams_ballot(live_key);

    Frag kf[NC], vf[kShared ? 1 : NC];
    rows_frag<DH, PB>(kf, a.k, a.ld_k, Row{key, h}, a.D);
    if constexpr (kShared) {
        const char *vp = (const char *)a.v + ((keys.begin + keys.first) * a.ld_v + (int64_t)h * a.D) * 2;
        const int64_t left = keys.count - 1 - keys.first;
        stage_rows<DH, PB, kManyRows>(vp, (int)(left < kManyRows - 1 ? left : kManyRows - 1), (uint32_t)(a.ld_v * 2), a.D, s_v);
    } else {
        rows_frag<DH, PB>(vf, a.v, a.ld_v, Row{key, h}, a.D);
    }
    const float c = a.scale * kLog2e;
    f32x16 ak[ND], av[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) ak[d] = av[d] = zero16();

    // rows a step ahead.  A row behind the last gets a log-sum-exp of +infinity, so that its weights are
    // zero; all rows of a sample have the same keys, so one without any has no live key either and is left out.
    if (lo < hi) {
        const Row w = row_at(a, q0, h, 0);
        const int bits = __builtin_amdgcn_readfirstlane((int)__float_as_uint(a.lse[w.query * a.H + w.head]));
        if (__uint_as_float((uint32_t)bits) == kNegInf) hi = lo;
    }
    RowStage<DH, PB, N> st;
    take_turns();
    const uint32_t row_at_lane = TL::row_base(), col_at_lane = TL::col_base();
    auto step = [&](int rb, char *qt, char *dt, char *qn, char *dn, int buf) {
        if (wave == 0 && lane < N) {
            s_lse[buf][lane] = rb + lane < hi ? st.lse * kLog2e : -kNegInf;
            s_delta[buf][lane] = st.delta;
        }
        staged();
        if (rb + N < hi) st.issue(a, h, q0, rb + N, hi, qn, dn);
#pragma unroll
        for (int t = 0; t < N / 32; ++t) {
            f32x16 s = zero16(), dp = zero16();
#pragma unroll
            for (int x = 0; x < NC; ++x) {
                s = mma32(TL::row_frag(qt, row_at_lane, 32 * t, x), kf[x], s);
                if constexpr (kShared) dp = mma32(TL::row_frag(dt, row_at_lane, 32 * t, x), VT::row_frag(s_v, row_at_lane, 32 * wave, x), dp);
                else dp = mma32(TL::row_frag(dt, row_at_lane, 32 * t, x), vf[x], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const float4 ls = *(const float4 *)&s_lse[buf][32 * t + entry_of(r, hh)];
                const float4 de = *(const float4 *)&s_delta[buf][32 * t + entry_of(r, hh)];
                const float lv[4] = {ls.x, ls.y, ls.z, ls.w}, dv[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[r + e] = __builtin_amdgcn_exp2f(s[r + e] * c - lv[e]);
                    dp[r + e] = s[r + e] * (dp[r + e] - dv[e]);
                }
            }
            if (all_live != ~0ull) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[r] = live_key ? s[r] : 0.f;
                    dp[r] = live_key ? dp[r] : 0.f;
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const Frag p = pack16(s, x), ds = pack16(dp, x);
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    av[d] = mma32(TL::col_frag(dt, col_at_lane, 32 * t + 16 * x, d), p, av[d]);
                    ak[d] = mma32(TL::col_frag(qt, col_at_lane, 32 * t + 16 * x, d), ds, ak[d]);
                }
            }
        }
    };
    if (lo < hi) st.issue(a, h, q0, lo, hi, s_q0, s_d0);
    for (int rb = lo; rb < hi; rb += 2 * N) {
        step(rb, s_q0, s_d0, s_q1, s_d1, 0);
        if (rb + N < hi) step(rb + N, s_q1, s_d1, s_q0, s_d0, 1);
    }
#pragma unroll
    for (int d = 0; d < ND; ++d) ak[d] *= a.scale;
    if (mine >= keys.count) return;
    if (a.nsplit > 1) {
        float *p = a.part_o + ((int64_t)wk.split * a.n_k * a.Hk + key * a.Hk + h) * 2 * a.D;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int x = 32 * d + entry_of(r, hh);
                if (x < a.D) p[x] = ak[d][r], p[a.D + x] = av[d][r];
            }
        return;
    }
    void *dk = (uint16_t *)a.dk + key * a.ld_dk + (int64_t)h * a.D, *dv = (uint16_t *)a.dv + key * a.ld_dv + (int64_t)h * a.D;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            store4<PB>(dk, 32 * d + entry_of(r, hh), a.D, ak[d][r], ak[d][r + 1], ak[d][r + 2], ak[d][r + 3]);
            store4<PB>(dv, 32 * d + entry_of(r, hh), a.D, av[d][r], av[d][r + 1], av[d][r + 2], av[d][r + 3]);
        }
}

// ------------------------------------------------------------------- host

// A block of attn_many.h has 128 rows of partial sums to write and join again: a split per compute unit, of 512
// entries at least.  Forward and backward, us at 256, 512 and 1024 entries: 64 queries over 1500 keys, 4 heads of 64,
// 37, 47 and 61; 2 samples of 1000 over 1500 89, 79 and 83; 16 of 100 queries, 8 heads of 64, over 600 73, 50 and 50.
// Up to two splits a unit: 8 samples of 128 queries over 12,000 keys, 4 heads of 128, 337 against 289.
inline int split_many(int64_t tiles, int64_t entries)
{
    if (tiles < 1) tiles = 1;
    const int64_t n = 256 / tiles < entries / 512 ? 256 / tiles : entries / 512;
    return n < 1 ? 1 : (int)n;
}

// Whether these kernels take the call, and how they cut it: from more than
// `from` rows of a sample on average.
inline bool cut_many(const ams_attn *at, int32_t B, int64_t n_q, int64_t keys, int from, Cut &c)
{
    const int64_t Hk = at->n_kv_heads, rows = n_q * (at->n_heads / Hk), samples = B < 1 ? 1 : B;
    if (rows <= from * samples) return false;
    int64_t busy = (rows + kManyRows - 1) >> kManyShift;
    if (busy < samples) busy = samples;
    c.nsplit = split_many(busy * Hk, keys);
    c.tiles = tiles_of(rows, kManyShift, B);
    c.blocks = c.tiles * Hk * c.nsplit;
    return true;
}

}  // namespace
