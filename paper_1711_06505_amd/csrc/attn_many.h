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
// product (relative 2^-9 at most, their sums are not rounded): a pair as in
// attn_device.h would add half of the second product's instructions here.
#pragma once

#include "attn_device.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

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
// entry of register r in lane half hh
__device__ __forceinline__ int entry_of(int r, int hh) { return 8 * (r >> 2) + 4 * hh + (r & 3); }

// A tile of 64 rows of DH bf16 values in shared memory.
template <int DH> struct Tile {
    static constexpr int kPieces = DH / 8, kRowBytes = DH * 2, kBytes = kManyStep * kRowBytes,
                         kPer = kManyStep * kPieces / kAttnThreads;      // pieces a thread stages
    __device__ static __forceinline__ int swizzle(int row) { return DH >= 64 ? row & 7 : (row >> 2) & 3; }
    __device__ static __forceinline__ uint32_t at(int row, int piece)
    {
        return (uint32_t)(row * kRowBytes + ((piece ^ swizzle(row)) << 4));
    }
    // rows `row0` + lane % 32 as operand of a contraction over the width, piece 2 c + lane / 32
    __device__ static __forceinline__ Frag row_frag(const char *t, int row0, int c)
    {
        const int lane = ams_lane(), row = row0 + (lane & 31);
        Frag f;
        *(uint4 *)f.u = *(const uint4 *)(t + at(row, 2 * c + (lane >> 5)));
        return f;
    }
    // operand of output columns 32 dt + lane % 32 for the contraction over rows row0 .. row0 + 15
    __device__ static __forceinline__ Frag col_frag(const char *t, int row0, int dt)
    {
        const int lane = ams_lane(), i = lane & 15;
        const int row = row0 + 4 * (lane >> 5) + (i >> 2), piece = 4 * dt + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
        Frag f;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(t + at(row, piece) + (i & 1) * 8));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(t + at(row + 8, piece) + (i & 1) * 8));
        *(s16x4 *)&f.u[0] = lo;
        *(s16x4 *)&f.u[2] = hi;
        return f;
    }
};

// Block of the work, so that neighbouring tiles (of one sample and key head,
// which read the same keys) run on one XCD and share its cache: hardware deals
// the blocks out to the 8 XCDs in turn.
__device__ __forceinline__ int64_t xcd_block()
{
    const int64_t b = blockIdx.x, per = gridDim.x / 8;
    return b < per * 8 ? (b % 8) * per + b / 8 : b;
}
__device__ __forceinline__ Work many_work(int64_t b, const AttnArgs &a)
{
    Work w;
    w.tile = b % a.tiles;
    b /= a.tiles;
    w.split = (int)(b % a.nsplit);
    w.h = (int)(b / a.nsplit);
    return w;
}

// The keys' side: 64 of K and V, a step ahead in registers, then in shared memory.
template <int DH> struct KeyStage {
    using TL = Tile<DH>;
    uint4 k[TL::kPer], v[TL::kPer];
    uint64_t live, next_live;

    __device__ __forceinline__ void load(const AttnArgs &a, int h, int k0, int kb, int hi)
    {
        const int lane = ams_lane(), last = hi - 1 - kb;
        bool on = kb + lane < hi;
        if (a.mask) on = on && a.mask[k0 + (on ? kb + lane : kb)] != 0;
        next_live = ams_ballot(on);
        const char *kp = (const char *)a.k + ((int64_t)(k0 + kb) * a.ld_k + (int64_t)h * a.D) * 2;
        const char *vp = (const char *)a.v + ((int64_t)(k0 + kb) * a.ld_v + (int64_t)h * a.D) * 2;
#pragma unroll
        for (int i = 0; i < TL::kPer; ++i) {
            const int at = i * kAttnThreads + threadIdx.x, row = at / TL::kPieces, piece = at % TL::kPieces;
            const uint32_t r = (uint32_t)min(row, last), col = piece * 8 < a.D ? piece * 16 : 0;
            k[i] = *(const uint4 *)(kp + (r * (uint32_t)(a.ld_k * 2) + col));
            v[i] = *(const uint4 *)(vp + (r * (uint32_t)(a.ld_v * 2) + col));
        }
    }
    // entries that take no part as zeros, whatever they hold
    __device__ __forceinline__ void store(const AttnArgs &a, char *kt, char *vt)
    {
        live = next_live;
        const bool whole = live == ~0ull && a.D == DH;
#pragma unroll
        for (int i = 0; i < TL::kPer; ++i) {
            const int at = i * kAttnThreads + threadIdx.x, row = at / TL::kPieces, piece = at % TL::kPieces;
            if (!whole && !((live >> row & 1) && piece * 8 < a.D)) k[i] = v[i] = make_uint4(0, 0, 0, 0);
            *(uint4 *)(kt + TL::at(row, piece)) = k[i];
            *(uint4 *)(vt + TL::at(row, piece)) = v[i];
        }
    }
};

// The wave's 32 rows as operand.
template <int DH>
__device__ __forceinline__ void rows_frag(Frag *f, const void *x, int64_t ld, const Row &row, int D)
{
    const char *p = (const char *)x + (row.query * ld + (int64_t)row.head * D) * 2;
    const int hh = ams_lane() >> 5;
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) {
        const int d = 16 * c + 8 * hh;
        *(uint4 *)f[c].u = *(const uint4 *)(p + (d < D ? d * 2 : 0));
        if (d >= D) *(uint4 *)f[c].u = make_uint4(0, 0, 0, 0);
    }
}

// Four consecutive values of a result row.
__device__ __forceinline__ void store4(void *row, int d, int D, float a, float b, float c, float e)
{
    if (d < D) *(uint2 *)((char *)row + d * 2) = make_uint2(pack_bf16(a, b), pack_bf16(c, e));
}

// ---------------------------------------------------------------- forward

template <int DH> __global__ __launch_bounds__(kAttnThreads, 2) void attn_fwd_many_k(AttnArgs a)
{
    using TL = Tile<DH>;
    constexpr int NC = DH / 16, ND = DH / 32;
    __shared__ __attribute__((aligned(16))) char s_k[2][TL::kBytes], s_v[2][TL::kBytes];
    const int lane = ams_lane(), hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE);
    const Work wk = many_work(xcd_block(), a);
    const int h = wk.h;
    const Span rows = span_of(a.q_off, a.B, a.n_q, a.G, kManyShift, wk.tile);
    const int64_t R = (int64_t)rows.count * a.G;
    if (rows.first < 0 || rows.first >= R) return;
    const int64_t r_mine = rows.first + wave * 32 + (lane & 31);
    const Row row = row_at(a, rows.begin, h, (int)(r_mine < R ? r_mine : R - 1));
    const int k0 = clamp_off(a.k_off[rows.i], a.n_k), k1 = clamp_off(a.k_off[rows.i + 1], a.n_k);
    int lo, hi;
    split_range(k1 > k0 ? k1 - k0 : 0, wk.split, a.nsplit, lo, hi);

    Frag qf[NC];
    rows_frag<DH>(qf, a.q, a.ld_q, row, a.D);
    // a positive factor, so that the maximum can be taken before it: a negative scale goes onto Q's signs
    const float c = fmaxf(fabsf(a.scale) * kLog2e, 1.2e-38f);
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
    KeyStage<DH> st;
    if (lo < hi) {
        st.load(a, h, k0, lo, hi);
        st.store(a, s_k[0], s_v[0]);
    }
    int buf = 0;
    for (int kb = lo; kb < hi; kb += kManyStep, buf ^= 1) {
        __syncthreads();                               // this tile is there, the other one free
        const bool more = kb + kManyStep < hi;
        const uint64_t live = st.live;
        if (more) st.load(a, h, k0, kb + kManyStep, hi);
        const char *kt = s_k[buf], *vt = s_v[buf];
        f32x16 s[2] = {zero16(), zero16()};
#pragma unroll
        for (int x = 0; x < NC; ++x)
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = mma32(TL::row_frag(kt, 32 * t, x), qf[x], s[t]);
        if (live != ~0ull) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(live >> (32 * t + entry_of(r, hh)) & 1)) s[t][r] = kNegInf;
        }
        // the running maximum may lag by 2^8: weights stay below 2^8, and the sums are rescaled that much less often
        float tm = kNegInf;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) tm = fmaxf(tm, s[t][r]);
        tm = fmaxf(tm, __shfl_xor(tm, 32, AMS_WAVE)) * c;
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
                s[t][r] = __builtin_amdgcn_exp2f(s[t][r] * c - base);
                l += s[t][r];
            }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const Frag p = pack16(s[t], x);
#pragma unroll
                for (int d = 0; d < ND; ++d) acc[d] = mma32(TL::col_frag(vt, 32 * t + 16 * x, d), p, acc[d]);
            }
        if (more) st.store(a, s_k[buf ^ 1], s_v[buf ^ 1]);
    }
    l += __shfl_xor(l, 32, AMS_WAVE);
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
            store4(out, 32 * d + entry_of(r, hh), a.D, acc[d][r] * inv, acc[d][r + 1] * inv, acc[d][r + 2] * inv,
                   acc[d][r + 3] * inv);
    if (a.lse && hh == 0) a.lse[at] = l == 0.f ? kNegInf : (mx + __builtin_amdgcn_logf(l)) * kLn2;
}

// -------------------------------------------------------------- dQ, delta

template <int DH> __global__ __launch_bounds__(kAttnThreads, 2) void attn_dq_many_k(AttnArgs a)
{
    using TL = Tile<DH>;
    constexpr int NC = DH / 16, ND = DH / 32;
    __shared__ __attribute__((aligned(16))) char s_k[2][TL::kBytes], s_v[2][TL::kBytes];
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
    rows_frag<DH>(qf, a.q, a.ld_q, row, a.D);
    rows_frag<DH>(df, a.dout, a.ld_dout, row, a.D);
    float delta = 0.f;
    {
        Frag of[NC];
        rows_frag<DH>(of, a.o, a.ld_o, row, a.D);
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
    KeyStage<DH> st;
    if (lo < hi) {
        st.load(a, h, k0, lo, hi);
        st.store(a, s_k[0], s_v[0]);
    }
    int buf = 0;
    for (int kb = lo; kb < hi; kb += kManyStep, buf ^= 1) {
        __syncthreads();
        const bool more = kb + kManyStep < hi;
        const uint64_t live = st.live;
        if (more) st.load(a, h, k0, kb + kManyStep, hi);
        const char *kt = s_k[buf], *vt = s_v[buf];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x16 s = zero16(), dp = zero16();
#pragma unroll
            for (int x = 0; x < NC; ++x) {
                s = mma32(TL::row_frag(kt, 32 * t, x), qf[x], s);
                dp = mma32(TL::row_frag(vt, 32 * t, x), df[x], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(s[r] * c - lse2);
                s[r] = p * (dp[r] - delta) * a.scale;
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
                for (int d = 0; d < ND; ++d) acc[d] = mma32(TL::col_frag(kt, 32 * t + 16 * x, d), p, acc[d]);
            }
        }
        if (more) st.store(a, s_k[buf ^ 1], s_v[buf ^ 1]);
    }
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
            store4(dq, 32 * d + entry_of(r, hh), a.D, acc[d][r], acc[d][r + 1], acc[d][r + 2], acc[d][r + 3]);
}

// ----------------------------------------------------------------- dK, dV

// 128 keys a block, 32 a wave in registers; rows in tiles of 64 with their
// log-sum-exp and delta.
template <int DH> __global__ __launch_bounds__(kAttnThreads) void attn_dkv_many_k(AttnArgs a)
{
    using TL = Tile<DH>;
    constexpr int NC = DH / 16, ND = DH / 32;
    __shared__ __attribute__((aligned(16))) char s_q[2][TL::kBytes], s_d[2][TL::kBytes];
    __shared__ __attribute__((aligned(16))) float s_lse[2][kManyStep], s_delta[2][kManyStep];
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

    Frag kf[NC], vf[NC];
    rows_frag<DH>(kf, a.k, a.ld_k, Row{key, h}, a.D);
    rows_frag<DH>(vf, a.v, a.ld_v, Row{key, h}, a.D);
    const float c = a.scale * kLog2e;
    f32x16 ak[ND], av[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) ak[d] = av[d] = zero16();

    // rows a step ahead; a row that is not there or has no keys comes as zeros with a log-sum-exp of
    // +infinity, so that its weights are zero
    uint4 qr[TL::kPer], dr[TL::kPer];
    float lr = 0.f, tr = 0.f;
    bool there[TL::kPer];
    auto load = [&](int rb) {
#pragma unroll
        for (int i = 0; i < TL::kPer; ++i) {
            const int p = i * kAttnThreads + threadIdx.x, r = rb + p / TL::kPieces, piece = p % TL::kPieces;
            const Row w = row_at(a, q0, h, r < hi ? r : hi - 1);
            const int64_t col = (int64_t)w.head * a.D + (piece * 8 < a.D ? piece * 8 : 0);
            qr[i] = *(const uint4 *)((const uint16_t *)a.q + w.query * a.ld_q + col);
            dr[i] = *(const uint4 *)((const uint16_t *)a.dout + w.query * a.ld_dout + col);
            there[i] = r < hi && piece * 8 < a.D && a.lse[w.query * a.H + w.head] != kNegInf;
        }
        if (threadIdx.x < kManyStep) {
            const int r = rb + threadIdx.x;
            const Row w = row_at(a, q0, h, r < hi ? r : hi - 1);
            const float x = a.lse[w.query * a.H + w.head];
            const bool ok = r < hi && x != kNegInf;
            lr = ok ? x * kLog2e : -kNegInf;
            tr = ok ? a.delta[w.query * a.H + w.head] : 0.f;
        }
    };
    auto store = [&](int b) {
#pragma unroll
        for (int i = 0; i < TL::kPer; ++i) {
            const int p = i * kAttnThreads + threadIdx.x, r = p / TL::kPieces, piece = p % TL::kPieces;
            if (!there[i]) qr[i] = dr[i] = make_uint4(0, 0, 0, 0);
            *(uint4 *)(s_q[b] + TL::at(r, piece)) = qr[i];
            *(uint4 *)(s_d[b] + TL::at(r, piece)) = dr[i];
        }
        if (threadIdx.x < kManyStep) {
            s_lse[b][threadIdx.x] = lr;
            s_delta[b][threadIdx.x] = tr;
        }
    };
    if (lo < hi) {
        load(lo);
        store(0);
    }
    int buf = 0;
    for (int rb = lo; rb < hi; rb += kManyStep, buf ^= 1) {
        __syncthreads();
        const bool more = rb + kManyStep < hi;
        if (more) load(rb + kManyStep);
        const char *qt = s_q[buf], *dt = s_d[buf];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x16 s = zero16(), dp = zero16();
#pragma unroll
            for (int x = 0; x < NC; ++x) {
                s = mma32(TL::row_frag(qt, 32 * t, x), kf[x], s);
                dp = mma32(TL::row_frag(dt, 32 * t, x), vf[x], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const float4 ls = *(const float4 *)&s_lse[buf][32 * t + entry_of(r, hh)];
                const float4 de = *(const float4 *)&s_delta[buf][32 * t + entry_of(r, hh)];
                const float lv[4] = {ls.x, ls.y, ls.z, ls.w}, dv[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[r + e] = __builtin_amdgcn_exp2f(s[r + e] * c - lv[e]);
                    dp[r + e] = s[r + e] * (dp[r + e] - dv[e]) * a.scale;
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
                    av[d] = mma32(TL::col_frag(dt, 32 * t + 16 * x, d), p, av[d]);
                    ak[d] = mma32(TL::col_frag(qt, 32 * t + 16 * x, d), ds, ak[d]);
                }
            }
        }
        if (more) store(buf ^ 1);
    }
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
            store4(dk, 32 * d + entry_of(r, hh), a.D, ak[d][r], ak[d][r + 1], ak[d][r + 2], ak[d][r + 3]);
            store4(dv, 32 * d + entry_of(r, hh), a.D, av[d][r], av[d][r + 1], av[d][r + 2], av[d][r + 3]);
        }
}

}  // namespace
