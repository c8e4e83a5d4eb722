// attn.hip -- multi-head attention of each sample's queries to that sample's
// keys, two lists of different lengths (the tiles are attn_device.h's).
//   ams_xattn_fwd  P = softmax(scale Q K^T) over the sample's live keys, O = P V
//   ams_xattn_bwd  with delta = rowsum(dO o O), in bf16 over few keys rowsum(P o dO V^T),
//                  and dS = scale P o (dO V^T - delta):
//                  dQ = dS K, dK = dS^T Q, dV = P^T dO, the last two summed over
//                  the query heads of a key head.
// The backward forms P again from the forward's log-sum-exp, in two kernels
// with one owner per result and no atomics: dQ's blocks own row tiles and
// stream keys as the forward does; dK's and dV's own keys, 16 a wave, and
// stream the rows (all heads of the group), so both their contractions have
// the operand layouts of the forward with rows and keys exchanged.  Where a
// sample's rows fit one tile (a few ads against a long list: bound by reading
// the keys and writing their gradients) a third kernel does all in one pass.
// bf16 samples of many rows, bound by the products, have attn_many.h's kernels.
#include <initializer_list>

#include "attn_device.h"
#include "attn_many.h"

namespace {

// delta = <dO, O> of the lane's row (pieces of it in each lane group).
template <class T, int NF> __device__ __forceinline__ float row_delta(const Frag *df, const Frag *of)
{
    float d = 0.f;
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                d += df[f].f[i] * of[f].f[i];
            } else {
                d += __uint_as_float(df[f].u[i] << 16) * __uint_as_float(of[f].u[i] << 16);
                d += __uint_as_float(df[f].u[i] & 0xffff0000u) * __uint_as_float(of[f].u[i] & 0xffff0000u);
            }
        }
    return sum_groups(d);
}

// Whether a list of n keys is step_delta's.
template <class T> __device__ __forceinline__ bool few_keys(int n) { return sizeof(T) == 2 && n <= 16; }

// delta of the lane's rows over a list of n <= 16 keys, as sum_j p_j <dO, V_j>.  The
// output that the forward stored is rounded to bf16, which shows where few keys
// make it up: dQ and dK are off by 2.8e-3 against 64 bits (by norm, normal inputs)
// at 2 to 4 keys, 2.0e-3 at 10 and 1.8e-3 at 20 with <dO, O>, by 1.7e-3 with the sum.
template <class T, int DH, int PB, int RT>
__device__ __forceinline__ void step_delta(const AttnArgs &a, const RowCols<T, DH, PB> &rc,
                                           const Frag (*qf)[DH / (4 * Num<T>::EP)],
                                           const Frag (*df)[DH / (4 * Num<T>::EP)], int k0, int n, int h, float c,
                                           const float *lse2, float *delta)
{
    constexpr int NF = DH / (4 * Num<T>::EP), ES = (int)sizeof(T);
    const int lane = ams_lane(), m = lane & 15, g = lane >> 4;
    const uint32_t live = live_bits(k0, k0 + n, a.mask);
    const int64_t key = k0 + min(m, n - 1), col = (int64_t)h * a.D;
    Frag kf[NF], vf[NF];
    rc.load(kf, (const char *)a.k + (key * a.ld_k + col) * ES, 0);
    rc.load(vf, (const char *)a.v + (key * a.ld_v + col) * ES, 0);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f}, dp = s;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            s = mma<T>(kf[f], qf[rt][f], s);
            dp = mma<T>(vf[f], df[rt][f], dp);
        }
        float d = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float x = __builtin_amdgcn_exp2f(s[r] * c - lse2[rt]) * dp[r];
            d += (live >> (4 * g + r) & 1) ? x : 0.f;
        }
        delta[rt] = sum_groups(d);
    }
}

// -------------------------------------------------------------- dQ, delta

// Tiles, waves and splits as the forward's.
template <class T, int DH, int PB, int RT, int WK>
__device__ __forceinline__ void dq_tile(const AttnArgs &a, int64_t block,
                                        float (*s_o)[WK > 1 ? kRowTile * RT : 1][DH + 4])
{
    constexpr int NF = DH / (4 * Num<T>::EP), VD = DH / 16, ES = (int)sizeof(T);
    constexpr int kRows = kRowTile * RT, kTileShift = RT == 2 ? 5 : 4;
    const int lane = ams_lane(), m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE);
    const Work wk = work_of(WK == 1 ? block * kAttnWaves + wave : block, a);
    const int h = wk.h;
    if (wk.tile >= a.tiles) return;
    const Span rows = span_of(a.q_off, a.B, a.n_q, a.G, kTileShift, wk.tile);
    const int64_t R = (int64_t)rows.count * a.G;
    if (rows.first < 0 || rows.first >= R || R <= a.few_rows) return;
    const int k0 = clamp_off(a.k_off[rows.i], a.n_k), k1 = clamp_off(a.k_off[rows.i + 1], a.n_k);
    int lo, hi;
    split_range(k1 > k0 ? k1 - k0 : 0, wk.split, a.nsplit, lo, hi);
    const bool first = wk.split == 0 && (WK == 1 || wave == 0);
    const bool summed = few_keys<T>(k1 - k0);         // all of such a list's keys are its first wave's

    const RowCols<T, DH, PB> rc(g, a.D);
    Frag qf[RT][NF], df[RT][NF];
    Row row[RT];
    float lse2[RT], delta[RT];
    bool on[RT];                                      // a row without keys: its upstream gradient goes nowhere
    const float c = a.scale * kLog2e;
    f32x4 acc[RT][VD];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int64_t r = rows.first + 16 * t + m;
        row[t] = row_at(a, rows.begin, h, (int)(r < R ? r : R - 1));
        const int64_t col = (int64_t)row[t].head * a.D;
        Frag of[NF];
        rc.load(qf[t], (const char *)a.q + (row[t].query * a.ld_q + col) * ES, 0);
        rc.load(df[t], (const char *)a.dout + (row[t].query * a.ld_dout + col) * ES, 0);
        if (!summed) rc.load(of, (const char *)a.o + (row[t].query * a.ld_o + col) * ES, 0);
        rc.clean(qf[t]);
        rc.clean(df[t]);
        if (!summed) rc.clean(of);
        const int64_t at = row[t].query * a.H + row[t].head;
        const float lse = a.lse[at];
        on[t] = lse != kNegInf;
        lse2[t] = on[t] ? lse * kLog2e : 0.f;
        delta[t] = 0.f;
        if (!summed) {
            delta[t] = row_delta<T, NF>(df[t], of);
            delta[t] = on[t] ? delta[t] : 0.f;
            if (first && g == 0 && r < R) a.delta[at] = delta[t];
        }
#pragma unroll
        for (int i = 0; i < VD; ++i) acc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if constexpr (sizeof(T) == 2) {
        if (summed && first) {
            if (lo < hi) step_delta<T, DH, PB, RT>(a, rc, qf, df, k0, hi, h, c, lse2, delta);
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const int64_t r = rows.first + 16 * t + m;
                const Row w = row_at(a, rows.begin, h, (int)(r < R ? r : R - 1));
                delta[t] = on[t] ? delta[t] : 0.f;
                if (g == 0 && r < R) a.delta[w.query * a.H + w.head] = delta[t];
            }
        }
    }
    const uint32_t ldk = (uint32_t)(a.ld_k * ES), ldv = (uint32_t)(a.ld_v * ES);
    uint32_t krow[2] = {m * ldk, (16 + m) * ldk}, vrow[2] = {m * ldv, (16 + m) * ldv}, srow[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) srow[j] = (uint32_t)stream_of(j, g) * ldk;
    const Cols<T, VD, PB> scol(m * VD, a.D);

    for (int kb = lo + (WK == 1 ? 0 : wave * kKeyTile); kb < hi; kb += WK * kKeyTile) {
        Frag kf[2][NF], vf[2][NF];
        Slice<T, DH> kk;
        const uint32_t live = live_bits(k0 + kb, k0 + hi, a.mask);
        if (kb + kKeyTile > hi) {
            const int last = hi - 1 - kb;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                krow[t] = (uint32_t)min(16 * t + m, last) * ldk;
                vrow[t] = (uint32_t)min(16 * t + m, last) * ldv;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) srow[j] = (uint32_t)min(stream_of(j, g), last) * ldk;
        }
        const char *kp = (const char *)a.k + ((int64_t)(k0 + kb) * a.ld_k + (int64_t)h * a.D) * ES;
        const char *vp = (const char *)a.v + ((int64_t)(k0 + kb) * a.ld_v + (int64_t)h * a.D) * ES;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            rc.load(kf[t], kp, krow[t]);
            rc.load(vf[t], vp, vrow[t]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) scol.load(kk.w[j], kp, srow[j]);
        if (live != 0xffffffffu) kk.keep(live, g);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float ds[8];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f}, dp = s;
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    s = mma<T>(kf[t][f], qf[rt][f], s);
                    dp = mma<T>(vf[t][f], df[rt][f], dp);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float p = __builtin_amdgcn_exp2f(s[r] * c - lse2[rt]);
                    ds[4 * t + r] = on[rt] ? p * (dp[r] - delta[rt]) * a.scale : 0.f;
                }
            }
            if (live != 0xffffffffu) {
#pragma unroll
                for (int j = 0; j < 8; ++j) ds[j] = (live >> (4 * g + stream_of(j, 0)) & 1) ? ds[j] : 0.f;
            }
            mma_slice<T, DH>(acc[rt], kk, Stream<T>(ds));
        }
    }
    if constexpr (WK == 1) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            if (rows.first + 16 * t + m >= R) continue;
            float o[4 * VD];
            acc_in_order<VD>(acc[t], 1.f, o);
            store_elems<T, 4 * VD, PB>((T *)a.dq + row[t].query * a.ld_dq + (int64_t)row[t].head * a.D, 4 * g * VD,
                                       a.D, o);
        }
        return;
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        float o[4 * VD];
        acc_in_order<VD>(acc[t], 1.f, o);
#pragma unroll
        for (int i = 0; i < 4 * VD; ++i) s_o[wave % WK][(16 * t + m) % (WK > 1 ? kRows : 1)][4 * g * VD + i] = o[i];
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int r = 16 * t + threadIdx.x / 16, d = (threadIdx.x % 16) * VD, rr = r % (WK > 1 ? kRows : 1);
        const int64_t ro = rows.first + r;
        if (ro >= R) return;
        float y[VD];
#pragma unroll
        for (int e = 0; e < VD; ++e)
            y[e] = (s_o[0][rr][d + e] + s_o[1 % WK][rr][d + e]) + (s_o[2 % WK][rr][d + e] + s_o[3 % WK][rr][d + e]);
        const Row ow = row_at(a, rows.begin, h, (int)ro);
        if (a.nsplit > 1) {
            float *p = a.part_o + ((int64_t)wk.split * a.n_q * a.H + ow.query * a.H + ow.head) * a.D;
#pragma unroll
            for (int e = 0; e < VD; ++e)
                if (d + e < a.D) p[d + e] = y[e];
            continue;
        }
        store_elems<T, VD, PB>((T *)a.dq + ow.query * a.ld_dq + (int64_t)ow.head * a.D, d, a.D, y);
    }
}

// Where attn_bwd_few_k has the small samples, the grid is a fixed number of
// blocks that first look whether there is any other (a.any_many).
template <class T, int DH, int PB, int RT, int WK>
__global__ __launch_bounds__(kAttnThreads, (waves_per_simd<T, DH, 2 * RT>())) void attn_dq_k(AttnArgs a)
{
    __shared__ float s_o[WK > 1 ? WK : 1][WK > 1 ? kRowTile * RT : 1][DH + 4];
    if (a.few_rows >= 0 && *a.any_many == 0) return;
    for (int64_t b = blockIdx.x; b < a.blocks; b += gridDim.x) {
        dq_tile<T, DH, PB, RT, WK>(a, b, s_o);
        __syncthreads();                               // s_o is free again
    }
}

// ----------------------------------------------------------------- dK, dV

// One wave per (16 keys of a sample, key head, split of the rows), four
// neighbouring key tiles to a block (they read the same rows).
template <class T, int DH, int PB> __device__ __forceinline__ void dkv_tile(const AttnArgs &a, int64_t block)
{
    constexpr int NF = DH / (4 * Num<T>::EP), VD = DH / 16, ES = (int)sizeof(T);
    const int lane = ams_lane(), m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE);
    const Work wk = work_of(block, a);
    const int h = wk.h;
    const Span keys = span_of(a.k_off, a.B, a.n_k, 1, 6, wk.tile);
    const int64_t first = keys.first + wave * 16;
    if (keys.first < 0 || first >= keys.count) return;
    const int q0 = clamp_off(a.q_off[keys.i], a.n_q), q1 = clamp_off(a.q_off[keys.i + 1], a.n_q);
    const int64_t R = q1 > q0 ? (int64_t)(q1 - q0) * a.G : 0;
    if (R <= a.few_rows) return;
    int lo, hi;
    split_range((int)R, wk.split, a.nsplit, lo, hi);

    const bool mine = first + m < keys.count;
    const int64_t key = keys.begin + (mine ? first + m : keys.count - 1);
    const bool live_key = mine && !(a.mask && a.mask[key] == 0);
    const RowCols<T, DH, PB> rc(g, a.D);
    const Cols<T, VD, PB> scol(m * VD, a.D);
    Frag kf[NF], vf[NF];
    rc.load(kf, (const char *)a.k + (key * a.ld_k + (int64_t)h * a.D) * ES, 0);
    rc.load(vf, (const char *)a.v + (key * a.ld_v + (int64_t)h * a.D) * ES, 0);
    rc.clean(kf);
    rc.clean(vf);
    const float c = a.scale * kLog2e;
    f32x4 ak[VD], av[VD];
#pragma unroll
    for (int t = 0; t < VD; ++t) ak[t] = av[t] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int rb = lo; rb < hi; rb += kKeyTile) {
        // the step's first query is the same in all lanes; a row lies at most 32 queries on
        const int qb = __builtin_amdgcn_readfirstlane(a.by_g.div(rb));
        const int64_t query = (int64_t)q0 + qb;
        const char *qp = (const char *)a.q + (query * a.ld_q + (int64_t)h * a.G * a.D) * ES;
        const char *dp_ = (const char *)a.dout + (query * a.ld_dout + (int64_t)h * a.G * a.D) * ES;
        const float *lp = a.lse + query * a.H + h * a.G, *tp = a.delta + query * a.H + h * a.G;
        Slice<T, DH> qs, os;
        Frag qf[2][NF], df[2][NF];
        float lse2[8], delta[8];
        bool live[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = rb + stream_of(j, g), rr = r < hi ? r : hi - 1, qq = a.by_g.div(rr), hh = rr - qq * a.G;
            const uint32_t dq = (uint32_t)(qq - qb), col = (uint32_t)(hh * a.D * ES);
            const float l = lp[dq * a.H + hh];
            live[j] = r < hi && l != kNegInf;
            lse2[j] = l * kLog2e;
            delta[j] = tp[dq * a.H + hh];
            scol.load(qs.w[j], qp, dq * (uint32_t)(a.ld_q * ES) + col);
            scol.load(os.w[j], dp_, dq * (uint32_t)(a.ld_dout * ES) + col);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int r = rb + 16 * t + m, rr = r < hi ? r : hi - 1, qq = a.by_g.div(rr), hh = rr - qq * a.G;
            const uint32_t dq = (uint32_t)(qq - qb), col = (uint32_t)(hh * a.D * ES);
            rc.load(qf[t], qp, dq * (uint32_t)(a.ld_q * ES) + col);
            rc.load(df[t], dp_, dq * (uint32_t)(a.ld_dout * ES) + col);
        }
        float p[8], ds[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f}, dp = s;
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                s = mma<T>(qf[t][f], kf[f], s);
                dp = mma<T>(df[t][f], vf[f], dp);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = 4 * t + e;
                const bool on = live[j] && live_key;
                p[j] = on ? __builtin_amdgcn_exp2f(s[e] * c - lse2[j]) : 0.f;
                ds[j] = on ? p[j] * (dp[e] - delta[j]) * a.scale : 0.f;
            }
        }
        bool all = true;
#pragma unroll
        for (int j = 0; j < 8; ++j) all = all && live[j];
        if (ams_ballot(!all)) {                        // rows behind the last, or without keys: whatever they hold
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (!live[j]) {
                    qs.zero(j);
                    os.zero(j);
                }
        }
        mma_slice<T, DH>(av, os, Stream<T>(p));
        mma_slice<T, DH>(ak, qs, Stream<T>(ds));
    }
    if (!mine) return;
    float o[4 * VD];
    if (a.nsplit > 1) {
        float *p = a.part_o + ((int64_t)wk.split * a.n_k * a.Hk + key * a.Hk + h) * 2 * a.D;
        acc_in_order<VD>(ak, 1.f, o);
#pragma unroll
        for (int i = 0; i < 4 * VD; ++i)
            if (4 * g * VD + i < a.D) p[4 * g * VD + i] = o[i];
        acc_in_order<VD>(av, 1.f, o);
#pragma unroll
        for (int i = 0; i < 4 * VD; ++i)
            if (4 * g * VD + i < a.D) p[a.D + 4 * g * VD + i] = o[i];
        return;
    }
    acc_in_order<VD>(ak, 1.f, o);
    store_elems<T, 4 * VD, PB>((T *)a.dk + key * a.ld_dk + (int64_t)h * a.D, 4 * g * VD, a.D, o);
    acc_in_order<VD>(av, 1.f, o);
    store_elems<T, 4 * VD, PB>((T *)a.dv + key * a.ld_dv + (int64_t)h * a.D, 4 * g * VD, a.D, o);
}

template <class T, int DH, int PB>
__global__ __launch_bounds__(kAttnThreads) void attn_dkv_k(AttnArgs a)
{
    if (a.few_rows >= 0 && *a.any_many == 0) return;
    for (int64_t b = blockIdx.x; b < a.blocks; b += gridDim.x) dkv_tile<T, DH, PB>(a, b);
}

// ------------------------------------------- dQ, dK, dV of few rows at once

// A sample whose rows fit one tile of 16 RT (a.few_rows; the others are left to
// the two kernels above): one wave per (sample, key head, split of the keys)
// keeps the rows in registers and reads each key once.  A key's scores are
// formed twice from the same operands, once with a row per lane (for dQ, which
// contracts over keys) and once with a key per lane (for dK and dV, which
// contract over rows); a key tile's dK and dV are complete at once.  One more
// block looks whether a sample has more rows than that.
template <class T, int DH, int PB, int RT>
__global__ __launch_bounds__(kAttnThreads, (DH == 128 ? 1 : waves_per_simd<T, DH, RT>())) void attn_bwd_few_k(AttnArgs a)
{
    if (blockIdx.x == gridDim.x - 1) {
        bool found = false;
#pragma unroll 16
        for (int s = threadIdx.x; s < a.B; s += kAttnThreads)
            found |= (int64_t)(clamp_off(a.q_off[s + 1], a.n_q) - clamp_off(a.q_off[s], a.n_q)) * a.G > a.few_rows;
        const int any = __syncthreads_or(found);
        if (threadIdx.x == 0) *a.any_many = any;
        return;
    }
    constexpr int NF = DH / (4 * Num<T>::EP), VD = DH / 16, ES = (int)sizeof(T);
    const int lane = ams_lane(), m = lane & 15, g = lane >> 4;
    const Work wk = work_of((int64_t)blockIdx.x * kAttnWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE), a);
    const int h = wk.h;
    if (wk.tile >= a.B) return;
    const int i = (int)wk.tile;
    const int q0 = clamp_off(a.q_off[i], a.n_q), q1 = clamp_off(a.q_off[i + 1], a.n_q);
    const int k0 = clamp_off(a.k_off[i], a.n_k), k1 = clamp_off(a.k_off[i + 1], a.n_k);
    const int64_t R64 = q1 > q0 ? (int64_t)(q1 - q0) * a.G : 0;
    if (R64 > a.few_rows) return;
    const int R = (int)R64;
    int lo, hi;
    split_range(k1 > k0 ? k1 - k0 : 0, wk.split, a.nsplit, lo, hi);
    const bool summed = few_keys<T>(k1 - k0);
    T *dkp = (T *)a.dk + (int64_t)h * a.D, *dvp = (T *)a.dv + (int64_t)h * a.D;
    if (R == 0) {                                     // keys that nothing attends to
        float z[4 * VD];
#pragma unroll
        for (int e = 0; e < 4 * VD; ++e) z[e] = 0.f;
        for (int key = k0 + lo + m; key < k0 + hi; key += 16) {
            store_elems<T, 4 * VD, PB>(dkp + (int64_t)key * a.ld_dk, 4 * g * VD, a.D, z);
            store_elems<T, 4 * VD, PB>(dvp + (int64_t)key * a.ld_dv, 4 * g * VD, a.D, z);
        }
        return;
    }

    const RowCols<T, DH, PB> rc(g, a.D);
    const Cols<T, VD, PB> scol(m * VD, a.D);
    Frag qf[RT][NF], df[RT][NF];
    Slice<T, DH> qs, os;                              // the rows again, as operands of a contraction over them
    float lse2[RT], delta[RT], lse2s[8], deltas[8];
    uint32_t on = 0;                                  // rows that attend to something: bits in stream_of's order
    f32x4 acc[RT][VD];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int r = 16 * t + m;
        const Row row = row_at(a, q0, h, r < R ? r : R - 1);
        const int64_t col = (int64_t)row.head * a.D;
        Frag of[NF];
        rc.load(qf[t], (const char *)a.q + (row.query * a.ld_q + col) * ES, 0);
        rc.load(df[t], (const char *)a.dout + (row.query * a.ld_dout + col) * ES, 0);
        if (!summed) rc.load(of, (const char *)a.o + (row.query * a.ld_o + col) * ES, 0);
        rc.clean(qf[t]);
        rc.clean(df[t]);
        if (!summed) rc.clean(of);
        const float lse = a.lse[row.query * a.H + row.head];
        const bool there = r < R && lse != kNegInf;
        on |= ((uint32_t)ams_ballot(there) & 0xffffu) << (16 * t);
        lse2[t] = there ? lse * kLog2e : 0.f;
        delta[t] = 0.f;
        if (!summed) {
            delta[t] = row_delta<T, NF>(df[t], of);
            delta[t] = there ? delta[t] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < VD; ++e) acc[t][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if constexpr (sizeof(T) == 2) {
        if (summed && lo < hi) {
            step_delta<T, DH, PB, RT>(a, rc, qf, df, k0, hi, h, a.scale * kLog2e, lse2, delta);
#pragma unroll
            for (int t = 0; t < RT; ++t) delta[t] = on >> (16 * t + m) & 1 ? delta[t] : 0.f;
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int r = stream_of(j, g);
        if (j >= 4 * RT) {                            // the second half of a step, which one tile does not have
            qs.zero(j);
            os.zero(j);
            lse2s[j] = deltas[j] = 0.f;
            continue;
        }
        const Row row = row_at(a, q0, h, r < R ? r : R - 1);
        const int64_t col = (int64_t)row.head * a.D;
        scol.load(qs.w[j], (const char *)a.q + (row.query * a.ld_q + col) * ES, 0);
        scol.load(os.w[j], (const char *)a.dout + (row.query * a.ld_dout + col) * ES, 0);
        // row r's values are lane r % 16's of tile r / 16
        lse2s[j] = __shfl(lse2[j >> 2], r & 15, AMS_WAVE);
        deltas[j] = __shfl(delta[j >> 2], r & 15, AMS_WAVE);
    }
    if (on != 0xffffffffu) {
        qs.keep(on, g);
        os.keep(on, g);
    }
    const float c = a.scale * kLog2e;
    const uint32_t ldk = (uint32_t)(a.ld_k * ES), ldv = (uint32_t)(a.ld_v * ES);
    uint32_t krow[2] = {m * ldk, (16 + m) * ldk}, vrow[2] = {m * ldv, (16 + m) * ldv}, srow[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) srow[j] = (uint32_t)stream_of(j, g) * ldk;

    for (int kb = lo; kb < hi; kb += kKeyTile) {
        Frag kf[2][NF], vf[2][NF];
        Slice<T, DH> kk;
        const uint32_t live = live_bits(k0 + kb, k0 + hi, a.mask);
        if (kb + kKeyTile > hi) {
            const int last = hi - 1 - kb;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                krow[t] = (uint32_t)min(16 * t + m, last) * ldk;
                vrow[t] = (uint32_t)min(16 * t + m, last) * ldv;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) srow[j] = (uint32_t)min(stream_of(j, g), last) * ldk;
        }
        const char *kp = (const char *)a.k + ((int64_t)(k0 + kb) * a.ld_k + (int64_t)h * a.D) * ES;
        const char *vp = (const char *)a.v + ((int64_t)(k0 + kb) * a.ld_v + (int64_t)h * a.D) * ES;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            rc.load(kf[t], kp, krow[t]);
            rc.load(vf[t], vp, vrow[t]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) scol.load(kk.w[j], kp, srow[j]);
        if (live != 0xffffffffu) kk.keep(live, g);

        // a row per lane: dQ
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float ds[8];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f}, dp = s;
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    s = mma<T>(kf[t][f], qf[rt][f], s);
                    dp = mma<T>(vf[t][f], df[rt][f], dp);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float p = __builtin_amdgcn_exp2f(s[r] * c - lse2[rt]);
                    ds[4 * t + r] = p * (dp[r] - delta[rt]) * a.scale;
                }
            }
            const bool mine = on >> (16 * rt + m) & 1;
            if (live != 0xffffffffu || on != 0xffffffffu) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    ds[j] = mine && (live >> (4 * g + stream_of(j, 0)) & 1) ? ds[j] : 0.f;
            }
            mma_slice<T, DH>(acc[rt], kk, Stream<T>(ds));
        }
        // a key per lane: dK and dV
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float p[8], ds[8];
#pragma unroll
            for (int rt = 0; rt < 2; ++rt) {
                if (rt >= RT) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) p[4 + r] = ds[4 + r] = 0.f;
                    continue;
                }
                f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f}, dp = s;
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    s = mma<T>(qf[rt % RT][f], kf[t][f], s);
                    dp = mma<T>(df[rt % RT][f], vf[t][f], dp);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 4 * rt + r;
                    p[j] = __builtin_amdgcn_exp2f(s[r] * c - lse2s[j]);
                    ds[j] = p[j] * (dp[r] - deltas[j]) * a.scale;
                }
            }
            const bool mine = live >> (16 * t + m) & 1;
            if (live != 0xffffffffu || on != 0xffffffffu) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool both = mine && (on >> (4 * g + stream_of(j, 0)) & 1);
                    p[j] = both ? p[j] : 0.f;
                    ds[j] = both ? ds[j] : 0.f;
                }
            }
            f32x4 ak[VD], av[VD];
#pragma unroll
            for (int e = 0; e < VD; ++e) ak[e] = av[e] = f32x4{0.f, 0.f, 0.f, 0.f};
            mma_slice<T, DH, RT == 1>(ak, qs, Stream<T>(ds));
            mma_slice<T, DH, RT == 1>(av, os, Stream<T>(p));
            const int key = kb + 16 * t + m;
            if (key < hi) {
                float o[4 * VD];
                acc_in_order<VD>(ak, 1.f, o);
                store_elems<T, 4 * VD, PB>(dkp + (int64_t)(k0 + key) * a.ld_dk, 4 * g * VD, a.D, o);
                acc_in_order<VD>(av, 1.f, o);
                store_elems<T, 4 * VD, PB>(dvp + (int64_t)(k0 + key) * a.ld_dv, 4 * g * VD, a.D, o);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int r = 16 * t + m;
        if (r >= R) continue;
        const Row row = row_at(a, q0, h, r);
        float o[4 * VD];
        acc_in_order<VD>(acc[t], 1.f, o);
        if (a.nsplit > 1) {
            float *p = a.part_o + ((int64_t)wk.split * a.n_q * a.H + row.query * a.H + row.head) * a.D;
#pragma unroll
            for (int e = 0; e < 4 * VD; ++e)
                if (4 * g * VD + e < a.D) p[4 * g * VD + e] = o[e];
        } else {
            store_elems<T, 4 * VD, PB>((T *)a.dq + row.query * a.ld_dq + (int64_t)row.head * a.D, 4 * g * VD, a.D, o);
        }
    }
}

// Partial sums of the splits added in their order: `per` = 1 (dQ, rows of
// q_off's samples) or 2 (dK then dV, keys of k_off's); one thread per element.
template <class T>
__global__ __launch_bounds__(kAttnThreads) void attn_sum_k(const float *part, int nsplit, int per, int heads, int D,
                                                           const int32_t *off, int B, int64_t n, T *x0, int64_t ld0,
                                                           T *x1, int64_t ld1)
{
    const int64_t width = (int64_t)heads * per * D, total = n * width;
    const int64_t lo = clamp_off(off[0], n), hi = clamp_off(off[B], n);
    for (int64_t e = (int64_t)blockIdx.x * kAttnThreads + threadIdx.x; e < total;
         e += (int64_t)gridDim.x * kAttnThreads) {
        const int64_t entry = e / width;
        if (entry < lo || entry >= hi) continue;       // no sample's: left as it was
        const int in = (int)(e - entry * width), head = in / (per * D), w = in - head * per * D;
        float y = 0.f;
#pragma unroll 4
        for (int s = 0; s < nsplit; ++s) y += part[s * total + e];
        T *dst = w < D ? x0 + entry * ld0 + (int64_t)head * D + w : x1 + entry * ld1 + (int64_t)head * D + w - D;
        store_elems<T, 1, (int)sizeof(T)>(dst, 0, 1, &y);
    }
}

// ------------------------------------------------------------------- host

struct Plan {
    Cut fwd, dq;
    bool many;                        // the kernels of attn_many.h
    int few_rows, few_rt, few_split;  // samples of at most few_rows rows go to attn_bwd_few_k (-1: none)
    int dkv;                          // splits of the rows
    int64_t key_tiles;
    size_t delta, total;              // workspace: delta's bytes, all
};

ams_status plan_of(const ams_attn *at, int32_t B, int64_t n_q, int64_t n_k, bool wide, Plan &p)
{
    const ams_status s = attn_shape(at);
    if (s != AMS_OK) return s;
    const int64_t G = at->n_heads / at->n_kv_heads, Hk = at->n_kv_heads;
    if (B < 0 || n_q < 0 || n_k < 0 || n_q > kAttnMaxEntries || n_q * G > kAttnMaxEntries || n_k > kAttnMaxEntries)
        return AMS_ERR_SIZE;
    const int64_t samples = B < 1 ? 1 : B, rows = n_q * G, keys = n_k / samples;
    p.fwd = p.dq = cut_rows(at, B, n_q, keys, wide);
    // from more rows than attn_bwd_few_k's tile holds (512 samples of 200 keys, 4 heads of 64, forward + backward:
    // 35 + 48 us at 32 rows against 39 + 136 with attn_many.h, 48 + 176 at 48 rows against 42 + 119)
    // and from 64 keys: with fewer the weights' rounding there shows next to the output's (dQ and dK off by 2.7e-3 at 8
    // keys, 2.4e-3 from 64 on, 1.9e-3 with pairs)
    p.many = at->dtype == AMS_BF16 && keys >= 64 &&
             cut_many(at, B, n_q, keys, at->head_dim <= 64 ? 32 : 16, p.fwd);
    if (p.many) p.dq = p.fwd;
    // one pass over the keys where most samples' rows fit one tile
    p.few_rt = wide && at->head_dim <= 64 && rows > 8 * samples ? 2 : 1;
    p.few_rows = rows <= 16 * p.few_rt * samples ? 16 * p.few_rt : -1;
    p.few_split = 1;
    if (p.few_rows > 0) {
        p.few_split = split_count((samples * Hk + 3) / 4, keys);      // a wave per split here
        p.dq.rt = p.few_rt, p.dq.wk = 4, p.dq.nsplit = p.few_split;
        p.dq.tiles = tiles_of(rows, p.dq.rt == 2 ? 5 : 4, B);
        p.dq.blocks = p.dq.tiles * Hk * p.dq.nsplit;
    }
    const int key_shift = p.many ? kManyShift : 6;
    p.key_tiles = tiles_of(n_k, key_shift, B);
    const int64_t kt = (n_k + (1 << key_shift) - 1) >> key_shift, ks = n_k < B ? n_k : B;
    const int64_t key_blocks = (kt > ks ? kt : ks) * Hk;
    p.dkv = p.few_rows > 0 ? 1 : (p.many ? split_many : split_count)(key_blocks, rows / samples);
    if (p.fwd.blocks > kAttnMaxBlocks || p.dq.blocks > kAttnMaxBlocks || p.key_tiles * Hk * p.dkv > kAttnMaxBlocks)
        return AMS_ERR_SIZE;
    const size_t all = (size_t)n_q * at->n_heads, D = at->head_dim, f = sizeof(float);
    const size_t fwd = p.fwd.nsplit > 1 ? align_up(p.fwd.nsplit * all * 2 * f) + p.fwd.nsplit * all * D * f : 0;
    const size_t dq = p.dq.nsplit > 1 ? p.dq.nsplit * all * D * f : 0;
    const size_t dkv = p.dkv > 1 ? (size_t)p.dkv * n_k * Hk * 2 * D * f : 0;
    p.delta = align_up(all * f) + 256;              // and any_many
    const size_t bwd = p.delta + (dq > dkv ? dq : dkv);
    p.total = 256 + (fwd > bwd ? fwd : bwd);
    return AMS_OK;
}

bool strides_ok(int64_t width, std::initializer_list<int64_t> lds)
{
    for (int64_t ld : lds)
        if (ld < width || ld > kAttnMaxStride) return false;
    return true;
}

AttnArgs args_of(const ams_attn *at, int32_t B, const int32_t *q_off, int64_t n_q, const int32_t *k_off, int64_t n_k,
                 const void *q, int64_t ld_q, const void *k, int64_t ld_k, const void *v, int64_t ld_v,
                 const uint8_t *mask)
{
    AttnArgs a{};
    a.B = B, a.H = at->n_heads, a.Hk = at->n_kv_heads, a.G = a.H / a.Hk, a.D = at->head_dim;
    a.by_g = fast_div((uint32_t)a.G);
    a.scale = at->scale;
    a.q_off = q_off, a.n_q = n_q, a.k_off = k_off, a.n_k = n_k;
    a.q = q, a.ld_q = ld_q, a.k = k, a.ld_k = ld_k, a.v = v, a.ld_v = ld_v, a.mask = mask;
    return a;
}

}  // namespace

extern "C" size_t ams_xattn_workspace(const ams_attn *attn, int32_t B, int64_t n_q, int64_t n_k)
{
    Plan p, q;                         // whichever pieces the call's addresses allow
    if (!attn || plan_of(attn, B, n_q, n_k, true, p) != AMS_OK || plan_of(attn, B, n_q, n_k, false, q) != AMS_OK) return 0;
    return p.total > q.total ? p.total : q.total;
}

extern "C" ams_status ams_xattn_fwd(const ams_attn *attn, int32_t B, const int32_t *q_off, int64_t n_q,
                                    const int32_t *k_off, int64_t n_k, const void *q, int64_t ld_q, const void *k,
                                    int64_t ld_k, const void *v, int64_t ld_v, const uint8_t *key_mask, void *out,
                                    int64_t ld_out, float *lse, void *ws, size_t ws_bytes, void *stream)
{
    if (!attn) return AMS_ERR_NULL;
    const int64_t ld[] = {ld_q, ld_k, ld_v, ld_out};
    const void *ptr[] = {q, k, v, out};
    const int pb = piece_bytes(attn->dtype == AMS_F32 ? 4 : 2, attn->head_dim, 4, ld, ptr);
    Plan pl;
    const ams_status s = plan_of(attn, B, n_q, n_k, pb == 16, pl);
    if (s != AMS_OK) return s;
    const int64_t wq = (int64_t)attn->n_heads * attn->head_dim, wk = (int64_t)attn->n_kv_heads * attn->head_dim;
    if (!strides_ok(wq, {ld_q, ld_out}) || !strides_ok(wk, {ld_k, ld_v})) return AMS_ERR_SIZE;
    if (B == 0 || n_q == 0) return AMS_OK;
    if (!q_off || !k_off || !q || !out || !ws || (n_k > 0 && (!k || !v))) return AMS_ERR_NULL;
    if (ws_bytes < pl.total) return AMS_ERR_WORKSPACE;
    AttnArgs a = args_of(attn, B, q_off, n_q, k_off, n_k, q, ld_q, k, ld_k, v, ld_v, key_mask);
    a.out = out, a.ld_out = ld_out, a.lse = lse, a.nsplit = pl.fwd.nsplit, a.tiles = pl.fwd.tiles;
    a.part_ml = (float *)align_up((size_t)ws);
    a.part_o = (float *)((char *)a.part_ml + align_up((size_t)a.nsplit * n_q * a.H * 2 * sizeof(float)));
    hipStream_t st = (hipStream_t)stream;
    return with_attn(attn->dtype, a.D, pb, [&](auto t, auto dh, auto piece) {
        using T = decltype(t);
        constexpr int DH = decltype(dh)::value, PB = decltype(piece)::value;
        if constexpr (sizeof(T) == 2) {
            if (pl.many) {
                AMS_LAUNCH("xattn_fwd_many", st,
                           attn_fwd_many_k<DH, PB, false><<<(unsigned)pl.fwd.blocks, kAttnThreads, 0, st>>>(a));
                if (a.nsplit > 1) launch_join<T>("xattn_join", a, st);
                return ams_launch_status();
            }
        }
        with_cut<T, DH, PB>(pl.fwd, [&](auto rt, auto wk) {
            AMS_LAUNCH("xattn_fwd", st,
                       attn_fwd_k<T, DH, PB, false, decltype(rt)::value, decltype(wk)::value>
                       <<<(unsigned)pl.fwd.blocks, kAttnThreads, 0, st>>>(a));
            return AMS_OK;
        });
        if (a.nsplit > 1) launch_join<T>("xattn_join", a, st);
        return ams_launch_status();
    });
}

extern "C" ams_status ams_xattn_bwd(const ams_attn *attn, int32_t B, const int32_t *q_off, int64_t n_q,
                                    const int32_t *k_off, int64_t n_k, const void *q, int64_t ld_q, const void *k,
                                    int64_t ld_k, const void *v, int64_t ld_v, const uint8_t *key_mask,
                                    const void *out, int64_t ld_out, const float *lse, const void *dout,
                                    int64_t ld_dout, void *dq, int64_t ld_dq, void *dk, int64_t ld_dk, void *dv,
                                    int64_t ld_dv, void *ws, size_t ws_bytes, void *stream)
{
    if (!attn) return AMS_ERR_NULL;
    const int64_t ld[] = {ld_q, ld_k, ld_v, ld_out, ld_dout, ld_dq, ld_dk, ld_dv};
    const void *ptr[] = {q, k, v, out, dout, dq, dk, dv};
    const int pb = piece_bytes(attn->dtype == AMS_F32 ? 4 : 2, attn->head_dim, 8, ld, ptr);
    Plan pl;
    const ams_status s = plan_of(attn, B, n_q, n_k, pb == 16, pl);
    if (s != AMS_OK) return s;
    const int64_t wq = (int64_t)attn->n_heads * attn->head_dim, wk = (int64_t)attn->n_kv_heads * attn->head_dim;
    if (!strides_ok(wq, {ld_q, ld_out, ld_dout, ld_dq}) || !strides_ok(wk, {ld_k, ld_v, ld_dk, ld_dv}))
        return AMS_ERR_SIZE;
    if (B == 0 || (n_q == 0 && n_k == 0)) return AMS_OK;
    if (!q_off || !k_off || !ws || (n_q > 0 && (!q || !out || !lse || !dout || !dq)) ||
        (n_k > 0 && (!k || !v || !dk || !dv)))
        return AMS_ERR_NULL;
    if (ws_bytes < pl.total) return AMS_ERR_WORKSPACE;
    AttnArgs a = args_of(attn, B, q_off, n_q, k_off, n_k, q, ld_q, k, ld_k, v, ld_v, key_mask);
    a.o = out, a.ld_o = ld_out, a.lse = (float *)lse, a.dout = dout, a.ld_dout = ld_dout;
    a.dq = dq, a.ld_dq = ld_dq, a.dk = dk, a.ld_dk = ld_dk, a.dv = dv, a.ld_dv = ld_dv;
    a.delta = (float *)align_up((size_t)ws);
    a.any_many = (int32_t *)((char *)a.delta + pl.delta - 256);
    a.part_o = (float *)((char *)a.delta + pl.delta);
    a.few_rows = pl.few_rows;
    // rows of one sample beyond a few: can there be any?
    const bool many = pl.few_rows < 0 || n_q * a.G > pl.few_rows;
    hipStream_t st = (hipStream_t)stream;
    return with_attn(attn->dtype, a.D, pb, [&](auto t, auto dh, auto piece) {
        using T = decltype(t);
        constexpr int DH = decltype(dh)::value, PB = decltype(piece)::value;
        auto sum = [&](int per, int heads, const int32_t *off, int64_t n, void *x0, int64_t ld0, void *x1, int64_t ld1) {
            const int64_t blocks = (n * heads * per * a.D + kAttnThreads - 1) / kAttnThreads;
            AMS_LAUNCH("xattn_sum", st,
                       attn_sum_k<T><<<(unsigned)(blocks < 8192 ? blocks : 8192), kAttnThreads, 0, st>>>(
                           a.part_o, a.nsplit, per, heads, a.D, off, B, n, (T *)x0, ld0, (T *)x1, ld1));
        };
        if constexpr (sizeof(T) == 2) {
            if (pl.many) {
                if (n_q > 0) {
                    a.nsplit = pl.dq.nsplit, a.tiles = pl.dq.tiles;
                    AMS_LAUNCH("xattn_dq_many", st,
                               attn_dq_many_k<DH, PB><<<(unsigned)pl.dq.blocks, kAttnThreads, 0, st>>>(a));
                    if (a.nsplit > 1) sum(1, a.H, q_off, n_q, dq, ld_dq, nullptr, 0);
                }
                if (n_k > 0) {
                    a.nsplit = pl.dkv, a.tiles = pl.key_tiles;
                    AMS_LAUNCH("xattn_dkv_many", st,
                               attn_dkv_many_k<DH, PB><<<(unsigned)(pl.key_tiles * a.Hk * a.nsplit), kAttnThreads, 0, st>>>(a));
                    if (a.nsplit > 1) sum(2, a.Hk, k_off, n_k, dk, ld_dk, dv, ld_dv);
                }
                return ams_launch_status();
            }
        }
        // beside attn_bwd_few_k usually nothing is left: blocks enough to fill the chip, each with several tiles
        auto grid = [&](int64_t blocks) { return (unsigned)(pl.few_rows > 0 && blocks > 1024 ? 1024 : blocks); };
        if (pl.few_rows > 0) {
            a.nsplit = pl.few_split;
            const int64_t waves = (int64_t)B * a.Hk * a.nsplit;
            const unsigned blocks = (unsigned)((waves + kAttnWaves - 1) / kAttnWaves) + 1;
            auto few = [&](auto rt) {
                AMS_LAUNCH("xattn_bwd_few", st,
                           attn_bwd_few_k<T, DH, PB, decltype(rt)::value><<<blocks, kAttnThreads, 0, st>>>(a));
            };
            if constexpr (PB == 16 && DH <= 64) {
                if (pl.few_rt == 2) few(std::integral_constant<int, 2>());
                else few(std::integral_constant<int, 1>());
            } else {
                few(std::integral_constant<int, 1>());
            }
        }
        if (n_q > 0) {
            a.nsplit = pl.dq.nsplit, a.tiles = pl.dq.tiles, a.blocks = pl.dq.blocks;
            if (many)
                with_cut<T, DH, PB>(pl.dq, [&](auto rt, auto wk) {
                    AMS_LAUNCH("xattn_dq", st,
                               attn_dq_k<T, DH, PB, decltype(rt)::value, decltype(wk)::value>
                               <<<grid(a.blocks), kAttnThreads, 0, st>>>(a));
                    return AMS_OK;
                });
            if (a.nsplit > 1) sum(1, a.H, q_off, n_q, dq, ld_dq, nullptr, 0);
        }
        if (n_k > 0 && many) {
            a.nsplit = pl.dkv, a.blocks = pl.key_tiles * a.Hk * a.nsplit;
            AMS_LAUNCH("xattn_dkv", st, attn_dkv_k<T, DH, PB><<<grid(a.blocks), kAttnThreads, 0, st>>>(a));
            if (a.nsplit > 1) sum(2, a.Hk, k_off, n_k, dk, ld_dk, dv, ld_dv);
        }
        return ams_launch_status();
    });
}
