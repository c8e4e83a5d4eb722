// attn.hip -- multi-head attention of each sample's queries to that sample's
// keys, two lists of different lengths (the tiles are attn_device.h's).
//   ams_xattn_fwd  P = softmax(scale Q K^T) over the sample's live keys, O = P V
//   ams_xattn_bwd  with delta = rowsum(dO o O) and dS = scale P o (dO V^T - delta):
//                  dQ = dS K, dK = dS^T Q, dV = P^T dO, the last two summed over
//                  the query heads of a key head.
// The backward forms P again from the forward's log-sum-exp, in two kernels
// with one owner per result and no atomics: dQ's blocks own row tiles and
// stream keys as the forward does; dK's and dV's own keys, 16 a wave, and
// stream the rows (all heads of the group), so both their contractions have
// the operand layouts of the forward with rows and keys exchanged.
#include "attn_device.h"

namespace {

// -------------------------------------------------------------- dQ, delta

template <class T, int DH, int PB>
__global__ __launch_bounds__(kAttnThreads) void attn_dq_k(AttnArgs a)
{
    constexpr int NF = DH / (4 * Num<T>::EP), VD = DH / 16;
    __shared__ float s_o[kAttnWaves][kRowTile][DH + 4];
    const int lane = ams_lane(), m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE);
    int64_t b = blockIdx.x;
    const int split = (int)(b % a.nsplit);
    b /= a.nsplit;
    const int h = (int)(b % a.Hk);
    const Span rows = span_of(a.q_off, a.B, a.n_q, a.G, 4, b / a.Hk);
    const int64_t R = (int64_t)rows.count * a.G;
    if (rows.first < 0 || rows.first >= R) return;
    const int64_t r_mine = rows.first + m;
    const Row row = row_at(a, rows.begin, h, (int)(r_mine < R ? r_mine : R - 1));
    const int k0 = clamp_off(a.k_off[rows.i], a.n_k), k1 = clamp_off(a.k_off[rows.i + 1], a.n_k);
    int lo, hi;
    split_range(k1 > k0 ? k1 - k0 : 0, split, a.nsplit, lo, hi);

    Frag qf[NF], df[NF], of[NF];
    load_row<T, DH, PB>(qf, (const T *)a.q + row.query * a.ld_q + (int64_t)row.head * a.D, g, a.D);
    load_row<T, DH, PB>(df, (const T *)a.dout + row.query * a.ld_dout + (int64_t)row.head * a.D, g, a.D);
    load_row<T, DH, PB>(of, (const T *)a.o + row.query * a.ld_o + (int64_t)row.head * a.D, g, a.D);
    const int64_t at = row.query * a.H + row.head;
    const float lse = a.lse[at];
    const bool live_row = lse != kNegInf;             // a row without keys: its upstream gradient goes nowhere
    float delta = 0.f;
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                delta += df[f].f[i] * of[f].f[i];
            } else {
                delta += __uint_as_float(df[f].u[i] << 16) * __uint_as_float(of[f].u[i] << 16);
                delta += __uint_as_float(df[f].u[i] & 0xffff0000u) * __uint_as_float(of[f].u[i] & 0xffff0000u);
            }
        }
    delta = live_row ? sum_groups(delta) : 0.f;
    if (split == 0 && wave == 0 && g == 0 && r_mine < R) a.delta[at] = delta;

    const float c = a.scale * kLog2e, lse2 = live_row ? lse * kLog2e : 0.f;
    f32x4 acc[VD];
#pragma unroll
    for (int t = 0; t < VD; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const T *kp = (const T *)a.k + (int64_t)h * a.D, *vp = (const T *)a.v + (int64_t)h * a.D;
    for (int kb = lo + wave * kKeyTile; kb < hi; kb += kAttnWaves * kKeyTile) {
        Slice<T, DH> kk;
        bool live[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            int key = kb + stream_of(j, g);
            live[j] = key < hi && live_row;
            key = k0 + (key < hi ? key : hi - 1);
            load_elems<T, VD, PB>(kk.w[j], kp + (int64_t)key * a.ld_k, m * VD, a.D);
            if (a.mask && a.mask[key] == 0) {
                live[j] = false;
                kk.zero(j);
            }
        }
        float ds[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            Frag kf[NF], vf[NF];
            int key = kb + 16 * t + m;
            key = k0 + (key < hi ? key : hi - 1);
            load_row<T, DH, PB>(kf, kp + (int64_t)key * a.ld_k, g, a.D);
            load_row<T, DH, PB>(vf, vp + (int64_t)key * a.ld_v, g, a.D);
            f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f}, dp = s;
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                s = mma<T>(kf[f], qf[f], s);
                dp = mma<T>(vf[f], df[f], dp);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = 4 * t + r;
                const float p = __builtin_amdgcn_exp2f(s[r] * c - lse2);
                ds[j] = live[j] ? p * (dp[r] - delta) * a.scale : 0.f;
            }
        }
        mma_slice<T, DH>(acc, kk, Stream<T>(ds));
    }
    float o[4 * VD];
    acc_in_order<VD>(acc, 1.f, o);
#pragma unroll
    for (int i = 0; i < 4 * VD; ++i) s_o[wave][m][4 * g * VD + i] = o[i];
    __syncthreads();
    const int r = threadIdx.x / 16, d = (threadIdx.x % 16) * VD;
    const int64_t ro = rows.first + r;
    if (ro >= R) return;
    float y[VD];
#pragma unroll
    for (int e = 0; e < VD; ++e) y[e] = (s_o[0][r][d + e] + s_o[1][r][d + e]) + (s_o[2][r][d + e] + s_o[3][r][d + e]);
    const Row ow = row_at(a, rows.begin, h, (int)ro);
    if (a.nsplit > 1) {
        float *p = a.part_o + ((int64_t)split * a.n_q * a.H + ow.query * a.H + ow.head) * a.D;
#pragma unroll
        for (int e = 0; e < VD; ++e)
            if (d + e < a.D) p[d + e] = y[e];
        return;
    }
    store_elems<T, VD, PB>((T *)a.dq + ow.query * a.ld_dq + (int64_t)ow.head * a.D, d, a.D, y);
}

// ----------------------------------------------------------------- dK, dV

// One block per (64 keys of a sample, key head, split of the rows).
template <class T, int DH, int PB>
__global__ __launch_bounds__(kAttnThreads) void attn_dkv_k(AttnArgs a)
{
    constexpr int NF = DH / (4 * Num<T>::EP), VD = DH / 16;
    const int lane = ams_lane(), m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE);
    int64_t b = blockIdx.x;
    const int split = (int)(b % a.nsplit);
    b /= a.nsplit;
    const int h = (int)(b % a.Hk);
    const Span keys = span_of(a.k_off, a.B, a.n_k, 1, 6, b / a.Hk);
    const int64_t first = keys.first + wave * 16;
    if (keys.first < 0 || first >= keys.count) return;
    const int q0 = clamp_off(a.q_off[keys.i], a.n_q), q1 = clamp_off(a.q_off[keys.i + 1], a.n_q);
    const int64_t R = q1 > q0 ? (int64_t)(q1 - q0) * a.G : 0;
    int lo, hi;
    split_range((int)R, split, a.nsplit, lo, hi);

    const bool mine = first + m < keys.count;
    const int64_t key = keys.begin + (mine ? first + m : keys.count - 1);
    const bool live_key = mine && !(a.mask && a.mask[key] == 0);
    Frag kf[NF], vf[NF];
    load_row<T, DH, PB>(kf, (const T *)a.k + key * a.ld_k + (int64_t)h * a.D, g, a.D);
    load_row<T, DH, PB>(vf, (const T *)a.v + key * a.ld_v + (int64_t)h * a.D, g, a.D);
    const float c = a.scale * kLog2e;
    f32x4 ak[VD], av[VD];
#pragma unroll
    for (int t = 0; t < VD; ++t) ak[t] = av[t] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int rb = lo; rb < hi; rb += kKeyTile) {
        Slice<T, DH> qs, os;
        float lse2[8], delta[8];
        bool live[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            int r = rb + stream_of(j, g);
            live[j] = r < hi;
            r = r < hi ? r : hi - 1;
            const Row w = row_at(a, q0, h, r);
            const int64_t at = w.query * a.H + w.head;
            const float l = a.lse[at];
            live[j] = live[j] && l != kNegInf;
            lse2[j] = l * kLog2e;
            delta[j] = a.delta[at];
            load_elems<T, VD, PB>(qs.w[j], (const T *)a.q + w.query * a.ld_q + (int64_t)w.head * a.D, m * VD, a.D);
            load_elems<T, VD, PB>(os.w[j], (const T *)a.dout + w.query * a.ld_dout + (int64_t)w.head * a.D, m * VD,
                                  a.D);
        }
        float p[8], ds[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            Frag qf[NF], df[NF];
            const int r = rb + 16 * t + m;
            const Row w = row_at(a, q0, h, r < hi ? r : hi - 1);
            load_row<T, DH, PB>(qf, (const T *)a.q + w.query * a.ld_q + (int64_t)w.head * a.D, g, a.D);
            load_row<T, DH, PB>(df, (const T *)a.dout + w.query * a.ld_dout + (int64_t)w.head * a.D, g, a.D);
            f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f}, dp = s;
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                s = mma<T>(qf[f], kf[f], s);
                dp = mma<T>(df[f], vf[f], dp);
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
        float *p = a.part_o + ((int64_t)split * a.n_k * a.Hk + key * a.Hk + h) * 2 * a.D;
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
    int fwd, dq, dkv;                 // splits
    int64_t row_tiles, key_tiles;
    size_t delta, total;              // workspace: delta's bytes, all
};

ams_status plan_of(const ams_attn *at, int32_t B, int64_t n_q, int64_t n_k, Plan &p)
{
    const ams_status s = attn_shape(at);
    if (s != AMS_OK) return s;
    const int64_t G = at->n_heads / at->n_kv_heads, Hk = at->n_kv_heads;
    if (B < 0 || n_q < 0 || n_k < 0 || n_q * G > INT32_MAX || n_k > INT32_MAX) return AMS_ERR_SIZE;
    const int64_t samples = B < 1 ? 1 : B;
    p.row_tiles = row_tiles(at, B, n_q);
    p.key_tiles = (n_k >> 6) + B;
    p.fwd = p.dq = split_count(busy_row_tiles(at, B, n_q), n_k / samples / 128);
    const int64_t kt = (n_k + 63) / 64, ks = n_k < B ? n_k : B;
    p.dkv = split_count((kt > ks ? kt : ks) * Hk, n_q * G / samples / 32);
    if (p.row_tiles * Hk * p.fwd > kAttnMaxBlocks || p.key_tiles * Hk * p.dkv > kAttnMaxBlocks) return AMS_ERR_SIZE;
    const size_t rows = (size_t)n_q * at->n_heads, D = at->head_dim, f = sizeof(float);
    const size_t fwd = p.fwd > 1 ? align_up(p.fwd * rows * 2 * f) + p.fwd * rows * D * f : 0;
    const size_t dq = p.dq > 1 ? p.dq * rows * D * f : 0;
    const size_t dkv = p.dkv > 1 ? (size_t)p.dkv * n_k * Hk * 2 * D * f : 0;
    p.delta = align_up(rows * f);
    const size_t bwd = p.delta + (dq > dkv ? dq : dkv);
    p.total = 256 + (fwd > bwd ? fwd : bwd);
    return AMS_OK;
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
    Plan p;
    return attn && plan_of(attn, B, n_q, n_k, p) == AMS_OK ? p.total : 0;
}

extern "C" ams_status ams_xattn_fwd(const ams_attn *attn, int32_t B, const int32_t *q_off, int64_t n_q,
                                    const int32_t *k_off, int64_t n_k, const void *q, int64_t ld_q, const void *k,
                                    int64_t ld_k, const void *v, int64_t ld_v, const uint8_t *key_mask, void *out,
                                    int64_t ld_out, float *lse, void *ws, size_t ws_bytes, void *stream)
{
    if (!attn) return AMS_ERR_NULL;
    Plan pl;
    const ams_status s = plan_of(attn, B, n_q, n_k, pl);
    if (s != AMS_OK) return s;
    const int64_t wq = (int64_t)attn->n_heads * attn->head_dim, wk = (int64_t)attn->n_kv_heads * attn->head_dim;
    if (ld_q < wq || ld_out < wq || ld_k < wk || ld_v < wk) return AMS_ERR_SIZE;
    if (B == 0 || n_q == 0) return AMS_OK;
    if (!q_off || !k_off || !q || !out || !ws || (n_k > 0 && (!k || !v))) return AMS_ERR_NULL;
    if (ws_bytes < pl.total) return AMS_ERR_WORKSPACE;
    AttnArgs a = args_of(attn, B, q_off, n_q, k_off, n_k, q, ld_q, k, ld_k, v, ld_v, key_mask);
    a.out = out, a.ld_out = ld_out, a.lse = lse, a.nsplit = pl.fwd;
    a.part_ml = (float *)align_up((size_t)ws);
    a.part_o = (float *)((char *)a.part_ml + align_up((size_t)pl.fwd * n_q * a.H * 2 * sizeof(float)));
    hipStream_t st = (hipStream_t)stream;
    const int64_t ld[] = {ld_q, ld_k, ld_v, ld_out};
    const void *ptr[] = {q, k, v, out};
    const int pb = piece_bytes(attn->dtype == AMS_F32 ? 4 : 2, a.D, 4, ld, ptr);
    return with_attn(attn->dtype, a.D, pb, [&](auto t, auto dh, auto piece) {
        using T = decltype(t);
        const unsigned blocks = (unsigned)(pl.row_tiles * a.Hk * a.nsplit);
        AMS_LAUNCH("xattn_fwd", st,
                   attn_fwd_k<T, decltype(dh)::value, decltype(piece)::value, false><<<blocks, kAttnThreads, 0, st>>>(a));
        if (a.nsplit > 1)
            AMS_LAUNCH("xattn_join", st,
                       attn_join_k<T><<<(unsigned)((n_q * a.H + kAttnWaves - 1) / kAttnWaves), kAttnThreads, 0, st>>>(a));
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
    Plan pl;
    const ams_status s = plan_of(attn, B, n_q, n_k, pl);
    if (s != AMS_OK) return s;
    const int64_t wq = (int64_t)attn->n_heads * attn->head_dim, wk = (int64_t)attn->n_kv_heads * attn->head_dim;
    if (ld_q < wq || ld_out < wq || ld_dout < wq || ld_dq < wq || ld_k < wk || ld_v < wk || ld_dk < wk || ld_dv < wk)
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
    a.part_o = (float *)((char *)a.delta + pl.delta);
    hipStream_t st = (hipStream_t)stream;
    const int64_t ld[] = {ld_q, ld_k, ld_v, ld_out, ld_dout, ld_dq, ld_dk, ld_dv};
    const void *ptr[] = {q, k, v, out, dout, dq, dk, dv};
    const int pb = piece_bytes(attn->dtype == AMS_F32 ? 4 : 2, a.D, 8, ld, ptr);
    return with_attn(attn->dtype, a.D, pb, [&](auto t, auto dh, auto piece) {
        using T = decltype(t);
        constexpr int DH = decltype(dh)::value, PB = decltype(piece)::value;
        auto sum = [&](int per, int heads, const int32_t *off, int64_t n, void *x0, int64_t ld0, void *x1, int64_t ld1) {
            const int64_t blocks = (n * heads * per * a.D + kAttnThreads - 1) / kAttnThreads;
            AMS_LAUNCH("xattn_sum", st,
                       attn_sum_k<T><<<(unsigned)(blocks < 8192 ? blocks : 8192), kAttnThreads, 0, st>>>(
                           a.part_o, a.nsplit, per, heads, a.D, off, B, n, (T *)x0, ld0, (T *)x1, ld1));
        };
        if (n_q > 0) {
            a.nsplit = pl.dq;
            AMS_LAUNCH("xattn_dq", st,
                       attn_dq_k<T, DH, PB><<<(unsigned)(pl.row_tiles * a.Hk * a.nsplit), kAttnThreads, 0, st>>>(a));
            if (a.nsplit > 1) sum(1, a.H, q_off, n_q, dq, ld_dq, nullptr, 0);
        }
        if (n_k > 0) {
            a.nsplit = pl.dkv;
            AMS_LAUNCH("xattn_dkv", st,
                       attn_dkv_k<T, DH, PB><<<(unsigned)(pl.key_tiles * a.Hk * a.nsplit), kAttnThreads, 0, st>>>(a));
            if (a.nsplit > 1) sum(2, a.Hk, k_off, n_k, dk, ld_dk, dv, ld_dv);
        }
        return ams_launch_status();
    });
}
