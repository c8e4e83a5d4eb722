// attn_device.h -- tiles and the forward kernel of the sequence attention,
// shared by attn.hip (keys and values as rows) and cache.hip (8-bit pages).
// Internal to the library; the public contract is include/ams.h.
//
// Rows.  The query heads of one key/value head that share a query form rows:
// row r of (sample i, key head h) is query q_off[i] + r / G, head h G + r % G,
// G heads per group, so one read of the keys serves the whole group.  Rows go
// in tiles of 16.  The host knows only n_q and B: sample i's tiles start at
// floor(q_off[i] G / 16) + i, which leaves every sample room for its own
// (a sample's share floor(b/16) - floor(a/16) + 1 is at least
// ceil((b - a) / 16)); a block finds its sample by search and leaves if its
// tile lies past the sample's rows.
//
// Products.  Both products of attention contract a tile of S^T = K Q^T: the
// matrix instruction's result has a row of Q per lane (lane % 16) and four
// consecutive keys per lane group, which is just the operand layout that the
// second product O^T = V^T P^T wants for its contraction over keys, if V's
// operand is read in the same order of keys.  So the probabilities never
// leave their lane: no transposition, no shared memory, and a row's maximum
// and sum are one value per lane.  Operands come from memory straight into
// registers; the four waves of a block take every fourth tile of 32 keys and
// are joined at the end.
#pragma once

#include <type_traits>

#include "ams_device.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kAttnThreads = 256, kAttnWaves = kAttnThreads / AMS_WAVE;
constexpr int kRowTile = 16;          // rows of a tile (lane % 16)
constexpr int kKeyTile = 32;          // streamed keys (or rows) per step of a wave
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_inff();

// A matrix operand of one instruction group, 16 bytes per lane: 8 bf16 (32
// contracted values over the four lane groups) or 4 floats (16 values).
union Frag {
    uint32_t u[4];
    float f[4];
    bf16x8 b;
};

template <class T> struct Num;
template <> struct Num<float> { static constexpr int EP = 4, SF = 2; };       // elements of a piece, fragments of 32
template <> struct Num<uint16_t> { static constexpr int EP = 8, SF = 1; };

template <class T> __device__ __forceinline__ f32x4 mma(const Frag &a, const Frag &b, f32x4 c)
{
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.b, b.b, c, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.f[e], b.f[e], c, 0, 0, 0);
        return c;
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const bf16x2 v = {(__bf16)lo, (__bf16)hi};       // round to nearest even
    return __builtin_bit_cast(uint32_t, v);
}

// r / G for r < 2^31, exact: with s = ceil(log2 G) and m = floor(2^32 (2^s - G) / G) + 1.
struct FastDiv {
    uint32_t m, s, d;
    __device__ __forceinline__ int div(int r) const { return (int)((__umulhi((uint32_t)r, m) + (uint32_t)r) >> s); }
};

inline FastDiv fast_div(uint32_t d)
{
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return {(uint32_t)(((1ull << 32) * ((1ull << s) - d)) / d + 1), s, d};
}

// NE elements of a row from element d on, in loads of at most PB bytes (the
// host picks PB so that every piece is aligned and lies within [0, D) or
// behind it).  Elements behind D are zero; nothing behind D is read.
template <class T, int NE, int PB>
__device__ __forceinline__ void load_elems(uint32_t *dst, const T *row, int d, int D)
{
    constexpr int BYTES = NE * (int)sizeof(T), W = BYTES < PB ? BYTES : PB, PE = W / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < BYTES / W; ++i) {
        const int di = d + i * PE;
        const bool in = di < D;
        const T *p = row + (in ? di : 0);
        if constexpr (W == 16) {
            const uint4 v = *(const uint4 *)p;
            dst[4 * i] = in ? v.x : 0, dst[4 * i + 1] = in ? v.y : 0;
            dst[4 * i + 2] = in ? v.z : 0, dst[4 * i + 3] = in ? v.w : 0;
        } else if constexpr (W == 8) {
            const uint2 v = *(const uint2 *)p;
            dst[2 * i] = in ? v.x : 0, dst[2 * i + 1] = in ? v.y : 0;
        } else if constexpr (W == 4) {
            const uint32_t v = *(const uint32_t *)p;
            dst[i] = in ? v : 0;
        } else {
            constexpr int PER = 4 / W;                // pieces of a word
            const uint32_t v = W == 2 ? (uint32_t)*(const uint16_t *)p : (uint32_t)*(const uint8_t *)p;
            const uint32_t x = in ? v : 0;
            if (i % PER) dst[i / PER] |= x << (8 * W * (i % PER));
            else dst[i / PER] = x;
        }
    }
}

// The reverse: NE floats rounded once to T.
template <class T, int NE, int PB>
__device__ __forceinline__ void store_elems(T *row, int d, int D, const float *v)
{
    constexpr int BYTES = NE * (int)sizeof(T), W = BYTES < PB ? BYTES : PB, PE = W / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < BYTES / W; ++i) {
        const int di = d + i * PE;
        if (di >= D) continue;
        uint32_t w[4] = {0, 0, 0, 0};
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < PE; ++e) w[e] = __float_as_uint(v[i * PE + e]);
        } else {
#pragma unroll
            for (int e = 0; e < PE; e += 2) w[e / 2] = pack_bf16(v[i * PE + e], PE > 1 ? v[i * PE + e + 1] : 0.f);
        }
        if constexpr (W == 16) *(uint4 *)(row + di) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (W == 8) *(uint2 *)(row + di) = make_uint2(w[0], w[1]);
        else if constexpr (W == 4) *(uint32_t *)(row + di) = w[0];
        else *(uint16_t *)(row + di) = (uint16_t)w[0];
    }
}

// A row as operand of a contraction over the head width: fragment c of lane
// group g holds the EP elements from (4 c + g) EP on.
template <class T, int DH, int PB>
__device__ __forceinline__ void load_row(Frag *f, const T *row, int g, int D)
{
    constexpr int EP = Num<T>::EP;
#pragma unroll
    for (int c = 0; c < DH / (4 * EP); ++c) load_elems<T, EP, PB>(f[c].u, row, (4 * c + g) * EP, D);
}

// Streamed entry j of lane group g within a step of 32 (the order in which
// both products see the streamed side).
__device__ __forceinline__ int stream_of(int j, int g) { return 16 * (j >> 2) + 4 * g + (j & 3); }

// The lane's slice of 8 streamed rows, elements (lane % 16) VD .. + VD of
// each, as raw words: operand of a contraction over the streamed rows.
template <class T, int DH> struct Slice {
    static constexpr int VD = DH / 16, WORDS = VD * (int)sizeof(T) / 4 > 0 ? VD * (int)sizeof(T) / 4 : 1;
    uint32_t w[8][WORDS];

    __device__ __forceinline__ void zero(int j)
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[j][i] = 0;
    }
    // operand of output tile t: element t of the 8 slices, in stream order
    __device__ __forceinline__ void frags(int t, Frag *f) const
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j >> 2].u[j & 3] = w[j][t];
        } else {
            const uint32_t sel = (t & 1) ? 0x07060302u : 0x05040100u;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                f[0].u[i] = __builtin_amdgcn_perm(w[2 * i + 1][t / 2], w[2 * i][t / 2], sel);
        }
    }
};

// Probabilities (or their gradients) of the lane's 8 streamed entries as
// operand.  bf16 takes each as a pair, its rounding and the rounded rest, so
// that it enters within 2^-17 of its float32 value: the second instruction
// costs nothing where these kernels run, which is bound by memory, and a
// rounding to 8 bits here would be as large an error as the output's own.
template <class T> struct Stream {
    Frag f[2];
    __device__ __forceinline__ explicit Stream(const float *p)
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j >> 2].f[j & 3] = p[j];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t h = pack_bf16(p[2 * i], p[2 * i + 1]);
                f[0].u[i] = h;
                f[1].u[i] = pack_bf16(p[2 * i] - __uint_as_float(h << 16),
                                      p[2 * i + 1] - __uint_as_float(h & 0xffff0000u));
            }
        }
    }
};

// acc[t] += slice tile t times the stream, over all VD tiles.
template <class T, int DH>
__device__ __forceinline__ void mma_slice(f32x4 *acc, const Slice<T, DH> &s, const Stream<T> &p)
{
#pragma unroll
    for (int t = 0; t < Slice<T, DH>::VD; ++t) {
        Frag f[Num<T>::SF];
        s.frags(t, f);
#pragma unroll
        for (int i = 0; i < 2; ++i) acc[t] = mma<T>(f[sizeof(T) == 4 ? i : 0], p.f[i], acc[t]);
    }
}

// The lane's accumulators in order of the head width: elements
// 4 g VD .. 4 (g + 1) VD of its row (acc[t][r] is element (4 g + r) VD + t).
template <int VD> __device__ __forceinline__ void acc_in_order(const f32x4 *acc, float f, float *v)
{
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < VD; ++t) v[r * VD + t] = acc[t][r] * f;
}

__device__ __forceinline__ float max_groups(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16, AMS_WAVE));
    return fmaxf(x, __shfl_xor(x, 32, AMS_WAVE));
}
__device__ __forceinline__ float sum_groups(float x)
{
    x += __shfl_xor(x, 16, AMS_WAVE);
    return x + __shfl_xor(x, 32, AMS_WAVE);
}

struct AttnArgs {
    int32_t B, H, Hk, G, D, nsplit;
    FastDiv by_g;
    float scale;
    const int32_t *q_off;
    int64_t n_q;
    const void *q;
    int64_t ld_q;
    // keys and values as rows
    const int32_t *k_off;
    int64_t n_k;
    const void *k, *v;
    int64_t ld_k, ld_v;
    const uint8_t *mask;
    // keys and values as 8-bit pages
    const int32_t *len, *page_table;
    int32_t max_pages, page_shift;
    int64_t n_pages;
    const uint8_t *kc, *vc;
    const float *ks, *vs;
    // results
    void *out;
    int64_t ld_out;
    float *lse;
    float *part_ml, *part_o;          // per split and (query, head): {maximum, sum} and D sums
    // backward
    const void *dout;
    int64_t ld_dout;
    const void *o;
    int64_t ld_o;
    float *delta;
    void *dq, *dk, *dv;
    int64_t ld_dq, ld_dk, ld_dv;
};

// Last sample i whose first tile, floor(off[i] mul / tile) + own i, is at most
// `at`, by a search of 64 probes at a time.
__device__ __forceinline__ int find_sample(const int32_t *off, int B, int64_t n, int mul, int tile_shift, int own,
                                           int64_t at)
{
    const int lane = ams_lane();
    int lo = 0, len = B;
    while (len > 1) {
        const int step = (len + AMS_WAVE - 1) / AMS_WAVE;
        const int i = lo + lane * step;
        bool le = false;
        if (lane * step < len) {
            int64_t o = off[i];
            o = o < 0 ? 0 : (o > n ? n : o);
            le = ((o * mul) >> tile_shift) + (int64_t)own * i <= at;
        }
        int c = __popcll(ams_ballot(le));
        c = c < 1 ? 1 : c;
        const int skip = (c - 1) * step;
        lo += skip;
        len = len - skip < step ? len - skip : step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ int clamp_off(int32_t o, int64_t n) { return o < 0 ? 0 : (o > n ? (int)n : o); }

// Sample, first entry and count of tile `at` (tile_shift as in find_sample).
struct Span {
    int i, begin, count;
    int64_t first;               // of the tile, in units of entries x mul
};
__device__ __forceinline__ Span span_of(const int32_t *off, int B, int64_t n, int mul, int tile_shift, int64_t at)
{
    Span s;
    s.i = find_sample(off, B, n, mul, tile_shift, 1, at);
    s.begin = clamp_off(off[s.i], n);
    const int end = clamp_off(off[s.i + 1], n);
    s.count = end > s.begin ? end - s.begin : 0;
    s.first = (at - ((((int64_t)s.begin * mul) >> tile_shift) + s.i)) << tile_shift;
    return s;
}

// A row's query and head.
struct Row {
    int64_t query;
    int head;
};
__device__ __forceinline__ Row row_at(const AttnArgs &a, int q0, int h, int r)
{
    const int q = a.by_g.div(r);
    return {(int64_t)q0 + q, h * a.G + (r - q * a.G)};
}

// The share of `count` streamed entries that split s of n takes: whole steps.
__device__ __forceinline__ void split_range(int count, int s, int n, int &lo, int &hi)
{
    const int steps = (count + kKeyTile - 1) / kKeyTile, per = (steps + n - 1) / n;
    const int64_t l = (int64_t)s * per * kKeyTile, h = l + (int64_t)per * kKeyTile;
    lo = l < count ? (int)l : count;
    hi = h < count ? (int)h : count;
}

// Eight codes (two words of e4m3) as bf16 or float: exact.
template <class T> __device__ __forceinline__ void decode4(uint32_t w, uint32_t *dst)
{
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    if constexpr (sizeof(T) == 4) {
        dst[0] = __float_as_uint(a[0]), dst[1] = __float_as_uint(a[1]);
        dst[2] = __float_as_uint(b[0]), dst[3] = __float_as_uint(b[1]);
    } else {
        // an e4m3 value's float has its low 16 bits clear: the high halves are the bf16 values
        dst[0] = __builtin_amdgcn_perm(__float_as_uint(a[1]), __float_as_uint(a[0]), 0x07060302u);
        dst[1] = __builtin_amdgcn_perm(__float_as_uint(b[1]), __float_as_uint(b[0]), 0x07060302u);
    }
}

// ---------------------------------------------------------------- forward

// One block per (row tile, key head, split of the keys).
template <class T, int DH, int PB, bool PAGED>
__global__ __launch_bounds__(kAttnThreads) void attn_fwd_k(AttnArgs a)
{
    constexpr int EP = Num<T>::EP, NF = DH / (4 * EP), VD = DH / 16;
    constexpr int CB = PB / (int)sizeof(T);           // codes of a piece: as many as elements
    constexpr int kPad = DH + 4;
    __shared__ float s_o[kAttnWaves][kRowTile][kPad];
    __shared__ float s_m[kAttnWaves][kRowTile], s_l[kAttnWaves][kRowTile];
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

    int k0 = 0, nk;
    const int32_t *pages = nullptr;
    if constexpr (PAGED) {
        const int64_t room = (int64_t)a.max_pages << a.page_shift;
        nk = clamp_off(a.len[rows.i], room);
        pages = a.page_table + (int64_t)rows.i * a.max_pages;
    } else {
        k0 = clamp_off(a.k_off[rows.i], a.n_k);
        const int k1 = clamp_off(a.k_off[rows.i + 1], a.n_k);
        nk = k1 > k0 ? k1 - k0 : 0;
    }
    int lo, hi;
    split_range(nk, split, a.nsplit, lo, hi);

    Frag qf[NF];
    load_row<T, DH, PB>(qf, (const T *)a.q + row.query * a.ld_q + (int64_t)row.head * a.D, g, a.D);
    const float c = a.scale * kLog2e;
    f32x4 acc[VD];
#pragma unroll
    for (int t = 0; t < VD; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float mx = kNegInf, l = 0.f;

    for (int kb = lo + wave * kKeyTile; kb < hi; kb += kAttnWaves * kKeyTile) {
        Frag kf[2][NF];
        Slice<T, DH> vv;
        bool live[8];
        float sk[2] = {1.f, 1.f}, sv[2] = {1.f, 1.f};
        if constexpr (PAGED) {
            const int P1 = (1 << a.page_shift) - 1;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                // 16 consecutive tokens lie in one page; a token behind the last reads the last one
                const int tok = kb + 16 * t < hi ? kb + 16 * t : kb;
                const int page = pages[tok >> a.page_shift];
                const bool ok = page >= 0 && page < a.n_pages;
                const int64_t at = (int64_t)(ok ? page : 0) * a.Hk + h;
                sk[t] = a.ks[at];
                sv[t] = a.vs[at];
                const uint8_t *kp = a.kc + (at << a.page_shift) * a.D;
                const uint8_t *vp = a.vc + (at << a.page_shift) * a.D;
                const int in = tok & P1;
                {
                    const uint8_t *r = kp + (int64_t)(in + m) * a.D;
#pragma unroll
                    for (int f = 0; f < NF; ++f) {
                        uint32_t w[EP / 4];
                        load_elems<uint8_t, EP, CB>(w, r, (4 * f + g) * EP, a.D);
#pragma unroll
                        for (int i = 0; i < EP / 4; ++i) decode4<T>(w[i], kf[t][f].u + i * (int)sizeof(T));
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 4 * t + r;
                    const uint8_t *p = vp + (int64_t)(in + 4 * g + r) * a.D;
                    uint32_t w[(VD + 3) / 4], x[8];
                    load_elems<uint8_t, VD, CB>(w, p, m * VD, a.D);
#pragma unroll
                    for (int i = 0; i < (VD + 3) / 4; ++i) decode4<T>(w[i], x + i * (int)sizeof(T));
#pragma unroll
                    for (int i = 0; i < Slice<T, DH>::WORDS; ++i) vv.w[j][i] = x[i];
                    live[j] = ok && kb + stream_of(j, g) < hi;
                }
            }
        } else {
            const T *kp = (const T *)a.k + (int64_t)h * a.D, *vp = (const T *)a.v + (int64_t)h * a.D;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                int key = kb + 16 * t + m;
                key = k0 + (key < hi ? key : hi - 1);
                load_row<T, DH, PB>(kf[t], kp + (int64_t)key * a.ld_k, g, a.D);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                int key = kb + stream_of(j, g);
                live[j] = key < hi;
                key = k0 + (key < hi ? key : hi - 1);
                load_elems<T, VD, PB>(vv.w[j], vp + (int64_t)key * a.ld_v, m * VD, a.D);
                if (a.mask) live[j] = live[j] && a.mask[key] != 0;
            }
        }
        float s[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int f = 0; f < NF; ++f) x = mma<T>(kf[t][f], qf[f], x);
            const float ct = PAGED ? c * sk[t] : c;
#pragma unroll
            for (int r = 0; r < 4; ++r) s[4 * t + r] = live[4 * t + r] ? x[r] * ct : kNegInf;
        }
        float tm = s[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) tm = fmaxf(tm, s[j]);
        tm = max_groups(tm);
        const float mn = fmaxf(mx, tm), base = mn == kNegInf ? 0.f : mn;
        const float alpha = __builtin_amdgcn_exp2f(mx - base);
        mx = mn;
        float p[8], ps = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            p[j] = __builtin_amdgcn_exp2f(s[j] - base);
            ps += p[j];
        }
        l = l * alpha + ps;
        if (ams_ballot(alpha != 1.f)) {
#pragma unroll
            for (int t = 0; t < VD; ++t) acc[t] *= alpha;
        }
        bool all = true;
#pragma unroll
        for (int j = 0; j < 8; ++j) all = all && live[j];
        if (ams_ballot(!all)) {                      // what a masked value holds (NaN too) must not count
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (!live[j]) vv.zero(j);
        }
        if constexpr (PAGED) {
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = live[j] ? p[j] * sv[j >> 2] : 0.f;      // a power of two: exact
        }
        mma_slice<T, DH>(acc, vv, Stream<T>(p));
    }

    // join the four waves
    l = sum_groups(l);
    float o[4 * VD];
    acc_in_order<VD>(acc, 1.f, o);
#pragma unroll
    for (int i = 0; i < 4 * VD; ++i) s_o[wave][m][4 * g * VD + i] = o[i];
    if (g == 0) {
        s_m[wave][m] = mx;
        s_l[wave][m] = l;
    }
    __syncthreads();
    const int r = threadIdx.x / 16, d = (threadIdx.x % 16) * VD;
    const int64_t ro = rows.first + r;
    if (ro >= R) return;
    float M = kNegInf, L = 0.f, y[VD];
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) M = fmaxf(M, s_m[w][r]);
    const float base = M == kNegInf ? 0.f : M;
#pragma unroll
    for (int e = 0; e < VD; ++e) y[e] = 0.f;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(s_m[w][r] - base);
        L += s_l[w][r] * f;
#pragma unroll
        for (int e = 0; e < VD; ++e) y[e] += s_o[w][r][d + e] * f;
    }
    const Row ow = row_at(a, rows.begin, h, (int)ro);
    const int64_t at = ow.query * a.H + ow.head;
    if (a.nsplit > 1) {
        const int64_t n_rows = a.n_q * a.H, p = (int64_t)split * n_rows + at;
        if (threadIdx.x % 16 == 0) {
            a.part_ml[2 * p] = M;
            a.part_ml[2 * p + 1] = L;
        }
#pragma unroll
        for (int e = 0; e < VD; ++e)
            if (d + e < a.D) a.part_o[p * a.D + d + e] = y[e];
        return;
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;       // no key: a zero row
#pragma unroll
    for (int e = 0; e < VD; ++e) y[e] *= inv;
    store_elems<T, VD, PB>((T *)a.out + ow.query * a.ld_out + (int64_t)ow.head * a.D, d, a.D, y);
    if (a.lse && threadIdx.x % 16 == 0)
        a.lse[at] = L == 0.f ? kNegInf : (M + __builtin_amdgcn_logf(L)) * kLn2;
}

// The splits of the keys joined: one wave per (query, head).
template <class T>
__global__ __launch_bounds__(kAttnThreads) void attn_join_k(AttnArgs a)
{
    const int lane = ams_lane();
    const int64_t at = (int64_t)blockIdx.x * kAttnWaves + threadIdx.x / AMS_WAVE, n_rows = a.n_q * a.H;
    if (at >= n_rows) return;
    const int64_t query = at / a.H;
    const int head = (int)(at % a.H);
    if (query < clamp_off(a.q_off[0], a.n_q) || query >= clamp_off(a.q_off[a.B], a.n_q)) return;   // no sample's row
    float M = kNegInf;
    for (int s = lane; s < a.nsplit; s += AMS_WAVE) M = fmaxf(M, a.part_ml[2 * (s * n_rows + at)]);
    M = ams_wave_max(M);
    const float base = M == kNegInf ? 0.f : M;
    float L = 0.f, y0 = 0.f, y1 = 0.f;
    const bool in0 = lane < a.D, in1 = lane + AMS_WAVE < a.D;
#pragma unroll 4
    for (int s = 0; s < a.nsplit; ++s) {
        const int64_t p = s * n_rows + at;
        const float f = __builtin_amdgcn_exp2f(a.part_ml[2 * p] - base);
        L += a.part_ml[2 * p + 1] * f;
        if (in0) y0 += a.part_o[p * a.D + lane] * f;
        if (in1) y1 += a.part_o[p * a.D + lane + AMS_WAVE] * f;
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    T *out = (T *)a.out + query * a.ld_out + (int64_t)head * a.D;
    y0 *= inv, y1 *= inv;
    if (in0) store_elems<T, 1, (int)sizeof(T)>(out, lane, a.D, &y0);
    if (in1) store_elems<T, 1, (int)sizeof(T)>(out, lane + AMS_WAVE, a.D, &y1);
    if (a.lse && lane == 0) a.lse[at] = L == 0.f ? kNegInf : (M + __builtin_amdgcn_logf(L)) * kLn2;
}

// ------------------------------------------------------------------- host

constexpr int64_t kAttnMaxBlocks = (1ll << 24) - 1;    // x 256 threads: below the grid's 2^32
constexpr int kAttnMaxDim = 128;

inline ams_status attn_shape(const ams_attn *at)
{
    if (at->dtype != AMS_F32 && at->dtype != AMS_BF16) return AMS_ERR_DTYPE;
    if (at->head_dim < 1 || at->head_dim > kAttnMaxDim || at->n_heads < 1 || at->n_heads > 4096 ||
        at->n_kv_heads < 1 || at->n_heads % at->n_kv_heads)
        return AMS_ERR_DIMS;
    return AMS_OK;
}

// Row tiles of all samples (each sample's own number is not known here).
inline int64_t row_tiles(const ams_attn *at, int32_t B, int64_t n_q)
{
    return (n_q * (at->n_heads / at->n_kv_heads) >> 4) + B;
}

// Splits of the streamed side so that about two blocks per compute unit are
// there: `tiles` are the tiles with work, `steps` the steps of 128 entries
// (one per wave) that a tile's share has on average.  One while there are
// 384 blocks without it; a split keeps two such steps at least, below which
// its partial sums cost more than it saves.
inline int split_count(int64_t tiles, int64_t steps)
{
    if (tiles < 1) tiles = 1;
    if (tiles >= 384) return 1;
    int64_t n = 512 / tiles;
    if (n > steps / 2) n = steps / 2;
    if (n > 256) n = 256;
    return n < 1 ? 1 : (int)n;
}

inline int64_t busy_row_tiles(const ams_attn *at, int32_t B, int64_t n_q)
{
    const int64_t t = (n_q * (at->n_heads / at->n_kv_heads) + 15) / 16, s = n_q < B ? n_q : B;
    return (t > s ? t : s) * at->n_kv_heads;
}

// Widest load (16, 8 or one element's bytes) for which a row's width, its
// stride and its address leave every piece aligned.
inline int piece_bytes(int esize, int32_t D, int n, const int64_t *ld, const void *const *p)
{
    uint64_t all = (uint64_t)D * esize;
    for (int i = 0; i < n; ++i) all |= (uint64_t)(ld[i] * esize) | (uint64_t)(uintptr_t)p[i];
    return !(all & 15) ? 16 : (!(all & 7) && esize < 4 ? 8 : esize);
}

// f(type, padded head width, piece bytes): f32 in 16, 32, 64 or 128, bf16 in 32, 64 or 128.
template <class F> ams_status with_attn(int32_t dtype, int32_t D, int pb, F f)
{
    auto dims = [&](auto t, auto piece) {
        if (D <= 16 && sizeof(t) == 4) return f(t, std::integral_constant<int, sizeof(t) == 4 ? 16 : 32>(), piece);
        if (D <= 32) return f(t, std::integral_constant<int, 32>(), piece);
        if (D <= 64) return f(t, std::integral_constant<int, 64>(), piece);
        return f(t, std::integral_constant<int, 128>(), piece);
    };
    if (dtype == AMS_F32) {
        if (pb == 16) return dims(0.f, std::integral_constant<int, 16>());
        return dims(0.f, std::integral_constant<int, 4>());
    }
    if (pb == 16) return dims((uint16_t)0, std::integral_constant<int, 16>());
    if (pb == 8) return dims((uint16_t)0, std::integral_constant<int, 8>());
    return dims((uint16_t)0, std::integral_constant<int, 2>());
}

inline size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace
