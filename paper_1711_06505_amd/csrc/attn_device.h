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
// registers: short lists are bound by instructions, so a step's addresses are
// one uniform base and lane offsets that do not change from step to step.
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

// Byte offsets of NE elements of a row from element d on, in pieces of at most
// PB bytes (the host picks PB so that every piece is aligned and lies within
// [0, D) or behind it).  A piece behind D is read at d = 0 instead; `in` says
// which pieces are there.
template <class T, int NE, int PB> struct Cols {
    static constexpr int BYTES = NE * (int)sizeof(T), W = BYTES < PB ? BYTES : PB, PE = W / (int)sizeof(T),
                         N = BYTES / W, WORDS = BYTES / 4 > 0 ? BYTES / 4 : 1;
    uint32_t o[N];

    __device__ __forceinline__ Cols() {}
    __device__ __forceinline__ Cols(int d, int D)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = d + i * PE < D ? (uint32_t)((d + i * PE) * (int)sizeof(T)) : 0u;
    }
    __device__ __forceinline__ void load(uint32_t *dst, const char *base, uint32_t row) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const char *p = base + (row + o[i]);
            if constexpr (W == 16) {
                const uint4 v = *(const uint4 *)p;
                dst[4 * i] = v.x, dst[4 * i + 1] = v.y, dst[4 * i + 2] = v.z, dst[4 * i + 3] = v.w;
            } else if constexpr (W == 8) {
                const uint2 v = *(const uint2 *)p;
                dst[2 * i] = v.x, dst[2 * i + 1] = v.y;
            } else if constexpr (W == 4) {
                dst[i] = *(const uint32_t *)p;
            } else {
                constexpr int PER = 4 / W;            // pieces of a word
                const uint32_t v = W == 2 ? (uint32_t)*(const uint16_t *)p : (uint32_t)*(const uint8_t *)p;
                if (i % PER) dst[i / PER] |= v << (8 * W * (i % PER));
                else dst[i / PER] = v;
            }
        }
    }
    // what lies behind D made zero
    __device__ __forceinline__ void mask(uint32_t *w, int d, int D) const
    {
#pragma unroll
        for (int e = 0; e < NE; ++e) {
            if (d + e < D) continue;
            if constexpr (sizeof(T) == 4) w[e] = 0;
            else w[e / 2] &= (e & 1) ? 0xffffu : 0xffff0000u;
        }
    }
};

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
// group g holds the EP elements from (4 c + g) EP on.  Of the two rows of a
// product one is loaded with zeros behind D (`clean`), so that it does not
// matter what the other one reads there (elements of its own row).
template <class T, int DH, int PB> struct RowCols {
    static constexpr int EP = Num<T>::EP, NF = DH / (4 * EP);
    Cols<T, EP, PB> c[NF];
    int d0, D;

    __device__ __forceinline__ RowCols(int g, int D_) : d0(g * EP), D(D_)
    {
#pragma unroll
        for (int f = 0; f < NF; ++f) c[f] = Cols<T, EP, PB>(4 * f * EP + d0, D);
    }
    __device__ __forceinline__ void load(Frag *f, const char *base, uint32_t row) const
    {
#pragma unroll
        for (int i = 0; i < NF; ++i) c[i].load(f[i].u, base, row);
    }
    __device__ __forceinline__ void clean(Frag *f) const
    {
        if (D == DH) return;
#pragma unroll
        for (int i = 0; i < NF; ++i) c[i].mask(f[i].u, 4 * i * EP + d0, D);
    }
};

// Streamed entry j of lane group g within a step of 32 (the order in which
// both products see the streamed side).
__device__ __forceinline__ int stream_of(int j, int g) { return 16 * (j >> 2) + 4 * g + (j & 3); }

// The lane's slice of 8 streamed rows, elements (lane % 16) VD .. + VD of
// each, as raw words: operand of a contraction over the streamed rows.
// (Elements behind D only reach results behind D, which nobody stores.)
template <class T, int DH> struct Slice {
    static constexpr int VD = DH / 16, WORDS = VD * (int)sizeof(T) / 4 > 0 ? VD * (int)sizeof(T) / 4 : 1;
    uint32_t w[8][WORDS];

    // entries not in `live` (bits of stream_of's order): whatever they hold (NaN too) must not count
    __device__ __forceinline__ void keep(uint32_t live, int g)
    {
        live >>= 4 * g;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!(live >> stream_of(j, 0) & 1)) zero(j);
    }

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

// acc[t] += slice tile t times the stream, over all VD tiles.  HALF: the stream's
// second 16 entries are zero (float has an instruction group for each half).
template <class T, int DH, bool HALF = false>
__device__ __forceinline__ void mma_slice(f32x4 *acc, const Slice<T, DH> &s, const Stream<T> &p)
{
#pragma unroll
    for (int t = 0; t < Slice<T, DH>::VD; ++t) {
        Frag f[Num<T>::SF];
        s.frags(t, f);
#pragma unroll
        for (int i = 0; i < (HALF && sizeof(T) == 4 ? 1 : 2); ++i)
            acc[t] = mma<T>(f[sizeof(T) == 4 ? i : 0], p.f[i], acc[t]);
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
    int64_t tiles;                    // of the grid, per key head and split
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
    int32_t few_rows;                 // samples of at most so many rows are attn_bwd_few_k's (-1: none)
    int32_t *any_many;                // whether there are others
    int64_t blocks;                   // of the whole work, where a grid may be smaller
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

// Which of the 32 entries from `at` on are there: below `end` and, with a
// mask, kept by it (a bit each, the same in all lanes).
__device__ __forceinline__ uint32_t live_bits(int at, int end, const uint8_t *mask)
{
    const int e = at + (ams_lane() & (kKeyTile - 1));
    bool on = e < end;
    if (mask) on = on && mask[on ? e : at] != 0;
    return (uint32_t)ams_ballot(on);
}

// Two waves per SIMD where their registers come to 256 or nearly.
template <class T, int DH, int RT> constexpr int waves_per_simd()
{
    return DH * RT * (int)sizeof(T) <= 256 ? 2 : 1;
}

// The lane's place in a list of rows: tile, key head and split of wave or block `b`.
struct Work {
    int split, h;
    int64_t tile;
};
__device__ __forceinline__ Work work_of(int64_t at, const AttnArgs &a)
{
    uint32_t b = (uint32_t)at;                         // below 4 kAttnMaxBlocks
    Work w;
    w.split = (int)(b % (uint32_t)a.nsplit);
    b /= (uint32_t)a.nsplit;
    w.h = (int)(b % (uint32_t)a.Hk);
    w.tile = b / (uint32_t)a.Hk;
    return w;
}

// ---------------------------------------------------------------- forward

// One tile of 16 RT rows per (row tile, key head, split of the keys), by WK
// waves: with WK = 4 the waves of a block take every fourth step of 32 keys
// and are joined at the end, with WK = 1 each wave has a tile of its own.
template <class T, int DH, int PB, bool PAGED, int RT, int WK>
__global__ __launch_bounds__(kAttnThreads, (waves_per_simd<T, DH, RT>())) void attn_fwd_k(AttnArgs a)
{
    constexpr int NF = DH / (4 * Num<T>::EP), VD = DH / 16, ES = (int)sizeof(T);
    constexpr int CB = PB / ES;                       // codes of a piece: as many as elements
    constexpr int kRows = kRowTile * RT, kTileShift = RT == 2 ? 5 : 4, kPad = DH + 4;
    __shared__ float s_o[WK > 1 ? WK : 1][WK > 1 ? kRows : 1][kPad];
    __shared__ float s_m[WK > 1 ? WK : 1][kRows], s_l[WK > 1 ? WK : 1][kRows];
    const int lane = ams_lane(), m = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE);
    const Work wk = work_of(WK == 1 ? (int64_t)blockIdx.x * kAttnWaves + wave : blockIdx.x, a);
    const int h = wk.h;
    if (wk.tile >= a.tiles) return;
    const Span rows = span_of(a.q_off, a.B, a.n_q, a.G, kTileShift, wk.tile);
    const int64_t R = (int64_t)rows.count * a.G;
    if (rows.first < 0 || rows.first >= R) return;

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
    split_range(nk, wk.split, a.nsplit, lo, hi);

    const RowCols<T, DH, PB> rc(g, a.D);
    Frag qf[RT][NF];
    Row row[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int64_t r = rows.first + 16 * t + m;
        row[t] = row_at(a, rows.begin, h, (int)(r < R ? r : R - 1));
        rc.load(qf[t], (const char *)a.q + (row[t].query * a.ld_q + (int64_t)row[t].head * a.D) * ES, 0);
    }
    const float c = a.scale * kLog2e;
    f32x4 acc[RT][VD];
    float mx[RT], l[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int i = 0; i < VD; ++i) acc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        mx[t] = kNegInf;
        l[t] = 0.f;
    }
    // lane offsets of a step
    const uint32_t ldk = PAGED ? (uint32_t)a.D : (uint32_t)(a.ld_k * ES);
    const uint32_t ldv = PAGED ? (uint32_t)a.D : (uint32_t)(a.ld_v * ES);
    uint32_t krow[2] = {m * ldk, (16 + m) * ldk}, vrow[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) vrow[j] = (uint32_t)(PAGED ? 4 * g + (j & 3) : stream_of(j, g)) * ldv;
    const Cols<T, VD, PB> vcol(m * VD, a.D);
    Cols<uint8_t, Num<T>::EP, CB> kc[PAGED ? NF : 1];
    const Cols<uint8_t, VD, CB> vc(m * VD, a.D);
    if constexpr (PAGED) {
#pragma unroll
        for (int f = 0; f < NF; ++f) kc[f] = Cols<uint8_t, Num<T>::EP, CB>((4 * f + g) * Num<T>::EP, a.D);
    }

    // A step's loads, issued a step ahead of their use: behind the last step the
    // last one's are read again, so that their number never changes.
    constexpr int kStep = WK * kKeyTile;
    struct Raw {
        Frag kf[PAGED ? 1 : 2][PAGED ? 1 : NF];
        Slice<T, DH> vv;
        uint32_t kw[2][PAGED ? NF : 1][Num<T>::EP / 4], vw[2][4][(VD + 3) / 4];
        float sk[2], sv[2];
        uint32_t there;                               // dense: the lane's mask byte; paged: which halves have a page
    };
    auto pages_of = [&](int kb, int *page) {
        if constexpr (PAGED) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
                // 16 consecutive tokens lie in one page; a step's second half behind the last reads the first half's page
                page[t] = pages[(kb + 16 * t < hi ? kb + 16 * t : kb) >> a.page_shift];
        }
    };
    auto issue = [&](Raw &x, int kb, const int *page) {
        if constexpr (PAGED) {
            x.there = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int tok = kb + 16 * t < hi ? kb + 16 * t : kb;
                const bool ok = page[t] >= 0 && page[t] < a.n_pages;
                x.there |= ok ? 0xffffu << (16 * t) : 0u;
                const int64_t at = (int64_t)(ok ? page[t] : 0) * a.Hk + h;
                x.sk[t] = a.ks[at];
                x.sv[t] = a.vs[at];
                const int64_t first = ((at << a.page_shift) + (tok & ((1 << a.page_shift) - 1))) * a.D;
                const char *kp = (const char *)a.kc + first, *vp = (const char *)a.vc + first;
#pragma unroll
                for (int f = 0; f < NF; ++f) kc[f].load(x.kw[t][f], kp, krow[0]);
#pragma unroll
                for (int r = 0; r < 4; ++r) vc.load(x.vw[t][r], vp, vrow[r]);
            }
        } else {
            if (kb + kKeyTile > hi) {                 // the last step: what lies behind it reads the last key
                const int last = hi - 1 - kb;
#pragma unroll
                for (int t = 0; t < 2; ++t) krow[t] = (uint32_t)min(16 * t + m, last) * ldk;
#pragma unroll
                for (int j = 0; j < 8; ++j) vrow[j] = (uint32_t)min(stream_of(j, g), last) * ldv;
            }
            const char *kp = (const char *)a.k + ((int64_t)(k0 + kb) * a.ld_k + (int64_t)h * a.D) * ES;
            const char *vp = (const char *)a.v + ((int64_t)(k0 + kb) * a.ld_v + (int64_t)h * a.D) * ES;
#pragma unroll
            for (int t = 0; t < 2; ++t) rc.load(x.kf[t], kp, krow[t]);
#pragma unroll
            for (int j = 0; j < 8; ++j) vcol.load(x.vv.w[j], vp, vrow[j]);
            x.there = 1;
            if (a.mask) x.there = a.mask[k0 + min(kb + (lane & (kKeyTile - 1)), hi - 1)];
        }
    };
    auto step = [&](Raw &x, int kb) {
        Frag pf[2][NF];
        uint32_t live = (uint32_t)ams_ballot(kb + (lane & (kKeyTile - 1)) < hi && (PAGED || x.there != 0));
        if constexpr (PAGED) {
            live &= x.there;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int i = 0; i < Num<T>::EP / 4; ++i) decode4<T>(x.kw[t][f][i], pf[t][f].u + i * ES);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    uint32_t y[8];
#pragma unroll
                    for (int i = 0; i < (VD + 3) / 4; ++i) decode4<T>(x.vw[t][r][i], y + i * ES);
#pragma unroll
                    for (int i = 0; i < Slice<T, DH>::WORDS; ++i) x.vv.w[4 * t + r][i] = y[i];
                }
            }
        }
        const Frag(*kf)[NF];
        if constexpr (PAGED) kf = pf;
        else kf = x.kf;
        Slice<T, DH> &vv = x.vv;
        if (live != 0xffffffffu) vv.keep(live, g);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float s[8];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int f = 0; f < NF; ++f) y = mma<T>(kf[t][f], qf[rt][f], y);
                const float ct = PAGED ? c * x.sk[t] : c;
#pragma unroll
                for (int r = 0; r < 4; ++r) s[4 * t + r] = y[r] * ct;
            }
            if (live != 0xffffffffu) {
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] = (live >> (4 * g + stream_of(j, 0)) & 1) ? s[j] : kNegInf;
            }
            float tm = s[0];
#pragma unroll
            for (int j = 1; j < 8; ++j) tm = fmaxf(tm, s[j]);
            tm = max_groups(tm);
            const float mn = fmaxf(mx[rt], tm), base = mn == kNegInf ? 0.f : mn;
            const float alpha = __builtin_amdgcn_exp2f(mx[rt] - base);
            mx[rt] = mn;
            float p[8], ps = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                p[j] = __builtin_amdgcn_exp2f(s[j] - base);
                ps += p[j];
            }
            l[rt] = l[rt] * alpha + ps;
            if (ams_ballot(alpha != 1.f)) {
#pragma unroll
                for (int i = 0; i < VD; ++i) acc[rt][i] *= alpha;
            }
            if constexpr (PAGED) {
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] = p[j] == 0.f ? 0.f : p[j] * x.sv[j >> 2];    // a power of two: exact
            }
            mma_slice<T, DH>(acc[rt], vv, Stream<T>(p));
        }
    };
    int kb = lo + (WK == 1 ? 0 : wave * kKeyTile);
    if (kb < hi) {
        Raw now, then;
        int page[2] = {0, 0};
        pages_of(kb, page);
        issue(now, kb, page);
        int next = kb + kStep < hi ? kb + kStep : kb;
        pages_of(next, page);
#pragma unroll
        for (int t = 0; t < RT; ++t) rc.clean(qf[t]);      // waits for the queries, behind the first keys' loads
        for (;;) {
            issue(then, next, page);
            const int after = next + kStep < hi ? next + kStep : next;
            pages_of(after, page);
            step(now, kb);
            if (next == kb) break;
            kb = next, next = after;
            now = then;
        }
    }

#pragma unroll
    for (int t = 0; t < RT; ++t) l[t] = sum_groups(l[t]);
    if constexpr (WK == 1) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            if (rows.first + 16 * t + m >= R) continue;
            const int64_t at = row[t].query * a.H + row[t].head;
            float o[4 * VD];                          // one split where a wave has a tile of its own
            acc_in_order<VD>(acc[t], l[t] == 0.f ? 0.f : 1.f / l[t], o);          // no key: a zero row
            store_elems<T, 4 * VD, PB>((T *)a.out + row[t].query * a.ld_out + (int64_t)row[t].head * a.D, 4 * g * VD,
                                       a.D, o);
            if (a.lse && g == 0) a.lse[at] = l[t] == 0.f ? kNegInf : (mx[t] + __builtin_amdgcn_logf(l[t])) * kLn2;
        }
        return;
    }
    // join the four waves
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        float o[4 * VD];
        acc_in_order<VD>(acc[t], 1.f, o);
#pragma unroll
        for (int i = 0; i < 4 * VD; ++i) s_o[wave % WK][(16 * t + m) % (WK > 1 ? kRows : 1)][4 * g * VD + i] = o[i];
        if (g == 0) {
            s_m[wave % WK][16 * t + m] = mx[t];
            s_l[wave % WK][16 * t + m] = l[t];
        }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int r = 16 * t + threadIdx.x / 16, d = (threadIdx.x % 16) * VD;
        const int64_t ro = rows.first + r;
        if (ro >= R) return;
        float M = kNegInf, L = 0.f, y[VD];
#pragma unroll
        for (int w = 0; w < WK; ++w) M = fmaxf(M, s_m[w][r]);
        const float base = M == kNegInf ? 0.f : M;
#pragma unroll
        for (int e = 0; e < VD; ++e) y[e] = 0.f;
#pragma unroll
        for (int w = 0; w < WK; ++w) {
            const float f = __builtin_amdgcn_exp2f(s_m[w][r] - base);
            L += s_l[w][r] * f;
#pragma unroll
            for (int e = 0; e < VD; ++e) y[e] += s_o[w][r % (WK > 1 ? kRows : 1)][d + e] * f;
        }
        const Row ow = row_at(a, rows.begin, h, (int)ro);
        const int64_t at = ow.query * a.H + ow.head;
        if (a.nsplit > 1) {
            const int64_t p = (int64_t)wk.split * (a.n_q * a.H) + at;
            if (threadIdx.x % 16 == 0) {
                a.part_ml[2 * p] = M;
                a.part_ml[2 * p + 1] = L;
            }
#pragma unroll
            for (int e = 0; e < VD; ++e)
                if (d + e < a.D) a.part_o[p * a.D + d + e] = y[e];
            continue;
        }
        const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
        for (int e = 0; e < VD; ++e) y[e] *= inv;
        store_elems<T, VD, PB>((T *)a.out + ow.query * a.ld_out + (int64_t)ow.head * a.D, d, a.D, y);
        if (a.lse && threadIdx.x % 16 == 0)
            a.lse[at] = L == 0.f ? kNegInf : (M + __builtin_amdgcn_logf(L)) * kLn2;
    }
}

// The splits of the keys joined: one block per (query, head), or four of them
// with a wave each (W = 1) where the splits are few.
template <class T, int W>
__global__ __launch_bounds__(kAttnThreads) void attn_join_k(AttnArgs a)
{
    __shared__ float s_y[W][2 * AMS_WAVE], s_l[W];
    const int lane = ams_lane(), wave = threadIdx.x / AMS_WAVE;
    const int64_t at = W == 1 ? (int64_t)blockIdx.x * kAttnWaves + wave : blockIdx.x, n_rows = a.n_q * a.H;
    if (at >= n_rows) return;
    const int64_t query = at / a.H;
    const int head = (int)(at - query * a.H);
    if (query < clamp_off(a.q_off[0], a.n_q) || query >= clamp_off(a.q_off[a.B], a.n_q)) return;   // no sample's row
    float M = kNegInf;
    for (int s = lane; s < a.nsplit; s += AMS_WAVE) M = fmaxf(M, a.part_ml[2 * (s * n_rows + at)]);
    M = ams_wave_max(M);
    const float base = M == kNegInf ? 0.f : M;
    float L = 0.f, y0 = 0.f, y1 = 0.f;
    const int d0 = lane < a.D ? lane : 0, d1 = lane + AMS_WAVE < a.D ? lane + AMS_WAVE : 0;
#pragma unroll 8
    for (int s = W == 1 ? 0 : wave; s < a.nsplit; s += W) {
        const int64_t p = s * n_rows + at;
        const float m = a.part_ml[2 * p], l = a.part_ml[2 * p + 1];
        const float x0 = a.part_o[p * a.D + d0], x1 = a.part_o[p * a.D + d1];
        const float f = __builtin_amdgcn_exp2f(m - base);
        L += l * f;
        y0 += x0 * f;
        y1 += x1 * f;
    }
    if constexpr (W > 1) {
        s_y[wave][lane] = y0;
        s_y[wave][AMS_WAVE + lane] = y1;
        if (lane == 0) s_l[wave] = L;
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int w = 1; w < W; ++w) {
            y0 += s_y[w][lane];
            y1 += s_y[w][AMS_WAVE + lane];
            L += s_l[w];
        }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    T *out = (T *)a.out + query * a.ld_out + (int64_t)head * a.D;
    y0 *= inv, y1 *= inv;
    if (lane < a.D) store_elems<T, 1, (int)sizeof(T)>(out, lane, a.D, &y0);
    if (lane + AMS_WAVE < a.D) store_elems<T, 1, (int)sizeof(T)>(out, lane + AMS_WAVE, a.D, &y1);
    if (a.lse && lane == 0) a.lse[at] = L == 0.f ? kNegInf : (M + __builtin_amdgcn_logf(L)) * kLn2;
}

template <class T> void launch_join(const char *name, const AttnArgs &a, hipStream_t st)
{
    const int64_t n = a.n_q * a.H;
    if (a.nsplit >= 8)
        AMS_LAUNCH(name, st, attn_join_k<T, kAttnWaves><<<(unsigned)n, kAttnThreads, 0, st>>>(a));
    else
        AMS_LAUNCH(name, st,
                   attn_join_k<T, 1><<<(unsigned)((n + kAttnWaves - 1) / kAttnWaves), kAttnThreads, 0, st>>>(a));
}

// ------------------------------------------------------------------- host

constexpr int64_t kAttnMaxBlocks = (1ll << 24) - 1;    // x 256 threads: below the grid's 2^32
constexpr int kAttnMaxDim = 128;
constexpr int64_t kAttnMaxEntries = 1 << 30;           // rows or keys: a step past the last one still fits 32 bits

inline ams_status attn_shape(const ams_attn *at)
{
    if (at->dtype != AMS_F32 && at->dtype != AMS_BF16) return AMS_ERR_DTYPE;
    if (at->head_dim < 1 || at->head_dim > kAttnMaxDim || at->n_heads < 1 || at->n_heads > 4096 ||
        at->n_kv_heads < 1 || at->n_heads % at->n_kv_heads)
        return AMS_ERR_DIMS;
    return AMS_OK;
}

constexpr int64_t kAttnMaxStride = 1 << 24;            // 32 rows' bytes fit the lanes' 32-bit offsets

// How a forward call (or dQ's) is cut.
struct Cut {
    int rt, wk, nsplit;
    int64_t tiles, blocks;
};

// Tiles of `rows` streamed against per sample: floor(n / size) + B of them are
// launched (each sample's own number is not known here).
inline int64_t tiles_of(int64_t n, int shift, int32_t B) { return (n >> shift) + B; }

// Splits of the streamed side when `tiles` blocks have work and a list has
// `entries` (over pages: room for them, which a sample may fill less): two blocks
// per compute unit while a split keeps 256 entries (two steps of the block; below
// that its partial sums cost more than it saves), four where each of them keeps
// 1200.  Numbers between the two leave units idle at the end.  Us with two and
// four a unit, at so many entries for each of the four: 8 users of 8,000..16,000
// 8-bit tokens, 8 key heads of 128, 48 and 50 at 1000 (61 at 10 splits between), 32 of
// 512..4096 51 and 55 at 1024; one query over 40,000 float32 keys, 8 samples, 4 heads of 64,
// 145 and 134 at 1250, over 60,000 bf16 keys, 3 samples, 8 heads of 128, 152 and 139 at
// 1430, over 80,000 188 and 170 at 1900.
inline int split_count(int64_t tiles, int64_t entries)
{
    if (tiles < 1) tiles = 1;
    const int64_t four = 1024 / tiles, two = 512 / tiles < entries / 256 ? 512 / tiles : entries / 256;
    const int64_t n = four > two && entries / 1200 >= four ? four : two;
    return n < 1 ? 1 : (n > 256 ? 256 : (int)n);
}

// rows: all samples' rows of one key head; keys: a sample's (on average).
// Two row tiles per wave once a sample has more than one on average (the keys
// are read and unpacked once for both), where the registers allow it.
inline Cut cut_rows(const ams_attn *at, int32_t B, int64_t n_q, int64_t keys, bool wide)
{
    const int64_t rows = n_q * (at->n_heads / at->n_kv_heads), Hk = at->n_kv_heads;
    const int64_t samples = B < 1 ? 1 : B;
    Cut c;
    c.rt = wide && rows > 16 * samples && (at->dtype == AMS_BF16 || at->head_dim <= 64) ? 2 : 1;
    const int shift = c.rt == 2 ? 5 : 4;
    c.tiles = tiles_of(rows, shift, B);
    int64_t busy = (rows + (1 << shift) - 1) >> shift;
    const int64_t with_rows = n_q < B ? n_q : B;
    busy = (busy > with_rows ? busy : with_rows) * Hk;
    // short lists and many of them: a wave per tile, nothing to join.  One query a sample, 4 heads, us with one wave and
    // with four: 1024 samples of 60 keys 12 and 18 (float32, 16 wide), 18 and 26 (bf16, 64 wide), of 250 29 and 42,
    // 48 and 48, of 500 54 and 81, 108 and 103; 512 samples of 250 keys 21 and 25, 33 and 28.
    c.wk = keys <= 256 && busy >= 1024 ? 1 : 4;
    c.nsplit = c.wk == 1 ? 1 : split_count(busy, keys);
    const int64_t work = c.tiles * Hk * c.nsplit;
    c.blocks = c.wk == 1 ? (work + kAttnWaves - 1) / kAttnWaves : work;
    return c;
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

// f(RT, WK): two row tiles only in the widest pieces, and not for 128 floats
// (whose operands alone would fill the registers).
template <class T, int DH, int PB, class F> ams_status with_cut(const Cut &c, F f)
{
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    using Four = std::integral_constant<int, 4>;
    if constexpr (PB == 16 && (sizeof(T) == 2 || DH <= 64)) {
        if (c.rt == 2) return c.wk == 1 ? f(Two(), One()) : f(Two(), Four());
    }
    return c.wk == 1 ? f(One(), One()) : f(One(), Four());
}

inline size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace
