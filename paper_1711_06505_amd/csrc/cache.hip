// cache.hip -- keys and values kept in 8-bit pages, and attention over them.
//   ams_cache_write  new tokens' keys and values into their samples' pages
//   ams_cache_attn   attention of each sample's queries to its cached tokens
//                    (attn_device.h's forward, with pages as the streamed side)
// A page holds 16 to 128 tokens of one sample; for each of its key heads the
// tokens' D values lie together as OCP e4m3 codes with one scale.  Scales are
// powers of two: a code times its scale, the division by a scale and the
// change of a page's scale are then exact but for the one rounding to 4
// significant bits, at the price of up to one bit of the 8-bit range.  Codes
// are exact in bf16, so the score product runs on them as they are and takes
// the page's scale afterwards; the value scale goes onto the weights.
#include "attn_device.h"
#include "attn_many.h"

namespace {

constexpr float kCodeMax = 448.f;                     // largest e4m3 value, 1.75 2^8
constexpr int kMinExp = -100;                         // of a scale: 2^kMinExp and its inverse are normal

// N (4 or 1) elements of a row, as they lie there and as floats.
template <class T, int N> struct Elems {
    typedef typename std::conditional<N == 1, T, typename std::conditional<sizeof(T) == 4, uint4, uint2>::type>::type raw;
    raw r;

    __device__ __forceinline__ void load(const T *p) { r = *(const raw *)p; }
    __device__ __forceinline__ void floats(float *x) const
    {
        if constexpr (N == 1) {
            if constexpr (sizeof(T) == 4) x[0] = r;
            else x[0] = ams_bf16_to_f32(r);
        } else if constexpr (sizeof(T) == 4) {
            x[0] = __uint_as_float(r.x), x[1] = __uint_as_float(r.y);
            x[2] = __uint_as_float(r.z), x[3] = __uint_as_float(r.w);
        } else {
            x[0] = __uint_as_float(r.x << 16), x[1] = __uint_as_float(r.x & 0xffff0000u);
            x[2] = __uint_as_float(r.y << 16), x[3] = __uint_as_float(r.y & 0xffff0000u);
        }
    }
};

// Round to e4m3, ties to even; beyond the largest value: that value (infinities too), NaN stays NaN.
__device__ __forceinline__ float into_range(float x)
{
    return x > kCodeMax ? kCodeMax : (x < -kCodeMax ? -kCodeMax : x);
}
template <int N> __device__ __forceinline__ void store_codes(uint8_t *dst, const float *x)
{
    if constexpr (N == 4) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(into_range(x[0]), into_range(x[1]), 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(into_range(x[2]), into_range(x[3]), w, true);
        *(uint32_t *)dst = (uint32_t)w;
    } else {
        *dst = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(into_range(x[0]), 0.f, 0, false);
    }
}

// Exponent of the least power of two 2^e, e >= kMinExp, with 448 2^e >= the
// magnitude whose bits these are (finite).
__device__ __forceinline__ int scale_exp(uint32_t bits)
{
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e > kMinExp ? e : kMinExp;
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

struct WriteArgs {
    int32_t B, Hk, D, max_pages, page_shift;
    int64_t n_pages, n_new, tiles;
    const int32_t *new_off, *start, *page_table;
    const void *x[2];
    int64_t ld[2];
    uint8_t *codes[2];
    float *scale[2];
    int32_t *status;
};

// One wave per (page that a sample's new tokens touch, key head, keys or
// values): the new tokens' largest magnitude, the page's scale, the codes
// that were there in the new scale where it grew, the new codes.  Bound by
// memory: the new rows stay in registers between the two, up to kHold pieces a
// lane (1024 pieces of 4 entries); a larger page's are read again.
constexpr int kHold = 16;
template <class T, int N>
__global__ __launch_bounds__(kAttnThreads) void cache_write_k(WriteArgs a)
{
    const int lane = ams_lane();
    uint32_t w = blockIdx.x * kAttnWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / AMS_WAVE);     // below 2^26
    if (w >= a.tiles * a.Hk * 2) return;
    const int kv = (int)(w & 1);
    w >>= 1;
    const int h = (int)(w % (uint32_t)a.Hk);
    const int64_t tile = w / (uint32_t)a.Hk;
    const int i = find_sample(a.new_off, a.B, a.n_new, 1, a.page_shift, 2, tile);
    const int n0 = clamp_off(a.new_off[i], a.n_new), n1 = clamp_off(a.new_off[i + 1], a.n_new);
    const int64_t start = a.start[i], P = 1ll << a.page_shift;
    const int64_t nth = tile - ((n0 >> a.page_shift) + 2ll * i);
    const int64_t pi = (start >> a.page_shift) + nth;           // page of the sample
    const int64_t lo = start > pi * P ? start : pi * P;
    const int64_t end = start + (n1 - n0), hi = end < (pi + 1) * P ? end : (pi + 1) * P;
    if (nth < 0 || lo >= hi) return;
    const int page = start < 0 || pi >= a.max_pages ? -1 : a.page_table[(int64_t)i * a.max_pages + pi];
    if (page < 0 || page >= a.n_pages) {                        // nowhere to put them: said, not written
        if (a.status && lane == 0) *a.status = AMS_ERR_ID_RANGE;
        return;
    }
    const int rows = (int)(hi - lo), in = (int)(lo - pi * P), per = a.D / N, units = rows * per;
    const T *x = (const T *)a.x[kv] + (n0 + (lo - start)) * a.ld[kv] + (int64_t)h * a.D;
    auto load = [&](Elems<T, N> &v, int u) {
        const int r = u / per, c = u - r * per;
        v.load(x + r * a.ld[kv] + c * N);
    };
    uint32_t most = 0;
    auto look = [&](const Elems<T, N> &e) {
        float v[N];
        e.floats(v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
            most = b < 0x7f800000u && b > most ? b : most;      // an infinity saturates, NaN stays
        }
    };
    const bool held = units <= kHold * AMS_WAVE;
    Elems<T, N> hold[kHold];
    if (held) {
#pragma unroll
        for (int i = 0; i < kHold; ++i)
            if (i * AMS_WAVE < units) load(hold[i], min(i * AMS_WAVE + lane, units - 1));
#pragma unroll
        for (int i = 0; i < kHold; ++i)
            if (i * AMS_WAVE < units) look(hold[i]);
    } else {
#pragma unroll 4
        for (int u = lane; u < units; u += AMS_WAVE) {
            Elems<T, N> v;
            load(v, u);
            look(v);
        }
    }
#pragma unroll
    for (int o = AMS_WAVE / 2; o > 0; o >>= 1) {
        const uint32_t y = __shfl_xor(most, o, AMS_WAVE);
        most = y > most ? y : most;
    }
    const int64_t at = (int64_t)page * a.Hk + h;
    uint8_t *codes = a.codes[kv] + (at << a.page_shift) * a.D;
    float s = pow2(scale_exp(most));
    if (in > 0) {                                               // tokens of before in this page
        const float old = a.scale[kv][at];
        if (old < s) {
            const float f = old / s;
            for (int u = lane; u < in * per; u += AMS_WAVE) {
                float v[N];
                if constexpr (N == 4) {
                    uint32_t d[4];
                    decode4<float>(*(const uint32_t *)(codes + u * 4), d);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(d[e]) * f;
                } else {
                    uint32_t d[4];
                    decode4<float>(codes[u], d);
                    v[0] = __uint_as_float(d[0]) * f;
                }
                store_codes<N>(codes + (int64_t)u * N, v);
            }
        } else {
            s = old;
        }
    }
    if (lane == 0) a.scale[kv][at] = s;
    const float f = 1.f / s;
    codes += (int64_t)in * a.D;
    auto put = [&](const Elems<T, N> &e, int u) {
        float v[N];
        e.floats(v);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= f;
        store_codes<N>(codes + (int64_t)u * N, v);
    };
    if (held) {
#pragma unroll
        for (int i = 0; i < kHold; ++i)
            if (i * AMS_WAVE + lane < units) put(hold[i], i * AMS_WAVE + lane);
    } else {
#pragma unroll 4
        for (int u = lane; u < units; u += AMS_WAVE) {
            Elems<T, N> v;
            load(v, u);
            put(v, u);
        }
    }
}

// ------------------------------------------------------------------- host

ams_status cache_shape(const ams_cache *c, int &page_shift)
{
    page_shift = 0;
    while (page_shift < 7 && (1 << page_shift) < c->page) ++page_shift;
    if (c->n_kv_heads < 1 || c->n_kv_heads > 4096 || c->head_dim < 1 || c->head_dim > kAttnMaxDim || c->page < 16 ||
        (1 << page_shift) != c->page)
        return AMS_ERR_DIMS;
    if (c->max_pages < 1 || c->n_pages < 1 || c->n_pages > INT32_MAX ||
        (int64_t)c->max_pages * c->page > kAttnMaxEntries)
        return AMS_ERR_SIZE;
    return AMS_OK;
}

// many: attn_many.h's kernel, which reads 16 codes at a time (`wide` for both: 16-byte pieces of the rows)
ams_status read_plan(const ams_attn *at, const ams_cache *c, int32_t B, int64_t n_q, bool wide, bool codes16, Cut &cut,
                     bool &many, size_t &total)
{
    ams_status s = attn_shape(at);
    int shift;
    if (s == AMS_OK) s = cache_shape(c, shift);
    if (s != AMS_OK) return s;
    if (at->n_kv_heads != c->n_kv_heads || at->head_dim != c->head_dim) return AMS_ERR_DIMS;
    if (B < 0 || n_q < 0 || n_q > kAttnMaxEntries || n_q * (at->n_heads / at->n_kv_heads) > kAttnMaxEntries)
        return AMS_ERR_SIZE;
    cut = cut_rows(at, B, n_q, (int64_t)c->max_pages * c->page, wide);
    // (128 samples of 2000..4000 tokens, 2 key heads of 128, 4 query heads each: 178 us at 80 rows against 183 with
    // it, 336 at 160 rows against 198; 64 wide: 102 against 127 and 159 against 135)
    many = wide && codes16 && at->dtype == AMS_BF16 && at->head_dim % 16 == 0 &&
           cut_many(at, B, n_q, (int64_t)c->max_pages * c->page, 96, cut);
    if (cut.blocks > kAttnMaxBlocks) return AMS_ERR_SIZE;
    const size_t rows = (size_t)n_q * at->n_heads;
    total = 256;
    if (cut.nsplit > 1)
        total += align_up(cut.nsplit * rows * 2 * sizeof(float)) + cut.nsplit * rows * at->head_dim * sizeof(float);
    return AMS_OK;
}

}  // namespace

extern "C" ams_status ams_cache_write(const ams_cache *cache, int32_t dtype, int32_t B, const int32_t *new_off,
                                      int64_t n_new, const int32_t *start, const int32_t *page_table, const void *k,
                                      int64_t ld_k, const void *v, int64_t ld_v, uint8_t *k_codes, float *k_scale,
                                      uint8_t *v_codes, float *v_scale, int32_t *dev_status, void *stream)
{
    if (!cache) return AMS_ERR_NULL;
    if (dtype != AMS_F32 && dtype != AMS_BF16) return AMS_ERR_DTYPE;
    WriteArgs a{};
    const ams_status s = cache_shape(cache, a.page_shift);
    if (s != AMS_OK) return s;
    const int64_t w = (int64_t)cache->n_kv_heads * cache->head_dim;
    if (B < 0 || n_new < 0 || n_new > kAttnMaxEntries || ld_k < w || ld_v < w) return AMS_ERR_SIZE;
    a.tiles = (n_new >> a.page_shift) + 2ll * B;
    const int64_t waves = a.tiles * cache->n_kv_heads * 2, blocks = (waves + kAttnWaves - 1) / kAttnWaves;
    if (blocks > kAttnMaxBlocks) return AMS_ERR_SIZE;
    if (B == 0 || n_new == 0) return AMS_OK;
    if (!new_off || !start || !page_table || !k || !v || !k_codes || !k_scale || !v_codes || !v_scale)
        return AMS_ERR_NULL;
    a.B = B, a.Hk = cache->n_kv_heads, a.D = cache->head_dim, a.max_pages = cache->max_pages;
    a.n_pages = cache->n_pages, a.n_new = n_new;
    a.new_off = new_off, a.start = start, a.page_table = page_table;
    a.x[0] = k, a.x[1] = v, a.ld[0] = ld_k, a.ld[1] = ld_v;
    a.codes[0] = k_codes, a.codes[1] = v_codes, a.scale[0] = k_scale, a.scale[1] = v_scale;
    a.status = dev_status;
    hipStream_t st = (hipStream_t)stream;
    const int es = dtype == AMS_F32 ? 4 : 2;
    const uint64_t rows = (uint64_t)(uintptr_t)k | (uint64_t)(uintptr_t)v | (uint64_t)(ld_k * es) | (uint64_t)(ld_v * es);
    const uint64_t codes = (uint64_t)(uintptr_t)k_codes | (uint64_t)(uintptr_t)v_codes;
    const bool four = a.D % 4 == 0 && !(rows & (4 * es - 1)) && !(codes & 3);
    auto go = [&](auto t, auto n) {
        AMS_LAUNCH("cache_write", st,
                   cache_write_k<decltype(t), decltype(n)::value><<<(unsigned)blocks, kAttnThreads, 0, st>>>(a));
        return ams_launch_status();
    };
    using One = std::integral_constant<int, 1>;
    using Four = std::integral_constant<int, 4>;
    if (dtype == AMS_F32) return four ? go(0.f, Four()) : go(0.f, One());
    return four ? go((uint16_t)0, Four()) : go((uint16_t)0, One());
}

extern "C" size_t ams_cache_workspace(const ams_attn *attn, const ams_cache *cache, int32_t B, int64_t n_q)
{
    // whichever pieces the call's addresses allow
    size_t most = 0;
    for (int way = 0; way < 3; ++way) {
        Cut cut;
        bool many;
        size_t need;
        if (!attn || !cache || read_plan(attn, cache, B, n_q, way > 0, way > 1, cut, many, need) != AMS_OK) return 0;
        most = need > most ? need : most;
    }
    return most;
}

extern "C" ams_status ams_cache_attn(const ams_attn *attn, const ams_cache *cache, int32_t B, const int32_t *q_off,
                                     int64_t n_q, const int32_t *lengths, const int32_t *page_table, const void *q,
                                     int64_t ld_q, const uint8_t *k_codes, const float *k_scale,
                                     const uint8_t *v_codes, const float *v_scale, void *out, int64_t ld_out,
                                     float *lse, void *ws, size_t ws_bytes, void *stream)
{
    if (!attn || !cache) return AMS_ERR_NULL;
    AttnArgs a{};
    const int64_t ld[] = {ld_q, ld_out};
    const void *ptr[] = {q, out};
    const int es = attn->dtype == AMS_F32 ? 4 : 2;
    int pb = piece_bytes(es, attn->head_dim, 2, ld, ptr);
    const uint64_t codes = (uint64_t)(uintptr_t)k_codes | (uint64_t)(uintptr_t)v_codes;
    if (codes & (pb / es - 1)) pb = es;                // a piece of codes has as many entries as one of q
    Cut cut;
    bool many;
    size_t total;
    const ams_status s = read_plan(attn, cache, B, n_q, pb == 16, !(codes & 15), cut, many, total);
    if (s != AMS_OK) return s;
    cache_shape(cache, a.page_shift);
    const int64_t w = (int64_t)attn->n_heads * attn->head_dim;
    if (ld_q < w || ld_out < w) return AMS_ERR_SIZE;
    if (B == 0 || n_q == 0) return AMS_OK;
    if (!q_off || !lengths || !page_table || !q || !k_codes || !k_scale || !v_codes || !v_scale || !out || !ws)
        return AMS_ERR_NULL;
    if (ws_bytes < total) return AMS_ERR_WORKSPACE;
    a.B = B, a.H = attn->n_heads, a.Hk = attn->n_kv_heads, a.G = a.H / a.Hk, a.D = attn->head_dim;
    a.by_g = fast_div((uint32_t)a.G);
    a.scale = attn->scale;
    a.q_off = q_off, a.n_q = n_q, a.q = q, a.ld_q = ld_q;
    a.len = lengths, a.page_table = page_table, a.max_pages = cache->max_pages, a.n_pages = cache->n_pages;
    a.kc = k_codes, a.vc = v_codes, a.ks = k_scale, a.vs = v_scale;
    a.out = out, a.ld_out = ld_out, a.lse = lse;
    a.part_ml = (float *)align_up((size_t)ws);
    a.part_o = (float *)((char *)a.part_ml + align_up((size_t)cut.nsplit * n_q * a.H * 2 * sizeof(float)));
    hipStream_t st = (hipStream_t)stream;
    a.nsplit = cut.nsplit, a.tiles = cut.tiles;
    return with_attn(attn->dtype, a.D, pb, [&](auto t, auto dh, auto piece) {
        using T = decltype(t);
        constexpr int DH = decltype(dh)::value, PB = decltype(piece)::value;
        if constexpr (PB == 16 && sizeof(T) == 2) {
            if (many) {
                AMS_LAUNCH("cache_attn_many", st,
                           attn_fwd_many_k<DH, PB, true><<<(unsigned)cut.blocks, kAttnThreads, 0, st>>>(a));
                if (a.nsplit > 1) launch_join<T>("cache_join", a, st);
                return ams_launch_status();
            }
        }
        with_cut<T, DH, PB>(cut, [&](auto rt, auto wk) {
            AMS_LAUNCH("cache_attn", st,
                       attn_fwd_k<T, DH, PB, true, decltype(rt)::value, decltype(wk)::value>
                       <<<(unsigned)cut.blocks, kAttnThreads, 0, st>>>(a));
            return AMS_OK;
        });
        if (a.nsplit > 1) launch_join<T>("cache_join", a, st);
        return ams_launch_status();
    });
}
