// lookup.hip -- token embeddings: the rows of a table times a scale, one per
// token, and the merged gradient of the touched rows.
//   ams_lookup_fwd  out[k] = scale table[ids[k]]
//   ams_lookup_bwd  grad[u] = scale sum of dout[k] over the tokens k of uniq[u]
// Both are bound by memory: a row is moved in the widest pieces that every
// address allows, by as many lanes as it has pieces (a power of two, 64 at
// most), so that a wave's load covers whole rows.  No float atomics: the
// backward reads the tokens in their sorted order (ams_dedup), in chunks of
// equal size whatever the rows' counts, and joins a row's pieces in the
// chunks' order.
#include <type_traits>

#include "ams_device.h"

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / AMS_WAVE;

template <int BYTES> struct Raw;
template <> struct Raw<16> { typedef uint4 type; };
template <> struct Raw<8> { typedef uint2 type; };
template <> struct Raw<4> { typedef uint32_t type; };
template <> struct Raw<2> { typedef uint16_t type; };

// A piece of a row: N elements of float or bf16 (uint16_t), moved by one
// load or store of N sizeof(T) bytes.
template <class T, int N> struct Piece {
    typedef typename Raw<N * (int)sizeof(T)>::type raw;
    union {
        raw r;
        T e[N];
    };
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(uint16_t x) { return ams_bf16_to_f32(x); }
template <class T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t from_f32<uint16_t>(float x) { return ams_f32_to_bf16(x); }

// Past the caches, which keep what is read again: the table here, the upstream
// rows in the backward that follows.  Us through the caches and past them, the
// lookup alone, repeated: 24 and 21 (823k x 32 float32), 24 and 21 (200k x 256
// bf16), 81 and 59 (64k x 2048 bf16); a step of it with dedup and gradient: 158
// and 147, 131 and 115, 231 and 218.  With nothing in the caches the lookup itself
// takes up to 4 % longer.
template <class T, int N> __device__ __forceinline__ void store_stream(T *p, const Piece<T, N> &x)
{
    constexpr int B = N * (int)sizeof(T);
    if constexpr (B >= 4) {
        typedef uint32_t vec __attribute__((ext_vector_type(B / 4)));
        __builtin_nontemporal_store(__builtin_bit_cast(vec, x), (vec *)p);
    } else {
        *(typename Piece<T, N>::raw *)p = x.r;
    }
}

// ---------------------------------------------------------------- forward

// L lanes per row; a wave takes 64 / L rows at a time, kRows such sets, every
// ID load, then every row load, in flight together.  bf16 products are
// rounded once, to the output.
template <class T, int N, int L>
__global__ __launch_bounds__(kThreads) void lookup_fwd_k(int nv, float scale, int pad_id,
                                                         const int32_t *__restrict__ ids, int64_t n,
                                                         const T *__restrict__ table, int64_t n_rows, int64_t ld_table,
                                                         T *__restrict__ out, int64_t ld_out)
{
    constexpr int kRows = 4, kPer = AMS_WAVE / L;
    const int lane = ams_lane(), g = lane / L, c0 = lane % L;
    const int64_t step = (int64_t)gridDim.x * kWaves * (kPer * kRows);
    for (int64_t k0 = ((int64_t)blockIdx.x * kWaves + threadIdx.x / AMS_WAVE) * (kPer * kRows) + g; k0 - g < n;
         k0 += step) {
        int id[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int64_t k = k0 + r * kPer;
            id[r] = k < n ? ids[k] : -1;
            if (id[r] == pad_id || id[r] >= n_rows) id[r] = -1;
        }
        for (int c = c0; c < nv; c += L) {
            Piece<T, N> x[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                x[r].r = typename Piece<T, N>::raw{};
                if (id[r] >= 0)
                    x[r].r = *(const typename Piece<T, N>::raw *)(table + id[r] * ld_table + (int64_t)c * N);
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const int64_t k = k0 + r * kPer;
                if (k >= n) continue;
#pragma unroll
                for (int e = 0; e < N; ++e) x[r].e[e] = id[r] >= 0 ? from_f32<T>(to_f32(x[r].e[e]) * scale) : (T)0;
                store_stream(out + k * ld_out + (int64_t)c * N, x[r]);
            }
        }
    }
}

// --------------------------------------------------------------- backward

// Chunks of C sorted positions, one wave each (and one column tile of L N
// elements).  A round takes 64 positions: lane t holds position t's token and
// row; the wave's 64 / L groups of lanes take L consecutive positions each,
// every group adding its rows one after the other.  A run of equal rows that
// began in another group gets that group's sum by a segmented scan over the
// groups, and one that began in another round by the carry.  A run that lies
// within the chunk is written to grad; else its part goes to the chunk's two
// partial rows: head (the run came from the chunk before) or tail (it began
// here and goes on).
template <class T, int N, int L>
__global__ __launch_bounds__(kThreads) void lookup_bwd_k(int D, int nv, int rounds, float scale, int pad_id, int64_t n,
                                                         const int32_t *__restrict__ uniq,
                                                         const int32_t *__restrict__ inv,
                                                         const int32_t *__restrict__ perm, int cap,
                                                         const T *__restrict__ dout, int64_t ld_dout,
                                                         float *__restrict__ grad, float *__restrict__ part)
{
    constexpr int G = AMS_WAVE / L;
    const int lane = ams_lane(), g = lane / L, wave = threadIdx.x / AMS_WAVE;
    // rows wider than a wave's 64 pieces: the block's waves take neighbouring column tiles of one chunk
    const int c = (L == AMS_WAVE ? blockIdx.y * kWaves + wave : blockIdx.y) * L + lane % L;
    const bool col = c < nv;
    const int64_t chunk = L == AMS_WAVE ? blockIdx.x : (int64_t)blockIdx.x * kWaves + wave;
    const int64_t p0 = chunk * rounds * AMS_WAVE;
    if (p0 >= n || (L == AMS_WAVE && c - lane >= nv)) return;

    auto row_of = [&](int64_t p, int &k) -> int {      // unique row of a sorted position (-1: none), and its token
        k = -1;
        if (p < 0 || p >= n) return -1;
        const int kk = perm[p];
        if (kk < 0 || kk >= n) return -1;
        const int u = inv[kk];
        if (u < 0 || u >= cap || u >= n) return -1;
        if (!(pad_id >= 0 && uniq[u] == pad_id)) k = kk;
        return u;
    };
    int k_next, u_before, u_now, k_now, dummy;
    u_before = row_of(p0 - 1, dummy);
    u_now = row_of(p0 + lane, k_now);
    const int u_first = __shfl(u_now, 0, AMS_WAVE);
    const bool from_before = p0 > 0 && u_first >= 0 && u_before == u_first;
    bool seen_end = false;                              // a run ended in this chunk already
    float carry[N];
#pragma unroll
    for (int e = 0; e < N; ++e) carry[e] = 0.f;

    auto store = [&](float *dst, const float *v) {
        if (!col) return;
        Piece<float, (N >= 4 ? 4 : N)> o;
#pragma unroll
        for (int q = 0; q < N; q += (N >= 4 ? 4 : N)) {
#pragma unroll
            for (int e = 0; e < (N >= 4 ? 4 : N); ++e) o.e[e] = v[q + e];
            *(typename Piece<float, (N >= 4 ? 4 : N)>::raw *)(dst + (int64_t)c * N + q) = o.r;
        }
    };

    for (int r = 0; r < rounds; ++r) {
        const int64_t pr = p0 + (int64_t)r * AMS_WAVE;
        if (pr >= n) break;
        // the next round's rows: where the last run of this one ends
        int u_next = row_of(pr + AMS_WAVE + lane, k_next);
        const int u_after = __shfl(u_next, 0, AMS_WAVE);
        int u_right = __shfl_down(u_now, 1, AMS_WAVE);
        if (lane == AMS_WAVE - 1) u_right = u_after;
        const uint64_t ends = ams_ballot(u_now >= 0 && u_right != u_now);

        float acc[N], head[N];
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = head[e] = 0.f;
        bool has_end = false;
        int head_u = -1;
        constexpr int kAhead = L < 8 ? L : 8;
        for (int j = 0; j < L; j += kAhead) {
            Piece<T, N> x[kAhead];
            int k[kAhead], u[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int t = g * L + j + a;
                k[a] = __shfl(k_now, t, AMS_WAVE);
                u[a] = __shfl(u_now, t, AMS_WAVE);
                x[a].r = typename Piece<T, N>::raw{};
                if (k[a] >= 0 && col)
                    x[a].r = *(const typename Piece<T, N>::raw *)(dout + k[a] * ld_dout + (int64_t)c * N);
            }
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int t = g * L + j + a;
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] += to_f32(x[a].e[e]);
                if ((ends >> t) & 1) {
                    if (has_end) {
                        float v[N];
#pragma unroll
                        for (int e = 0; e < N; ++e) v[e] = acc[e] * scale;
                        store(grad + (int64_t)u[a] * D, v);
                    } else {
                        has_end = true;
                        head_u = u[a];
#pragma unroll
                        for (int e = 0; e < N; ++e) head[e] = acc[e];
                    }
#pragma unroll
                    for (int e = 0; e < N; ++e) acc[e] = 0.f;
                }
            }
        }
        // carry into each group: the sum of the open run before it
        float in[N], sum[N];
        bool closed = has_end;
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] = acc[e];
#pragma unroll
        for (int o = 1; o < G; o <<= 1) {
            const bool pc = __shfl_up((int)closed, o * L, AMS_WAVE);
            const bool take = g >= o && !closed;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float pv = __shfl_up(sum[e], o * L, AMS_WAVE);
                if (take) sum[e] = pv + sum[e];
            }
            if (take) closed = pc;
        }
        bool before_closed = false;
#pragma unroll
        for (int e = 0; e < N; ++e) in[e] = 0.f;
        if (G > 1) {
            before_closed = __shfl_up((int)closed, L, AMS_WAVE) && g > 0;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float pv = __shfl_up(sum[e], L, AMS_WAVE);
                in[e] = g > 0 ? pv : 0.f;
            }
        }
        if (!before_closed) {
#pragma unroll
            for (int e = 0; e < N; ++e) in[e] += carry[e];
        }
        if (has_end) {                                  // the run that came into the group ends here
            const uint64_t below = g == 0 ? 0ull : ends & (~0ull >> (AMS_WAVE - g * L));
            float v[N];
            if (!seen_end && below == 0 && from_before) {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = in[e] + head[e];
                store(part + chunk * 2 * D, v);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = (in[e] + head[e]) * scale;
                store(grad + (int64_t)head_u * D, v);
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float out = closed ? sum[e] : sum[e] + carry[e];
            carry[e] = __shfl(out, AMS_WAVE - L + lane % L, AMS_WAVE);
        }
        seen_end = seen_end || ends != 0;
        // an open run at the chunk's end
        const bool last = r + 1 == rounds;
        const int u_end = __shfl(u_now, AMS_WAVE - 1, AMS_WAVE);
        if (last && u_end >= 0 && u_end == u_after && g == 0)
            store(part + chunk * 2 * D + (!seen_end && from_before ? 0 : D), carry);
        u_now = u_next;
        k_now = k_next;
    }
}

// Runs over several chunks: the chunk where such a run begins adds its tail
// and the heads of the chunks behind, up to the run's end.  One block per
// chunk and column tile; its lane groups take every (groups)-th chunk, their
// sums are added in order.
template <int N, int L>
__global__ __launch_bounds__(kThreads) void lookup_join_k(int D, int nv, int64_t C, float scale, int64_t n,
                                                          const int32_t *__restrict__ inv,
                                                          const int32_t *__restrict__ perm,
                                                          const int32_t *__restrict__ uniq_off, int cap,
                                                          const float *__restrict__ part, float *__restrict__ grad)
{
    constexpr int G = kThreads / L;
    __shared__ float red[kThreads * N];
    const int64_t chunk = blockIdx.x;
    const int64_t p1 = (chunk + 1) * C;                // first position behind the chunk
    if (p1 >= n) return;
    const int ka = perm[p1 - 1], kb = perm[p1];
    if (ka < 0 || ka >= n || kb < 0 || kb >= n) return;
    const int u = inv[ka];
    if (u < 0 || u >= cap || u >= n || inv[kb] != u) return;
    const int64_t s = uniq_off[u], e1 = uniq_off[u + 1];
    if (s < chunk * C || s >= p1 || e1 <= p1 || e1 > n) return;
    const int64_t last = (e1 - 1) / C;
    const int g = threadIdx.x / L;
    const int c = blockIdx.y * L + threadIdx.x % L;
    float acc[N];
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
    if (c < nv) {
#pragma unroll 4
        for (int64_t q = chunk + g; q <= last; q += G) {
            const float *p = part + q * 2 * D + (q == chunk ? D : 0) + (int64_t)c * N;
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += p[e];
        }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) red[e * kThreads + threadIdx.x] = acc[e];
    __syncthreads();
    if (g == 0 && c < nv) {
        const int64_t m = last - chunk + 1 < G ? last - chunk + 1 : G;
        for (int64_t h = 1; h < m; ++h)
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += red[e * kThreads + h * L + threadIdx.x];
#pragma unroll
        for (int e = 0; e < N; ++e) grad[(int64_t)u * D + (int64_t)c * N + e] = acc[e] * scale;
    }
}

// ------------------------------------------------------------------- host

// Elements of a piece: the widest of 16, 8, 4 (, 2) bytes that divides a
// row's width, its stride and every base address.
int piece_elems(int esize, int32_t D, int64_t ld_a, int64_t ld_b, const void *a, const void *b)
{
    const uint64_t all = (uint64_t)D * esize | (uint64_t)(ld_a * esize) | (uint64_t)(ld_b * esize) |
                         (uint64_t)(uintptr_t)a | (uint64_t)(uintptr_t)b;
    int bytes = 16;
    while (bytes > esize && (all & (bytes - 1))) bytes >>= 1;
    return bytes / esize;
}

int lanes_of(int nv)
{
    int L = 1;
    while (L < nv && L < AMS_WAVE) L <<= 1;
    return L;
}

// Positions per chunk, in rounds of 64: one round while the chunks are few, which
// keeps more waves at work; four where there are enough, which leaves fewer partial
// rows (with one and with four, us: 32 floats 12 and 17 at 131072 tokens, 18 and 20
// at 262144, 44 and 39 at 823k, 109 and 89 at 2M; 512 bf16 28 and 61 at 64k,
// 47 and 64 at 131072, 110 and 101 at 262144).
constexpr int64_t kFourRounds = 262144;
int bwd_rounds(int64_t n) { return n >= kFourRounds ? 4 : 1; }

template <class F> ams_status with_lanes(int L, F f)
{
    switch (L) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 4: return f(std::integral_constant<int, 4>());
    case 8: return f(std::integral_constant<int, 8>());
    case 16: return f(std::integral_constant<int, 16>());
    case 32: return f(std::integral_constant<int, 32>());
    default: return f(std::integral_constant<int, 64>());
    }
}

// f(type, piece elements)
template <class F> ams_status with_piece(int32_t dtype, int N, F f)
{
    if (dtype == AMS_F32) {
        switch (N) {
        case 4: return f(0.f, std::integral_constant<int, 4>());
        case 2: return f(0.f, std::integral_constant<int, 2>());
        default: return f(0.f, std::integral_constant<int, 1>());
        }
    }
    switch (N) {
    case 8: return f((uint16_t)0, std::integral_constant<int, 8>());
    case 4: return f((uint16_t)0, std::integral_constant<int, 4>());
    case 2: return f((uint16_t)0, std::integral_constant<int, 2>());
    default: return f((uint16_t)0, std::integral_constant<int, 1>());
    }
}

constexpr int64_t kMaxTok = (1ll << 30) - 1;           // as ams_dedup
constexpr int32_t kMaxWidth = 65536;
constexpr int64_t kMaxBlocks = 1 << 20;

}  // namespace

extern "C" ams_status ams_lookup_fwd(int32_t dtype, int32_t D, float scale, int32_t pad_id, const int32_t *ids,
                                     int64_t n, const void *table, int64_t n_rows, int64_t ld_table, void *out,
                                     int64_t ld_out, void *stream)
{
    if (dtype != AMS_F32 && dtype != AMS_BF16) return AMS_ERR_DTYPE;
    if (D < 1 || D > kMaxWidth) return AMS_ERR_DIMS;
    if (n < 0 || n > kMaxTok || n_rows < 0 || ld_table < D || ld_out < D) return AMS_ERR_SIZE;
    if (n == 0) return AMS_OK;
    if (!ids || !out || (!table && n_rows > 0)) return AMS_ERR_NULL;
    const int esize = dtype == AMS_F32 ? 4 : 2;
    hipStream_t st = (hipStream_t)stream;
    const int N = piece_elems(esize, D, ld_table, ld_out, table, out);
    const int nv = D / N, L = lanes_of(nv);
    return with_piece(dtype, N, [&](auto t, auto np) {
        using T = decltype(t);
        return with_lanes(L, [&](auto nl) {
            constexpr int NP = decltype(np)::value, NL = decltype(nl)::value;
            const int64_t per = (int64_t)(AMS_WAVE / NL) * 4 * kWaves;
            const int64_t blocks = (n + per - 1) / per;
            AMS_LAUNCH("lookup_fwd", st,
                       lookup_fwd_k<T, NP, NL><<<(unsigned)(blocks < kMaxBlocks ? blocks : kMaxBlocks), kThreads, 0, st>>>(
                           nv, scale, pad_id, ids, n, (const T *)table, n_rows, ld_table, (T *)out, ld_out));
            return ams_launch_status();
        });
    });
}

extern "C" size_t ams_lookup_workspace(int64_t n, int32_t D)
{
    if (n < 0 || n > kMaxTok || D < 1 || D > kMaxWidth) return 0;
    // one round per chunk below the switch, so that a smaller n never needs more
    const int64_t few = n < kFourRounds ? n : kFourRounds - 1;
    const int64_t a = (few + AMS_WAVE - 1) / AMS_WAVE;
    const int64_t b = n < kFourRounds ? 0 : (n + 4 * AMS_WAVE - 1) / (4 * AMS_WAVE);
    return (size_t)(a > b ? a : b) * 2 * D * sizeof(float) + 256;
}

extern "C" ams_status ams_lookup_bwd(int32_t dtype, int32_t D, float scale, int32_t pad_id, int64_t n,
                                     const int32_t *uniq, const int32_t *inv, const int32_t *occ_perm,
                                     const int32_t *uniq_off, const int32_t *n_uniq, int32_t n_uniq_cap,
                                     const void *dout, int64_t ld_dout, float *grad, void *ws, size_t ws_bytes,
                                     void *stream)
{
    if (dtype != AMS_F32 && dtype != AMS_BF16) return AMS_ERR_DTYPE;
    if (D < 1 || D > kMaxWidth) return AMS_ERR_DIMS;
    if (n < 0 || n > kMaxTok || n_uniq_cap < 0 || ld_dout < D) return AMS_ERR_SIZE;
    if (n == 0 || n_uniq_cap == 0) return AMS_OK;
    if (!uniq || !inv || !occ_perm || !uniq_off || !n_uniq || !dout || !grad || !ws) return AMS_ERR_NULL;
    if (ws_bytes < ams_lookup_workspace(n, D)) return AMS_ERR_WORKSPACE;
    const int esize = dtype == AMS_F32 ? 4 : 2;
    hipStream_t st = (hipStream_t)stream;
    float *part = (float *)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
    int N = piece_elems(esize, D, ld_dout, ld_dout, dout, dout);
    while (N > 1 && ((uintptr_t)grad & (N >= 4 ? 15 : N * 4 - 1))) N >>= 1;
    const int nv = D / N, L = lanes_of(nv), rounds = bwd_rounds(n);
    const int64_t C = (int64_t)rounds * AMS_WAVE, chunks = (n + C - 1) / C;
    return with_piece(dtype, N, [&](auto t, auto np) {
        using T = decltype(t);
        return with_lanes(L, [&](auto nl) {
            constexpr int NP = decltype(np)::value, NL = decltype(nl)::value;
            const unsigned tiles = (unsigned)((nv + NL - 1) / NL);
            const dim3 g1 = NL == AMS_WAVE ? dim3((unsigned)chunks, (tiles + kWaves - 1) / kWaves)
                                           : dim3((unsigned)((chunks + kWaves - 1) / kWaves), tiles);
            AMS_LAUNCH("lookup_bwd", st,
                       lookup_bwd_k<T, NP, NL><<<g1, kThreads, 0, st>>>(D, nv, rounds, scale, pad_id, n, uniq, inv,
                                                                       occ_perm, n_uniq_cap, (const T *)dout, ld_dout,
                                                                       grad, part));
            if (chunks > 1)
                AMS_LAUNCH("lookup_join", st,
                           lookup_join_k<NP, NL><<<dim3((unsigned)chunks, tiles), kThreads, 0, st>>>(
                               D, nv, C, scale, n, inv, occ_perm, uniq_off, n_uniq_cap, part, grad));
            return ams_launch_status();
        });
    });
}
