// gfx950 kernels for the attention that cached rows get, and for dropping the rows that get least.
//
// The weight of row p of a KV head is the sum, over queries i and the heads that share the KV head, of exp(s_ip - lse_i): the softmax weights that attention
// has given the row.  The results are fp32 sums of many positive terms, and an error of the scores is a relative one of the weights, so scores are made to
// 22 bits: each turned key and query is a sum of two fp16 numbers, and three of the four products of those are taken, on the matrix cores in fp32.
// Keys and queries are divided by powers of two of their own (largest element of a row 2^12 .. 2^13), which come back in fp32: fp16 holds any magnitude.
//
//   k_weights_few      up to 16 queries of a unit: rows stream by, queries stay
//   k_weights_queries  more: the queries as operands, turned, in fragment order
//   k_weights          ... keys stay, in registers, and queries stream by
//   k_weights_join     ... parts of the queries brought together, in order
//   k_evict_select     which rows of a head stay: the `keep` largest weights (a radix selection), in their order
//   k_evict_move       their keys and values move up
#include "freqkv_internal.h"
#include "freqkv_lanes.h"
#include "freqkv_turn.h"

#include <type_traits>

namespace freqkv {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Eight adjacent values, as stored and as floats.
template <typename T> struct Eight;
template <> struct Eight<uint16_t> { u32x4 a; };
template <> struct Eight<float> { u32x4 a, b; };
__device__ __forceinline__ void read8(const __amdgpu_buffer_rsrc_t& buf, uint32_t at, Eight<uint16_t>& x) { x.a = __builtin_amdgcn_raw_buffer_load_b128(buf, at, 0, 0); }
__device__ __forceinline__ void read8(const __amdgpu_buffer_rsrc_t& buf, uint32_t at, Eight<float>& x)
{
    x.a = __builtin_amdgcn_raw_buffer_load_b128(buf, at, 0, 0);
    x.b = __builtin_amdgcn_raw_buffer_load_b128(buf, at + 16, 0, 0);
}
__device__ __forceinline__ void read8(const uint16_t* p, Eight<uint16_t>& x) { x.a = *(const u32x4*)p; }
__device__ __forceinline__ void read8(const float* p, Eight<float>& x) { x.a = *(const u32x4*)p; x.b = *(const u32x4*)(p + 4); }
template <int I> __device__ __forceinline__ float at8(const Eight<uint16_t>& x) { return __uint_as_float(I & 1 ? x.a[I / 2] & 0xffff0000u : x.a[I / 2] << 16); }
template <int I> __device__ __forceinline__ float at8(const Eight<float>& x) { return __uint_as_float(I < 4 ? x.a[I & 3] : x.b[I & 3]); }

// The power of two that brings a row whose largest magnitude is `most` to 2^12 .. 2^13, and its inverse.
struct Power { float down, up; };
__device__ __forceinline__ Power power_for(float most)
{
    const int e = max(-110, min(exponent_of(most), 126)) - 12;
    return Power{ldexpf(1.f, -e), ldexpf(1.f, e)};
}

// Eight floats as sums of two fp16 numbers.
__device__ __forceinline__ void split8(const float (&x)[8], half8& hi, half8& lo)
{
    static_for<4>([&](auto i) {
        const half2v h = halves(x[2 * i.value], x[2 * i.value + 1]);
        const half2v l = halves(x[2 * i.value] - (float)h[0], x[2 * i.value + 1] - (float)h[1]);
        hi[2 * i.value] = h[0]; hi[2 * i.value + 1] = h[1];
        lo[2 * i.value] = l[0]; lo[2 * i.value + 1] = l[1];
    });
}

// log2(e) times a query's lse, to be taken from its scores.  One that saw no row (-inf) adds nothing.
__device__ __forceinline__ float taken(float lse) { return lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f; }

}  // namespace

// Up to 16 queries: bound by the rows.  A wave has tiles of 16 rows; a lane (c, g) = (lane & 15, lane >> 4) has of row c the channels 32 p + 8 g .. + 7 for every p,
// so that a rotary pair is in one lane, and gets the scores of row c with the queries 4 g .. 4 g + 3.
template <typename T, int D>
__global__ __launch_bounds__(256, (D == 256 ? 1 : 2))
void k_weights_few(const WeightGeom, const T* __restrict__ q, const float* __restrict__ lse, const TurnTable rt, float* __restrict__ weights,
                   const SlabTable tab)
{
    const WeightGeom g = first_argument<decltype(k_weights_few<T, D>)>();
    constexpr int KS = D / 32, HP = KS / 2;         // k-steps; of a half
    __shared__ __attribute__((aligned(16))) float2 turns[4][D / 2];
    const int lane = threadIdx.x & 63, c = lane & 15, gq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = g.by_chunk.quotient(blockIdx.x), ck = blockIdx.x - unit * g.n_chunk;
    const int layer = g.by_layer.quotient(unit), rem = unit - layer * g.units_per_layer;
    const int b = g.by_kv.quotient(rem), kvh = rem - b * g.n_kv;
    int cur_len = g.cur_len;
    if (g.cur_lens) cur_len = max(0, min(g.cur_lens[b], g.cur_len));
    const int row0 = ck * g.chunk, row_end = min(row0 + g.chunk, cur_len);
    if (row0 >= row_end) return;
    const uint32_t row_bytes = (uint32_t)g.stride_token * (uint32_t)sizeof(T);
    const char* const kbase = tab.base[layer] + ((long long)b * g.stride_batch + (long long)kvh * g.stride_head) * (long long)sizeof(T);
    const __amdgpu_buffer_rsrc_t kbuf = __builtin_amdgcn_make_buffer_rsrc((void*)kbase, 0, (int)((uint32_t)(row_end - 1) * row_bytes + (uint32_t)(D * sizeof(T))), kBufferFlags);
    float* const wout = weights + (long long)unit * g.capacity;

    const int wrow = row0 + 16 * wave, tiles = wrow < row_end ? (row_end - wrow + kTurnStep - 1) / kTurnStep : 0;
    Eight<T> lo[HP], up[HP];
    auto load = [&](int n) {
        const uint32_t at = (uint32_t)(wrow + n * kTurnStep + c) * row_bytes + (uint32_t)(8 * gq) * (uint32_t)sizeof(T);
        static_for<HP>([&](auto p) {
            read8(kbuf, at + p.value * 32 * (uint32_t)sizeof(T), lo[p.value]);
            read8(kbuf, at + (D / 2 + p.value * 32) * (uint32_t)sizeof(T), up[p.value]);
        });
    };
    load(0);
    float co[HP][8], si[HP][8], cd[HP][8], sd[HP][8];
    float2* const own = turns[wave];
    auto seed = [&](int n) {
        wave_turns<D>(rt, wrow + n * kTurnStep - (cur_len - 1), own, lane);
        static_for<HP>([&](auto p) { seeds<D, 8>(rt, own, c, 32 * p.value + 8 * gq, co[p.value], si[p.value]); });
    };
    static_for<HP>([&](auto p) { steps<8>(rt, 32 * p.value + 8 * gq, cd[p.value], sd[p.value]); });
    seed(0);

    // ---- queries: the lane's is c; of those that its scores are of, factors, lse and last rows
    half8 qh[KS], ql[KS];
    const long long head0 = (long long)unit * g.M;
    const int mine = min(c, g.M - 1), place = mine - g.by_q.quotient(mine) * g.q_len;
    float qfactor;
    {
        Eight<T> a[HP], bb[HP];
        const T* const qp = q + (head0 + mine) * D + 8 * gq;
        float most = 0.f;
        static_for<HP>([&](auto p) {
            read8(qp + 32 * p.value, a[p.value]);
            read8(qp + D / 2 + 32 * p.value, bb[p.value]);
            static_for<8>([&](auto i) { most = fmaxf(most, fmaxf(fabsf(at8<i.value>(a[p.value])), fabsf(at8<i.value>(bb[p.value])))); });
        });
        most = fold<32>(fold<16>(most, Max{}), Max{});
        const Power pw = power_for(most);
        qfactor = pw.up * g.qscale;
        static_for<HP>([&](auto p) {
            float x[8], y[8];
            static_for<8>([&](auto i) { x[i.value] = at8<i.value>(a[p.value]) * pw.down; y[i.value] = at8<i.value>(bb[p.value]) * pw.down; });
            if (g.q_len > 1) {
                static_for<8>([&](auto i) {
                    const float l = x[i.value], u = y[i.value];
                    const CosSin t = turn(rt.quarters[32 * p.value + 8 * gq + i.value], place + 1 - g.q_len);
                    x[i.value] = fmaf(l, t.c, -(u * t.s));
                    y[i.value] = fmaf(u, t.c, l * t.s);
                    if constexpr (i.value % 4 == 3) __builtin_amdgcn_sched_barrier(0);    // (all at once, they take more registers than there are)
                });
            }
            split8(x, qh[p.value], ql[p.value]);
            split8(y, qh[HP + p.value], ql[HP + p.value]);
        });
    }
    const float taken_mine = c < g.M ? taken(lse[head0 + mine]) : INFINITY;      // (no query there: nothing is added)
    float factor[4], minus[4];
    int last[4];                                     // row of the query
    static_for<4>([&](auto r) {
        factor[r.value] = __shfl(qfactor, 4 * gq + r.value);
        minus[r.value] = -__shfl(taken_mine, 4 * gq + r.value);
        last[r.value] = cur_len - g.q_len + __shfl(place, 4 * gq + r.value);
    });

    for (int n = 0; n < tiles; ++n) {
        if (n > 0 && n % 64 == 0) seed(n);
        half8 kh[KS], kl[KS];
        float most = 0.f;
        static_for<HP>([&](auto p) {
            static_for<8>([&](auto i) { most = fmaxf(most, fmaxf(fabsf(at8<i.value>(lo[p.value])), fabsf(at8<i.value>(up[p.value])))); });
        });
        most = fold<32>(fold<16>(most, Max{}), Max{});
        const Power pw = power_for(most);
        static_for<HP>([&](auto p) {
            float x[8], y[8];
            static_for<8>([&](auto i) {
                constexpr int P = p.value, I = i.value;
                const float l = at8<I>(lo[P]) * pw.down, u = at8<I>(up[P]) * pw.down;
                x[I] = fmaf(l, co[P][I], -(u * si[P][I]));
                y[I] = fmaf(u, co[P][I], l * si[P][I]);
                const float cn = fmaf(co[P][I], cd[P][I], -(si[P][I] * sd[P][I]));
                si[P][I] = fmaf(si[P][I], cd[P][I], co[P][I] * sd[P][I]);
                co[P][I] = cn;
            });
            split8(x, kh[p.value], kl[p.value]);
            split8(y, kh[HP + p.value], kl[HP + p.value]);
        });
        if (n + 1 < tiles) load(n + 1);
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        static_for<KS>([&](auto k) {
            s = __builtin_amdgcn_mfma_f32_16x16x32_f16(ql[k.value], kh[k.value], s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x32_f16(qh[k.value], kl[k.value], s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x32_f16(qh[k.value], kh[k.value], s, 0, 0, 0);
        });
        const int row = wrow + n * kTurnStep + c;
        float w = 0.f;
        static_for<4>([&](auto r) {
            const float e = exp2_fast(fmaf(s[r.value], factor[r.value] * pw.up, minus[r.value]));
            w += row <= last[r.value] ? e : 0.f;
        });
        w = fold<32>(fold<16>(w, Add{}), Add{});
        if (gq == 0 && row < row_end) wout[row] = g.accumulate ? wout[row] + w : w;
    }
}

// Queries as operands: a workgroup has a tile of 32, eight threads to a query.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_weights_queries(const WeightGeom, const T* __restrict__ q, const float* __restrict__ lse, const TurnTable rt,
                                                         _Float16* __restrict__ operands, float2* __restrict__ factors)
{
    const WeightGeom g = first_argument<decltype(k_weights_queries<T, D>)>();
    constexpr int N = D / 16;                       // pairs of a thread
    const int unit = g.by_split.quotient(blockIdx.x), tile = blockIdx.x - unit * g.q_tiles;      // (by_split: of q_tiles here)
    const int j = threadIdx.x >> 3, sub = threadIdx.x & 7, mine = kWeightTile * tile + j;
    const bool there = mine < g.M;
    const long long head = (long long)unit * g.M + (there ? mine : 0);
    const int place = there ? mine - g.by_q.quotient(mine) * g.q_len : 0;
    const T* const qp = q + head * D + N * sub;
    float a[N], bb[N], most = 0.f;
    static_for<N>([&](auto i) {
        if constexpr (sizeof(T) == 2) {
            a[i.value] = __uint_as_float((uint32_t)qp[i.value] << 16);
            bb[i.value] = __uint_as_float((uint32_t)qp[D / 2 + i.value] << 16);
        } else {
            a[i.value] = qp[i.value];
            bb[i.value] = qp[D / 2 + i.value];
        }
        most = fmaxf(most, fmaxf(fabsf(a[i.value]), fabsf(bb[i.value])));
    });
    most = fmaxf(most, dpp<0xB1>(most));
    most = fmaxf(most, dpp<0x4E>(most));
    most = fmaxf(most, dpp<0x141>(most));
    const Power pw = power_for(most);
    _Float16* const to = operands + ((long long)unit * g.q_tiles + tile) * (2 * kWeightTile * D);
    static_for<N>([&](auto i) {
        const int ch = N * sub + i.value;
        const float l = a[i.value] * pw.down, u = bb[i.value] * pw.down;
        const CosSin t = turn(rt.quarters[ch], place + 1 - g.q_len);
        const float xy[2] = {there ? l * t.c - u * t.s : 0.f, there ? u * t.c + l * t.s : 0.f};
        static_for<2>([&](auto n) {
            const int at = ch + n.value * (D / 2);      // k-step at / 16, lane (at / 8 & 1) * 32 + j, place at % 8
            const _Float16 h = (_Float16)xy[n.value];
            _Float16* const p = to + ((at / 16) * 64 + (at / 8 & 1) * 32 + j) * 8 + at % 8;
            p[0] = h;
            p[kWeightTile * D] = (_Float16)(xy[n.value] - (float)h);
        });
    });
    if (sub == 0) factors[((long long)unit * g.q_tiles + tile) * kWeightTile + j] = float2{there ? pw.up * g.qscale : 0.f, there ? -taken(lse[head]) : -INFINITY};
}

// More queries: bound by the matrix cores.  A wave has 32 keys, a workgroup 128; v_mfma_f32_32x32x16_f16, queries x keys, so that a lane gets 16 queries' scores with one
// key, and adds up weights without an exchange.
template <typename T, int D>
__global__ __launch_bounds__(256, (D == 256 ? 1 : 2))
void k_weights(const WeightGeom, const _Float16* __restrict__ operands, const float2* __restrict__ factors, const TurnTable rt,
               float* __restrict__ parts, float* __restrict__ weights, const SlabTable tab)
{
    const WeightGeom g = first_argument<decltype(k_weights<T, D>)>();
    constexpr int KS = D / 16, HP = KS / 2;         // k-steps; of a half
    static_assert(kWeightTile <= kTurnRows, "rows of a tile");
    __shared__ __attribute__((aligned(16))) float2 turns[4][D / 2];
    const int lane = threadIdx.x & 63, l32 = lane & 31, hw = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // part of the queries, then unit, then keys
    const int us = g.by_keys.quotient(blockIdx.x), kb = blockIdx.x - us * g.key_blocks;
    const int unit = g.by_split.quotient(us), split = us - unit * g.n_split;
    const int layer = g.by_layer.quotient(unit), rem = unit - layer * g.units_per_layer;
    const int b = g.by_kv.quotient(rem), kvh = rem - b * g.n_kv;
    int cur_len = g.cur_len;
    if (g.cur_lens) cur_len = max(0, min(g.cur_lens[b], g.cur_len));
    const int row0 = kb * kWeightKeys + wave * kWeightTile, row = row0 + l32;
    if (row0 >= cur_len) return;
    const uint32_t row_bytes = (uint32_t)g.stride_token * (uint32_t)sizeof(T);
    const char* const kbase = tab.base[layer] + ((long long)b * g.stride_batch + (long long)kvh * g.stride_head) * (long long)sizeof(T);
    const __amdgpu_buffer_rsrc_t kbuf = __builtin_amdgcn_make_buffer_rsrc((void*)kbase, 0, (int)((uint32_t)(cur_len - 1) * row_bytes + (uint32_t)(D * sizeof(T))), kBufferFlags);

    half8 kh[KS], kl[KS];
    float kfactor;
    {
        Eight<T> lo[HP], up[HP];
        const uint32_t at = (uint32_t)row * row_bytes + (uint32_t)(8 * hw) * (uint32_t)sizeof(T);
        float most = 0.f;
        static_for<HP>([&](auto p) {
            read8(kbuf, at + p.value * 16 * (uint32_t)sizeof(T), lo[p.value]);
            read8(kbuf, at + (D / 2 + p.value * 16) * (uint32_t)sizeof(T), up[p.value]);
        });
        static_for<HP>([&](auto p) {
            static_for<8>([&](auto i) { most = fmaxf(most, fmaxf(fabsf(at8<i.value>(lo[p.value])), fabsf(at8<i.value>(up[p.value])))); });
        });
        most = fold<32>(most, Max{});
        const Power pw = power_for(most);
        kfactor = pw.up;
        float2* const own = turns[wave];
        wave_turns<D>(rt, row0 - (cur_len - 1), own, lane);
        static_for<HP>([&](auto p) {
            float x[8], y[8], tc[8], ts[8];
            seeds<D, 8>(rt, own, l32, 16 * p.value + 8 * hw, tc, ts);
            static_for<8>([&](auto i) {
                const float l = at8<i.value>(lo[p.value]) * pw.down, u = at8<i.value>(up[p.value]) * pw.down;
                x[i.value] = fmaf(l, tc[i.value], -(u * ts[i.value]));
                y[i.value] = fmaf(u, tc[i.value], l * ts[i.value]);
            });
            split8(x, kh[p.value], kl[p.value]);
            split8(y, kh[HP + p.value], kl[HP + p.value]);
        });
    }

    const int t0 = split * g.split_tiles, t1 = min(t0 + g.split_tiles, g.q_tiles);
    float sum = 0.f;
    for (int t = t0; t < t1; ++t) {
        // places of the tile's queries: from place0 on, and from 0 again where a head's chunk ends
        const int j0 = t * kWeightTile, n = min(kWeightTile, g.M - j0), place0 = j0 - g.by_q.quotient(j0) * g.q_len;
        const bool wraps = place0 + n > g.q_len;
        const int past = cur_len - g.q_len;          // row of the query at place 0
        if (row0 > past + (wraps ? g.q_len - 1 : place0 + n - 1)) continue;      // no query of the tile sees a key of the wave
        const bool masked = row0 + kWeightTile - 1 > past + (wraps ? 0 : place0);
        const half8* const op = (const half8*)(operands + ((long long)unit * g.q_tiles + t) * (2 * kWeightTile * D)) + lane;
        f32x16 s;
        static_for<16>([&](auto r) { s[r.value] = 0.f; });
        static_for<KS>([&](auto k) {
            const half8 h = op[k.value * 64], l = op[(KS + k.value) * 64];
            s = __builtin_amdgcn_mfma_f32_32x32x16_f16(l, kh[k.value], s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x16_f16(h, kl[k.value], s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x16_f16(h, kh[k.value], s, 0, 0, 0);
        });
        const float2* const fa = factors + ((long long)unit * g.q_tiles + t) * kWeightTile;
        static_for<16>([&](auto r) {
            const int j = 8 * (r.value / 4) + 4 * hw + r.value % 4;
            const float2 f = fa[j];
            float e = exp2_fast(fmaf(s[r.value], kfactor * f.x, f.y));
            if (masked) {
                const int at = j0 + j, place = at - g.by_q.quotient(at) * g.q_len;
                e = row <= past + place && at < g.M ? e : 0.f;
            }
            sum += e;
        });
    }
    sum = fold<32>(sum, Add{});
    if (hw == 0 && row < cur_len) {
        if (g.n_split > 1) {
            parts[((long long)split * g.units + unit) * g.cur_len + row] = sum;
        } else {
            float* const w = weights + (long long)unit * g.capacity + row;
            *w = g.accumulate ? *w + sum : sum;
        }
    }
}

__global__ __launch_bounds__(256) void k_weights_join(const WeightGeom g, const float* __restrict__ parts, float* __restrict__ weights)
{
    const int blocks = (g.cur_len + 255) / 256, unit = blockIdx.x / blocks, row = (blockIdx.x - unit * blocks) * 256 + (int)threadIdx.x;
    const int b = (unit % g.units_per_layer) / g.n_kv;
    int cur_len = g.cur_len;
    if (g.cur_lens) cur_len = max(0, min(g.cur_lens[b], g.cur_len));
    if (row >= cur_len) return;
    float sum = 0.f;
    for (int s = 0; s < g.n_split; ++s) sum += parts[((long long)s * g.units + unit) * g.cur_len + row];
    float* const w = weights + (long long)unit * g.capacity + row;
    *w = g.accumulate ? *w + sum : sum;
}

// ---------------------------------------------------------------------------------------------
// eviction
// ---------------------------------------------------------------------------------------------

namespace {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64, kBins = 2048;

// Larger weights have larger orders; +0 and -0 the same one, NaN the least.
__device__ __forceinline__ uint32_t order_of(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
    return u >> 31 ? ~u : u | 0x80000000u;
}

// Rows of a sequence and of what competes in it.
struct Span { int n, lo, hi; bool due; };
__device__ __forceinline__ Span span_of(const EvictGeom& g, int b)
{
    Span s;
    s.n = g.cur_lens ? max(0, min(g.cur_lens[b], g.cur_len)) : g.cur_len;
    s.lo = min(g.n_sink, s.n);
    s.hi = max(s.lo, s.n - g.n_recent);
    s.due = s.hi - s.lo > g.keep;
    return s;
}

}  // namespace

// A workgroup to a unit.  The keep-th largest order is found 11, 11 and 10 bits at a time, from counts of the rows that agree in the bits before; of the rows
// that have it the first ones stay.  Then rows are gone through in their order, 1024 at a time, and each of those that stay has its place from the
// counts of those before it.  weights_out may be weights: rows are read ahead of a barrier, and move to lower places only.
__global__ __launch_bounds__(kSelectThreads) void k_evict_select(const EvictGeom g, const float* weights, float* weights_out, int* __restrict__ kept, int* __restrict__ new_lens)
{
    __shared__ uint32_t hist[kBins];
    __shared__ int above[kSelectWaves], chosen[2], counts[2][2][kSelectWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int unit = blockIdx.x, layer = g.by_layer.quotient(unit), rem = unit - layer * g.units_per_layer;
    const int b = g.by_kv.quotient(rem), kvh = rem - b * g.n_kv;
    const Span s = span_of(g, b);
    const float* const w = weights + (long long)unit * g.capacity;
    float* const wo = weights_out ? weights_out + (long long)unit * g.capacity : nullptr;
    int* const out = kept + (long long)unit * g.keep;
    const int new_len = s.due ? s.lo + g.keep + (s.n - s.hi) : s.n;
    if (new_lens && layer == 0 && kvh == 0 && tid == 0) new_lens[b] = new_len;
    if (!s.due) {
        for (int j = tid; j < g.keep; j += kSelectThreads) out[j] = s.lo + j < s.hi ? s.lo + j : -1;
        if (wo) {
            if (wo != w)
                for (int r = tid; r < s.n; r += kSelectThreads) wo[r] = w[r];
            for (int r = s.n + tid; r < g.cur_len; r += kSelectThreads) wo[r] = 0.f;
        }
        return;
    }
    uint32_t found = 0;                              // bits of the keep-th largest order
    int need = g.keep;                               // rows still to be taken among those that agree with them
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int i = tid; i < kBins; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        for (int r = s.lo + tid; r < s.hi; r += kSelectThreads) {
            const uint32_t u = order_of(w[r]);
            if (pass == 0 || u >> (shift + bits) == found >> (shift + bits)) atomicAdd(&hist[u >> shift & ((1u << bits) - 1)], 1u);
        }
        __syncthreads();
        // thread t has the bins 2047 - 2 t and 2046 - 2 t, from the largest down; the rows above them by a sum over the threads before
        const int top = kBins - 1 - 2 * tid, c0 = (int)hist[top], c1 = (int)hist[top - 1];
        int before = c0 + c1;
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(before, o);
            if (lane >= o) before += x;
        }
        if (lane == 63) above[wave] = before;
        __syncthreads();
        before -= c0 + c1;
        for (int i = 0; i < wave; ++i) before += above[i];
        if (before < need && before + c0 >= need) { chosen[0] = top; chosen[1] = before; }
        else if (before + c0 < need && before + c0 + c1 >= need) { chosen[0] = top - 1; chosen[1] = before + c0; }
        __syncthreads();
        found |= (uint32_t)chosen[0] << shift;
        need -= chosen[1];
        __syncthreads();
    }
    if (wo && wo != w)
        for (int r = tid; r < s.lo; r += kSelectThreads) wo[r] = w[r];
    int larger = 0, equal = 0;                       // among the rows so far
    for (int r0 = s.lo, flip = 0; r0 < s.hi; r0 += kSelectThreads, flip ^= 1) {
        const int r = r0 + tid;
        const float x = r < s.hi ? w[r] : 0.f;
        const uint32_t u = order_of(x);
        const bool gt = r < s.hi && u > found, eq = r < s.hi && u == found;
        const uint64_t mg = __builtin_amdgcn_ballot_w64(gt), me = __builtin_amdgcn_ballot_w64(eq);
        if (lane == 0) { counts[flip][0][wave] = __popcll(mg); counts[flip][1][wave] = __popcll(me); }
        __syncthreads();
        int g0 = larger, e0 = equal;
        for (int i = 0; i < kSelectWaves; ++i) {
            if (i < wave) { g0 += counts[flip][0][i]; e0 += counts[flip][1][i]; }
            larger += counts[flip][0][i];
            equal += counts[flip][1][i];
        }
        const uint64_t below = ((uint64_t)1 << lane) - 1;
        g0 += __popcll(mg & below);
        e0 += __popcll(me & below);
        if (gt || (eq && e0 < need)) {
            const int at = g0 + min(e0, need);
            out[at] = r;
            if (wo) wo[s.lo + at] = x;
        }
    }
    if (!wo) return;
    for (int r0 = s.hi; r0 < s.n; r0 += kSelectThreads) {
        const int r = r0 + tid;
        const float x = r < s.n ? w[r] : 0.f;
        __syncthreads();
        if (r < s.n) wo[s.lo + g.keep + (r - s.hi)] = x;
    }
    __syncthreads();
    for (int r = new_len + tid; r < g.cur_len; r += kSelectThreads) wo[r] = 0.f;
}

// A workgroup moves a slice of all rows of a head-tensor, in their order: 64 KB are read, and after a barrier written, to lower rows.  No row is written that is
// still to be read: the i-th row that stays lies at lo + i or above, and the rows written until then are those up to there.
constexpr int kMovePieces = 4;
__global__ __launch_bounds__(1024) void k_evict_move(const EvictGeom, const int* __restrict__ kept, const SlabTable tab)
{
    const EvictGeom g = first_argument<decltype(k_evict_move)>();
    const int us = g.by_slice.quotient(blockIdx.x), slice = blockIdx.x - us * g.slices, unit = us >> 1, kv = us & 1;
    const int layer = g.by_layer.quotient(unit), rem = unit - layer * g.units_per_layer;
    const int b = g.by_kv.quotient(rem), kvh = rem - b * g.n_kv;
    const Span s = span_of(g, b);
    if (!s.due) return;
    char* const base = tab.base[2 * layer + kv] + (long long)b * g.stride_batch + (long long)kvh * g.stride_head + (long long)slice * g.slice_pieces * 16;
    const int* const from = kept + (long long)unit * g.keep;
    const int rows = g.keep + (s.n - s.hi);
    const int per_step = 1024 * kMovePieces;
    const long long pieces = (long long)rows * g.slice_pieces;
    for (long long p0 = 0; p0 < pieces; p0 += per_step) {
        u32x4 x[kMovePieces];
        char* to[kMovePieces];
        static_for<kMovePieces>([&](auto i) {
            const long long p = p0 + i.value * 1024 + (int)threadIdx.x;
            to[i.value] = nullptr;
            if (p < pieces) {
                const int row = g.by_pieces.quotient((int)p), piece = (int)p - row * g.slice_pieces;
                const int src = row < g.keep ? from[row] : s.hi + (row - g.keep);
                x[i.value] = *(const u32x4*)(base + (long long)src * g.stride_token + piece * 16);
                to[i.value] = base + (long long)(s.lo + row) * g.stride_token + piece * 16;
            }
        });
        __syncthreads();
        static_for<kMovePieces>([&](auto i) { if (to[i.value]) *(u32x4*)to[i.value] = x[i.value]; });
    }
}

// ---------------------------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------------------------

template <class F> static hipError_t by_type(const WeightGeom& g, F&& f)
{
    switch (g.d) {
        case 64:  return g.elem_bytes == 2 ? f(uint16_t{}, IC<64>{}) : f(float{}, IC<64>{});
        case 128: return g.elem_bytes == 2 ? f(uint16_t{}, IC<128>{}) : f(float{}, IC<128>{});
        case 256: return g.elem_bytes == 2 ? f(uint16_t{}, IC<256>{}) : f(float{}, IC<256>{});
        default:  return hipErrorInvalidValue;
    }
}

hipError_t launch_weights_few(const SlabTable& tab, const WeightGeom& g, const void* q, const float* lse, const TurnTable& rt, float* weights, hipStream_t st)
{
    if (g.M < 1 || g.M > kWeightFew || g.n_chunk < 1 || g.chunk % kTurnStep || (long long)g.n_chunk * g.chunk < g.cur_len) return hipErrorInvalidValue;
    return by_type(g, [&](auto t, auto d) {
        typedef decltype(t) T;
        hipLaunchKernelGGL((k_weights_few<T, decltype(d)::value>), dim3((unsigned)(g.units * g.n_chunk)), dim3(256), 0, st, g, (const T*)q, lse, rt, weights, tab);
        return hipGetLastError();
    });
}

hipError_t launch_weights_queries(const WeightGeom& g, const void* q, const float* lse, const TurnTable& rt, void* operands, float2* factors, hipStream_t st)
{
    WeightGeom h = g;
    h.by_split = divisor(g.q_tiles);
    return by_type(g, [&](auto t, auto d) {
        typedef decltype(t) T;
        hipLaunchKernelGGL((k_weights_queries<T, decltype(d)::value>), dim3((unsigned)(g.units * g.q_tiles)), dim3(256), 0, st, h, (const T*)q, lse, rt,
                           (_Float16*)operands, factors);
        return hipGetLastError();
    });
}

hipError_t launch_weights(const SlabTable& tab, const WeightGeom& g, const void* operands, const float2* factors, const TurnTable& rt, float* parts,
                          float* weights, hipStream_t st)
{
    if (g.key_blocks != (g.cur_len + kWeightKeys - 1) / kWeightKeys || (long long)g.n_split * g.split_tiles < g.q_tiles) return hipErrorInvalidValue;
    hipError_t e = by_type(g, [&](auto t, auto d) {
        typedef decltype(t) T;
        hipLaunchKernelGGL((k_weights<T, decltype(d)::value>), dim3((unsigned)(g.units * g.n_split * g.key_blocks)), dim3(256), 0, st, g,
                           (const _Float16*)operands, factors, rt, parts, weights, tab);
        return hipGetLastError();
    });
    if (e != hipSuccess || g.n_split < 2) return e;
    hipLaunchKernelGGL(k_weights_join, dim3((unsigned)(g.units * ((g.cur_len + 255) / 256))), dim3(256), 0, st, g, parts, weights);
    return hipGetLastError();
}

hipError_t launch_evict_select(const EvictGeom& g, const float* weights, float* weights_out, int* kept, int* new_lens, hipStream_t st)
{
    hipLaunchKernelGGL(k_evict_select, dim3((unsigned)g.units), dim3(kSelectThreads), 0, st, g, weights, weights_out, kept, new_lens);
    return hipGetLastError();
}

hipError_t launch_evict_move(const SlabTable& tab, const EvictGeom& g, const int* kept, hipStream_t st)
{
    hipLaunchKernelGGL(k_evict_move, dim3((unsigned)(2 * g.units * g.slices)), dim3(1024), 0, st, g, kept, tab);
    return hipGetLastError();
}

}  // namespace freqkv
