// gfx950 kernels for the attention that cached rows get, and for dropping the rows that get least.
//
// The weight of row p of a KV head is the sum, over queries i and the heads that share the KV head, of exp(s_ip - lse_i): the softmax weights that attention
// has given the row.  The results are fp32 sums of many positive terms, and an error of the scores is a relative one of the weights, so scores are made to
// 22 bits or more: in fp32 where there are few queries, else each turned key and query is a sum of two fp16 numbers, and three of the four products of those are taken.
// Queries, and tiles of keys, are then divided by powers of two (largest element 2^12 .. 2^13), which come back in fp32: fp16 holds any magnitude.
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

// Sums of two values over lanes O apart: the lanes without O in their index get that of x, the others that of y.
template <int O> __device__ __forceinline__ float halved(float x, float y)
{
    const auto s = O == 16 ? __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false)
                           : __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

__device__ __forceinline__ void pin(half8& x) { asm volatile("" : "+v"(x) :: "memory"); }

// log2(e) times a query's lse, to be taken from its scores.  One that saw no row (-inf) adds nothing.
__device__ __forceinline__ float taken(float lse) { return lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f; }

}  // namespace

// Up to 16 queries: bound by the rows.  A wave has tiles of 16 rows, kTurnStep apart; a lane (c, g) = (lane & 15, lane >> 4) has of row c the channels 32 p + 8 g .. + 7 for every p,
// so that a rotary pair is in one lane.  Products and sums are fp32 (with keys and queries as sums of two fp16 a tile took 390 vector instructions instead of 190):
//   SETS 1, 2   up to four or eight queries: v_mfma_f32_4x4x1_16b_f32, a quad of lanes' four rows times the queries that the lanes' places in the quad name, a product of each
//               channel group; sums over the groups by exchanges that halve the rows, to one score of each set to a lane
//   SETS 0      up to 16: v_mfma_f32_16x16x4_f32, to the scores of row c with the queries 4 g .. 4 g + 3; four times as long on the matrix cores as a set
// Tiles are copied to LDS, SLOTS of them under way for each wave, a row's pieces of 16 bytes
// turned by the row, and their weights stay there to the end, when all of the chunk's are written, or added to what is there, together: with rows in registers a tile ahead, and weights
// added as they came, 16 sequences of 4096 to 8192 rows of 8 KV heads of 4 took 78 us; now 49, 3.9 TB/s.
template <typename T, int D, int SETS>
__global__ __launch_bounds__(256, (D == 256 || sizeof(T) == 4 ? 1 : 2))
void k_weights_few(const WeightGeom, const T* __restrict__ q, const float* __restrict__ lse, const TurnTable tables, float* __restrict__ weights,
                   const SlabTable tab)
{
    const WeightGeom g = first_argument<decltype(k_weights_few<T, D, SETS>)>();
    constexpr int HP = D / 64;                      // pieces of eight channels of a lane in each half
    constexpr int RB = D * (int)sizeof(T), PIECES = RB / 16, TILE = 16 * RB, N = TILE / 1024, ROWS = 16 / N;      // bytes, pieces of 16 of a row; copies of a tile, rows of one
    constexpr int SLOTS = D == 256 && sizeof(T) == 4 ? 2 : 3, TABLES = (3 + 16) * (D / 2) * 8, TIN = (TABLES + 1023) / 1024;
    __shared__ __attribute__((aligned(1024))) char pool[4][SLOTS][TILE];
    __shared__ __attribute__((aligned(1024))) char tsm[TIN * 1024];       // the start of the tables: frequencies, rotations by a step, 16 rows
    __shared__ __attribute__((aligned(16))) float2 turns[4][D / 2];
    __shared__ float sums[kWeightFewChunk];
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
    const int wrow = row0 + 16 * wave, tiles = wrow < row_end ? (row_end - wrow + kTurnStep - 1) / kTurnStep : 0;
    const long long head0 = (long long)unit * g.M;

    // ---- copies: tables, a fourth of them each wave, and queries, each wave its own, in the last slot; then the first tiles
    typedef __attribute__((address_space(3))) char* lptr_t;
    const uint32_t ring = (uint32_t)(uintptr_t)(lptr_t)&pool[wave][0][0];
    const int crow = lane / PIECES;                 // row of a copy; its piece is turned by the row of the tile
    auto piece_at = [&](auto i) { return (uint32_t)(((lane % PIECES) ^ ((i.value * ROWS + crow) & 7)) * 16); };
    auto ask = [&](int n) {
        const int first = wrow + n * kTurnStep;
        const char* const from = kbase + (uint32_t)first * row_bytes;
        static_for<N>([&](auto i) {                 // (past the end: the last row again)
            const int row = min(i.value * ROWS + crow, row_end - 1 - first);
            lds_dma16(ring + (uint32_t)(n % SLOTS * TILE + i.value * 1024), from, (uint32_t)row * row_bytes + piece_at(i));
        });
    };
    auto landed = [](auto n) { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(decltype(n)::value) : "memory"); };      // all copies but the last n
    static_for<(TIN + 3) / 4>([&](auto i) {
        const int part = i.value * 4 + wave;
        if (part < TIN) lds_dma16((uint32_t)(uintptr_t)(lptr_t)tsm + (uint32_t)part * 1024, tables.quarters, (uint32_t)(part * 1024 + lane * 16));
    });
    static_for<N>([&](auto i) {
        lds_dma16(ring + (uint32_t)((SLOTS - 1) * TILE + i.value * 1024), (const char*)(q + head0 * D), (uint32_t)(min(i.value * ROWS + crow, g.M - 1) * RB) + piece_at(i));
    });
    if (tiles > 0) ask(0);
    if (SLOTS == 3 && tiles > 1) {
        ask(1);
        landed(IC<2 * N>{});
    } else if (tiles > 0) {
        landed(IC<N>{});
    } else {
        landed(IC<0>{});
    }
    lds_barrier();
    const double* const quarters = (const double*)tsm;
    const float2 *const step = (const float2*)(tsm + D * 4), *const rows = (const float2*)(tsm + D * 12);

    float co[HP][8], si[HP][8];
    float2* const own = turns[wave];
    auto seed = [&](int n) {
        wave_turns<D>(quarters, wrow + n * kTurnStep - (cur_len - 1), own, lane);
        static_for<HP>([&](auto p) { seeds<D, 8>(rows, own, c, 32 * p.value + 8 * gq, co[p.value], si[p.value]); });
    };
    seed(0);
    // eight channels of a row of a tile
    auto eight = [&](const char* tile, int row, int channel, Eight<T>& x) {
        const int piece = channel * (int)sizeof(T) / 16;
        const char* const at = tile + row * RB;
        x.a = *(const u32x4*)(at + (piece ^ (row & 7)) * 16);
        if constexpr (sizeof(T) == 4) x.b = *(const u32x4*)(at + ((piece + 1) ^ (row & 7)) * 16);
    };

    // ---- the lane's queries (of each set lane & 3, or c), scaled by log2(e) / sqrt(d), turned by their places less the last one's; of those that its scores are of, lse and last rows
    constexpr int NQ = SETS ? SETS : 1;
    float ql[NQ][HP][8], qu[NQ][HP][8];
    auto place_of = [&](int j) { return j - g.by_q.quotient(j) * g.q_len; };
    static_for<NQ>([&](auto set) {
        constexpr int Q = set.value;
        const int mine = min(SETS ? 4 * Q + (lane & 3) : c, g.M - 1), place = place_of(mine);
        static_for<HP>([&](auto p) {
            Eight<T> a, bb;
            eight(&pool[wave][SLOTS - 1][0], mine, 32 * p.value + 8 * gq, a);
            eight(&pool[wave][SLOTS - 1][0], mine, D / 2 + 32 * p.value + 8 * gq, bb);
            static_for<8>([&](auto i) { ql[Q][p.value][i.value] = at8<i.value>(a) * g.qscale; qu[Q][p.value][i.value] = at8<i.value>(bb) * g.qscale; });
            if (g.q_len > 1) {
                static_for<8>([&](auto i) {
                    const float l = ql[Q][p.value][i.value], u = qu[Q][p.value][i.value];
                    const CosSin t = turn(quarters[32 * p.value + 8 * gq + i.value], place + 1 - g.q_len);
                    ql[Q][p.value][i.value] = fmaf(l, t.c, -(u * t.s));
                    qu[Q][p.value][i.value] = fmaf(u, t.c, l * t.s);
                    if constexpr (i.value % 4 == 3) __builtin_amdgcn_sched_barrier(0);    // (all at once, they take more registers than there are)
                });
            }
        });
    });
    constexpr int NS = SETS ? SETS : 4;
    float less[NS];
    int last[NS];                                    // row of the query
    static_for<NS>([&](auto r) {
        // (of a query that there is not nothing is added; by scalar loads, which do not queue behind the copies)
        less[r.value] = INFINITY;
        static_for<4>([&](auto of) {
            const int j = SETS ? 4 * r.value + of.value : 4 * of.value + r.value;
            const float x = j < g.M ? taken(lse[head0 + j]) : INFINITY;
            less[r.value] = (SETS ? lane & 3 : gq) == of.value ? x : less[r.value];
        });
        last[r.value] = cur_len - g.q_len + place_of(min(SETS ? 4 * r.value + (lane & 3) : 4 * gq + r.value, g.M - 1));
    });
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // (queries read, before rows are written there)
    if (tiles > SLOTS - 1) ask(SLOTS - 1);

    for (int n = 0; n < tiles; ++n) {
        if (n > 0 && n % 64 == 0) seed(n);
        if (SLOTS == 3 && n + 2 < tiles) landed(IC<2 * N>{});
        else if (n + 1 < tiles) landed(IC<N>{});
        else landed(IC<0>{});
        const char* const tile = &pool[wave][n % SLOTS][0];
        Eight<T> lo[HP], up[HP];
        static_for<HP>([&](auto p) {
            eight(tile, c, 32 * p.value + 8 * gq, lo[p.value]);
            eight(tile, c, D / 2 + 32 * p.value + 8 * gq, up[p.value]);
        });
        f32x4 s[NQ];
        static_for<NQ>([&](auto set) { s[set.value] = f32x4{0.f, 0.f, 0.f, 0.f}; });
        int ln = lane;
        asm volatile("" : "+v"(ln));                 // (rotations are read in every step, and not kept in registers from before the loop)
        static_for<HP>([&](auto p) {
            static_for<8>([&](auto i) {
                constexpr int P = p.value, I = i.value;
                const float l = at8<I>(lo[P]), u = at8<I>(up[P]);
                const float x = fmaf(l, co[P][I], -(u * si[P][I])), y = fmaf(u, co[P][I], l * si[P][I]);
                const float2 by = step[32 * P + 8 * (ln >> 4) + I];
                const float cn = fmaf(co[P][I], by.x, -(si[P][I] * by.y));
                si[P][I] = fmaf(si[P][I], by.x, co[P][I] * by.y);
                co[P][I] = cn;
                if constexpr (SETS == 0) {
                    s[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(ql[0][P][I], x, s[0], 0, 0, 0);
                    s[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(qu[0][P][I], y, s[0], 0, 0, 0);
                } else {
                    static_for<NQ>([&](auto set) { s[set.value] = __builtin_amdgcn_mfma_f32_4x4x1f32(x, ql[set.value][P][I], s[set.value], 0, 0, 0); });
                    static_for<NQ>([&](auto set) { s[set.value] = __builtin_amdgcn_mfma_f32_4x4x1f32(y, qu[set.value][P][I], s[set.value], 0, 0, 0); });
                }
            });
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (read, before it is written again)
        if (n + SLOTS < tiles) ask(n + SLOTS);
        float w = 0.f;
        if constexpr (SETS == 0) {
            const int row = wrow + n * kTurnStep + c;
            static_for<4>([&](auto r) {
                const float e = exp2_fast(s[0][r.value] - less[r.value]);
                w += row <= last[r.value] ? e : 0.f;
            });
            w = fold<32>(fold<16>(w, Add{}), Add{});
            if (gq == 0) sums[row - row0] = w;
        } else {
            // the lane's row is the g-th of its quad's four
            const int row = wrow + n * kTurnStep + (c & 12) + gq;
            static_for<NQ>([&](auto set) {
                const float score = halved<32>(halved<16>(s[set.value][0], s[set.value][1]), halved<16>(s[set.value][2], s[set.value][3]));
                const float e = exp2_fast(score - less[set.value]);
                w += row <= last[set.value] ? e : 0.f;
            });
            w += dpp<0xB1>(w);
            w += dpp<0x4E>(w);
            if ((lane & 3) == 0) sums[row - row0] = w;
        }
    }
    lds_barrier();
    float* const wout = weights + (long long)unit * g.capacity;
    for (int r = row0 + (int)threadIdx.x; r < row_end; r += 256) wout[r] = g.accumulate ? wout[r] + sums[r - row0] : sums[r - row0];
}

// Queries as operands: a workgroup has a tile of 32, eight threads to a query.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_weights_queries(const WeightGeom, const T* __restrict__ q, const float* __restrict__ lse, const TurnTable rt,
                                                         char* __restrict__ operands)
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
    char* const block = operands + ((long long)unit * g.q_tiles + tile) * weight_operand_bytes(D);
    _Float16* const to = (_Float16*)block;
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
    if (sub == 0) ((float2*)(block + 4 * kWeightTile * D))[j] = float2{there ? pw.up * g.qscale : 0.f, there ? -taken(lse[head]) : -INFINITY};
}

// More queries: bound by the matrix cores.  A wave has KT tiles of 32 keys, in registers; v_mfma_f32_32x32x16_f16, keys x queries, so that a lane has one query's
// scores with 16 keys of a tile: its lse and factor are one number each, and weights add up, over all queries, without an exchange until the end.  A tile of queries, 16 KB
// at d = 128, is copied to LDS once for the workgroup's four waves, two tiles ahead, and each wave uses it for two tiles of keys.  64 queries on 4 x 8192
// rows, 8 KV heads of 4: 64 us, 0.8 PFLOP/s with the three products of each.  (Keys loaded to registers, 16 bytes a lane of 32 rows, with their angles from memory, and queries for
// each wave from the L2: 75.)
template <typename T, int D>
__global__ __launch_bounds__(256, (D == 256 ? 1 : 2))
void k_weights(const WeightGeom, const _Float16* __restrict__ operands, const TurnTable tables, float* __restrict__ parts, float* __restrict__ weights, const SlabTable tab)
{
    const WeightGeom g = first_argument<decltype(k_weights<T, D>)>();
    constexpr int KS = D / 16, HP = KS / 2, KT = weight_key_tiles(D), KEYS = kWeightTile * KT;         // k-steps; of a half; keys of a wave
    constexpr int RB = D * (int)sizeof(T), PIECES = RB / 16, KTILE = kWeightTile * RB, KN = KTILE / 1024, ROWS = kWeightTile / KN;      // of a tile of keys as it is cached
    constexpr int QTILE = 4 * kWeightTile * D, QN = QTILE / 4096, SLOTS = 3;       // of a tile of queries; copies of it by each wave
    constexpr int TABLES = (3 + kWeightTile) * (D / 2) * 8, TIN = (TABLES + 1023) / 1024;
    static_assert(kWeightTile <= kTurnRows, "rows of a tile");
    constexpr bool STAGED = 4 * KTILE <= SLOTS * QTILE;                     // keys of 16 bits by way of LDS; of 32 there is no room for them
    __shared__ __attribute__((aligned(1024))) char pool[SLOTS * QTILE];       // a tile of keys of each wave, then tiles of queries
    __shared__ __attribute__((aligned(1024))) char tsm[TIN * 1024];       // the start of the tables: frequencies, rotations by a step, 32 rows
    __shared__ __attribute__((aligned(256))) float2 fsm[4][SLOTS][kWeightTile];
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
    const int first_row = kb * 4 * KEYS, row0 = first_row + wave * KEYS;
    if (first_row >= cur_len) return;
    const uint32_t row_bytes = (uint32_t)g.stride_token * (uint32_t)sizeof(T);
    const char* const kbase = tab.base[layer] + ((long long)b * g.stride_batch + (long long)kvh * g.stride_head) * (long long)sizeof(T);

    // ---- keys: a tile of each wave at a time, through LDS a row's pieces of 16 bytes turned by the row
    typedef __attribute__((address_space(3))) char* lptr_t;
    auto landed = [](auto n) { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(decltype(n)::value) : "memory"); };      // all copies but the last n
    const char* const own_tile = pool + wave * KTILE;
    auto ask_keys = [&](int kt) {
        if constexpr (!STAGED) return;
        const int first = row0 + kt * kWeightTile;
        static_for<KN>([&](auto i) {                // (past the end: the last row again)
            const int r = i.value * ROWS + lane / PIECES, row = min(first + r, cur_len - 1);
            lds_dma16((uint32_t)(uintptr_t)(lptr_t)(pool + wave * KTILE) + (uint32_t)(i.value * 1024), kbase,
                      (uint32_t)row * row_bytes + (uint32_t)(((lane % PIECES) ^ (r & 7)) * 16));
        });
    };
    static_for<(TIN + 3) / 4>([&](auto i) {
        const int part = i.value * 4 + wave;
        if (part < TIN) lds_dma16((uint32_t)(uintptr_t)(lptr_t)tsm + (uint32_t)part * 1024, tables.quarters, (uint32_t)(part * 1024 + lane * 16));
    });
    ask_keys(0);
    landed(IC<0>{});
    lds_barrier();
    const double* const quarters = (const double*)tsm;
    const float2* const rows = (const float2*)(tsm + D * 12);

    // turned by their position less the last row's, divided by a power of two common to a tile
    half8 kh[KT][KS], kl[KT][KS];
    float kfactor[KT];
    float2* const own = turns[wave];
    static_for<KT>([&](auto kt) {
        const int first = row0 + kt.value * kWeightTile;
        Eight<T> lo[HP], up[HP];
        float most = 0.f;
        auto eight = [&](int channel, Eight<T>& x) {
            if constexpr (!STAGED) {
                const char* const from = kbase + (uint32_t)min(first + l32, cur_len - 1) * row_bytes + channel * (int)sizeof(T);
                x.a = *(const u32x4*)from;
                if constexpr (sizeof(T) == 4) x.b = *(const u32x4*)(from + 16);
                return;
            }
            const int piece = channel * (int)sizeof(T) / 16;
            x.a = *(const u32x4*)(own_tile + l32 * RB + (piece ^ (l32 & 7)) * 16);
        };
        if constexpr (STAGED && kt.value > 0) landed(IC<0>{});
        static_for<HP>([&](auto p) {
            eight(16 * p.value + 8 * hw, lo[p.value]);
            eight(D / 2 + 16 * p.value + 8 * hw, up[p.value]);
        });
        if constexpr (STAGED) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (read, before it is written again)
        if constexpr (kt.value + 1 < KT) ask_keys(kt.value + 1);
        wave_turns<D>(quarters, first - (cur_len - 1), own, lane);
        static_for<HP>([&](auto p) {
            static_for<8>([&](auto i) {
                // (of finite values: a row that is not keeps to itself)
                const float a = fabsf(at8<i.value>(lo[p.value])), c = fabsf(at8<i.value>(up[p.value]));
                most = fmaxf(most, fmaxf(a < INFINITY ? a : 0.f, c < INFINITY ? c : 0.f));
            });
        });
        const Power pw = power_for(wave_fold(most, Max{}));
        kfactor[kt.value] = pw.up;
        static_for<HP>([&](auto p) {
            float x[8], y[8], tc[8], ts[8];
            seeds<D, 8>(rows, own, l32, 16 * p.value + 8 * hw, tc, ts);
            static_for<8>([&](auto i) {
                const float l = at8<i.value>(lo[p.value]) * pw.down, u = at8<i.value>(up[p.value]) * pw.down;
                x[i.value] = fmaf(l, tc[i.value], -(u * ts[i.value]));
                y[i.value] = fmaf(u, tc[i.value], l * ts[i.value]);
            });
            split8(x, kh[kt.value][p.value], kl[kt.value][p.value]);
            split8(y, kh[kt.value][HP + p.value], kl[kt.value][HP + p.value]);
            // (worked out here, one after the other: all at once they take more registers than there are)
            pin(kh[kt.value][p.value]); pin(kl[kt.value][p.value]); pin(kh[kt.value][HP + p.value]); pin(kl[kt.value][HP + p.value]);
            __builtin_amdgcn_sched_barrier(0);
        });
    });
    lds_barrier();                                   // (all keys read, before queries are written there)

    // ---- queries, tile by tile.  Places go from place0 on, and from 0 again where a head's chunk ends; `past` is the row of the query at place 0.
    const int t0 = split * g.split_tiles, t1 = min(t0 + g.split_tiles, g.q_tiles), past = cur_len - g.q_len;
    auto place_of = [&](int j) { return j - g.by_q.quotient(j) * g.q_len; };
    auto last_row = [&](int t) {                     // of the queries of a tile
        const int j0 = t * kWeightTile, n = min(kWeightTile, g.M - j0), place0 = place_of(j0);
        return past + (place0 + n > g.q_len ? g.q_len - 1 : place0 + n - 1);
    };
    auto next = [&](int t) {                         // the next tile that sees a key of the workgroup
        while (t < t1 && last_row(t) < first_row) ++t;
        return t;
    };
    const char* const ops = (const char*)operands + (long long)unit * g.q_tiles * weight_operand_bytes(D);
    auto ask = [&](int t, int slot) {
        const char* const from = ops + (long long)t * weight_operand_bytes(D);
        static_for<QN>([&](auto i) {
            const uint32_t at = (uint32_t)((i.value * 4 + wave) * 1024);
            lds_dma16((uint32_t)(uintptr_t)(lptr_t)pool + (uint32_t)(slot * QTILE) + at, from, at + (uint32_t)(lane * 16));
        });
        if (lane < kWeightTile * 8 / 16) lds_dma16((uint32_t)(uintptr_t)(lptr_t)&fsm[wave][slot][0], from, (uint32_t)(QTILE + lane * 16));
    };
    f32x16 sum[KT];
    static_for<KT>([&](auto kt) { static_for<16>([&](auto r) { sum[kt.value][r.value] = 0.f; }); });
    int ta = next(t0), tb = next(ta + 1);
    if (ta < t1) ask(ta, 0);
    if (tb < t1) ask(tb, 1);
    for (int slot = 0; ta < t1;) {
        const int tc = next(tb + 1), after = slot == 0 ? 2 : slot - 1;       // the slot of the tile before
        if (tb < t1) landed(IC<QN + 1>{});
        else landed(IC<0>{});
        lds_barrier();
        if (tc < t1) ask(tc, after);
        const int t = ta, j0 = t * kWeightTile, place0 = place_of(j0);
        const half8* const op = (const half8*)(pool + slot * QTILE) + lane;
        const float2 of_query = fsm[wave][slot][l32];
        ta = tb;
        tb = tc;
        slot = slot == 2 ? 0 : slot + 1;
        if (row0 > last_row(t)) continue;            // no query of the tile sees a key of the wave
        f32x16 s[KT];
        static_for<KT>([&](auto kt) { static_for<16>([&](auto r) { s[kt.value][r.value] = 0.f; }); });
        static_for<KS>([&](auto k) {
            const half8 h = op[k.value * 64], l = op[(KS + k.value) * 64];
            static_for<KT>([&](auto kt) { s[kt.value] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kl[kt.value][k.value], h, s[kt.value], 0, 0, 0); });
            static_for<KT>([&](auto kt) { s[kt.value] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kh[kt.value][k.value], l, s[kt.value], 0, 0, 0); });
            static_for<KT>([&](auto kt) { s[kt.value] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kh[kt.value][k.value], h, s[kt.value], 0, 0, 0); });
        });
        const bool masked = row0 + KEYS - 1 > past + (place0 + min(kWeightTile, g.M - j0) > g.q_len ? 0 : place0);
        const int last = past + place_of(j0 + l32);  // row of the lane's query (one that there is not adds nothing)
        static_for<KT>([&](auto kt) {
            const float f = kfactor[kt.value] * of_query.x;
            static_for<16>([&](auto r) {
                float e = exp2_fast(fmaf(s[kt.value][r.value], f, of_query.y));
                if (masked) e = row0 + kt.value * kWeightTile + 8 * (r.value / 4) + 4 * hw + r.value % 4 <= last ? e : 0.f;
                sum[kt.value][r.value] += e;
            });
        });
    }
    // ---- over the queries of a tile; then lane r of 16 has the key of the register r
    static_for<KT>([&](auto kt) {
        float mine = 0.f;
        static_for<16>([&](auto r) {
            float x = sum[kt.value][r.value];
            x += dpp<0xB1>(x);
            x += dpp<0x4E>(x);
            x += dpp<0x141>(x);
            x = fold<16>(fold<8>(x, Add{}), Add{});
            mine = (lane & 15) == r.value ? x : mine;
        });
        const int r = lane & 15, row = row0 + kt.value * kWeightTile + 8 * (r / 4) + 4 * hw + r % 4;
        if ((lane & 16) == 0 && row < cur_len) {
            if (g.n_split > 1) {
                parts[((long long)split * g.units + unit) * g.cur_len + row] = mine;
            } else {
                float* const w = weights + (long long)unit * g.capacity + row;
                *w = g.accumulate ? *w + mine : mine;
            }
        }
    });
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

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kSelectBins = 2048, kSelectCopies = 4; // of a digit of 11 bits, two to a thread; of each count, one for each fourth lane

// Larger weights have larger orders; +0 and -0 the same one, NaN the least.
__device__ __forceinline__ uint32_t order_of(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
    return u >> 31 ? ~u : u | 0x80000000u;
}

// Sum over the 16 lanes of a row, common to the wave where all rows have the same.  (Sixteen counts read by every lane, 16 waves of them, are what LDS would be busy with.)
__device__ __forceinline__ int sum16(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x140, 0xf, 0xf, true);
    return __builtin_amdgcn_readfirstlane(x);
}

// Sums over the lanes up to each.
__device__ __forceinline__ int scan_wave(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);       // lanes 1, 2, 4 and 8 below, in rows of 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // the last lane of a row to the next
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);      // ... of the second row to the third and fourth
    return x;
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

// A workgroup to a unit, a thread with R rows of its own, 1024 apart, in registers (R 0: more rows than that, read again each time).  The keep-th largest order is found
// by its digits, of 11, 11 and 10 bits, from counts in LDS of the rows that have each and the digits before it as found, until just the rows that stay are; of the rows that have
// it the first ones stay.  Four counts of each digit, for lanes four apart and in different banks: rows of the same weight queue for one of them (8 heads of 8192 rows, of any weights
// 9.2 us, all equal 13; with one count 9.1 and 28; digits of one bit, counted by ballots, 14 and 17; of eight, with their few exponents, 22).  Bound by the three rounds of counts,
// barriers and sums.  Then every row that stays has its place from the counts of those before it, by 64s, which a scan gives.  weights_out may be weights: all rows are read ahead of
// a barrier.
template <int R>
__global__ __launch_bounds__(kSelectThreads) void k_evict_select(const EvictGeom, const float* weights, float* weights_out, int* __restrict__ kept, int* __restrict__ new_lens)
{
    const EvictGeom g = first_argument<decltype(k_evict_select<R>)>();
    constexpr int W = kSelectWaves, N = R ? R : 1;
    static_assert(W == 16 && kSelectBins == 2 * kSelectThreads, "a count to each lane of 16; two digits to a thread");
    __shared__ int counts[2][2][W];                  // R 0
    __shared__ int larger[N * W], equal[N * W];      // of each 64 rows, then of all rows before them
    __shared__ int sums[2][W];
    __shared__ __attribute__((aligned(16))) int bins[kSelectCopies][kSelectBins + 8];      // (copies of a digit's count in different banks)
    __shared__ int digit[3];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
    const int rows = s.hi - s.lo, tiles = (rows + kSelectThreads - 1) / kSelectThreads;
    static_for<kSelectCopies>([&](auto c) { *(u32x2*)&bins[c.value][2 * tid] = u32x2{0u, 0u}; });
    __syncthreads();
    float x[N];
    uint32_t u[N];
    static_for<R>([&](auto i) { const int r = i.value * kSelectThreads + tid; x[i.value] = r < rows ? w[s.lo + r] : 0.f; });
    static_for<R>([&](auto i) { u[i.value] = order_of(x[i.value]); });
    static_for<R>([&](auto i) { u[i.value] = i.value * kSelectThreads + tid < rows ? u[i.value] : 0u; });
    // every row's order, tile by tile; rows past the end have the least, 0
    auto each = [&](auto&& f) {
        if constexpr (R > 0) {
            static_for<R>([&](auto i) { f(i.value, i.value * kSelectThreads + tid < rows, u[i.value], x[i.value]); });
        } else {
            for (int i = 0; i < tiles; ++i) {
                const int r = i * kSelectThreads + tid;
                const float y = r < rows ? w[s.lo + r] : 0.f;
                f(i, r < rows, r < rows ? order_of(y) : 0u, y);
            }
        }
    };
    uint32_t found = 0;
    int need = g.keep;                               // of the rows whose upper bits are found's
    static_for<3>([&](auto pass) {
        constexpr int SHIFT = pass.value == 0 ? 21 : pass.value == 1 ? 10 : 0, BITS = pass.value == 2 ? 10 : 11;
        if (need == 0) return;
        each([&](int, bool there, uint32_t v, float) {
            if (there && (pass.value == 0 || ((v ^ found) >> SHIFT) >> BITS == 0)) atomicAdd(&bins[lane & (kSelectCopies - 1)][v >> SHIFT & ((1 << BITS) - 1)], 1);
        });
        lds_barrier();
        // a thread has two digits, the largest ones first; the rows of those before them
        const int d0 = kSelectBins - 1 - 2 * tid;
        int c0 = 0, c1 = 0;
        static_for<kSelectCopies>([&](auto c) {
            u32x2* const both = (u32x2*)&bins[c.value][d0 - 1];
            c0 += (int)(*both)[1];
            c1 += (int)(*both)[0];
            *both = u32x2{0u, 0u};
        });
        const int upto = scan_wave(c0 + c1);
        if (lane == 63) counts[0][0][wave] = upto;
        lds_barrier();
        const int before = upto - c0 - c1 + sum16((lane & 15) < wave ? counts[0][0][lane & 15] : 0);
        if (before < need && need <= before + c0 + c1) {
            const bool first = need <= before + c0;
            digit[0] = first ? d0 : d0 - 1;
            digit[1] = first ? before : before + c0;     // rows above it
            digit[2] = first ? c0 : c1;
        }
        lds_barrier();
        found |= (uint32_t)__builtin_amdgcn_readfirstlane(digit[0]) << SHIFT;
        need -= __builtin_amdgcn_readfirstlane(digit[1]);
        if (need == __builtin_amdgcn_readfirstlane(digit[2]) && found > 0) {       // just the rows that stay: all above the next lower order
            --found;
            need = 0;
        }
    });
    // ---- rows above and at the order found, by 64s; `place` of the first row that stays of each
    auto prefix = [&](int i, int& above, int& at) {  // counts of a tile's waves, and those before
        above = larger[(R ? i : 0) * W + wave];
        at = equal[(R ? i : 0) * W + wave];
    };
    int all_above = 0, all_at = 0;                   // R 0: of the tiles before
    auto put = [&](int i, bool there, uint32_t v, float y, int need) {
        const bool gt = there && v > found, eq = there && v == found;
        const uint64_t mg = __builtin_amdgcn_ballot_w64(gt), me = __builtin_amdgcn_ballot_w64(eq), below = ((uint64_t)1 << lane) - 1;
        int above, at;
        prefix(i, above, at);
        above += __popcll(mg & below);
        at += __popcll(me & below);
        if (gt || (eq && at < need)) {
            const int place = above + min(at, need);
            out[place] = s.lo + i * kSelectThreads + tid;
            if (wo) wo[s.lo + place] = y;
        }
    };
    if constexpr (R > 0) {
        static_for<R>([&](auto i) {
            const bool there = i.value * kSelectThreads + tid < rows;
            const uint64_t mg = __builtin_amdgcn_ballot_w64(there && u[i.value] > found), me = __builtin_amdgcn_ballot_w64(there && u[i.value] == found);
            if (lane == 0) { larger[i.value * W + wave] = __popcll(mg); equal[i.value * W + wave] = __popcll(me); }
        });
        __syncthreads();
        // thread t < 16 R has the t-th 64 rows
        const int a = tid < N * W ? larger[tid] : 0, e = tid < N * W ? equal[tid] : 0;
        int ia = a, ie = e;
        for (int o = 1; o < 64; o <<= 1) {
            const int ya = __shfl_up(ia, o), ye = __shfl_up(ie, o);
            if (lane >= o) { ia += ya; ie += ye; }
        }
        if (lane == 63) { sums[0][wave] = ia; sums[1][wave] = ie; }
        __syncthreads();
        const int sa = sums[0][lane & 15], se = sums[1][lane & 15], total = sum16(sa);
        const int ba = sum16((lane & 15) < wave ? sa : 0), be = sum16((lane & 15) < wave ? se : 0);
        if (tid < N * W) { larger[tid] = ba + ia - a; equal[tid] = be + ie - e; }
        __syncthreads();
        each([&](int i, bool there, uint32_t v, float y) { put(i, there, v, y, g.keep - total); });
    } else {
        int total = 0;
        each([&](int, bool there, uint32_t v, float) { total += __popcll(__builtin_amdgcn_ballot_w64(there && v > found)); });
        if (lane == 0) sums[0][wave] = total;
        __syncthreads();
        total = sum16(sums[0][lane & 15]);
        for (int i = 0, flip = 0; i < tiles; ++i, flip ^= 1) {
            const int r = i * kSelectThreads + tid;
            const float y = r < rows ? w[s.lo + r] : 0.f;
            const uint32_t v = order_of(y);
            const uint64_t mg = __builtin_amdgcn_ballot_w64(r < rows && v > found), me = __builtin_amdgcn_ballot_w64(r < rows && v == found);
            if (lane == 0) { counts[flip][0][wave] = __popcll(mg); counts[flip][1][wave] = __popcll(me); }
            __syncthreads();
            const int ca = counts[flip][0][lane & 15], ce = counts[flip][1][lane & 15];
            const int above = all_above + sum16((lane & 15) < wave ? ca : 0), at = all_at + sum16((lane & 15) < wave ? ce : 0);
            all_above += sum16(ca);
            all_at += sum16(ce);
            if (lane == 0) { larger[wave] = above; equal[wave] = at; }
            asm volatile("" ::: "memory");           // (a wave's own, in order)
            put(i, r < rows, v, y, g.keep - total);
        }
    }
    if (!wo) return;
    if (wo != w)
        for (int r = tid; r < s.lo; r += kSelectThreads) wo[r] = w[r];
    for (int r0 = s.hi; r0 < s.n; r0 += kSelectThreads) {
        const int r = r0 + tid;
        const float y = r < s.n ? w[r] : 0.f;
        __syncthreads();
        if (r < s.n) wo[s.lo + g.keep + (r - s.hi)] = y;
    }
    __syncthreads();
    for (int r = new_len + tid; r < g.cur_len; r += kSelectThreads) wo[r] = 0.f;
}

// A workgroup moves a slice of all rows of a head-tensor, in their order, 64 KB at a time: read, and after a barrier written, to lower rows.  No row is written that is
// still to be read: the i-th row that stays lies at lo + i or above, and the rows written until then are those up to there; so the next 64 KB are asked for ahead of the
// writes, and which rows they are another step ahead.  A barrier waits for the rows asked for before it alone.  Slices of a head-tensor's rows go to one XCD, whose L2 puts lines
// together.  (32 layers, 8192 rows to 4100: 203 us, 5.3 TB/s; one layer 8.5.)
constexpr int kMovePieces = 4;
__device__ __forceinline__ void awaited(u32x4& x) { asm volatile("" : "+v"(x)); }
__global__ __launch_bounds__(1024) void k_evict_move(const EvictGeom, const int* __restrict__ kept, const SlabTable tab)
{
    const EvictGeom g = first_argument<decltype(k_evict_move)>();
    int us = blockIdx.x, slice = 0;
    if (g.slices > 1) share_out(g.slices, us, slice);
    const int unit = us >> 1, kv = us & 1;
    const int layer = g.by_layer.quotient(unit), rem = unit - layer * g.units_per_layer;
    const int b = g.by_kv.quotient(rem), kvh = rem - b * g.n_kv;
    const Span s = span_of(g, b);
    if (!s.due) return;
    char* const base = tab.base[2 * layer + kv] + (long long)b * g.stride_batch + (long long)kvh * g.stride_head + (long long)slice * g.slice_pieces * 16;
    const int* const from = kept + (long long)unit * g.keep;
    constexpr int STEP = 1024 * kMovePieces;
    const int pieces = (g.keep + (s.n - s.hi)) * g.slice_pieces, steps = (pieces + STEP - 1) / STEP;
    // the i-th piece of a step that a thread has: row it comes from (past the end: the last one's again, not written)
    struct Step { u32x4 x[kMovePieces]; };
    int src[kMovePieces];
    auto which = [&](int t) {
        static_for<kMovePieces>([&](auto i) {
            const int row = g.by_pieces.quotient(min(t * STEP + i.value * 1024 + (int)threadIdx.x, pieces - 1));
            src[i.value] = row < g.keep ? from[row] : s.hi + (row - g.keep);
        });
    };
    auto ask = [&](Step& x, int t) {
        static_for<kMovePieces>([&](auto i) {
            const int p = min(t * STEP + i.value * 1024 + (int)threadIdx.x, pieces - 1), row = g.by_pieces.quotient(p);
            x.x[i.value] = *(const u32x4*)(base + (long long)src[i.value] * g.stride_token + (p - row * g.slice_pieces) * 16);
        });
    };
    auto put = [&](const Step& x, int t) {
        static_for<kMovePieces>([&](auto i) {
            const int p = t * STEP + i.value * 1024 + (int)threadIdx.x, row = g.by_pieces.quotient(p);
            if (p < pieces) *(u32x4*)(base + (long long)(s.lo + row) * g.stride_token + (p - row * g.slice_pieces) * 16) = x.x[i.value];
        });
    };
    auto arrived = [&](Step& x) {                    // ... in all threads of the workgroup
        static_for<kMovePieces>([&](auto i) { awaited(x.x[i.value]); });
        asm volatile("s_barrier" ::: "memory");
    };
    Step a, c;
    which(0);
    ask(a, 0);
    if (steps > 1) which(1);
    for (int t = 0; t < steps; t += 2) {
        arrived(a);
        if (t + 1 < steps) {
            ask(c, t + 1);
            if (t + 2 < steps) which(t + 2);
        }
        put(a, t);
        if (t + 1 >= steps) break;
        arrived(c);
        if (t + 2 < steps) {
            ask(a, t + 2);
            if (t + 3 < steps) which(t + 3);
        }
        put(c, t + 1);
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
    if (g.M < 1 || g.M > kWeightFew || g.n_chunk < 1 || g.chunk % kTurnStep || g.chunk > kWeightFewChunk || (long long)g.n_chunk * g.chunk < g.cur_len) return hipErrorInvalidValue;
    return by_type(g, [&](auto t, auto d) {
        typedef decltype(t) T;
        auto launch = [&](auto sets) {
            hipLaunchKernelGGL((k_weights_few<T, decltype(d)::value, decltype(sets)::value>), dim3((unsigned)(g.units * g.n_chunk)), dim3(256), 0, st, g, (const T*)q, lse, rt,
                               weights, tab);
            return hipGetLastError();
        };
        return g.M <= 4 ? launch(IC<1>{}) : g.M <= 8 ? launch(IC<2>{}) : launch(IC<0>{});
    });
}

hipError_t launch_weights_queries(const WeightGeom& g, const void* q, const float* lse, const TurnTable& rt, void* operands, hipStream_t st)
{
    WeightGeom h = g;
    h.by_split = divisor(g.q_tiles);
    return by_type(g, [&](auto t, auto d) {
        typedef decltype(t) T;
        hipLaunchKernelGGL((k_weights_queries<T, decltype(d)::value>), dim3((unsigned)(g.units * g.q_tiles)), dim3(256), 0, st, h, (const T*)q, lse, rt,
                           (char*)operands);
        return hipGetLastError();
    });
}

hipError_t launch_weights(const SlabTable& tab, const WeightGeom& g, const void* operands, const TurnTable& rt, float* parts,
                          float* weights, hipStream_t st)
{
    if (g.key_blocks != (g.cur_len + weight_keys(g.d) - 1) / weight_keys(g.d) || (long long)g.n_split * g.split_tiles < g.q_tiles) return hipErrorInvalidValue;
    hipError_t e = by_type(g, [&](auto t, auto d) {
        typedef decltype(t) T;
        hipLaunchKernelGGL((k_weights<T, decltype(d)::value>), dim3((unsigned)(g.units * g.n_split * g.key_blocks)), dim3(256), 0, st, g,
                           (const _Float16*)operands, rt, parts, weights, tab);
        return hipGetLastError();
    });
    if (e != hipSuccess || g.n_split < 2) return e;
    hipLaunchKernelGGL(k_weights_join, dim3((unsigned)(g.units * ((g.cur_len + 255) / 256))), dim3(256), 0, st, g, parts, weights);
    return hipGetLastError();
}

hipError_t launch_evict_select(const EvictGeom& g, const float* weights, float* weights_out, int* kept, int* new_lens, hipStream_t st)
{
    const int tiles = (g.cur_len + kSelectThreads - 1) / kSelectThreads;       // (rows that compete: at most)
    auto launch = [&](auto r) {
        hipLaunchKernelGGL(k_evict_select<decltype(r)::value>, dim3((unsigned)g.units), dim3(kSelectThreads), 0, st, g, weights, weights_out, kept, new_lens);
        return hipGetLastError();
    };
    return tiles <= 2 ? launch(IC<2>{}) : tiles <= 8 ? launch(IC<8>{}) : tiles <= 32 ? launch(IC<32>{}) : launch(IC<0>{});
}

hipError_t launch_evict_move(const SlabTable& tab, const EvictGeom& g, const int* kept, hipStream_t st)
{
    hipLaunchKernelGGL(k_evict_move, dim3((unsigned)(2 * g.units * g.slices)), dim3(1024), 0, st, g, kept, tab);
    return hipGetLastError();
}

}  // namespace freqkv
