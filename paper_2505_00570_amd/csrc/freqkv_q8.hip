// gfx950 kernels for caches held in 8 bits.
//
// A head's rows lie as codes of one byte, int8 or e4m3 (1 sign, 4 exponent, 3 mantissa bits, largest value 448), and every block of 16 to 128 tokens of a
// head has a scale: a value is code * scale.  The scale is the smallest number by which no value of the block exceeds the largest code, of
// 8 significant bits for int8 (so that code * 127 and code * scale are exact in fp32, as is the remainder of a quotient, and with it every
// rounding of value / scale), a power of two for e4m3 (a quotient is then the value itself with another exponent).
//
//   k_quantize     rows -> codes and scales, a workgroup to a block
//   k_dequantize   codes -> rows
//   k_attend_q8    attention over the codes
#include "freqkv_internal.h"
#include "freqkv_lanes.h"
#include "freqkv_turn.h"

#include <type_traits>

namespace freqkv {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));

constexpr float kMinusBig = -1.0e30f;
constexpr float kLeastScale = 7.888609052210118e-31f;      // 2^-100
template <int FMT> constexpr float kMostCode = FMT == kInt8 ? 127.f : 448.f;

template <int FMT> __device__ __forceinline__ void values_of(uint32_t codes, float (&x)[4])
{
    if constexpr (FMT == kInt8) {
        static_for<4>([&](auto i) { x[i.value] = (float)(int)(signed char)(codes >> 8 * i.value); });
    } else {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
        x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
    }
}

// Codes of four quotients that are rounded already (int8) or that the conversion rounds, to even (e4m3).
template <int FMT> __device__ __forceinline__ uint32_t codes_of(const float (&y)[4])
{
    if constexpr (FMT == kInt8) {
        uint32_t w = 0;
        static_for<4>([&](auto i) { w |= ((uint32_t)(int)y[i.value] & 0xff) << 8 * i.value; });
        return w;
    } else {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    }
}

// Value over scale, rounded to the nearest code, a tie to the even one.  int8: the product with an inexact 1 / scale may be on the wrong side of a
// border; the remainder x - q scale is exact (see above) and says so.
template <int FMT> __device__ __forceinline__ float quotient(float x, float scale, float inverse)
{
    if constexpr (FMT == kInt8) {
        float q = rintf(x * inverse);
        const float r = fmaf(-q, scale, x), half = 0.5f * scale;
        const bool wrong = fabsf(r) > half || (fabsf(r) == half && ((int)q & 1));
        return wrong ? q + copysignf(1.f, r) : q;
    } else {
        return x * inverse;
    }
}

// The scale of a block whose largest magnitude is amax, which is finite.
template <int FMT> __device__ __forceinline__ float fresh_scale(float amax)
{
    if (amax == 0.f) return 0.f;
    float s;
    if constexpr (FMT == kInt8) {
        s = __uint_as_float(__float_as_uint(amax * (1.f / 127.f)) & 0xffff0000u);
        s = fmaxf(s, kLeastScale);
        static_for<2>([&](auto) { if (127.f * s < amax) s = __uint_as_float(__float_as_uint(s) + 0x10000u); });
    } else {
        // amax = m 2^e, 448 = 1.75 * 2^8
        const uint32_t u = __float_as_uint(amax);
        const int e = (int)(u >> 23) - 127 - ((u & 0x7fffff) > 0x600000 ? 7 : 8);
        s = e < -100 ? kLeastScale : __uint_as_float((uint32_t)(e + 127) << 23);
    }
    return s;
}

// Eight consecutive values of a row.
__device__ __forceinline__ void load8(const char* p, u32x4 (&w)[1]) { w[0] = *(const u32x4*)p; }
__device__ __forceinline__ void load8(const char* p, u32x4 (&w)[2]) { w[0] = *(const u32x4*)p; w[1] = *(const u32x4*)(p + 16); }
__device__ __forceinline__ float value8(const u32x4 (&w)[1], int i) { return __uint_as_float(i & 1 ? w[0][i / 2] & 0xffff0000u : w[0][i / 2] << 16); }
__device__ __forceinline__ float value8(const u32x4 (&w)[2], int i) { return __uint_as_float(w[i / 4][i & 3]); }

constexpr int kMoveThreads = 256;

}  // namespace

// A workgroup has one block of a head-tensor, whose new rows stay in registers between the search for their largest magnitude and their conversion: read once, written
// once, bound by memory: K and V of 8 heads of 8192 rows, bf16 to int8, 16.9 us, of bytes that a copy moves in 10.  A block that holds rows already keeps its scale, or has it doubled until the new rows fit, and its older codes are rounded again (so that
// a row's error is below one step of the block's scale, whatever the number of calls that filled it; a new scale for every row that is
// a little larger would round all rows again each time).
template <int FMT, int E, int PIECES, int THREADS>
__global__ __launch_bounds__(THREADS) void k_quantize(const Q8MoveGeom, const SlabTable rows, const SlabTable codes)
{
    const Q8MoveGeom g = first_argument<decltype(k_quantize<FMT, E, PIECES, THREADS>)>();
    __shared__ uint32_t most[THREADS / 64];
    const int tid = threadIdx.x, slab = blockIdx.y;
    const int ht = g.by_blk.quotient(blockIdx.x), i = blockIdx.x - ht * g.n_blk;
    const int b = g.by_heads.quotient(ht), h = ht - b * g.n_heads;
    int start = g.code_row;
    if (g.code_rows) {
        start = g.code_rows[b];
        if (start < 0 || start > g.capacity - g.n_rows) return;          // a sequence that is not written to
    }
    const int block = (start >> g.block_shift) + i, first = block << g.block_shift;
    const int lo = max(start, first), hi = min(start + g.n_rows, first + (1 << g.block_shift));
    if (lo >= hi) return;
    const int per_row = g.d / 8, pieces = (hi - lo) * per_row;
    const char* const from = rows.base[slab] + (long long)b * g.stride_batch + (long long)h * g.stride_head + (long long)(g.row + lo - start) * g.stride_token;
    char* const to = codes.base[slab] + (long long)b * g.code_batch + (long long)h * g.code_head + (long long)first * g.code_token;
    float* const scale_at = (slab & 1 ? g.v_scale : g.k_scale) + (long long)(slab >> 1) * g.scale_layer + (long long)b * g.scale_batch +
                            (long long)h * g.scale_head + block;
    const float held = lo > first ? *scale_at : 0.f;

    u32x4 x[PIECES][E / 2];
    uint32_t bits = 0;
    static_for<PIECES>([&](auto p) {
        const int piece = tid + p.value * THREADS;
        static_for<E / 2>([&](auto j) { x[p.value][j.value] = u32x4{0u, 0u, 0u, 0u}; });
        if (piece < pieces) {
            const int row = g.by_pieces.quotient(piece);
            load8(from + (long long)row * g.stride_token + (piece - row * per_row) * (8 * E), x[p.value]);
        }
    });
    static_for<PIECES>([&](auto p) {
        static_for<8>([&](auto j) { bits = max(bits, __float_as_uint(value8(x[p.value], j.value)) & 0x7fffffffu); });
    });
    for (int o = 32; o; o >>= 1) bits = max(bits, (uint32_t)__shfl_xor((int)bits, o));
    if constexpr (THREADS > 64) {
        if ((tid & 63) == 0) most[tid >> 6] = bits;
        __syncthreads();
        static_for<THREADS / 64>([&](auto w) { bits = max(bits, most[w.value]); });
    }
    const float amax = __uint_as_float(bits);

    // the block's scale after the call, and by how many doublings an older one grows
    float scale;
    int doubled = 0;
    if (bits >= 0x7f800000u || !(held >= 0.f && held < INFINITY)) {
        scale = __uint_as_float(0x7fc00000u);              // inf or NaN among the values: the block's values are NaN
    } else if (held == 0.f) {
        scale = fresh_scale<FMT>(amax);
    } else {
        const float limit = kMostCode<FMT> * held;
        if (limit < amax) {
            doubled = max(exponent_of(amax) - exponent_of(limit), 0);
            if (ldexpf(limit, doubled) < amax) ++doubled;
        }
        scale = ldexpf(held, doubled);
    }
    const bool none = !(scale > 0.f);
    const float inverse = none ? 0.f : 1.f / scale;
    static_for<PIECES>([&](auto p) {
        const int piece = tid + p.value * THREADS;
        if (piece >= pieces) return;
        const int row = g.by_pieces.quotient(piece);
        u32x2 w;
        static_for<2>([&](auto half) {
            float y[4];
            static_for<4>([&](auto j) { y[j.value] = none ? 0.f : quotient<FMT>(value8(x[p.value], 4 * half.value + j.value), scale, inverse); });
            w[half.value] = codes_of<FMT>(y);
        });
        *(u32x2*)(to + (long long)(row + lo - first) * g.code_token + (piece - row * per_row) * 8) = w;
    });
    if (doubled > 0 && !none) {
        const float shrink = doubled > 100 ? 0.f : ldexpf(1.f, -doubled);
        for (int piece = tid; piece < (lo - first) * per_row; piece += THREADS) {
            const int row = g.by_pieces.quotient(piece);
            u32x2* const at = (u32x2*)(to + (long long)row * g.code_token + (piece - row * per_row) * 8);
            u32x2 w = *at;
            static_for<2>([&](auto half) {
                float y[4];
                values_of<FMT>(w[half.value], y);
                static_for<4>([&](auto j) { y[j.value] = FMT == kInt8 ? rintf(y[j.value] * shrink) : y[j.value] * shrink; });
                w[half.value] = codes_of<FMT>(y);
            });
            *at = w;
        }
    }
    if (tid == 0) *scale_at = scale;
}

// Codes times scale, in fp32 (exact: 8 significant bits times 8), rounded once to the type of the rows; 16 codes a lane, several pieces of each asked for ahead of the first
// conversion.  Bound by memory (the same rows: 11.5 us, of 10).
template <int FMT, int E, int PIECES>
__global__ __launch_bounds__(kMoveThreads) void k_dequantize(const Q8MoveGeom, const SlabTable codes, const SlabTable rows)
{
    const Q8MoveGeom g = first_argument<decltype(k_dequantize<FMT, E, PIECES>)>();
    const int slab = blockIdx.y;
    const int ht = g.by_blk.quotient(blockIdx.x), i = blockIdx.x - ht * g.n_blk;
    const int b = g.by_heads.quotient(ht), h = ht - b * g.n_heads;
    const char* const from = codes.base[slab] + (long long)b * g.code_batch + (long long)h * g.code_head;
    char* const to = rows.base[slab] + (long long)b * g.stride_batch + (long long)h * g.stride_head;
    const float* const scales = (slab & 1 ? g.v_scale : g.k_scale) + (long long)(slab >> 1) * g.scale_layer + (long long)b * g.scale_batch + (long long)h * g.scale_head;
    const int per_row = g.d / 16, pieces = g.n_rows * per_row;
    u32x4 w[PIECES];
    float scale[PIECES];
    static_for<PIECES>([&](auto p) {
        const int piece = (i * PIECES + p.value) * kMoveThreads + (int)threadIdx.x;
        if (piece < pieces) {
            const int row = g.by_pieces.quotient(piece), at = row + g.code_row;
            w[p.value] = *(const u32x4*)(from + (long long)at * g.code_token + (piece - row * per_row) * 16);
            scale[p.value] = scales[at >> g.block_shift];
        }
    });
    static_for<PIECES>([&](auto p) {
        const int piece = (i * PIECES + p.value) * kMoveThreads + (int)threadIdx.x;
        if (piece >= pieces) return;
        const int row = g.by_pieces.quotient(piece);
        char* const at = to + (long long)(row + g.row) * g.stride_token + (piece - row * per_row) * (16 * E);
        static_for<E>([&](auto o) {                          // 16 bytes of the row at a time: 8 values or 4
            u32x4 y;
            static_for<4 / E>([&](auto j) {
                float x[4];
                values_of<FMT>(w[p.value][o.value * (4 / E) + j.value], x);
                static_for<4>([&](auto n) { x[n.value] *= scale[p.value]; });
                if constexpr (E == 2) {
                    static_for<2>([&](auto n) {
                        const f32x2 v = {x[2 * n.value], x[2 * n.value + 1]};
                        y[2 * j.value + n.value] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
                    });
                } else {
                    static_for<4>([&](auto n) { y[n.value] = __float_as_uint(x[n.value]); });
                }
            });
            *(u32x4*)(at + 16 * o.value) = y;
        });
    });
}

// ---------------------------------------------------------------------------------------------
// attention over the codes
// ---------------------------------------------------------------------------------------------

__global__ void k_turn_table(char* at, int d, double base)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x, half = d / 2, row = i / half, j = i - row * half;
    if (row > kTurnRows + 1) return;
    const double theta = base > 0.0 ? pow(base, -2.0 * (double)j / (double)d) : 0.0;       // no rotary embedding: every angle is zero
    if (row == 0) ((double*)at)[j] = theta * 0.6366197723675814;
    // rows 0 and 1: the steps; row r + 2: the angle of row r
    double s, c;
    sincos((double)(row == 0 ? kTurnStep : row == 1 ? 2 * kTurnStep : row - 2) * theta, &s, &c);
    const int place = row < 2 ? j : 2 * ((j / 2) ^ ((row - 2) & 7)) + j % 2;
    ((float2*)(at + d * 4))[row * half + place] = float2{(float)c, (float)s};
}

namespace {

constexpr float kSlack = 8.0f;       // log2 of the largest un-rescaled softmax weight (times at most 4 an fp16 operand)
constexpr int kReseedSteps = 32;     // steps between exact recomputations of the rows' cos/sin

// Byte CH of the codes of two rows, as fp16 (exact).  RAW, of int8: the byte plus 128, times 2^-24, as the fp16 number that has just it as its bits.
template <int FMT, int CH, bool RAW> __device__ __forceinline__ half2v pair_of(uint32_t row0, uint32_t row1)
{
    if constexpr (RAW) {
        return __builtin_bit_cast(half2v, __builtin_amdgcn_perm(row1, row0, 0x0c000c00u | (4u + CH) << 16 | CH));      // (of rows whose bytes are plus 128)
    } else if constexpr (FMT == kInt8) {
        // (code + 128) behind the byte 0x64 is 1024 + 128 + code in fp16
        const uint32_t u = __builtin_amdgcn_perm(row1, row0, 0x0c000c00u | (4u + CH) << 16 | CH) ^ 0x64806480u;
        return __builtin_bit_cast(half2v, u) - half2v{(_Float16)1152.f, (_Float16)1152.f};
    } else {
        const uint32_t u = __builtin_amdgcn_perm(row1, row0, CH < 2 ? 0x05010400u : 0x07030602u);
        return __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, 1.0f, CH & 1));
    }
}

// x is used from here on: what is made of it is not made earlier.
__device__ __forceinline__ void here(uint32_t& x) { asm volatile("" : "+v"(x)); }

// What stands behind is not done ahead of what stands before, loads from LDS among it.
__device__ __forceinline__ void apart()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// x of this lane where the banks (4 lanes of 16) are not named, else y of the lane 8 away
template <int BANKS> __device__ __forceinline__ uint32_t of_pair(uint32_t x, uint32_t y)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)y, 0x128, 0xf, BANKS, false);
}

}  // namespace

// Attention of up to 16 queries of a unit (heads that share a KV head, and of a chunk several of each) over a chunk of its rows, one pass with the running
// maximum and sum of a softmax.  A wave has two tiles of 16 rows in a step, 64 rows apart, of the four waves' 128:
//   scores     v_mfma_f32_16x16x32_f16, rows of the tile x queries.  A lane (c, g) = (lane & 15, lane >> 4) has of row c a sixteenth
//              of the channels in each half, so that a rotary pair is in one lane; codes become fp32, turn by the row's position less the last one's, and are rounded to
//              fp16 (11 bits; fp32 queries: two fp16, 22 bits).  A query is divided by a power of two that brings its largest element to 2^6 .. 2^7, so that
//              magnitudes do not matter; scale of the block and power come back in one factor per score, in fp32.
//   softmax    lane (c, g) has the scores of query c with the rows 4 g .. 4 g + 3 of both tiles: in-lane but for two exchanges.
//   values     the same instruction, channels x queries over the 32 rows: the weights are, as they lie, the second operand.  They take the block's
//              scale with them (relative to a power of two that follows the largest, so that fp16 holds them), codes are exact in fp16.
// cos/sin of a row advance by a fixed rotation from seeds made anew every kReseedSteps steps (of fp64 angles): once in a step, by its 128 rows, as the second tile's keys turn by the
// first one's angles and meet queries turned back by the 64 rows between them; with 256 channels and fp32 queries, which leave no registers for two sets of queries, for each tile.
// Bound by the rows where workgroups fill the device (32 layers of 8 KV heads of 4, 8192 rows: 101 us, 5.3 TB/s; 16 sequences of 4096 to 8192 rows 50 us), by the start of a
// workgroup, its merge and the call where they do not (8 KV heads of 6147 rows: 10.2 us).  Without copies to LDS, and keys of both tiles turned by angles of their own, all layers took 112.
// Scores of rows that a query does not see are -inf, their weights zero whatever the scale.
template <int FMT, int D, bool F32, bool ONE>
__global__ __launch_bounds__(kQ8Waves * 64, (D == 256 || F32 ? 1 : 2))
void k_attend_q8(const Q8AttGeom, const void* __restrict__ q, const TurnTable tables, float* __restrict__ part_acc, float* __restrict__ part_ml,
                 void* __restrict__ out, float* __restrict__ lse, const SlabTable tab)
{
    const Q8AttGeom g = first_argument<decltype(k_attend_q8<FMT, D, F32, ONE>)>();
    constexpr int W = kQ8Waves, NQ = kQ8Queries;
    constexpr int HC = D / 8;                        // pairs of a key that a lane has
    constexpr int PC = HC < 16 ? HC : 16, NP = HC / PC;   // in pieces of PC channels, NP to a half
    constexpr int KS = D / 32;                       // k-steps of a score
    constexpr int NV = D / 16;                       // channels of a value that a lane has = tiles of channels
    constexpr int VW = NV / 4;                       // ... in words
    constexpr bool TIGHT = D == 256;                 // few registers to spare: what need not be at once is kept apart
    typedef typename std::conditional<F32, float, uint16_t>::type T;

    constexpr int SLOTS = TIGHT && F32 ? 1 : 2;      // steps whose rows LDS holds
    constexpr int RINGS = W * SLOTS * 2 * 32 * D, RED = D + 4, ENDS = W * NQ * RED * 4, TABLES = (3 + 16) * (D / 2) * 8;
    __shared__ __attribute__((aligned(1024))) char pool[RINGS > ENDS ? RINGS : ENDS];     // rows of SLOTS steps, of each wave; then their sums
    __shared__ __attribute__((aligned(1024))) char tsm[(TABLES + 1023) / 1024 * 1024];    // the start of the tables: frequencies, rotations by a step, 16 rows
    float (*const red)[NQ][RED] = (float (*)[NQ][RED])pool;      // (four more to a row: queries in different banks)
    __shared__ float xm[W][NQ], xl[W][NQ];
    __shared__ half8 qsm[D == 256 && F32 ? 2 * KS : 1][64];
    __shared__ __attribute__((aligned(16))) float2 turns[W][D / 2];

    const int lane = threadIdx.x & 63, c = lane & 15, gq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int chunk_id = blockIdx.x, part = blockIdx.y;
    if (g.parts > 1 && gridDim.y == 1) share_out(g.parts, chunk_id, part);
    const int unit = g.by_split.quotient(chunk_id), split = chunk_id - unit * g.n_split;
    const int layer = g.by_layer.quotient(unit), rem = unit - layer * g.units_per_layer;
    const int b = g.by_kv.quotient(rem), kvh = rem - b * g.n_kv;
    const int j0 = part * NQ, queries = min(NQ, g.M - j0);
    const long long head0 = (long long)unit * g.M + j0;

    int cur_len = g.cur_len;
    if (g.cur_lens) cur_len = max(0, min(g.cur_lens[b], g.cur_len));
    // places of the queries in their chunk: of the lane's, and the least and the last of the workgroup's
    const int mine = j0 + min(c, queries - 1);
    const int place = mine - g.by_q.quotient(mine) * g.q_len;
    const int place0 = j0 - g.by_q.quotient(j0) * g.q_len;
    const bool wraps = place0 + queries > g.q_len;
    const int past = cur_len - g.q_len + 1;
    const int row0 = split * g.chunk;
    const int row_end = min(row0 + g.chunk, past + (wraps ? g.q_len - 1 : place0 + queries - 1));   // <= row0: no rows
    const int limit = min(row_end, past + place), seen = min(row_end, past + (wraps ? 0 : place0));
    const int nit = row_end > row0 ? (row_end - row0 + kQ8StepRows - 1) / kQ8StepRows : 0;

    const long long head_off = (long long)b * g.code_batch + (long long)kvh * g.code_head;
    const uint32_t row_bytes = (uint32_t)g.code_token;
    const char* const kbase = tab.base[2 * layer] + head_off;
    const char* const vbase = tab.base[2 * layer + 1] + head_off;
    const long long scale_off = (long long)layer * g.scale_layer + (long long)b * g.scale_batch + (long long)kvh * g.scale_head;
    const float* const ks = g.k_scale + scale_off;
    const float* const vs = g.v_scale + scale_off;
    const int last_block = max(row_end - 1, 0) >> g.block_shift;

    // ---- rows of a step, two tiles of 16: copied to the wave's part of LDS two steps ahead, 16 bytes a lane, whole rows side by side.  (Loaded as they are used, with the four
    // lanes that share a row 16 apart, a load's 64 pieces were 64 requests of the first-level cache.)  Keys lie with their pieces of 16 bytes turned by row, so that lanes that
    // read the same piece of eight rows find them in different banks.  Rows past the end are the last one's again.
    constexpr int IN = D / 64, PIECES = D / 16, ROWS = 64 / PIECES;     // copies of a tile, pieces of a row, rows of a copy
    constexpr int TILE = 16 * D, SLOT = 2 * TILE;
    const int wrow = row0 + 16 * wave;               // first row of the wave's first tile
    char* const ring = pool + wave * SLOTS * 2 * SLOT;       // [slot][keys, values][tile][row][D]
    typedef __attribute__((address_space(3))) char* lptr_t;
    const uint32_t ring_lds = (uint32_t)(uintptr_t)(lptr_t)ring;
    auto slot_of = [](int it) { return SLOTS == 2 ? (it & 1) * 2 * SLOT : 0; };
    auto turned = [](int row, int piece) { return piece ^ (D == 64 ? row >> 1 & 3 : row & 7); };
    // a lane's copies of a step: where they lie, from the step's first row on (the last step's rows past the end: the last row's again)
    uint32_t key_at[2 * IN], val_at[2 * IN];
    static_for<2 * IN>([&](auto i) {
        const int row = (i.value % IN) * ROWS + lane / PIECES, piece = lane % PIECES;
        const uint32_t at = (uint32_t)(16 * wave + i.value / IN * kTurnStep + row) * row_bytes;
        key_at[i.value] = at + (uint32_t)(turned(row, piece) * 16);
        val_at[i.value] = at + (uint32_t)(piece * 16);
    });
    auto ask = [&](int it, uint32_t lds, const char* base, const uint32_t (&at)[2 * IN], auto is_keys) {
        const int first = row0 + it * kQ8StepRows;
        const char* const from = base + (uint32_t)first * row_bytes;
        if (first + kQ8StepRows <= row_end) {
            static_for<2 * IN>([&](auto i) { lds_dma16(lds + (uint32_t)(slot_of(it) + i.value * 1024), from, at[i.value]); });
        } else {
            static_for<2 * IN>([&](auto i) {
                const int r = (i.value % IN) * ROWS + lane / PIECES, piece = lane % PIECES;
                const int row = min(16 * wave + i.value / IN * kTurnStep + r, row_end - 1 - first);
                lds_dma16(lds + (uint32_t)(slot_of(it) + i.value * 1024), from,
                          (uint32_t)row * row_bytes + (uint32_t)((decltype(is_keys)::value ? turned(r, piece) : piece) * 16));
            });
        }
    };
    auto ask_keys = [&](int it) { ask(it, ring_lds, kbase, key_at, IC<1>{}); };
    auto ask_values = [&](int it) { ask(it, ring_lds + SLOT, vbase, val_at, IC<0>{}); };
    auto landed = [](auto n) { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(decltype(n)::value) : "memory"); };      // all copies but the last n
    auto words = [](const char* p, auto& to, auto n) {
        if constexpr (decltype(n)::value == 4) {
            const u32x4 w = *(const u32x4*)p;
            static_for<4>([&](auto i) { to[i.value] = w[i.value]; });
        } else if constexpr (decltype(n)::value == 2) {
            const u32x2 w = *(const u32x2*)p;
            static_for<2>([&](auto i) { to[i.value] = w[i.value]; });
        } else {
            to[0] = *(const uint32_t*)p;
        }
    };
    struct Keys { uint32_t lo[NP][PC / 4], up[NP][PC / 4]; };
    auto load_keys = [&](const char* tile, Keys& key) {
        static_for<NP>([&](auto p) {
            constexpr int HALF = PIECES / 2;
            if constexpr (PC == 16) {
                words(tile + c * D + turned(c, gq + 4 * p.value) * 16, key.lo[p.value], IC<4>{});
                words(tile + c * D + turned(c, HALF + gq + 4 * p.value) * 16, key.up[p.value], IC<4>{});
            } else {
                words(tile + c * D + turned(c, gq >> 1) * 16 + (gq & 1) * 8, key.lo[p.value], IC<2>{});
                words(tile + c * D + turned(c, HALF + (gq >> 1)) * 16 + (gq & 1) * 8, key.up[p.value], IC<2>{});
            }
        });
    };
    uint32_t val[2][4][VW];                          // D = 128: [half][row of the four] as they lie, then [tile][row]
    auto load_values = [&](const char* slot) {
        if constexpr (D == 128) {
            // 16 bytes a lane, 8 lanes to a row; lanes with 8 in their index have the second tile's rows
            const char* const p = slot + (lane >> 3 & 1) * TILE + 4 * gq * D + 16 * (lane & 7);
            static_for<4>([&](auto r) {
                const u32x4 w = *(const u32x4*)(p + r.value * D);
                static_for<2>([&](auto i) { val[0][r.value][i.value] = w[i.value]; val[1][r.value][i.value] = w[2 + i.value]; });
            });
        } else {
            static_for<2>([&](auto t) {
                static_for<4>([&](auto r) { words(slot + t.value * TILE + (4 * gq + r.value) * D + NV * c, val[t.value][r.value], IC<VW>{}); });
            });
        }
    };
    auto block_of = [&](int it, int t) { return min((wrow + it * kQ8StepRows + t * kTurnStep) >> g.block_shift, last_block); };
    // first channel of the lane `c` of a tile of values: the tile `ct` has the channel ct behind it
    auto channel0 = [](int c) { return D == 128 ? 16 * (c & 7) + 8 * (c >> 3) : NV * c; };

    // ---- the start: tables, a fourth of them each wave, and queries, each wave its own, in the last slot; then the rows of the first step.  All are copies: what came back to
    // registers would be awaited with all copies asked for before it, which for the first rows, asked for by all workgroups at once, are microseconds.
    constexpr int N = 2 * IN;                        // copies of a step's keys, and of its values
    constexpr int QB = D * (int)sizeof(T), QPIECES = QB / 16, QROWS = 64 / QPIECES, QIN = NQ / QROWS;    // of a query; copies of all
    char* const qraw = ring + (SLOTS - 1) * 2 * SLOT;
    static_assert(NQ * QB <= 2 * SLOT, "a slot holds the queries");
    constexpr int TIN = (TABLES + 1023) / 1024;
    static_for<(TIN + W - 1) / W>([&](auto i) {
        const int part = i.value * W + wave;
        if (part < TIN) lds_dma16((uint32_t)(uintptr_t)(lptr_t)tsm + (uint32_t)part * 1024, tables.quarters, (uint32_t)(part * 1024 + lane * 16));
    });
    static_for<QIN>([&](auto i) {
        const int r = i.value * QROWS + lane / QPIECES, piece = (lane % QPIECES) ^ (r & 7);
        lds_dma16(ring_lds + (uint32_t)((SLOTS - 1) * 2 * SLOT + i.value * 1024), (const char*)q + head0 * QB, (uint32_t)(min(r, queries - 1) * QB + piece * 16));
    });
    if (SLOTS == 2 && nit > 0) {
        ask_keys(0);
        ask_values(0);
        landed(IC<2 * N>{});
    } else {
        landed(IC<0>{});
    }
    lds_barrier();
    const struct { const double* quarters; const float2 *step, *step2, *rows; } rt = {(const double*)tsm, (const float2*)(tsm + D * 4), (const float2*)(tsm + D * 8),
                                                                                   (const float2*)(tsm + D * 12)};

    // ---- the rotary state of the lane's pairs
    float co[HC], si[HC], cd[TIGHT ? 8 : HC], sd[TIGHT ? 8 : HC];
    auto pair_index = [&](int i) { return PC * (gq + 4 * (i / PC)) + i % PC; };
    float2* const own = turns[wave];
    auto seed = [&](int it) {
        wave_turns<D>(rt.quarters, wrow + it * kQ8StepRows - (cur_len - 1), own, lane);
        static_for<NP>([&](auto p) { seeds<D, PC>(rt.rows, own, c, PC * (gq + 4 * p.value), co + PC * p.value, si + PC * p.value); });
    };
    // PAIRED: the keys of a step's two tiles turn by the same angle, and the second tile meets queries that are turned back by the rows between them
    constexpr bool PAIRED = !(TIGHT && F32);
    const float2* const advance = PAIRED ? rt.step2 : rt.step;
    // (TIGHT: the rotations by a step stay in LDS)
    if constexpr (!TIGHT) static_for<NP>([&](auto p) { rotations<PC>(advance + PC * (gq + 4 * p.value), cd + PC * p.value, sd + PC * p.value); });
    seed(0);

    // ---- the lane's query c: channels of the group gq, turned by its place less the last one's
    constexpr bool QLDS = TIGHT && F32;              // (in LDS there: all waves have the same)
    constexpr int SETS = PAIRED ? 2 : 1;
    half8 qh[SETS][QLDS ? 1 : KS], ql[SETS][F32 && !QLDS ? KS : 1];
    float qfactor;
    {
        float a[HC], bb[HC], most = 0.f;
        constexpr int CH = 16 / (int)sizeof(T);       // channels to 16 bytes
        static_for<HC / CH>([&](auto i) {
            const int piece = pair_index(i.value * CH) / CH;
            const u32x4 x = *(const u32x4*)(qraw + c * QB + (piece ^ (c & 7)) * 16), y = *(const u32x4*)(qraw + c * QB + ((QPIECES / 2 + piece) ^ (c & 7)) * 16);
            static_for<CH>([&](auto j) {
                constexpr int to = i.value * CH + j.value;
                a[to] = __uint_as_float(F32 ? x[j.value % 4] : j.value & 1 ? x[j.value / 2] & 0xffff0000u : x[j.value / 2] << 16);
                bb[to] = __uint_as_float(F32 ? y[j.value % 4] : j.value & 1 ? y[j.value / 2] & 0xffff0000u : y[j.value / 2] << 16);
                most = fmaxf(most, fmaxf(fabsf(a[to]), fabsf(bb[to])));
            });
        });
        most = fold<32>(fold<16>(most, Max{}), Max{});
        const int e = max(-110, min(exponent_of(most), 126)) - 6;        // largest element -> 2^6 .. 2^7
        qfactor = ldexpf(g.qscale, e);
        const float down = ldexpf(1.f, -e);
        static_for<HC>([&](auto i) { a[i.value] *= down; bb[i.value] *= down; });
        if (g.q_len > 1) {
            static_for<HC>([&](auto i) {
                const float x = a[i.value], y = bb[i.value];
                const CosSin t = turn(rt.quarters[pair_index(i.value)], place + 1 - g.q_len);
                a[i.value] = fmaf(x, t.c, -(y * t.s));
                bb[i.value] = fmaf(y, t.c, x * t.s);
                if constexpr (i.value % 4 == 3) __builtin_amdgcn_sched_barrier(0);        // (all at once, they take more registers than there are)
            });
        }
        static_for<SETS>([&](auto set) {
            if constexpr (set.value > 0) {
                static_for<NP>([&](auto p) {
                    float sc[PC], ss[PC];
                    rotations<PC>(rt.step + PC * (gq + 4 * p.value), sc, ss);
                    static_for<PC>([&](auto i) {
                        constexpr int at = PC * p.value + i.value;
                        const float x = a[at], y = bb[at];
                        a[at] = fmaf(x, sc[i.value], y * ss[i.value]);
                        bb[at] = fmaf(y, sc[i.value], -(x * ss[i.value]));
                    });
                });
            }
            static_for<KS>([&](auto k) {
                half8 hi, lo;
                static_for<8>([&](auto i) {
                    constexpr int at = k.value % (KS / 2) * 8 + i.value;
                    const float x = k.value < KS / 2 ? a[at] : bb[at];
                    hi[i.value] = (_Float16)x;
                    lo[i.value] = (_Float16)(x - (float)(_Float16)x);
                });
                if constexpr (QLDS) {
                    if (wave == k.value % W) { qsm[k.value][lane] = hi; qsm[KS + k.value][lane] = lo; }
                } else {
                    qh[set.value][k.value] = hi;
                    if constexpr (F32) ql[set.value][k.value] = lo;
                }
            });
        });
        if constexpr (QLDS) lds_barrier();
    }

    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // (queries read, before rows are written there)
    if (SLOTS == 2 && nit > 1) {
        ask_keys(1);
        ask_values(1);
    }

    float m = kMinusBig, lsum = 0.f, vref = 0.f;     // vref: the power of two that the sums are relative to
    f32x4 acc[NV];
    static_for<NV>([&](auto ct) { acc[ct.value] = f32x4{0.f, 0.f, 0.f, 0.f}; });
    // RAW: int8 codes go to the matrix cores as bytes plus 128, times 2^-24 (the numbers below fp16's normal ones: no conversion), and what the 128 add to each sum, the weights' sum times
    // 128, is added up beside.  Fp32 queries would lose two of their bits by the difference.
    constexpr bool RAW = FMT == kInt8 && !F32;
    f32x4 off = {0.f, 0.f, 0.f, 0.f};

    for (int it = 0; it < nit; ++it) {
        if (it > 0 && it % kReseedSteps == 0) seed(it);
        // behind the step's keys were asked for: its values, and keys and values of the next step
        if constexpr (SLOTS == 1) {
            ask_keys(it);
            ask_values(it);
            landed(IC<N>{});
        } else if (it + 1 < nit) {
            landed(IC<3 * N>{});
        } else {
            landed(IC<N>{});
        }
        const char* const kslot = ring + slot_of(it);
        const float kscale[2] = {ks[block_of(it, 0)], ks[block_of(it, 1)]};
        const float vscale[2] = {vs[block_of(it, 0)], vs[block_of(it, 1)]};
        // ---- scores
        float ka[4], kb[4];
        uint32_t ln = lane;
        if constexpr (TIGHT) here(ln);                   // (what is read from LDS is read in every step, and not kept in registers from before the loop)
        f32x4 sc[2];
        static_for<2>([&](auto t) {
            sc[t.value] = f32x4{0.f, 0.f, 0.f, 0.f};
            Keys key;
            load_keys(kslot + t.value * TILE, key);
            static_for<KS / 2>([&](auto k) {             // eight pairs: a k-step of the lower half and one of the upper
                half8 kh[2], kl[2];
                if constexpr (TIGHT && (!PAIRED || t.value == 1)) {
                    static_for<4>([&](auto n) {
                        const f32x4 w = *(const f32x4*)(advance + PC * ((int)(ln >> 4) + 4 * (8 * k.value / PC)) + (8 * k.value + 2 * n.value) % PC);
                        cd[2 * n.value] = w[0]; sd[2 * n.value] = w[1];
                        cd[2 * n.value + 1] = w[2]; sd[2 * n.value + 1] = w[3];
                    });
                }
                static_for<4>([&](auto n) {
                    constexpr int i = 8 * k.value + 2 * n.value, w = i / 4;
                    if constexpr (n.value % 2 == 0) {
                        if constexpr (TIGHT) {
                            here(key.lo[w / (PC / 4)][w % (PC / 4)]);
                            here(key.up[w / (PC / 4)][w % (PC / 4)]);
                        }
                        values_of<FMT>(key.lo[w / (PC / 4)][w % (PC / 4)], ka);
                        values_of<FMT>(key.up[w / (PC / 4)][w % (PC / 4)], kb);
                    }
                    float lo[2], up[2];
                    static_for<2>([&](auto o) {
                        constexpr int j = 2 * (n.value % 2) + o.value, at = i + o.value, by = TIGHT ? at % 8 : at;
                        lo[o.value] = fmaf(ka[j], co[at], -(kb[j] * si[at]));
                        up[o.value] = fmaf(kb[j], co[at], ka[j] * si[at]);
                        if constexpr (!PAIRED || t.value == 1) {
                            const float cn = fmaf(co[at], cd[by], -(si[at] * sd[by]));
                            si[at] = fmaf(si[at], cd[by], co[at] * sd[by]);
                            co[at] = cn;
                        }
                    });
                    const half2v l = halves(lo[0], lo[1]), u = halves(up[0], up[1]);
                    kh[0][2 * n.value] = l[0]; kh[0][2 * n.value + 1] = l[1];
                    kh[1][2 * n.value] = u[0]; kh[1][2 * n.value + 1] = u[1];
                    if constexpr (F32) {
                        const half2v l2 = halves(lo[0] - (float)l[0], lo[1] - (float)l[1]), u2 = halves(up[0] - (float)u[0], up[1] - (float)u[1]);
                        kl[0][2 * n.value] = l2[0]; kl[0][2 * n.value + 1] = l2[1];
                        kl[1][2 * n.value] = u2[0]; kl[1][2 * n.value + 1] = u2[1];
                    }
                });
                static_for<2>([&](auto h) {
                    constexpr int at = k.value + h.value * (KS / 2);
                    half8 qa, qb;
                    if constexpr (QLDS) { qa = qsm[at][ln]; qb = qsm[KS + at][ln]; }
                    else { qa = qh[PAIRED ? t.value : 0][at]; if constexpr (F32) qb = ql[PAIRED ? t.value : 0][at]; }
                    if constexpr (F32) {
                        sc[t.value] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kl[h.value], qa, sc[t.value], 0, 0, 0);
                        sc[t.value] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh[h.value], qb, sc[t.value], 0, 0, 0);
                    }
                    sc[t.value] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh[h.value], qa, sc[t.value], 0, 0, 0);
                });
                if constexpr (TIGHT) apart();
            });
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (read, before they are written again)
        if (SLOTS == 2 && it + 2 < nit) ask_keys(it + 2);
        static_for<2>([&](auto t) { sc[t.value] *= kscale[t.value] * qfactor; });
        // rows that not all queries see: which of the lane's (bit 4 t + r) its query does not
        const bool tail = row0 + (it + 1) * kQ8StepRows > seen;
        uint32_t hidden = 0;
        if (tail) {
            static_for<8>([&](auto i) {
                const bool no = wrow + it * kQ8StepRows + i.value / 4 * kTurnStep + 4 * gq + i.value % 4 >= limit;
                hidden |= no ? 1u << i.value : 0u;
                sc[i.value / 4][i.value % 4] = no ? -INFINITY : sc[i.value / 4][i.value % 4];
            });
        }
        // ---- softmax: the reference point m only moves when a score exceeds it by more than 2^kSlack
        float mx = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])), fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
        mx = fold<32>(fold<16>(mx, Max{}), Max{});
        const bool grow = mx > m + kSlack;
        if (__builtin_amdgcn_ballot_w64(grow) != 0) {
            const float mn = grow ? mx : m, f = exp2_fast(m - mn);
            m = mn;
            lsum *= f;
            static_for<NV>([&](auto ct) { acc[ct.value] *= f; });
            if constexpr (RAW) off *= f;
        }
        const float larger = fmaxf(vscale[0], vscale[1]);
        if (larger > 4.f * vref && larger < INFINITY) {
            const float to = __uint_as_float(__float_as_uint(larger) & 0x7f800000u), f = vref / to;
            vref = to;
            static_for<NV>([&](auto ct) { acc[ct.value] *= f; });
            if constexpr (RAW) off *= f;
        }
        const float per = vref > 0.f ? 1.f / vref : 0.f;
        half8 ph, pl;
        float x[8];
        static_for<8>([&](auto i) {
            const float p = exp2_fast(sc[i.value / 4][i.value % 4] - m);
            lsum += p;
            x[i.value] = p * (vscale[i.value / 4] * per);
        });
        if (tail) static_for<8>([&](auto i) { x[i.value] = hidden >> i.value & 1 ? 0.f : x[i.value]; });      // (a scale may be NaN)
        static_for<4>([&](auto i) {
            const half2v h = halves(x[2 * i.value], x[2 * i.value + 1]);
            ph[2 * i.value] = h[0]; ph[2 * i.value + 1] = h[1];
            if constexpr (F32) {
                const half2v l = halves(x[2 * i.value] - (float)h[0], x[2 * i.value + 1] - (float)h[1]);
                pl[2 * i.value] = l[0]; pl[2 * i.value + 1] = l[1];
            }
        });
        // ---- values: behind them were asked for keys and values of the next step, and keys of the one after
        if (SLOTS == 2 && it + 2 < nit) landed(IC<3 * N>{});
        else if (SLOTS == 2 && it + 1 < nit) landed(IC<2 * N>{});
        else landed(IC<0>{});
        load_values(kslot + SLOT);
        if constexpr (D == 128) {
            // (as loaded: [lower or upper 8 channels][row])  Lanes 8 apart have the same 16 channels of the two tiles: after the exchange each has half of the channels of both.
            static_for<4>([&](auto r) {
                static_for<2>([&](auto w) {
                    const uint32_t lo = val[0][r.value][w.value], up = val[1][r.value][w.value];
                    val[0][r.value][w.value] = of_pair<0xc>(lo, up);
                    val[1][r.value][w.value] = of_pair<0x3>(up, lo);
                });
            });
        }
        if constexpr (RAW) {
            static_for<8>([&](auto r) { static_for<VW>([&](auto w) { val[r.value / 4][r.value % 4][w.value] ^= 0x80808080u; }); });
            half8 offset;
            static_for<8>([&](auto i) { offset[i.value] = __builtin_bit_cast(_Float16, (uint16_t)128); });
            off = __builtin_amdgcn_mfma_f32_16x16x32_f16(offset, ph, off, 0, 0, 0);
        }
        static_for<VW>([&](auto w) {
            if constexpr (TIGHT) static_for<8>([&](auto r) { here(val[r.value / 4][r.value % 4][w.value]); });
            static_for<4>([&](auto ch) {
                half8 a;
                static_for<4>([&](auto r) {
                    constexpr int t = r.value / 2, n = r.value % 2 * 2;
                    const half2v x = pair_of<FMT, ch.value, RAW>(val[t][n][w.value], val[t][n + 1][w.value]);
                    a[2 * r.value] = x[0];
                    a[2 * r.value + 1] = x[1];
                });
                constexpr int ct = 4 * w.value + ch.value;
                if constexpr (F32) acc[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, pl, acc[ct], 0, 0, 0);
                acc[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, ph, acc[ct], 0, 0, 0);
            });
            if constexpr (TIGHT) apart();
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (SLOTS == 2 && it + 2 < nit) ask_values(it + 2);
    }

    // ---- the waves' states: common reference point, sums, results of the chunk
    lsum = fold<32>(fold<16>(lsum, Add{}), Add{});
    if (gq == 0) xm[wave][c] = m;
    lds_barrier();
    float M = xm[0][c];
    static_for<W - 1>([&](auto w) { M = fmaxf(M, xm[w.value + 1][c]); });
    const float f = exp2_fast(m - M);
    if (gq == 0) xl[wave][c] = lsum * f;
    const float ends = f * vref;
    if (c < queries) {
        static_for<NV / 4>([&](auto ct) {
            static_for<4>([&](auto r) {
                f32x4 x;
                static_for<4>([&](auto i) {
                    const float y = acc[4 * ct.value + i.value][r.value];
                    x[i.value] = (RAW ? (y - off[r.value]) * 16777216.f : y) * ends;
                });
                *(f32x4*)&red[wave][c][channel0(4 * gq + r.value) + 4 * ct.value] = x;
            });
        });
    }
    lds_barrier();
    for (int idx = threadIdx.x; idx < queries * (D / 2); idx += W * 64) {
        const int j = idx / (D / 2), ch = 2 * (idx - j * (D / 2));
        f32x2 sum = {0.f, 0.f};
        static_for<W>([&](auto w) { sum += *(const f32x2*)&red[w.value][j][ch]; });
        if constexpr (ONE) {
            float L = 0.f;
            static_for<W>([&](auto w) { L += xl[w.value][j]; });
            store2((T*)out + (head0 + j) * D + ch, L == 0.f ? 0.f : sum[0] / L, L == 0.f ? 0.f : sum[1] / L);
        } else {
            *(f32x2*)(part_acc + ((head0 + j) * g.n_split + split) * D + ch) = sum;
        }
    }
    if ((int)threadIdx.x < queries) {
        const int j = threadIdx.x;
        float Mj = xm[0][j], L = 0.f;
        static_for<W>([&](auto w) { Mj = fmaxf(Mj, xm[w.value][j]); L += xl[w.value][j]; });
        if constexpr (ONE) {
            if (lse) lse[head0 + j] = 0.6931471805599453f * (Mj + log2f(L));
        } else {
            *(f32x2*)(part_ml + ((head0 + j) * g.n_split + split) * 2) = f32x2{Mj, L};
        }
    }
}

// ---------------------------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------------------------

template <int FMT, int E>
static hipError_t launch_quantize_t(const SlabTable& rows, const SlabTable& codes, const Q8MoveGeom& g, int slabs, hipStream_t st)
{
    const dim3 grid((unsigned)(g.n_blk * g.hts), (unsigned)slabs);
    const int tokens = 1 << g.block_shift, pieces = (tokens < g.n_rows ? tokens : g.n_rows) * (g.d / 8), need = (pieces + kMoveThreads - 1) / kMoveThreads;
    auto launch_of = [&](auto pieces, auto threads) {
        hipLaunchKernelGGL((k_quantize<FMT, E, decltype(pieces)::value, decltype(threads)::value>), grid, dim3(threads.value), 0, st, g, rows, codes);
        return hipGetLastError();
    };
    auto launch = [&](auto n) { return launch_of(n, IC<kMoveThreads>{}); };
    // a wave to a block where it has a piece for each lane, at most: no barrier, and a fourth of the waves (a token of 32 layers x 8 sequences x 8 heads: 6.7 us, of four waves 9.1)
    if (pieces <= 64) return launch_of(IC<1>{}, IC<64>{});
    if (need <= 1) return launch(IC<1>{});
    if (need <= 2) return launch(IC<2>{});
    if (need <= 4) return launch(IC<4>{});
    if (need <= 8) return launch(IC<8>{});
    return need <= 16 ? launch(IC<16>{}) : hipErrorInvalidValue;
}

hipError_t launch_quantize(const SlabTable& rows, const SlabTable& codes, const Q8MoveGeom& g, int slabs, hipStream_t st)
{
    if (g.format == kInt8) return g.elem_bytes == 2 ? launch_quantize_t<kInt8, 2>(rows, codes, g, slabs, st) : launch_quantize_t<kInt8, 4>(rows, codes, g, slabs, st);
    return g.elem_bytes == 2 ? launch_quantize_t<kE4M3, 2>(rows, codes, g, slabs, st) : launch_quantize_t<kE4M3, 4>(rows, codes, g, slabs, st);
}

hipError_t launch_dequantize(const SlabTable& codes, const SlabTable& rows, const Q8MoveGeom& g, int slabs, hipStream_t st)
{
    const dim3 grid((unsigned)(g.n_blk * g.hts), (unsigned)slabs), block(kMoveThreads);
    auto launch = [&](auto fmt, auto e) {
        hipLaunchKernelGGL((k_dequantize<decltype(fmt)::value, decltype(e)::value, kDequantPieces>), grid, block, 0, st, g, codes, rows);
        return hipGetLastError();
    };
    if (g.format == kInt8) return g.elem_bytes == 2 ? launch(IC<kInt8>{}, IC<2>{}) : launch(IC<kInt8>{}, IC<4>{});
    return g.elem_bytes == 2 ? launch(IC<kE4M3>{}, IC<2>{}) : launch(IC<kE4M3>{}, IC<4>{});
}

hipError_t launch_turn_table(void* at, int d, double base, hipStream_t st)
{
    hipLaunchKernelGGL(k_turn_table, dim3((unsigned)((2 + kTurnRows) * (d / 2) + 255) / 256), dim3(256), 0, st, (char*)at, d, base);
    return hipGetLastError();
}

template <int FMT, int D>
static hipError_t launch_q8_d(const SlabTable& tab, const Q8AttGeom& g, const void* q, const TurnTable& rt, float* part_acc, float* part_ml, void* out,
                              float* lse, hipStream_t st)
{
    const long long chunks = (long long)g.units * g.n_split;
    const dim3 grid = chunks * g.parts < 1 << 23 ? dim3((unsigned)(chunks * g.parts)) : dim3((unsigned)chunks, (unsigned)g.parts);
    auto launch = [&](auto f32, auto one) {
        hipLaunchKernelGGL((k_attend_q8<FMT, D, decltype(f32)::value != 0, decltype(one)::value != 0>), grid, dim3(kQ8Waves * 64), 0, st, g, q, rt,
                           part_acc, part_ml, out, lse, tab);
        return hipGetLastError();
    };
    if (g.n_split == 1) return g.f32 ? launch(IC<1>{}, IC<1>{}) : launch(IC<0>{}, IC<1>{});
    return g.f32 ? launch(IC<1>{}, IC<0>{}) : launch(IC<0>{}, IC<0>{});
}

hipError_t launch_attend_q8(const SlabTable& tab, const Q8AttGeom& g, const void* q, const TurnTable& rt, float* part_acc, float* part_ml, void* out,
                            float* lse, hipStream_t st)
{
    if (g.units < 1 || g.n_split < 1 || g.chunk < 1 || g.chunk % kQ8StepRows || g.cur_len < 1 || g.M < 1 || g.parts != (g.M + kQ8Queries - 1) / kQ8Queries)
        return hipErrorInvalidValue;
    if ((long long)(g.n_split - 1) * g.chunk >= g.cur_len || (long long)g.n_split * g.chunk < g.cur_len) return hipErrorInvalidValue;
    auto by_d = [&](auto fmt) {
        constexpr int F = decltype(fmt)::value;
        switch (g.d) {
            case 64:  return launch_q8_d<F, 64>(tab, g, q, rt, part_acc, part_ml, out, lse, st);
            case 128: return launch_q8_d<F, 128>(tab, g, q, rt, part_acc, part_ml, out, lse, st);
            case 256: return launch_q8_d<F, 256>(tab, g, q, rt, part_acc, part_ml, out, lse, st);
            default:  return hipErrorInvalidValue;
        }
    };
    return g.format == kInt8 ? by_d(IC<kInt8>{}) : by_d(IC<kE4M3>{});
}

}  // namespace freqkv
