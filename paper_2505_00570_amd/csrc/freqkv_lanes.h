// What the kernels of attention and of 8-bit caches share: vector types, loops over constants, exchanges between the lanes of a wave.
#pragma once
#include "freqkv_internal.h"

namespace freqkv {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int I> struct IC { static constexpr int value = I; };
template <int N, int I = 0, class F>
__device__ __forceinline__ void static_for(F&& f)
{
    if constexpr (I < N) {
        f(IC<I>{});
        static_for<N, I + 1>(f);
    }
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Lane exchange inside a row of 16 lanes through the data-parallel primitives (no LDS traffic).
template <int CTRL> __device__ __forceinline__ float dpp(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
// Barrier for what the workgroup keeps in LDS.  (The other one would wait for all loads as well, those of rows past the end of a chunk among
// them, which nobody uses: 2000 cycles at the end of every workgroup.)
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// x op (x of the lane O further or nearer), in every lane; O = 4, 8, 16 or 32.  On the vector units: a shuffle goes through LDS, and
// a chain of them is what the end of a short call waits for.
template <int O, class F> __device__ __forceinline__ float fold(float x, F&& op)
{
    if constexpr (O == 4) {
        return op(x, dpp<0x141>(dpp<0x1B>(x)));  // mirrored in the quad [3,2,1,0], then in the half row
    } else if constexpr (O == 8) {
        return op(x, dpp<0x128>(x));             // the row of 16 turned by 8
    } else if constexpr (O == 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
    } else {
        static_assert(O == 32);
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
    }
}
// ... over the lanes O, 2 O, ... 32 apart
template <int O, class F> __device__ __forceinline__ float fold_from(float x, F&& op)
{
    x = fold<O>(x, op);
    if constexpr (O < 32) x = fold_from<2 * O>(x, op);
    return x;
}
// ... over all 64 lanes
template <class F> __device__ __forceinline__ float wave_fold(float x, F&& op)
{
    x = op(x, dpp<0xB1>(x));                     // lanes 1, 2 and 4 apart (quads exchange halves, half rows of 8 mirror)
    x = op(x, dpp<0x4E>(x));
    x = op(x, dpp<0x141>(x));
    return fold_from<8>(x, op);
}
struct Add { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct Max { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };

// Two adjacent results, rounded once.
__device__ __forceinline__ void store2(uint16_t* p, float a, float b)
{
    f32x2 v = {a, b};
    *(uint32_t*)p = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ void store2(float* p, float a, float b) { *(f32x2*)p = f32x2{a, b}; }

// Workgroups that read the same rows, for query heads beyond those of one, follow each other on one XCD (they are dealt round-robin to 8) and
// find them in its L2 (8 query heads to each of 4 KV heads x 8192 rows x 32 layers 181 -> 159 us, of 8 x 4000 x 32 167 -> 155; with all
// first parts ahead of all second ones, rows came from memory again).
[[maybe_unused]] __device__ __forceinline__ void share_out(int parts, int& chunk_id, int& part)
{
    const int chunks = (int)gridDim.x / parts, whole = chunks & ~7, at = chunk_id - whole * parts;
    if (at < 0) {
        const int grp = chunk_id / (8 * parts), local = chunk_id - grp * 8 * parts;
        part = local >> 3;
        chunk_id = grp * 8 + (local & 7);
    } else {
        part = at / (chunks - whole);
        chunk_id = whole + at - part * (chunks - whole);
    }
}

}  // namespace

}  // namespace freqkv
