// Angles of rotary pairs, powers of two and fp16 pairs, for the kernels over 8-bit caches and those of attention weights.
#pragma once
#include "freqkv_lanes.h"

namespace freqkv {

namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int exponent_of(float x) { return (int)(__float_as_uint(x) >> 23 & 0xff) - 127; }

struct CosSin { float c, s; };
// cos and sin of pos times an angle given in quarter turns: quarters in fp64, the rest, at most an eighth of a turn, by Taylor sums in fp32 (cut off
// below 3e-9).
__device__ __forceinline__ CosSin turn(double quarters, int pos)
{
    const double t = (double)pos * quarters, k = rint(t);
    const float x = (float)(t - k) * 1.5707963267948966f, x2 = x * x;
    float s = fmaf(x2, 1.f / 362880.f, -1.f / 5040.f);
    s = fmaf(x2, s, 1.f / 120.f);
    s = fmaf(x2, s, -1.f / 6.f);
    s = fmaf(x2 * x, s, x);
    float c = fmaf(x2, -1.f / 3628800.f, 1.f / 40320.f);
    c = fmaf(x2, c, -1.f / 720.f);
    c = fmaf(x2, c, 1.f / 24.f);
    c = fmaf(x2, c, -0.5f);
    c = fmaf(x2, c, 1.f);
    const int n = (int)k;
    CosSin r = {n & 1 ? s : c, n & 1 ? c : s};
    if ((n + 1) & 2) r.c = -r.c;
    if (n & 2) r.s = -r.s;
    return r;
}

// cos and sin of a position common to the wave, of all pairs, to the wave's own part of LDS (a wave's LDS instructions take effect in order).
template <int D> __device__ __forceinline__ void wave_turns(const double* quarters, int pos, float2* own, int lane)
{
    static_for<(D / 2 + 63) / 64>([&](auto n) {
        const int j = n.value * 64 + lane;
        if (D / 2 >= 64 || j < D / 2) {
            const CosSin x = turn(quarters[j], pos);
            own[j] = float2{x.c, x.s};
        }
    });
    asm volatile("" ::: "memory");
}
// ... times those of a row from there on, of N adjacent pairs (N even): the lane's seeds
template <int D, int N> __device__ __forceinline__ void seeds(const float2* rows, const float2* own, int row, int pair, float* c, float* s)
{
    static_for<N / 2>([&](auto i) {
        const f32x4 w = *(const f32x4*)(own + pair + 2 * i.value), r = *(const f32x4*)(rows + row * (D / 2) + 2 * ((pair / 2 + i.value) ^ (row & 7)));
        static_for<2>([&](auto n) {
            constexpr int k = 2 * n.value;
            c[2 * i.value + n.value] = fmaf(w[k], r[k], -(w[k + 1] * r[k + 1]));
            s[2 * i.value + n.value] = fmaf(w[k + 1], r[k], w[k] * r[k + 1]);
        });
    });
}
// N adjacent pairs (N even) of a table of rotations.
template <int N> __device__ __forceinline__ void rotations(const float2* from, float* c, float* s)
{
    static_for<N / 2>([&](auto i) {
        const f32x4 w = *(const f32x4*)(from + 2 * i.value);
        c[2 * i.value] = w[0]; s[2 * i.value] = w[1];
        c[2 * i.value + 1] = w[2]; s[2 * i.value + 1] = w[3];
    });
}

__device__ __forceinline__ half2v halves(float a, float b)
{
    const f32x2 v = {a, b};
    return __builtin_convertvector(v, half2v);
}

}  // namespace

}  // namespace freqkv
