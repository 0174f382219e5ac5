// What the appends to the paged caches share (cache.hip, latent.hip): e4m3 values and their scales,
// rotation by a position.
#pragma once

#include "paged.h"

namespace cospec {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float floatx2;

constexpr float kLowestScale = 7.888609052210118e-31f;   // 2^-100

__device__ inline uint32_t bf16_pair(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
}

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Four values -> four e4m3 bytes, round to nearest even, NaN beyond the largest.
__device__ inline uint32_t f8_quad(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

__device__ inline uint32_t f8_byte(float a) {
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(a, a, 0, false)) & 0xffu;
}

__device__ inline float f8_value(uint32_t byte) {
    return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(byte), 0);
}

// Four e4m3 bytes, each times f (a power of two), rounded anew.
__device__ inline uint32_t f8_rescaled(uint32_t w, float f) {
    const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
    const floatx2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
    return f8_quad(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}

// The smallest power of two s >= 2^-100 with amax <= 448 s: 448 is 1.75 * 2^8.
__device__ inline float scale_for(float amax) {
    const uint32_t w = __float_as_uint(amax);
    const int e = static_cast<int>(w >> 23) - 127 - 8 + ((w & 0x7fffffu) > 0x600000u);
    return e < -100 ? kLowestScale : __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}

// The power of two of a scale (its mantissa bits are not used).
__device__ inline float power_of(float s) { return __uint_as_float(__float_as_uint(s) & 0x7f800000u); }

// cos and sin of 2 pi f, |f| <= 1/2.  The nearest quarter turn is taken off, which leaves x, |x| <= pi / 4,
// for the Taylor sums of sin to x^9 and cos to x^10 (the next terms are below 2e-9 and 2e-10);
// the quarter turns swap them and set the signs.
__device__ inline float2 cos_sin_turns(float f) {
    const float q = rintf(4.f * f);
    const float x = 6.28318530717958648f * fmaf(q, -0.25f, f), z = x * x;
    float s = fmaf(z, 2.75573192e-6f, -1.98412698e-4f);
    s = fmaf(z, s, 8.33333333e-3f);
    s = fmaf(z, s, -1.66666667e-1f);
    s = fmaf(z * x, s, x);
    float c = fmaf(z, -2.75573192e-7f, 2.48015873e-5f);
    c = fmaf(z, c, -1.38888889e-3f);
    c = fmaf(z, c, 4.16666667e-2f);
    c = fmaf(z, c, -0.5f);
    c = fmaf(z, c, 1.f);
    const int n = static_cast<int>(q);
    const float u = n & 1 ? s : c, v = n & 1 ? c : s;
    return make_float2(__uint_as_float(__float_as_uint(u) ^ (((n + 1) & 2) ? 0x80000000u : 0u)),
                       __uint_as_float(__float_as_uint(v) ^ ((n & 2) ? 0x80000000u : 0u)));
}

// Turns of a pair per position, in double precision, and cos and sin at a position: the product is
// reduced to a fraction of a turn in double precision (far positions then lose nothing; the rest,
// sine and cosine of a fraction, is fp32).
__device__ inline double turns_of(float inv_freq) { return static_cast<double>(inv_freq) * 0.15915494309189535; }

__device__ inline float2 turn(int64_t position, double turns) {
    const double t = static_cast<double>(position) * turns;
    return cos_sin_turns(static_cast<float>(t - rint(t)));
}

__device__ inline float finite_abs(float x) {
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.f;     // false for NaN too
}

// A token's head of D components is handled in units of sixteen: two runs of eight, `a` and `b`,
// that hold the two halves of eight pairs where the unit is rotated.
struct Unit {
    int a, b;      // first component of each run
    int pair;      // first of the eight pairs, or -1: not rotated
};

__device__ inline Unit unit_of(int u, int rot, int interleaved) {
    if (16 * u >= rot) return Unit{16 * u, 16 * u + 8, -1};
    if (interleaved) return Unit{16 * u, 16 * u + 8, 8 * u};
    return Unit{8 * u, rot / 2 + 8 * u, 8 * u};
}

__device__ inline void unpack8(u32x4 w, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(w[i]);
        x[2 * i + 1] = bf16_hi(w[i]);
    }
}

// The unit's sixteen values: run a, then run b.
__device__ inline void load_unit(const char *row, const Unit &u, u32x4 (&w)[2]) {
    w[0] = *reinterpret_cast<const u32x4 *>(row + u.a * 2);
    w[1] = *reinterpret_cast<const u32x4 *>(row + u.b * 2);
}

// Pair i of the unit rotated by t = {cos, sin}.
template <int INTERLEAVED> __device__ inline void rotate_pair(float *x, int i, float2 t) {
    const int p1 = INTERLEAVED ? 2 * i : i, p2 = INTERLEAVED ? 2 * i + 1 : i + 8;
    const float x1 = x[p1], x2 = x[p2];
    x[p1] = x1 * t.x - x2 * t.y;
    x[p2] = x2 * t.x + x1 * t.y;
}

__device__ inline void store_bf16(char *row, const Unit &u, const float *x) {
    *reinterpret_cast<u32x4 *>(row + u.a * 2) =
        u32x4{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])};
    *reinterpret_cast<u32x4 *>(row + u.b * 2) =
        u32x4{bf16_pair(x[8], x[9]), bf16_pair(x[10], x[11]), bf16_pair(x[12], x[13]), bf16_pair(x[14], x[15])};
}

}  // namespace
}  // namespace cospec
