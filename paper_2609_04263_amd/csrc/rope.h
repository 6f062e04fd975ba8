// Rotary positions and per-head RMS norms of queries and keys, as functions of
// the registers that hold a row: shared by the rope kernel and the append
// kernels.  The result is a bit-exact function of the input (include/kvq.h
// has the steps): binary32 operations in a fixed order without contraction,
// sums of squares and angles in binary64.
//
// Angles.  Position t of a pair that makes `turn` turns per position is at
// f = t turn - rint(t turn) turns, one rounding of the exact value (a fused
// multiply-add): in binary32 a position of 10^5 would be 6e-3 radians off.
// With q = rint(4 f) and x = 2 pi (f - q / 4), |x| <= pi / 4, the series
//     sin x = x - x^3/3! + .. - x^15/15!,  cos x = 1 - x^2/2! + .. + x^16/16!
// leave less than 5e-17, so the binary32 cosine is the nearest one in all but
// 1 of 10^8 cases.  Binary64 operations run at the rate of (unpacked) binary32
// ones on this chip: 35 of them per pair.
#pragma once

#include "kvq_device.h"
#include "kvq_internal.h"

namespace kvq {

__device__ __forceinline__ float2 rope_cos_sin(int t, double turn, float scale)
{
#pragma clang fp contract(off)
    const double p = (double)t, n = __builtin_rint(p * turn);
    const double f = __builtin_fma(p, turn, -n), q = __builtin_rint(4.0 * f);
    const double x = (f - 0.25 * q) * 6.283185307179586477, z = x * x;
    double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
    s = __builtin_fma(s, z, 1.0 / 6227020800.0);
    s = __builtin_fma(s, z, -1.0 / 39916800.0);
    s = __builtin_fma(s, z, 1.0 / 362880.0);
    s = __builtin_fma(s, z, -1.0 / 5040.0);
    s = __builtin_fma(s, z, 1.0 / 120.0);
    s = __builtin_fma(s, z, -1.0 / 6.0);
    s = __builtin_fma(s * z, x, x);
    c = __builtin_fma(c, z, -1.0 / 87178291200.0);
    c = __builtin_fma(c, z, 1.0 / 479001600.0);
    c = __builtin_fma(c, z, -1.0 / 3628800.0);
    c = __builtin_fma(c, z, 1.0 / 40320.0);
    c = __builtin_fma(c, z, -1.0 / 720.0);
    c = __builtin_fma(c, z, 1.0 / 24.0);
    c = __builtin_fma(c, z, -0.5);
    c = __builtin_fma(c, z, 1.0);
    const int k = (int)q;
    const double a = k & 1 ? s : c, b = k & 1 ? c : s;  // |cos|, |sin| up to signs
    const double m = (double)scale;
    return make_float2((float)((k + 1) & 2 ? -(a * m) : a * m), (float)(k & 2 ? -(b * m) : b * m));
}

// bf16 pairs -> fp32, and back (round to nearest even).
__device__ __forceinline__ void widen8(const u32x4& w, float* v)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
}

__device__ __forceinline__ u32x4 narrow8(const float* v)
{
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        w[j] = f32_to_bf16(v[2 * j]) | ((uint32_t)f32_to_bf16(v[2 * j + 1]) << 16);
    return w;
}

// Sum over the `LANES` lanes (4 .. 32, a power of two, aligned) that hold a row.
// Every lane adds the same two numbers at each step, so all get the same bits.
template <int CTRL>
__device__ __forceinline__ double dpp_f64(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)u, CTRL, 0xF, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(u >> 32), CTRL, 0xF, 0xF, false);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}

template <int LANES>
__device__ __forceinline__ double row_sum(double x)
{
    x += dpp_f64<0xB1>(x);       // quad_perm [1, 0, 3, 2]
    x += dpp_f64<0x4E>(x);       // quad_perm [2, 3, 0, 1]
    if constexpr (LANES >= 8)
        x += dpp_f64<0x141>(x);  // row_half_mirror
    if constexpr (LANES >= 16)
        x += dpp_f64<0x140>(x);  // row_mirror
    if constexpr (LANES >= 32)
        x += __shfl_xor(x, 16);
    return x;
}

// Sum of squares of eight bf16 values (in binary64 each square is exact and none
// leaves the range).
__device__ __forceinline__ double squares8(const float* v)
{
#pragma clang fp contract(off)
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        s = __builtin_fma((double)v[e], (double)v[e], s);
    return s;
}

// The factor of a row with sum of squares `sum`.
__device__ __forceinline__ float norm_factor(double sum, int D, float eps)
{
#pragma clang fp contract(off)
    return (float)(1.0 / __builtin_sqrt(sum / (double)D + (double)eps));
}

__device__ __forceinline__ void norm8(float* v, float r, const float* w)
{
#pragma clang fp contract(off)
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = (v[e] * r) * w[e];
}

// (a, b) turned by (c, s).
__device__ __forceinline__ void turn_pair(float& a, float& b, float c, float s)
{
#pragma clang fp contract(off)
    const float x = a * c - b * s, y = b * c + a * s;
    a = x;
    b = y;
}

}  // namespace kvq
