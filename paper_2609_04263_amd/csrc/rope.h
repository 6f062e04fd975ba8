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
// ones on this chip: about 35 of them per pair.
#pragma once

#include <type_traits>

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

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// bf16 pairs -> fp32, and back (round to nearest even: one conversion a pair).
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
        w[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v[2 * j], v[2 * j + 1]}), bf16x2));
    return w;
}

// Sum over the `LANES` lanes (4 .. 32, a power of two, aligned) that hold a row.
// Every lane adds the same two numbers at each step, so all get the same bits.
template <int CTRL>
__device__ __forceinline__ double dpp_f64(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)u, CTRL, 0xF, 0xF, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(u >> 32), CTRL, 0xF, 0xF, true);
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

// The sum of squares of a row from those of its pieces of eight channels: one order, to
// the bit, for kvq_rope_qk and for appends.  Pairs in halves of a whole head: the two pieces
// with a pair's members first, then neighbours of these sums.  Else: neighbours first.
//
// Whether pairs in halves are of a part of the head, and rows are normed.
__host__ __device__ __forceinline__ bool part_in_halves(const RopeArgs& r, int D)
{
    return r.layout == KVQ_ROPE_HALF && r.rot < D && r.rot > 16 && (r.wq || r.wk);
}

// Lane l of D / 16 holds two pieces' sums, a and b (rope_rows), which come together in
// that order.  PART (part_in_halves): those of the rotated part are l and hp + l instead, so
// they are added up side by side up to the hp lanes that hold them, or, where hp is no power of
// two, exchanged (3 x 999 tokens of 40 normed heads of 128: 13.7 us in a's and b's own order, 14.1
// and 14.3 so; an instance of its own, so that the others' registers stay).
template <int D, bool PART>
__device__ __forceinline__ double row_squares(const RopeArgs& r, int l, double a, double b)
{
    constexpr int LPR = D / 16;
    if constexpr (!PART) {
        return row_sum<LPR>(a + b);
    } else {
        const int hp = r.rot / 16;
        if ((hp & (hp - 1)) == 0) {
            double x = l < hp ? a : a + b, y = l < hp ? b : 0.0;
            const auto step = [&](auto ctrl, int n) {
                if (n == hp)
                    x += y;
                x += dpp_f64<ctrl.value>(x);
                if (n < hp)
                    y += dpp_f64<ctrl.value>(y);
            };
            step(std::integral_constant<int, 0xB1>{}, 1);
            step(std::integral_constant<int, 0x4E>{}, 2);
            if constexpr (LPR >= 8)
                step(std::integral_constant<int, 0x141>{}, 4);
            if constexpr (LPR >= 16)
                step(std::integral_constant<int, 0x140>{}, 8);
            return x;
        }
        const int row = (threadIdx.x & 63) - l;
        const auto piece = [&](int P) {  // where it is: lane, and which of its two
            const int lane = P < hp ? P : P < 2 * hp ? P - hp : P >> 1;
            const double x = __shfl(a, row + lane), y = __shfl(b, row + lane);
            return P < hp || (P >= 2 * hp && P % 2 == 0) ? x : y;
        };
        const double even = piece(2 * l), odd = piece(2 * l + 1);
        return row_sum<LPR>(even + odd);
    }
}

// The same where lane P of D / 8 holds piece P's (appends).
template <int D>
__device__ __forceinline__ double row_squares(const RopeArgs& r, int P, double s)
{
    if (r.layout != KVQ_ROPE_HALF || r.rot != D)
        return row_sum<D / 8>(s);
    const uint64_t u = __builtin_bit_cast(uint64_t, s);
    const auto other = [&](uint32_t x) -> uint32_t {  // of lane P ^ (D / 16)
        if constexpr (D == 64) {
            const uint32_t m = __builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, true);
            return __builtin_amdgcn_update_dpp(0, m, 0x1B, 0xF, 0xF, true);
        } else if constexpr (D == 128) {
            return __builtin_amdgcn_update_dpp(0, x, 0x128, 0xF, 0xF, true);
        } else {
            const auto rows = __builtin_amdgcn_permlane16_swap(x, x, false, false);
            return P & 16 ? rows[0] : rows[1];
        }
    };
    const uint64_t v = ((uint64_t)other((uint32_t)(u >> 32)) << 32) | other((uint32_t)u);
    return row_sum<D / 16>(s + __builtin_bit_cast(double, v));
}

// The factor of a row with sum of squares `sum`: 1 / sqrt(v) by the hardware's
// estimate y (2^-23 or better) and one step of third order, y (1 + e / 2 + 3 e^2 / 8)
// with e = 1 - v y^2 (binary64: off by 2^-51, so the binary32 result is the nearest
// in all but 1 of 10^8 cases).
__device__ __forceinline__ float norm_factor(double sum, int D, float eps)
{
#pragma clang fp contract(off)
    const double v = sum * (1.0 / D) + (double)eps, y = __builtin_amdgcn_rsq(v);
    const double e = __builtin_fma(-(v * y), y, 1.0);
    return (float)__builtin_fma(y * e, __builtin_fma(0.375, e, 0.5), y);
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

// One wave's share of rotating queries and keys: ITER iterations of 1024 / D heads of
// one token, all loaded before the angles are computed; lds: D / 2 of the wave.
//
// A lane holds sixteen channels of a row, such that both members of each of its
// eight pairs are its own and the pairs are 8 l .. 8 l + 7 in either layout:
//     halves       channels 8 l .. and rot / 2 + 8 l ..  (l < rot / 16)
//     interleaved  channels 16 l .. 16 l + 15, as are those that are not rotated
// (two 16-byte loads), so rotating needs no exchange, and lane l's eight cosines
// and sines are the same for every head of a token: the wave's lanes compute each
// once, pass them on through LDS and keep their eight in registers.
// KEYS: there may be keys beside the queries.  PART: part_in_halves.
template <int D, int ITER, bool KEYS, bool PART>
__device__ __forceinline__ void rope_rows(const RopeQkParams& p, const RopeArgs& r, uint32_t token, int part, float2* lds)
{
    constexpr int LPR = D / 16, RPI = 64 / LPR;  // lanes of a row, rows of an iteration
    const int lane = threadIdx.x & 63, l = lane & (LPR - 1);
    const bool half = r.layout == KVQ_ROPE_HALF && l < r.rot / 16;
    const int c0 = half ? 8 * l : 16 * l, c1 = half ? r.rot / 2 + 8 * l : 16 * l + 8;
    u32x4 w[ITER][2];
    const int heads = p.H_q + (KEYS ? p.H : 0), h0 = part * ITER * RPI + lane / LPR;
    const auto row_of = [&](const uint16_t* q, const uint16_t* k, int h) {
        if constexpr (KEYS)
            return h < p.H_q ? q + ((size_t)token * p.H_q + h) * D : k + ((size_t)token * p.H + (h - p.H_q)) * D;
        else
            return q + ((size_t)token * p.H_q + h) * D;
    };
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int h = h0 + i * RPI;
        if (h < heads) {
            const uint16_t* row = row_of(p.q, p.k, h);
            w[i][0] = *(const u32x4*)(row + c0);
            w[i][1] = *(const u32x4*)(row + c1);
        }
    }
    float cs[8], sn[8];
    if (r.rot > 0) {
        const int t = r.pos ? r.pos[token] : r.pos0 + (int)(token % (uint32_t)p.n);
#pragma unroll
        for (int i = lane; i < D / 2; i += 64)
            if (i < r.rot / 2)
                lds[i] = rope_cos_sin(t, r.turns[i], r.scale);
        asm volatile("" ::: "memory");  // LDS accesses of a wave are performed in order
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const float4 x = *(const float4*)&lds[8 * l + j];
            cs[j] = x.x, sn[j] = x.y, cs[j + 1] = x.z, sn[j + 1] = x.w;
        }
    }
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int h = h0 + i * RPI;
        if (i > 0 && (part * ITER + i) * RPI >= heads)
            break;
        float v[16];
        widen8(w[i][0], v);
        widen8(w[i][1], v + 8);
        if (r.wq || (KEYS && r.wk)) {  // (every lane of a row takes part in its sum)
            const bool is_q = !KEYS || h < p.H_q;
            const uint16_t* any = KEYS && !r.wq ? r.wk : r.wq;
            const uint16_t* weight = !KEYS || is_q ? r.wq : r.wk;
            float f = norm_factor(row_squares<D, PART>(r, l, squares8(v), squares8(v + 8)), D, r.eps);
            float g[16];
            const uint16_t* at = weight ? weight : any;
            widen8(*(const u32x4*)(at + c0), g);
            widen8(*(const u32x4*)(at + c1), g + 8);
            if (KEYS && (!r.wq || !r.wk)) {  // rows of the kind without a norm: times one, twice
                f = weight ? f : 1.0f;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    g[e] = weight ? g[e] : 1.0f;
            }
            norm8(v, f, g);
            norm8(v + 8, f, g + 8);
        }
        if (16 * l < r.rot) {
            if (half) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    turn_pair(v[j], v[j + 8], cs[j], sn[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    turn_pair(v[2 * j], v[2 * j + 1], cs[j], sn[j]);
            }
        }
        if (h < heads) {
            uint16_t* row = const_cast<uint16_t*>(row_of(p.qo, p.ko, h));
            *(u32x4*)(row + c0) = narrow8(v);
            *(u32x4*)(row + c1) = narrow8(v + 8);
        }
    }
}

}  // namespace kvq
