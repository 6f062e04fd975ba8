// Attention of a batch whose sequences share long prefixes
// (kvq_decode_attn_shared, kvq_prefill_attn_shared): one softmax over the
// tokens of a sequence's prefix, a sequence of the prefix cache that its whole
// group reads, and of its own suffix.
//
// The two caches are two segments.  A segment's unit (cache sequence, KV head)
// meets a set of query rows (sequence, chunk token, head): all rows of the
// group for a prefix unit, one sequence's rows for a suffix unit.  A work item
// is a range of a unit's 32-token blocks and up to 16 kTiles kWaves of its
// rows; every item writes an unnormalized partial (m, l, o) per row, and a
// second kernel joins a row's partials of both segments:
//     M = max m,  O = sum 2^(m - M) o / sum 2^(m - M) l.
// So the codes of a prefix are read once per work item of its group's rows
// instead of once per sequence.
//
// Inside an item eight waves, two per SIMD, alternate between two phases:
//   build    the waves turn the next kImages blocks into images in LDS, kParts
//            waves per block: operand fragments of
//            v_mfma_f32_16x16x32_f16, in the order in which the cache stores
//            its codes (a 1 KiB fragment is one 16-byte piece per lane);
//   consume  each wave multiplies its query rows with its share of the images.
// With R row waves (the fewest powers of two that hold the rows) a wave has up
// to kTiles tiles of 16 rows and every kWaves / R-th image, so that few rows
// still occupy all waves.  What a block costs to convert is paid once for all
// rows of the item, where decode attention, which converts in registers, pays
// it once per 16 rows.
//
// An image holds
//   keys    per-token groups: the codes, centred (c - (2^b - 1) / 2, or c -
//           2^(b-1) when symmetric), exact in fp16, with scales and offsets s, z'
//           beside them: S = sum_g s_g (A_g . q_g) + z'_g sum q_g, the offsets
//           by one fp32 MFMA of four groups.  Per-channel groups: the
//           reconstructed key times a power of two, as fp16 hi + lo (22 bits);
//   values  the reconstructed value times a power of two, hi + lo.
// and the product of the values with the probabilities (hi + lo as well) is
// three MFMAs, all but the 2^-22 of lo x lo.  Values as codes with p s as the
// other operand take two, but cost each tile 40 vector operations per value
// group, and a bias in the codes costs precision where outputs are small
// beside the values: 32768 tokens of flat attention were 4.7e-4 off with
// decode attention's operands and 1e-6 with these.
// fp16 tokens (window, sink) are images as they are, with a lo half of zero.
//
// Softmax: online per column in base 2, the running maximum raised only when a
// block exceeds it by more than kTau; probabilities are at most 2^(kTau +
// kPBits).  Causal rows (suffix segments of a chunk) are masked per column, and
// blocks that no row of a wave sees are skipped.
#pragma once

#include <type_traits>

#include "kvq_device.h"
#include "kvq_internal.h"

namespace kvq {
namespace shr {
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr float kTau = 4.0f;     // lazy rescale threshold, log2 units
constexpr float kPBits = 10.0f;  // probabilities are kept times 2^kPBits, so that their lo half is exact
constexpr float kNegInf = -__builtin_inff();

// 16-row tiles per wave: 32 rows' accumulators and queries fit 256 registers
// up to D = 128.
__host__ __device__ constexpr int tiles(int D)
{
    return D == 256 ? 1 : 2;
}

// Images of a build phase (LDS), and waves that build one.
__host__ __device__ constexpr int images(int D)
{
    return 512 / D;
}

__host__ __device__ constexpr int parts(int D)
{
    return kWaves / images(D);
}

__host__ __device__ constexpr int item_rows(int D)
{
    return 16 * tiles(D) * kWaves;
}

// ---- LDS: the images, then per image its scales and offsets ([group][32]
// each) and two scalars, then 2 KiB per wave to pass a block's metadata
// between lanes.  The merge of the waves reuses it from the start.
__host__ __device__ constexpr int key_bytes(int D, bool hilo)
{
    return 64 * D * (hilo ? 2 : 1);
}

__host__ __device__ constexpr int image_bytes(int D, bool hilo)
{
    return key_bytes(D, hilo) + 128 * D;
}

__host__ __device__ constexpr int meta_bytes(int D)
{
    return 2 * (D / 32) * 128 + 16;
}

constexpr int kStage = 2048;

__host__ __device__ constexpr int lds_bytes(int D, bool hilo)
{
    const int walk = images(D) * (image_bytes(D, hilo) + meta_bytes(D)) + kWaves * kStage;
    const int merge = kWaves * 16 * (D + 2) * 4;
    return walk > merge ? walk : merge;
}

__device__ __forceinline__ float sum_rows(float v)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ float max_rows(float v)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

template <int CTRL>
__device__ __forceinline__ float dpp_f32(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, false));
}

// The largest x >= 0 of the wave.
__device__ __forceinline__ float wave_max(float x)
{
    x = fmaxf(x, dpp_f32<0xB1>(x));   // quad_perm [1, 0, 3, 2]
    x = fmaxf(x, dpp_f32<0x4E>(x));   // quad_perm [2, 3, 0, 1]
    x = fmaxf(x, dpp_f32<0x141>(x));  // row_half_mirror
    x = fmaxf(x, dpp_f32<0x140>(x));  // row_mirror
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(max_rows(x))));
}

// A power of two f with x f in (2^8, 2^12], its exponent a multiple of four, so
// that neighbouring blocks mostly share it (x >= 0; f is kept within 2^-115 .. 2^113).
__device__ __forceinline__ float scale_to_range(float x)
{
    const uint32_t e = min(max(((__float_as_uint(x) >> 23) + 4) & ~3u, 26u), 254u);  // x < 2^(e - 127)
    return __uint_as_float((254 + 12 - e) << 23);
}

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// fp32 -> fp16 hi + lo, both to nearest: |v - hi - lo| <= 2^-23 |v| (2^-25
// absolute where lo is subnormal).  Pairs, for the packed conversion.
__device__ __forceinline__ void split_nearest(const float* v, half8* hi, half8* lo)
{
    u32x4 h, l;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f16x2 a = __builtin_convertvector((f32x2{v[2 * j], v[2 * j + 1]}), f16x2);
        const f16x2 b = __builtin_convertvector((f32x2{v[2 * j] - (float)a.x, v[2 * j + 1] - (float)a.y}), f16x2);
        h[j] = __builtin_bit_cast(uint32_t, a);
        l[j] = __builtin_bit_cast(uint32_t, b);
    }
    *hi = __builtin_bit_cast(half8, h);
    *lo = __builtin_bit_cast(half8, l);
}

// LDS accesses of a wave are performed in order; the compiler keeps them in
// order too, whatever their types.
__device__ __forceinline__ void lds_order()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// This wave's LDS accesses are done and every wave is past the same point.
// (Loads from global memory stay in flight.)
__device__ __forceinline__ void sync_lds()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// ------------------------------------------------------------ images

// How codes become operands (uniform).
struct Coding {
    float mid;        // the operand of code c is c - mid
    uint32_t centre;  // fp16 pair added to the biased code (see centred)
};

template <int BITS>
__device__ __forceinline__ Coding coding(bool affine)
{
    // 8 bits: 1024 + c - 1152; 4 bits: 16 + c - 23.5 or - 24; 2 bits: 4 + c - 5.5 or - 6
    Coding c;
    c.mid = BITS == 8 ? 128.0f : affine ? (float)((1 << BITS) - 1) * 0.5f : (float)(1 << (BITS - 1));
    c.centre = BITS == 8 ? 0xE480E480u : BITS == 4 ? (affine ? 0xCDE0CDE0u : 0xCE00CE00u)
                                                   : (affine ? 0xC580C580u : 0xC600C600u);
    return c;
}

// Piece k (eight codes) of the words -> (c_j - mid, c_{j+4} - mid) in dword j,
// i.e. element e holds code perm4(e): the code as mantissa bits under an
// exponent that gives them unit weight, then one exact packed addition.
template <int BITS>
__device__ __forceinline__ half8 centred(const uint32_t* w, int k, uint32_t centre)
{
    u32x4 v;
    if constexpr (BITS == 8) {
        const uint32_t lo = w[2 * k], hi = w[2 * k + 1];
        v.x = __builtin_amdgcn_perm(hi, lo, 0x0c040c00u) | 0x64006400u;
        v.y = __builtin_amdgcn_perm(hi, lo, 0x0c050c01u) | 0x64006400u;
        v.z = __builtin_amdgcn_perm(hi, lo, 0x0c060c02u) | 0x64006400u;
        v.w = __builtin_amdgcn_perm(hi, lo, 0x0c070c03u) | 0x64006400u;
    } else if constexpr (BITS == 4) {
        const uint32_t x = w[k];
        v.x = ((x << 6) & 0x03C003C0u) | 0x4C004C00u;
        v.y = ((x << 2) & 0x03C003C0u) | 0x4C004C00u;
        v.z = ((x >> 2) & 0x03C003C0u) | 0x4C004C00u;
        v.w = ((x >> 6) & 0x03C003C0u) | 0x4C004C00u;
    } else {
        // bytes (c0..c3) and (c4..c7) of the piece to bytes 0 and 2
        const uint32_t z = __builtin_amdgcn_perm(0u, w[k >> 1], (k & 1) ? 0x0c030c02u : 0x0c010c00u);
        v.x = ((z << 8) & 0x03000300u) | 0x44004400u;
        v.y = ((z << 6) & 0x03000300u) | 0x44004400u;
        v.z = ((z << 4) & 0x03000300u) | 0x44004400u;
        v.w = ((z << 2) & 0x03000300u) | 0x44004400u;
    }
    const f16x2 c = __builtin_bit_cast(f16x2, centre);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        v[j] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, (uint32_t)v[j]) + c);
    return __builtin_bit_cast(half8, v);
}

// The loads of one wave's part of a coded block: four key pieces and four
// value pieces per lane, and chunk `lane` (four numbers) of the block's key and
// of its value scales and offsets.
template <int KB, int VB, bool M16>
struct Raw {
    uint32_t k[KB], v[VB];  // 4 pieces of KB / 4 words
    u32x4 ks, kz, vs, vz;
};

// N bytes (4 to 32, naturally aligned) from global memory, streaming.
template <int N>
__device__ __forceinline__ void load_bytes(const uint8_t* at, uint32_t* w)
{
    if constexpr (N == 4) {
        w[0] = __builtin_nontemporal_load((const uint32_t*)at);
    } else if constexpr (N == 8) {
        const u32x2 x = __builtin_nontemporal_load((const u32x2*)at);
        w[0] = x.x;
        w[1] = x.y;
    } else {
#pragma unroll
        for (int i = 0; i < N / 16; ++i) {
            const u32x4 x = __builtin_nontemporal_load((const u32x4*)at + i);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[4 * i + e] = x[e];
        }
    }
}

// The builder's view of a segment's unit: a wave's part of its images.
template <int D, bool KH, int KB, int VB, bool M16>
struct Builder {
    static constexpr int NKB = D / 32, NMB = D / 16, PB = parts(D);
    const AttnParams& p;
    int unit, part, lane;
    int nkc, nvc;      // chunks of a block's key and value scales
    bool kaff, vaff;
    const uint8_t *k, *v, *ks, *vs;  // this lane's pieces and chunks of block 0
    long dkz, dvz;                   // offsets - scales (0 when symmetric: the scales once more)

    // piece i of the lane: half block and 32-channel block
    __device__ __forceinline__ int half(int i) const { return PB == 1 ? i >> 1 : PB == 2 ? part : part >> 1; }
    __device__ __forceinline__ int kblock(int i) const { return PB == 1 ? i & 1 : PB == 2 ? i : 4 * (part & 1) + i; }

    __device__ __forceinline__ Builder(const AttnParams& p_, int unit_, int part_, int lane_)
        : p(p_), unit(unit_), part(part_), lane(lane_)
    {
        const size_t ub0 = (size_t)unit * (p.T >> 5);
        constexpr int ESZ = M16 ? 2 : 4;
        nkc = KH ? D / 4 : 8 * (D / p.k_group);
        nvc = 8 * (D / p.v_group);
        kaff = p.k_mode == KVQ_AFFINE;
        vaff = p.v_mode == KVQ_AFFINE;
        k = (const uint8_t*)p.kc + ((ub0 * 2 + half(0)) * 64 + lane) * (NKB * KB) + kblock(0) * KB;
        v = (const uint8_t*)p.vc + (ub0 * 64 + lane) * (NMB * VB) + 4 * part * VB;
        ks = (const uint8_t*)p.ks + (ub0 * nkc + min(lane, nkc - 1)) * (4 * ESZ);
        vs = (const uint8_t*)p.vs + (ub0 * nvc + min(lane, nvc - 1)) * (4 * ESZ);
        dkz = kaff ? (const uint8_t*)p.kz - (const uint8_t*)p.ks : 0;
        dvz = vaff ? (const uint8_t*)p.vz - (const uint8_t*)p.vs : 0;
    }

    __device__ __forceinline__ u32x4 load_chunk(const uint8_t* at) const
    {
        if constexpr (M16) {
            const u32x2 x = __builtin_nontemporal_load((const u32x2*)at);
            return u32x4{x.x, x.y, 0u, 0u};
        } else {
            return __builtin_nontemporal_load((const u32x4*)at);
        }
    }

    // Every lane issues the same loads whatever the block.
    __device__ __forceinline__ void load(Raw<KB, VB, M16>& r, int blk) const
    {
        constexpr int ESZ = M16 ? 2 : 4;
        const uint8_t* kb = k + (size_t)blk * (2 * 64 * NKB * KB);
        if constexpr (PB == 1) {
            load_bytes<2 * KB>(kb, r.k);
            load_bytes<2 * KB>(kb + 64 * NKB * KB, r.k + KB / 2);
        } else {
            load_bytes<4 * KB>(kb, r.k);
        }
        load_bytes<4 * VB>(v + (size_t)blk * (64 * NMB * VB), r.v);
        const uint8_t *a = ks + (size_t)blk * (nkc * 4 * ESZ), *b = vs + (size_t)blk * (nvc * 4 * ESZ);
        r.ks = load_chunk(a);
        r.kz = load_chunk(a + dkz);
        r.vs = load_chunk(b);
        r.vz = load_chunk(b + dvz);
    }

    // The numbers of a chunk pair: scale, and offset of the centred code.
    // Dead slots (a chunk is four tokens of a group, unless `whole`) give zeros.
    __device__ __forceinline__ void widen(const u32x4& s, const u32x4& z, bool aff, float mid, int live, bool whole,
                                          float* sv, float* zv) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sv[e] = M16 ? f16_bits_to_f32((uint16_t)(s[e >> 1] >> (16 * (e & 1)))) : __uint_as_float(s[e]);
            zv[e] = M16 ? f16_bits_to_f32((uint16_t)(z[e >> 1] >> (16 * (e & 1)))) : __uint_as_float(z[e]);
            const bool on = whole || 4 * (lane & 7) + e < live;
            sv[e] = on ? sv[e] : 0.0f;
            zv[e] = on && aff ? fmaf(mid, sv[e], zv[e]) : 0.0f;
        }
    }

    // This wave's part of the image of a coded block whose first `live` tokens
    // exist.  img: the image; meta: its scales; st: this wave's stage.
    __device__ __forceinline__ void coded_image(const Raw<KB, VB, M16>& r, int live, uint8_t* img, float* meta,
                                                float* st) const
    {
        const int qg = lane >> 4;
        // ---- keys
        const Coding kc = coding<KB>(kaff);
        float ksv[4], kzv[4], kf = 1.0f;
        widen(r.ks, r.kz, kaff, kc.mid, live, KH, ksv, kzv);
        if constexpr (KH) {
            // times a power of two that brings the block's keys to 2^12 at most:
            // hi + lo then holds them to 2^-37 of the largest
            float top = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                top = fmaxf(top, fmaf(kc.mid, ksv[e], fabsf(kzv[e])));
            kf = scale_to_range(wave_max(lane < nkc ? top : 0.0f));
            // channel c: scale at st[c], offset at st[D + c]
            if (lane < nkc) {
                *(float4*)(st + 4 * lane) = float4{ksv[0] * kf, ksv[1] * kf, ksv[2] * kf, ksv[3] * kf};
                *(float4*)(st + D + 4 * lane) = float4{kzv[0] * kf, kzv[1] * kf, kzv[2] * kf, kzv[3] * kf};
            }
            lds_order();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int kb = kblock(i);
                const float* s = st + 32 * kb + 8 * qg;
                const float4 s0 = *(const float4*)s, s1 = *(const float4*)(s + 4);
                const float4 z0 = *(const float4*)(s + D), z1 = *(const float4*)(s + D + 4);
                const float sn[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
                const float zn[8] = {z0.x, z0.y, z0.z, z0.w, z1.x, z1.y, z1.z, z1.w};
                const half8 a = centred<KB>(r.k, i, kc.centre);
                float x[8];
                half8 hi, lo;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[j] = fmaf((float)a[j], sn[perm4(j)], zn[perm4(j)]);
                split_nearest(x, &hi, &lo);
                uint8_t* at = img + 1024 * (half(i) * NKB + kb) + 16 * lane;
                *(half8*)at = hi;
                *(half8*)(at + 64 * D) = lo;
            }
            lds_order();
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(half8*)(img + 1024 * (half(i) * NKB + kblock(i)) + 16 * lane) = centred<KB>(r.k, i, kc.centre);
            if (part == 0 && lane < nkc) {
                const float f = p.sm_log2;
                *(float4*)(meta + 4 * lane) = float4{ksv[0] * f, ksv[1] * f, ksv[2] * f, ksv[3] * f};
                *(float4*)(meta + D + 4 * lane) = float4{kzv[0] * f, kzv[1] * f, kzv[2] * f, kzv[3] * f};
            }
        }
        __builtin_amdgcn_sched_barrier(0);  // (the registers of one side at a time)
        // ---- values, likewise; group g's scales at st[32 g], offsets at st[D + 32 g]
        const Coding vc = coding<VB>(vaff);
        float vsv[4], vzv[4], top = 0.0f;
        widen(r.vs, r.vz, vaff, vc.mid, live, false, vsv, vzv);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            top = fmaxf(top, fmaf(vc.mid, vsv[e], fabsf(vzv[e])));
        const float vf = scale_to_range(wave_max(lane < nvc ? top : 0.0f));
        if (lane < nvc) {
            *(float4*)(st + 4 * lane) = float4{vsv[0] * vf, vsv[1] * vf, vsv[2] * vf, vsv[3] * vf};
            *(float4*)(st + D + 4 * lane) = float4{vzv[0] * vf, vzv[1] * vf, vzv[2] * vf, vzv[3] * vf};
        }
        lds_order();
        const int lg = 31 - __builtin_clz(p.v_group);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int mb = 4 * part + i;
            const float* s = st + 32 * (16 * mb >> lg) + 8 * qg;
            const float4 s0 = *(const float4*)s, s1 = *(const float4*)(s + 4);
            const float4 z0 = *(const float4*)(s + D), z1 = *(const float4*)(s + D + 4);
            const float sn[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
            const float zn[8] = {z0.x, z0.y, z0.z, z0.w, z1.x, z1.y, z1.z, z1.w};
            const half8 c = centred<VB>(r.v, i, vc.centre);
            float x[8];
            half8 hi, lo;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = fmaf((float)c[j], sn[perm4(j)], zn[perm4(j)]);
            split_nearest(x, &hi, &lo);
            uint8_t* at = img + key_bytes(D, KH) + 1024 * mb + 16 * lane;
            *(half8*)at = hi;
            *(half8*)(at + 64 * D) = lo;
            __builtin_amdgcn_sched_barrier(0);
        }
        if (part == 0 && lane == 0) {
            meta[2 * D] = vf;
            meta[2 * D + 1] = KH ? p.sm_log2 * (1.0f / kf) : 0.0f;
        }
    }

    // This wave's part of the image of a block of fp16 rows: token i is row
    // (first + i) % ring of kr, vr [.][D], the first `live` exist.
    __device__ __forceinline__ void rows_image(const uint16_t* kr, const uint16_t* vr, int first, int ring, int live,
                                               uint8_t* img, float* meta) const
    {
        const int qg = lane >> 4, hh = lane & 15;
        const half8 zero = {};
        // (dead tokens read a live row and are cleared: no load waits for a branch)
        u32x4 kw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = min(8 * (hh >> 2) + 4 * half(i) + (hh & 3), live - 1);
            kw[i] = *(const u32x4*)(kr + (uint32_t)((first + t) % ring * D + 32 * kblock(i) + 8 * qg));
        }
        uint32_t row[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            row[j] = (first + min(8 * qg + perm4(j), live - 1)) % ring * D + 64 * part + hh;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool on = 8 * (hh >> 2) + 4 * half(i) + (hh & 3) < live;
            u32x4 a;  // dword j: channels j and j + 4
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t x = kw[i][j >> 1], y = kw[i][2 + (j >> 1)];
                a[j] = !on ? 0u : j & 1 ? (x >> 16) | (y & 0xFFFF0000u) : (x & 0xFFFFu) | (y << 16);
            }
            uint8_t* at = img + 1024 * (half(i) * NKB + kblock(i)) + 16 * lane;
            *(u32x4*)at = a;
            if constexpr (KH)
                *(half8*)(at + 64 * D) = zero;
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            uint16_t h[2][8];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    h[u][j] = vr[row[j] + 16 * (i + u)];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                u32x4 w;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    w[j] = 8 * qg + j < live ? h[u][2 * j] : 0u;
                    w[j] |= 8 * qg + j + 4 < live ? (uint32_t)h[u][2 * j + 1] << 16 : 0u;
                }
                uint8_t* at = img + key_bytes(D, KH) + 1024 * (4 * part + i + u) + 16 * lane;
                *(u32x4*)at = w;
                *(half8*)(at + 64 * D) = zero;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (part == 0) {
            if (!KH && lane < nkc) {
                const float f = p.sm_log2;
                *(float4*)(meta + 4 * lane) = float4{f, f, f, f};
                *(float4*)(meta + D + 4 * lane) = float4{0.0f, 0.0f, 0.0f, 0.0f};
            }
            if (lane == 0) {
                meta[2 * D] = 1.0f;
                meta[2 * D + 1] = p.sm_log2;
            }
        }
    }
};

// ------------------------------------------------------------ rows

// A wave's state: NT tiles of 16 query rows (columns of the MFMAs).  KG: key
// group size / 32 (0: reconstructed keys, hi + lo).  ROT: rotated queries, hi + lo.
template <int D, int KG, bool ROT>
struct Rows {
    static constexpr int CT = tiles(D), NKB = D / 32, NMB = D / 16;
    static constexpr bool KH = KG == 0;
    static constexpr int KS = KH ? NKB : KG, NG = NKB / KS, NZ = (NG + 3) / 4;
    half8 q[CT][NKB], ql[ROT ? CT : 1][ROT ? NKB : 1];
    float qz[CT][NZ];        // lane (col, qg): the query's sum over group 4 j + qg
    floatx4 oacc[CT][NMB];
    float m[CT], lsum[CT];   // running max (log2 units), lane partial sum (times 2^kPBits)
    float vf;                // power of two that the accumulated values carry (uniform)
    int lim[CT];             // tail tokens that this lane's column sees (may be negative: only sink tokens)
    int lim0, lim1;          // the least and the most of the wave's rows (uniform)

    // Query rows of tile c, this lane's at src (channels 32 kb + 8 qg .. + 7 of it).
    __device__ __forceinline__ void load_query(int c, const uint16_t* src, float rot_c, int lane)
    {
        const int qg = lane >> 4;
        float v[NKB][8];
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
            const u32x4 w = *(const u32x4*)(src + 32 * kb + 8 * qg);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[kb][2 * j] = __uint_as_float(w[j] << 16);
                v[kb][2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
            }
        }
        if constexpr (ROT) {
            // the transform's butterflies commute: channel bits 0..2 and 5.. are
            // in this lane's registers, bits 3 and 4 are lanes 16 and 32 apart
#pragma unroll
            for (int h = 1; h < 8; h <<= 1)
#pragma unroll
                for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (!(j & h)) {
                            const float a = v[kb][j], b = v[kb][j + h];
                            v[kb][j] = a + b;
                            v[kb][j + h] = a - b;
                        }
#pragma unroll
            for (int h = 1; h < NKB; h <<= 1)
#pragma unroll
                for (int kb = 0; kb < NKB; ++kb)
                    if (!(kb & h))
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float a = v[kb][j], b = v[kb + h][j];
                            v[kb][j] = a + b;
                            v[kb + h][j] = a - b;
                        }
            const float s16 = qg & 1 ? -1.0f : 1.0f, s32 = qg & 2 ? -1.0f : 1.0f;
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t x = __float_as_uint(v[kb][j]);
                    auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
                    const uint32_t y = __float_as_uint(fmaf(s16, __uint_as_float(a[1]), __uint_as_float(a[0])));
                    auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
                    v[kb][j] = fmaf(s32, __uint_as_float(b[1]), __uint_as_float(b[0]));
                }
        }
        float sum[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g)
            sum[g] = 0.0f;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = v[kb][perm4(j)] * (ROT ? rot_c : 1.0f);
                sum[kb / KS] += x[j];
            }
            if constexpr (ROT)
                split_nearest(x, &q[c][kb], &ql[c][kb]);
            else
                q[c][kb] = pack_half8(x);
        }
        if constexpr (!KH) {
#pragma unroll
            for (int j = 0; j < NZ; ++j)
                qz[c][j] = 0.0f;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const float s = sum_rows(sum[g]);
                qz[c][g / 4] = qg == g % 4 ? s : qz[c][g / 4];
            }
        }
    }

    __device__ __forceinline__ void init()
    {
        vf = 0.0f;
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            m[c] = kNegInf;
            lsum[c] = 0.0f;
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb)
                oacc[c][mb] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }

    // One image: tokens t0 .. t0 + 31 (tail indices; with `off` = the sink's size
    // for sink blocks), the first `live` of which exist.
    template <int NT>
    __device__ __forceinline__ void consume(const uint8_t* img, const float* meta, int t0, int off, int live, int lane)
    {
        const int qg = lane >> 4, hh = lane & 15;
        const uint8_t* fb = img + 16 * lane;
        const auto frag = [&](int at) { return *(const half8*)(fb + at); };
        const float f = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(meta[2 * D])));
        // ---- scores: l[c][4 e + i] is token 8 qg + 4 e + i
        float l[NT][8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            floatx4 S[NT];
#pragma unroll
            for (int c = 0; c < NT; ++c)
                S[c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (!KH) {
                // offsets of four groups at once: row hh of the half is token 8 (hh / 4) + 4 e + hh % 4
                const int tok = 8 * (hh >> 2) + 4 * e + (hh & 3);
#pragma unroll
                for (int j = 0; j < NZ; ++j) {
                    const float z = meta[D + 32 * min(4 * j + qg, NG - 1) + tok];  // (times a zero sum past the last group)
#pragma unroll
                    for (int c = 0; c < NT; ++c)
                        S[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(z, qz[c][j], S[c], 0, 0, 0);
                }
            }
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                floatx4 acc[NT];
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    acc[c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int u = 0; u < KS; ++u) {
                    const int kb = g * KS + u;
                    const half8 a = frag(1024 * (e * NKB + kb));
#pragma unroll
                    for (int c = 0; c < NT; ++c)
                        acc[c] = mfma16(a, q[c][kb], acc[c]);
                    if constexpr (ROT) {
#pragma unroll
                        for (int c = 0; c < NT; ++c)
                            acc[c] = mfma16(a, ql[c][kb], acc[c]);
                    }
                    if constexpr (KH) {
                        const half8 b = frag(64 * D + 1024 * (e * NKB + kb));
#pragma unroll
                        for (int c = 0; c < NT; ++c)
                            acc[c] = mfma16(b, q[c][kb], acc[c]);
                    }
                }
                if constexpr (KH) {
                    const float sm = meta[2 * D + 1];
#pragma unroll
                    for (int c = 0; c < NT; ++c)
                        S[c] = acc[c] * sm;
                } else {
                    const floatx4 s4 = *(const floatx4*)(meta + 32 * g + 8 * qg + 4 * e);
#pragma unroll
                    for (int c = 0; c < NT; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            S[c][i] = fmaf(s4[i], acc[c][i], S[c][i]);
                }
            }
#pragma unroll
            for (int c = 0; c < NT; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    l[c][4 * e + i] = S[c][i];
        }
        if (live < 32 || t0 + 32 > lim0 + off) {
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                const int valid = min(live, lim[c] + off - t0);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    l[c][k] = 8 * qg + k < valid ? l[c][k] : kNegInf;
            }
        }
        // ---- the values' power of two: accumulators follow the largest values
        float bias = kPBits, back = 1.0f;
        if (f != vf) {
            const int d = (int)(__float_as_uint(f) >> 23) - (int)(__float_as_uint(vf) >> 23);  // log2(f / vf)
            const float r = __uint_as_float((uint32_t)min(max(127 + d, 0), 254) << 23);
            if (vf == 0.0f || d < 0) {
                if (vf != 0.0f) {
#pragma unroll
                    for (int c = 0; c < CT; ++c)
#pragma unroll
                        for (int mb = 0; mb < NMB; ++mb)
                            oacc[c][mb] *= r;
                }
                vf = f;
            } else {
                // smaller values: their probabilities make up for it
                bias = kPBits - (float)d;
                back = r;
            }
        }
        // ---- softmax, and the probabilities' operands
        half8 ph[NT], pl[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            float bm = fmaxf(fmaxf(fmaxf(l[c][0], l[c][1]), fmaxf(l[c][2], l[c][3])),
                             fmaxf(fmaxf(l[c][4], l[c][5]), fmaxf(l[c][6], l[c][7])));
            if (__any(bm > m[c] + kTau)) {
                bm = max_rows(bm);
                const float mn = bm > m[c] + kTau ? bm : m[c];
                const float alpha = m[c] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m[c] - mn);
                m[c] = mn;
                lsum[c] *= alpha;
#pragma unroll
                for (int mb = 0; mb < NMB; ++mb)
                    oacc[c][mb] *= alpha;
            }
            // (a column that has seen no token keeps m = -inf and gets zeros)
            const float shift = bias - (m[c] == kNegInf ? 0.0f : m[c]);
            float pv[8], ps = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                pv[j] = __builtin_amdgcn_exp2f(l[c][perm4(j)] + shift);
                ps += pv[j];
            }
            lsum[c] = fmaf(ps, back, lsum[c]);
            split_nearest(pv, &ph[c], &pl[c]);
        }
        // ---- values
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb) {
            const half8 a = frag(key_bytes(D, KH) + 1024 * mb), b = frag(key_bytes(D, KH) + 64 * D + 1024 * mb);
#pragma unroll
            for (int c = 0; c < NT; ++c)
                oacc[c][mb] = mfma16(a, ph[c], oacc[c][mb]);
#pragma unroll
            for (int c = 0; c < NT; ++c)
                oacc[c][mb] = mfma16(a, pl[c], oacc[c][mb]);
#pragma unroll
            for (int c = 0; c < NT; ++c)
                oacc[c][mb] = mfma16(b, ph[c], oacc[c][mb]);
        }
    }
};

// ------------------------------------------------------------ work items

// The work item of a workgroup (all uniform).
struct Item {
    int seg, unit, j;    // segment, unit (sequence H + j) and KV head
    int seq0;            // first batch sequence of the rows
    int r0, rows;        // first row of the item, rows of the unit
    int split, part;     // range of blocks, and its place among a row's partials
    int v0, v1;          // blocks v0 .. v1 - 1 (sink blocks first, then the tail's)
    int lim, causal;     // limit of row 0, and whether a row of chunk token c sees c more
};

__device__ __forceinline__ Item find_item(const SharedParams& p)
{
    Item it;
    int x = blockIdx.x;
    const int per = p.tile_rows;
    if (x < p.items0) {
        // prefix: ranges of a tile apart, tiles of a unit next to each other
        const AttnParams& a = p.seg[0];
        it.seg = 0;
        const int t = x % p.tiles0;
        it.split = x / p.tiles0;
        it.part = it.split;
        int g = 0, hi = p.P;  // tile0[g] <= t < tile0[hi]
        while (hi - g > 1) {
            const int mid = (g + hi) >> 1;
            if (p.tile0[mid] <= t)
                g = mid;
            else
                hi = mid;
        }
        it.seq0 = p.first[g];
        it.rows = (p.first[g + 1] - it.seq0) * p.C * a.G;
        const int n = (it.rows + per - 1) / per, u = t - p.tile0[g];
        it.j = u / n;
        it.r0 = (u - it.j * n) * per;
        it.unit = g * a.H + it.j;
        it.lim = a.n;
        it.causal = 0;
    } else {
        const AttnParams& a = p.seg[1];
        x -= p.items0;
        it.seg = 1;
        it.rows = p.C * a.G;
        const int n = (it.rows + per - 1) / per;
        const int t = x / p.S[1];
        it.split = x - t * p.S[1];
        it.part = p.S[0] + it.split;
        it.unit = t / n;
        it.r0 = (t - it.unit * n) * per;
        it.seq0 = it.unit / a.H;
        it.j = it.unit - it.seq0 * a.H;
        it.lim = a.n - p.C + 1;
        it.causal = 1;
    }
    return it;
}

// Row of O [B][C][H_q][D] (and of Q, and of the partials) of a unit's row r.
__device__ __forceinline__ size_t global_row(const SharedParams& p, const Item& it, int G, int r)
{
    const int t = r / G;
    return ((size_t)it.seq0 * p.C + t) * p.H_q + (size_t)it.j * G + (r - t * G);
}

template <int D, int KG, int KB, int VB, bool M16, bool ROT>
__global__ __launch_bounds__(kThreads, 2) void shared_kernel(SharedParams sp)
{
    constexpr bool KH = KG == 0;
    constexpr int CT = tiles(D), NI = images(D), PB = parts(D), NMB = D / 16;
    constexpr int BI = image_bytes(D, KH), BM = meta_bytes(D);
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, hh = lane & 15, qg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const Item it = find_item(sp);
    const AttnParams& p = sp.seg[it.seg];
    const int G = p.G, left = min(it.rows - it.r0, item_rows(D));

    // ---- this wave's rows and images: R row waves (at least what the images leave)
    const int nt16 = (left + 15) >> 4;
    int R = kWaves / NI;
    while (R * CT < nt16)
        R *= 2;
    const int rw = wave & (R - 1), bw = wave / R, BW = kWaves / R;
    const int nt = nt16 > rw ? (nt16 - rw + R - 1) / R : 0;  // tiles rw, rw + R, ..
    Rows<D, KG, ROT> T;
    T.init();
    T.lim0 = it.lim + (it.causal ? (it.r0 + 16 * rw) / G : 0);
    {
        const int last = min(left, 16 * (rw + R * (nt - 1)) + 16) - 1;
        T.lim1 = nt > 0 ? it.lim + (it.causal ? (it.r0 + last) / G : 0) : -(1 << 30);
    }

    // ---- the blocks that some row sees: sink blocks, then the tail's
    const int nsb = (p.n_sink + 31) >> 5;
    const int top = it.lim + (it.causal ? (it.r0 + left - 1) / G : 0);  // the most that a row sees
    const int nv = min(nsb, (top + p.sink + 31) >> 5) + (top > 0 ? (top + 31) >> 5 : 0);
    const int v0 = min(nv, it.split * sp.bps[it.seg]), v1 = min(nv, v0 + sp.bps[it.seg]);
    const Builder<D, KH, KB, VB, M16> B(p, it.unit, wave % PB, lane);
    const int own = wave / PB;  // the image of a phase that this wave builds
    // Block v's loads, or of the nearest coded block (fp16 blocks are read when
    // they are built): without branches, so that nothing waits for them early.
    const int ncb = (p.nq + 31) >> 5;
    const auto prefetch = [&](int v) {
        Raw<KB, VB, M16> r;
        if (ncb > 0)
            B.load(r, min(max(min(v, v1 - 1) - nsb, 0), ncb - 1));
        return r;
    };
    Raw<KB, VB, M16> raw = prefetch(v0 + own);

#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int r = 16 * (rw + R * c) + hh, rc = min(r, left - 1);
        T.lim[c] = it.lim + (it.causal ? (it.r0 + rc) / G : 0);
        T.load_query(c, sp.q + global_row(sp, it, G, it.r0 + rc) * D, p.rot_c, lane);
    }

    uint8_t* metas = lds + NI * BI;
    float* st = (float*)(metas + NI * BM + kStage * wave);
    // (two loops, so that the registers of a wave's tiles have one place in each)
    const auto walk = [&](auto tiles_now) __attribute__((always_inline)) {
        constexpr int NT = decltype(tiles_now)::value;
        for (int v = v0; v < v1; v += NI) {
            // ---- build
            const int mine = v + own;
            if (mine < v1) {
                uint8_t* img = lds + own * BI;
                float* meta = (float*)(metas + own * BM);
                const int tb = mine - nsb;
                if (tb >= 0 && 32 * tb < p.nq) {
                    B.coded_image(raw, min(32, p.nq - 32 * tb), img, meta, st);
                } else {
                    const bool sink = tb < 0;
                    const int first = sink ? 32 * mine : 32 * tb, rows = sink ? p.sink : p.ring;
                    const size_t at = (size_t)it.unit * rows * D;
                    B.rows_image((sink ? p.kq : p.kr) + at, (sink ? p.vq : p.vr) + at, first, rows,
                                 (sink ? p.n_sink : p.n) - first, img, meta);
                }
            }
            raw = prefetch(mine + NI);
            sync_lds();
            // ---- consume
            for (int i = bw; i < NI && v + i < v1; i += BW) {
                const int tb = v + i - nsb;
                const bool sink = tb < 0;
                const int t0 = sink ? 32 * (v + i) : 32 * tb, off = sink ? p.sink : 0;
                if (t0 >= T.lim1 + off)
                    continue;
                const int live = sink ? p.n_sink - t0 : p.n - t0;
                const uint8_t* img = lds + i * BI;
                const float* meta = (const float*)(metas + i * BM);
                T.template consume<NT>(img, meta, t0, off, live, lane);
            }
            sync_lds();
        }
    };
    if (CT == 1 || nt <= 1)
        walk(std::integral_constant<int, 1>{});
    else
        walk(std::integral_constant<int, CT>{});

    // ---- partials: of each wave when its rows are its own, else merged in LDS
    const float inv = T.vf == 0.0f ? 0.0f : 1.0f / T.vf;
    float* lo = (float*)lds;              // [waves][16][D]
    float* lml = lo + kWaves * 16 * D;    // [waves][16][2]
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const float l = sum_rows(T.lsum[c]);
        const int r = 16 * (rw + R * c) + hh;
        if (BW == 1) {
            if (r < left) {
                const size_t row = (size_t)it.part * sp.rows + global_row(sp, it, G, it.r0 + r);
#pragma unroll
                for (int mb = 0; mb < NMB; ++mb)
                    *(floatx4*)(sp.part_o + row * D + 16 * mb + 4 * qg) = T.oacc[c][mb] * inv;
                if (qg == 0)
                    *(float2*)(sp.part_ml + 2 * row) = make_float2(T.m[c], l);
            }
            continue;
        }
        if (c > 0)
            sync_lds();
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb)
            *(floatx4*)(lo + ((size_t)wave * 16 + hh) * D + 16 * mb + 4 * qg) = T.oacc[c][mb] * inv;
        if (qg == 0)
            *(float2*)(lml + 2 * (wave * 16 + hh)) = make_float2(T.m[c], l);
        sync_lds();
        for (int idx = threadIdx.x; idx < 16 * R * (D / 4); idx += kThreads) {
            const int row = idx / (D / 4), d = 4 * (idx % (D / 4)), w0 = row >> 4, rr = 16 * (w0 + R * c) + (row & 15);
            if (rr >= left)
                continue;
            float M = kNegInf;
            for (int w = w0; w < kWaves; w += R)
                M = fmaxf(M, lml[2 * (w * 16 + (row & 15))]);
            floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
            float L = 0.0f;
            if (M != kNegInf) {
                for (int w = w0; w < kWaves; w += R) {
                    const float2 ml = *(const float2*)(lml + 2 * (w * 16 + (row & 15)));
                    const float sc = __builtin_amdgcn_exp2f(ml.x - M);
                    acc += *(const floatx4*)(lo + ((size_t)w * 16 + (row & 15)) * D + d) * sc;
                    L += sc * ml.y;
                }
            }
            const size_t at = (size_t)it.part * sp.rows + global_row(sp, it, G, it.r0 + rr);
            *(floatx4*)(sp.part_o + at * D + d) = acc;
            if (d == 0)
                *(float2*)(sp.part_ml + 2 * at) = make_float2(M, L);
        }
    }
}

template <int D, int KG, int KB, int VB, bool M16, bool ROT>
hipError_t launch_instance(const SharedParams& p, int items, hipStream_t stream)
{
    launch_kernel(shared_kernel<D, KG, KB, VB, M16, ROT>, dim3(items), dim3(kThreads), (size_t)lds_bytes(D, KG == 0),
                  stream, p);
    return hipGetLastError();
}

template <int D, int KG, bool M16, bool ROT>
hipError_t launch_widths(const SharedParams& p, int items, hipStream_t stream)
{
    const AttnParams& a = p.seg[0];
    if (a.k_bits == 8)  // 8-bit codes come as K and V both 8-bit
        return launch_instance<D, KG, 8, 8, M16, ROT>(p, items, stream);
    if (a.k_bits == 4)
        return a.v_bits == 4 ? launch_instance<D, KG, 4, 4, M16, ROT>(p, items, stream)
                             : launch_instance<D, KG, 4, 2, M16, ROT>(p, items, stream);
    return a.v_bits == 4 ? launch_instance<D, KG, 2, 4, M16, ROT>(p, items, stream)
                         : launch_instance<D, KG, 2, 2, M16, ROT>(p, items, stream);
}

// The kernels of one head size and key grouping.
template <int D, int KG>
hipError_t launch_family(const SharedParams& p, int items, hipStream_t stream)
{
    if (p.rotate)
        return p.seg[0].meta16 ? launch_widths<D, KG, true, true>(p, items, stream)
                               : launch_widths<D, KG, false, true>(p, items, stream);
    return p.seg[0].meta16 ? launch_widths<D, KG, true, false>(p, items, stream)
                           : launch_widths<D, KG, false, false>(p, items, stream);
}

}  // namespace shr
}  // namespace kvq
