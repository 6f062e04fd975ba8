// Attention of a batch whose sequences share long prefixes
// (kvq_decode_attn_shared, kvq_prefill_attn_shared): one softmax over the
// tokens of a sequence's prefix, a sequence of the prefix cache that its whole
// group reads, and of its own suffix.
//
// The two caches are two segments.  A segment's unit (cache sequence, KV head)
// meets a set of query rows (sequence, chunk token, head): all rows of the
// group for a prefix unit, one sequence's rows for a suffix unit.  A work item
// is a range of a unit's 32-token blocks and a tile of its rows; every item
// writes an unnormalized partial (m, l, o) per row, and a last kernel joins a
// row's partials of both segments:
//     M = max m,  O = sum 2^(m - M) o / sum 2^(m - M) l.
// So the codes of a prefix are read once per tile of its group's rows instead
// of once per sequence.  Two kernels (shared.hip has the rule):
//
//   image_kernel   much work.  One workgroup per CU, of eight waves (sixteen at
//                  D = 64) and up to 16 tiles(D) waves(D) rows.  In turns, the
//                  waves convert the next images(D) blocks into images in LDS
//                  (parts(D) waves per block), then multiply their own rows with
//                  them.  With R row waves a wave has up to tiles(D) tiles of 16
//                  rows and every waves(D) / R-th image.  (Two buffers with one
//                  barrier per turn leave room for half the images, and every
//                  wave that takes part in a block repeats the work on its
//                  scales: 3 to 15% slower, in either order of the halves.)
//   direct_kernel  little work, or few rows per unit (a suffix's queries, few
//                  samples): 16 or 32 rows, four waves, each with blocks of its
//                  own, whose codes become operands in registers.
//
// Operands are in the order in which the cache stores its codes, that of
// v_mfma_f32_16x16x32_f16 (a 1 KiB fragment is one 16-byte piece per lane).
// Codes are centred (c - (2^b - 1) / 2, or c - 2^(b-1) when symmetric), exact in
// fp16; s and z' are a group's scale and the offset of its centred codes:
//   keys in per-token groups
//           the codes: S = sum_g s_g (A_g . q_g) + z'_g sum q_g;
//   keys with per-channel scales, values
//           image_kernel: reconstructed, times a power of two, as fp16 hi + lo
//           (22 bits); direct_kernel: the codes, and the other side takes the
//           scales: (q s) . c + q . z', (p s) . c + p . z', q s and p s as hi + lo.
// The product of reconstructed values with the probabilities (hi + lo as well) is
// three MFMAs, all but the 2^-22 of lo x lo, that with codes two.  But the scaled
// side costs a tile 24 vector operations (96 cycles) per value group and block
// where an image shares the 50 of a reconstructed fragment among up to 16 tiles.
// Direct, D = 256, groups of 64: 55 us with reconstructed values, 46 with codes.
// (Codes that are not centred cost precision where outputs are small beside the
// values: 32768 tokens of flat attention were 4.7e-4 off with decode attention's
// operands and are 4e-7 with these.)
// fp16 tokens (window, sink) are operands as they are, with a lo half of zero.
//
// What bounds them (MI355X): image_kernel, 64 sequences x 4 heads per KV head, 32768
// rotated tokens at D = 128, 92 us: the matrix pipes 0.42 and the vector pipes 0.39 of
// its waves' time, which add up instead of overlapping whatever the waves' order,
// priority or number (sixteen waves at D = 128: 15% slower); without LDS reads 2% faster.
// 930 TFLOP/s of executed products, where a large library product reaches 1160.
// direct_kernel: vector operations of the conversions, and at small sizes the
// latency of one block after another.
//
// Softmax: online per column in base 2, by the size of the products rather than
// that of the weights.  A token's values are multiplied by its own power of two f_t
// (largest magnitude 2^11 to 2^12), and its score x_t (log2 units) is taken as
//     x'_t = x_t - log2 f_t + 10,
// so that a reference R that follows max x' makes p'_t = 2^(x'_t - R + kPBits) and
// f_t v_t fp16 operands with all of their bits wherever p v is not negligible beside the
// row's largest product, however far apart values and weights are:
//     sum_t p'_t (f_t v_t) = 2^(kPBits + 10) sum_t 2^(x_t - R) v_t,
//     sum_t p'_t (f_t / 2^10) = 2^kPBits sum_t 2^(x_t - R).
// (With one power of two per block, for which the probabilities of smaller values made
// up, outputs beside blocks of values 2^20 times theirs and no weight were up to 8e-4
// off, D = 256; they are 4e-7 off with these.)  The scores are multiplied by
// their query's power of two anyway, so the addition of 10 - log2 f_t costs nothing; a
// block costs its tokens' maxima: -3 to +4% of listed calls with the queries' powers.
// R is an integer, raised only when a block exceeds it by more than kTau: rescaling is
// exact, p' at most 2^(kTau + kPBits).  Causal rows (suffix segments of a chunk) are
// masked per column, and blocks that no row of a wave sees are skipped.
#pragma once

#include <type_traits>

#include "kvq_device.h"
#include "kvq_internal.h"

namespace kvq {
namespace shr {
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr float kTau = 4.0f;     // lazy rescale threshold, log2 units
constexpr float kPBits = 10.0f;  // probabilities are kept times 2^kPBits, so that their lo half is exact
constexpr float kNegInf = -__builtin_inff();

// ---- image_kernel
// Waves of a workgroup, the only one on its CU, and 16-row tiles of a wave.  The
// accumulators and queries of 32 rows at D = 128 and of 16 at D = 256 fit the
// 256 registers of two waves per SIMD; at D = 64 16 rows fit the 128 of four (200
// tokens after 2048: 3% faster than 32 rows in two).
__host__ __device__ constexpr int waves(int D)
{
    return D == 64 ? 16 : 8;
}

__host__ __device__ constexpr int tiles(int D)
{
    return D == 128 ? 2 : 1;
}

__host__ __device__ constexpr int item_rows(int D)
{
    return 16 * tiles(D) * waves(D);
}

// Images of a turn, and waves that build one: four key and four value pieces
// per lane.
__host__ __device__ constexpr int images(int D)
{
    return 512 / D;
}

__host__ __device__ constexpr int parts(int D)
{
    return waves(D) / images(D);
}

// LDS: the images, per image its key scales and offsets ([group][32] each), its
// tokens' powers of two (see TokenPowers) and two scalars, then per wave room to
// pass a block's scales and offsets between lanes.  The merge of the waves reuses
// it from the start.
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
    return 2 * (D / 32) * 128 + 256 + 16;
}

__host__ __device__ constexpr int stage_bytes(int D)
{
    return 8 * D;
}

// Floats per row of the waves' partials in LDS (16 rows next to each other are
// written at once: a pitch of D would be one bank for all of them).
__host__ __device__ constexpr int merge_pitch(int D)
{
    return D + 4;
}

__host__ __device__ constexpr int image_lds(int D, bool hilo)
{
    const int walk = images(D) * (image_bytes(D, hilo) + meta_bytes(D)) + waves(D) * stage_bytes(D);
    const int merge = waves(D) * 16 * (merge_pitch(D) + 2) * 4;
    return walk > merge ? walk : merge;
}

// Waves that share an item's rows, of n16 tiles; waves(D) / it take turns at the images.
__host__ __device__ constexpr int row_waves(int D, int n16)
{
    int R = waves(D) / images(D);
    while (R * tiles(D) < n16)
        R *= 2;
    return R;
}

// ---- direct_kernel
constexpr int kDirectWaves = 4, kDirectThreads = 64 * kDirectWaves;

// 16-row tiles of a wave, which shares a block's codes between them: as many as
// fit the registers beside wide codes or the conversion of fp16 tokens and, at
// D = 128, the lo halves of rotated queries or the scales of groups of 32.  Two tiles /
// one, us: 96 sequences at D = 64 26 / 37, D = 128 (4-bit groups of 64) 256 rows
// 50 / 50 (16384 tokens), 71 / 89 (32768); where two spill, 32 sequences of 4096 tokens
// and more: rotated 41 / 31, 4-bit groups of 32 62 / 34, 2-bit 50 / 28.
__host__ __device__ constexpr int direct_tiles(int D, int kg, int bits, bool rot, bool fp16)
{
    return D == 256 || bits == 8 || fp16 || (D == 128 && (kg == 1 || rot)) ? 1 : 2;
}

// Per wave: what an image has of scales, offsets and powers, then the block's value
// scales and offsets, or (fp16 tokens) its values transposed, [D][kVtPitch].
constexpr int kVtPitch = 40;  // halves

__host__ __device__ constexpr int direct_region(int D, bool fp16)
{
    return meta_bytes(D) + (fp16 ? 2 * kVtPitch * D : stage_bytes(D));
}

__host__ __device__ constexpr int direct_lds(int D, bool fp16)
{
    const int walk = kDirectWaves * direct_region(D, fp16), merge = kDirectWaves * 16 * (merge_pitch(D) + 2) * 4;
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

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t x)
{
    return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, false);
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

// A power of two f with x f in (2^11, 2^12] (x >= 0; f is kept within 2^-115 .. 2^113).
__device__ __forceinline__ float scale_to_range(float x)
{
    const uint32_t e = min(max((__float_as_uint(x) >> 23) + 1, 26u), 254u);  // x < 2^(e - 127)
    return __uint_as_float((254 + 12 - e) << 23);
}

// The larger of two pairs of 16-bit numbers.
__device__ __forceinline__ uint32_t max_pairs(uint32_t a, uint32_t b)
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// The powers of two of a token's values: f brings its largest magnitude x (below
// 2^(e - 127)) to 2^12 at most; start is what its scores begin with, 10 - log2 f;
// weight, 2^-start, makes p' a weight again.  e >= 101 (f <= 2^38) leaves room
// for every coded token, whose scale is 1e-8 or more.
struct TokenPowers {
    static constexpr uint32_t kLeast = 101;
    uint32_t e;
    __device__ __forceinline__ explicit TokenPowers(uint32_t e_, uint32_t least = kLeast) : e(min(max(e_, least), 254u)) {}
    // Of a row of fp16 numbers with the sum of squares n2: f within fp16, 2^-8 .. 2^15
    static __device__ __forceinline__ TokenPowers of_row(float n2)
    {
        return TokenPowers((uint32_t)max(127 + (((int)(__float_as_uint(n2) >> 23) - 125) >> 1), 0), 124);
    }
    __device__ __forceinline__ float f(int log2_pre = 0) const { return __uint_as_float((266 + log2_pre - e) << 23); }
    __device__ __forceinline__ float start() const { return (float)((int)e - 129); }
    __device__ __forceinline__ float weight() const { return __uint_as_float((256 - e) << 23); }
};

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float add_squares(const u32x4& w, float sum)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f16x2 x = __builtin_bit_cast(f16x2, (uint32_t)w[j]);
        sum = __builtin_amdgcn_fdot2(x, x, sum, false);
    }
    return sum;
}

// A value operand times its tokens' powers, fp16 pairs (f_j, f_(j + 4)).
__device__ __forceinline__ half8 times_powers(const u32x4& v, const u32x4& f)
{
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        w[j] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, (uint32_t)v[j]) *
                                                __builtin_bit_cast(f16x2, (uint32_t)f[j]));
    return __builtin_bit_cast(half8, w);
}

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

// The loads of one wave's part of a coded block: NK key pieces and NV value
// pieces per lane, and of the block's key and value scales and offsets (at most
// D of each) NM = D / 64 numbers, the keys' in NW words.
template <int KB, int VB, int NK, int NV, int NM, int NW>
struct Raw {
    uint32_t k[NK * KB / 4], v[NV * VB / 4];
    uint32_t ks[NW], kz[NW], vs[NM], vz[NM];
};

// N bytes (2 to 128, aligned to N or 16) from global memory, streaming.
template <int N>
__device__ __forceinline__ void load_bytes(const uint8_t* at, uint32_t* w)
{
    if constexpr (N == 2) {
        w[0] = __builtin_nontemporal_load((const uint16_t*)at);
    } else if constexpr (N == 4) {
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

// Conversion of a segment's unit: part `part` of PB of every block.
template <int D, bool KH, int KB, int VB, bool M16, int PB>
struct Builder {
    static constexpr int NKB = D / 32, NMB = D / 16, NK = 2 * NKB / PB, NV = NMB / PB;
    static constexpr int NM = D / 64, ESZ = M16 ? 2 : 4;  // numbers of a lane, and their bytes
    typedef Raw<KB, VB, NK, NV, NM, (NM * ESZ + 3) / 4> Loads;
    const AttnParams& p;
    int unit, part, lane;
    int nk, nv;        // key and value scales of a block
    bool kaff, vaff;
    const uint8_t *k, *v, *ks;       // this lane's pieces and numbers of block 0
    const uint8_t* vs;               // the unit's value scales
    uint32_t vlane;                  // this lane's first of a block
    long dkz, dvz;                   // offsets - scales (0 when symmetric: the scales once more)

    // key piece i of the lane: half block and 32-channel block
    __device__ __forceinline__ int half(int i) const { return PB == 1 ? i / NKB : (part * NK + i) / NKB; }
    __device__ __forceinline__ int kblock(int i) const { return PB == 1 ? i % NKB : (part * NK + i) % NKB; }

    __device__ __forceinline__ Builder(const AttnParams& p_, int unit_, int part_, int lane_)
        : p(p_), unit(unit_), part(part_), lane(lane_)
    {
        const size_t ub0 = (size_t)unit * (p.T >> 5);
        nk = KH ? D : 32 * (D / p.k_group);
        nv = 32 * (D / p.v_group);
        kaff = p.k_mode == KVQ_AFFINE;
        vaff = p.v_mode == KVQ_AFFINE;
        k = (const uint8_t*)p.kc + ((ub0 * 2 + half(0)) * 64 + lane) * (NKB * KB) + kblock(0) * KB;
        v = (const uint8_t*)p.vc + (ub0 * 64 + lane) * (NMB * VB) + NV * part * VB;
        ks = (const uint8_t*)p.ks + (ub0 * nk + min(NM * lane, nk - NM)) * ESZ;
        vs = (const uint8_t*)p.vs + ub0 * nv * ESZ;
        vlane = (nv < 64 ? lane & 31 : lane) * ESZ;
        dkz = kaff ? (const uint8_t*)p.kz - (const uint8_t*)p.ks : 0;
        dvz = vaff ? (const uint8_t*)p.vz - (const uint8_t*)p.vs : 0;
    }

    // Every lane issues the same loads whatever the block.
    __device__ __forceinline__ void load(Loads& r, int blk) const
    {
        const uint8_t* kb = k + (size_t)blk * (2 * 64 * NKB * KB);
        if constexpr (PB == 1) {
            load_bytes<NKB * KB>(kb, r.k);
            load_bytes<NKB * KB>(kb + 64 * NKB * KB, r.k + NKB * KB / 4);
        } else {
            load_bytes<NK * KB>(kb, r.k);
        }
        load_bytes<NV * VB>(v + (size_t)blk * (64 * NMB * VB), r.v);
        const uint8_t *a = ks + (size_t)blk * (nk * ESZ), *b = vs + (size_t)blk * (nv * ESZ);
        load_bytes<NM * ESZ>(a, r.ks);
        load_bytes<NM * ESZ>(a + dkz, r.kz);
        // Value numbers 64 e + lane, so that a lane's are all of one token, lane % 32
        // (past the last group: the first ones once more).
#pragma unroll
        for (int e = 0; e < NM; ++e) {
            const uint8_t* at = b + (64 * e < nv ? 64 * e * ESZ : 0);
            load_bytes<ESZ>(at + vlane, r.vs + e);
            load_bytes<ESZ>(at + dvz + vlane, r.vz + e);
        }
    }

    // A scale and the offset of its centred codes; zeros of a dead token.
    __device__ __forceinline__ void widen(uint16_t s, uint16_t z, bool aff, float mid, bool on, float* sv, float* zv) const
    {
        widen(f16_bits_to_f32(s), f16_bits_to_f32(z), aff, mid, on, sv, zv);
    }

    __device__ __forceinline__ void widen(float s, float z, bool aff, float mid, bool on, float* sv, float* zv) const
    {
        *sv = on ? s : 0.0f;
        *zv = on && aff ? fmaf(mid, *sv, z) : 0.0f;
    }

    // This lane's key scales and offsets (number NM lane + e is token (NM lane + e) % 32
    // of a group, unless `whole`).
    __device__ __forceinline__ void widen_keys(const Loads& r, float mid, int live, bool whole, float* sv, float* zv) const
    {
#pragma unroll
        for (int e = 0; e < NM; ++e) {
            const bool on = whole || ((NM * lane + e) & 31) < live;
            if constexpr (M16)
                widen((uint16_t)(r.ks[e >> 1] >> (16 * (e & 1))), (uint16_t)(r.kz[e >> 1] >> (16 * (e & 1))), kaff, mid, on,
                      sv + e, zv + e);
            else
                widen(__uint_as_float(r.ks[e]), __uint_as_float(r.kz[e]), kaff, mid, on, sv + e, zv + e);
        }
    }

    // This lane's numbers (of n) times f to st (scales) and st + D (offsets).
    __device__ __forceinline__ void put(float* st, const float* sv, const float* zv, float f, int n) const
    {
        if (NM * lane < n) {
#pragma unroll
            for (int e = 0; e < NM; ++e) {
                st[NM * lane + e] = sv[e] * f;
                st[D + NM * lane + e] = zv[e] * f;
            }
        }
    }

    // A power of two that brings the block's largest magnitude |offset| + mid
    // scale to 2^12 at most: hi + lo then holds every element to 2^-37 of it.
    __device__ __forceinline__ float range_scale(const float* sv, const float* zv, float mid, int n) const
    {
        float top = 0.0f;
#pragma unroll
        for (int e = 0; e < NM; ++e)
            top = fmaxf(top, fmaf(mid, sv[e], fabsf(zv[e])));
        return scale_to_range(wave_max(NM * lane < n ? top : 0.0f));
    }

    // The key scales of a coded block: per-token groups (times sm_scale log2 e) to
    // meta, [group][32] scales and offsets; per-channel ones (times a power of two
    // and pre) to st, [channel].  Returns what the scores of the latter take.
    __device__ __forceinline__ float key_scales(const Loads& r, int live, float* meta, float* st, float pre = 1.0f) const
    {
        float sv[NM], zv[NM];
        const float mid = coding<KB>(kaff).mid;
        widen_keys(r, mid, live, KH, sv, zv);
        if constexpr (KH) {
            const float f = range_scale(sv, zv, mid, nk) * pre;
            put(st, sv, zv, f, nk);
            return p.sm_log2 * (1.0f / f);
        } else {
            put(meta, sv, zv, p.sm_log2, nk);
            return 0.0f;
        }
    }

    // The value scales of a coded block, times 2^LOG2_PRE and each token's power of
    // two, to st, [group][32], and the powers (start, weight: [32] each) to at.  Whether a
    // token has 2^66 or more (uniform).
    template <int LOG2_PRE>
    __device__ __forceinline__ bool value_scales(const Loads& r, int live, float* st, float* at) const
    {
        float sv[NM], zv[NM], top = 0.0f;
        const float mid = coding<VB>(vaff).mid;
        const bool on = (lane & 31) < live;
#pragma unroll
        for (int e = 0; e < NM; ++e) {
            if constexpr (M16)
                widen((uint16_t)r.vs[e], (uint16_t)r.vz[e], vaff, mid, on, sv + e, zv + e);
            else
                widen(__uint_as_float(r.vs[e]), __uint_as_float(r.vz[e]), vaff, mid, on, sv + e, zv + e);
            top = fmaxf(top, fmaf(mid, sv[e], fabsf(zv[e])));
        }
        auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
        const TokenPowers t((__float_as_uint(top) >> 23) + 1);
        // (numbers past the last group go to room that nobody reads)
#pragma unroll
        for (int e = 0; e < NM; ++e) {
            st[64 * e + lane] = sv[e] * t.f(LOG2_PRE);
            st[D + 64 * e + lane] = zv[e] * t.f(LOG2_PRE);
        }
        if (part == 0 && lane < 32) {
            at[lane] = t.start();
            at[32 + lane] = t.weight();
        }
        return __any(top >= 0x1p66f);
    }

    // Eight reconstructed elements of the codes' operand a, hi + lo; s: their
    // scales (natural order), offsets D further.
    static __device__ __forceinline__ void reconstruct(const half8& a, const float* s, half8* hi, half8* lo)
    {
        const float4 s0 = *(const float4*)s, s1 = *(const float4*)(s + 4);
        const float4 z0 = *(const float4*)(s + D), z1 = *(const float4*)(s + D + 4);
        const float sn[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
        const float zn[8] = {z0.x, z0.y, z0.z, z0.w, z1.x, z1.y, z1.z, z1.w};
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            x[j] = fmaf((float)a[j], sn[perm4(j)], zn[perm4(j)]);
        split_nearest(x, hi, lo);
    }

    __device__ __forceinline__ half8 key_codes(const Loads& r, int i) const
    {
        return centred<KB>(r.k, i, coding<KB>(kaff).centre);
    }

    __device__ __forceinline__ half8 value_codes(const Loads& r, int i) const
    {
        return centred<VB>(r.v, i, coding<VB>(vaff).centre);
    }

    // Key piece i: the codes (lo untouched), or the reconstructed keys.
    __device__ __forceinline__ void key_piece(const Loads& r, int i, const float* st, half8* hi, half8* lo) const
    {
        const half8 a = key_codes(r, i);
        if constexpr (KH)
            reconstruct(a, st + 32 * kblock(i) + 8 * (lane >> 4), hi, lo);
        else
            *hi = a;
    }

    // Value piece i (channels 16 (NV part + i) + lane % 16).
    __device__ __forceinline__ void value_piece(const Loads& r, int i, const float* st, half8* hi, half8* lo) const
    {
        const int g = 16 * (NV * part + i) >> (31 - __builtin_clz(p.v_group));
        reconstruct(value_codes(r, i), st + 32 * g + 8 * (lane >> 4), hi, lo);
    }

    // This wave's part of the image of a coded block whose first `live` tokens
    // exist.  img: the image; meta: its scales and powers; st: this wave's stage.
    __device__ __forceinline__ void coded_image(const Loads& r, int live, uint8_t* img, float* meta, float* st) const
    {
        const float ksm = KH || part == 0 ? key_scales(r, live, meta, st) : 0.0f;
        lds_order();
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            half8 hi, lo;
            key_piece(r, i, st, &hi, &lo);
            uint8_t* at = img + 1024 * (half(i) * NKB + kblock(i)) + 16 * lane;
            *(half8*)at = hi;
            if constexpr (KH)
                *(half8*)(at + 64 * D) = lo;
        }
        lds_order();
        const bool huge = value_scales<0>(r, live, st, meta + 2 * D);
        lds_order();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            half8 hi, lo;
            value_piece(r, i, st, &hi, &lo);
            uint8_t* at = img + key_bytes(D, KH) + 1024 * (NV * part + i) + 16 * lane;
            *(half8*)at = hi;
            *(half8*)(at + 64 * D) = lo;
        }
        if (part == 0 && lane == 0) {
            meta[2 * D + 64] = ksm;
            meta[2 * D + 65] = huge;
        }
    }

    // ---- Blocks of fp16 rows: token i is row (first + i) % ring of kr, vr [.][D],
    // the first `live` exist.  (Dead tokens read a live row and are cleared: no
    // load waits for a branch.)
    __device__ __forceinline__ int key_token(int i) const { return 8 * ((lane & 15) >> 2) + 4 * half(i) + (lane & 3); }

    __device__ __forceinline__ u32x4 load_key_row(const uint16_t* kr, int first, int ring, int live, int i) const
    {
        const int t = min(key_token(i), live - 1);
        return *(const u32x4*)(kr + (uint32_t)((first + t) % ring * D + 32 * kblock(i) + 8 * (lane >> 4)));
    }

    __device__ __forceinline__ half8 key_row_piece(const u32x4& w, int live, int i) const
    {
        const bool on = key_token(i) < live;
        u32x4 a;  // dword j: channels j and j + 4
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x = w[j >> 1], y = w[2 + (j >> 1)];
            a[j] = !on ? 0u : j & 1 ? (x >> 16) | (y & 0xFFFF0000u) : (x & 0xFFFFu) | (y << 16);
        }
        return __builtin_bit_cast(half8, a);
    }

    // Element offsets of this lane's eight tokens (operand order) in vr.
    __device__ __forceinline__ void value_rows(int first, int ring, int live, uint32_t* row) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            row[j] = (uint32_t)((first + min(8 * (lane >> 4) + perm4(j), live - 1)) % ring * D + (lane & 15));
    }

    __device__ __forceinline__ u32x4 value_row_piece(const uint16_t* vr, const uint32_t* row, int live, int i) const
    {
        uint16_t h[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            h[j] = vr[row[j] + 16 * (NV * part + i)];
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = 8 * (lane >> 4) + j < live ? h[2 * j] : 0u;
            w[j] |= 8 * (lane >> 4) + j + 4 < live ? (uint32_t)h[2 * j + 1] << 16 : 0u;
        }
        return w;
    }

    // A row's powers to at (start, weight), `start` more of the scores' start.
    __device__ __forceinline__ void put_powers(const TokenPowers& t, int token, float* at, int start) const
    {
        at[token] = t.start() + (float)start;
        at[32 + token] = t.weight() * __uint_as_float((uint32_t)(127 - start) << 23);
    }

    // The scales of fp16 rows: ones (times the softmax scale for code operands).
    __device__ __forceinline__ void row_scales(float* meta) const
    {
        if (part != 0)
            return;
        if constexpr (!KH) {
            if (NM * lane < nk) {
#pragma unroll
                for (int e = 0; e < NM; ++e)
                    meta[NM * lane + e] = p.sm_log2;
            }
        }
        if (lane == 0) {
            meta[2 * D + 64] = p.sm_log2;
            meta[2 * D + 65] = 0.0f;
        }
    }

    // The image of a block of fp16 rows in two parts, a barrier between them: the
    // rows, whose tokens' largest magnitudes among this wave's values (pairs of fp16,
    // tokens 8 qg + j and + 4) go to st; then the values times their tokens' powers, from
    // the maxima of all of the block's waves (their stages lie at sts).  (Every wave
    // reading all of the values for their maxima is a read's latency more per turn: 158
    // us instead of 145, 200 KIVI tokens after 2048 at D = 256.)
    __device__ __forceinline__ void rows_image(const uint16_t* kr, const uint16_t* vr, int first, int ring, int live,
                                               uint8_t* img, float* meta, float* st) const
    {
        const half8 zero = {};
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            uint8_t* at = img + 1024 * (half(i) * NKB + kblock(i)) + 16 * lane;
            *(half8*)at = key_row_piece(load_key_row(kr, first, ring, live, i), live, i);
            if constexpr (KH)
                *(half8*)(at + 64 * D) = zero;
        }
        uint32_t row[8];
        value_rows(first, ring, live, row);
        u32x4 top = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            uint8_t* at = img + key_bytes(D, KH) + 1024 * (NV * part + i) + 16 * lane;
            const u32x4 v = value_row_piece(vr, row, live, i);
            *(u32x4*)at = v;
            *(half8*)(at + 64 * D) = zero;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                top[j] = max_pairs(top[j], v[j] & 0x7FFF7FFFu);
        }
        row_scales(meta);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t x = top[j];
            x = max_pairs(x, dpp_u32<0xB1>(x));  // the 16 lanes of a token
            x = max_pairs(x, dpp_u32<0x4E>(x));
            x = max_pairs(x, dpp_u32<0x141>(x));
            x = max_pairs(x, dpp_u32<0x140>(x));
            top[j] = x;
        }
        if ((lane & 15) == 0)
            *(u32x4*)(st + (lane >> 2)) = top;
    }

    __device__ __forceinline__ void rows_scale(const uint8_t* sts, uint8_t* img, float* meta) const
    {
        const int qg = lane >> 4;
        u32x4 f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            f[j] = 0;
#pragma unroll
        for (int q = 0; q < PB; ++q) {
            const u32x4 x = *(const u32x4*)(sts + stage_bytes(D) * q + 16 * qg);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                f[j] = max_pairs(f[j], x[j]);
        }
        // fp16 exponents E, at least 11: a magnitude is below 2^(E - 14), f = 2^(26 - E)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            f[j] = max_pairs(f[j] & 0x7C007C00u, 0x2C002C00u);
        if (part == 0 && (lane & 15) == 0) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                put_powers(TokenPowers(113 + (f[k & 3] >> (k < 4 ? 10 : 26) & 31)), 8 * qg + k, meta + 2 * D, 0);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            f[j] = 0xA400A400u - f[j];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            uint8_t* at = img + key_bytes(D, KH) + 1024 * (NV * part + i) + 16 * lane;
            *(half8*)at = times_powers(*(const u32x4*)at, f);
        }
    }
};

// ------------------------------------------------------------ rows

// A power of two <= 1 by which scales in range_scale's range are at most one
// (mid scale <= 2^12): the row side's operand x scale is no larger than x then.
template <int BITS>
__host__ __device__ constexpr int log2_to_one()
{
    return BITS == 8 ? -5 : BITS == 4 ? -9 : -11;
}

template <int BITS>
__device__ __forceinline__ constexpr float to_one()
{
    return 1.0f / (float)(1 << -log2_to_one<BITS>());
}

// A wave's state: NT tiles of 16 query rows (columns of the MFMAs).  KG: key
// group size / 32 (0: per-channel scales).  ROT: rotated queries, hi + lo.
// DIRECT: direct_kernel's, which takes value offsets apart.  (The scores l of a block
// include the tokens' starts; nl: where a block's starts and weights are.)
template <int D, int KG, bool ROT, int CT, bool DIRECT>
struct Rows {
    static constexpr int NKB = D / 32, NMB = D / 16;
    static constexpr bool KH = KG == 0;
    static constexpr int KS = KH ? NKB : KG, NG = NKB / KS;
    // Offsets of up to two groups are added by vector operations (eight per group
    // and tile, 32 cycles), of more by an fp32 MFMA per four (two of 32 cycles).
    static constexpr bool ZM = NG > 2;
    static constexpr int NZ = ZM ? (NG + 3) / 4 : NG;
    half8 q[CT][NKB], ql[ROT ? CT : 1][ROT ? NKB : 1];
    float qz[CT][NZ];        // lane (col, qg): the query's sum over group 4 j + qg (ZM), or over group j
    float qinv[CT];          // q and qz are this column's query divided by it
    floatx4 oacc[CT][NMB];
    float zacc[CT][DIRECT ? D / 32 : 1];  // this lane's sum of p x value offset, at the first 32 channels of each group
    float m[CT], lsum[CT];   // reference of the probabilities (an integer), lane partial sum (times 2^kPBits)
    bool apart;              // a token is so large that the sums are taken apart (uniform)
    int lim[CT];             // tail tokens that this lane's column sees (may be negative: only sink tokens)
    int lim0, lim1;          // the least and the most of the wave's rows (uniform)

    // Query rows of tile c, this lane's at src (channels 32 kb + 8 qg .. + 7 of it),
    // each times a power of two of its own that brings its largest element to 2^7 ..
    // 2^8 (the transform adds at most four bits): fp16 operands of small queries would
    // be subnormal.  (Per row, not per workgroup: a row of a padded batch may hold
    // anything.)  Queries of 2^-10: 1e-5 off without it, 3e-4 with per-channel keys;
    // 5e-7 and 7e-7 with it.  It costs the scores of keys in groups a product.
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
        float top = 0.0f;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                top = fmaxf(top, fabsf(v[kb][j]));
        const uint32_t e = max(__float_as_uint(max_rows(top)) >> 23, 34u);  // top < 2^(e - 126)
        const float g = __uint_as_float((261 - e) << 23) * (ROT ? rot_c : 1.0f);
        qinv[c] = __uint_as_float((e - 7) << 23);
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
                x[j] = v[kb][perm4(j)] * g;
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
                qz[c][j] = ZM ? 0.0f : sum_rows(sum[j]);
#pragma unroll
            for (int g = 0; ZM && g < NG; ++g) {
                const float s = sum_rows(sum[g]);
                qz[c][g / 4] = qg == g % 4 ? s : qz[c][g / 4];
            }
        }
    }

    __device__ __forceinline__ void init()
    {
        apart = false;
#pragma unroll
        for (int c = 0; c < CT; ++c) {
#pragma unroll
            for (float& z : zacc[c])
                z = 0.0f;
            m[c] = kNegInf;
            lsum[c] = 0.0f;
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb)
                oacc[c][mb] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }

    // ---- A block takes four steps: scores (matrix products), settle (masks,
    // running maxima), probabilities (vector operations), values (matrix
    // products).

    __device__ __forceinline__ void scale_offsets(int c, float by)
    {
        if constexpr (DIRECT) {
#pragma unroll
            for (float& z : zacc[c])
                z *= by;
        }
    }

    // Masks and the running references; shift is for probabilities().  The block is
    // tokens t0 .. t0 + 31 (tail indices; with `off` = the sink's size for sink
    // blocks), the first `live` of which exist.
    template <int NT>
    __device__ __forceinline__ void settle(float (*l)[8], const float* nl, int t0, int off, int live, int lane, float* shift)
    {
        const int qg = lane >> 4;
        if (live < 32 || t0 + 32 > lim0 + off) {
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                const int valid = min(live, lim[c] + off - t0);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    l[c][k] = 8 * qg + k < valid ? l[c][k] : kNegInf;
            }
        }
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            float bm = fmaxf(fmaxf(fmaxf(l[c][0], l[c][1]), fmaxf(l[c][2], l[c][3])),
                             fmaxf(fmaxf(l[c][4], l[c][5]), fmaxf(l[c][6], l[c][7])));
            if (__any(bm > m[c] + kTau)) {
                bm = max_rows(bm);
                const float mn = bm > m[c] + kTau ? __builtin_rintf(bm) : m[c];
                const float alpha = m[c] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m[c] - mn);
                m[c] = mn;
                lsum[c] *= alpha;
#pragma unroll
                for (int mb = 0; mb < NMB; ++mb)
                    oacc[c][mb] *= alpha;
                scale_offsets(c, alpha);
            }
            // (a column that has seen no token keeps m = -inf and gets zeros)
            shift[c] = kPBits - (m[c] == kNegInf ? 0.0f : m[c]);
        }
        // Beside values of 2^66 and more the probabilities of small ones leave
        // binary32's range, but their weights are to be counted.
        if (apart) {
            float start[8];
            load_natural(nl + 8 * qg, start);
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                float top = kNegInf, sum = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    top = fmaxf(top, l[c][k] - start[k]);
                top = max_rows(top);
                top = top == kNegInf ? 0.0f : top;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    sum += __builtin_amdgcn_exp2f(l[c][k] - start[k] - top);
                lsum[c] = fmaf(sum, __builtin_amdgcn_exp2f(top + shift[c]), lsum[c]);
            }
        }
    }

    // The probabilities of tile c in operand order; summed as weights.
    __device__ __forceinline__ void exponentials(int c, const float* l, const float* weight, float shift, float* pv)
    {
        float ps = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            pv[j] = __builtin_amdgcn_exp2f(l[perm4(j)] + shift);
            ps = fmaf(pv[j], weight[perm4(j)], ps);
        }
        lsum[c] += apart ? 0.0f : ps;
    }

    template <int NT>
    __device__ __forceinline__ void probabilities(const float (*l)[8], const float* nl, const float* shift, int lane,
                                                  half8* ph, half8* pl)
    {
        float weight[8];
        load_natural(nl + 32 + 8 * (lane >> 4), weight);
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            float pv[8];
            exponentials(c, l[c], weight, shift[c], pv);
            split_nearest(pv, &ph[c], &pl[c]);
        }
    }

    static __device__ __forceinline__ void load_natural(const float* at, float* x)
    {
        const float4 a = *(const float4*)at, b = *(const float4*)(at + 4);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
        x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    }

    // ---- The matrix products of an image in LDS.  Its fragments are read in the
    // order of use, kAhead of them ahead of their products, through one ring
    // of registers: keys, then values, then the keys of the next image.  (Left
    // to itself the compiler reads each fragment right before its products,
    // whose wait for LDS is longer than the products.)
    static constexpr int kAhead = 4, NKF = 2 * NKB * (KH ? 2 : 1), NF = NKF + 2 * NMB;
    static_assert(NKF % kAhead == 0 && NF % kAhead == 0, "a fragment's slot does not depend on the image");

    // fragment k at fb (the image + 16 lane): (half, 32 channels, hi / lo) of the keys, (16 channels, hi / lo) of the values
    static __device__ __forceinline__ half8 fragment(const uint8_t* fb, int k)
    {
        const int at = k >= NKF ? key_bytes(D, KH) + 1024 * ((k - NKF) >> 1) + 64 * D * ((k - NKF) & 1)
                       : KH     ? 1024 * (k >> 1) + 64 * D * (k & 1)
                                : 1024 * k;
        return *(const half8*)(fb + at);
    }

    // S += offset x sum of the group's query, of half e: all groups, and one group.
    template <int NT>
    __device__ __forceinline__ void add_offset_products(floatx4* S, const float* meta, int e, int lane)
    {
        // row hh of the half is token 8 (hh / 4) + 4 e + hh % 4
        const int qg = lane >> 4, hh = lane & 15, tok = 8 * (hh >> 2) + 4 * e + (hh & 3);
#pragma unroll
        for (int j = 0; j < NZ; ++j) {
            const float z = meta[D + 32 * min(4 * j + qg, NG - 1) + tok];  // (times a zero sum past the last group)
#pragma unroll
            for (int c = 0; c < NT; ++c)
                S[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(z, qz[c][j], S[c], 0, 0, 0);
        }
    }

    template <int NT>
    __device__ __forceinline__ void add_group_offset(floatx4* S, const float* meta, int g, int e, int lane)
    {
        const floatx4 z = *(const floatx4*)(meta + D + 32 * g + 8 * (lane >> 4) + 4 * e);
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                S[c][i] = fmaf(z[i], qz[c][g], S[c][i]);
    }

    // The scores of half e from its sums and the tokens' starts; sm: what the sums take beside the query's power.
    template <int NT>
    __device__ __forceinline__ void finish(const floatx4* S, float sm, const float* nl, int e, int lane, float (*l)[8]) const
    {
        const floatx4 start = *(const floatx4*)(nl + 8 * (lane >> 4) + 4 * e);
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                l[c][4 * e + i] = fmaf(S[c][i], sm * qinv[c], start[i]);
    }

    // The scores of the image at fb; the ring holds its first fragments.
    template <int NT>
    __device__ __forceinline__ void image_scores(half8* ring, const uint8_t* fb, const float* meta, bool affine, int lane,
                                                 float (*l)[8])
    {
        const int qg = lane >> 4;
        constexpr int PER = KH ? 2 : 1, GF = KS * PER;  // fragments of a key piece, and of a group
        const float ksm = KH ? meta[2 * D + 64] : 0.0f;
        floatx4 S[NT], acc[NT], s4;
#pragma unroll
        for (int k = 0; k < NKF; ++k) {
            const int e = k / (NKF / 2), kk = k % (NKF / 2), g = kk / GF, kb = kk / PER;
            if (kk == 0) {
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    S[c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
                if constexpr (!KH && ZM) {
                    if (affine)
                        add_offset_products<NT>(S, meta, e, lane);
                }
            }
            if (kk % GF == 0) {
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    acc[c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
                if constexpr (!KH)
                    s4 = *(const floatx4*)(meta + 32 * g + 8 * qg + 4 * e);
            }
            const half8 a = ring[k % kAhead];
#pragma unroll
            for (int c = 0; c < NT; ++c)
                acc[c] = mfma16(a, q[c][kb], acc[c]);
            if constexpr (ROT) {
                if (!KH || k % 2 == 0) {  // (all but lo x lo)
#pragma unroll
                    for (int c = 0; c < NT; ++c)
                        acc[c] = mfma16(a, ql[c][kb], acc[c]);
                }
            }
            ring[k % kAhead] = fragment(fb, k + kAhead);
            __builtin_amdgcn_sched_barrier(0);
            if (kk % GF == GF - 1) {
#pragma unroll
                for (int c = 0; c < NT; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        S[c][i] = KH ? acc[c][i] : fmaf(s4[i], acc[c][i], S[c][i]);
                if constexpr (!KH && !ZM) {
                    if (affine)
                        add_group_offset<NT>(S, meta, g, e, lane);
                }
            }
            if (kk == NKF / 2 - 1)
                finish<NT>(S, KH ? ksm : 1.0f, meta + 2 * D, e, lane, l);
        }
    }

    // The value products of the image at fb; the ring goes on with the image at `next`.
    template <int NT>
    __device__ __forceinline__ void image_values(half8* ring, const uint8_t* fb, const uint8_t* next, const half8* ph,
                                                 const half8* pl)
    {
#pragma unroll
        for (int k = NKF; k < NF; ++k) {
            const int mb = (k - NKF) >> 1;
            const half8 a = ring[k % kAhead];
#pragma unroll
            for (int c = 0; c < NT; ++c)
                oacc[c][mb] = mfma16(a, ph[c], oacc[c][mb]);
            if ((k - NKF) % 2 == 0) {
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    oacc[c][mb] = mfma16(a, pl[c], oacc[c][mb]);
            }
            ring[k % kAhead] = k + kAhead < NF ? fragment(fb, k + kAhead) : fragment(next, k + kAhead - NF);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // ---- One block of codes or fp16 rows in registers, of a wave with NT tiles.
    // The pieces are made one at a time (left to itself the compiler makes
    // them all ahead of their products, in registers that there are not).

    // l[c][4 e + i]: the score of token 8 qg + 4 e + i, in log2 units, from key(e, kb)
    // and meta's scales.
    template <int NT, class Key>
    __device__ __forceinline__ void group_scores(Key key, const float* meta, bool affine, int lane, float (*l)[8])
    {
        const int qg = lane >> 4;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            floatx4 S[NT];
#pragma unroll
            for (int c = 0; c < NT; ++c)
                S[c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (ZM) {
                if (affine)
                    add_offset_products<NT>(S, meta, e, lane);
            }
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                floatx4 acc[NT];
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    acc[c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int kb = g * KS; kb < (g + 1) * KS; ++kb) {
                    const half8 a = key(e, kb);
#pragma unroll
                    for (int c = 0; c < NT; ++c)
                        acc[c] = mfma16(a, q[c][kb], acc[c]);
                    if constexpr (ROT) {
#pragma unroll
                        for (int c = 0; c < NT; ++c)
                            acc[c] = mfma16(a, ql[c][kb], acc[c]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                const floatx4 s4 = *(const floatx4*)(meta + 32 * g + 8 * qg + 4 * e);
#pragma unroll
                for (int c = 0; c < NT; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        S[c][i] = fmaf(s4[i], acc[c][i], S[c][i]);
                if constexpr (!ZM) {
                    if (affine)
                        add_group_offset<NT>(S, meta, g, e, lane);
                }
            }
            finish<NT>(S, 1.0f, meta + 2 * D, e, lane, l);
        }
    }

    // Eight scales and offsets (D further) at `at`, in operand order.
    static __device__ __forceinline__ void load_scales(const float* at, float* sn)
    {
        const float4 a = *(const float4*)at, b = *(const float4*)(at + 4);
        const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            sn[j] = x[perm4(j)];
    }

    // The same with per-channel scales (s at st, offsets z D further):
    // sum_d q_d (s_d c_d + z_d) = (q s) . c + q . z.
    template <int NT, class Key>
    __device__ __forceinline__ void channel_scores(Key key, const float* st, float ksm, const float* nl, int lane,
                                                   float (*l)[8])
    {
        const int qg = lane >> 4;
        floatx4 acc[NT][2];
        float z[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            acc[c][0] = acc[c][1] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
            z[c] = 0.0f;
        }
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
            half8 hi[NT], lo[NT];
            float sn[8], zn[8];
            load_scales(st + 32 * kb + 8 * qg, sn);
            load_scales(st + D + 32 * kb + 8 * qg, zn);
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float qf = (float)q[c][kb][j] + (ROT ? (float)ql[c][ROT ? kb : 0][j] : 0.0f);
                    x[j] = qf * sn[j];
                    z[c] = fmaf(qf, zn[j], z[c]);
                }
                split_nearest(x, &hi[c], &lo[c]);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const half8 a = key(e, kb);
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    acc[c][e] = mfma16(a, hi[c], acc[c][e]);
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    acc[c][e] = mfma16(a, lo[c], acc[c][e]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int c = 0; c < NT; ++c)
            z[c] = sum_rows(z[c]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            floatx4 S[NT];
#pragma unroll
            for (int c = 0; c < NT; ++c)
                S[c] = acc[c][e] + z[c];
            finish<NT>(S, ksm, nl, e, lane, l);
        }
    }

    // The same of fp16 rows, key(e, kb) after load(e); sm: what their products take.
    template <int NT, class Load, class Key>
    __device__ __forceinline__ void row_scores(Load load, Key key, float sm, const float* nl, int lane, float (*l)[8])
    {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            load(e);
            floatx4 acc[NT];
#pragma unroll
            for (int c = 0; c < NT; ++c)
                acc[c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb) {
                const half8 a = key(e, kb);
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    acc[c] = mfma16(a, q[c][kb], acc[c]);
                if constexpr (ROT) {
#pragma unroll
                    for (int c = 0; c < NT; ++c)
                        acc[c] = mfma16(a, ql[c][kb], acc[c]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            finish<NT>(acc, sm, nl, e, lane, l);
        }
    }

    // Values of codes(mb), scales s at st (offsets z D further) of `group` channels:
    // sum_t p_t (s_t c_t + z_t) = (p s) . c + p . z.
    template <int NT, class Codes>
    __device__ __forceinline__ void group_values(Codes codes, const float* st, int group, bool affine,
                                                 const float (*pv)[8], int lane)
    {
        half8 hi[NT], lo[NT];
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb) {
            if (mb % 2 == 0 && (16 * mb & (group - 1)) == 0) {
                const float* at = st + 32 * (16 * mb >> (31 - __builtin_clz(group))) + 8 * (lane >> 4);
                float sn[8];
                load_scales(at, sn);
#pragma unroll
                for (int c = 0; c < NT; ++c) {
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        x[j] = pv[c][j] * sn[j];
                    split_nearest(x, &hi[c], &lo[c]);
                }
                if (affine) {
                    load_scales(at + D, sn);
#pragma unroll
                    for (int c = 0; c < NT; ++c)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            zacc[c][mb / 2] = fmaf(pv[c][j], sn[j], zacc[c][mb / 2]);
                }
            }
            value_products<NT>(codes(mb), mb, hi, lo);
        }
    }

    template <int NT>
    __device__ __forceinline__ void value_products(const half8& a, int mb, const half8* hi, const half8* lo)
    {
#pragma unroll
        for (int c = 0; c < NT; ++c)
            oacc[c][mb] = mfma16(a, hi[c], oacc[c][mb]);
#pragma unroll
        for (int c = 0; c < NT; ++c)
            oacc[c][mb] = mfma16(a, lo[c], oacc[c][mb]);
        __builtin_amdgcn_sched_barrier(0);
    }

    // Values that are operands as they are.
    template <int NT, class Value>
    __device__ __forceinline__ void row_values(Value value, const float (*pv)[8])
    {
        half8 hi[NT], lo[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c)
            split_nearest(pv[c], &hi[c], &lo[c]);
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb)
            value_products<NT>(value(mb), mb, hi, lo);
    }

    // The value offsets join their channels.
    __device__ __forceinline__ void add_offsets(int group)
    {
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            float z = 0.0f;
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb) {
                if (mb % 2 == 0 && (16 * mb & (group - 1)) == 0)
                    z = sum_rows(zacc[c][mb / 2]);
                oacc[c][mb] += z;
            }
        }
    }

    // The partial of tile c: (m, l) with l in [1, 2), so that m is a weight's and not
    // that of a product, and what the accumulators (of 2^(kPBits + 10) `pre`; this lane's
    // channels 16 mb + 4 qg .. + 3 of row lane % 16) take.  Powers of two.
    __device__ __forceinline__ float2 partial(int c, int log2_pre, float* scale) const
    {
        const uint32_t u = __float_as_uint(sum_rows(lsum[c])), e = u >> 23;  // e = 0: no token seen
        *scale = e ? __uint_as_float((254 - e) << 23) * __uint_as_float((uint32_t)(117 - log2_pre) << 23) : 0.0f;
        return e ? make_float2(m[c] + (float)((int)e - 127), __uint_as_float((u & 0x7FFFFFu) | 0x3F800000u))
                 : make_float2(kNegInf, 0.0f);
    }
};

// ------------------------------------------------------------ work items

// The work item of a workgroup (all uniform).
struct Item {
    int seg, unit, j;    // segment, unit (sequence H + j) and KV head
    int seq0;            // first batch sequence of the rows
    int r0, rows;        // first row of the item, rows of the unit
    int split, part;     // range of blocks, and its place among a row's partials
    int lim, causal;     // limit of row 0, and whether a row of chunk token c sees c more
};

// Item x of a kernel that takes `per` rows per item.
__device__ __forceinline__ Item find_item(const SharedParams& p, int x, int per)
{
    Item it;
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

// Row R of O [B][C][H_q][D] (and of Q, and of the partials) of a unit's row r.
__device__ __forceinline__ size_t global_row(const SharedParams& p, const Item& it, int G, int r)
{
    const int t = r / G;
    return ((size_t)it.seq0 * p.C + t) * p.H_q + (size_t)it.j * G + (r - t * G);
}

// The blocks of an item that some of its `left` rows see, in the order sink
// blocks, coded blocks, window blocks.
struct Blocks {
    int v0, v1;  // v0 .. v1 - 1
    int nsb;     // sink blocks come first; block v is tail block v - nsb after them
    int ncb;     // coded blocks of the tail

    __device__ __forceinline__ Blocks(const SharedParams& sp, const AttnParams& p, const Item& it, int left)
    {
        nsb = (p.n_sink + 31) >> 5;
        ncb = (p.nq + 31) >> 5;
        const int top = it.lim + (it.causal ? (it.r0 + left - 1) / p.G : 0);  // the most that a row sees
        const int nv = min(nsb, (top + p.sink + 31) >> 5) + (top > 0 ? (top + 31) >> 5 : 0);
        v0 = min(nv, it.split * sp.bps[it.seg]);
        v1 = min(nv, v0 + sp.bps[it.seg]);
    }

    __device__ __forceinline__ bool coded(int v) const { return v >= nsb && v - nsb < ncb; }
    // the coded block nearest to block v of this item
    __device__ __forceinline__ int nearest(int v) const { return min(max(min(v, v1 - 1) - nsb, 0), ncb - 1); }
};

// Where fp16 block v's rows are.
struct RowBlock {
    const uint16_t *k, *v;
    int first, ring, live;

    __device__ __forceinline__ RowBlock(const AttnParams& p, int unit, const Blocks& b, int blk, int D)
    {
        const bool sink = blk < b.nsb;
        first = 32 * (sink ? blk : blk - b.nsb);
        ring = sink ? p.sink : p.ring;
        live = (sink ? p.n_sink : p.n) - first;
        const size_t at = (size_t)unit * ring * D;
        k = (sink ? p.kq : p.kr) + at;
        v = (sink ? p.vq : p.vr) + at;
    }
};

// Block v's first token, what is added to the rows' limits, and its live tokens.
struct Span {
    int t0, off, live;

    __device__ __forceinline__ Span(const AttnParams& p, const Blocks& b, int v)
    {
        const bool sink = v < b.nsb;
        t0 = 32 * (sink ? v : v - b.nsb);
        off = sink ? p.sink : 0;
        live = (sink ? p.n_sink : p.n) - t0;
    }
};

// One row's partial, merged over waves first, first + 1, .. of lo [waves][16][merge_pitch]
// and lml [waves][16][2] (row r of each), four channels from d.
template <int D>
__device__ __forceinline__ void merge_row(const SharedParams& sp, const float* lo, const float* lml, int first,
                                          int waves, int r, int d, size_t at)
{
    float M = kNegInf, L = 0.0f;
    for (int w = first; w < waves; ++w)
        M = fmaxf(M, lml[2 * (w * 16 + r)]);
    floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    if (M != kNegInf) {
        for (int w = first; w < waves; ++w) {
            const float2 ml = *(const float2*)(lml + 2 * (w * 16 + r));
            const float sc = __builtin_amdgcn_exp2f(ml.x - M);
            acc += *(const floatx4*)(lo + (w * 16 + r) * merge_pitch(D) + d) * sc;
            L += sc * ml.y;
        }
    }
    *(floatx4*)(sp.part_o + at * D + d) = acc;
    if (d == 0)
        *(float2*)(sp.part_ml + 2 * at) = make_float2(M, L);
}

// ROWS (of both kernels): the format has fp16 tokens (their conversion in the
// loop costs the other formats registers that the loop spills).
template <int D, int KG, int KB, int VB, bool M16, bool ROT, bool ROWS>
__global__ __launch_bounds__(64 * waves(D), waves(D) / 4) void image_kernel(SharedParams sp)
{
    constexpr bool KH = KG == 0;
    constexpr int W = waves(D), CT = tiles(D), NI = images(D), PB = parts(D), NMB = D / 16;
    constexpr int BI = image_bytes(D, KH), BM = meta_bytes(D);
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, hh = lane & 15, qg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const Item it = find_item(sp, blockIdx.x, item_rows(D));
    const AttnParams& p = sp.seg[it.seg];
    const int G = p.G, left = min(it.rows - it.r0, item_rows(D));
    const Blocks bl(sp, p, it, left);

    // ---- this wave's part of the images: block v0 + turn NI + own
    typedef Builder<D, KH, KB, VB, M16, PB> Build;
    const Build B(p, it.unit, wave % PB, lane);
    const int own = wave / PB;
    // (the nearest coded block's loads, fp16 blocks are read when they are
    // built: without branches, so that nothing waits for them early)
    const auto prefetch = [&](int v) {
        typename Build::Loads r;
        if (!ROWS || bl.ncb > 0)
            B.load(r, bl.nearest(v));
        return r;
    };
    typename Build::Loads raw = prefetch(bl.v0 + own);

    // ---- this wave's rows and its images of a turn
    const int nt16 = (left + 15) >> 4;
    const int R = row_waves(D, nt16);
    const int BW = W / R, rw = wave / BW, bw = wave - rw * BW;
    const int nt = nt16 > rw ? (nt16 - rw + R - 1) / R : 0;  // tiles rw, rw + R, ..
    Rows<D, KG, ROT, CT, false> T;
    T.lim0 = it.lim + (it.causal ? (it.r0 + 16 * rw) / G : 0);
    {
        const int last = min(left, 16 * (rw + R * (nt - 1)) + 16) - 1;
        T.lim1 = nt > 0 ? it.lim + (it.causal ? (it.r0 + last) / G : 0) : -(1 << 30);
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int rc = min(16 * (rw + R * c) + hh, left - 1);
        T.lim[c] = it.lim + (it.causal ? (it.r0 + rc) / G : 0);
        T.load_query(c, sp.q + global_row(sp, it, G, it.r0 + rc) * D, p.rot_c, lane);
    }

    T.init();
    uint8_t* metas = lds + NI * BI;
    float* st = (float*)(metas + NI * BM + stage_bytes(D) * wave);
    const auto build = [&](int v) __attribute__((always_inline)) {  // the turn that starts at block v
        const int mine = v + own;
        uint8_t* img = lds + own * BI;
        float* meta = (float*)(metas + own * BM);
        if (mine < bl.v1) {
            if (!ROWS || bl.coded(mine)) {
                B.coded_image(raw, min(32, p.nq - 32 * (mine - bl.nsb)), img, meta, st);
            } else {
                const RowBlock rb(p, it.unit, bl, mine, D);
                B.rows_image(rb.k, rb.v, rb.first, rb.ring, rb.live, img, meta, st);
            }
        }
        raw = prefetch(mine + NI);
        if constexpr (ROWS) {
            if (v < bl.nsb || min(v + NI, bl.v1) > bl.nsb + bl.ncb) {  // a turn with fp16 rows
                sync_lds();
                if (mine < bl.v1 && !bl.coded(mine))
                    B.rows_scale(metas + NI * BM + stage_bytes(D) * own * PB, img, meta);
            }
        }
    };
    // (two loops, so that the registers of a wave's tiles have one place in each)
    const auto walk = [&](auto tiles_now) __attribute__((always_inline)) {
        constexpr int NT = decltype(tiles_now)::value;
        const auto consume = [&](int v) __attribute__((always_inline)) {
            // images bw, bw + BW, .. that some of this wave's rows see
            const int n = min(NI, bl.v1 - v);
            const auto seen = [&](int i) {  // the first of them from i on
                while (i < n) {
                    const Span s(p, bl, v + i);
                    if (s.t0 < T.lim1 + s.off)
                        break;
                    i += BW;
                }
                return i;
            };
            int i = seen(bw);
            if (i >= n)
                return;
            T.apart |= __any(((const uint32_t*)(metas + min(lane, n - 1) * BM))[2 * D + 65] != 0);
            half8 ring[T.kAhead];
#pragma unroll
            for (int k = 0; k < T.kAhead; ++k)
                ring[k] = T.fragment(lds + i * BI + 16 * lane, k);
            while (i < n) {
                const int j = seen(i + BW);
                const uint8_t *fb = lds + i * BI + 16 * lane, *next = j < n ? lds + j * BI + 16 * lane : fb;
                const float* meta = (const float*)(metas + i * BM);
                const Span s(p, bl, v + i);
                const bool affine = B.kaff && (!ROWS || bl.coded(v + i));  // (fp16 rows have no offsets)
                float l[NT][8], shift[NT];
                half8 ph[NT], pl[NT];
                T.template image_scores<NT>(ring, fb, meta, affine, lane, l);
                T.template settle<NT>(l, meta + 2 * D, s.t0, s.off, s.live, lane, shift);
                T.template probabilities<NT>(l, meta + 2 * D, shift, lane, ph, pl);
                T.template image_values<NT>(ring, fb, next, ph, pl);
                i = j;
            }
        };
        for (int v = bl.v0; v < bl.v1; v += NI) {
            build(v);
            sync_lds();
            consume(v);
            sync_lds();
        }
    };
    if (CT == 1 || nt <= 1)
        walk(std::integral_constant<int, 1>{});
    else
        walk(std::integral_constant<int, CT>{});

    // ---- partials: of each wave when its rows are its own, else merged in LDS
    float* lo = (float*)lds;                     // [waves][16][pitch]
    float* lml = lo + W * 16 * merge_pitch(D);   // [waves][16][2]
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        if (R * c >= nt16)
            break;
        float scale;
        const float2 ml = T.partial(c, 0, &scale);
        const int r = 16 * (rw + R * c) + hh;
        if (BW == 1) {
            if (r < left) {
                const size_t row = (size_t)it.part * sp.rows + global_row(sp, it, G, it.r0 + r);
#pragma unroll
                for (int mb = 0; mb < NMB; ++mb)
                    *(floatx4*)(sp.part_o + row * D + 16 * mb + 4 * qg) = T.oacc[c][mb] * scale;
                if (qg == 0)
                    *(float2*)(sp.part_ml + 2 * row) = ml;
            }
            continue;
        }
        if (c > 0)
            sync_lds();
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb)
            *(floatx4*)(lo + (wave * 16 + hh) * merge_pitch(D) + 16 * mb + 4 * qg) = T.oacc[c][mb] * scale;
        if (qg == 0)
            *(float2*)(lml + 2 * (wave * 16 + hh)) = ml;
        sync_lds();
        for (int idx = threadIdx.x; idx < 16 * R * (D / 4); idx += 64 * W) {
            const int row = idx / (D / 4), d = 4 * (idx % (D / 4)), w = row >> 4, rr = 16 * (w + R * c) + (row & 15);
            if (rr < left)
                merge_row<D>(sp, lo, lml, w * BW, w * BW + BW, row & 15, d,
                             (size_t)it.part * sp.rows + global_row(sp, it, G, it.r0 + rr));
        }
    }
}

// Waves per SIMD that the registers are held to.
__host__ __device__ constexpr int direct_waves(int D)
{
    return D == 64 ? 3 : 2;
}

template <int D, int KG, int KB, int VB, bool M16, bool ROT, bool ROWS>
__global__ __launch_bounds__(kDirectThreads, direct_waves(D)) void direct_kernel(SharedParams sp)
{
    constexpr int NMB = D / 16, NKB = D / 32, W = kDirectWaves, CT = direct_tiles(D, KG, KB, ROT, ROWS), PER = 16 * CT;
    // (two blocks' loads, or both halves of a block of fp16 keys, do not fit the
    // registers of the widest heads)
    constexpr bool kAhead = D < 256;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, hh = lane & 15, qg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const Item it = find_item(sp, blockIdx.x + sp.direct0, PER);
    const AttnParams& p = sp.seg[it.seg];
    const int G = p.G, left = min(it.rows - it.r0, PER);
    const Blocks bl(sp, p, it, left);

    typedef Builder<D, KG == 0, KB, VB, M16, 1> Build;
    const Build B(p, it.unit, 0, lane);
    const auto prefetch = [&](int v) {
        typename Build::Loads r;
        if (!ROWS || bl.ncb > 0)
            B.load(r, bl.nearest(v));
        return r;
    };
    int vc = bl.v0 + wave;  // this wave's first block after the sink's
    while (ROWS && vc < bl.nsb)
        vc += W;
    typename Build::Loads raw;
    if constexpr (kAhead || !ROWS)
        raw = prefetch(vc);
    Rows<D, KG, ROT, CT, true> T;
    T.lim0 = it.lim + (it.causal ? it.r0 / G : 0);
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int rc = min(16 * c + hh, left - 1);
        T.lim[c] = it.lim + (it.causal ? (it.r0 + rc) / G : 0);
        T.load_query(c, sp.q + global_row(sp, it, G, it.r0 + rc) * D, p.rot_c, lane);
    }
    T.init();
    float* meta = (float*)(lds + wave * direct_region(D, p.ring || p.sink));
    float* st = meta + meta_bytes(D) / 4;
    // (two loops, so that the registers of a wave's tiles have one place in each)
    const auto walk = [&](auto tiles_now) __attribute__((always_inline)) {
        constexpr int NT = decltype(tiles_now)::value;
        // (loops of one kind of block, sink rows, codes, window rows: a loop of all
        // spills the registers that their branches differ in)
        int v = bl.v0 + wave;
        const auto fp16_blocks = [&](int end) __attribute__((always_inline)) {
            for (; v < end; v += W) {
                const Span s(p, bl, v);
                float l[NT][8], pv[NT][8], shift[NT], weight[8];
                lds_order();
                const RowBlock rb(p, it.unit, bl, v, D);
                Build A = B;  // (the addresses below are made here, not kept in registers over the loop)
                asm volatile("" : "+v"(A.lane));
                // Values are transposed through LDS, 128 channels at a time: a lane has 8
                // channels of tokens t and t + 4, neighbours in the operand, 16 such
                // pairs and 4 lanes of channels at a time: two lanes per bank.
                constexpr int NV = (D < 128 ? D : 128) / 32;
                constexpr int KN = kAhead ? 2 * NKB : NKB;  // key pieces at a time
                u32x4 kw[KN];
                float n2[2] = {0.0f, 0.0f};  // sums of squares of tokens t0 and t0 + 4
                uint16_t* vt = (uint16_t*)st;
                const int pair = A.lane >> 2, t0 = 2 * (pair & ~3) + (pair & 3), c8 = 8 * (A.lane & 3);
                const uint32_t keep = (t0 < rb.live ? 0xFFFFu : 0u) | (t0 + 4 < rb.live ? 0xFFFF0000u : 0u);
#pragma unroll
                for (int u = 0; u < D / 32; u += NV) {
                    u32x4 vw[NV][2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int t = min(t0 + 4 * h, rb.live - 1);
                        const uint16_t* row = rb.v + (uint32_t)((rb.first + t) % rb.ring * D + c8);
#pragma unroll
                        for (int i = 0; i < NV; ++i)
                            vw[i][h] = *(const u32x4*)(row + 32 * (u + i));
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < NV; ++i)
                            n2[h] = add_squares(vw[i][h], n2[h]);
                    if (u + NV >= D / 32) {
#pragma unroll
                        for (int i = 0; i < KN; ++i)
                            kw[i] = A.load_key_row(rb.k, rb.first, rb.ring, rb.live, i);
                    }
#pragma unroll
                    for (int i = 0; i < NV; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            *(uint32_t*)(vt + (32 * (u + i) + c8 + j) * kVtPitch + 2 * pair) =
                                keep & __builtin_amdgcn_perm(vw[i][1][j >> 1], vw[i][0][j >> 1],
                                                         j & 1 ? 0x07060302u : 0x05040100u);
                    __builtin_amdgcn_sched_barrier(0);
                }
                // the tokens' powers: starts and weights, and (where a coded block has its key
                // offsets) fp16 pairs for the transposed values
                float* nl = meta + 2 * D;
                uint32_t* pairs = (uint32_t*)(meta + D);
                {
                    uint32_t f2 = 0;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        n2[h] += dpp_f32<0xB1>(n2[h]);  // the four lanes of a token
                        n2[h] += dpp_f32<0x4E>(n2[h]);
                        const TokenPowers t = TokenPowers::of_row(n2[h]);
                        A.put_powers(t, t0 + 4 * h, nl, log2_to_one<VB>());
                        f2 |= (uint32_t)f32_to_f16_bits(t.f()) << (16 * h);
                    }
                    pairs[pair] = f2;
                }
                lds_order();
                const auto load = [&](int e) {
#pragma unroll
                    for (int i = NKB; i < NKB + KN && !kAhead && e == 1; ++i)
                        kw[i - NKB] = A.load_key_row(rb.k, rb.first, rb.ring, rb.live, i);
                };
                const auto key = [&](int e, int kb) {
                    return A.key_row_piece(kw[(e * NKB + kb) % KN], rb.live, e * NKB + kb);
                };
                T.template row_scores<NT>(load, key, p.sm_log2, nl, lane, l);
                T.template settle<NT>(l, nl, s.t0, s.off, s.live, lane, shift);
                T.load_natural(nl + 32 + 8 * qg, weight);
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    T.exponentials(c, l[c], weight, shift[c], pv[c]);
                const uint16_t* at = vt + hh * kVtPitch + 8 * qg;
                const u32x4 powers = *(const u32x4*)(pairs + 4 * qg);
                T.template row_values<NT>(
                    [&](int mb) { return times_powers(*(const u32x4*)(at + 16 * mb * kVtPitch), powers); }, pv);
            }
        };
        const int codes = ROWS ? min(bl.v1, bl.nsb + bl.ncb) : bl.v1;
        for (int part = 0; part < (ROWS ? 2 : 1); ++part) {
            if constexpr (ROWS)
                fp16_blocks(part ? bl.v1 : min(bl.v1, bl.nsb));
            if constexpr (!kAhead && ROWS) {
                if (v < codes)
                    raw = prefetch(v);
            }
            for (; v < codes; v += W) {
                const Span s(p, bl, v);
                float l[NT][8], pv[NT][8], shift[NT], weight[8], *nl = meta + 2 * D;
                lds_order();
                const typename Build::Loads now = raw;
                if constexpr (kAhead)
                    raw = prefetch(v + W);
                const int live = min(32, p.nq - s.t0);
                const float ksm = B.key_scales(now, live, meta, meta, to_one<KB>());
                T.apart |= B.template value_scales<log2_to_one<VB>()>(now, live, st, nl);
                lds_order();
                const auto key = [&](int e, int kb) { return B.key_codes(now, e * NKB + kb); };
                if constexpr (KG == 0)
                    T.template channel_scores<NT>(key, meta, ksm, nl, lane, l);
                else
                    T.template group_scores<NT>(key, meta, B.kaff, lane, l);
                T.template settle<NT>(l, nl, s.t0, s.off, s.live, lane, shift);
                T.load_natural(nl + 32 + 8 * qg, weight);
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    T.exponentials(c, l[c], weight, shift[c], pv[c]);
                T.template group_values<NT>([&](int mb) { return B.value_codes(now, mb); }, st, p.v_group, B.vaff, pv, lane);
                if constexpr (!kAhead)
                    raw = prefetch(v + W);
            }
        }
    };
    if (CT == 1 || left <= 16)
        walk(std::integral_constant<int, 1>{});
    else
        walk(std::integral_constant<int, CT>{});
    T.add_offsets(p.v_group);

    // ---- the waves' partials merged
    float* lo = (float*)lds;
    float* lml = lo + W * 16 * merge_pitch(D);
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        if (16 * c >= left)
            break;
        float scale;
        const float2 ml = T.partial(c, log2_to_one<VB>(), &scale);
        __syncthreads();
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb)
            *(floatx4*)(lo + (wave * 16 + hh) * merge_pitch(D) + 16 * mb + 4 * qg) = T.oacc[c][mb] * scale;
        if (qg == 0)
            *(float2*)(lml + 2 * (wave * 16 + hh)) = ml;
        __syncthreads();
        for (int idx = threadIdx.x; idx < min(left - 16 * c, 16) * (D / 4); idx += kDirectThreads) {
            const int r = idx / (D / 4), d = 4 * (idx % (D / 4));
            merge_row<D>(sp, lo, lml, 0, W, r, d, (size_t)it.part * sp.rows + global_row(sp, it, G, it.r0 + 16 * c + r));
        }
    }
}

// Items [0, image_items) by the image kernel, then direct_items by the direct one.
template <int D, int KG, int KB, int VB, bool M16, bool ROT>
hipError_t launch_instance(const SharedParams& p, hipStream_t stream)
{
    const bool rows = p.seg[0].ring > 0 || p.seg[0].sink > 0;
    constexpr bool kWindow = KG == 0;  // (per-channel keys come with a window)
    if (p.image_items > 0)
        launch_kernel(rows ? image_kernel<D, KG, KB, VB, M16, ROT, true> : image_kernel<D, KG, KB, VB, M16, ROT, kWindow>,
                      dim3(p.image_items), dim3(64 * waves(D)), (size_t)image_lds(D, KG == 0), stream, p);
    if (p.direct_items > 0)
        launch_kernel(rows ? direct_kernel<D, KG, KB, VB, M16, ROT, true>
                           : direct_kernel<D, KG, KB, VB, M16, ROT, kWindow>,
                      dim3(p.direct_items), dim3(kDirectThreads), (size_t)direct_lds(D, rows), stream, p);
    return hipGetLastError();
}

template <int D, int KG, bool M16, bool ROT>
hipError_t launch_widths(const SharedParams& p, hipStream_t stream)
{
    const AttnParams& a = p.seg[0];
    if (a.k_bits == 8)  // 8-bit codes come as K and V both 8-bit
        return launch_instance<D, KG, 8, 8, M16, ROT>(p, stream);
    if (a.k_bits == 4)
        return a.v_bits == 4 ? launch_instance<D, KG, 4, 4, M16, ROT>(p, stream)
                             : launch_instance<D, KG, 4, 2, M16, ROT>(p, stream);
    return a.v_bits == 4 ? launch_instance<D, KG, 2, 4, M16, ROT>(p, stream)
                         : launch_instance<D, KG, 2, 2, M16, ROT>(p, stream);
}

// The kernels of one head size and key grouping.
template <int D, int KG>
hipError_t launch_family(const SharedParams& p, hipStream_t stream)
{
    if (p.rotate)
        return p.seg[0].meta16 ? launch_widths<D, KG, true, true>(p, stream) : launch_widths<D, KG, false, true>(p, stream);
    return p.seg[0].meta16 ? launch_widths<D, KG, true, false>(p, stream) : launch_widths<D, KG, false, false>(p, stream);
}

}  // namespace shr
}  // namespace kvq
