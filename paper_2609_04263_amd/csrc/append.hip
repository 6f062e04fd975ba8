// Quantize-and-pack append into the physically packed incremental cache
// (Sec. 3.1 of the paper: new key/value states are coded with Eq. (3) or the
// symmetric control, bit-packed and appended; KIVI keeps an fp16 window).
//
// Bit-exactness: codes and metadata must equal the CPU reference bit for
// bit, so this file is compiled with -ffp-contract=off and the coder takes
// exactly the reference's IEEE binary32 steps: subtract, correctly rounded
// divide, round half to even, clamp (the rounded quotient comes from a
// reciprocal product wherever that provably gives the same code; see
// rint_quotient).  Min/max are exact.
//
// One workgroup (256 threads) codes one aligned block of 32 tokens of one
// (sequence, KV head): a thread holds eight channels of one or a few rows
// (rotated by the fixed Hadamard butterflies when the format rotates, rounded
// to fp16 when a window exists), group statistics are reduced per (token,
// group) or per channel, and every output piece (eight codes) is assembled by
// one thread, keys first, then values.  V codes are packed along tokens: a
// piece shared with tokens outside the block range keeps earlier tokens' bits
// and clears later ones, so the image is independent of call boundaries.
//
// Pieces are stored in the order the decode kernel consumes them (per
// 32-token block, a 64-lane MFMA layout; see include/kvq.h): token tau of a
// block is row 4 (tau / 8) + tau % 4 of half (tau / 4) % 2, and the lane of
// key piece P is row + 16 (P % 4); value piece (octet o, channel d) belongs
// to lane d % 16 + 16 o.

#include <type_traits>

#include "coder.h"
#include "kvq_device.h"
#include "kvq_internal.h"
#include "rope.h"

namespace kvq {
namespace {

// The file is built for two kinds of parameters P: AppendParams, and (with
// KVQ_APPEND_ROPE) AppendRopeParams, whose keys are normed and rotated (rope.h) and rounded to
// bf16 as they are loaded, so that the coder sees what kvq_rope_qk would have
// written, and whose rows may be chosen by an index.
template <typename P>
constexpr bool kRope = std::is_same<P, AppendRopeParams>::value;

// Row [sequence, token] of kin and vin that token i of the call is taken from.
template <typename P>
__device__ __forceinline__ size_t input_row(const P& p, int b, int i)
{
    if constexpr (kRope<P>) {
        const int r = p.rows ? p.rows[(size_t)b * p.n_new + i] : i;
        return (size_t)b * p.n_in + min(max(r, 0), p.n_in - 1);
    } else {
        return (size_t)b * p.n_new + i;
    }
}

// Position of token i of the call.
__device__ __forceinline__ int input_position(const AppendRopeParams& p, int b, int i)
{
    return p.rope.pos ? p.rope.pos[(size_t)b * p.n_new + i] : p.rope.pos0 + i;
}

// The angles of K rows held by D / 8 consecutive lanes, eight channels each (piece P
// of the row).  In the half layout a piece and its partner rot / 16 pieces on need
// the same eight: each computes four, and they exchange them.  s has the sign of
// the partner's part: y = c x + s x_partner.
struct Angles {
    float c[8], s[8];

    __device__ __forceinline__ Angles() {}
    __device__ __forceinline__ Angles(const RopeArgs& r, int t, int P)
    {
        if (r.layout == KVQ_ROPE_HALF) {
            const int hp = r.rot / 16;
            const bool in = P < 2 * hp, up = in && P >= hp;
            const int base = up ? 8 * (P - hp) + 4 : 8 * P, other = partner(r, P);
            float2 mine[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                mine[j] = in ? rope_cos_sin(t, r.turns[base + j], r.scale) : make_float2(1.0f, 0.0f);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float oc = __shfl(mine[j].x, other), os = __shfl(mine[j].y, other);
                c[j] = up ? oc : mine[j].x, s[j] = up ? os : -mine[j].y;
                c[j + 4] = up ? mine[j].x : oc, s[j + 4] = up ? mine[j].y : -os;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 cs = 8 * P < r.rot ? rope_cos_sin(t, r.turns[4 * P + j], r.scale) : make_float2(1.0f, 0.0f);
                c[j] = cs.x, s[j] = cs.y;
            }
        }
    }

    // The lane of a piece's partner in the half layout, its own where it has none.
    static __device__ __forceinline__ int partner(const RopeArgs& r, int P)
    {
        const int hp = r.rot / 16, lane = threadIdx.x & 63;
        return P < hp ? lane + hp : P < 2 * hp ? lane - hp : lane;
    }

    // The row normed (by weights `norm`), turned and rounded to bf16.
    template <int D>
    __device__ __forceinline__ void turn(const RopeArgs& r, const u32x4& norm, int P, float* v) const
    {
#pragma clang fp contract(off)
        if (r.wk) {
            const float f = norm_factor(row_squares<D>(r, P, squares8(v)), D, r.eps);
            float g[8];
            widen8(norm, g);
            norm8(v, f, g);
        }
        if (r.layout == KVQ_ROPE_HALF) {
            float y[8];
            exchange<D>(r, P, v, y);
            if (8 * P < r.rot) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] = v[e] * c[e] + y[e] * s[e];
            }
        } else if (8 * P < r.rot) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                turn_pair(v[2 * j], v[2 * j + 1], c[j], s[j]);
        }
        const u32x4 w = narrow8(v);
        widen8(w, v);
    }

    template <int D>
    __device__ __forceinline__ void turn(const RopeArgs& r, int P, float* v) const
    {
        turn<D>(r, r.wk ? *(const u32x4*)(r.wk + 8 * P) : u32x4{0u, 0u, 0u, 0u}, P, v);
    }

    // The partner's channels: half a row away when all of the head is rotated (a
    // vector operation each; LDS exchanges otherwise).
    template <int D>
    static __device__ __forceinline__ void exchange(const RopeArgs& r, int P, const float* v, float* y)
    {
        if (r.rot == D) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t x = __float_as_uint(v[e]);
                if constexpr (D == 64) {  // lane ^ 4: lane ^ 7, then ^ 3
                    const uint32_t m = __builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, true);
                    y[e] = __uint_as_float(__builtin_amdgcn_update_dpp(0, m, 0x1B, 0xF, 0xF, true));
                } else if constexpr (D == 128) {  // lane ^ 8
                    y[e] = __uint_as_float(__builtin_amdgcn_update_dpp(0, x, 0x128, 0xF, 0xF, true));
                } else {  // lane ^ 16
                    const auto rows = __builtin_amdgcn_permlane16_swap(x, x, false, false);
                    y[e] = __uint_as_float(P & 16 ? rows[0] : rows[1]);
                }
            }
        } else {
            const int other = partner(r, P);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                y[e] = __shfl(v[e], other);
        }
    }
};
struct NoAngles {};

constexpr int kThreads = 256;
constexpr int kBlockTok = 32;

// Index of key piece P (channels 8P..8P+7) of position tau in block `blk`
// (blk counted over the whole section: unit * NB + block).
template <int D>
__device__ __forceinline__ size_t key_piece(size_t blk, int tau, int P)
{
    const int row = 4 * (tau >> 3) + (tau & 3), half = (tau >> 2) & 1;
    return ((blk * 2 + half) * 64 + row + 16 * (P & 3)) * (D / 32) + (P >> 2);
}

// Index of value piece (octet o of the block, channel d).
template <int D>
__device__ __forceinline__ size_t value_piece(size_t blk, int o, int d)
{
    return (blk * 64 + (d & 15) + 16 * o) * (D / 16) + (d >> 4);
}

// The normalized transform of one row held by D / 8 consecutive lanes, eight
// channels each (piece `piece` of the row): half widths 1, 2, 4 inside a lane,
// 8 .. D / 2 across lanes, then one multiply by c.  Every butterfly adds or
// subtracts the same two values as the serial transform, so results are
// identical.
template <int D>
__device__ __forceinline__ void rotate8(float* r, int piece, float c)
{
#pragma unroll
    for (int hw = 1; hw < 8; hw <<= 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e & hw)
                continue;
            const float a = r[e], b = r[e + hw];
            r[e] = a + b;
            r[e + hw] = a - b;
        }
    }
#pragma unroll
    for (int hl = 1; hl < D / 8; hl <<= 1) {
        const bool upper = (piece & hl) != 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float other = __shfl_xor(r[e], hl);
            r[e] = upper ? other - r[e] : r[e] + other;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        r[e] *= c;
}

// Staging of the block's rows of K (which = 0) or V (which = 1) as the coder
// sees them.  Row i is token tb + i; rows outside [q0, q1) are zero.  Thread
// j moves eight channels of one row per step (one 16-byte load); the D / 8
// threads of a row are consecutive lanes of one wave.
template <int D>
struct RowStage {
    static constexpr int kSteps = kBlockTok * (D / 8) / kThreads;
    static_assert(kSteps >= 1 && kBlockTok * (D / 8) % kThreads == 0, "uniform staging steps");
    u32x4 w[kSteps];

    __device__ static int row(int k) { return ((int)threadIdx.x + kThreads * k) / (D / 8); }
    __device__ static int chan(int k) { return 8 * (((int)threadIdx.x + kThreads * k) % (D / 8)); }

    // The angles of step k's row, a token of this call.
    __device__ static __forceinline__ Angles angles(const AppendRopeParams& p, int b, int tb, int k)
    {
        return Angles(p.rope, input_position(p, b, tb + row(k) - p.n0), chan(k) >> 3);
    }

    // Issue the loads (bf16 input for tokens of this call, fp16 window slots
    // for tokens appended earlier).
    template <typename P>
    __device__ __forceinline__ void load(const P& p, int which, int b, int h, int tb)
    {
        const uint16_t* in = which ? p.vin : p.kin;
        const uint16_t* ring = which ? p.vr : p.kr;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int t = tb + row(k), d8 = chan(k);
            w[k] = u32x4{0u, 0u, 0u, 0u};
            if (t >= p.q0 && t < p.q1)
                w[k] = t >= p.n0 ? *(const u32x4*)(in + (input_row(p, b, t - p.n0) * p.H + h) * D + d8)
                                 : *(const u32x4*)(ring + (((size_t)b * p.H + h) * p.ring + t % p.ring) * D + d8);
        }
    }

    // The eight values of step k as the coder sees them: widened to fp32; for
    // tokens of this call (keys: turned by the angles `turn`) rotated, and rounded
    // to fp16 when a window exists.
    template <typename P, typename A>
    __device__ __forceinline__ void widen(const P& p, int tb, int k, float* v, const A& turn) const
    {
        const int t = tb + row(k);
        const bool fresh = !(t >= p.q0 && t < p.q1) || t >= p.n0;  // bf16 (zero rows: zero words)
        const uint32_t ww[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (fresh) {
                v[2 * q] = __uint_as_float(ww[q] << 16);
                v[2 * q + 1] = __uint_as_float(ww[q] & 0xFFFF0000u);
            } else {
                v[2 * q] = f16_bits_to_f32((uint16_t)ww[q]);
                v[2 * q + 1] = f16_bits_to_f32((uint16_t)(ww[q] >> 16));
            }
        }
        const bool input = t >= p.q0 && t < p.q1 && t >= p.n0;
        if constexpr (std::is_same<A, Angles>::value) {
            if (input)  // (all lanes of a row or none)
                turn.template turn<D>(p.rope, chan(k) >> 3, v);
        }
        if (p.rotate) {
            float r[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                r[e] = v[e];
            rotate8<D>(r, chan(k) >> 3, p.rot_c);
            if (input) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] = r[e];
            }
        }
        if (p.ring && input) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = f16_bits_to_f32(f32_to_f16_bits(v[e]));
        }
    }
};

// 16-byte copy of `bytes` (a multiple of 16) from LDS to global memory.
__device__ __forceinline__ void copy_out(const uint8_t* src, uint8_t* dst, int bytes)
{
    for (int off = 16 * (int)threadIdx.x; off < bytes; off += 16 * kThreads)
        *(u32x4*)(dst + off) = *(const u32x4*)(src + off);
}

#ifndef KVQ_APPEND_ROPE
// A block shared with earlier or later calls (per-token groups: a block of
// per-channel keys is one whole group), written piece by piece: value pieces
// keep the bits of tokens appended earlier.  vcode: 32 D bytes of LDS for the
// value codes [token][D].
template <int D>
__device__ __forceinline__ void edge_block(const AppendParams& p, int unit, int tb, uint8_t* vcode)
{
    const int b = unit / p.H, h = unit % p.H;
    const int lo = max(p.q0, tb), hi = min(p.q1, tb + kBlockTok);

    // ------------------------------------------------------------ keys
    const size_t blk = (size_t)unit * (size_t)(p.T / kBlockTok) + (size_t)(tb / kBlockTok);
    RowStage<D> kst, vst;
    kst.load(p, 0, b, h, tb);
    vst.load(p, 1, b, h, tb);  // in flight while the keys are coded
    const int kb = p.k_bits;
    {
        const int lanes = p.k_group / 8, ng = D / p.k_group;
        const size_t mbase = blk * (size_t)(ng * kBlockTok);
#pragma unroll
        for (int k = 0; k < RowStage<D>::kSteps; ++k) {
            const int i = RowStage<D>::row(k), P = RowStage<D>::chan(k) / 8, t = tb + i;
            float x[8];
            kst.widen(p, tb, k, x, NoAngles());
            float s, z;
            piece_group_stats(x, lanes, p.k_mode, kb, &s, &z);
            round_meta(p.meta16, &s, &z);
            if (t < lo || t >= hi)
                continue;
            if (P % lanes == 0) {
                const size_t mi = mbase + (size_t)(P / lanes) * kBlockTok + i;
                store_meta(p.ks, mi, s, p.meta16);
                if (p.k_mode == KVQ_AFFINE)
                    store_meta(p.kz, mi, z, p.meta16);
            }
            const float r = code_reciprocal(s);
            uint64_t word = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                word |= (uint64_t)code_one(x[e], s, r, z, p.k_mode, kb) << (kb * e);
            store_piece(p.kc, key_piece<D>(blk, i, P), kb, word);
        }
    }

    // ---------------------------------------------------------- values
    const int vb = p.v_bits;
    const int vlanes = p.v_group / 8;
    const size_t mbase = blk * (size_t)((D / p.v_group) * kBlockTok);
#pragma unroll
    for (int k = 0; k < RowStage<D>::kSteps; ++k) {
        const int i = RowStage<D>::row(k), P = RowStage<D>::chan(k) / 8, t = tb + i;
        float x[8];
        vst.widen(p, tb, k, x, NoAngles());
        float s, z;
        piece_group_stats(x, vlanes, p.v_mode, vb, &s, &z);
        round_meta(p.meta16, &s, &z);
        if (t >= lo && t < hi && P % vlanes == 0) {
            const size_t mi = mbase + (size_t)(P / vlanes) * kBlockTok + i;
            store_meta(p.vs, mi, s, p.meta16);
            if (p.v_mode == KVQ_AFFINE)
                store_meta(p.vz, mi, z, p.meta16);
        }
        const float r = code_reciprocal(s);
        uint32_t c[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            c[e] = code_one(x[e], s, r, z, p.v_mode, vb);
        *(uint2*)(vcode + i * D + 8 * P) =
            make_uint2(c[0] | (c[1] << 8) | (c[2] << 16) | (c[3] << 24), c[4] | (c[5] << 8) | (c[6] << 16) | (c[7] << 24));
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < (kBlockTok / 8) * D; idx += kThreads) {
        int o = idx / D, d = idx % D;
        int tfirst = tb + 8 * o;
        if (tfirst + 8 <= lo || tfirst >= hi)
            continue;
        uint64_t word = 0;
        if (tfirst < lo) {  // keep the bits of tokens appended earlier
            int keep_n = lo - tfirst;
            word = load_piece(p.vc, value_piece<D>(blk, o, d), vb) & low_codes(vb, keep_n);
        }
        for (int e = 0; e < 8; ++e) {
            int t = tfirst + e;
            if (t < lo || t >= hi)
                continue;
            word |= (uint64_t)vcode[(t - tb) * D + d] << (vb * e);
        }
        store_piece(p.vc, value_piece<D>(blk, o, d), vb, word);
    }
}

// ---- blocks

// Whether finite numbers can leave a group of BITS-bit codes a scale s without a
// hardware reciprocal: with more bits a range is divided by 7 at least.
template <int BITS>
__device__ __forceinline__ bool no_reciprocal(float s)
{
    return BITS == 2 && s > kMostReciprocal;
}

// The eight codes of a piece.  The quotient is the product with the hardware
// reciprocal wherever that provably rounds to the same code (rint_quotient);
// the eight distances to the rounded values are folded into one test, and a
// piece with a near tie takes the exact divisions.  Codes are packed by fp32
// sums (below 2^24, exact), one conversion per 16 bits: conversions, shifts
// and the per-element branch took half of the instructions before.  `divide`: a
// scale has no reciprocal (no_reciprocal), so all take the divisions.
template <int BITS>
__device__ __forceinline__ uint64_t piece_codes(const float* x, const float* s, const float* r, const float* z, int mode,
                                                bool divide)
{
#pragma clang fp contract(off)
    const float top = (float)((1 << BITS) - 1), qmax = (float)((1 << (BITS - 1)) - 1), half = (float)(1 << (BITS - 1));
    const bool aff = mode == KVQ_AFFINE;
    // The product q is within 2^-22 |d / s| of fl(d / s): 2^-23 of the reciprocal
    // and two roundings.  Below 2^BITS that is 2^(BITS - 22), beyond it both clamp;
    // so the codes can differ only where q is as near to a half-integer.  (Four
    // times that.  2048 tokens of 8 x 8 heads of 256, 4 bits: 61 us, 64 with 2^-10 at
    // any width.)
    constexpr float kNear = BITS == 8 ? 0x1p-12f : BITS == 4 ? 0x1p-16f : 0x1p-18f;
    float c[8], worst = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = aff ? x[e] - z[e] : x[e], q = d * r[e];
        c[e] = __builtin_rintf(q);
        worst = fmaxf(worst, fabsf(q - c[e]));
    }
    if (worst >= 0.5f - kNear || divide) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            c[e] = __builtin_rintf((aff ? x[e] - z[e] : x[e]) / s[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        c[e] = aff ? __builtin_amdgcn_fmed3f(c[e], 0.0f, top) : __builtin_amdgcn_fmed3f(c[e], -qmax, qmax) + half;
    constexpr int N = 16 / BITS;  // codes per 16 bits
    uint64_t word = 0;
#pragma unroll
    for (int k = 0; k < 8 / N; ++k) {
        float v = 0.0f;
#pragma unroll
        for (int e = N - 1; e >= 0; --e)
            v = __builtin_fmaf(v, (float)(1 << BITS), c[N * k + e]);
        if constexpr (BITS == 8)
            word |= (uint64_t)(uint32_t)v << (16 * k);
        else
            word = (uint32_t)word | ((uint32_t)v << (16 * k));
    }
    return word;
}

#endif

// The value of lane l ^ 8 (a rotation by half a 16-lane row).
__device__ __forceinline__ float row_ror8(float v)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x128, 0xF, 0xF, false));
}

#ifndef KVQ_APPEND_ROPE
// One workgroup per 32-token block of one (sequence, KV head); a block this
// call does not write whole takes edge_block (in a launch of its own it cost
// 5 to 10 us a call).  Per-token groups: each thread takes the eight channels of one piece, the
// group's statistics are reduced across the group's lanes.  Per-channel keys:
// a thread's eight channels of its rows are reduced over the rows in
// registers, by shuffles and over the four waves.  Key pieces go to LDS as
// they are; value words (eight channels of one token) are transposed there,
// one thread per (octet, eight channels).  Each section holds a block's bytes
// as one range, written with contiguous 16-byte stores.
// Vector work bounds it.  A KIVI chunk of 2048 tokens (B = 32, 8 heads of 128,
// 348 MB) took 164 us with rows staged in LDS, one thread per channel for the
// statistics, codes as bytes and 64-bit shifts; 115 now, window rows included.
template <int D, bool PERCH, int KB, int VB>
__global__ __launch_bounds__(kThreads) void append_block_kernel(AppendParams p)
{
    constexpr int PPT = D / 8, kOut = 4 * D * (KB > VB ? KB : VB);
    // a section's pieces, and the value codes by token (edge_block: all of it)
    constexpr int kPool = kOut + 4 * D * VB > 32 * D ? kOut + 4 * D * VB : 32 * D;
    __shared__ __attribute__((aligned(16))) uint8_t pool[kPool];
    uint8_t* ob = pool;
    uint32_t* vw = (uint32_t*)(pool + kOut);
    __shared__ __attribute__((aligned(16))) float mb[2][kBlockTok * 8];  // its scales, offsets (<= 1 KB each)
    __shared__ __attribute__((aligned(16))) float red[PERCH ? 2 : 1][PERCH ? 4 : 1][PERCH ? D : 4];
    __shared__ __attribute__((aligned(16))) float cs[PERCH ? 3 : 1][PERCH ? D : 4];  // channel scales, reciprocals, offsets
    constexpr int kSteps = RowStage<D>::kSteps;

    const int unit = blockIdx.y;
    const int b = unit / p.H, h = unit % p.H;
    const int tb = (p.q0 / kBlockTok + (int)blockIdx.x) * kBlockTok;
    if constexpr (!PERCH) {
        if (tb < p.q0 || tb + kBlockTok > p.q1) {
            edge_block<D>(p, unit, tb, pool);
            return;
        }
    }
    const int msz = p.meta16 ? 2 : 4;
    const size_t blk = (size_t)unit * (size_t)(p.T / kBlockTok) + (size_t)(tb / kBlockTok);
    RowStage<D> kst, vst;
    kst.load(p, 0, b, h, tb);
    vst.load(p, 1, b, h, tb);  // in flight while the keys are coded

    // ------------------------------------------------------------ keys
    int kmeta;  // metadata elements per block
    if constexpr (!PERCH) {
        const int lanes = p.k_group / 8;
        kmeta = D / p.k_group * kBlockTok;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int i = RowStage<D>::row(k), P = RowStage<D>::chan(k) / 8;
            float x[8], s, z;
            kst.widen(p, tb, k, x, NoAngles());
            piece_group_stats(x, lanes, p.k_mode, KB, &s, &z);
            round_meta(p.meta16, &s, &z);
            if (P % lanes == 0) {
                store_meta(mb[0], (P / lanes) * kBlockTok + i, s, p.meta16);
                if (p.k_mode == KVQ_AFFINE)
                    store_meta(mb[1], (P / lanes) * kBlockTok + i, z, p.meta16);
            }
            const float r = __builtin_amdgcn_rcpf(s);
            const float s8[8] = {s, s, s, s, s, s, s, s}, r8[8] = {r, r, r, r, r, r, r, r}, z8[8] = {z, z, z, z, z, z, z, z};
            store_piece(ob, key_piece<D>(0, i, P), KB, piece_codes<KB>(x, s8, r8, z8, p.k_mode, no_reciprocal<KB>(s)));
        }
    } else {
        kmeta = D;
        float x[kSteps][8], mn[8], mx[8];
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
            kst.widen(p, tb, k, x[k], NoAngles());
        const bool aff = p.k_mode == KVQ_AFFINE;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            mn[e] = x[0][e];
            mx[e] = aff ? x[0][e] : fabsf(x[0][e]);
#pragma unroll
            for (int k = 1; k < kSteps; ++k) {
                mn[e] = fminf(mn[e], x[k][e]);
                mx[e] = fmaxf(mx[e], aff ? x[k][e] : fabsf(x[k][e]));
            }
            // (shuffles are LDS operations, which the vector-bound large chunks
            // do not notice: row swaps instead took 125 against 115 us)
            if constexpr (PPT <= 8) {
                mn[e] = fminf(mn[e], row_ror8(mn[e]));
                mx[e] = fmaxf(mx[e], row_ror8(mx[e]));
            }
#pragma unroll
            for (int off = PPT < 16 ? 16 : PPT; off < 64; off <<= 1) {
                mn[e] = fminf(mn[e], __shfl_xor(mn[e], off));
                mx[e] = fmaxf(mx[e], __shfl_xor(mx[e], off));
            }
        }
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c8 = RowStage<D>::chan(0);
        if (lane < PPT) {
            *(float4*)&red[0][wave][c8] = make_float4(mn[0], mn[1], mn[2], mn[3]);
            *(float4*)&red[0][wave][c8 + 4] = make_float4(mn[4], mn[5], mn[6], mn[7]);
            *(float4*)&red[1][wave][c8] = make_float4(mx[0], mx[1], mx[2], mx[3]);
            *(float4*)&red[1][wave][c8 + 4] = make_float4(mx[4], mx[5], mx[6], mx[7]);
        }
        __syncthreads();
        for (int d = threadIdx.x; d < D; d += kThreads) {
            const float lo[1] = {fminf(fminf(red[0][0][d], red[0][1][d]), fminf(red[0][2][d], red[0][3][d]))};
            const float hi = fmaxf(fmaxf(red[1][0][d], red[1][1][d]), fmaxf(red[1][2][d], red[1][3][d]));
            // group_stats of the group's extremes: the same minimum, maximum
            // and magnitude, so the same scale and offset
            const float ends[2] = {aff ? lo[0] : hi, hi};
            float s, z;
            group_stats(ends, 1, 2, p.k_mode, KB, &s, &z);
            round_meta(p.meta16, &s, &z);
            cs[0][d] = s;
            cs[1][d] = __builtin_amdgcn_rcpf(s);
            cs[2][d] = z;
            store_meta(mb[0], d, s, p.meta16);
            if (aff)
                store_meta(mb[1], d, z, p.meta16);
        }
        __syncthreads();
        float s8[8], r8[8], z8[8];
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
            *(float4*)(s8 + e) = *(const float4*)&cs[0][c8 + e];
            *(float4*)(r8 + e) = *(const float4*)&cs[1][c8 + e];
            *(float4*)(z8 + e) = *(const float4*)&cs[2][c8 + e];
        }
        // (a window's numbers, and so the scales, are below 2^17)
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
            store_piece(ob, key_piece<D>(0, RowStage<D>::row(k), c8 / 8), KB, piece_codes<KB>(x[k], s8, r8, z8, p.k_mode, false));
    }
    __syncthreads();
    copy_out(ob, (uint8_t*)p.kc + blk * (size_t)(4 * D * KB), 4 * D * KB);
    copy_out((const uint8_t*)mb[0], (uint8_t*)p.ks + blk * (size_t)(kmeta * msz), kmeta * msz);
    if (p.k_mode == KVQ_AFFINE)
        copy_out((const uint8_t*)mb[1], (uint8_t*)p.kz + blk * (size_t)(kmeta * msz), kmeta * msz);
    __syncthreads();  // the key copies have read ob and mb

    // ---------------------------------------------------------- values
    const int vlanes = p.v_group / 8, vmeta = (D / p.v_group) * kBlockTok;
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        const int i = RowStage<D>::row(k), P = RowStage<D>::chan(k) / 8;
        float x[8], s, z;
        vst.widen(p, tb, k, x, NoAngles());
        piece_group_stats(x, vlanes, p.v_mode, VB, &s, &z);
        round_meta(p.meta16, &s, &z);
        if (P % vlanes == 0) {
            store_meta(mb[0], (P / vlanes) * kBlockTok + i, s, p.meta16);
            if (p.v_mode == KVQ_AFFINE)
                store_meta(mb[1], (P / vlanes) * kBlockTok + i, z, p.meta16);
        }
        const float r = __builtin_amdgcn_rcpf(s);
        const float s8[8] = {s, s, s, s, s, s, s, s}, r8[8] = {r, r, r, r, r, r, r, r}, z8[8] = {z, z, z, z, z, z, z, z};
        store_piece(vw, i * PPT + P, VB, piece_codes<VB>(x, s8, r8, z8, p.v_mode, no_reciprocal<VB>(s)));
    }
    __syncthreads();
    // (octet o, channels 8 P .. 8 P + 7): the eight tokens' words transposed
    for (int idx = threadIdx.x; idx < 4 * PPT; idx += kThreads) {
        const int o = idx / PPT, P = idx % PPT;
        uint64_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            w[j] = load_piece(vw, (8 * o + j) * PPT + P, VB);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (VB == 8) {
                uint64_t v = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    v |= (w[j] >> (8 * e) & 0xFFu) << (8 * j);
                store_piece(ob, value_piece<D>(0, o, 8 * P + e), VB, v);
            } else {
                uint32_t v = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    v |= ((uint32_t)w[j] >> (VB * e) & ((1u << VB) - 1u)) << (VB * j);
                store_piece(ob, value_piece<D>(0, o, 8 * P + e), VB, v);
            }
        }
    }
    __syncthreads();
    copy_out(ob, (uint8_t*)p.vc + blk * (size_t)(4 * D * VB), 4 * D * VB);
    copy_out((const uint8_t*)mb[0], (uint8_t*)p.vs + blk * (size_t)(vmeta * msz), vmeta * msz);
    if (p.v_mode == KVQ_AFFINE)
        copy_out((const uint8_t*)mb[1], (uint8_t*)p.vz + blk * (size_t)(vmeta * msz), vmeta * msz);
}

#endif

#ifndef KVQ_APPEND_ROPE
// One decoded token per (sequence, KV head) without a window: a workgroup of
// D threads, thread d owning channel d of the token's K and V.  Every load
// (the token's K and V, and the value piece it shares with earlier tokens)
// is issued first; the rotation runs as the same butterflies as rotate8;
// group statistics are all-reduced across the group's threads (min, max and
// max-magnitude are exact in any order, so they equal the block kernel's),
// then each thread codes its channel, key pieces are OR-reduced over eight
// lanes and each value piece is merged with the bits of earlier tokens.
template <int D>
__device__ __forceinline__ float group_reduce(float v, int g, bool is_max, float* red, int slot)
{
    const int lanes = g < 64 ? g : 64;
    for (int off = 1; off < lanes; off <<= 1) {
        const float o = __shfl_xor(v, off);
        v = is_max ? fmaxf(v, o) : fminf(v, o);
    }
    if (g > 64) {
        // one value per wave, combined over the g / 64 waves of the group
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
            red[slot * 4 + wave] = v;
        __syncthreads();
        const int w0 = (wave / (g / 64)) * (g / 64);
        v = red[slot * 4 + w0];
        for (int w = 1; w < g / 64; ++w)
            v = is_max ? fmaxf(v, red[slot * 4 + w0 + w]) : fminf(v, red[slot * 4 + w0 + w]);
    }
    return v;
}

template <int D>
__global__ __launch_bounds__(D) void append_token_kernel(AppendParams p)
{
    __shared__ float xs[2][D];
    __shared__ float red[8 * 4];
    const int unit = blockIdx.x, b = unit / p.H, h = unit % p.H, d = threadIdx.x;
    const int t = p.n0, tau = t & 31, j = t & 7;
    const size_t blk = (size_t)unit * (p.T / kBlockTok) + (size_t)(t / kBlockTok);
    const size_t vpi = value_piece<D>(blk, tau >> 3, d);
    const size_t in = ((size_t)b * p.H + h) * D + d;  // n_new == 1
    float x[2] = {bf16_to_f32(p.kin[in]), bf16_to_f32(p.vin[in])};
    const uint64_t old = load_piece(p.vc, vpi, p.v_bits);
    if (p.rotate) {
        xs[0][d] = x[0];
        xs[1][d] = x[1];
        __syncthreads();
        for (int hw = 1; hw < D; hw <<= 1) {
            float nv[2];
#pragma unroll
            for (int w = 0; w < 2; ++w)
                nv[w] = (d & hw) ? xs[w][d - hw] - xs[w][d] : xs[w][d] + xs[w][d + hw];
            __syncthreads();
            xs[0][d] = nv[0];
            xs[1][d] = nv[1];
            __syncthreads();
        }
        x[0] = xs[0][d] * p.rot_c;
        x[1] = xs[1][d] * p.rot_c;
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int mode = w ? p.v_mode : p.k_mode, bits = w ? p.v_bits : p.k_bits;
        const int g = w ? p.v_group : p.k_group, gi = d / g, ng = D / g;
        float s, z;
        if (mode == KVQ_AFFINE) {
            const float mn = group_reduce<D>(x[w], g, false, red, 2 * w);
            const float mx = group_reduce<D>(x[w], g, true, red, 2 * w + 1);
            const float top = (float)((1 << bits) - 1);
            s = (mx - mn) / top;
            if (!(s >= 1e-8f))
                s = 1e-8f;
            z = mn + 0.0f;  // canonical +0 for a signed-zero minimum
        } else {
            const float ma = group_reduce<D>(fabsf(x[w]), g, true, red, 2 * w);
            const float qmax = (float)((1 << (bits - 1)) - 1);
            s = ma / qmax;
            if (!(s >= 1e-8f))
                s = 1e-8f;
            z = 0.0f;
        }
        round_meta(p.meta16, &s, &z);
        const uint32_t c = code_one(x[w], s, code_reciprocal(s), z, mode, bits);
        if (d % g == 0) {
            const size_t mi = (blk * ng + gi) * kBlockTok + tau;
            store_meta(w ? p.vs : p.ks, mi, s, p.meta16);
            if (mode == KVQ_AFFINE)
                store_meta(w ? p.vz : p.kz, mi, z, p.meta16);
        }
        if (w == 0) {
            // key piece d / 8: codes of channels 8P .. 8P + 7 at bits k_bits e,
            // OR-reduced as two 32-bit halves
            const uint64_t mine = (uint64_t)c << (bits * (d & 7));
            uint32_t lo32 = (uint32_t)mine, hi32 = (uint32_t)(mine >> 32);
#pragma unroll
            for (int off = 1; off < 8; off <<= 1) {
                lo32 |= __shfl_xor(lo32, off);
                hi32 |= __shfl_xor(hi32, off);
            }
            if ((d & 7) == 0)
                store_piece(p.kc, key_piece<D>(blk, tau, d >> 3), bits, ((uint64_t)hi32 << 32) | lo32);
        } else {
            const uint64_t keep = low_codes(bits, j);
            store_piece(p.vc, vpi, bits, (old & keep) | ((uint64_t)c << (bits * j)));
        }
    }
}

#endif

// fp16 window: slot t mod (R + F) <- fp16 of token t (rotated first when
// the format rotates), for t in [ring_lo, n0 + n_new).  Runs after the coder
// of the same call, which may still read the slots being replaced.  The
// sink rows are written by the same kernel with ring = sink (slot t).
// A thread moves eight channels of one row of K and of V with 16-byte loads and
// stores, a workgroup kRingRows<D> rows (one row per workgroup with 2-byte
// loads: 128 rows of 256 units 33 us, now 8).
template <int D>
constexpr int kRingRows = kThreads / (D / 8);

template <int D, typename Params>
__device__ __forceinline__ void write_rows(const Params& p, int hi, int unit, int first)
{
    const int b = unit / p.H, h = unit % p.H;
    const int c8 = 8 * ((int)threadIdx.x % (D / 8));
    const int t = first + (int)threadIdx.x / (D / 8);
    u32x4 w[2] = {u32x4{0u, 0u, 0u, 0u}, u32x4{0u, 0u, 0u, 0u}};
    if (t < hi) {
        const size_t at = (input_row(p, b, t - p.n0) * p.H + h) * D + c8;
        w[0] = *(const u32x4*)(p.kin + at);
        w[1] = *(const u32x4*)(p.vin + at);
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const uint32_t ww[4] = {w[q].x, w[q].y, w[q].z, w[q].w};
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = __uint_as_float((e & 1) ? ww[e >> 1] & 0xFFFF0000u : ww[e >> 1] << 16);
        if constexpr (kRope<Params>) {
            if (q == 0 && t < hi)
                Angles(p.rope, input_position(p, b, t - p.n0), c8 >> 3).template turn<D>(p.rope, c8 >> 3, v);
        }
        if (p.rotate)  // (every lane of a row takes part)
            rotate8<D>(v, c8 >> 3, p.rot_c);
        if (t < hi) {
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                o[e] = f32_to_f16_bits(v[2 * e]) | ((uint32_t)f32_to_f16_bits(v[2 * e + 1]) << 16);
            *(u32x4*)((q ? p.vr : p.kr) + ((size_t)unit * p.ring + t % p.ring) * D + c8) = u32x4{o[0], o[1], o[2], o[3]};
        }
    }
}

template <int D, typename Params>
__global__ __launch_bounds__(kThreads) void append_ring_kernel(Params p, int hi)
{
    write_rows<D>(p, hi, blockIdx.y, p.ring_lo + kRingRows<D> * (int)blockIdx.x);
}

template <int D, typename P>
void launch_ring(const P& p, int hi, hipStream_t stream)
{
    launch_kernel((append_ring_kernel<D, P>), dim3((hi - p.ring_lo + kRingRows<D> - 1) / kRingRows<D>, p.B * p.H), dim3(kThreads),
                  0, stream, p, hi);
}

#ifdef KVQ_APPEND_ROPE
// Per-token groups of `size` channels (a power of two; by shifts, a division of
// integers is 20 to 30 vector operations): lanes of one, how many of a row.
template <int D>
struct Groups {
    int shift, lanes, count;
    __device__ __forceinline__ explicit Groups(int size)
        : shift(__builtin_ctz(size) - 3), lanes(1 << shift), count((D / 8) >> shift) {}
    __device__ __forceinline__ bool first(int piece) const { return (piece & (lanes - 1)) == 0; }
    __device__ __forceinline__ int of(int piece) const { return piece >> shift; }
};

// What a group's codes are made with: its scale, that one's reciprocal and its offset, of
// numbers times 2^-8, so that no finite number's difference from the offset overflows and no
// reciprocal is subnormal below an infinite scale (2^127 here: every code is 0, or the
// middle).  Between numbers of magnitude up to `most` of which one is the offset the scale is
// no less than most 2^-32, so raising it to most 2^-120 changes nothing; where fp16 holds the
// offset of a larger constant, it keeps the quotients finite and beyond every code's.
struct Divisor {
    float s, y, z;
    __device__ __forceinline__ Divisor(float scale, float offset, float most)
        : s(__builtin_amdgcn_fmed3f(scale * 0x1p-8f, most * 0x1p-128f, 0x1p127f)), y(1.0f / s), z(offset * 0x1p-8f) {}
};

// fl(x - offset) 2^-8.
__device__ __forceinline__ float from_offset(float x, float z)
{
    return __builtin_fmaf(x, 0x1p-8f, -z);
}

// The coder of code_heads: the codes, scales and offsets of piece_group_stats,
// round_meta and piece_codes in fewer operations.  A symmetric group is one with
// offset zero and other limits (`bias` makes its codes unsigned); the sums of a
// group meet by DPP, and a group's range is divided by 2^b - 1 as
//     q = fl(d fl(1 / n)),  s = fl(q + fl(d - q n) fl(1 / n)),
// the correctly rounded quotient (checked for every mantissa and n = 1, 3, 7, 15,
// 127, 255; where it would be subnormal the scale is 1e-8), infinite where d is.
template <int BITS, bool PLAIN>
struct Coder {
    float n, inv, lo, hi, bias;  // bias: of 16 / BITS codes in their places
    bool affine;

    __device__ __forceinline__ explicit Coder(int mode) : affine(PLAIN || mode == KVQ_AFFINE)
    {
        constexpr float top = (float)((1 << BITS) - 1), qmax = (float)((1 << (BITS - 1)) - 1);
        constexpr float half = (float)(1 << (BITS - 1));
        n = affine ? top : qmax;
        inv = affine ? 1.0f / top : 1.0f / qmax;
        lo = affine ? 0.0f : -qmax;
        hi = n;
        bias = affine ? 0.0f : half * (65535.0f / top);
    }

    template <int CTRL>
    static __device__ __forceinline__ float dpp(float x)
    {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xF, 0xF, true));
    }

    // Over `lanes` (4, 8, 16 or 32) lanes.
    template <typename F>
    static __device__ __forceinline__ float reduce(float x, int lanes, F f)
    {
        x = f(x, dpp<0xB1>(x));
        x = f(x, dpp<0x4E>(x));
        if (lanes > 4)
            x = f(x, dpp<0x141>(x));
        if (lanes > 8)
            x = f(x, dpp<0x140>(x));
        if (lanes > 16)
            x = f(x, __shfl_xor(x, 16));
        return x;
    }

    __device__ __forceinline__ Divisor scale(const float* x, int lanes, int meta16, float* s, float* z) const
    {
#pragma clang fp contract(off)
        const auto least = [](float a, float b) { return fminf(a, b); };
        const auto most = [](float a, float b) { return fmaxf(a, b); };
        float d, large = 0.0f;
        if (affine) {
            float mn = x[0], mx = x[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) {
                mn = fminf(mn, x[e]);
                mx = fmaxf(mx, x[e]);
            }
            mn = reduce(mn, lanes, least);
            mx = reduce(mx, lanes, most);
            d = mx - mn;
            large = fmaxf(fabsf(mn), fabsf(mx));
            *z = mn + 0.0f;  // canonical +0 for a signed-zero minimum
        } else {
            float ma = fabsf(x[0]);
#pragma unroll
            for (int e = 1; e < 8; ++e)
                ma = fmaxf(ma, fabsf(x[e]));
            d = reduce(ma, lanes, most);
            *z = 0.0f;
        }
        *s = over_n(d);
        round_meta(meta16, s, z);
        return Divisor(*s, *z, large);
    }

    __device__ __forceinline__ float over_n(float d) const
    {
        const float q = fminf(d * inv, 0x1.fffffep127f);
        return fmaxf(__builtin_fmaf(__builtin_fmaf(-q, n, d), inv, q), 1e-8f);
    }

    __device__ __forceinline__ uint64_t piece(const float* x, const Divisor& by) const
    {
        return piece(x, [&](int) { return by.s; }, [&](int) { return by.y; }, [&](int) { return by.z; });
    }

    // Element e's Divisor.
    // fl(d / s) by two corrections of fl(d y): the first leaves less than an ulp, from
    // which the second gives the correctly rounded quotient (Markstein's theorem; no
    // exception in 2 10^9 pairs).  Numbers on a grid, as bf16 rows are, meet ties of their
    // codes in 8 of 10 waves' pieces, so a branch to exact divisions costs more.
    template <typename S, typename Y, typename Z>
    __device__ __forceinline__ uint64_t piece(const float* x, S s, Y y, Z z) const
    {
#pragma clang fp contract(off)
        float c[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = from_offset(x[e], z(e));
            float q = d * y(e);
            q = __builtin_fmaf(__builtin_fmaf(-q, s(e), d), y(e), q);
            q = __builtin_fmaf(__builtin_fmaf(-q, s(e), d), y(e), q);
            c[e] = __builtin_rintf(q);
        }
        constexpr int N = 16 / BITS;  // codes per 16 bits
        uint64_t word = 0;
#pragma unroll
        for (int k = 0; k < 8 / N; ++k) {
            float v = 0.0f;
#pragma unroll
            for (int e = N - 1; e >= 0; --e)
                v = __builtin_fmaf(v, (float)(1 << BITS), __builtin_amdgcn_fmed3f(c[N * k + e], lo, hi));
            const uint32_t w = (uint32_t)(v + bias);
            if constexpr (BITS == 8)
                word |= (uint64_t)w << (16 * k);
            else
                word = (uint32_t)word | (w << (16 * k));
        }
        return word;
    }
};

// Tokens t0 .. t0 + 2048 / D - 1 of one sequence's heads h0 .., all of them coded by
// this call, per-token groups: a thread owns eight channels of one token, so that
// its keys turn by the same eight angles in every head, which cost as much as a
// third of a head's coding.  (With a 32-token block of one head per workgroup, as
// code_block, a thread has the angles of up to four rows: 64 registers where heads
// are to share them.)
// The codes of a head meet in one of two LDS buffers, so one barrier a head is
// enough: key pieces in their final order (eight runs of 32 pieces), value words by
// token, of which each thread then makes one piece of eight tokens, and the scales
// and offsets.  The next head's rows are loaded meanwhile.
// PLAIN: affine codes of tokens that are all this call's, without a transform or a
// window; what the call decides at run time otherwise costs a fifth of the work.
template <int D, int KB, int VB, bool PLAIN>
__device__ __forceinline__ void code_heads(const AppendRopeParams& p, int b, int h0, int heads, int t0)
{
    constexpr int PPT = D / 8, T = kThreads / PPT;
    struct Buffer {
        uint8_t k[kThreads * KB], v[kThreads * VB];
        float meta[4][64];  // key scales, offsets, value scales, offsets: [groups][T]
    };
    __shared__ __attribute__((aligned(16))) Buffer buffers[2];
    const int tid = threadIdx.x, i = tid / PPT, P = tid % PPT, t = t0 + i;
    const bool fresh = PLAIN || t >= p.n0;
    const size_t row = fresh ? input_row(p, b, t - p.n0) * p.H : ((size_t)b * p.H) * p.ring + t % p.ring;
    const size_t step = fresh ? D : (size_t)p.ring * D;  // from head to head
    const uint16_t* ksrc = (fresh ? p.kin : p.kr) + row * D + h0 * step + 8 * P;
    const uint16_t* vsrc = (fresh ? p.vin : p.vr) + row * D + h0 * step + 8 * P;
    u32x4 kw = *(const u32x4*)ksrc, vw = *(const u32x4*)vsrc, norm = {0u, 0u, 0u, 0u};
    if (p.rope.wk)
        norm = *(const u32x4*)(p.rope.wk + 8 * P);
    const Angles turn = fresh ? Angles(p.rope, input_position(p, b, t - p.n0), P) : Angles();

    const Coder<KB, PLAIN> kcode(p.k_mode);
    const Coder<VB, PLAIN> vcode(p.v_mode);
    const int tau = t % kBlockTok, o0 = t0 % kBlockTok / 8;
    const Groups<D> kg(p.k_group), vg(p.v_group);
    // this thread's key piece in its buffer: run (half, P % 4), row of the run, P / 4
    const int kp = (((tau >> 2 & 1) * 4 + (P & 3)) * (T / 2) + 4 * ((tau >> 3) - o0) + (tau & 3)) * (D / 32) + (P >> 2);
    // the value piece it makes (octet, channel) of words vfirst, vfirst + PPT, ..
    const int vd = 16 * (tid % (D / 16)) + tid / (D / 16) % 16, vfirst = 8 * (tid / D) * PPT + vd / 8;
    // the metadata element it stores: of array tid / 64, group and token
    const int ma = __builtin_amdgcn_readfirstlane(tid >> 6), mg = (tid & 63) / T, ng = ma < 2 ? kg.count : vg.count;
    const bool stores = mg < ng && (!(ma & 1) || (ma == 1 ? p.k_mode : p.v_mode) == KVQ_AFFINE);
    float* meta = ma == 0 ? p.ks : ma == 1 ? p.kz : ma == 2 ? p.vs : p.vz;
    // of head h0; every head is `blocks` blocks on
    const size_t blk = (size_t)(b * p.H + h0) * (size_t)(p.T / kBlockTok) + (size_t)(t0 / kBlockTok), blocks = p.T / kBlockTok;
    const int run = tid / (2 * KB);
    uint8_t* kdst = (uint8_t*)p.kc + (blk * (size_t)(4 * D) + (size_t)(((run >> 2) * 64 + 16 * (run & 3) + 4 * o0) * (D / 32))) * KB +
                    16 * (tid % (2 * KB));
    uint8_t* vdst = (uint8_t*)p.vc + (blk * (size_t)(4 * D) + (size_t)(16 * o0 * (D / 16)) + tid) * VB;
    size_t mdst = (blk * ng + mg) * kBlockTok + 8 * o0 + (tid & 63) % T;
    const auto widen = [&](const u32x4& w, float* x) {
        if (fresh) {
            widen8(w, x);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                x[2 * q] = f16_bits_to_f32((uint16_t)w[q]);
                x[2 * q + 1] = f16_bits_to_f32((uint16_t)(w[q] >> 16));
            }
        }
    };
    const auto to_cache = [&](float* x) {  // as the coder sees it (a window's slots hold rows that are)
        if (!PLAIN && p.rotate && fresh)  // (all lanes of a row or none)
            rotate8<D>(x, P, p.rot_c);
        if (!PLAIN && p.ring && fresh) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = f16_bits_to_f32(f32_to_f16_bits(x[e]));
        }
    };
    for (int j = 0; j < heads; ++j) {
        Buffer& buf = buffers[j & 1];
        float x[8], s, z;
        widen(kw, x);
        ksrc += step;
        if (j + 1 < heads)
            kw = *(const u32x4*)ksrc;
        if (fresh)
            turn.template turn<D>(p.rope, norm, P, x);
        to_cache(x);
        const Divisor kdiv = kcode.scale(x, kg.lanes, p.meta16, &s, &z);
        if (kg.first(P)) {
            buf.meta[0][kg.of(P) * T + i] = s;
            buf.meta[1][kg.of(P) * T + i] = z;
        }
        store_piece(buf.k, kp, KB, kcode.piece(x, kdiv));
        widen(vw, x);
        vsrc += step;
        if (j + 1 < heads)
            vw = *(const u32x4*)vsrc;
        to_cache(x);
        const Divisor vdiv = vcode.scale(x, vg.lanes, p.meta16, &s, &z);
        if (vg.first(P)) {
            buf.meta[2][vg.of(P) * T + i] = s;
            buf.meta[3][vg.of(P) * T + i] = z;
        }
        store_piece(buf.v, i * PPT + P, VB, vcode.piece(x, vdiv));
        __syncthreads();
        if (tid < 16 * KB)  // 16 bytes of the key pieces
            *(u32x4*)kdst = *(const u32x4*)(buf.k + 16 * tid);
        uint64_t word = 0;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const uint64_t w = load_piece(buf.v, vfirst + q * PPT, VB);
            if constexpr (VB == 8)
                word |= (w >> (8 * (vd & 7)) & 0xFFu) << (8 * q);
            else
                word |= (uint32_t)((uint32_t)w >> (VB * (vd & 7)) & ((1u << VB) - 1u)) << (VB * q);
        }
        store_piece(vdst, 0, VB, word);
        if (stores)
            store_meta(meta, mdst, buf.meta[ma][tid & 63], p.meta16);
        kdst += blocks * (size_t)(4 * D * KB);
        vdst += blocks * (size_t)(4 * D * VB);
        mdst += blocks * (size_t)(ng * kBlockTok);
    }
}

// The part of block tb that this call codes, tokens lo .. hi - 1 of one head (per-token
// groups; never of a window, which is coded by whole blocks).  Value pieces keep the
// bits of tokens appended earlier and clear later ones; those of the first octet are
// loaded first, with the rows.  Bound by latency: five tokens of 16 x 8 heads of 128 take
// 5.2 us; 7.0 where a thread codes a key and then a value, which more tokens than T / 2
// do (31 of 8 x 8 heads of 256: 10.4, 12.7 with keys and values apart); 11.0 where all 32
// rows are taken and old pieces are loaded when they are needed.
template <int D, int KB, int VB, bool PLAIN>
__device__ __forceinline__ void code_edge(const AppendRopeParams& p, int unit, int tb)
{
    constexpr int PPT = D / 8, T = kThreads / PPT;
    __shared__ __attribute__((aligned(16))) uint8_t words[4 * D * VB];  // [token][PPT]
    const int tid = threadIdx.x, P = tid % PPT, b = unit / p.H, h = unit % p.H;
    const int lo = max(p.q0, tb), hi = min(p.q1, tb + kBlockTok), o0 = (lo - tb) >> 3, o1 = (hi - 1 - tb) >> 3;
    const size_t blk = (size_t)unit * (size_t)(p.T / kBlockTok) + (size_t)(tb / kBlockTok);
    uint64_t old = 0;
    if ((lo & 7) && tid < D)
        old = load_piece(p.vc, value_piece<D>(blk, o0, tid), VB) & low_codes(VB, lo & 7);
    const Coder<KB, PLAIN> kcode(p.k_mode);
    const Coder<VB, PLAIN> vcode(p.v_mode);
    const Groups<D> kg(p.k_group), vg(p.v_group);
    const auto load = [&](const uint16_t* in, int t) {
        return *(const u32x4*)(in + (input_row(p, b, t - p.n0) * p.H + h) * D + 8 * P);
    };
    const auto key = [&](int t, const u32x4& w) {
        float x[8], s, z;
        const Angles turn(p.rope, input_position(p, b, t - p.n0), P);
        widen8(w, x);
        turn.template turn<D>(p.rope, P, x);
        if (!PLAIN && p.rotate)
            rotate8<D>(x, P, p.rot_c);
        const Divisor by = kcode.scale(x, kg.lanes, p.meta16, &s, &z);
        if (kg.first(P)) {
            const size_t mi = (blk * kg.count + kg.of(P)) * kBlockTok + (t - tb);
            store_meta(p.ks, mi, s, p.meta16);
            if (kcode.affine)
                store_meta(p.kz, mi, z, p.meta16);
        }
        store_piece(p.kc, key_piece<D>(blk, t - tb, P), KB, kcode.piece(x, by));
    };
    const auto value = [&](int t, const u32x4& w) {
        float x[8], s, z;
        widen8(w, x);
        if (!PLAIN && p.rotate)
            rotate8<D>(x, P, p.rot_c);
        const Divisor by = vcode.scale(x, vg.lanes, p.meta16, &s, &z);
        if (vg.first(P)) {
            const size_t mi = (blk * vg.count + vg.of(P)) * kBlockTok + (t - tb);
            store_meta(p.vs, mi, s, p.meta16);
            if (vcode.affine)
                store_meta(p.vz, mi, z, p.meta16);
        }
        store_piece(words, (t - tb) * PPT + P, VB, vcode.piece(x, by));
    };
    const int row = tid / PPT;  // (all lanes of a row or none)
    if (hi - lo <= T / 2) {  // keys by two waves, values by the others
        const bool keys = row < T / 2;
        const int t = lo + row % (T / 2);
        if (t < hi) {
            const u32x4 w = load(keys ? p.kin : p.vin, t);
            if (keys)
                key(t, w);
            else
                value(t, w);
        }
    } else {
        for (int t = lo + row; t < hi; t += T) {
            const u32x4 kw = load(p.kin, t), vw = load(p.vin, t);
            key(t, kw);
            value(t, vw);
        }
    }
    __syncthreads();
    for (int idx = tid; idx < (o1 - o0 + 1) * D; idx += kThreads) {
        const int o = o0 + idx / D, d = idx % D;
        uint64_t word = idx < D ? old : 0;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int t = tb + 8 * o + q;
            const uint64_t c = load_piece(words, (8 * o + q) * PPT + d / 8, VB) >> (VB * (d & 7)) & ((1u << VB) - 1u);
            word |= t >= lo && t < hi ? c << (VB * q) : 0;
        }
        store_piece(p.vc, value_piece<D>(blk, o, d), VB, word);
    }
}

// Block tb of one sequence's heads h0 .. with per-channel keys: a thread owns eight
// channels of D / 64 tokens.  The angles of the block's tokens are computed once, for
// all heads, and kept in LDS (ANGLES: 16 KiB at D = 128; at 256 they would leave one
// workgroup per CU, so a workgroup takes one head and computes its own); 16-byte
// pieces of them are swapped by row and lane so that 16 lanes hit 16 different ones.
template <int D, int KB, int VB>
__device__ __forceinline__ void code_channels(const AppendRopeParams& p, int b, int h0, int heads, int tb)
{
    constexpr int PPT = D / 8, kSteps = RowStage<D>::kSteps;
    constexpr bool kAngles = D <= 128;
    __shared__ __attribute__((aligned(16))) uint8_t kbuf[4 * D * KB], vbuf[4 * D * VB];
    __shared__ __attribute__((aligned(16))) float meta[2][kBlockTok * 8];  // value scales, offsets: [groups][32]
    __shared__ __attribute__((aligned(16))) float red[2][4][D], cs[3][D];  // extremes by wave; each channel's Divisor
    __shared__ __attribute__((aligned(16))) float4 angles[kAngles ? kBlockTok : 1][kAngles ? D / 4 : 1];
    const int tid = threadIdx.x, P = tid % PPT, lane = tid & 63, wave = tid >> 6;
    const Coder<KB, false> kcode(p.k_mode);
    const Coder<VB, false> vcode(p.v_mode);
    const Groups<D> vg(p.v_group);
    const int ng = vg.count;
    const auto fresh = [&](int k) { return tb + RowStage<D>::row(k) >= p.n0; };  // (all lanes of a row or none)
    RowStage<D> kst, vst;
    kst.load(p, 0, b, h0, tb);
    vst.load(p, 1, b, h0, tb);
    // where row i's angles of pairs 8 u + 2 j, 8 u + 2 j + 1 are
    const auto place = [&](int i, int u, int j) { return 4 * u + (j ^ ((u + i) & 3)); };
    if constexpr (kAngles) {
        for (int x = tid; x < kBlockTok * (D / 4); x += kThreads) {
            const int i = x / (D / 4), c = x % (D / 4);  // pairs 2 c, 2 c + 1
            const int t = tb + i;
            if (t < p.n0 || 4 * c >= p.rope.rot)
                continue;
            const int at = input_position(p, b, t - p.n0);
            const float2 a = rope_cos_sin(at, p.rope.turns[2 * c], p.rope.scale);
            const float2 d = rope_cos_sin(at, p.rope.turns[2 * c + 1], p.rope.scale);
            angles[i][place(i, c >> 2, c & 3)] = make_float4(a.x, a.y, d.x, d.y);
        }
        __syncthreads();
    }
    const auto angles_of = [&](int k) {
        if constexpr (kAngles) {
            const int i = RowStage<D>::row(k), hp = p.rope.rot / 16;
            const bool half = p.rope.layout == KVQ_ROPE_HALF, up = half && P >= hp;
            Angles a;
            if (8 * P < p.rope.rot) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (half) {
                        const float4 x = angles[i][place(i, up ? P - hp : P, j)];
                        a.c[2 * j] = x.x, a.c[2 * j + 1] = x.z;
                        a.s[2 * j] = up ? x.y : -x.y, a.s[2 * j + 1] = up ? x.w : -x.w;
                    } else if (j < 2) {
                        const float4 x = angles[i][place(i, P >> 1, 2 * (P & 1) + j)];
                        a.c[2 * j] = x.x, a.c[2 * j + 1] = x.z;
                        a.s[2 * j] = x.y, a.s[2 * j + 1] = x.w;
                    }
                }
            }
            return a;
        } else {
            return RowStage<D>::angles(p, b, tb, k);
        }
    };
    for (int h = h0; h < h0 + heads; ++h) {
        const size_t blk = (size_t)(b * p.H + h) * (size_t)(p.T / kBlockTok) + (size_t)(tb / kBlockTok);
        float x[kSteps][8], mn[8], mx[8];
        asm volatile("" ::: "memory");  // (angles are read again for every head, not kept in 16 registers a row)
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
            kst.widen(p, tb, k, x[k], fresh(k) ? angles_of(k) : Angles());
        if (h + 1 < h0 + heads)
            kst.load(p, 0, b, h + 1, tb);
        const bool aff = kcode.affine;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            mn[e] = x[0][e];
            mx[e] = aff ? x[0][e] : fabsf(x[0][e]);
#pragma unroll
            for (int k = 1; k < kSteps; ++k) {
                mn[e] = fminf(mn[e], x[k][e]);
                mx[e] = fmaxf(mx[e], aff ? x[k][e] : fabsf(x[k][e]));
            }
            if constexpr (PPT <= 8) {
                mn[e] = fminf(mn[e], row_ror8(mn[e]));
                mx[e] = fmaxf(mx[e], row_ror8(mx[e]));
            }
#pragma unroll
            for (int off = PPT < 16 ? 16 : PPT; off < 64; off <<= 1) {
                mn[e] = fminf(mn[e], __shfl_xor(mn[e], off));
                mx[e] = fmaxf(mx[e], __shfl_xor(mx[e], off));
            }
        }
        if (lane < PPT) {
            *(float4*)&red[0][wave][8 * P] = make_float4(mn[0], mn[1], mn[2], mn[3]);
            *(float4*)&red[0][wave][8 * P + 4] = make_float4(mn[4], mn[5], mn[6], mn[7]);
            *(float4*)&red[1][wave][8 * P] = make_float4(mx[0], mx[1], mx[2], mx[3]);
            *(float4*)&red[1][wave][8 * P + 4] = make_float4(mx[4], mx[5], mx[6], mx[7]);
        }
        __syncthreads();
        if (tid < D) {
            const float lo = fminf(fminf(red[0][0][tid], red[0][1][tid]), fminf(red[0][2][tid], red[0][3][tid]));
            const float hi = fmaxf(fmaxf(red[1][0][tid], red[1][1][tid]), fmaxf(red[1][2][tid], red[1][3][tid]));
            float s = kcode.over_n(aff ? hi - lo : hi), z = aff ? lo + 0.0f : 0.0f;
            round_meta(p.meta16, &s, &z);
            const Divisor by(s, z, aff ? fmaxf(fabsf(lo), fabsf(hi)) : 0.0f);
            cs[0][tid] = by.s;
            cs[1][tid] = by.y;
            cs[2][tid] = by.z;
            store_meta(p.ks, blk * D + tid, s, p.meta16);
            if (aff)
                store_meta(p.kz, blk * D + tid, z, p.meta16);
        }
        __syncthreads();
        float s8[8], r8[8], z8[8];
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
            *(float4*)(s8 + e) = *(const float4*)&cs[0][8 * P + e];
            *(float4*)(r8 + e) = *(const float4*)&cs[1][8 * P + e];
            *(float4*)(z8 + e) = *(const float4*)&cs[2][8 * P + e];
        }
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
            store_piece(kbuf, key_piece<D>(0, RowStage<D>::row(k), P), KB,
                        kcode.piece(x[k], [&](int e) { return s8[e]; }, [&](int e) { return r8[e]; }, [&](int e) { return z8[e]; }));
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int i = RowStage<D>::row(k);
            float v[8], s, z;
            vst.widen(p, tb, k, v, NoAngles());
            const Divisor by = vcode.scale(v, vg.lanes, p.meta16, &s, &z);
            if (vg.first(P)) {
                meta[0][vg.of(P) * kBlockTok + i] = s;
                meta[1][vg.of(P) * kBlockTok + i] = z;
            }
            store_piece(vbuf, i * PPT + P, VB, vcode.piece(v, by));
        }
        if (h + 1 < h0 + heads)
            vst.load(p, 1, b, h + 1, tb);
        // (what the next head writes before its second barrier, nobody reads behind this one)
        __syncthreads();
        for (int at = 16 * tid; at < 4 * D * KB; at += 16 * kThreads)
            *(u32x4*)((uint8_t*)p.kc + blk * (size_t)(4 * D * KB) + at) = *(const u32x4*)(kbuf + at);
#pragma unroll
        for (int x0 = 0; x0 < 4 * D; x0 += kThreads) {  // value piece x: octet, channel
            const int at = x0 + tid, d = 16 * (at % (D / 16)) + at / (D / 16) % 16, first = 8 * (at / D) * PPT + d / 8;
            uint64_t word = 0;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const uint64_t w = load_piece(vbuf, first + q * PPT, VB);
                if constexpr (VB == 8)
                    word |= (w >> (8 * (d & 7)) & 0xFFu) << (8 * q);
                else
                    word |= (uint32_t)((uint32_t)w >> (VB * (d & 7)) & ((1u << VB) - 1u)) << (VB * q);
            }
            store_piece(p.vc, blk * (size_t)(4 * D) + at, VB, word);
        }
        for (int at = tid; at < ng * kBlockTok; at += kThreads) {
            store_meta(p.vs, blk * (size_t)(ng * kBlockTok) + at, meta[0][at], p.meta16);
            if (vcode.affine)
                store_meta(p.vz, blk * (size_t)(ng * kBlockTok) + at, meta[1][at], p.meta16);
        }
    }
}

// A wave's share of a call's queries.
template <int D, int ITER>
__device__ __forceinline__ void rope_queries(const AppendRopeParams& p, uint32_t token, int part, float2* lds)
{
    if (part_in_halves(p.rope, D))
        rope_rows<D, ITER, false, true>(p.queries, p.rope, token, part, lds);
    else
        rope_rows<D, ITER, false, false>(p.queries, p.rope, token, part, lds);
}

// One token per sequence without a window (a decode step), a wave per (sequence, KV
// head): lanes 0 .. D / 8 - 1 hold eight channels each of its key, those from lane 32 on
// of its value, so nothing waits for another wave; further waves rotate queries.  The
// value pieces that it shares with earlier tokens are loaded first.  Bound by one chain
// of latencies, its own instructions' fetch among them: 4 heads of 64 take 3.9 us, 8 of
// 256 of 8 sequences 4.2.  With a thread per channel and reductions through LDS 4.5 and
// 5.4; as this, but widths decided at run time (169 branches), 4.5 and 4.8.
template <int D, int KB, int VB>
__global__ __launch_bounds__(64) void append_token_rope_kernel(AppendRopeParams p)
{
#pragma clang fp contract(off)
    constexpr int PPT = D / 8;
    __shared__ __attribute__((aligned(16))) float2 angles[D / 2];
    const uint32_t x = wg_index();
    if (x >= p.code_wgs) {
        const uint32_t item = x - p.code_wgs, parts = (uint32_t)p.queries.parts, token = item / parts;
        if (token < (uint32_t)p.queries.tokens)
            rope_queries<D, 1>(p, token, (int)(item - token * parts), angles);
        return;
    }
    const int unit = (int)x, b = unit / p.H, h = unit - b * p.H, lane = threadIdx.x, P = lane & 31;
    const bool value = lane >= 32, live = P < PPT;
    const int t = p.n0, tau = t & 31, j = t & 7;
    const size_t blk = (size_t)unit * (size_t)(p.T / kBlockTok) + (size_t)(t / kBlockTok);
    const int bits = value ? VB : KB, group = value ? p.v_group : p.k_group;
    const int log2 = value ? __builtin_ctz(p.v_group) : __builtin_ctz(p.k_group);
    const bool affine = (value ? p.v_mode : p.k_mode) == KVQ_AFFINE;
    const size_t at = (input_row(p, b, 0) * p.H + h) * D + 8 * P;
    u32x4 w = {0u, 0u, 0u, 0u};
    uint64_t old[8];
    if (live)
        w = *(const u32x4*)((value ? p.vin : p.kin) + at);
    if (live && value && j) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            old[e] = load_piece(p.vc, value_piece<D>(blk, tau >> 3, 8 * P + e), VB);
    }
    float v[8];
    if (live && !value) {
        const Angles turn(p.rope, input_position(p, b, 0), P);
        widen8(w, v);
        turn.template turn<D>(p.rope, P, v);
    } else {
        widen8(w, v);
    }
    if (p.rotate)  // (every lane of a row takes part)
        rotate8<D>(v, P, p.rot_c);
    // the group's extremes, over group / 8 lanes
    float mn = v[0], mx = v[0], ma;
#pragma unroll
    for (int e = 1; e < 8; ++e) {
        mn = fminf(mn, v[e]);
        mx = fmaxf(mx, v[e]);
    }
    const auto step = [&](float a, float c) {
        mn = fminf(mn, a);
        mx = fmaxf(mx, c);
    };
    typedef Coder<4, true> Dpp;
    step(Dpp::dpp<0xB1>(mn), Dpp::dpp<0xB1>(mx));
    step(Dpp::dpp<0x4E>(mn), Dpp::dpp<0x4E>(mx));
    float a = Dpp::dpp<0x141>(mn), c = Dpp::dpp<0x141>(mx);
    if (group > 32)
        step(a, c);
    a = Dpp::dpp<0x140>(mn), c = Dpp::dpp<0x140>(mx);
    if (group > 64)
        step(a, c);
    a = __shfl_xor(mn, 16), c = __shfl_xor(mx, 16);
    if (group > 128)
        step(a, c);
    ma = fmaxf(fabsf(mn), fabsf(mx));
    const float top = (float)((1 << bits) - 1), qmax = (float)((1 << (bits - 1)) - 1);
    float s = fmaxf((affine ? mx - mn : ma) / (affine ? top : qmax), 1e-8f), z = affine ? mn + 0.0f : 0.0f;
    round_meta(p.meta16, &s, &z);
    const Divisor by(s, z, affine ? ma : 0.0f);
    const float lo = affine ? 0.0f : -qmax, hi = affine ? top : qmax, half = affine ? 0.0f : (float)(1 << (bits - 1));
    uint32_t code[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {  // (Coder::piece)
        const float d = from_offset(v[e], by.z);
        float q = d * by.y;
        q = __builtin_fmaf(__builtin_fmaf(-q, by.s, d), by.y, q);
        q = __builtin_fmaf(__builtin_fmaf(-q, by.s, d), by.y, q);
        code[e] = (uint32_t)(__builtin_amdgcn_fmed3f(__builtin_rintf(q), lo, hi) + half);
    }
    if (!live)
        return;
    if ((8 * P & (group - 1)) == 0) {
        const size_t mi = (blk * (size_t)(D >> log2) + (size_t)(8 * P >> log2)) * kBlockTok + tau;
        store_meta(value ? p.vs : p.ks, mi, s, p.meta16);
        if (affine)
            store_meta(value ? p.vz : p.kz, mi, z, p.meta16);
    }
    if (value) {
        const uint64_t keep = low_codes(VB, j);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            store_piece(p.vc, value_piece<D>(blk, tau >> 3, 8 * P + e), VB,
                        (j ? old[e] & keep : 0) | ((uint64_t)code[e] << (VB * j)));
    } else {
        uint64_t word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            word |= (uint64_t)code[e] << (KB * e);
        store_piece(p.kc, key_piece<D>(blk, tau, P), KB, word);
    }
}

// One launch for all that an append with positions does: workgroups that code
// blocks, the longest, come first, then those that write window rows and those that
// rotate queries (four waves of rope_rows).
constexpr int kQueryIter = 4;  // iterations of a wave

// Waves per SIMD that the registers are held to.  (Five with per-token groups spill 16
// to 24 registers: 2048 tokens 3% faster, five tokens 12% slower.)
__host__ __device__ constexpr int append_waves(int D, bool perch)
{
    return !perch ? 4 : D == 256 ? 2 : D == 128 ? 3 : 4;
}

template <int D, bool PERCH, int KB, int VB, bool PLAIN>
__global__ __launch_bounds__(kThreads, append_waves(D, PERCH)) void append_rope_kernel(AppendRopeParams p)
{
    uint32_t x = wg_index();
    if (x < p.code_wgs) {
        const uint32_t units = p.B * p.H, singles = units * p.edges;  // blocks at the ends, by head
        if (!PERCH && x < singles) {
            const int e = (int)(x / units), unit = (int)(x - e * units);
            code_edge<D, KB, VB, PLAIN>(p, unit, kBlockTok * (e == 0 && p.q0 % kBlockTok ? p.q0 / kBlockTok : p.q1 / kBlockTok));
        } else {
            constexpr int T = PERCH ? kBlockTok : 2048 / D, PARTS = kBlockTok / T;
            x -= singles;
            const uint32_t hg = (p.H + p.heads - 1) / p.heads, y = x / hg, h0 = (x - y * hg) * p.heads;
            const uint32_t b = y / (p.blocks * PARTS), part = y - b * (p.blocks * PARTS);
            const int heads = min(p.heads, p.H - (int)h0), t0 = (p.q0 + kBlockTok - 1) / kBlockTok * kBlockTok + (int)part * T;
            if constexpr (PERCH)
                code_channels<D, KB, VB>(p, (int)b, (int)h0, heads, t0);
            else
                code_heads<D, KB, VB, PLAIN>(p, (int)b, (int)h0, heads, t0);
        }
        return;
    }
    x -= p.code_wgs;
    if (x < p.row_wgs) {
        const uint32_t per = p.row_wgs / (p.B * p.H), unit = x / per;
        write_rows<D>(p, p.n0 + p.n_new, (int)unit, p.ring_lo + kRingRows<D> * (int)(x - unit * per));
        return;
    }
    __shared__ __attribute__((aligned(16))) float2 angles[kThreads / 64][D / 2];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const uint32_t item = (x - p.row_wgs) * (kThreads / 64) + wave, token = item / (uint32_t)p.queries.parts;
    if (token < (uint32_t)p.queries.tokens)
        rope_queries<D, kQueryIter>(p, token, (int)(item - token * (uint32_t)p.queries.parts), angles[wave]);
}

template <int D>
void launch_token(const AppendRopeParams& p, dim3 g, hipStream_t stream)
{
    if (p.k_bits == 8)
        launch_kernel(append_token_rope_kernel<D, 8, 8>, g, dim3(64), 0, stream, p);
    else if (p.k_bits == 4 && p.v_bits == 4)
        launch_kernel(append_token_rope_kernel<D, 4, 4>, g, dim3(64), 0, stream, p);
    else if (p.k_bits == 4)
        launch_kernel(append_token_rope_kernel<D, 4, 2>, g, dim3(64), 0, stream, p);
    else if (p.v_bits == 4)
        launch_kernel(append_token_rope_kernel<D, 2, 4>, g, dim3(64), 0, stream, p);
    else
        launch_kernel(append_token_rope_kernel<D, 2, 2>, g, dim3(64), 0, stream, p);
}

template <int D, bool PERCH, bool PLAIN>
void launch_blocks(const AppendRopeParams& p, uint32_t grid, hipStream_t stream)
{
    const dim3 g = grid_of(grid), t(kThreads);
    if (p.k_bits == 8)
        launch_kernel((append_rope_kernel<D, PERCH, 8, 8, PLAIN>), g, t, 0, stream, p);
    else if (p.k_bits == 4 && p.v_bits == 4)
        launch_kernel((append_rope_kernel<D, PERCH, 4, 4, PLAIN>), g, t, 0, stream, p);
    else if (p.k_bits == 4)
        launch_kernel((append_rope_kernel<D, PERCH, 4, 2, PLAIN>), g, t, 0, stream, p);
    else if (p.v_bits == 4)
        launch_kernel((append_rope_kernel<D, PERCH, 2, 4, PLAIN>), g, t, 0, stream, p);
    else
        launch_kernel((append_rope_kernel<D, PERCH, 2, 2, PLAIN>), g, t, 0, stream, p);
}

template <int D>
hipError_t launch_append_d(AppendRopeParams p, hipStream_t stream)
{
    const int units = p.B * p.H, n1 = p.n0 + p.n_new;
    if (p.n_new == 1 && p.ring == 0 && p.k_axis == KVQ_PER_TOKEN) {
        constexpr int RPI = 1024 / D;
        p.queries.parts = p.queries.tokens > 0 ? (p.queries.H_q + RPI - 1) / RPI : 1;
        p.code_wgs = (uint32_t)units;
        launch_token<D>(p, grid_of(p.code_wgs + (uint32_t)(p.queries.tokens * p.queries.parts)), stream);
        return hipGetLastError();
    }
    // whole blocks by code_heads or code_channels, those at the ends by code_edge
    const int lo = (p.q0 + kBlockTok - 1) / kBlockTok, hi = p.q1 / kBlockTok;
    const bool perch = p.k_axis == KVQ_PER_CHANNEL;  // (whole blocks only)
    p.blocks = hi < lo ? 0 : hi - lo;
    p.edges = p.q1 <= p.q0 || perch ? 0 : hi < lo ? 1 : (p.q0 % kBlockTok != 0) + (p.q1 % kBlockTok != 0);
    const long long parts = (long long)p.blocks * p.B * (perch ? 1 : kBlockTok * D / 2048);
    p.heads = 1;
    while (p.heads < (perch && D == 256 ? 1 : 4) && p.heads < p.H && parts * p.H > (perch ? 1024 : 4096) * p.heads)
        p.heads *= 2;
    p.code_wgs = (uint32_t)(parts * ((p.H + p.heads - 1) / p.heads)) + (uint32_t)(p.edges * units);
    // the window's rows beside the coder, if none takes the slot of a token that is coded from it
    const bool ring = p.ring && n1 > p.ring_lo, together = ring && n1 - p.ring <= p.q0;
    p.row_wgs = together ? (uint32_t)((n1 - p.ring_lo + kRingRows<D> - 1) / kRingRows<D>) * (uint32_t)units : 0;
    uint32_t others = p.row_wgs;
    p.queries.parts = 1;  // (a divisor, without queries too)
    if (p.queries.tokens > 0) {
        constexpr int RPI = 1024 / D;
        p.queries.parts = (p.queries.H_q + RPI * kQueryIter - 1) / (RPI * kQueryIter);
        others += (uint32_t)(((long long)p.queries.tokens * p.queries.parts + kThreads / 64 - 1) / (kThreads / 64));
    }
    const uint32_t grid = p.code_wgs + others;
    if (grid > 0) {
        if (perch)
            launch_blocks<D, true, false>(p, grid, stream);
        else if (p.k_mode == KVQ_AFFINE && p.v_mode == KVQ_AFFINE && !p.rotate && !p.ring)
            launch_blocks<D, false, true>(p, grid, stream);
        else
            launch_blocks<D, false, false>(p, grid, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    if (ring && !together)
        launch_ring<D>(p, n1, stream);
    return hipGetLastError();
}

typedef AppendRopeParams Params;
#else
template <int D, bool PERCH>
void launch_blocks(const AppendParams& p, int blocks, int units, hipStream_t stream)
{
    const dim3 g(blocks, units), t(kThreads);
    if (p.k_bits == 8)  // 8-bit codes come as K and V both 8-bit
        launch_kernel((append_block_kernel<D, PERCH, 8, 8>), g, t, 0, stream, p);
    else if (p.k_bits == 4 && p.v_bits == 4)
        launch_kernel((append_block_kernel<D, PERCH, 4, 4>), g, t, 0, stream, p);
    else if (p.k_bits == 4)
        launch_kernel((append_block_kernel<D, PERCH, 4, 2>), g, t, 0, stream, p);
    else if (p.v_bits == 4)
        launch_kernel((append_block_kernel<D, PERCH, 2, 4>), g, t, 0, stream, p);
    else
        launch_kernel((append_block_kernel<D, PERCH, 2, 2>), g, t, 0, stream, p);
}

template <int D>
hipError_t launch_append_d(const AppendParams& p, hipStream_t stream)
{
    const int units = p.B * p.H;
    if (p.n_new == 1 && p.ring == 0 && p.k_axis == KVQ_PER_TOKEN) {
        launch_kernel(append_token_kernel<D>, dim3(units), dim3(D), 0, stream, p);
        return hipGetLastError();
    }
    if (p.q1 > p.q0) {
        const int blocks = (p.q1 + kBlockTok - 1) / kBlockTok - p.q0 / kBlockTok;
        if (p.k_axis == KVQ_PER_CHANNEL)
            launch_blocks<D, true>(p, blocks, units, stream);
        else
            launch_blocks<D, false>(p, blocks, units, stream);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    const int n1 = p.n0 + p.n_new;
    if (p.ring && n1 > p.ring_lo)
        launch_ring<D>(p, n1, stream);
    return hipGetLastError();
}

typedef AppendParams Params;
#endif

template <int D>
hipError_t launch_rows_d(const Params& p, int hi, hipStream_t stream)
{
    if (hi > p.ring_lo)
        launch_ring<D>(p, hi, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append_rows(const Params& p, int D, int hi, hipStream_t stream)
{
    switch (D) {
    case 64:
        return launch_rows_d<64>(p, hi, stream);
    case 128:
        return launch_rows_d<128>(p, hi, stream);
    case 256:
        return launch_rows_d<256>(p, hi, stream);
    default:
        return hipErrorInvalidValue;
    }
}

hipError_t launch_append(const Params& p, int D, hipStream_t stream)
{
    switch (D) {
    case 64:
        return launch_append_d<64>(p, stream);
    case 128:
        return launch_append_d<128>(p, stream);
    case 256:
        return launch_append_d<256>(p, stream);
    default:
        return hipErrorInvalidValue;
    }
}

}  // namespace kvq
