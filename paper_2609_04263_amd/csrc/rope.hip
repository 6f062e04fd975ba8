// Rotary positions of queries and keys with the RMS norm of each head in the
// same pass (kvq_rope_qk).  rope.h has the arithmetic.
//
// A lane holds sixteen channels of a row, such that both members of each of its
// eight pairs are its own and the pairs are 8 l .. 8 l + 7 in either layout:
//     halves       channels 8 l .. and rot / 2 + 8 l ..  (l < rot / 16)
//     interleaved  channels 16 l .. 16 l + 15, as are those that are not rotated
// (two 16-byte loads), so rotating needs no exchange, and lane l's eight cosines
// and sines are the same for every head of a token.  A wave takes some of the
// heads of one token, 1024 / D rows at a time: its lanes compute each cosine
// once, pass them on through LDS and keep their eight in registers.
#include "rope.h"

namespace kvq {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// ITER: rows of a wave are ITER times 1024 / D, all loaded before the angles are
// computed.
template <int D, int ITER>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeQkParams p)
{
    constexpr int LPR = D / 16, RPI = 64 / LPR;  // lanes of a row, rows of an iteration
    __shared__ __attribute__((aligned(16))) float2 lds[kWaves][D / 2];
    const int lane = threadIdx.x & 63, l = lane & (LPR - 1);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const uint32_t item = blockIdx.x * kWaves + wave, token = item / (uint32_t)p.parts;
    const int part = (int)(item - token * (uint32_t)p.parts);
    if (token >= (uint32_t)p.tokens)  // (waves of a workgroup do not wait for each other)
        return;
    const RopeArgs& r = p.rope;
    const bool half = r.layout == KVQ_ROPE_HALF && l < r.rot / 16;
    const int c0 = half ? 8 * l : 16 * l, c1 = half ? r.rot / 2 + 8 * l : 16 * l + 8;

    u32x4 w[ITER][2];
    const int heads = p.H_q + p.H, h0 = part * ITER * RPI + lane / LPR;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int h = h0 + i * RPI;
        if (h < heads) {
            const uint16_t* row = h < p.H_q ? p.q + ((size_t)token * p.H_q + h) * D
                                            : p.k + ((size_t)token * p.H + (h - p.H_q)) * D;
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
                lds[wave][i] = rope_cos_sin(t, r.turns[i], r.scale);
        asm volatile("" ::: "memory");  // LDS accesses of a wave are performed in order
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const float4 x = *(const float4*)&lds[wave][8 * l + j];
            cs[j] = x.x, sn[j] = x.y, cs[j + 1] = x.z, sn[j + 1] = x.w;
        }
    }
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int h = h0 + i * RPI;
        float v[16];
        widen8(w[i][0], v);
        widen8(w[i][1], v + 8);
        const bool is_q = h < p.H_q;
        const uint16_t* weight = is_q ? r.wq : r.wk;
        const bool live = h < heads;
        if (r.wq || r.wk) {  // (every lane of a row takes part in its sum)
            const double sum = row_sum<LPR>(squares8(v) + squares8(v + 8));
            if (live && weight) {
                const float f = norm_factor(sum, D, r.eps);
                float g[8];
                widen8(*(const u32x4*)(weight + c0), g);
                norm8(v, f, g);
                widen8(*(const u32x4*)(weight + c1), g);
                norm8(v + 8, f, g);
            }
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
        if (live) {
            uint16_t* row = is_q ? p.qo + ((size_t)token * p.H_q + h) * D : p.ko + ((size_t)token * p.H + (h - p.H_q)) * D;
            *(u32x4*)(row + c0) = narrow8(v);
            *(u32x4*)(row + c1) = narrow8(v + 8);
        }
    }
}

template <int D>
hipError_t launch_d(RopeQkParams p, hipStream_t stream)
{
    constexpr int RPI = 1024 / D;
    const int iters = (p.H_q + p.H + RPI - 1) / RPI;
    // few tokens: a wave per RPI rows; else up to four iterations of a wave
    const int iter = p.tokens * iters <= 1024 ? 1 : (iters + (iters + 3) / 4 - 1) / ((iters + 3) / 4);
    p.parts = (iters + iter - 1) / iter;
    const dim3 g((unsigned)((p.tokens * p.parts + kWaves - 1) / kWaves)), t(kThreads);
    if (iter == 1)
        launch_kernel((rope_kernel<D, 1>), g, t, 0, stream, p);
    else if (iter == 2)
        launch_kernel((rope_kernel<D, 2>), g, t, 0, stream, p);
    else if (iter == 3)
        launch_kernel((rope_kernel<D, 3>), g, t, 0, stream, p);
    else
        launch_kernel((rope_kernel<D, 4>), g, t, 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeQkParams& p, int D, hipStream_t stream)
{
    switch (D) {
    case 64:
        return launch_d<64>(p, stream);
    case 128:
        return launch_d<128>(p, stream);
    case 256:
        return launch_d<256>(p, stream);
    default:
        return hipErrorInvalidValue;
    }
}

}  // namespace kvq
