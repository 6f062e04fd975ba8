// Rotary positions of queries and keys with the RMS norm of each head in the
// same pass (kvq_rope_qk): rope_rows in rope.h, a wave per token and some of its
// heads.  Bound by HBM: 16384 tokens of 24 normed heads of 256 (402 MB) take 80 us,
// 5.0 TB/s, as a copy of 1 GiB does; small calls by the launch (one token 2.3 us).
#include "rope.h"

namespace kvq {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

template <int D, int ITER, bool PART>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeQkParams p, RopeArgs r)
{
    __shared__ __attribute__((aligned(16))) float2 lds[kWaves][D / 2];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const uint32_t item = wg_index() * kWaves + wave, token = item / (uint32_t)p.parts;
    if (token < (uint32_t)p.tokens)  // (waves of a workgroup do not wait for each other)
        rope_rows<D, ITER, true, PART>(p, r, token, (int)(item - token * (uint32_t)p.parts), lds[wave]);
}

template <int D, bool PART>
hipError_t launch_d(RopeQkParams p, const RopeArgs& rope, hipStream_t stream)
{
    constexpr int RPI = 1024 / D;
    const int iters = (p.H_q + p.H + RPI - 1) / RPI;
    // Few tokens: a wave per RPI rows (latency), many: up to four iterations of a wave,
    // which share its angles.  One / up to four, us: 192 tokens of 24 heads of 256 3.6 /
    // 4.7, 400 of 40 of 128 3.7 / 4.3, 2000 of 24 of 256 12.6 / 12.1.
    const int iter = (long long)p.tokens * iters <= 8192 ? 1 : (iters + (iters + 3) / 4 - 1) / ((iters + 3) / 4);
    p.parts = (iters + iter - 1) / iter;
    const dim3 g = grid_of((uint32_t)(((long long)p.tokens * p.parts + kWaves - 1) / kWaves)), t(kThreads);
    if (iter == 1)
        launch_kernel((rope_kernel<D, 1, PART>), g, t, 0, stream, p, rope);
    else if (iter == 2)
        launch_kernel((rope_kernel<D, 2, PART>), g, t, 0, stream, p, rope);
    else if (iter == 3)
        launch_kernel((rope_kernel<D, 3, PART>), g, t, 0, stream, p, rope);
    else
        launch_kernel((rope_kernel<D, 4, PART>), g, t, 0, stream, p, rope);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeQkParams& p, const RopeArgs& rope, int D, hipStream_t stream)
{
    switch (D) {
    case 64:
        return part_in_halves(rope, D) ? launch_d<64, true>(p, rope, stream) : launch_d<64, false>(p, rope, stream);
    case 128:
        return part_in_halves(rope, D) ? launch_d<128, true>(p, rope, stream) : launch_d<128, false>(p, rope, stream);
    case 256:
        return part_in_halves(rope, D) ? launch_d<256, true>(p, rope, stream) : launch_d<256, false>(p, rope, stream);
    default:
        return hipErrorInvalidValue;
    }
}

}  // namespace kvq
