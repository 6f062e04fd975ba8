// Shared-prefix attention: work planning, dispatch to the kernel families
// (shared_part.hip) and the kernel that joins a row's partials.

#include "shared_impl.h"

namespace kvq {

#define KVQ_FAMILY(D, KG) hipError_t launch_shared_##D##_##KG(const SharedParams& p, int items, hipStream_t stream);
KVQ_FAMILY(64, 0) KVQ_FAMILY(64, 1) KVQ_FAMILY(64, 2)
KVQ_FAMILY(128, 0) KVQ_FAMILY(128, 1) KVQ_FAMILY(128, 2) KVQ_FAMILY(128, 4)
KVQ_FAMILY(256, 0) KVQ_FAMILY(256, 1) KVQ_FAMILY(256, 2) KVQ_FAMILY(256, 4) KVQ_FAMILY(256, 8)
#undef KVQ_FAMILY

namespace {

// A workgroup fills a compute unit, so a round is one work item per CU.
constexpr int kRound = 256;

int ceil_div(int a, int b)
{
    return (a + b - 1) / b;
}

// Ranges that a segment of `tiles` tiles is cut into, at most.
int shared_splits(long long tiles)
{
    return tiles > 0 && tiles < kRound ? (int)(kRound / tiles) : 1;
}

// Joins the partials of a row: one thread per four output channels,
// O = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s, then the inverse rotation
// of a rotating format (the normalized transform is its own inverse) in LDS.
constexpr int kJoinThreads = 256;

template <int D>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(SharedParams p)
{
    constexpr int R = kJoinThreads / (D / 4);  // rows per workgroup
    __shared__ __attribute__((aligned(16))) float x[R * D];
    const int rl = threadIdx.x / (D / 4), d = 4 * (threadIdx.x % (D / 4));
    const size_t row = (size_t)blockIdx.x * R + rl;
    const int S = p.S[0] + p.S[1];
    floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    float M = -INFINITY, L = 0.0f;
    if (row < p.rows) {
        for (int s = 0; s < S; ++s)
            M = fmaxf(M, p.part_ml[2 * ((size_t)s * p.rows + row)]);
#pragma unroll 4
        for (int s = 0; s < S; ++s) {
            const size_t at = (size_t)s * p.rows + row;
            const float2 ml = *(const float2*)(p.part_ml + 2 * at);
            const floatx4 o = *(const floatx4*)(p.part_o + at * D + d);
            const float w = ml.x == -INFINITY ? 0.0f : fast_exp2(ml.x - M);
            acc += o * w;
            L += ml.y * w;
        }
    }
    acc *= 1.0f / L;  // every row sees a token
    if (!p.rotate) {
        if (row < p.rows)
            *(floatx4*)(p.out + row * D + d) = acc;
        return;
    }
    *(floatx4*)(x + rl * D + d) = acc;
    __syncthreads();
    for (int h = 1; h < D; h <<= 1) {
        for (int i = threadIdx.x; i < R * (D / 2); i += kJoinThreads) {
            const int r = i / (D / 2), k = i % (D / 2), jj = r * D + (k / h) * 2 * h + (k % h);
            const float a = x[jj], c = x[jj + h];
            x[jj] = a + c;
            x[jj + h] = a - c;
        }
        __syncthreads();
    }
    if (row < p.rows)
        *(floatx4*)(p.out + row * D + d) = *(const floatx4*)(x + rl * D + d) * p.rot_c;
}

template <int D>
void launch_join(const SharedParams& p, hipStream_t stream)
{
    constexpr int R = kJoinThreads / (D / 4);
    launch_kernel(join_kernel<D>, dim3((unsigned)((p.rows + R - 1) / R)), dim3(kJoinThreads), 0, stream, p);
}

}  // namespace

// Work items.  Prefix items are long (many rows) and few, suffix items short
// and many; the former start first and the latter fill the CUs that they leave.
// So prefix units are cut for one round of their own, at most: ranges of
// blocks of a whole number of build phases.
int shared_plan(SharedParams* p, int D, int B)
{
    const AttnParams &a = p->seg[0], &b = p->seg[1];
    const int per = shr::item_rows(D), NI = shr::images(D);
    p->tile_rows = per;
    p->tiles0 = 0;
    for (int g = 0; g < p->P; ++g) {
        p->tile0[g] = p->tiles0;
        p->tiles0 += a.H * ceil_div((p->first[g + 1] - p->first[g]) * p->C * a.G, per);
    }
    p->tile0[p->P] = p->tiles0;
    const int tiles[2] = {p->tiles0, B * a.H * ceil_div(p->C * a.G, per)};
    for (int k = 0; k < 2; ++k) {
        const AttnParams& s = k ? b : a;
        const int blocks = ceil_div(s.n_sink, 32) + ceil_div(s.n > 0 ? s.n : 0, 32);
        const int want = shared_splits(tiles[k]);
        p->bps[k] = blocks > 0 ? ceil_div(ceil_div(blocks, want), NI) * NI : NI;
        p->S[k] = ceil_div(blocks, p->bps[k]);
    }
    p->items0 = p->tiles0 * p->S[0];
    return p->items0 + tiles[1] * p->S[1];
}

int shared_split_bound(int B, int H, int D, int C, int G)
{
    // the groups' tiles are never fewer than one group's of all rows
    const int per = shr::item_rows(D);
    return shared_splits((long long)H * ceil_div(B * C * G, per)) +
           shared_splits((long long)B * H * ceil_div(C * G, per));
}

hipError_t launch_shared(const SharedParams& p, int D, int items, hipStream_t stream)
{
    const AttnParams& a = p.seg[0];
    const int kg = a.k_axis == KVQ_PER_CHANNEL ? 0 : a.k_group / 32;
    hipError_t e = hipErrorInvalidValue;
    switch (1000 * D + kg) {
#define KVQ_FAMILY(D, KG)                           \
    case 1000 * D + KG:                             \
        e = launch_shared_##D##_##KG(p, items, stream); \
        break;
        KVQ_FAMILY(64, 0)
        KVQ_FAMILY(64, 1)
        KVQ_FAMILY(64, 2)
        KVQ_FAMILY(128, 0)
        KVQ_FAMILY(128, 1)
        KVQ_FAMILY(128, 2)
        KVQ_FAMILY(128, 4)
        KVQ_FAMILY(256, 0)
        KVQ_FAMILY(256, 1)
        KVQ_FAMILY(256, 2)
        KVQ_FAMILY(256, 4)
        KVQ_FAMILY(256, 8)
#undef KVQ_FAMILY
    }
    if (e != hipSuccess)
        return e;
    if (D == 64)
        launch_join<64>(p, stream);
    else if (D == 128)
        launch_join<128>(p, stream);
    else
        launch_join<256>(p, stream);
    return hipGetLastError();
}

}  // namespace kvq
