// Shared-prefix attention: work planning, dispatch to the kernel families
// (shared_part.hip) and the kernel that joins a row's partials.

#include "shared_impl.h"

namespace kvq {

#define KVQ_FAMILY(D, KG) hipError_t launch_shared_##D##_##KG(const SharedParams& p, hipStream_t stream);
KVQ_FAMILY(64, 0) KVQ_FAMILY(64, 1) KVQ_FAMILY(64, 2)
KVQ_FAMILY(128, 0) KVQ_FAMILY(128, 1) KVQ_FAMILY(128, 2) KVQ_FAMILY(128, 4)
KVQ_FAMILY(256, 0) KVQ_FAMILY(256, 1) KVQ_FAMILY(256, 2) KVQ_FAMILY(256, 4) KVQ_FAMILY(256, 8)
#undef KVQ_FAMILY

namespace {

// Work items of a round: one image_kernel workgroup per CU, two direct_kernel
// workgroups (three or four: up to 20% slower).
constexpr int kImageRound = 256, kDirectRound = 512;
constexpr int kTile = 16;  // rows of an MFMA

int ceil_div(int a, int b)
{
    return (a + b - 1) / b;
}

// Key group size / 32, 0 for per-channel keys.
int key_groups(const AttnParams& a)
{
    return a.k_axis == KVQ_PER_CHANNEL ? 0 : a.k_group / 32;
}

// How a segment's rows are taken.
struct Kind {
    bool direct;
    int per, step, round;  // rows per item, blocks that a range is a multiple of, items of a round
    int most;              // direct: the work up to which it takes everything (all_direct), in 1024s
};

Kind direct_kind(int D, int kg, int bits, bool rot, bool fp16)
{
    const int tiles = shr::direct_tiles(D, kg, bits, rot, fp16);
    const int most = D == 256 ? 12 : tiles == 2 ? 64 : bits == 8 || fp16 ? 24 : 40;
    return {true, kTile * tiles, shr::kDirectWaves, kDirectRound, most};
}

Kind direct_kind(int D, const AttnParams& a)
{
    return direct_kind(D, key_groups(a), a.k_bits, a.rotate, a.ring > 0 || a.sink > 0);
}

Kind image_kind(int D, int rows)
{
    const int per = shr::item_rows(D), n16 = ceil_div(rows < per ? rows : per, 16);
    return {false, per, shr::waves(D) / shr::row_waves(D, n16), kImageRound, 0};
}

// Whether the direct kernel takes everything: `rows` the most that a unit of the
// prefix has, `work` the 32-token blocks of all 16-row tiles of both segments, k
// the direct kernel's.  It converts a block's codes once per one or two tiles, the
// image kernel once per 128 or 256 rows; but a call of that one has to pay a
// launch of its own, the conversion before its first product, the merge of a wave's
// partials and the join of more of them: 16 to 25 us.  Direct / image, us, at
// `work` in 1024s:
//     two tiles  D = 64    64 rows  29 / 37 (32)   256 rows  42 / 48 (64)   72 / 70 (128)
//                D = 128   64 rows  44 / 53 (32)   256 rows  71 / 77 (64)   98 / 94 (96)
//     one tile, no wide codes or fp16 tokens
//                D = 128, rotated   128 rows  52 / 57 (32)  72 / 68 (48)    256 rows  51 / 68 (32)  90 / 84 (64)
//                groups of 32       128 rows  58 / 72 (32)  81 / 88 (48)    256 rows  56 / 74 (32)  99 / 98 (64)
//     one tile   D = 128, per-channel keys   64 rows  40 / 44 (16)  52 / 51 (24)   256 rows  63 / 62 (32)
//                8 bits                      64 rows  32 / 32 (8)   62 / 51 (24)   256 rows  79 / 62 (32)
//                D = 64, 8 bits              64 rows  33 / 36 (32)                 256 rows  31 / 36 (32)  54 / 48 (64)
//                D = 256   64 rows  44 / 46 (8)   128 rows  49 / 52 (8)  69 / 62 (16)   256 rows  54 / 66 (9)
// Units of two tiles would leave most of an image kernel's waves idle: 32 rows of
// 8192 tokens, 8 prefixes, D = 256, 110 / 141 us.
bool all_direct(int rows, long long work, const Kind& k)
{
    return rows <= 2 * kTile || work <= k.most * 1024;
}

// Ranges that a segment of `tiles` tiles is cut into, at most.
int shared_splits(long long tiles, int round)
{
    return tiles > 0 && tiles < round ? (int)(round / tiles) : 1;
}

// Joins the partials of a row: D / 4 threads, four output channels each, take
// every J-th partial, J of them side by side,
//     O = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s,
// with a running M over batches of kJoinBatch; then their sums meet in LDS and a
// rotating format's rows are rotated back over the threads' registers (the
// normalized transform is its own inverse).  Bound by the latency of its loads:
// of 33 partials, 2048 rows at D = 128 take 10 us, 17 when one thread per
// four channels walks them and 12 when M is found in a pass before.
constexpr int kJoinThreads = 256, kJoinBatch = 4;

template <int D>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(SharedParams p, int J)
{
    constexpr int TR = D / 4, SLOTS = kJoinThreads / TR;  // threads of a row, rows J = 1 would take
    __shared__ __attribute__((aligned(16))) float x[SLOTS * D];
    __shared__ float2 xml[SLOTS];
    const int slot = threadIdx.x / TR, d = 4 * (threadIdx.x % TR);
    const int R = SLOTS / J, rl = slot % R, j = slot / R;
    const size_t row = (size_t)blockIdx.x * R + rl;
    const size_t at = row < p.rows ? row : p.rows - 1;
    const int S = p.S[0] + p.S[1];
    floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    float M = -INFINITY, L = 0.0f;
    const auto raise = [&](float m) {  // M to at least m
        if (m > M) {
            const float w = fast_exp2(M - m);
            acc *= w;
            L *= w;
            M = m;
        }
    };
    for (int s0 = j; s0 < S; s0 += kJoinBatch * J) {
        float2 ml[kJoinBatch];
        floatx4 o[kJoinBatch];
#pragma unroll
        for (int k = 0; k < kJoinBatch; ++k) {
            const size_t i = (size_t)min(s0 + k * J, S - 1) * p.rows + at;
            ml[k] = *(const float2*)(p.part_ml + 2 * i);
            o[k] = *(const floatx4*)(p.part_o + i * D + d);
        }
        float m = -INFINITY;
#pragma unroll
        for (int k = 0; k < kJoinBatch; ++k) {
            ml[k].x = s0 + k * J < S ? ml[k].x : -INFINITY;
            m = fmaxf(m, ml[k].x);
        }
        raise(m);
#pragma unroll
        for (int k = 0; k < kJoinBatch; ++k) {
            const float w = ml[k].x == -INFINITY ? 0.0f : fast_exp2(ml[k].x - M);
            acc += o[k] * w;
            L += ml[k].y * w;
        }
    }
    if (J > 1) {
        *(floatx4*)(x + slot * D + d) = acc;
        if (d == 0)
            xml[slot] = make_float2(M, L);
        __syncthreads();
        for (int k = 1; k < J && slot < R; ++k) {
            const float2 ml = xml[slot + k * R];
            raise(ml.x);
            const float w = ml.x == -INFINITY ? 0.0f : fast_exp2(ml.x - M);
            acc += *(const floatx4*)(x + (slot + k * R) * D + d) * w;
            L += ml.y * w;
        }
    }
    acc *= 1.0f / L;  // every row sees a token
    if (p.rotate) {
        const float a = acc[0] + acc[1], b = acc[0] - acc[1], c = acc[2] + acc[3], e = acc[2] - acc[3];
        acc = floatx4{a + c, b + e, a - c, b - e} * p.rot_c;
#pragma unroll
        for (int h = 1; h < TR; h <<= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float y = __shfl_xor(acc[i], h);
                acc[i] = threadIdx.x & h ? y - acc[i] : acc[i] + y;
            }
    }
    if (slot < R && row < p.rows)
        *(floatx4*)(p.out + row * D + d) = acc;
}

template <int D>
void launch_join(const SharedParams& p, hipStream_t stream)
{
    constexpr int SLOTS = kJoinThreads / (D / 4);
    const int S = p.S[0] + p.S[1];
    int J = 1;
    while (2 * J <= SLOTS && 4 * J <= S)
        J *= 2;
    const size_t R = SLOTS / J;
    launch_kernel(join_kernel<D>, dim3((unsigned)((p.rows + R - 1) / R)), dim3(kJoinThreads), 0, stream, p, J);
}

}  // namespace

// Each segment is cut into ranges for one round of its kernel's workgroups, a
// range a multiple of the blocks that a workgroup takes at a time.  When both
// segments go to one kernel the prefix' items, the longer ones, start first,
// and the suffix is cut for what they leave of their round: its later items
// begin where others end, and more of them only add their fixed cost (200 tokens
// after 2048, D = 64: 64 us with one range of a suffix, 76 with two).  If they
// leave nothing the suffix is a round of its own (512 tokens after 8192,
// D = 256: 389 us with one range of a suffix, 377 with two).  `kernels`: 0 by
// the rule above, 1 and 2 the direct and the image kernel only.
void shared_plan(SharedParams* p, int D, int B, int kernels)
{
    const AttnParams &a = p->seg[0], &b = p->seg[1];
    const auto blocks = [](const AttnParams& s) { return ceil_div(s.n_sink, 32) + ceil_div(s.n > 0 ? s.n : 0, 32); };
    const int nb[2] = {blocks(a), blocks(b)}, own = p->C * a.G;
    int most = 0;
    long long work = (long long)B * a.H * ceil_div(own, kTile) * nb[1];
    for (int g = 0; g < p->P; ++g) {
        const int rows = (p->first[g + 1] - p->first[g]) * own;
        most = rows > most ? rows : most;
        work += (long long)a.H * ceil_div(rows, kTile) * nb[0];
    }
    const Kind few = direct_kind(D, a);
    const bool direct = kernels ? kernels == 1 : all_direct(most, work, few);
    const Kind kind[2] = {direct ? few : image_kind(D, most),
                          direct || (!kernels && own <= 2 * kTile) ? few : image_kind(D, own)};
    p->tiles0 = 0;
    for (int g = 0; g < p->P; ++g) {
        p->tile0[g] = p->tiles0;
        p->tiles0 += a.H * ceil_div((p->first[g + 1] - p->first[g]) * p->C * a.G, kind[0].per);
    }
    p->tile0[p->P] = p->tiles0;
    const int tiles[2] = {p->tiles0, B * a.H * ceil_div(p->C * a.G, kind[1].per)};
    for (int k = 0; k < 2; ++k) {
        int round = kind[k].round;
        if (k && kind[1].direct == kind[0].direct && tiles[0] * p->S[0] < round)
            round -= tiles[0] * p->S[0];
        const int want = shared_splits(tiles[k], round), step = kind[k].step;
        p->bps[k] = nb[k] > 0 ? ceil_div(ceil_div(nb[k], want), step) * step : step;
        p->S[k] = ceil_div(nb[k], p->bps[k]);
    }
    p->items0 = tiles[0] * p->S[0];
    const int items1 = tiles[1] * p->S[1];
    p->image_items = (kind[0].direct ? 0 : p->items0) + (kind[1].direct ? 0 : items1);
    p->direct0 = p->image_items;
    p->direct_items = p->items0 + items1 - p->image_items;
}

size_t shared_partials_bound(int B, int H, int D, int C, int G)
{
    // A segment of `units` units of u rows is cut into S <= max(1, round / tiles)
    // ranges, its tiles never fewer than units ceil(u / per) (the groups' not fewer
    // than one group's of all rows): units u S <= max(units u, round min(u, per)).
    // Unlike S this does not fall as C grows.
    const auto segment = [&](size_t units, int u) {
        size_t most = units * u;
        for (const Kind& k : {image_kind(D, u), direct_kind(D, 2, 2, false, false)}) {
            const size_t cut = (size_t)k.round * (u < k.per ? u : k.per);
            most = cut > most ? cut : most;
        }
        return most;
    };
    return segment(H, B * C * G) + segment((size_t)B * H, C * G);
}

hipError_t launch_shared(const SharedParams& p, int D, hipStream_t stream)
{
    const AttnParams& a = p.seg[0];
    hipError_t e = hipErrorInvalidValue;
    switch (1000 * D + key_groups(a)) {
#define KVQ_FAMILY(D, KG)                           \
    case 1000 * D + KG:                             \
        e = launch_shared_##D##_##KG(p, stream);        \
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
