// Copying whole sequences of a packed cache (kvq_cache_gather): forking a
// prompt's cache, reordering beams, moving the survivors of a batch together.
//
// A sequence's live bytes are at the same offsets within each (sequence, KV
// head) slab of every section, so the copy is a set of columns: 16 bytes at
// one offset of one head, taken through the list of (source, destination)
// sequences.  One thread owns a column for the operations it is given: it
// loads the column of up to kGatherBatch sources, then stores them, so
// operations of one batch may overwrite each other's sources (a cycle of up
// to kGatherBatch sequences is one batch).  The host orders dependent
// operations (kvq_cache_gather in kvq_api.cpp); a thread's own accesses to
// one address are performed in program order, so they need no barrier and no
// staging memory, and the copy can run in place.  Batches that do not depend
// on each other go to different workgroups (grid y).
//
// Bound by HBM: every distinct source is read once (operations of one source
// are adjacent and share the load), every destination written once.

#include "kvq_device.h"
#include "kvq_internal.h"

namespace kvq {
namespace {

constexpr int kGatherThreads = 256;

__global__ __launch_bounds__(kGatherThreads) void gather_kernel(GatherParams p)
{
    // the span of this workgroup (uniform)
    int k = 0;
    while (k + 1 < p.spans && (int)blockIdx.x >= p.span[k + 1].wg0)
        ++k;
    const GatherSpan sp = p.span[k];
    const uint32_t w = blockIdx.x - sp.wg0, h = w / sp.wgs;
    const size_t c = (size_t)(w - h * sp.wgs) * kGatherThreads + threadIdx.x, o = 16 * c;
    if (c >= sp.len16)
        return;
    const uint8_t* src = p.src + sp.src_off + h * sp.src_stride + o;
    uint8_t* dst = p.dst + sp.dst_off + h * sp.dst_stride + o;
    const size_t src_row = sp.src_stride * p.H, dst_row = sp.dst_stride * p.H;
    for (int b = blockIdx.y; b < p.batches; b += gridDim.y) {
        const GatherOp* op = p.op + b * kGatherBatch;
        u32x4 v[kGatherBatch];
#pragma unroll
        for (int i = 0; i < kGatherBatch; ++i) {
            if (op[i].dst < 0)
                continue;
            if (i > 0 && op[i].src == op[i > 0 ? i - 1 : 0].src)
                v[i] = v[i > 0 ? i - 1 : 0];
            else
                v[i] = *(const u32x4*)(src + (size_t)op[i].src * src_row);
        }
#pragma unroll
        for (int i = 0; i < kGatherBatch; ++i)
            if (op[i].dst >= 0)
                *(u32x4*)(dst + (size_t)op[i].dst * dst_row) = v[i];
    }
}

}  // namespace

hipError_t launch_gather(GatherParams p, bool ordered, hipStream_t stream)
{
    int wgs = 0;
    for (int k = 0; k < p.spans; ++k) {
        p.span[k].wg0 = wgs;
        p.span[k].wgs = (uint32_t)((p.span[k].len16 + kGatherThreads - 1) / kGatherThreads);
        wgs += (int)p.span[k].wgs * p.H;
    }
    launch_kernel(gather_kernel, dim3(wgs, ordered ? 1 : p.batches), dim3(kGatherThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace kvq
