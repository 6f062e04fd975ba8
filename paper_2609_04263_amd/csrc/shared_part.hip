// Shared-prefix attention kernels of one head size (KVQ_PART_D), for plain or
// rotated queries (KVQ_PART_ROT): built once per pair, so that they compile in
// parallel.
#include "shared_impl.h"

#if !defined(KVQ_PART_D) || !defined(KVQ_PART_ROT)
#error "shared_part.hip is compiled once per family with KVQ_PART_D and KVQ_PART_ROT defined"
#endif

#define KVQ_CAT2(a, b, c) a##_##b##_##c
#define KVQ_CAT(a, b, c) KVQ_CAT2(a, b, c)

namespace kvq {

hipError_t KVQ_CAT(launch_shared, KVQ_PART_D, KVQ_PART_ROT)(const SharedParams& p, int items, hipStream_t stream)
{
    // 8-bit codes come as keys and values both
    return p.seg[0].k_bits == 8 ? shr::launch_groups<KVQ_PART_D, true, KVQ_PART_ROT != 0>(p, items, stream)
                                : shr::launch_groups<KVQ_PART_D, false, KVQ_PART_ROT != 0>(p, items, stream);
}

}  // namespace kvq
