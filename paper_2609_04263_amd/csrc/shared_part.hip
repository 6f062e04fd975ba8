// Shared-prefix attention kernels of one head size (KVQ_PART_D) and key
// grouping (KVQ_PART_KG: per-token group size / 32, 0 for per-channel keys):
// built once per pair, so that they compile in parallel.
#include "shared_impl.h"

#if !defined(KVQ_PART_D) || !defined(KVQ_PART_KG)
#error "shared_part.hip is compiled once per family with KVQ_PART_D and KVQ_PART_KG defined"
#endif

#define KVQ_CAT2(a, b, c) a##_##b##_##c
#define KVQ_CAT(a, b, c) KVQ_CAT2(a, b, c)

namespace kvq {

hipError_t KVQ_CAT(launch_shared, KVQ_PART_D, KVQ_PART_KG)(const SharedParams& p, hipStream_t stream)
{
    return shr::launch_family<KVQ_PART_D, KVQ_PART_KG>(p, stream);
}

}  // namespace kvq
