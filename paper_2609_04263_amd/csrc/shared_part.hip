// Shared-prefix attention kernels of one head size (KVQ_PART_D) and key
// grouping (KVQ_PART_KG: per-token group size / 32, 0 for per-channel keys):
// built once per pair, so that they compile in parallel, and once more for the
// calls of drafted trees (KVQ_PART_TREE).
#include "shared_impl.h"

#if !defined(KVQ_PART_D) || !defined(KVQ_PART_KG)
#error "shared_part.hip is compiled once per family with KVQ_PART_D and KVQ_PART_KG defined"
#endif
#ifdef KVQ_PART_TREE
#define KVQ_LAUNCH launch_tree
#else
#define KVQ_LAUNCH launch_shared
#endif

#define KVQ_CAT2(a, b, c) a##_##b##_##c
#define KVQ_CAT(a, b, c) KVQ_CAT2(a, b, c)

namespace kvq {

hipError_t KVQ_CAT(KVQ_LAUNCH, KVQ_PART_D, KVQ_PART_KG)(const SharedParams& p, hipStream_t stream)
{
#ifdef KVQ_PART_TREE
    return shr::launch_family<KVQ_PART_D, KVQ_PART_KG, true>(p, stream);
#else
    return shr::launch_family<KVQ_PART_D, KVQ_PART_KG, false>(p, stream);
#endif
}

}  // namespace kvq
