// Attention over the paged KV cache: the kernels for capped scores, whatever else their shape has.
#include "mma_attention_kernels.h"

namespace mma {

hipError_t launch_attention_capped(const CappedArgs& a, const AttnPlan& p, const OpsKind& k, hipStream_t stream) {
  return by_type(a, p, k, stream);
}

}  // namespace mma
