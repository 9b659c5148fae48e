// Attention over the paged KV cache: the kernels for plain scores.
#include "mma_attention_kernels.h"

namespace mma {

hipError_t launch_attention(const AttnArgs& a, const AttnPlan& p, const OpsKind& k, hipStream_t stream) {
  return by_type(a, p, k, stream);
}

}  // namespace mma
