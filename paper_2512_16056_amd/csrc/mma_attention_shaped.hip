// Attention over the paged KV cache: the kernels for scores that are biased by distance, kept to a window, or seen both ways in
// a prefix. A file of its own, as the capped ones have, so that all sets are compiled side by side.
#include "mma_attention_kernels.h"

namespace mma {

hipError_t launch_attention_shaped(const ShapedArgs& a, const AttnPlan& p, const OpsKind& k, hipStream_t stream) {
  return by_type(a, p, k, stream);
}

}  // namespace mma
