// Launches of the attention of a chunk of new tokens, of one kind of cache.
#pragma once
#include "attn_kernel.h"

namespace bpc {

template <AttnKind KIND, bool LSE>
static hipError_t launch_chunk_lse(const AttnArgs& a, const AttnPlan& p) {
  hipError_t e;
  if (p.rb == 1) {
    e = p.once ? launch_attn_shape<1, 4, 32, KIND, true, LSE>(a) : launch_attn_shape<1, 4, 32, KIND, false, LSE>(a);
  } else if (p.rb == 4) {
    e = launch_attn_shape<4, 1, 64, KIND, false, LSE>(a);
  } else {
    e = launch_attn_shape<8, 1, 64, KIND, false, LSE>(a);
  }
  return e;
}

template <AttnKind KIND>
static hipError_t launch_chunk_as(const AttnArgs& a, const AttnPlan& p) {
  return a.lse ? launch_chunk_lse<KIND, true>(a, p) : launch_chunk_lse<KIND, false>(a, p);
}

}  // namespace bpc
