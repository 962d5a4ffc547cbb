// Attention of a chunk of new tokens over a paged cache.
#include "attn_chunk.h"

namespace bpc {

hipError_t launch_chunk_paged(const AttnArgs& a, const AttnPlan& p) { return launch_chunk_as<kPagedChunk>(a, p); }

}  // namespace bpc
