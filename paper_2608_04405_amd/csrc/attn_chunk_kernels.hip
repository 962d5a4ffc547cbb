// Attention of a chunk of new tokens over a contiguous cache, the cut of its calls
// over either cache, and the join of their pieces.
#include <algorithm>

#include "attn_chunk.h"

namespace bpc {

// The model of a prefill over the slots that a workgroup's rows see.
AttnPlan chunk_plan(int B, int Hkv, int G, int T, int N, int window, int sinks) {
  if (window) N = (int)std::min<int64_t>(N, (int64_t)window + sinks + std::min(T, 256 / G));
  AttnPlan p = attn_plan(B, Hkv, G, T, N, false);
  if (p.splits > 1) {
    p.off_e = p.total;
    p.total += ((size_t)B * Hkv * T * G * p.splits * sizeof(float) + 255) / 256 * 256;
  }
  return p;
}

hipError_t launch_chunk(AttnArgs a, const AttnPlan& p) {
  a.div_G = FastDiv::by(a.G), a.div_Hkv = FastDiv::by(a.Hkv), a.div_splits = FastDiv::by(a.splits);
  const int pieces = a.B * a.Hkv * a.splits;
  a.rounds = pieces % 8 == 0 || pieces >= 32;
  const hipError_t e = a.table ? launch_chunk_paged(a, p) : launch_chunk_as<kChunk>(a, p);
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t rows = (int64_t)a.B * a.Hkv * a.T * a.G;
  auto* join = a.lse ? attn_merge_kernel<false, true, true> : attn_merge_kernel<false, true, false>;
  join<<<(unsigned)((rows + 3) / 4), 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

}  // namespace bpc
