// Attention of a chunk of new tokens over a contiguous cache, the cut of its calls
// over either cache, and the join of their pieces.
#include <algorithm>

#include "attn_chunk.h"

namespace bpc {

// The model of a prefill over the slots that a workgroup's rows see.
AttnPlan chunk_plan(int B, int Hkv, int G, int T, int N, int window, int sinks) {
  const int64_t all = N;
  if (window) N = (int)std::min<int64_t>(N, (int64_t)window + sinks + std::min(T, 256 / G));
  AttnPlan p = attn_plan(B, Hkv, G, T, N, false);
  if (getenv("BPC_RB") && atoi(getenv("BPC_RB"))) p.rb = atoi(getenv("BPC_RB"));
  if (getenv("BPC_S") && atoi(getenv("BPC_S"))) p.splits = atoi(getenv("BPC_S"));
  // the most steps of a row block
  const int64_t keys = p.rb == 1 ? 32 : 64, group = p.rb == 1 ? 4 : 1;
  int64_t tiles = (all + keys - 1) / keys;
  if (window) tiles = std::min(tiles, (sinks + keys - 1) / keys + ((int64_t)window + std::min<int64_t>(T, (p.rb * 32 + G - 1) / G + 1)) / keys + 2);
  const int64_t steps = (tiles + group - 1) / group;
  p.unit = (int)((steps + p.splits - 1) / p.splits);
  p.splits = (int)((steps + p.unit - 1) / p.unit);
  p.total = 0;
  if (p.splits > 1) {
    const size_t n = (size_t)B * Hkv * T * G * p.splits;
    auto take = [&](size_t bytes) {
      const size_t at = p.total;
      p.total += (bytes + 255) / 256 * 256;
      return at;
    };
    p.off_ml = take(n * sizeof(float2));
    p.off_e = take(n * sizeof(float));
    p.off_o = take(n * kHeadDim * sizeof(float));
  }
  return p;
}

hipError_t launch_chunk(AttnArgs a, const AttnPlan& p) {
  a.div_G = FastDiv::by(a.G), a.div_Hkv = FastDiv::by(a.Hkv), a.div_splits = FastDiv::by(a.splits);
  const int pieces = a.B * a.Hkv * a.splits;
  a.unit = p.unit, a.tile_keys = p.rb == 1 ? 32 : 64, a.tile_group = p.rb == 1 ? 4 : 1, a.block_rows = p.rb * kBlockRows;
  a.rounds = pieces % 8 == 0 || pieces >= 32;
  const hipError_t e = a.table ? launch_chunk_paged(a, p) : launch_chunk_as<kChunk>(a, p);
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t rows = (int64_t)a.B * a.Hkv * a.T * a.G;
  auto* join = a.lse ? attn_merge_kernel<false, true, true> : attn_merge_kernel<false, true, false>;
  join<<<(unsigned)((rows + 3) / 4), 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

}  // namespace bpc
