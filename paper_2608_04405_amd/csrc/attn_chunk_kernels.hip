// Attention of a chunk of new tokens over a contiguous cache, the cut of its calls
// over either cache, and the join of their pieces.
#include <algorithm>

#include "attn_chunk.h"

namespace bpc {

// Pieces go round the XCDs where each gets as many, or nearly, so that long sequences'
// pieces do not come to one; else each XCD gets a run of row blocks.
static bool pieces_go_round(int64_t pieces) { return pieces % 8 == 0 || pieces >= 32; }

// How a call is cut, by a model of its time (us) over the shapes and the lengths of
// a piece: row blocks of 32 rows a workgroup, steps (tiles, or groups of four) of a
// piece.  A round of workgroups costs 3, a step of one, four or eight row blocks as in
// the comment of attn_plan but for the last, 1.95; with several sequences whose
// pieces go round the XCDs a quarter of the work is taken to be missing (some are
// shorter than the longest, where no window makes them alike), and pieces fill up each
// other's rounds.  The join costs 2.5 and its partial results' way out
// and back.  Measured (us; S: pieces of the longest sequence; lengths from half of the
// longest up; * the choice):
//   2048 tokens of 2 requests over 32768 slots: eight row blocks 1430, 1469, 1371, 1316*,
//   1326, 1378 with S = 1 to 6, four 1423, 1457, 1412 with S = 1, 2, 4
//   1000 tokens of 2 requests over 16384 slots, cap and bias: eight 636, 643, 474, 517*, 478,
//   494, four 456, 540, 462: where the last round ends depends on lengths that are not
//   known here, and decides more than the model's terms
//   1000 tokens of 4 requests over 16384 slots: eight 692, 725, 692*, 722, 730, 737, four 725, 668, 665
//   512 tokens of 4 requests over 8192 slots: eight 229*, 252, 223, 222, 242, 238, four 196, 228, 209
//   257 tokens of 3 requests: one row block 23.0, four 14.7*, eight 20.5
//   one token, window 4096: S = 4, 17*: 20.5, 12.9
// The quarter is a guess about lengths.  Without it the first two calls take S = 1: 1430
// and 636, 9 and 23 % more.  Requests that are all as long as the longest pay for it: these
// calls take 2176 and 740 us with S = 4, 2060 and 685 with S = 1; the third 1130 and 1041;
// the fourth has S = 1 in both.
AttnPlan chunk_plan(int B, int Hkv, int G, int T, int N, int window, int sinks) {
  AttnPlan p{};
  const int64_t rows = (int64_t)T * G, bh = (int64_t)B * Hkv;
  double best = 0;
  int64_t best_pieces = 1;
  // (as in attn_plan; of a window's slots only those are read)
  const int64_t seen = window ? std::min<int64_t>(N, (int64_t)window + sinks + T) : N;
  const bool ragged = B > 1 && 2 * seen > N;
  for (int rb = 1; rb <= 8; rb = rb == 1 ? 4 : 2 * rb) {
    if (rb > 1 && rows <= rb / 2 * kBlockRows) break;
    const int64_t nrb = (rows + rb * kBlockRows - 1) / (rb * kBlockRows);
    const int slots = rb == 4 ? 512 : 256;
    // the most steps of a row block
    const int64_t keys = rb == 1 ? 32 : 64, group = rb == 1 ? 4 : 1;
    int64_t tiles = (N + keys - 1) / keys;
    if (window) tiles = std::min(tiles, (sinks + keys - 1) / keys + ((int64_t)window + std::min<int64_t>(T, (rb * 32 + G - 1) / G + 1)) / keys + 2);
    const int64_t steps = (tiles + group - 1) / group;
    for (int64_t want = 1; want <= kMaxSplits && want <= steps; ++want) {
      const int64_t unit = (steps + want - 1) / want, pieces = (steps + unit - 1) / unit;
      if (pieces != want) continue;
      const double wgs = (double)(bh * nrb * pieces);
      const bool spread = pieces_go_round(bh * pieces);
      const double full = (double)(spread ? (bh * pieces + 7) / 8 * nrb : (bh * pieces * nrb + 7) / 8) / (slots / 8);
      const double busy = ragged ? 0.75 * wgs : wgs;
      const double step = rb == 8 ? 1.95 : rb == 4 ? (wgs > 256 ? 2.1 : 1.5) : nrb > 1 ? 1.4 : busy > 161 ? 2.7 * (busy < 256 ? busy / 256 : 1) : 1.7;
      // rounds of workgroups; a last one that is not full takes as long as another
      double rounds = full <= 1 ? 1 : full < 8 ? ceil(full) : full;
      if (ragged && spread && full > 1) rounds = std::max(1.0, 0.75 * full + 0.5);
      const double mean = rounds <= 1 || window ? 1 : 1.2 - 0.5 * (T < N ? (double)T / N : 1);
      const double join = pieces == 1 ? 0 : 2.5 + (ragged ? 0.75 : 1) * (double)(bh * rows) * pieces * (2 * (kHeadDim + 2) * sizeof(float)) / 4e6;
      const double us = 3 + rounds * (3 + std::min(mean, 1.0) * (double)unit * step) + join;
      if (!p.rb || us < best) best = us, p.rb = rb, p.unit = (int)unit, best_pieces = pieces;
    }
  }
  p.splits = (int)best_pieces;
  p.once = rows <= kBlockRows && bh * seen * (4 * kHeadDim) > (int64_t)320 << 20;
  if (p.splits > 1) {
    const size_t n = (size_t)(bh * rows) * p.splits;
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
  a.div_G = FastDiv::by(a.G), a.div_Hkv = FastDiv::by(a.Hkv), a.div_bh = FastDiv::by(a.B * a.Hkv);
  a.unit = p.unit, a.tile_keys = p.rb == 1 ? 32 : 64, a.tile_group = p.rb == 1 ? 4 : 1, a.block_rows = p.rb * kBlockRows;
  a.rounds = pieces_go_round((int64_t)a.B * a.Hkv * a.splits);
  const hipError_t e = a.table ? launch_chunk_paged(a, p) : launch_chunk_as<kChunk>(a, p);
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t rows = (int64_t)a.B * a.Hkv * a.T * a.G;
  auto* join = a.lse ? attn_merge_kernel<false, true, true> : attn_merge_kernel<false, true, false>;
  join<<<(unsigned)((rows + 3) / 4), 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

}  // namespace bpc
