// Prefill and tree attention: how their calls are cut, and their launches.
#include "attn_kernel.h"

namespace bpc {

// How a call is cut, by a model of its time (us) over the shapes and numbers of
// pieces S of the key axis.  A workgroup of a shape handles `keys` keys a step
// and `slots` of them are resident on the chip.  A round of workgroups costs 3,
// a step of 4 row blocks 1.5, or 2.1 where two workgroups share a compute unit,
// one of 8 row blocks 2.0 (these read each key once for twice the rows);
// a step of one row block (64 KiB of keys and values) 1.4 where neighbouring row
// blocks find them in L2, else 1.7, or the memory's 2.7 with every compute unit
// at it.  The join costs 2.5 and its partial results' way out and back.  Where
// there are several rounds, workgroups of fewer keys make room for others: a
// causal prefill's mean is less than its longest, ragged sequences' about 0.8.
// Measured, one row block against four, and S against its neighbours:
//   257 tokens, 8 heads (2 KV): 9.8 and 11.7 us; S = 2: 11.7
//   1024 tokens, 32 heads: 45.8 and 28.2 us; S = 2: 41.3
//   64 queries over 4096 keys: S = 4 of one row block 21.8, S = 16 of four 24.6
//   512 queries over 65536 keys: four row blocks 563, eight 530 us
//   4096 tokens, 32 heads: four row blocks 157, eight 147 us
//   4000 tokens, 4 heads (4 KV): S = 1 of one row block 69.5, S = 4 of four 47.8
//   512 queries over 16384 keys: S = 2, 4, 8: 180, 152, 159 us
//   one token over 4 x 4096 slots: S = 4, 8, 16: 22.9, 18.1, 24.0 us
//   24 drafts over 8 x 32768 slots: S = 4, 8, 16: 239, 168, 172 us
AttnPlan attn_plan(int B, int Hkv, int G, int T, int N, bool tree) {
  AttnPlan p{};
  const int64_t rows = (int64_t)T * G, bh = (int64_t)B * Hkv;
  double best = 0;
  for (int rb = 1; rb <= (tree ? 4 : 8); rb = rb == 1 ? 4 : 2 * rb) {
    if (rb > 1 && rows <= rb / 2 * kBlockRows) break;
    const int64_t nrb = (rows + rb * kBlockRows - 1) / (rb * kBlockRows);
    const int keys = rb == 1 ? 128 : 64, slots = rb == 4 ? 512 : 256;
    const int64_t steps = ((int64_t)N + keys - 1) / keys;
    for (int S = 1; S <= kMaxSplits && (S == 1 || S <= steps); S *= 2) {
      const double wgs = (double)(bh * nrb * S), full = wgs / slots;
      // a last round that is not full takes as long as another, at first
      const double rounds = full <= 1 ? 1 : full < 8 ? 0.5 * (full + ceil(full)) : full;
      const double step = rb == 8 ? 2.0 : rb == 4 ? (wgs > 256 ? 2.1 : 1.5) : nrb > 1 ? 1.4 : wgs > 161 ? 2.7 * (wgs < 256 ? wgs / 256 : 1) : 1.7;
      const double mean = rounds == 1 ? 1 : tree ? 0.8 : 1.2 - 0.5 * (T < N ? (double)T / N : 1);
      const double join = S == 1 ? 0 : 2.5 + (double)(bh * rows) * S * (2 * (kHeadDim + 2) * sizeof(float)) / 5e6;
      const double us = 3 + rounds * (3 + mean * (double)((steps + S - 1) / S) * step) + join;
      if (!p.rb || us < best) best = us, p.rb = rb, p.splits = S;
    }
  }
  // Keys that one row block reads, and more of them than the last-level cache
  // (256 MB) holds until the next call, pass it by.  One token over 16 sequences, 8 KV
  // heads, kept and streamed: 4096 slots (268 MB) 49.5 and 49.5 us, 5120 65.6 and
  // 60.7, 8192 104 and 89, 32768 377 and 325 (pages of 64: 52.3 and 52.0, 64.5 and
  // 61.3, 100 and 87, 363 and 323).  Of a cache that is filled in part, streaming what
  // would have fitted costs little: 2000 of 131072 slots 32.9 and 32.9, 4000 48.8 and
  // 50.4, 8000 104 and 85.  Several row blocks read each key again: 168 and 174 (16
  // tokens over 8 x 32768 slots), 1094 and 1116 (2 x 8192 causal tokens).
  p.once = rows <= kBlockRows && bh * N * (4 * kHeadDim) > (int64_t)320 << 20;
  size_t o = 0;
  auto take = [&](size_t bytes) {
    size_t at = o;
    o += (bytes + 255) / 256 * 256;
    return at;
  };
  if (p.splits > 1) {
    const size_t n = (size_t)(bh * rows) * p.splits;
    p.off_ml = take(n * sizeof(float2));
    p.off_o = take(n * kHeadDim * sizeof(float));
  }
  p.total = o;
  return p;
}

template <AttnKind KIND>
static hipError_t launch_attn_as(const AttnArgs& a, const AttnPlan& p) {
  hipError_t e;
  if (p.rb == 1) {
    e = p.once ? launch_attn_shape<1, 4, 32, KIND, true>(a) : launch_attn_shape<1, 4, 32, KIND>(a);
  } else if (KIND != kPrefill || p.rb == 4) {  // (a tree's plan has no eight)
    e = launch_attn_shape<4, 1, 64, KIND>(a);
  } else {
    e = launch_attn_shape<8, 1, 64, kPrefill>(a);
  }
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t rows = (int64_t)a.B * a.Hkv * a.T * a.G;
  attn_merge_kernel<KIND != kPrefill><<<(unsigned)((rows + 3) / 4), 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_attn(AttnArgs a, const AttnPlan& p) {
  a.div_G = FastDiv::by(a.G), a.div_Hkv = FastDiv::by(a.Hkv), a.div_splits = FastDiv::by(a.splits);
  return !a.lens ? launch_attn_as<kPrefill>(a, p) : a.table ? launch_attn_as<kPagedTree>(a, p) : launch_attn_as<kTree>(a, p);
}

}  // namespace bpc
