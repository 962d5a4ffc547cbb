// Dense attention of many query rows: a masked prefill, a tree of drafted
// tokens over a contiguous or paged cache, and a chunk of few new tokens over either
// (of many: chunk_rows_kernel).
//
// The G query heads of a KV head share its keys, so a row of the product is a
// (token, head) pair, r = t G + g, and 32 rows make a row block.  A wavefront
// computes, for 32 rows and tiles of 32 keys,
//   S^T = K Q^T   (32x32x16 bf16 MFMA: a lane holds 16 scores of ONE row)
//   O^T += V^T P^T
// with the softmax's running maximum and sum in that lane, so neither needs
// more than one exchange with the other half of the wavefront per tile.  The
// keys a lane holds in S^T are those its half supplies to the second product,
// so the probabilities go from the accumulators to bf16 operands in place;
// rounding them to bf16 (2^-9 relative each, averaged by the sum) is what lets
// both products run on the matrix cores.  Sums and statistics stay fp32.
//
// K and V tiles go from global memory to LDS without passing registers, double
// buffered.  A row of 256 bytes holds its sixteen 16-byte chunks at position
// chunk ^ swz(row): sixteen consecutive rows' equal chunks (the K operand) and
// four consecutive rows' neighbouring four chunks (the transposing reads that
// make the V operand) then lie in different banks.
//
// Where rows are many a SIMD's two wavefronts are in the same phase of a tile, so
// products and softmax run almost one after the other: 2 x 8192 causal tokens, 32
// heads, 1.04 ms, 1.05 PFLOP/s of visible pairs, matrix units busy 46 % of the cycles,
// other vector instructions 35 % and more; 512 queries over 65536 keys with a bias
// 0.57 ms, 41 and 50 %; capped scores (8001 tokens in documents, 0.19 ms, 0.55 PFLOP/s)
// 22 and 37 %, three of their instructions transcendental.  Where rows are few by
// memory (8 tokens over 16 x 131072 slots: 0.94 ms, 6.8 TB/s; one token over the last
// 16384 of 16 sequences' slots: 0.165 ms, 6.5 TB/s).
#pragma once
#include <math.h>

#include <atomic>
#include <type_traits>

#include "bpc_internal.h"

namespace bpc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr float kLog2e = 1.4426950408889634f;
// instruction kinds of __builtin_amdgcn_sched_group_barrier
constexpr int kSchedValu = 0x2, kSchedMfma = 0x8, kSchedLds = 0x100;
constexpr int kRowBytes = kHeadDim * 2;
constexpr int kBlockRows = 32;  // query rows of a wavefront
constexpr int kMaxSplits = 64;  // pieces of the key axis
constexpr float kFarScore = 0x1p24f;  // in log2: from here on fp32 holds no score to better than one

__device__ __forceinline__ uint32_t swz(uint32_t row) {
  return ((row & 3u) << 2) | ((row >> 2) & 3u);
}

__device__ __forceinline__ uint32_t cvt_pk_bf16(float lo, float hi) {
  bf16x2 p;
  p[0] = (__bf16)lo, p[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, p);
}

// maximum of a lane's value and that of the lane 32 away, in both
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ int wave_min(int x) { return wave_reduce_maxmin<false>(x); }
__device__ __forceinline__ int wave_max(int x) { return wave_reduce_maxmin<true>(x); }

// What a unit of the running maximum is in log2: capped scores are held in units
// of log2, others in those of the products, which need no multiplication.
template <bool CAP>
__device__ __forceinline__ float log2_units(float sm_scale) {
  return CAP ? 1.f : sm_scale * kLog2e;
}

// The reference point that a maximum m stands for, in log2: the rounded product
// m * unit, so that an exponent is one multiply-add away from a score.  Far from
// zero its rounding would take the largest score's exponential from one to any
// power of two, out of range in the end: there it is the product itself, and the
// difference of score and maximum comes first.
__device__ __forceinline__ bool far_from_zero(float m, float unit) { return fabsf(m * unit) > kFarScore; }
// From the reference point of b to that of a.
template <bool CAP>
__device__ __forceinline__ float reference_step(float a, float b, float unit) {
  if (CAP) return a - b;
  return far_from_zero(b, unit) ? (a - b) * unit : a * unit - b * unit;
}

// The natural logarithm of `sum` exponentials that count from the reference point
// of m; no exponentials: -inf.
constexpr float kLn2 = 0.6931471805599453f;
template <bool CAP>
__device__ __forceinline__ float log_of_sum(float m, float sum, float unit) {
  return sum == 0.f ? -INFINITY : (m * unit + __builtin_amdgcn_logf(sum)) * kLn2;
}

// a value equal in all lanes, in scalar registers
__device__ __forceinline__ uint64_t uniform64(uint64_t x) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)x) |
         (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32;
}
// 64 lanes' 16 bytes each, from `base` + their own offset to LDS at `dst` +
// 16 lane.  Written out because the compiler would otherwise wait for every
// such copy in flight before any LDS read; the kernel waits by itself (dma_wait).
// No register is written, so there is nothing in flight that the compiler does
// not know of but the LDS bytes, which it cannot touch before dma_wait.
// ONCE: bytes that need not stay in a cache, as no other workgroup reads them (but
// where sequences have pages in common).
template <bool ONCE>
__device__ __forceinline__ void dma16(const char* base, uint32_t off, uint32_t dst) {
  if (ONCE)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt"
                 :
                 : "v"(off), "s"(base), "s"(dst)
                 : "memory");
  else
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(off), "s"(base), "s"(dst)
                 : "memory");
}
template <int N>
__device__ __forceinline__ void dma_wait() {  // until at most N copies of this wavefront are in flight
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ void lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

// LDS at `at` + a constant, which goes into the instruction
template <typename T>
__device__ __forceinline__ T lds_read(uint32_t at, int offset) {
  return *(__attribute__((address_space(3))) T*)((lds_char*)at + offset);
}
// four rows' columns: lane i of each 16 gets column i of the 4 x 16 block whose
// row i / 4, columns 4 (i % 4) .. + 3 it addresses
__device__ __forceinline__ s16x4 lds_read_tr(uint32_t at, int offset) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)((lds_char*)at + offset));
}
// x, as a value that the compiler does not take apart again
__device__ __forceinline__ uint32_t opaque(uint32_t x) {
  asm("" : "+v"(x));
  return x;
}

// a value that every lane reads at the same address, through the scalar cache
// (a vector load would have to wait for the copies in flight before it)
__device__ __forceinline__ int32_t uniform_load(const int32_t* p) {
  return *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)p;
}

// The kernel's arguments, read again: what only the end of a kernel or a rare
// path needs would otherwise hold scalar registers through the loop.
typedef const __attribute__((address_space(4))) AttnArgs* LateArgs;
__device__ __forceinline__ LateArgs late_args() {
  LateArgs p = (LateArgs)__builtin_amdgcn_kernarg_segment_ptr();  // (the kernel's first argument)
  asm volatile("" : "+s"(p));
  return p;
}

// RB row blocks of 32 rows by KW groups of wavefronts that take alternate key
// tiles of KT keys; RB KW wavefronts.
enum AttnKind { kPrefill, kTree, kPagedTree, kChunk, kPagedChunk };
constexpr bool is_tree(AttnKind kind) { return kind == kTree || kind == kPagedTree; }
constexpr bool is_chunk(AttnKind kind) { return kind == kChunk || kind == kPagedChunk; }

// New tokens of sequence b, which stand at slots first .. first + the number
// returned - 1; 0 where these are not all below N.
template <typename Args>
__device__ __forceinline__ int chunk_tokens(const Args& a, int b, int first) {
  const int n = a.count ? min(max(uniform_load(a.count + b), 0), a.T) : a.T;
  return first < 0 || first > a.N - n ? 0 : n;
}

// The slots that rows row0 .. row0 + span - 1 of a chunk's `rows` see, in tiles of
// `keys`: all tiles up to slot `end`, but that those from the `near`th on are `gap`
// further on, past slots that lie behind the first ones and before every window.
struct ChunkSlots {
  int p0, p1, end, near, gap, tiles;
};
template <typename Args>
__device__ __forceinline__ ChunkSlots chunk_slots(const Args& a, const FastDiv& div_G, int first, int rows, int row0, int span, int keys) {
  ChunkSlots s;
  s.p0 = first + div_G.quotient(row0), s.p1 = first + div_G.quotient(min(rows, row0 + span) - 1);
  s.end = s.p1 + 1, s.near = s.gap = 0;
  if (a.window) {
    const int lo = max(0, s.p0 - a.window + 1);
    s.near = (min(a.sinks, lo) + keys - 1) / keys, s.gap = max(0, lo / keys - s.near);
  }
  s.tiles = (s.end + keys - 1) / keys - s.gap;
  return s;
}


template <int KW, int KT>
struct AttnShape {
  static constexpr int kTileBytes = KT * kRowBytes;    // K or V of a tile
  static constexpr int kLds = KW * 2 * 2 * kTileBytes;  // K and V, two buffers, per group
};

// LSE: the logarithm of each row's sum of exponentials is wanted.  It is of the
// exponentials before they are rounded, a sum of its own.
template <int RB, int KW, int KT, AttnKind KIND, bool CAP, bool BIAS, bool ONCE, bool LSE = false>
__global__ __launch_bounds__(RB* KW * 64, KW > 1 ? 1 : 2) void attn_kernel(AttnArgs a) {
  using S = AttnShape<KW, KT>;
  constexpr bool TREE = is_tree(KIND), CHUNK = is_chunk(KIND), paged = KIND == kPagedTree || KIND == kPagedChunk;
  constexpr int NB = KT / 32;   // 32-key blocks of a tile
  constexpr int RPW = KT / RB;  // rows of a tile's K (and V) that a wavefront copies
  static_assert(RPW % 4 == 0, "a copy moves four rows");
  extern __shared__ __attribute__((aligned(64))) char smem[];  // (the halves of V's operands are an exclusive or of 32 apart)
  __shared__ uint64_t odd_rows[2][RB * KW];
  __shared__ int draft_place[TREE && BIAS ? 64 : 1];
  // Consecutive workgroups go to different XCDs.  A prefill gives each XCD a run
  // of consecutive items, whose row blocks share their keys in its L2 (later row
  // blocks first: they see more keys).  In a tree only the row blocks of one
  // piece share keys, and the sequences' lengths differ: pieces go round the XCDs.
  const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3;
  int rb, piece;
  if (TREE || (CHUNK && a.rounds)) {
    const int round = a.div_nrb.quotient(turn);
    rb = turn - round * a.nrb, piece = round * 8 + xcd;
    if (piece * a.nrb >= a.items) return;
    if (CHUNK) rb = a.nrb - 1 - rb;
  } else {
    const int item = xcd * ((a.items + 7) >> 3) + turn;
    if (item >= a.items || turn >= (a.items + 7) >> 3) return;
    piece = a.div_nrb.quotient(item), rb = a.nrb - 1 - (item - piece * a.nrb);
  }
  // (a chunk's pieces begin with the first of every KV head, so that those that short
  // sequences do not have come to no XCD more than to others)
  const int whole = CHUNK ? a.div_bh.quotient(piece) : a.div_splits.quotient(piece);
  const int bh = CHUNK ? piece - whole * a.B * a.Hkv : whole, split = CHUNK ? whole : piece - bh * a.splits;
  const int b = a.div_Hkv.quotient(bh), h = bh - b * a.Hkv;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = wid / RB, rbw = wid % RB;
  const int half = lane >> 5, col = lane & 31;
  const int G = a.G;
  const int first = CHUNK ? uniform_load(a.lens + b) : 0;  // slot of a chunk's first token
  const int rows = (CHUNK ? chunk_tokens(a, b, first) : a.T) * G;
  const int wg_row0 = rb * RB * kBlockRows;
  if (CHUNK && wg_row0 >= rows) return;  // these rows stay as they are

  // ---- the keys that any row of the workgroup sees -------------------------
  int klo = 0, khi = 0, len = 0;
  int wg_all_lo = 0, wg_all_hi = 0;  // and those that every row sees
  int near = 0, gap = 0;
  if (TREE) {
    len = uniform_load(a.lens + b);
    if (len < 0 || len > a.N - a.T) return;  // no such sequence: its rows stay as they are
    khi = len + a.T;
    wg_all_hi = len;
  } else if (CHUNK) {
    const ChunkSlots s = chunk_slots(a, a.div_G, first, rows, wg_row0, RB * kBlockRows, KT);
    khi = s.end, wg_all_hi = s.p0 + 1, near = s.near, gap = s.gap;
    if (a.window) wg_all_lo = max(0, s.p1 - a.window + 1);
  } else {
    const int t0 = a.div_G.quotient(wg_row0), t1 = a.div_G.quotient(min(rows - 1, wg_row0 + RB * kBlockRows - 1));
    int lo = INT32_MAX, hi = 0, all_lo = 0, all_hi = INT32_MAX;
    for (int t = t0 + lane; t <= t1; t += 64) {
      const int f = a.key_begin ? max(a.key_begin[b * a.s_begin + t], 0) : 0;
      const int e = a.key_end ? min(a.key_end[b * a.s_end + t], a.N) : (int)min((int64_t)a.N, (int64_t)a.pos0 + t + 1);
      if (f < e) lo = min(lo, f), hi = max(hi, e);
      all_lo = max(all_lo, f), all_hi = min(all_hi, e);
    }
    klo = wave_min(lo), khi = wave_max(hi);
    wg_all_lo = wave_max(all_lo), wg_all_hi = wave_min(all_hi);
    if (klo >= khi) klo = khi = 0;
  }

  // ---- tiles of this workgroup ---------------------------------------------
  const int base0 = klo / KT * KT;
  const int total = (khi - base0 - gap * KT + KT * KW - 1) / (KT * KW);
  // Pieces of a chunk are of equal length, so that those of short sequences take
  // no longer than others; a prefill's and a tree's are as many for all rows.
  const int per = CHUNK ? a.unit : a.div_splits.quotient(total + a.splits - 1);
  const int it0 = split * per, it1 = min(total, it0 + per);
  if (CHUNK && it0 >= total) return;
  const bool joined = CHUNK ? total > per : a.splits > 1;  // a second launch joins this row block's pieces
  auto tile_key = [&](int it) {  // first key of a tile
    const int v = it * KW + grp;
    return CHUNK ? (v < near ? v : v + gap) * KT : base0 + v * KT;
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem;
  const uint32_t ldsK = lds0 + grp * 4 * S::kTileBytes, ldsV = ldsK + 2 * S::kTileBytes;

  const int32_t* table = paged ? a.table + b * a.st_b : nullptr;
  const char* Kb = reinterpret_cast<const char*>(a.K + (paged ? 0 : b * a.sK_b) + h * a.sK_h);
  const char* Vb = reinterpret_cast<const char*>(a.V + (paged ? 0 : b * a.sV_b) + h * a.sV_h);
  const int64_t kstep = a.sK_n * 2, vstep = a.sV_n * 2;
  const int pmask = (1 << a.page_shift) - 1;
  constexpr int RU = RPW < 16 ? RPW : 16;  // a wavefront copies rows in runs of RU, which no page border cuts
  const int r4 = lane >> 4;                // row within a copy's four
  uint32_t chunk[RU / 4], koff[RU / 4], voff[RU / 4];
#pragma unroll
  for (int i = 0; i < RU / 4; ++i) {
    chunk[i] = (((uint32_t)lane & 15u) ^ swz((uint32_t)(rbw * RPW + 4 * i + r4))) * 16;
    koff[i] = (4 * i + r4) * (uint32_t)kstep + chunk[i];
    voff[i] = (4 * i + r4) * (uint32_t)vstep + chunk[i];
  }
  // Pages of the next tile to be copied, one per 16 keys.
  // A page that is not in the pool hides its keys: pages_bad has a bit for each
  // such 16 keys of the tile copied last (page 0 is read in its place).
  constexpr int NP = KT / 16;
  uint32_t pages[NP], pages_bad = 0;
  auto look_up = [&](int it) {
    const int n0 = tile_key(it);
#pragma unroll
    for (int u = 0; u < NP; ++u) pages[u] = (uint32_t)uniform_load(table + (min(n0 + 16 * u, khi - 1) >> a.page_shift));
  };
  // A chunk's workgroups of several row blocks look up 64 entries at a time, a lane
  // each, a tile before they are needed: they lie in registers by then, where a
  // scalar load would be waited for in every tile (260 tokens of 2 requests behind a window
  // of 500 and 600 first slots, pages of 16: 43.0 -> 41.5 us; 257 of 3: 15.0 -> 14.7).
  constexpr bool AHEAD = CHUNK && paged && RB > 1;
  constexpr int kAhead = 64 / NP;  // tiles whose entries a wavefront holds
  uint32_t entry = 0, next_entry = 0;
  uint64_t entry_bad = 0;
  auto fetch_entries = [&](int it) {
    const int n = min(tile_key(it + lane / NP) + 16 * (lane % NP), khi - 1);
    next_entry = (uint32_t)table[n >> a.page_shift];
  };
  auto take_entries = [&]() {
    const bool bad = next_entry >= (uint32_t)a.num_pages;
    entry_bad = __ballot(bad), entry = bad ? 0u : next_entry;
  };
  auto issue = [&](int it, int buf) {
    const int n0 = tile_key(it) + rbw * RPW;
    const int held = (it - it0) % kAhead * NP;  // this tile's entries
    if (AHEAD) {
      pages_bad = (uint32_t)(entry_bad >> held) & ((1u << NP) - 1u);
    } else if (paged) {
      pages_bad = 0;
#pragma unroll
      for (int u = 0; u < NP; ++u) {
        if (pages[u] >= (uint32_t)a.num_pages) pages_bad |= 1u << u, pages[u] = 0;
      }
    }
#pragma unroll
    for (int u = 0; u < RPW / RU; ++u) {
      const int nu = min(n0 + RU * u, khi - 1);
      const char *kt, *vt;
      if (paged) {
        static_assert(!paged || RPW % 16 == 0 || 16 % RPW == 0, "a run of a wavefront's rows lies in one page entry");
        int64_t page;
        if (AHEAD) {
          page = (uint32_t)__builtin_amdgcn_readlane((int)entry, held + rbw * RPW / 16 + u);
        } else {
          page = pages[u];
#pragma unroll
          for (int w = 1; w < RB; ++w) page = rbw == w ? pages[(w * RPW) / 16 + u] : page;
        }
        kt = Kb + page * a.sK_b * 2 + (nu & pmask) * kstep;
        vt = Vb + page * a.sV_b * 2 + (nu & pmask) * vstep;
      } else {
        kt = Kb + nu * kstep, vt = Vb + nu * vstep;
      }
      kt = reinterpret_cast<const char*>(uniform64(reinterpret_cast<uint64_t>(kt)));
      vt = reinterpret_cast<const char*>(uniform64(reinterpret_cast<uint64_t>(vt)));
      const uint32_t dst = (uint32_t)buf * S::kTileBytes + (rbw * RPW + RU * u) * kRowBytes;
      const int last = khi - 1 - nu;  // last row that may be read, from kt and vt on
      if (last >= RU - 1) {
#pragma unroll
        for (int i = 0; i < RU / 4; ++i) {
          dma16<ONCE>(kt, koff[i], ldsK + dst + 4 * i * kRowBytes);
          dma16<ONCE>(vt, voff[i], ldsV + dst + 4 * i * kRowBytes);
        }
      } else {
#pragma unroll
        for (int i = 0; i < RU / 4; ++i) {
          const uint32_t r = min(4 * i + r4, last);
          dma16<ONCE>(kt, r * (uint32_t)kstep + chunk[i], ldsK + dst + 4 * i * kRowBytes);
          dma16<ONCE>(vt, r * (uint32_t)vstep + chunk[i], ldsV + dst + 4 * i * kRowBytes);
        }
      }
    }
  };
  constexpr int kCopies = 2 * (RPW / 4);  // copies a wavefront issues per tile

  if (AHEAD) fetch_entries(it0), take_entries();
  else if (paged && it0 < it1) look_up(it0);

  // ---- this lane's row ------------------------------------------------------
  const int row = wg_row0 + rbw * kBlockRows + col;
  const bool live = row < rows;
  const int t = live ? a.div_G.quotient(row) : 0, g = live ? row - t * G : 0;
  int lo = INT32_MIN, hi = INT32_MAX;  // rows past the last see everything: they never make a tile partial
  uint64_t sees = ~0ull;
  int place = 0;  // position, for the distance
  if (TREE) {
    hi = len;
    if (live) {
      const uint64_t all = a.T >= 64 ? ~0ull : (1ull << a.T) - 1;
      sees = (a.tree ? a.tree[b * a.s_tree + t] : (2ull << t) - 1) & all;
      place = len + __popcll(sees & ~(1ull << t));
    }
  } else if (CHUNK) {
    if (live) place = first + t, lo = a.window ? max(0, place - a.window + 1) : 0, hi = place + 1;
  } else if (live) {
    lo = a.key_begin ? max(a.key_begin[b * a.s_begin + t], 0) : 0;
    hi = a.key_end ? min(a.key_end[b * a.s_end + t], a.N) : (int)min((int64_t)a.N, (int64_t)a.pos0 + t + 1);
    // A bias counts from the nearest key that the row sees: what all of its keys
    // have in common falls out of the softmax, and would cost fp32 what they differ in.
    if (lo < hi) place = min(max(a.pos0 + t, lo), hi - 1);
  }
  // every row's keys cover [all_lo, all_hi); no row sees a key outside [any_lo, any_hi)
  int all_lo = 0, all_hi = len, any_lo = 0, any_hi = wg_row0 + rbw * kBlockRows < rows ? khi : 0;
  if (!TREE) {
    all_lo = wave_max(lo), all_hi = wave_min(hi);
    any_lo = wave_min(live && lo < hi ? lo : INT32_MAX), any_hi = wave_max(live && lo < hi ? hi : 0);
  }
  if (TREE && BIAS) {
    // the distance counts a draft at its depth in the tree
    if (threadIdx.x < a.T) {
      const int j = threadIdx.x;
      const uint64_t js = (a.tree ? a.tree[b * a.s_tree + j] : (2ull << j) - 1) & (a.T >= 64 ? ~0ull : (1ull << a.T) - 1);
      draft_place[j] = len + __popcll(js & ~(1ull << j));
    }
    __syncthreads();
  }
  // in units of log2 behind a cap, else of the products: the scale follows later
  const float slope = BIAS && live ? a.slopes[h * G + g] * (CAP ? kLog2e : 1.f / a.sm_scale) : 0.f;

  bf16x8 qf[8];
  {
    const uint16_t* qp = a.q + b * a.sq_b + (int64_t)(h * G + g) * a.sq_h + (int64_t)t * a.sq_t + 8 * half;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      u32x4 x = live ? *reinterpret_cast<const u32x4*>(qp + 16 * s) : u32x4{0, 0, 0, 0};
      qf[s] = __builtin_bit_cast(bf16x8, x);
    }
  }
  // the first tile is under way while the queries arrive
  if (it0 < it1) issue(it0, 0);
  if (RB == 1 && paged && it0 + 1 < it1) look_up(it0 + 1);
  // waited for here, not at their first use: a wait there would be one for the copies
#pragma unroll
  for (int s = 0; s < 8; ++s) asm volatile("" : "+v"(qf[s]));

  f32x16 o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) {
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  }
  // maximum, what a score has to exceed to move it, reference point (log2), sum
  float mrun = -INFINITY, limit = -INFINITY, mu = 0.f, lsum = 0.f;
  float esum = 0.f;  // LSE: the sum of the exponentials that were not rounded

  const uint32_t kswz = swz(col & 15) ^ half;
  uint32_t kaddr[8], vaddr[4];
#pragma unroll
  for (int s = 0; s < 8; ++s) kaddr[s] = ldsK + col * kRowBytes + ((2 * s) ^ kswz) * 16;
  {
    const int i16 = lane & 15, gd = r4 & 1;
    const uint32_t chunk = 2 * gd + ((i16 & 3) >> 1), f = swz(4 * half + (i16 >> 2));
#pragma unroll
    for (int d = 0; d < 4; ++d)
      vaddr[d] = ldsV + (4 * half + (i16 >> 2)) * kRowBytes + ((4 * d + chunk) ^ f) * 16 + (i16 & 1) * 8;
  }
  // Of the uncapped scores' units (the products') one is c1 in log2, 8 are c8.
  const float c1 = log2_units<CAP>(a.sm_scale), c8 = 8.f / c1;
  const float cap2 = a.softcap * kLog2e, capk = CAP ? 2.f * kLog2e * a.sm_scale / a.softcap : 0.f;

  auto compute = [&](int it, int buf, uint32_t bad, bool cleared, uint64_t odd) {
    const int n0 = tile_key(it);
    const bool sunk = CHUNK && n0 + KT <= a.sinks;  // a tile of slots that every later token sees
    if (n0 >= any_hi || (n0 + KT <= any_lo && !(CHUNK && n0 < a.sinks))) return;
    const bool full = (n0 >= all_lo || sunk) && n0 + KT <= all_hi && !bad;  // every row sees every key
    const uint32_t bo = buf * S::kTileBytes;
    uint32_t ka[8], va[4], vb[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) ka[i] = opaque(kaddr[i] + bo);
#pragma unroll
    for (int i = 0; i < 4; ++i) va[i] = opaque(vaddr[i] + bo), vb[i] = opaque(va[i] ^ 32u);
    f32x16 acc[NB];
#pragma unroll
    for (int k = 0; k < NB; ++k) {
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const bf16x8 kf = __builtin_bit_cast(bf16x8, lds_read<u32x4>(ka[s], k * 32 * kRowBytes));
        acc[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], s ? acc[k] : f32x16{}, 0, 0, 0);
      }
    }
    // the operand of a product is read four products ahead
    __builtin_amdgcn_sched_group_barrier(kSchedLds, 4, 0);
#pragma unroll
    for (int i = 0; i < 8 * NB - 4; ++i) {
      __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kSchedLds, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kSchedMfma, 4, 0);
    // key of score e of block k: n0 + 32 k + 8 (e / 4) + 4 half + e % 4
    const int nl = n0 + 4 * half;
    if (CAP || BIAS) {
      // (a distance beyond 2^24 is rounded to fp32 before it is weighed)
      const float ahead = (float)(place - nl);
      const bool drafts = TREE && BIAS && n0 + KT > len;
#pragma unroll
      for (int k = 0; k < NB; ++k) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int at = 32 * k + 8 * (e / 4) + e % 4;
          float z = acc[k][e];
          // in units of log2: cap tanh(x) = cap - 2 cap / (1 + e^2x)
          if (CAP) z = fmaf(-2.f * cap2, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * capk)), cap2);
          if (BIAS) {
            float dist = ahead - (float)at;
            if (TREE && drafts) {
              const uint32_t j = (uint32_t)(nl + at - len);
              if (j < (uint32_t)a.T) dist = (float)(place - draft_place[j]);
            }
            z = fmaf(-slope, fabsf(dist), z);
          }
          acc[k][e] = z;
        }
      }
    }
    auto visible = [&](int n) {
      if (!TREE) return (n >= lo || (CHUNK && n < a.sinks)) && n < hi;
      const uint32_t j = (uint32_t)(n - len);
      return n < len || (j < 64u && ((sees >> (j & 63u)) & 1u));
    };
    if (!full) {
#pragma unroll
      for (int k = 0; k < NB; ++k) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int n = nl + 32 * k + 8 * (e / 4) + e % 4;
          acc[k][e] = visible(n) && n < khi && !(paged && (bad >> (2 * k + e / 8) & 1)) ? acc[k][e] : -INFINITY;
        }
      }
    }
    float mt = acc[0][0];
#pragma unroll
    for (int k = 0; k < NB; ++k) {
#pragma unroll
      for (int e = 0; e < 16; ++e) mt = fmaxf(mt, acc[k][e]);
    }
    mt = max_halves(mt);
    // the reference point of the exponentials moves only when a score lies more
    // than 2^8 above it, so that the products are seldom rescaled; any point
    // gives the same quotient
    if (__any(mt > limit)) {
      const float mn = fmaxf(mrun, mt);
      const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(reference_step<CAP>(mrun, mn, c1));
      mrun = mn;
      lsum *= f;
      if (LSE) esum *= f;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] *= f;
      }
      limit = mn + (CAP ? 8.f : c8);
      const float ref = mn == -INFINITY ? 0.f : mn;
      mu = CAP ? ref : ref * c1;
      const bool far = !CAP && far_from_zero(ref, c1);
      if (__any(far)) {  // every tile of such a row comes this way
        if (far) limit = -INFINITY, mu = 0.f;
#pragma unroll
        for (int k = 0; k < NB; ++k) {
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[k][e] -= far ? ref : 0.f;
        }
      }
    }
    u32x4 pw[NB][2];
#pragma unroll
    for (int k = 0; k < NB; ++k) {
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        float p[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
          p[i] = __builtin_amdgcn_exp2f(CAP ? acc[k][e + i] - mu : fmaf(acc[k][e + i], c1, -mu));
        if (LSE) esum += p[0] + p[1];
        const bf16x2 pp = {(__bf16)p[0], (__bf16)p[1]};
        lsum = __builtin_amdgcn_fdot2_f32_bf16(pp, bf16x2{(__bf16)1.f, (__bf16)1.f}, lsum, false);
        pw[k][e / 8][e % 8 / 2] = __builtin_bit_cast(uint32_t, pp);
      }
    }
#pragma unroll
    for (int k = 0; k < NB; ++k) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const bf16x8 pf = __builtin_bit_cast(bf16x8, pw[k][s]);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          // keys 16 s + 4 half + j and 16 s + 8 + 4 half + j: the second lies eight
          // rows on, whose swizzle differs in bit 1
          const uint32_t at = (32 * k + 16 * s) * kRowBytes;
          const s16x8 vf = __builtin_shufflevector(lds_read_tr(va[d], at), lds_read_tr(vb[d], at + 8 * kRowBytes), 0, 1,
                                                   2, 3, 4, 5, 6, 7);
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf), pf, o[d], 0, 0, 0);
        }
      }
    }
    // V is read, and the next 16 keys' probabilities are computed, in the shadow
    // of the products
    __builtin_amdgcn_sched_group_barrier(kSchedLds, 8, 1);
    __builtin_amdgcn_sched_group_barrier(kSchedValu, 24, 1);
#pragma unroll
    for (int i = 0; i < 8 * NB; ++i) {
      __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 1);
      __builtin_amdgcn_sched_group_barrier(kSchedLds, 2, 1);
      __builtin_amdgcn_sched_group_barrier(kSchedValu, 5, 1);
    }
    if (cleared && RB > 1) {
      odd = 0;
#pragma unroll
      for (int w = 0; w < RB; ++w) odd |= odd_rows[buf][grp * RB + w];
      odd = uniform64(odd);
    }
    while (odd) {  // values of V that clear_odd() took out of the tile
      const int i = __ffsll((long long)odd) - 1, n = n0 + i;
      odd &= odd - 1;
      if (n >= khi) continue;
      const LateArgs la = late_args();
      const char* vr = Vb + n * la->sV_n * 2;
      if (paged) {
        const uint32_t pg = (uint32_t)uniform_load(table + (n >> la->page_shift));
        if (pg >= (uint32_t)la->num_pages) continue;
        vr = Vb + (pg * la->sV_b + (n & ((1 << la->page_shift) - 1)) * la->sV_n) * 2;
      }
      const bool see = visible(n);
#pragma unroll
      for (int c = 0; c < 16; ++c) {  // coordinates 8 c + 4 half + 0..3
        const u32x2 x = *reinterpret_cast<const u32x2*>(vr + 16 * c + 8 * half);
        const uint32_t w[4] = {x[0] << 16, x[0] & 0xFFFF0000u, x[1] << 16, x[1] & 0xFFFF0000u};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (see && (w[e] & 0x7F800000u) == 0x7F800000u) o[c / 4][4 * (c % 4) + e] += __uint_as_float(w[e]);
        // (else the compiler holds 64 masks at once, and the loop's scalars in vector registers)
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  // A key that a row does not see must not reach it through 0 * V either: where
  // some row sees only part of a tile, values of V that are not finite are
  // cleared, and added afterwards (from memory) to the rows that see them.  A
  // wavefront does this for the rows that it copied; the result has a bit for
  // each row of the tile that held such a value.
  auto clear_odd = [&](int buf) {
    uint64_t rows_odd = 0;
#pragma unroll
    for (int i = 0; i < RPW / 4; ++i) {
      const uint32_t at = ldsV + buf * S::kTileBytes + (rbw * RPW + 4 * i) * kRowBytes + 16 * lane;
      u32x4 x = lds_read<u32x4>(at, 0);
      uint32_t seen = 0;  // an exponent of all ones carries into bits 15 and 31
#pragma unroll
      for (int e = 0; e < 4; ++e) seen |= (x[e] & 0x7F807F80u) + 0x00800080u;
      seen &= 0x80008000u;
      const uint64_t lanes = __ballot(seen != 0);
      if (lanes) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if ((x[e] & 0x7F80u) == 0x7F80u) x[e] &= 0xFFFF0000u;
          if ((x[e] & 0x7F800000u) == 0x7F800000u) x[e] &= 0x0000FFFFu;
        }
        *(__attribute__((address_space(3))) u32x4*)(lds_char*)at = x;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if ((lanes >> (16 * r)) & 0xFFFFu) rows_odd |= 1ull << (rbw * RPW + 4 * i + r);
      }
    }
    return rows_odd;
  };

  for (int it = it0; it < it1; ++it) {
    const int buf = (it - it0) & 1;
    const uint32_t bad = pages_bad;  // of this tile: issue() turns to the next
    // (pages are looked up where copies are waited for: a scalar load in flight
    // would make every read of LDS wait for it)
    if (RB > 1) {
      if (paged && !AHEAD && it + 1 < it1) look_up(it + 1);
      dma_wait<0>();
    } else if (it + 1 < it1) {  // the other buffer is this wavefront's own: its next tile can be under way already
      issue(it + 1, buf ^ 1);
      if (paged && it + 2 < it1) look_up(it + 2);
      dma_wait<kCopies>();
    } else {
      dma_wait<0>();
    }
    const int n0 = tile_key(it);
    const bool partial = n0 + KT > wg_all_hi || (n0 < wg_all_lo && !(CHUNK && n0 + KT <= a.sinks)) || bad;
    uint64_t odd = 0;
    if (partial) {
      odd = clear_odd(buf);
      if (RB > 1 && lane == 0) odd_rows[buf][wid] = odd;
      lds_done();
    }
    if (RB > 1) {
      // past this point every wavefront's part of this tile is there, and no one
      // reads the other buffer any more
      __builtin_amdgcn_s_barrier();
      asm volatile("" : : : "memory");
      if (AHEAD && (it + 1 - it0) % kAhead == 0) take_entries();
      if (it + 1 < it1) issue(it + 1, buf ^ 1);
      if (AHEAD && (it + 2 - it0) % kAhead == 0) fetch_entries(it + 2);
    }
    asm volatile("" : : : "memory");
    compute(it, buf, bad, partial, odd);
    lds_done();  // the reads of this buffer, before it is filled again
  }

  // ---- results ---------------------------------------------------------------
  lsum = sum_halves(lsum);
  if (LSE) esum = sum_halves(esum);
  // coordinates 8 c + 4 half + 0..3 of this lane's row
  auto sums = [&](int c) { return make_float4(o[c / 4][4 * (c % 4)], o[c / 4][4 * (c % 4) + 1], o[c / 4][4 * (c % 4) + 2], o[c / 4][4 * (c % 4) + 3]); };
  constexpr int CW = 16 / KW;  // such groups of coordinates that a wavefront writes, from c0 on
  float4 res[CW];
  if (KW == 1) {
#pragma unroll
    for (int c = 0; c < CW; ++c) res[c] = sums(c);
  } else {
    // The groups of a row block join in LDS, each wavefront a quarter of the
    // coordinates: sums [group][c][half][row], then (max, sum) [group][row].
    static_assert(KW == 1 || RB == 1, "one row block");
    static_assert(KW * (16 * 2 * kBlockRows * (int)sizeof(float4) + kBlockRows * (int)(sizeof(float2) + sizeof(float))) <= S::kLds, "fits the tiles' LDS");
    float4* so = reinterpret_cast<float4*>(smem);
    float2* sm = reinterpret_cast<float2*>(so + KW * 16 * 2 * kBlockRows);
    float* se = reinterpret_cast<float*>(sm + KW * kBlockRows);
    const float unit = log2_units<CAP>(late_args()->sm_scale);
    __syncthreads();
#pragma unroll
    for (int c = 0; c < 16; ++c) so[((grp * 16 + c) * 2 + half) * kBlockRows + col] = sums(c);
    if (half == 0) sm[grp * kBlockRows + col] = make_float2(mrun, lsum);
    if (LSE && half == 0) se[grp * kBlockRows + col] = esum;
    __syncthreads();
    float2 st[KW];
    float mx = -INFINITY;
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      st[k] = sm[k * kBlockRows + col];
      mx = fmaxf(mx, st[k].x);
    }
    float tot = 0.f, f[KW];
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      f[k] = st[k].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(reference_step<CAP>(st[k].x, mx, unit));
      tot = fmaf(st[k].y, f[k], tot);
    }
    if (LSE) {
      esum = 0.f;
#pragma unroll
      for (int k = 0; k < KW; ++k) esum = fmaf(se[k * kBlockRows + col], f[k], esum);
    }
#pragma unroll
    for (int c = 0; c < CW; ++c) {
      res[c] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        const float4 x = so[((k * 16 + grp * CW + c) * 2 + half) * kBlockRows + col];
        res[c].x = fmaf(x.x, f[k], res[c].x), res[c].y = fmaf(x.y, f[k], res[c].y);
        res[c].z = fmaf(x.z, f[k], res[c].z), res[c].w = fmaf(x.w, f[k], res[c].w);
      }
    }
    mrun = mx, lsum = tot;
  }
  const LateArgs la = late_args();
  const int d0 = 8 * CW * (KW > 1 ? grp : 0) + 4 * half;
  const int end_row = (rb * RB + rbw) * kBlockRows + col, end_rows = la->T * la->G;
  if (end_row >= (CHUNK ? rows : end_rows)) return;
  if (joined) {
    const int64_t at = ((int64_t)bh * end_rows + end_row) * la->splits + split;
    if (d0 == 0) la->part_ml[at] = make_float2(mrun, lsum);
    if (LSE && d0 == 0) la->part_e[at] = esum;
    if (lsum == 0.f) return;
    float* po = la->part_o + at * kHeadDim + d0;
#pragma unroll
    for (int c = 0; c < CW; ++c) *reinterpret_cast<float4*>(po + 8 * c) = res[c];
    return;
  }
  const float inv = lsum == 0.f ? 0.f : 1.f / lsum;  // a row that sees no key: zeros
  const FastDiv by_G{la->div_G.mul, la->div_G.shift}, by_Hkv{la->div_Hkv.mul, la->div_Hkv.shift};
  const int end_t = by_G.quotient(end_row), end_b = by_Hkv.quotient(bh);
  const int head = (bh - end_b * la->Hkv) * la->G + end_row - end_t * la->G;
  uint16_t* op = la->out + end_b * la->so_b + head * la->so_h + end_t * la->so_t + d0;
  if (LSE && d0 == 0)
    la->lse[end_b * la->sl_b + head * la->sl_h + end_t] = log_of_sum<CAP>(mrun, esum, log2_units<CAP>(la->sm_scale));
#pragma unroll
  for (int c = 0; c < CW; ++c)
    *reinterpret_cast<uint2*>(op + 8 * c) =
        make_uint2(cvt_pk_bf16(res[c].x * inv, res[c].y * inv), cvt_pk_bf16(res[c].z * inv, res[c].w * inv));
}

// The splits of a row joined: a wavefront per row.  Lane s holds split s's
// (max, sum) and so its weight; then each half of the wavefront adds every other
// split's 128 sums, four coordinates per lane, four loads in flight.  (32 rows of
// 32 splits: 4 us; of 16 in one loop of dependent loads it was 11.)
static_assert(kMaxSplits <= 64, "a lane per split");
template <bool TREE, bool CHUNK = false, bool LSE = false>
__global__ __launch_bounds__(256) void attn_merge_kernel(AttnArgs a) {
  const int rows = a.T * a.G, lane = threadIdx.x & 63, half = lane >> 5, d = 4 * (lane & 31);
  const uint32_t r = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // (bh, t, g)
  const int bh = (int)(r / (uint32_t)rows);
  if (bh >= a.B * a.Hkv) return;
  const int row = (int)r - bh * rows, t = a.div_G.quotient(row), g = row - t * a.G;
  const int b = a.div_Hkv.quotient(bh), h = bh - b * a.Hkv;
  if (TREE) {
    const int len = uniform_load(a.lens + b);
    if (len < 0 || len > a.N - a.T) return;
  }
  int splits = a.splits;
  if (CHUNK) {
    const int first = uniform_load(a.lens + b), tokens = chunk_tokens(a, b, first), span = a.block_rows;
    if (t >= tokens) return;
    const ChunkSlots s = chunk_slots(a, a.div_G, first, tokens * a.G, row & -span, span, a.tile_keys);
    splits = (s.tiles + a.tile_group * a.unit - 1) / (a.tile_group * a.unit);
    if (splits == 1) return;
  }
  const float2* ml = a.part_ml + (int64_t)r * a.splits;
  const float* po = a.part_o + (int64_t)r * a.splits * kHeadDim + d;
  float2 mine = make_float2(-INFINITY, 0.f);
  if (lane < splits) mine = ml[lane];
  // a split that saw no key of this row has the sum 0, and its o was not written;
  // one whose weight is 0 beside the others' counts, for the NaN it may hold
  const uint64_t seen = __ballot(mine.y != 0.f);
  float mx = mine.y == 0.f ? -INFINITY : mine.x;
#pragma unroll
  for (int o = 32; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
  const float unit = a.softcap > 0.f ? log2_units<true>(a.sm_scale) : log2_units<false>(a.sm_scale);
  const float w = mine.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(reference_step<false>(mine.x, mx, unit));
  float tot = mine.y * w;
#pragma unroll
  for (int o = 32; o; o >>= 1) tot += __shfl_xor(tot, o, 64);
  if (LSE) {
    float e = mine.y == 0.f ? 0.f : a.part_e[(int64_t)r * a.splits + lane] * w;
#pragma unroll
    for (int o = 32; o; o >>= 1) e += __shfl_xor(e, o, 64);
    if (lane == 0) a.lse[b * a.sl_b + (int64_t)(h * a.G + g) * a.sl_h + t] = log_of_sum<false>(mx, e, unit);
  }
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = 0; s0 < splits; s0 += 8) {
    float4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = *reinterpret_cast<const float4*>(po + (int64_t)min(s0 + 2 * i + half, splits - 1) * kHeadDim);
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // (lanes from `splits` on have seen nothing)
      const float f = __shfl(w, (s0 + 2 * i + half) & 63, 64);
      const bool on = (seen >> ((s0 + 2 * i + half) & 63)) & 1;
      x.x = on ? fmaf(v[i].x, f, x.x) : x.x, x.y = on ? fmaf(v[i].y, f, x.y) : x.y;
      x.z = on ? fmaf(v[i].z, f, x.z) : x.z, x.w = on ? fmaf(v[i].w, f, x.w) : x.w;
    }
  }
  const float inv = tot == 0.f ? 0.f : 1.f / tot;
  x.x = sum_halves(x.x) * inv, x.y = sum_halves(x.y) * inv, x.z = sum_halves(x.z) * inv, x.w = sum_halves(x.w) * inv;
  uint16_t* op = a.out + b * a.so_b + (int64_t)(h * a.G + g) * a.so_h + (int64_t)t * a.so_t;
  if (half == 0) *reinterpret_cast<uint2*>(op + d) = make_uint2(cvt_pk_bf16(x.x, x.y), cvt_pk_bf16(x.z, x.w));
}

static hipError_t allow_lds(const void* f, int bytes, std::atomic<uint64_t>& allowed) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (allowed.load() & bit)) return hipSuccess;
  e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess && dev < 64) allowed.fetch_or(bit);
  return e;
}

template <int RB, int KW, int KT, AttnKind KIND, bool ONCE = false, bool LSE = false>
static hipError_t launch_attn_shape(AttnArgs a) {
  const int rows = a.T * a.G, nrb = (rows + RB * kBlockRows - 1) / (RB * kBlockRows);
  const int items = a.B * a.Hkv * nrb * a.splits;
  a.nrb = nrb, a.items = items, a.div_nrb = FastDiv::by(nrb);
  const int grid = is_tree(KIND) || (is_chunk(KIND) && a.rounds) ? (items / nrb + 7) / 8 * 8 * nrb : (items + 7) / 8 * 8;
#define BPC_ATTN(CAP, BIAS)                                                                                       \
  {                                                                                                               \
    auto* f = attn_kernel<RB, KW, KT, KIND, CAP, BIAS, ONCE, LSE>;                                                      \
    constexpr int lds = AttnShape<KW, KT>::kLds;                                                                  \
    static std::atomic<uint64_t> allowed{0}; /* devices on which the kernel may use that much LDS */               \
    if (hipError_t e = allow_lds(reinterpret_cast<const void*>(f), lds, allowed); e != hipSuccess) return e;      \
    f<<<grid, RB * KW * 64, lds, a.stream>>>(a);                                                      \
  }
  if (a.softcap > 0.f) {
    if (a.slopes) BPC_ATTN(true, true) else BPC_ATTN(true, false)
  } else {
    if (a.slopes) BPC_ATTN(false, true) else BPC_ATTN(false, false)
  }
#undef BPC_ATTN
  return hipGetLastError();
}

}  // namespace bpc
