// Eviction from a cache by the weight that its slots have gathered: which slots
// stay, and their rows on the way to a smaller cache.
//
// The slots that stay are the first `sinks`, the last `recent`, and those of the
// largest weights between them, found by a radix select over an order key of the
// float (11, 11 and 10 bits, most significant first; a NaN lies below all, both
// zeros are one).  Ties go to the lowest slot.
//
// A workgroup holds a segment of 16384 slots' weights in registers, 16 a thread,
// and counts its keys' digits in LDS.  Up to one segment it finds all three digits
// and writes the slots by itself; else there is a launch for each digit, whose
// workgroups all add up what the one before counted, in the order of the segments,
// so that each knows how many slots before its own stay as well (of many segments a launch
// between the two adds up).  Weights of a
// kind have few exponents, so the first digit's counters are few: four of each,
// in neighbouring banks, for every fourth lane.
//
// Measured: 4096 slots 9.6 us in one launch, three rounds of count and scan; more slots
// 7.4 (8 x 8 rows of 32749) to 9.1 us (4 x 8 of 131072) for each of four launches, most
// of it the way from length to weights to counters; a workgroup with 32768 slots, 32 a
// thread, takes 57 us.  The copy of 8001 rows of 64 heads takes 101 to 114 us, 5.2 to 4.6
// TB/s read and written, that of 65536 of 32 heads 409 to 430: a copy's rate.
#include "bpc_internal.h"

namespace bpc {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kSelectThreads = 1024;
constexpr int kSelectBins = 2048;
constexpr int kSelectRounds = 16;
constexpr int kSegSlots = kSelectRounds * kSelectThreads;
constexpr int kCopies = 4;  // of each counter
// workspace of a segment: three digits' counts, then its state
constexpr int kSegWords = 3 * kSelectBins + 4;

__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);  // -0 + 0 = 0
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// ONE: all of it; else launch `pass` of four: it settles digit pass - 1, then
// counts digit `pass`, or (the last) writes the slots that stay.
template <bool ONE, int ROUNDS>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a, int pass) {
  constexpr int NW = kSelectThreads / 64;
  __shared__ __attribute__((aligned(16))) uint32_t hist[kSelectBins * kCopies];
  static_assert(__alignof__(hist) >= alignof(uint4), "cleared and read 16 bytes at a time");
  __shared__ int wave_tot[NW];
  __shared__ int found[4];
  __shared__ int2 wave_cnt[NW];
  const int segs = ONE ? 1 : a.segs;
  const int bh = ONE ? (int)blockIdx.x : (int)(blockIdx.x / (uint32_t)segs), seg = ONE ? 0 : (int)blockIdx.x - bh * segs;
  const int b = bh / a.Hkv, h = bh - b * a.Hkv, t = threadIdx.x;
  const int lane = t & 63, wid = __builtin_amdgcn_readfirstlane(t >> 6);
  // weights, state and length are on their way at once (the weights of all N slots are there)
  const float* w = a.weights + b * a.sw_b + h * a.sw_h;
  const int slot0 = seg * kSegSlots + wid * (ROUNDS * 64) + lane;
  float x[ROUNDS];
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    const int i = slot0 + 64 * j;
    x[j] = w[min(i, a.N - 1)];
  }
  const int n = a.lens[b];
  if (n < 0 || n > a.N) return;
  const int stay = min(n, a.keep);
  const bool all = n <= a.keep;
  const int lo = all ? n : a.sinks, hi = all ? n : n - a.recent;  // the slots between are chosen from
  const int m = all ? 0 : a.keep - a.sinks - a.recent;
  if (!ONE && pass < 3 && m == 0) return;
  // segments that hold slots of the sequence; the others have nothing to say
  const int used = ONE ? 1 : max(1, (n + kSegSlots - 1) / kSegSlots);
  if (seg >= used) return;

  auto shift_of = [](int p) { return p == 0 ? 21 : p == 1 ? 10 : 0; };
  auto mask_of = [](int p) { return p == 2 ? 1023u : 2047u; };
  uint32_t prefix = 0u, pmask = 0u;
  int need = m;      // slots of the key looked for and below, within the prefix
  int before = 0, ties = 0;  // slots of earlier segments above the prefix, and equal to the key
  uint32_t* counts = ONE ? nullptr : a.counts + ((int64_t)bh * segs) * kSegWords;
  uint32_t* state = ONE ? nullptr : counts + (int64_t)seg * kSegWords + 3 * kSelectBins;

  auto count = [&](int p) {
    const int shift = shift_of(p);
    const uint32_t mask = mask_of(p);
    uint4* zero = reinterpret_cast<uint4*>(hist);
#pragma unroll
    for (int i = 0; i < kSelectBins * kCopies / 4 / kSelectThreads; ++i) zero[t + i * kSelectThreads] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ROUNDS; ++j) {
      const int i = slot0 + 64 * j;
      const uint32_t k = weight_key(x[j]);
      if (i >= lo && i < hi && (k & pmask) == prefix)
        atomicAdd(&hist[((k >> shift) & mask) * kCopies + (lane & (kCopies - 1))], 1u);
    }
    __syncthreads();
  };
  // thread t's counters: the bins 2047 - 2t and 2046 - 2t
  auto counted = [&](int bin) {
    const uint4 c = *reinterpret_cast<const uint4*>(&hist[bin * kCopies]);
    return (int)(c.x + c.y + c.z + c.w);
  };
  const int bin_top = kSelectBins - 1 - 2 * t, bin_low = bin_top - 1;
  // digit p: the one in which the `need`th largest key lies
  auto settle = [&](int p) {
    int top = 0, low = 0, pre_top = 0, pre_low = 0;
    if (ONE) {
      top = counted(bin_top), low = counted(bin_low);
    } else {
      const uint32_t* c = counts + p * kSelectBins + bin_low;
      if (a.totals) {
        const uint2 v = *reinterpret_cast<const uint2*>(c + (int64_t)seg * kSegWords);
        const uint2 all = *reinterpret_cast<const uint2*>(a.totals + (int64_t)bh * kSelectBins + bin_low);
        pre_top = (int)v.y, pre_low = (int)v.x, top = (int)all.y, low = (int)all.x;
      } else {
#pragma unroll 8
        for (int s = 0; s < used; ++s) {
          const uint2 v = *reinterpret_cast<const uint2*>(c + (int64_t)s * kSegWords);
          if (s < seg) pre_top += (int)v.y, pre_low += (int)v.x;
          top += (int)v.y, low += (int)v.x;
        }
      }
    }
    if (t < 4) found[t] = 0;
    int total;
    const int above_top = block_exclusive_scan<kSelectThreads>(top + low, wave_tot, total), above_low = above_top + top;
    if (above_top < need && need <= above_top + top) found[0] = bin_top, found[1] = above_top, found[3] = pre_top;
    if (above_low < need && need <= above_low + low) found[0] = bin_low, found[1] = above_low, found[3] = pre_low;
    __syncthreads();
    const int digit = found[0];
    if (!ONE) {
      int pre = (bin_top > digit ? pre_top : 0) + (bin_low > digit ? pre_low : 0);
#pragma unroll
      for (int o = 32; o; o >>= 1) pre += __shfl_xor(pre, o, 64);
      if (lane == 0 && pre) atomicAdd(&found[2], pre);
      __syncthreads();
      before += found[2], ties = found[3];
    }
    prefix |= (uint32_t)digit << shift_of(p);
    pmask |= mask_of(p) << shift_of(p);
    need -= found[1];
    __syncthreads();
  };

  if (m > 0) {
    if (ONE) {
#pragma unroll 1
      for (int p = 0; p < 3; ++p) {
        count(p);
        settle(p);
      }
    } else {
      if (pass > 1) {
        prefix = state[0], need = (int)state[1], before = (int)state[2];
        pmask = ~0u << shift_of(pass - 2);
      }
      if (pass > 0) settle(pass - 1);
      if (pass < 3) {
        count(pass);
        *reinterpret_cast<uint2*>(counts + (int64_t)seg * kSegWords + pass * kSelectBins + bin_low) =
            make_uint2((uint32_t)counted(bin_low), (uint32_t)counted(bin_top));
        if (t == 0) state[0] = prefix, state[1] = (uint32_t)need, state[2] = (uint32_t)before;
        return;
      }
    }
  }

  // ---- the slots that stay, in order: `need` of those equal to the key ---------
  int32_t* kept = a.kept + (int64_t)bh * a.keep;
  float* wo = a.weights_out ? a.weights_out + b * a.swo_b + h * a.swo_h : nullptr;
  for (int64_t i = stay + seg * kSelectThreads + t; i < a.keep; i += used * kSelectThreads) kept[i] = -1;
  if (wo)
    for (int64_t i = stay + seg * kSelectThreads + t; i < a.cap; i += used * kSelectThreads) wo[i] = 0.f;
  int above = 0, equal = 0;  // in this wavefront
  if (m > 0) {
#pragma unroll
    for (int j = 0; j < ROUNDS; ++j) {
      const int i = slot0 + 64 * j;
      const bool in = i >= lo && i < hi;
      const uint32_t k = weight_key(x[j]);
      above += __popcll(__ballot(in && k > prefix)), equal += __popcll(__ballot(in && k == prefix));
    }
    if (lane == 0) wave_cnt[wid] = make_int2(above, equal);
    __syncthreads();
    above = before, equal = ties;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const int2 c = wave_cnt[v];
      if (v < wid) above += c.x, equal += c.y;
    }
  }
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    const int i = slot0 + 64 * j;
    bool mine = i < n && (i < lo || i >= hi);
    int rank = i < lo ? i : a.keep - (n - i);
    if (m > 0) {
      const bool in = i >= lo && i < hi;
      const uint32_t k = weight_key(x[j]);
      const bool more = in && k > prefix, same = in && k == prefix;
      const uint64_t mb = __ballot(more), sb = __ballot(same);
      const int a0 = above + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mb >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mb, 0u));
      const int e0 = equal + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(sb >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)sb, 0u));
      if (more || (same && e0 < need)) mine = true, rank = lo + a0 + min(e0, need);
      above += __popcll(mb), equal += __popcll(sb);
    }
    if (mine) {
      kept[rank] = i;
      if (wo) wo[rank] = x[j];
    }
  }
}

// Many segments: their counters of a digit added up once, a thread a counter, to those
// of the segments before each and of all.
constexpr int kTotalThreads = 256;
__global__ __launch_bounds__(kTotalThreads) void evict_totals_kernel(EvictArgs a, int pass) {
  constexpr int kBlocks = kSelectBins / kTotalThreads, R = 16;
  const int bh = (int)(blockIdx.x / kBlocks), bin = (int)(blockIdx.x % kBlocks) * kTotalThreads + threadIdx.x;
  const int n = a.lens[bh / a.Hkv];
  if (n <= a.keep || n > a.N || a.keep == a.sinks + a.recent) return;
  const int used = (n + kSegSlots - 1) / kSegSlots;
  uint32_t* c = a.counts + (int64_t)bh * a.segs * kSegWords + pass * kSelectBins + bin;
  uint32_t before = 0u;
  for (int s0 = 0; s0 < used; s0 += R) {
    uint32_t x[R];
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = c[(int64_t)min(s0 + i, used - 1) * kSegWords];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (s0 + i < used) c[(int64_t)(s0 + i) * kSegWords] = before, before += x[i];
    }
  }
  a.totals[(int64_t)bh * kSelectBins + bin] = before;
}

// The rows that stay.  A wavefront moves 16 of each tensor, 16 lanes a row, all
// under way at once; the 16 rows written lie in one page.
constexpr int kCopyRows = 16;
int64_t evict_blocks(int B, int Hkv, int keep) { return (int64_t)B * Hkv * ((keep + 4 * kCopyRows - 1) / (4 * kCopyRows)); }

__global__ __launch_bounds__(256) void evict_copy_kernel(EvictArgs a) {
  const int blocks = (a.keep + 4 * kCopyRows - 1) / (4 * kCopyRows);
  const int bh = (int)(blockIdx.x / (uint32_t)blocks), block = (int)blockIdx.x - bh * blocks, b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int base = (block * 4 + wid) * kCopyRows;
  if (base >= a.keep) return;
  const int part = lane & 15, row0 = base + (lane >> 4);
  const int32_t* kept = a.kept + (int64_t)bh * a.keep;
  constexpr int R = kCopyRows / 4;
  int slot[R];
#pragma unroll
  for (int i = 0; i < R; ++i) slot[i] = kept[min(row0 + 4 * i, a.keep - 1)];
  const int n = a.lens[b];
  const int stay = min(n, a.keep);
  if (n < 0 || n > a.N || base >= stay) return;
#pragma unroll
  for (int i = 0; i < R; ++i) slot[i] = max(slot[i], 0);  // (rows past the last one)
  int64_t page_out = b, at_out = row0;
  bool room = true;
  if (a.table_out) {
    page_out = a.table_out[b * a.sto_b + (base >> a.out_shift)], at_out = row0 & ((1 << a.out_shift) - 1);
    room = (uint64_t)page_out < (uint64_t)a.out_pages;
    if (!room) page_out = 0;
  }
  int64_t page[R], at[R];
  bool on[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    page[i] = b, at[i] = slot[i];
    on[i] = room && row0 + 4 * i < stay;
  }
  if (a.table) {
#pragma unroll
    for (int i = 0; i < R; ++i) page[i] = a.table[b * a.st_b + (slot[i] >> a.page_shift)];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      at[i] = slot[i] & ((1 << a.page_shift) - 1);
      const bool there = (uint64_t)page[i] < (uint64_t)a.num_pages;
      on[i] = on[i] && there, page[i] = there ? page[i] : 0;
    }
  }
  u32x4 kr[R], vr[R];
#pragma unroll
  for (int i = 0; i < R; ++i) kr[i] = *reinterpret_cast<const u32x4*>(a.K + page[i] * a.sK_b + h * a.sK_h + at[i] * a.sK_n + 8 * part);
#pragma unroll
  for (int i = 0; i < R; ++i) vr[i] = *reinterpret_cast<const u32x4*>(a.V + page[i] * a.sV_b + h * a.sV_h + at[i] * a.sV_n + 8 * part);
  if (a.codes && part < a.W) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (row0 + 4 * i < stay)
        a.codes_out[b * a.sCo_b + h * a.sCo_h + (int64_t)(row0 + 4 * i) * a.W + part] = a.codes[b * a.sC_b + h * a.sC_h + (int64_t)slot[i] * a.W + part];
    }
  }
  uint16_t* ko = a.K_out + page_out * a.sKo_b + h * a.sKo_h + at_out * a.sKo_n + 8 * part;
  uint16_t* vo = a.V_out + page_out * a.sVo_b + h * a.sVo_h + at_out * a.sVo_n + 8 * part;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (on[i]) {
      *reinterpret_cast<u32x4*>(ko + 4 * i * a.sKo_n) = kr[i];
      *reinterpret_cast<u32x4*>(vo + 4 * i * a.sVo_n) = vr[i];
    }
  }
}

int evict_segments(int N) { return (N + kSegSlots - 1) / kSegSlots; }

// Whether the segments' counters are added up by launches of their own.  Where each
// workgroup adds up all of them, the work grows with the square of the segments: 8, 32, 64,
// 128 and 256 segments of 8 heads take 38, 52, 110, 288 and 884 us, with three launches more
// 42, 53, 88, 156 and 286; of 32 heads 50, 169, 394 and 1321 (up to 128), and 54, 143, 250 and 510.
static bool evict_adds_up(int segs) { return segs >= 32; }

size_t evict_workspace(int B, int Hkv, int N) {
  const int segs = evict_segments(N);
  const size_t bh = (size_t)B * Hkv;
  return segs == 1 ? 0 : (bh * segs * kSegWords + (evict_adds_up(segs) ? bh * kSelectBins : 0)) * sizeof(uint32_t);
}

hipError_t launch_evict(EvictArgs a) {
  const int bh = a.B * a.Hkv;
  a.segs = evict_segments(a.N);
  if (a.segs == 1) {
    auto* f = a.N <= 4 * kSelectThreads ? evict_select_kernel<true, 4> : evict_select_kernel<true, kSelectRounds>;
    f<<<bh, kSelectThreads, 0, a.stream>>>(a, 0);
  } else {
    a.totals = evict_adds_up(a.segs) ? a.counts + (int64_t)bh * a.segs * kSegWords : nullptr;
    for (int pass = 0; pass < 4; ++pass) {
      evict_select_kernel<false, kSelectRounds><<<bh * a.segs, kSelectThreads, 0, a.stream>>>(a, pass);
      if (a.totals && pass < 3) evict_totals_kernel<<<bh * (kSelectBins / kTotalThreads), kTotalThreads, 0, a.stream>>>(a, pass);
    }
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  evict_copy_kernel<<<(unsigned)evict_blocks(a.B, a.Hkv, a.keep), 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

}  // namespace bpc
