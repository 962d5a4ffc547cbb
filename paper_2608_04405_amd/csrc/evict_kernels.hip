// Eviction from a cache by the weight that its slots have gathered: which slots
// stay, and their rows on the way to a smaller cache.
//
// The slots that stay are the first `sinks`, the last `recent`, and those of the
// largest weights between them, found by a radix select over an order key of the
// float (11, 11 and 10 bits, most significant first; a NaN lies below all, both
// zeros are one).  Ties go to the lowest slot.
#include "bpc_internal.h"

namespace bpc {

constexpr int kSelectThreads = 1024;
constexpr int kSelectBins = 2048;

__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);  // -0 + 0 = 0
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t hist[kSelectBins];
  __shared__ int wave_tot[kSelectThreads / 64];
  __shared__ int found[2];
  const int bh = blockIdx.x, b = bh / a.Hkv, h = bh - b * a.Hkv, t = threadIdx.x;
  const int n = a.lens[b];
  if (n < 0 || n > a.N) return;
  const float* w = a.weights + b * a.sw_b + h * a.sw_h;
  int32_t* kept = a.kept + (int64_t)bh * a.keep;
  float* wo = a.weights_out ? a.weights_out + b * a.swo_b + h * a.swo_h : nullptr;
  const int stay = min(n, a.keep);
  for (int i = stay + t; i < a.keep; i += kSelectThreads) kept[i] = -1;
  if (wo)
    for (int i = stay + t; i < a.cap; i += kSelectThreads) wo[i] = 0.f;
  if (n <= a.keep) {
    for (int i = t; i < n; i += kSelectThreads) {
      kept[i] = i;
      if (wo) wo[i] = w[i];
    }
    return;
  }
  const int lo = a.sinks, hi = n - a.recent;
  const int m = a.keep - a.sinks - a.recent;  // of [lo, hi), which has more
  uint32_t prefix = 0u, pmask = 0u;
  int need = m;
  constexpr int kShift[3] = {21, 10, 0}, kBits[3] = {11, 11, 10};
  if (m > 0) {
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = kShift[pass];
      const uint32_t dmask = (1u << kBits[pass]) - 1u;
      hist[2 * t] = 0u, hist[2 * t + 1] = 0u;
      __syncthreads();
      for (int i = lo + t; i < hi; i += kSelectThreads) {
        const uint32_t k = weight_key(w[i]);
        if ((k & pmask) == prefix) atomicAdd(&hist[(k >> shift) & dmask], 1u);
      }
      __syncthreads();
      // thread t holds bins 2047 - 2t and 2046 - 2t: the scan counts the bins above
      const int top = (int)hist[kSelectBins - 1 - 2 * t], low = (int)hist[kSelectBins - 2 - 2 * t];
      int total;
      const int above_top = block_exclusive_scan<kSelectThreads>(top + low, wave_tot, total), above_low = above_top + top;
      if (above_top < need && need <= above_top + top) found[0] = kSelectBins - 1 - 2 * t, found[1] = above_top;
      if (above_low < need && need <= above_low + low) found[0] = kSelectBins - 2 - 2 * t, found[1] = above_low;
      __syncthreads();
      prefix |= (uint32_t)found[0] << shift;
      pmask |= dmask << shift;
      need -= found[1];
      __syncthreads();
    }
  }
  // `need` slots of weight `prefix`, the lowest first, and all above it
  int written = 0, ties = 0;
  for (int c0 = 0; c0 < n; c0 += kSelectThreads) {
    const int i = c0 + t;
    const bool inside = i < n, middle = i >= lo && i < hi;
    const float x = inside ? w[i] : 0.f;
    const uint32_t k = weight_key(x);
    const bool tie = m > 0 && inside && middle && k == prefix;
    const bool sure = inside && (!middle || (m > 0 && k > prefix));
    int tot;
    const int pre = block_exclusive_scan<kSelectThreads>(((int)tie << 16) | (int)sure, wave_tot, tot);
    const int rank_tie = ties + (pre >> 16);
    const int rank = written + (pre & 0xFFFF) + min(rank_tie, need) - min(ties, need);
    if (sure || (tie && rank_tie < need)) {
      kept[rank] = i;
      if (wo) wo[rank] = x;
    }
    written += (tot & 0xFFFF) + min(ties + (tot >> 16), need) - min(ties, need);
    ties += tot >> 16;
  }
}

// A wavefront copies rows four at a time, 16 lanes a row.
constexpr int kCopyRows = 16;  // of a wavefront
int64_t evict_blocks(int B, int Hkv, int keep) { return (int64_t)B * Hkv * ((keep + 4 * kCopyRows - 1) / (4 * kCopyRows)); }
__global__ __launch_bounds__(256) void evict_copy_kernel(EvictArgs a) {
  const int blocks = (a.keep + 4 * kCopyRows - 1) / (4 * kCopyRows);
  const int bh = blockIdx.x / blocks, block = blockIdx.x - bh * blocks, b = bh / a.Hkv, h = bh - b * a.Hkv;
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int n = a.lens[b];
  if (n < 0 || n > a.N) return;
  const int stay = min(n, a.keep);
  const int base = (block * 4 + wid) * kCopyRows;
  const int part = lane & 15, pmask = (1 << a.page_shift) - 1, omask = (1 << a.out_shift) - 1;
  const int32_t* kept = a.kept + (int64_t)bh * a.keep;
  uint4 kr[kCopyRows / 4], vr[kCopyRows / 4];
  bool on[kCopyRows / 4];
#pragma unroll
  for (int i = 0; i < kCopyRows / 4; ++i) {
    const int row = base + 4 * i + (lane >> 4);
    on[i] = row < stay;
    if (!on[i]) continue;
    const int s = kept[row];
    int64_t page = b, at = s;
    if (a.table) {
      page = a.table[b * a.st_b + (s >> a.page_shift)], at = s & pmask;
      if ((uint64_t)page >= (uint64_t)a.num_pages) on[i] = false;
    }
    if (on[i]) {
      kr[i] = *reinterpret_cast<const uint4*>(a.K + page * a.sK_b + h * a.sK_h + at * a.sK_n + 8 * part);
      vr[i] = *reinterpret_cast<const uint4*>(a.V + page * a.sV_b + h * a.sV_h + at * a.sV_n + 8 * part);
    }
    if (a.codes && part < a.W)
      a.codes_out[b * a.sCo_b + h * a.sCo_h + (int64_t)row * a.W + part] = a.codes[b * a.sC_b + h * a.sC_h + (int64_t)s * a.W + part];
  }
#pragma unroll
  for (int i = 0; i < kCopyRows / 4; ++i) {
    const int row = base + 4 * i + (lane >> 4);
    if (!on[i]) continue;
    int64_t page = b, at = row;
    if (a.table_out) {
      page = a.table_out[b * a.sto_b + (row >> a.out_shift)], at = row & omask;
      if ((uint64_t)page >= (uint64_t)a.out_pages) continue;
    }
    *reinterpret_cast<uint4*>(a.K_out + page * a.sKo_b + h * a.sKo_h + at * a.sKo_n + 8 * part) = kr[i];
    *reinterpret_cast<uint4*>(a.V_out + page * a.sVo_b + h * a.sVo_h + at * a.sVo_n + 8 * part) = vr[i];
  }
}

hipError_t launch_evict(const EvictArgs& a) {
  const int bh = a.B * a.Hkv;
  evict_select_kernel<<<bh, kSelectThreads, 0, a.stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  evict_copy_kernel<<<bh * ((a.keep + 4 * kCopyRows - 1) / (4 * kCopyRows)), 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

}  // namespace bpc
