// The attention weight that each cached slot gathers from a chunk of tokens:
// w_n = decay w_n + sum over the (token, head) pairs r of a KV head of
// exp(s_rn - lse_r), s = Q K^T as in the attention of the same chunk.
//
// The sum runs over rows, so the product is taken the other way round than the
// attention takes it: S = Q K^T with 32x32x16 bf16 MFMA, rows of Q as the first
// operand, and a lane holds 16 rows' scores of ONE key, which it adds up by
// itself.  A wavefront keeps its keys (32 or 64) in registers for the whole call
// and the rows come by in tiles of 64 through LDS, so that every key is read once
// and no two wavefronts add to the same weight: the result does not depend on the
// order of workgroups.  Scores, exponentials and sums are fp32; the sum over tiles
// carries its rounding errors along (Knuth's two-sum), as there may be 10^5 rows.
//
// Keys come by way of LDS too, 32 of a wavefront at a time in the buffers that the
// rows' tiles use afterwards: a load straight into the operand's layout touches 32
// lines of 128 bytes for 16 bytes of each, four times over, and streamed 4.2 TB/s.
//
// Up to 64 rows (a step, a few drafts) it is the rows that stay in registers, and each
// wavefront runs through keys of its own, 32 at a time, the next on their way.
//
// Measured with 32 heads (8 KV heads): 500 tokens of 2 requests over 32768 slots 0.20 ms,
// 0.78 PFLOP/s of visible pairs, matrix units busy 33 % of the cycles, other vector
// instructions 35 to 43 % (an exponential, a multiply-add and an addition a score; with
// them spread evenly over the products it took as long); one token over 16 x 65536 slots 0.30 ms, 5.5 TB/s
// (6.2 to 6.8 where no weight is written: reads and writes take turns at the memory).
#include <algorithm>

#include "attn_kernel.h"

namespace bpc {

constexpr int kSchedTrans = 0x400;  // (as kSchedValu)
constexpr int kTileRows = 64;
constexpr int kWeightThreads = 256;
constexpr int kWeightWaves = kWeightThreads / 64;

// What scores come from, in units of log2: cap tanh(y) = cap - 2 cap / (1 + e^2y).
struct ScoreUnits {
  float c1, cap2, capk;
};
template <bool CAP>
__device__ __forceinline__ ScoreUnits score_units(const WeightArgs& a) {
  return {a.sm_scale * kLog2e, a.softcap * kLog2e, CAP ? 2.f * kLog2e * a.sm_scale / a.softcap : 0.f};
}
// exp(score - lse) of a product z
template <bool CAP, bool BIAS>
__device__ __forceinline__ float share(float z, const ScoreUnits& u, float lse, float slope, int away) {
  if (!CAP && !BIAS) return __builtin_amdgcn_exp2f(fmaf(z, u.c1, -lse));
  float x = CAP ? fmaf(-2.f * u.cap2, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * u.capk)), u.cap2) : z * u.c1;
  if (BIAS) x = fmaf(-slope, (float)away, x);
  return __builtin_amdgcn_exp2f(x - lse);
}
// whether a row at slot `place` (-1: no row) sees the slot `away` before it, `n`
__device__ __forceinline__ bool sees(const WeightArgs& a, int place, int away, int n) {
  return away >= 0 && (!a.window || away < a.window || n < a.sinks) && place >= 0;
}

template <int KB, bool CAP, bool BIAS>
__global__ __launch_bounds__(kWeightThreads, 2) void key_weights_kernel(WeightArgs a) {
  constexpr int kKeys = 32 * KB * kWeightWaves;
  extern __shared__ __attribute__((aligned(256))) char weight_tiles[];  // two tiles of rows, or 32 keys of each wavefront
  __shared__ __attribute__((aligned(16))) float row_lse[2][kTileRows];  // in log2; +inf: the row adds nothing
  __shared__ __attribute__((aligned(16))) int row_place[2][kTileRows];  // slot of the row's token, -1: none
  __shared__ __attribute__((aligned(16))) float row_slope[2][BIAS ? kTileRows : 4];
  __shared__ int odd_rows[2];
  static_assert(2 * kTileRows == 32 * kWeightWaves, "the buffers' two uses");
  const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3;
  int bh, block;
  if (a.rounds) {
    const int round = a.div_blocks.quotient(turn);
    block = turn - round * a.blocks, bh = round * 8 + xcd;
    if (bh >= a.B * a.Hkv) return;
  } else {
    const int per = (a.B * a.Hkv * a.blocks + 7) >> 3, item = xcd * per + turn;
    if (turn >= per || item >= a.B * a.Hkv * a.blocks) return;
    bh = a.div_blocks.quotient(item), block = item - bh * a.blocks;
  }
  const int b = a.div_Hkv.quotient(bh), h = bh - b * a.Hkv;
  const int first = uniform_load(a.pos + b);
  const int given = a.count ? min(max(uniform_load(a.count + b), 0), a.T) : a.T;
  if (first < 0 || first > a.N - given) return;
  const int khi = first + given;
  const int n_wg = block * kKeys, G = a.G;
  if (n_wg >= khi) return;

  // ---- the rows that see any of the workgroup's keys ------------------------
  const int n_end = min(n_wg + kKeys, khi);
  int t0 = max(0, n_wg - first), t1 = given;
  if (a.window && n_wg >= a.sinks) t1 = (int)min((int64_t)t1, (int64_t)n_end - 1 + a.window - first);
  const int r0 = t0 * G, r1 = max(t0, t1) * G;
  if (r0 == r1 && a.decay == 1.f) return;

  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int n_wave = n_wg + wid * 32 * KB;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)weight_tiles, ldsK = lds0 + wid * 32 * kRowBytes;

  // ---- this lane's keys -----------------------------------------------------
  // 16 keys at a time lie in one page; the pages are looked up at once
  constexpr int NP = 2 * KB;
  uint32_t pages[NP];
  uint32_t bad = 0;
  if (a.table) {
#pragma unroll
    for (int u = 0; u < NP; ++u) pages[u] = (uint32_t)uniform_load(a.table + b * a.st_b + (min(n_wave + 16 * u, khi - 1) >> a.page_shift));
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      if (pages[u] >= (uint32_t)a.num_pages) bad |= 1u << u, pages[u] = 0;
    }
  }
  const uint32_t kstep = (uint32_t)a.sK_n * 2;
  const int pmask = (1 << a.page_shift) - 1, r4 = lane >> 4;
  auto copy_keys = [&](int k) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int nu = min(n_wave + 32 * k + 16 * u, khi - 1), last = khi - 1 - nu;
      const uint16_t* base = a.K + h * a.sK_h;
      base += a.table ? pages[2 * k + u] * a.sK_b + (int64_t)(nu & pmask) * a.sK_n : b * a.sK_b + (int64_t)nu * a.sK_n;
      const char* from = reinterpret_cast<const char*>(uniform64(reinterpret_cast<uint64_t>(base)));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t row = 16 * u + 4 * i + r4;
        const uint32_t off = min(4 * i + r4, last) * kstep + (((uint32_t)lane & 15u) ^ swz(row)) * 16;
        dma16<false>(from, off, ldsK + (16 * u + 4 * i) * kRowBytes);
      }
    }
  };
  copy_keys(0);

  // ---- tiles of rows: global memory -> registers -> LDS ----------------------
  const int part = threadIdx.x & 15, line = threadIdx.x >> 4;  // 16 bytes of rows line + 16 i
  u32x4 qr[4];
  float lse_r = 0.f, slope_r = 0.f;
  int place_r = -1;
  // Where G divides a tile's 64 rows, a tile's rows lie 64 / G tokens behind the last
  // tile's, head for head.
  const int tokens = kTileRows / G;
  const bool even = tokens * G == kTileRows;
  const uint16_t* qp[4];
  const float* lp = a.lse;
  int place_lp = 0;
  auto fetch = [&](int r) {
    if (!even || r == r0 || r + kTileRows > r1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = min(r + line + 16 * i, r1 - 1), t = a.div_G.quotient(row), g = row - t * G;
        qp[i] = a.q + b * a.sq_b + (int64_t)(h * G + g) * a.sq_h + (int64_t)t * a.sq_t + 8 * part;
      }
      if (threadIdx.x < kTileRows) {
        const int row = min(r + (int)threadIdx.x, r1 - 1), t = a.div_G.quotient(row), g = row - t * G;
        lp = a.lse + b * a.sl_b + (int64_t)(h * G + g) * a.sl_h + t;
        place_lp = first + t;
        if (BIAS) slope_r = a.slopes[h * G + g] * kLog2e;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) qp[i] += tokens * a.sq_t;
      lp += tokens, place_lp += tokens;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) qr[i] = *reinterpret_cast<const u32x4*>(qp[i]);
    if (threadIdx.x < kTileRows) {
      lse_r = INFINITY, place_r = -1;
      if (r + (int)threadIdx.x < r1) {
        const float x = *lp * kLog2e;
        if (x != -INFINITY) lse_r = x, place_r = place_lp;
      }
    }
  };
  auto store = [&](int buf) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t row = line + 16 * i;
      *reinterpret_cast<u32x4*>(&weight_tiles[(buf * kTileRows + row) * kRowBytes + ((uint32_t)part ^ swz(row)) * 16]) = qr[i];
    }
    if (threadIdx.x < kTileRows) {
      row_lse[buf][threadIdx.x] = lse_r, row_place[buf][threadIdx.x] = place_r;
      if (BIAS) row_slope[buf][threadIdx.x] = slope_r;
      const bool odd = __any(place_r < 0);
      if (threadIdx.x == 0) odd_rows[buf] = odd;
    }
  };
  if (r0 < r1) fetch(r0);
  float* wp = a.weights + b * a.sw_b + h * a.sw_h;
  float old[KB];
#pragma unroll
  for (int k = 0; k < KB; ++k) old[k] = a.decay != 0.f ? wp[min(n_wave + 32 * k + col, khi - 1)] : 0.f;

  const uint32_t kswz = swz(col & 15) ^ half;
  bf16x8 kf[KB][8];
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    if (k) copy_keys(k);
    dma_wait<0>();
#pragma unroll
    for (int s = 0; s < 8; ++s) kf[k][s] = __builtin_bit_cast(bf16x8, lds_read<u32x4>(ldsK + col * kRowBytes + ((2 * s) ^ kswz) * 16, 0));
    lds_done();
    // (read before the next copies, or the rows, overwrite them)
#pragma unroll
    for (int s = 0; s < 8; ++s) asm volatile("" : "+v"(kf[k][s]));
  }
  __syncthreads();

  const ScoreUnits units = score_units<CAP>(a);
  float sum[KB], lost[KB];
#pragma unroll
  for (int k = 0; k < KB; ++k) sum[k] = lost[k] = 0.f;

  int buf = 0;
  for (int r = r0; r < r1; r += kTileRows, buf ^= 1) {
    store(buf);
    __syncthreads();
    if (r + kTileRows < r1) fetch(r + kTileRows);
    const bool odd = __builtin_amdgcn_readfirstlane(odd_rows[buf]);
    // a row block of 32 rows against 32 keys is a unit: products, then what a lane's
    // 16 rows add to its key
    constexpr int kUnits = kTileRows / 32 * KB;
    f32x16 acc[2];
    bf16x8 qf[8];
    auto read_rows = [&](int sub) {
#pragma unroll
      for (int s = 0; s < 8; ++s)
        qf[s] = __builtin_bit_cast(bf16x8, lds_read<u32x4>(lds0 + (buf * kTileRows + 32 * sub + col) * kRowBytes + ((2 * s) ^ kswz) * 16, 0));
    };
    auto products = [&](int k, f32x16& z) {
#pragma unroll
      for (int s = 0; s < 8; ++s) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[s], kf[k][s], s ? z : f32x16{}, 0, 0, 0);
    };
    auto add_up = [&](int k, float add) {  // and what the rounding of the sum lost
      const float s = sum[k] + add, bb = s - sum[k];
      lost[k] += (sum[k] - (s - bb)) + (add - bb);
      sum[k] = s;
    };
    auto gather = [&](int sub, int k, const f32x16& z) {
      const int n = n_wave + 32 * k + col;
      float add = 0.f;
#pragma unroll
      for (int e4 = 0; e4 < 4; ++e4) {
        const int at = 32 * sub + 8 * e4 + 4 * half;
        const float4 L = *reinterpret_cast<const float4*>(&row_lse[buf][at]);
        const float l[4] = {L.x, L.y, L.z, L.w};
        const int4 P = *reinterpret_cast<const int4*>(&row_place[buf][at]);
        const int place[4] = {P.x, P.y, P.z, P.w};
        float sl[4] = {};
        if (BIAS) {
          const float4 x = *reinterpret_cast<const float4*>(&row_slope[buf][at]);
          sl[0] = x.x, sl[1] = x.y, sl[2] = x.z, sl[3] = x.w;
        }
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int away = place[i] - n;
          p[i] = share<CAP, BIAS>(z[4 * e4 + i], units, l[i], sl[i], away);
          p[i] = sees(a, place[i], away, n) ? p[i] : 0.f;
        }
        add += (p[0] + p[1]) + (p[2] + p[3]);
      }
      add_up(k, add);
    };
    const int p0 = first + a.div_G.quotient(r), p1 = first + a.div_G.quotient(min(r + kTileRows, r1) - 1);
    const int n_last = n_wave + 32 * KB - 1;
    if (r + kTileRows <= r1 && !odd && n_last <= p0 && (!a.window || n_wave > p1 - a.window || n_last < a.sinks)) {
      // every row sees every key: a unit's exponentials run beside the next one's products
      float l[16];
      auto read_lse = [&](int sub) {
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const float4 x = *reinterpret_cast<const float4*>(&row_lse[buf][32 * sub + 8 * e4 + 4 * half]);
          l[4 * e4] = x.x, l[4 * e4 + 1] = x.y, l[4 * e4 + 2] = x.z, l[4 * e4 + 3] = x.w;
        }
      };
      auto whole = [&](int sub, int k, const f32x16& z) {
        float p[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int r = 32 * sub + 8 * (e / 4) + 4 * half + e % 4;
          p[e] = share<CAP, BIAS>(z[e], units, l[e], BIAS ? row_slope[buf][r] : 0.f, BIAS ? row_place[buf][r] - (n_wave + 32 * k + col) : 0);
        }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) {
#pragma unroll
          for (int e = 0; e < 16; e += 2 * o) p[e] += p[e + o];
        }
        add_up(k, p[0]);
      };
      read_rows(0);
      read_lse(0);
      __builtin_amdgcn_sched_barrier(0);
      products(0, acc[0]);
#pragma unroll
      for (int u = 1; u <= kUnits; ++u) {
        __builtin_amdgcn_sched_barrier(0);
        const bool next_rows = u < kUnits && u % KB == 0;
        if (next_rows) read_rows(u / KB);
        whole((u - 1) / KB, (u - 1) % KB, acc[(u - 1) & 1]);
        if (u < kUnits) products(u % KB, acc[u & 1]);
        if (next_rows) read_lse(u / KB);
        if (next_rows) {
          __builtin_amdgcn_sched_group_barrier(kSchedLds, 8, 0);
          __builtin_amdgcn_sched_group_barrier(kSchedValu, 16, 0);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
          __builtin_amdgcn_sched_group_barrier(kSchedValu, 5, 0);
          __builtin_amdgcn_sched_group_barrier(kSchedTrans, 2, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    } else {
#pragma unroll 1
      for (int sub = 0; sub < kTileRows / 32; ++sub) {
        const int s0 = r + 32 * sub;
        if (s0 >= r1) break;
        const int first_p = first + a.div_G.quotient(s0), last_p = first + a.div_G.quotient(min(s0 + 31, r1 - 1));
        if (n_wave > last_p) continue;  // no row sees any key of the wavefront
        if (a.window && n_wave >= a.sinks && n_last < first_p - a.window + 1) continue;
        read_rows(sub);
#pragma unroll
        for (int k = 0; k < KB; ++k) {
          products(k, acc[0]);
          gather(sub, k, acc[0]);
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    const int n = n_wave + 32 * k + col;
    // (what an infinite sum lost is not a number)
    const float x = sum_halves(fabsf(sum[k]) < INFINITY ? sum[k] + lost[k] : sum[k]);
    const float base = a.decay != 0.f ? a.decay * old[k] : 0.f;
    if (half == 0 && n < khi) wp[n] = base + ((bad >> (2 * k + (col >> 4)) & 1) ? 0.f : x);
  }
}

// Up to 32 SUB rows; a workgroup's run of a.run keys.  The run's page entries are there
// before it begins, and its sums go to memory when it is over: a look-up and a store
// between the copies of each 32 keys cost 9 and 12 % of the bandwidth.
constexpr int kMaxRun = 2048;
template <int SUB, bool CAP, bool BIAS, bool ONCE>
__global__ __launch_bounds__(kWeightThreads, 2) void key_weights_stream_kernel(WeightArgs a) {
  constexpr int kBuffer = 32 * kRowBytes;
  extern __shared__ __attribute__((aligned(256))) char stream_tiles[];  // two buffers of each wavefront
  __shared__ __attribute__((aligned(16))) float row_lse[32 * SUB];
  __shared__ __attribute__((aligned(16))) int row_place[32 * SUB];
  __shared__ __attribute__((aligned(16))) float row_slope[BIAS ? 32 * SUB : 4];
  __shared__ float sums[kMaxRun];
  __shared__ uint32_t entries[kMaxRun / 16];
  // pieces go round the XCDs: sequences' lengths differ
  const int bh = a.div_blocks.quotient(blockIdx.x), block = blockIdx.x - bh * a.blocks;
  const int b = a.div_Hkv.quotient(bh), h = bh - b * a.Hkv;
  const int first = uniform_load(a.pos + b);
  const int given = a.count ? min(max(uniform_load(a.count + b), 0), a.T) : a.T;
  if (first < 0 || first > a.N - given) return;
  const int khi = first + given, G = a.G, rows = given * G;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int from = block * a.run, to = min(from + a.run, khi);
  if (from >= khi) return;

  // ---- rows -------------------------------------------------------------------
  if ((int)threadIdx.x < 32 * SUB) {
    float lse = INFINITY, slope = 0.f;
    int place = -1;
    if ((int)threadIdx.x < rows) {
      const int t = a.div_G.quotient(threadIdx.x), g = threadIdx.x - t * G;
      const float x = a.lse[b * a.sl_b + (int64_t)(h * G + g) * a.sl_h + t] * kLog2e;
      if (x != -INFINITY) lse = x, place = first + t;
      if (BIAS) slope = a.slopes[h * G + g] * kLog2e;
    }
    row_lse[threadIdx.x] = lse, row_place[threadIdx.x] = place;
    if (BIAS) row_slope[threadIdx.x] = slope;
  }
  if (a.table && (int)threadIdx.x < a.run / 16)
    entries[threadIdx.x] = (uint32_t)a.table[b * a.st_b + (min(from + 16 * (int)threadIdx.x, khi - 1) >> a.page_shift)];
  bf16x8 qf[SUB][8];
#pragma unroll
  for (int sub = 0; sub < SUB; ++sub) {
    const int row = 32 * sub + col;
    const bool live = row < rows;
    const int t = live ? a.div_G.quotient(row) : 0, g = live ? row - t * G : 0;
    const uint16_t* qp = a.q + b * a.sq_b + (int64_t)(h * G + g) * a.sq_h + (int64_t)t * a.sq_t + 8 * half;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const u32x4 x = live ? *reinterpret_cast<const u32x4*>(qp + 16 * s) : u32x4{0, 0, 0, 0};
      qf[sub][s] = __builtin_bit_cast(bf16x8, x);
    }
  }
  __syncthreads();
  float lse[SUB][16];
  uint32_t live[SUB][16];  // all ones where the row adds something
#pragma unroll
  for (int sub = 0; sub < SUB; ++sub) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int r = 32 * sub + 8 * (e / 4) + 4 * half + e % 4;
      lse[sub][e] = row_lse[r], live[sub][e] = row_place[r] >= 0 ? ~0u : 0u;
    }
  }

  // ---- the keys that some row sees: blocks b0 .. and, behind a gap, b0 + near + gap .. ----
  float* wp = a.weights + b * a.sw_b + h * a.sw_h;
  const int p1 = khi - 1;  // the last row's slot, and before it all keys of this call
  const int b0 = from / 32, b1 = (to + 31) / 32;
  int near = b1 - b0, gap = 0, total = near;
  if (!rows) {
    near = total = 0, gap = b1 - b0;
  } else if (a.window) {
    const int lo = max(0, first - a.window + 1) / 32;
    near = max(0, min(b1, (min(a.sinks, khi) + 31) / 32) - b0);
    gap = max(0, min(b1, lo) - (b0 + near));
    total = b1 - b0 - gap;
  }
  // the wavefronts take turns, so that a workgroup reads one stream
  const int turns = (total - wid + kWeightWaves - 1) / kWeightWaves;
  auto block_key = [&](int turn) {
    const int i = turn * kWeightWaves + wid;
    return 32 * (b0 + (i < near ? i : i + gap));
  };

  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)stream_tiles + wid * 2 * kBuffer;
  const uint32_t kstep = (uint32_t)a.sK_n * 2;
  const int pmask = (1 << a.page_shift) - 1, r4 = lane >> 4;
  uint32_t bad_next = 0;
  auto issue = [&](int i, int buf) {
    const int n0 = block_key(i);
    const uint32_t dst = lds0 + buf * kBuffer;
    bad_next = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int nu = min(n0 + 16 * u, khi - 1), last = khi - 1 - nu;
      const uint16_t* base = a.K + h * a.sK_h;
      if (a.table) {
        uint32_t page = __builtin_amdgcn_readfirstlane(entries[((n0 - from) >> 4) + u]);
        if (page >= (uint32_t)a.num_pages) bad_next |= 1u << u, page = 0;
        base += page * a.sK_b + (int64_t)(nu & pmask) * a.sK_n;
      } else {
        base += b * a.sK_b + (int64_t)nu * a.sK_n;
      }
      const char* src = reinterpret_cast<const char*>(uniform64(reinterpret_cast<uint64_t>(base)));
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint32_t row = 16 * u + 4 * x + r4;
        dma16<ONCE>(src, min(4 * x + r4, last) * kstep + (((uint32_t)lane & 15u) ^ swz(row)) * 16, dst + (16 * u + 4 * x) * kRowBytes);
      }
    }
  };
  if (turns > 0) issue(0, 0);
#pragma unroll
  for (int sub = 0; sub < SUB; ++sub) {
#pragma unroll
    for (int s = 0; s < 8; ++s) asm volatile("" : "+v"(qf[sub][s]));
  }
  const ScoreUnits units = score_units<CAP>(a);
  const uint32_t kaddr = col * kRowBytes + (swz(col & 15) ^ half) * 16;
  for (int i = 0; i < turns; ++i) {
    const int buf = i & 1, n0 = block_key(i), n = n0 + col;
    const uint32_t bad = bad_next;
    if (i + 1 < turns) {
      issue(i + 1, buf ^ 1);
      dma_wait<8>();
    } else {
      dma_wait<0>();
    }
    const uint32_t at = lds0 + buf * kBuffer;
    bf16x8 kf[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) kf[s] = __builtin_bit_cast(bf16x8, lds_read<u32x4>(opaque(at + (kaddr ^ 32u * s)), 0));
    const bool full = n0 + 31 <= first && (!a.window || n0 > p1 - a.window || n0 + 32 <= a.sinks);
    float sum = 0.f;
#pragma unroll
    for (int sub = 0; sub < SUB; ++sub) {
      f32x16 acc;
#pragma unroll
      for (int s = 0; s < 8; ++s) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[sub][s], kf[s], s ? acc : f32x16{}, 0, 0, 0);
      float p[16];
      if (!BIAS && full) {
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = __uint_as_float(__float_as_uint(share<CAP, BIAS>(acc[e], units, lse[sub][e], 0.f, 0)) & live[sub][e]);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int r = 32 * sub + 8 * (e / 4) + 4 * half + e % 4, place = row_place[r], away = place - n;
          p[e] = share<CAP, BIAS>(acc[e], units, lse[sub][e], BIAS ? row_slope[r] : 0.f, away);
          p[e] = sees(a, place, away, n) ? p[e] : 0.f;
        }
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) {
#pragma unroll
        for (int e = 0; e < 16; e += 2 * o) p[e] += p[e + o];
      }
      sum += p[0];
    }
    sum = sum_halves(sum);
    if (half == 0) sums[n - from] = bad >> (col >> 4) & 1 ? 0.f : sum;
    lds_done();  // the reads of this buffer, before it is filled again
  }
  __syncthreads();
  for (int n = from + (int)threadIdx.x; n < to; n += kWeightThreads) {
    const int i = n / 32 - b0;
    const bool unseen = i >= near && i < near + gap;
    if (unseen && a.decay == 1.f) continue;
    const float x = unseen ? 0.f : sums[n - from];
    wp[n] = a.decay != 0.f ? a.decay * wp[n] + x : x;
  }
}

template <int KB>
static hipError_t launch_weights(WeightArgs a) {
  const int keys = 32 * KB * kWeightWaves;
  a.blocks = (a.N + keys - 1) / keys, a.div_blocks = FastDiv::by(a.blocks);
  const int64_t bh = (int64_t)a.B * a.Hkv;
  a.rounds = bh % 8 == 0 || bh >= 32;
  const int64_t grid = a.rounds ? (bh + 7) / 8 * 8 * a.blocks : (bh * a.blocks + 7) / 8 * 8;
  auto* f = a.softcap > 0.f ? (a.slopes ? key_weights_kernel<KB, true, true> : key_weights_kernel<KB, true, false>)
                            : (a.slopes ? key_weights_kernel<KB, false, true> : key_weights_kernel<KB, false, false>);
  f<<<(unsigned)grid, kWeightThreads, 2 * kTileRows * kRowBytes, a.stream>>>(a);
  return hipGetLastError();
}

template <int SUB>
static hipError_t launch_stream(WeightArgs a) {
  const int64_t bh = (int64_t)a.B * a.Hkv, keys = bh * a.N;
  // A workgroup's run: four rounds of two a compute unit, where there are so many keys.
  a.run = (int)std::max<int64_t>(64 * kWeightWaves, std::min<int64_t>(kMaxRun, (keys / 2048 + 255) / 256 * 256));
  a.blocks = (a.N + a.run - 1) / a.run, a.div_blocks = FastDiv::by(a.blocks);
  const bool once = keys * kRowBytes > (int64_t)320 << 20;  // as in attn_plan
#define BPC_STREAM(CAP, BIAS)                                                                                                              \
  {                                                                                                                                        \
    auto* f = once ? key_weights_stream_kernel<SUB, CAP, BIAS, true> : key_weights_stream_kernel<SUB, CAP, BIAS, false>;                   \
    constexpr int lds = 2 * kWeightWaves * 32 * kRowBytes;                                                                                 \
    static std::atomic<uint64_t> allowed[2];                                                                                               \
    if (hipError_t e = allow_lds(reinterpret_cast<const void*>(f), lds, allowed[once]); e != hipSuccess) return e;                         \
    f<<<(unsigned)(bh * a.blocks), kWeightThreads, lds, a.stream>>>(a);                                                                    \
  }
  if (a.softcap > 0.f) {
    if (a.slopes) BPC_STREAM(true, true) else BPC_STREAM(true, false)
  } else {
    if (a.slopes) BPC_STREAM(false, true) else BPC_STREAM(false, false)
  }
#undef BPC_STREAM
  return hipGetLastError();
}

int64_t weights_blocks(int B, int Hkv, int N) { return ((int64_t)B * Hkv + 7) / 8 * 8 * ((N + 127) / 128); }

hipError_t launch_key_weights(WeightArgs a) {
  a.div_G = FastDiv::by(a.G), a.div_Hkv = FastDiv::by(a.Hkv);
  const int64_t rows = (int64_t)a.T * a.G;
  if (rows <= 32) return launch_stream<1>(a);
  if (rows <= 64) return launch_stream<2>(a);
  // 64 keys a wavefront where that leaves the chip full (500 tokens of 2 requests over
  // 32768 slots: 197 us, with 32 keys 209)
  return weights_blocks(a.B, a.Hkv, a.N) < 1024 ? launch_weights<1>(a) : launch_weights<2>(a);
}

}  // namespace bpc
