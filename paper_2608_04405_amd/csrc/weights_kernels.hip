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
#include <algorithm>

#include "attn_kernel.h"

namespace bpc {

constexpr int kTileRows = 64;
constexpr int kWeightThreads = 256;

template <int KB, bool CAP, bool BIAS>
__global__ __launch_bounds__(kWeightThreads, 2) void key_weights_kernel(WeightArgs a) {
  constexpr int kKeys = 32 * KB * (kWeightThreads / 64);
  __shared__ __attribute__((aligned(16))) char tile[2][kTileRows * kRowBytes];
  __shared__ __attribute__((aligned(16))) float row_lse[2][kTileRows];  // in log2; +inf: the row adds nothing
  __shared__ __attribute__((aligned(16))) int row_place[2][kTileRows];  // slot of the row's token, -1: none
  __shared__ __attribute__((aligned(16))) float row_slope[2][BIAS ? kTileRows : 4];
  __shared__ int odd_rows[2];
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

  // ---- this lane's keys -----------------------------------------------------
  bf16x8 kf[KB][8];
  float old[KB];
  bool there[KB];
  float* wp = a.weights + b * a.sw_b + h * a.sw_h;
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    const int n = min(n_wave + 32 * k + col, khi - 1);
    const uint16_t* row;
    there[k] = true;
    if (a.table) {
      uint32_t page = (uint32_t)a.table[b * a.st_b + (n >> a.page_shift)];
      there[k] = page < (uint32_t)a.num_pages;
      if (!there[k]) page = 0;
      row = a.K + page * a.sK_b + h * a.sK_h + (n & ((1 << a.page_shift) - 1)) * a.sK_n;
    } else {
      row = a.K + b * a.sK_b + h * a.sK_h + n * a.sK_n;
    }
#pragma unroll
    for (int s = 0; s < 8; ++s) kf[k][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(row + 16 * s + 8 * half));
    old[k] = a.decay != 0.f ? wp[n] : 0.f;
  }

  // ---- tiles of rows: global memory -> registers -> LDS ----------------------
  const int part = threadIdx.x & 15, line = threadIdx.x >> 4;  // 16 bytes of rows line + 16 i
  u32x4 qr[4];
  float lse_r = 0.f, slope_r = 0.f;
  int place_r = -1;
  auto fetch = [&](int r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = min(r + line + 16 * i, r1 - 1), t = a.div_G.quotient(row), g = row - t * G;
      qr[i] = *reinterpret_cast<const u32x4*>(a.q + b * a.sq_b + (int64_t)(h * G + g) * a.sq_h + (int64_t)t * a.sq_t + 8 * part);
    }
    if (threadIdx.x < kTileRows) {
      const int row = r + (int)threadIdx.x;
      lse_r = INFINITY, place_r = -1;
      if (row < r1) {
        const int t = a.div_G.quotient(row), g = row - t * G;
        const float x = a.lse[b * a.sl_b + (int64_t)(h * G + g) * a.sl_h + t] * kLog2e;
        if (x != -INFINITY) lse_r = x, place_r = first + t;
        if (BIAS) slope_r = a.slopes[h * G + g] * kLog2e;
      }
    }
  };
  auto store = [&](int buf) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t row = line + 16 * i;
      *reinterpret_cast<u32x4*>(&tile[buf][row * kRowBytes + ((uint32_t)part ^ swz(row)) * 16]) = qr[i];
    }
    if (threadIdx.x < kTileRows) {
      row_lse[buf][threadIdx.x] = lse_r, row_place[buf][threadIdx.x] = place_r;
      if (BIAS) row_slope[buf][threadIdx.x] = slope_r;
      const bool odd = __any(place_r < 0);
      if (threadIdx.x == 0) odd_rows[buf] = odd;
    }
  };

  const float c1 = a.sm_scale * kLog2e;
  const float cap2 = a.softcap * kLog2e, capk = CAP ? 2.f * kLog2e * a.sm_scale / a.softcap : 0.f;
  float sum[KB], lost[KB];
#pragma unroll
  for (int k = 0; k < KB; ++k) sum[k] = lost[k] = 0.f;
  const uint32_t kswz = swz(col & 15) ^ half;

  if (r0 < r1) fetch(r0);
  int buf = 0;
  for (int r = r0; r < r1; r += kTileRows, buf ^= 1) {
    store(buf);
    __syncthreads();
    if (r + kTileRows < r1) fetch(r + kTileRows);
    const bool odd = odd_rows[buf];
#pragma unroll
    for (int sub = 0; sub < kTileRows / 32; ++sub) {
      const int s0 = r + 32 * sub;
      if (s0 >= r1) break;
      const int p0 = first + a.div_G.quotient(s0), p1 = first + a.div_G.quotient(min(s0 + 31, r1 - 1));
      if (n_wave > p1) continue;  // no row sees any key of the wavefront
      if (a.window && n_wave >= a.sinks && n_wave + 32 * KB <= p0 - a.window + 1) continue;
      bf16x8 qf[8];
#pragma unroll
      for (int s = 0; s < 8; ++s)
        qf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(&tile[buf][(32 * sub + col) * kRowBytes + ((2 * s) ^ kswz) * 16]));
      f32x16 acc[KB];
#pragma unroll
      for (int k = 0; k < KB; ++k) {
#pragma unroll
        for (int s = 0; s < 8; ++s) acc[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[s], kf[k][s], s ? acc[k] : f32x16{}, 0, 0, 0);
      }
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        const int n0 = n_wave + 32 * k, n = n0 + col;
        const bool full = !odd && n0 + 31 <= p0 && (!a.window || n0 > p1 - a.window || n0 + 32 <= a.sinks);
        float add = 0.f;
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const int at = 32 * sub + 8 * e4 + 4 * half;
          const float4 L = *reinterpret_cast<const float4*>(&row_lse[buf][at]);
          const int4 P = *reinterpret_cast<const int4*>(&row_place[buf][at]);
          const float l[4] = {L.x, L.y, L.z, L.w};
          const int place[4] = {P.x, P.y, P.z, P.w};
          float sl[4] = {};
          if (BIAS) {
            const float4 x = *reinterpret_cast<const float4*>(&row_slope[buf][at]);
            sl[0] = x.x, sl[1] = x.y, sl[2] = x.z, sl[3] = x.w;
          }
          float part4 = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float z = acc[k][4 * e4 + i];
            float x;
            if (CAP || BIAS) {
              // cap tanh(y) = cap - 2 cap / (1 + e^2y), in log2
              x = CAP ? fmaf(-2.f * cap2, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * capk)), cap2) : z * c1;
              if (BIAS) x = fmaf(-sl[i], (float)(place[i] - n), x);
              x -= l[i];
            } else {
              x = fmaf(z, c1, -l[i]);
            }
            float p = __builtin_amdgcn_exp2f(x);
            if (!full) {
              const int away = place[i] - n;
              p = away >= 0 && (!a.window || away < a.window || n < a.sinks) && place[i] >= 0 ? p : 0.f;
            }
            part4 += p;
          }
          add += part4;
        }
        // sum + add, and what that rounding lost
        const float s = sum[k] + add, bb = s - sum[k];
        lost[k] += (sum[k] - (s - bb)) + (add - bb);
        sum[k] = s;
      }
    }
  }
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    const int n = n_wave + 32 * k + col;
    const float x = sum_halves(sum[k] + lost[k]);
    const float base = a.decay != 0.f ? a.decay * old[k] : 0.f;
    if (half == 0 && n < khi) wp[n] = base + (there[k] ? x : 0.f);
  }
}

template <int KB>
static hipError_t launch_weights(WeightArgs a) {
  const int keys = 32 * KB * (kWeightThreads / 64);
  a.blocks = (a.N + keys - 1) / keys, a.div_blocks = FastDiv::by(a.blocks);
  const int64_t bh = (int64_t)a.B * a.Hkv;
  a.rounds = bh % 8 == 0 || bh >= 32;
  const int64_t grid = a.rounds ? (bh + 7) / 8 * 8 * a.blocks : (bh * a.blocks + 7) / 8 * 8;
  auto* f = a.softcap > 0.f ? (a.slopes ? key_weights_kernel<KB, true, true> : key_weights_kernel<KB, true, false>)
                            : (a.slopes ? key_weights_kernel<KB, false, true> : key_weights_kernel<KB, false, false>);
  f<<<(unsigned)grid, kWeightThreads, 0, a.stream>>>(a);
  return hipGetLastError();
}

// workgroups of a call; a launch has fewer than 2^32 threads
int64_t weights_blocks(int B, int Hkv, int N) { return ((int64_t)B * Hkv + 7) / 8 * 8 * ((N + 127) / 128); }

hipError_t launch_key_weights(WeightArgs a) {
  a.div_G = FastDiv::by(a.G), a.div_Hkv = FastDiv::by(a.Hkv);
  return weights_blocks(a.B, a.Hkv, a.N) >= 512 ? launch_weights<2>(a) : launch_weights<1>(a);
}

}  // namespace bpc
