// Rows on their way into the cache: the RMS norm of a query or key row, the
// rotation by its token's position, and the store to a tensor or to a page.
//
// A row of 128 bf16 is 16 lanes of 16 bytes, so that a wavefront works on four
// rows (heads) of one token at once.  The mean of squares is a sum over 16
// lanes; the partner of coordinate d in a rotation by halves (d +- R/2) lies
// R / 16 lanes away and is fetched with one shuffle per 4 bytes of the raw row
// (the norm's factor is the same for both), that of a rotation in adjacent
// pairs lies in the same lane.  A lane holds the cosines and sines of its eight
// coordinates for all heads of the token.
#include "bpc_internal.h"

namespace bpc {

constexpr int kRopeThreads = 256;
constexpr int kRopeWaves = kRopeThreads / 64;
constexpr int kRowLanes = kHeadDim / 8;     // lanes per row
constexpr int kRowsPerPass = 64 / kRowLanes;  // rows of a wavefront at once
constexpr int kRopeBatch = 4;               // passes whose loads are issued before the first is used

// The bf16 nearest to x, ties to even (the compiler's conversion instruction).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  bf2 p;
  p[0] = (__bf16)lo, p[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// What a lane keeps for the rows of one token and one tensor: its eight norm
// weights, its partner's, and the token's cosines and sines (of the lane's four
// pairs in the first four entries where pairs are adjacent).
struct RopeLane {
  float c[8], s[8];
  int partner;  // lane of the partner chunk (itself outside the rotation)
  bool turn;    // the lane's coordinates are rotated
};

__device__ __forceinline__ RopeLane rope_lane(const float* __restrict__ cs, int R, int inter) {
  RopeLane r;
  const int lane = threadIdx.x & 63, j = lane % kRowLanes;
  r.turn = 8 * j < R;
  r.partner = lane;
#pragma unroll
  for (int e = 0; e < 8; ++e) r.c[e] = 1.f, r.s[e] = 0.f;
  if (!r.turn) return r;
  const int half = R / 2;
  if (inter) {
    const float4 c = *reinterpret_cast<const float4*>(cs + 4 * j), s = *reinterpret_cast<const float4*>(cs + half + 4 * j);
    r.c[0] = c.x, r.c[1] = c.y, r.c[2] = c.z, r.c[3] = c.w;
    r.s[0] = s.x, r.s[1] = s.y, r.s[2] = s.z, r.s[3] = s.w;
    return r;
  }
  const int hl = R / 16;  // lanes per half
  const bool second = j >= hl;
  r.partner = second ? lane - hl : lane + hl;
  const float4* pc = reinterpret_cast<const float4*>(cs + 8 * (second ? j - hl : j));
  const float4* ps = reinterpret_cast<const float4*>(cs + half + 8 * (second ? j - hl : j));
  const float4 c0 = pc[0], c1 = pc[1], s0 = ps[0], s1 = ps[1];
  const float g = second ? 1.f : -1.f;  // x1 c - x2 s, x2 c + x1 s
  r.c[0] = c0.x, r.c[1] = c0.y, r.c[2] = c0.z, r.c[3] = c0.w;
  r.c[4] = c1.x, r.c[5] = c1.y, r.c[6] = c1.z, r.c[7] = c1.w;
  r.s[0] = g * s0.x, r.s[1] = g * s0.y, r.s[2] = g * s0.z, r.s[3] = g * s0.w;
  r.s[4] = g * s1.x, r.s[5] = g * s1.y, r.s[6] = g * s1.z, r.s[7] = g * s1.w;
  return r;
}

// Norm (with `w`, the row's 128 weights, else none) and rotation of the row
// whose chunk `x` this lane holds; every lane of the wavefront calls it.
__device__ __forceinline__ uint4 rope_row(uint4 x, const uint16_t* w, float eps, const RopeLane& rl, int R, int inter) {
  const uint32_t xr[4] = {x.x, x.y, x.z, x.w};
  float v[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[2 * e] = lo_f32(xr[e]), v[2 * e + 1] = hi_f32(xr[e]);
  float rstd = 1.f;
  if (w) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(v[e], v[e], ss);
#pragma unroll
    for (int o = 1; o < kRowLanes; o <<= 1) ss += __shfl_xor(ss, o, 64);
    rstd = rsqrtf(ss * (1.f / kHeadDim) + eps);
  }
  const int j = threadIdx.x % kRowLanes;
  if (w) {
    const uint4 wx = *reinterpret_cast<const uint4*>(w + 8 * j);
    const uint32_t wr[4] = {wx.x, wx.y, wx.z, wx.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[2 * e] *= rstd * lo_f32(wr[e]), v[2 * e + 1] *= rstd * hi_f32(wr[e]);
  }
  float y[8];
  if (R == 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = v[e];
  } else if (inter) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float a = v[2 * e], b = v[2 * e + 1];
      y[2 * e] = rl.turn ? a * rl.c[e] - b * rl.s[e] : a;
      y[2 * e + 1] = rl.turn ? b * rl.c[e] + a * rl.s[e] : b;
    }
  } else {
    float u[8];
    uint32_t pr[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) pr[e] = (uint32_t)__shfl((int)xr[e], rl.partner, 64);
#pragma unroll
    for (int e = 0; e < 4; ++e) u[2 * e] = lo_f32(pr[e]), u[2 * e + 1] = hi_f32(pr[e]);
    if (w) {
      const uint4 wx = *reinterpret_cast<const uint4*>(w + 8 * (rl.partner % kRowLanes));
      const uint32_t wr[4] = {wx.x, wx.y, wx.z, wx.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) u[2 * e] *= rstd * lo_f32(wr[e]), u[2 * e + 1] *= rstd * hi_f32(wr[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = rl.turn ? v[e] * rl.c[e] + u[e] * rl.s[e] : v[e];
  }
  return make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}

// ---------------------------------------------------------------------------
// qk_norm_rope: a wavefront takes one token and up to `per` of its heads, the
// query heads before the key heads.  Bound by memory.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(RopeArgs a, int per, int parts) {
  const int64_t wave = (int64_t)blockIdx.x * kRopeWaves + (threadIdx.x >> 6);
  const int64_t tok = wave / parts;
  if (tok >= (int64_t)a.B * a.T) return;
  const int h0 = (int)(wave - tok * parts) * per;
  const int b = (int)(tok / a.T), t = (int)(tok - (int64_t)b * a.T);
  const int lane = threadIdx.x & 63, sub = lane / kRowLanes, d0 = 8 * (lane % kRowLanes);
  const float* cs = nullptr;
  if (a.R) {
    const int p = a.pos[b * a.sp_b + t];
    if (p < 0 || p >= a.table_rows) return;  // no such position: the token's rows stay as they are
    cs = a.cos_sin + (int64_t)p * a.R;
  }
  const RopeLane rl = rope_lane(cs, a.R, a.inter);
  const int H = a.q.H + a.k.H, h1 = min(H, h0 + per);
  for (int hb = h0; hb < h1; hb += kRopeBatch * kRowsPerPass) {
    uint4 x[kRopeBatch];
    uint16_t* dst[kRopeBatch];
    const uint16_t* w[kRopeBatch];
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      const int h = min(hb + i * kRowsPerPass + sub, h1 - 1);
      const RopeTensor& s = h < a.q.H ? a.q : a.k;
      const int hh = h < a.q.H ? h : h - a.q.H;
      x[i] = *reinterpret_cast<const uint4*>(s.in + b * s.si_b + hh * s.si_h + t * s.si_t + d0);
      dst[i] = s.out + b * s.so_b + hh * s.so_h + t * s.so_t + d0;
      w[i] = s.w ? s.w + hh * s.sw_h : nullptr;
    }
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      if (hb + i * kRowsPerPass >= h1) break;
      const uint4 y = rope_row(x[i], w[i], a.eps, rl, a.R, a.inter);
      if (hb + i * kRowsPerPass + sub < h1) *reinterpret_cast<uint4*>(dst[i]) = y;
    }
  }
}

hipError_t launch_qk_norm_rope(const RopeArgs& a) {
  const int H = a.q.H + a.k.H;
  const int64_t tokens = (int64_t)a.B * a.T;
  int per = H, parts = 1;
  // few tokens: their heads are spread over wavefronts
  while (per > kRowsPerPass && tokens * parts < 2048) {
    per = ((per + 1) / 2 + kRowsPerPass - 1) / kRowsPerPass * kRowsPerPass;
    parts = (H + per - 1) / per;
  }
  const int64_t waves = tokens * parts;
  qk_norm_rope_kernel<<<(unsigned)((waves + kRopeWaves - 1) / kRopeWaves), kRopeThreads, 0, a.stream>>>(a, per, parts);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// append_kv_paged: as above, the key heads (normed and rotated) before the
// value heads (copied), stored at the token's row of its page.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(kRopeThreads) void append_paged_kernel(AppendPagedArgs a, int per, int parts) {
  const int64_t wave = (int64_t)blockIdx.x * kRopeWaves + (threadIdx.x >> 6);
  const int64_t tok = wave / parts;
  if (tok >= (int64_t)a.B * a.T) return;
  const int h0 = (int)(wave - tok * parts) * per;
  const int b = (int)(tok / a.T), t = (int)(tok - (int64_t)b * a.T);
  if (a.count && t >= a.count[b]) return;
  const int64_t slot = (int64_t)a.pos[b] + t;
  if (slot < 0 || (slot >> a.page_shift) >= a.max_pages) return;
  const int page = a.table[b * a.st_b + (slot >> a.page_shift)];
  if (page < 0 || page >= a.num_pages) return;
  const int64_t row = slot & ((1 << a.page_shift) - 1);
  const float* cs = nullptr;
  if (a.R) {
    const int64_t p = a.rope_pos ? a.rope_pos[b * a.sr_b + t] : slot;
    if (p < 0 || p >= a.table_rows) return;
    cs = a.cos_sin + p * a.R;
  }
  const int lane = threadIdx.x & 63, sub = lane / kRowLanes, d0 = 8 * (lane % kRowLanes);
  const RopeLane rl = rope_lane(cs, a.R, a.inter);
  const int H = 2 * a.Hkv, h1 = min(H, h0 + per);
  for (int hb = h0; hb < h1; hb += kRopeBatch * kRowsPerPass) {
    uint4 x[kRopeBatch];
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      const int h = min(hb + i * kRowsPerPass + sub, h1 - 1);
      const uint16_t* src = h < a.Hkv ? a.kn + b * a.skn_b + h * a.skn_h + t * a.skn_t
                                      : a.vn + b * a.svn_b + (h - a.Hkv) * a.svn_h + t * a.svn_t;
      x[i] = *reinterpret_cast<const uint4*>(src + d0);
    }
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      if (hb + i * kRowsPerPass >= h1) break;
      const int h = hb + i * kRowsPerPass + sub;
      uint4 y = x[i];
      if (hb + i * kRowsPerPass < a.Hkv && (a.R || a.wk)) {  // some of the wavefront's rows are keys
        const int hk = min(h, a.Hkv - 1);
        const uint4 turned = rope_row(x[i], a.wk ? a.wk + hk * a.sw_h : nullptr, a.eps, rl, a.R, a.inter);
        if (h < a.Hkv) y = turned;
      }
      if (h < h1) {
        uint16_t* dst = h < a.Hkv ? a.K + page * a.sK_p + h * a.sK_h + row * a.sK_n
                                  : a.V + page * a.sV_p + (h - a.Hkv) * a.sV_h + row * a.sV_n;
        *reinterpret_cast<uint4*>(dst + d0) = y;
      }
    }
  }
}

hipError_t launch_append_paged(const AppendPagedArgs& a) {
  const int H = 2 * a.Hkv;
  const int64_t tokens = (int64_t)a.B * a.T;
  int per = H, parts = 1;
  while (per > kRowsPerPass && tokens * parts < 2048) {
    per = ((per + 1) / 2 + kRowsPerPass - 1) / kRowsPerPass * kRowsPerPass;
    parts = (H + per - 1) / per;
  }
  const int64_t waves = tokens * parts;
  append_paged_kernel<<<(unsigned)((waves + kRopeWaves - 1) / kRopeWaves), kRopeThreads, 0, a.stream>>>(a, per, parts);
  return hipGetLastError();
}

}  // namespace bpc
