// Rows on their way into the cache: the RMS norm of a query or key row, the
// rotation by its token's position, and the store to a tensor or to a page.
//
// A row of 128 bf16 is 16 lanes of 16 bytes, so that a wavefront works on four
// rows (heads) of one token at once, a "pass", and goes through the token's
// heads pass by pass.  With the norm's factor r, the weights w and the token's
// cosines and sines every coordinate becomes
//     y_e = r (v_e C_e + u_e S_e),   C_e = w_e c,   S_e = -+ w_u s,
// u its partner in the pair: C and S hold for all heads of the token, so a row
// costs two multiply-adds and a product per coordinate, the mean of squares (a
// sum over 16 lanes by DPP rotations, equal in all of them), and the partner's
// raw values: R / 16 lanes away for pairs (i, i + R/2), where R = 128 is one
// DPP rotation by eight lanes, or in the same 32-bit word for adjacent pairs.
// Bound by memory: the loads of kRopeBatch passes are issued before the first is
// used.  32749 tokens of 40 heads take 124 us (5.5 TB/s; a copy of as many bytes
// runs at 5.4), the append of 4 x 8192 tokens of 8 heads 38 us, one token 2.5 us.
#include "bpc_internal.h"

namespace bpc {

constexpr int kRopeThreads = 256;
constexpr int kRopeWaves = kRopeThreads / 64;
constexpr int kRowLanes = kHeadDim / 8;       // lanes per row
constexpr int kPassRows = 64 / kRowLanes;     // rows of a pass
constexpr int kRopeBatch = 4;                 // passes whose loads are issued before the first is used

// where the partner of a coordinate lies
enum Pairing {
  kPairNone,     // no rotation
  kPairEight,    // eight lanes on: halves of R = 128
  kPairLanes,    // R / 16 lanes on: halves of a smaller R
  kPairAdjacent  // in the same word
};

// The bf16 nearest to x, ties to even (the compiler's conversion instruction).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  bf2 p;
  p[0] = (__bf16)lo, p[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// x of the lane N further on (mod 16) within the 16 lanes of a row
template <int N>
__device__ __forceinline__ uint32_t row_rotate(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xF, 0xF, true);
}
template <int N>
__device__ __forceinline__ float row_rotate_add(float x) {
  return x + __uint_as_float(row_rotate<N>(__float_as_uint(x)));
}

__device__ __forceinline__ void unpack8(const uint4& x, float v[8]) {
  v[0] = lo_f32(x.x), v[1] = hi_f32(x.x), v[2] = lo_f32(x.y), v[3] = hi_f32(x.y);
  v[4] = lo_f32(x.z), v[5] = hi_f32(x.z), v[6] = lo_f32(x.w), v[7] = hi_f32(x.w);
}

// a lane's place in the rotation of its token: cosines and signed sines of its
// eight coordinates (1 and -0 outside, where x + 0 * -0 is x for every x), and its
// partner's lane
struct Turn {
  float c[8], s[8];
  int partner;
  uint32_t keep;  // all ones where the partner counts
};

template <Pairing PAIR>
__device__ __forceinline__ Turn token_turn(const float* __restrict__ cs, int R) {
  Turn r;
  const int lane = threadIdx.x & 63, j = lane % kRowLanes, half = R / 2;
  r.partner = lane, r.keep = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) r.c[e] = 1.f, r.s[e] = -0.f;
  if (PAIR == kPairNone || 8 * j >= R) return r;
  r.keep = 0xFFFFFFFFu;
  if (PAIR == kPairAdjacent) {
    const float4 c = *reinterpret_cast<const float4*>(cs + 4 * j), s = *reinterpret_cast<const float4*>(cs + half + 4 * j);
    const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      r.c[2 * e] = r.c[2 * e + 1] = cc[e];
      r.s[2 * e] = -ss[e], r.s[2 * e + 1] = ss[e];
    }
    return r;
  }
  const int hl = R / 16;  // lanes per half
  const bool second = j >= hl;
  r.partner = second ? lane - hl : lane + hl;
  const int f = 8 * (second ? j - hl : j);
  const float4* pc = reinterpret_cast<const float4*>(cs + f);
  const float4* ps = reinterpret_cast<const float4*>(cs + half + f);
  const float4 c0 = pc[0], c1 = pc[1], s0 = ps[0], s1 = ps[1];
  const float cc[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
  const float ss[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) r.c[e] = cc[e], r.s[e] = second ? ss[e] : -ss[e];
  return r;
}

// C and S of a row with weights w (or none)
template <Pairing PAIR>
__device__ __forceinline__ void row_factors(const Turn& t, const uint16_t* w, float C[8], float S[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) C[e] = t.c[e], S[e] = t.s[e];
  if (!w) return;
  float wv[8], wu[8];
  unpack8(*reinterpret_cast<const uint4*>(w + 8 * (threadIdx.x % kRowLanes)), wv);
  if (PAIR == kPairAdjacent) {
#pragma unroll
    for (int e = 0; e < 8; ++e) wu[e] = wv[e ^ 1];
  } else if (PAIR != kPairNone) {
    unpack8(*reinterpret_cast<const uint4*>(w + 8 * (t.partner % kRowLanes)), wu);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    C[e] *= wv[e];
    if (PAIR == kPairEight || (PAIR != kPairNone && t.keep)) S[e] *= wu[e];
  }
}

// the row whose chunk `x` this lane holds; every lane of the wavefront calls it
template <Pairing PAIR>
__device__ __forceinline__ uint4 turn_row(const uint4& x, bool norm, float eps, const Turn& t, const float C[8], const float S[8]) {
  float v[8], y[8];
  unpack8(x, v);
  float r = 1.f;
  if (norm) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(v[e], v[e], ss);
    ss = row_rotate_add<1>(row_rotate_add<2>(row_rotate_add<4>(row_rotate_add<8>(ss))));
    r = rsqrtf(fmaf(ss, 1.f / kHeadDim, eps));
  }
  if (PAIR == kPairNone) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = v[e] * C[e];
  } else {
    const uint32_t xr[4] = {x.x, x.y, x.z, x.w};
    float u[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t p;
      if (PAIR == kPairAdjacent) p = __builtin_amdgcn_alignbit(xr[e], xr[e], 16);
      if (PAIR == kPairEight) p = row_rotate<8>(xr[e]);
      if (PAIR == kPairLanes) p = (uint32_t)__shfl((int)xr[e], t.partner, 64);
      if (PAIR != kPairEight) p &= t.keep;  // outside the rotation: no partner, whatever its value
      u[2 * e] = lo_f32(p), u[2 * e + 1] = hi_f32(p);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = fmaf(u[e], S[e], v[e] * C[e]);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] *= r;
  return make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}

// 16 bytes of a row; STREAM: past the caches
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <bool STREAM>
__device__ __forceinline__ uint4 load_chunk(const uint16_t* p) {
  const u32x4* at = reinterpret_cast<const u32x4*>(p);
  const u32x4 x = STREAM ? __builtin_nontemporal_load(at) : *at;
  return make_uint4(x[0], x[1], x[2], x[3]);
}
template <bool STREAM>
__device__ __forceinline__ void store_chunk(uint16_t* p, const uint4& y) {
  u32x4* at = reinterpret_cast<u32x4*>(p);
  const u32x4 x = {y.x, y.y, y.z, y.w};
  if (STREAM)
    __builtin_nontemporal_store(x, at);
  else
    *at = x;
}

// Passes [p0, p1) of a token's heads through `row(chunk, head)`, from `src` with
// head stride ss to `dst` with head stride sd: up to kRopeBatch passes' loads
// before the first is used.
template <int N, bool STREAM, class Row>
__device__ __forceinline__ void move_passes(const uint16_t* src, int64_t ss, uint16_t* dst, int64_t sd, int H, int p, Row row) {
  const int sub = (threadIdx.x & 63) / kRowLanes, d0 = 8 * (threadIdx.x % kRowLanes);
  uint4 x[N];
#pragma unroll
  for (int i = 0; i < N; ++i)
    x[i] = load_chunk<STREAM>(src + min((p + i) * kPassRows + sub, H - 1) * ss + d0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int h = (p + i) * kPassRows + sub;
    const uint4 y = row(x[i], min(h, H - 1));
    if (h < H) store_chunk<STREAM>(dst + h * sd + d0, y);
  }
}
template <bool STREAM, class Row>
__device__ __forceinline__ void move_heads(const uint16_t* src, int64_t ss, uint16_t* dst, int64_t sd, int H, int p0, int p1, Row row) {
  int p = p0;
  for (; p + kRopeBatch <= p1; p += kRopeBatch) move_passes<kRopeBatch, STREAM>(src, ss, dst, sd, H, p, row);
  if (p + 2 <= p1) move_passes<2, STREAM>(src, ss, dst, sd, H, p, row), p += 2;
  if (p < p1) move_passes<1, STREAM>(src, ss, dst, sd, H, p, row);
}

// rows of H heads of one token; PER_HEAD: weights of their own for every head
template <Pairing PAIR, bool PER_HEAD, bool STREAM>
__device__ __forceinline__ void turn_heads(const uint16_t* src, int64_t ss, uint16_t* dst, int64_t sd, const uint16_t* w,
                                           int64_t sw, float eps, const Turn& t, int H, int p0, int p1) {
  float C[8], S[8];
  if (!PER_HEAD) row_factors<PAIR>(t, w, C, S);
  move_heads<STREAM>(src, ss, dst, sd, H, p0, p1, [&](const uint4& x, int h) {
    if (PER_HEAD) row_factors<PAIR>(t, w ? w + h * sw : nullptr, C, S);
    return turn_row<PAIR>(x, w != nullptr, eps, t, C, S);
  });
}

// ---------------------------------------------------------------------------
// qk_norm_rope: a wavefront takes `per` of the passes of one token, those of the
// query heads before those of the key heads
// ---------------------------------------------------------------------------
template <Pairing PAIR, bool PER_HEAD, bool STREAM>
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(RopeArgs a, int per, int parts) {
  const uint32_t wave = blockIdx.x * kRopeWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t tok = wave / (uint32_t)parts;
  if (tok >= (uint32_t)a.B * (uint32_t)a.T) return;
  const int b = (int)(tok / (uint32_t)a.T), t = (int)(tok - (uint32_t)b * (uint32_t)a.T);
  const float* cs = nullptr;
  if (PAIR != kPairNone) {
    const int p = a.pos[b * a.sp_b + t];
    if (p < 0 || p >= a.table_rows) return;  // no such position: the token's rows stay as they are
    cs = a.cos_sin + (int64_t)p * a.R;
  }
  const Turn turn = token_turn<PAIR>(cs, a.R);
  const int nq = (a.q.H + kPassRows - 1) / kPassRows, nk = (a.k.H + kPassRows - 1) / kPassRows;
  const int p0 = (int)(wave - tok * (uint32_t)parts) * per, p1 = min(nq + nk, p0 + per);
  if (p0 < nq)
    turn_heads<PAIR, PER_HEAD, STREAM>(a.q.in + b * a.q.si_b + t * a.q.si_t, a.q.si_h, a.q.out + b * a.q.so_b + t * a.q.so_t,
                               a.q.so_h, a.q.w, a.q.sw_h, a.eps, turn, a.q.H, p0, min(p1, nq));
  if (p1 > nq)
    turn_heads<PAIR, PER_HEAD, STREAM>(a.k.in + b * a.k.si_b + t * a.k.si_t, a.k.si_h, a.k.out + b * a.k.so_b + t * a.k.so_t,
                               a.k.so_h, a.k.w, a.k.sw_h, a.eps, turn, a.k.H, max(p0 - nq, 0), p1 - nq);
}

// Passes per wavefront: all of a token's, or while the wavefronts are few, down
// to one (a wavefront per SIMD and more hide each other's latency).
static int passes_per_wave(int64_t tokens, int passes) {
  int per = passes;
  while (per > 1 && tokens * ((passes + per - 1) / per) < 4096) per = (per + 1) / 2;
  return per;
}

static Pairing pairing_of(int R, int inter) {
  return R == 0 ? kPairNone : inter ? kPairAdjacent : R == kHeadDim ? kPairEight : kPairLanes;
}

#define BPC_BY_PAIRING(KERNEL, ...)                             \
  switch (pairing_of(a.R, a.inter)) {                           \
    case kPairNone: KERNEL(kPairNone, __VA_ARGS__) break;         \
    case kPairEight: KERNEL(kPairEight, __VA_ARGS__) break;       \
    case kPairLanes: KERNEL(kPairLanes, __VA_ARGS__) break;       \
    case kPairAdjacent: KERNEL(kPairAdjacent, __VA_ARGS__) break; \
  }

hipError_t launch_qk_norm_rope(const RopeArgs& a) {
  const int passes = (a.q.H + kPassRows - 1) / kPassRows + (a.k.H + kPassRows - 1) / kPassRows;
  const int64_t tokens = (int64_t)a.B * a.T;
  const int per = passes_per_wave(tokens, passes), parts = (passes + per - 1) / per;
  const unsigned grid = (unsigned)((tokens * parts + kRopeWaves - 1) / kRopeWaves);
  const bool per_head = (a.q.w && a.q.sw_h) || (a.k.w && a.k.sw_h);
  // More rows than the last-level cache (256 MB) could hold for their reader pass
  // it by: 32749 tokens of 40 heads (335 MB out) 136 and 124 us.
  const bool stream = tokens * (a.q.H + a.k.H) * (kHeadDim * 2) > (int64_t)256 << 20;
#define BPC_QK(PAIR, PER_HEAD, STREAM) \
  qk_norm_rope_kernel<PAIR, PER_HEAD, STREAM><<<grid, kRopeThreads, 0, a.stream>>>(a, per, parts);
  if (per_head) {
    if (stream) BPC_BY_PAIRING(BPC_QK, true, true) else BPC_BY_PAIRING(BPC_QK, true, false)
  } else {
    if (stream) BPC_BY_PAIRING(BPC_QK, false, true) else BPC_BY_PAIRING(BPC_QK, false, false)
  }
#undef BPC_QK
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// append_kv_paged: as above, the key heads (normed and rotated) before the
// value heads (copied), stored at the token's row of its page
// ---------------------------------------------------------------------------
template <Pairing PAIR, bool PER_HEAD>
__global__ __launch_bounds__(kRopeThreads) void append_paged_kernel(AppendPagedArgs a, int per, int parts) {
  const uint32_t wave = blockIdx.x * kRopeWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t tok = wave / (uint32_t)parts;
  if (tok >= (uint32_t)a.B * (uint32_t)a.T) return;
  const int b = (int)(tok / (uint32_t)a.T), t = (int)(tok - (uint32_t)b * (uint32_t)a.T);
  if (a.count && t >= a.count[b]) return;
  const int64_t slot = (int64_t)a.pos[b] + t;
  if (slot < 0 || (slot >> a.page_shift) >= a.max_pages) return;
  const int page = a.table[b * a.st_b + (slot >> a.page_shift)];
  if (page < 0 || page >= a.num_pages) return;
  const int64_t row = slot & ((1 << a.page_shift) - 1);
  const float* cs = nullptr;
  if (PAIR != kPairNone) {
    const int64_t p = a.rope_pos ? a.rope_pos[b * a.sr_b + t] : slot;
    if (p < 0 || p >= a.table_rows) return;
    cs = a.cos_sin + p * a.R;
  }
  const int n = (a.Hkv + kPassRows - 1) / kPassRows;
  const int p0 = (int)(wave - tok * (uint32_t)parts) * per, p1 = min(2 * n, p0 + per);
  if (p0 < n)
    turn_heads<PAIR, PER_HEAD, false>(a.kn + b * a.skn_b + t * a.skn_t, a.skn_h, a.K + page * a.sK_p + row * a.sK_n, a.sK_h,
                               a.wk, a.sw_h, a.eps, token_turn<PAIR>(cs, a.R), a.Hkv, p0, min(p1, n));
  if (p1 > n)
    move_heads<false>(a.vn + b * a.svn_b + t * a.svn_t, a.svn_h, a.V + page * a.sV_p + row * a.sV_n, a.sV_h, a.Hkv, max(p0 - n, 0),
               p1 - n, [](const uint4& x, int) { return x; });
}

hipError_t launch_append_paged(const AppendPagedArgs& a) {
  const int passes = 2 * ((a.Hkv + kPassRows - 1) / kPassRows);
  const int64_t tokens = (int64_t)a.B * a.T;
  const int per = passes_per_wave(tokens, passes), parts = (passes + per - 1) / per;
  const unsigned grid = (unsigned)((tokens * parts + kRopeWaves - 1) / kRopeWaves);
#define BPC_APPEND(PAIR, PER_HEAD) append_paged_kernel<PAIR, PER_HEAD><<<grid, kRopeThreads, 0, a.stream>>>(a, per, parts);
  if (a.wk && a.sw_h) {
    BPC_BY_PAIRING(BPC_APPEND, true)
  } else {
    BPC_BY_PAIRING(BPC_APPEND, false)
  }
#undef BPC_APPEND
  return hipGetLastError();
}
#undef BPC_BY_PAIRING

}  // namespace bpc
