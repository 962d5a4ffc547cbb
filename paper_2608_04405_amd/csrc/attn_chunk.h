// Attention of a chunk of new tokens, over one kind of cache: the kernel for many
// rows, and the launches.
#pragma once
#include "attn_kernel.h"

namespace bpc {

// Eight row blocks of 32 rows a workgroup, a wavefront each, two wavefronts a SIMD:
// tiles, operands and statistics as in attn_kernel, but a wavefront's work on a tile
// is in two parts, products (O^T += V^T P^T of the tile before, S^T = K Q^T of this
// one) and softmax, with a barrier behind each, and one half of the wavefronts is
// one barrier behind the other.  So a SIMD's two wavefronts are never in the same
// part: one's products run beside the other's exponentials, where attn_kernel's run
// almost in turn.  A wavefront sends off its share of tile t + 3 between the products of t and
// waits for it at those of t + 2, so that even pages from memory, in any
// order, are there in time (and scalar arithmetic, 50 instructions a tile for pages, runs
// beside the matrix unit; before the exponentials it cost 26 %).  Where wavefronts 0-3
// are at the products of t + 1, the others are at the softmax of t and then at t + 1: V of
// t and all from there to t + 4 are in use, five buffers, and four of K.
//
// Measured with 32 heads (8 KV heads), attn_kernel's time with as many row blocks
// first; matrix units and other vector instructions as shares of the cycles:
//   2048 tokens of 2 requests over 32768 slots in pages of 64: 1.73 -> 1.25 ms, 1.0
//   PFLOP/s of visible pairs; 45 and 36 to 42 %, compute units busy 89 %, at the clock
//   (1.8 GHz) that the power limit leaves
//   1000 tokens of 2 requests over 16384 slots, cap and bias: 0.76 -> 0.49 ms; 25 and 44
//   to 54 %, compute units busy 75 % (the last round of pieces is not full)
//   8001 tokens, window 1024 and 16 first slots: 0.24 -> 0.20 ms; 30 and 27 to 31 %: a
//   third of a row block's 19 tiles are masked in part, and each block begins anew
constexpr int kPairRows = 8 * kBlockRows;
constexpr int kPairKeys = 64;
constexpr int kPairTile = kPairKeys * kRowBytes;
constexpr int kPairLds = 9 * kPairTile;

// What a workgroup does: a row block of a piece of the slots of one KV head.
struct PairItem {
  int bh, b, h, split, rb;
};
template <typename Args>
__device__ __forceinline__ PairItem pair_item(const Args& a) {
  const FastDiv by_nrb{a.div_nrb.mul, a.div_nrb.shift}, by_bh{a.div_bh.mul, a.div_bh.shift}, by_Hkv{a.div_Hkv.mul, a.div_Hkv.shift};
  const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3;
  PairItem x{-1, 0, 0, 0, 0};
  int piece;
  if (a.rounds) {
    const int round = by_nrb.quotient(turn);
    x.rb = a.nrb - 1 - (turn - round * a.nrb), piece = round * 8 + xcd;
    if (piece * a.nrb >= a.items) return x;
  } else {
    const int per = (a.items + 7) >> 3, item = xcd * per + turn;
    if (item >= a.items || turn >= per) return x;
    piece = by_nrb.quotient(item), x.rb = a.nrb - 1 - (item - piece * a.nrb);
  }
  x.split = by_bh.quotient(piece), x.bh = piece - x.split * a.B * a.Hkv;
  x.b = by_Hkv.quotient(x.bh), x.h = x.bh - x.b * a.Hkv;
  return x;
}

template <bool paged, bool CAP, bool BIAS, bool LSE>
__global__ __launch_bounds__(512, 2) void chunk_rows_kernel(AttnArgs a) {
  constexpr int KT = kPairKeys, NB = KT / 32, RPW = KT / 8;
  constexpr int kShare = 2 * RPW / 4;  // copies of a wavefront for a tile
  extern __shared__ __attribute__((aligned(256))) char pair_tiles[];
  __shared__ uint64_t odd_rows[5][8];
  const PairItem item = pair_item(a);
  if (item.bh < 0) return;
  const int b = item.b, h = item.h;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool behind = wid >= 4;
  const int half = lane >> 5, col = lane & 31;
  const int G = a.G;
  const int first = uniform_load(a.lens + b);
  const int rows = chunk_tokens(a, b, first) * G;
  const int wg_row0 = item.rb * kPairRows;
  if (wg_row0 >= rows) return;  // these rows stay as they are
  const ChunkSlots slots = chunk_slots(a, a.div_G, first, rows, wg_row0, kPairRows, KT);
  const int khi = slots.end, wg_all_hi = slots.p0 + 1, wg_all_lo = a.window ? max(0, slots.p1 - a.window + 1) : 0;
  const int it0 = item.split * a.unit, it1 = min(slots.tiles, it0 + a.unit);
  if (it0 >= slots.tiles) return;
  auto tile_key = [&](int it) { return (it < slots.near ? it : it + slots.gap) * KT; };
  auto kbuf = [&](int it) { return (uint32_t)((it - it0) & 3) * kPairTile; };
  int v5 = 0;  // V of tile `it` of the loop lies in this one of five buffers, that of it + k in vslot(k)
  auto vslot = [&](int k) {
    const int x = v5 + k;
    return k < 0 ? (x < 0 ? x + 5 : x) : (x >= 5 ? x - 5 : x);
  };

  const uint32_t ldsK = (uint32_t)(uintptr_t)(lds_char*)pair_tiles, ldsV = ldsK + 4 * kPairTile;
  const char* Kb = reinterpret_cast<const char*>(a.K + (paged ? 0 : b * a.sK_b) + h * a.sK_h);
  const char* Vb = reinterpret_cast<const char*>(a.V + (paged ? 0 : b * a.sV_b) + h * a.sV_h);
  const uint32_t kstep = (uint32_t)a.sK_n * 2, vstep = (uint32_t)a.sV_n * 2;
  const int64_t kpage = paged ? a.sK_b * 2 : 0, vpage = paged ? a.sV_b * 2 : 0;
  const uint32_t pmask = (1u << a.page_shift) - 1;
  const int r4 = lane >> 4;
  uint32_t chunk[RPW / 4], koff[RPW / 4], voff[RPW / 4];
#pragma unroll
  for (int i = 0; i < RPW / 4; ++i) {
    chunk[i] = (((uint32_t)lane & 15u) ^ swz((uint32_t)(wid * RPW + 4 * i + r4))) * 16;
    koff[i] = (4 * i + r4) * kstep + chunk[i];
    voff[i] = (4 * i + r4) * vstep + chunk[i];
  }
  // 64 page entries at a time, a lane each, one per 16, 32 or 64 slots: looked up a
  // tile before they are needed
  const int per_entry = paged ? min(a.page_shift, 6) : 6;        // (log2 of the slots)
  const int ahead = 1 << per_entry;                              // tiles whose entries a wavefront holds
  uint32_t entry = 0, next_entry = 0;
  uint64_t entry_bad = 0;
  auto fetch_entries = [&](int it) {
    const int n = min(tile_key(it + (lane >> (6 - per_entry))) + ((lane << per_entry) & (KT - 1)), khi - 1);
    const LateArgs la = late_args();
    next_entry = (uint32_t)la->table[b * la->st_b + (n >> la->page_shift)];
  };
  auto take_entries = [&]() {
    const bool bad = next_entry >= (uint32_t)late_args()->num_pages;
    entry_bad = __ballot(bad), entry = bad ? 0u : next_entry;
  };
  auto entry_of = [&](int it, int n) { return ((it - it0) & (ahead - 1)) << (6 - per_entry) | n >> per_entry; };  // slot n of the tile
  auto bad_of = [&](int it) {  // a bit per 16 slots
    uint32_t bad = 0;
    if (paged && entry_bad) {
#pragma unroll
      for (int u = 0; u < KT / 16; ++u) bad |= (uint32_t)(entry_bad >> entry_of(it, 16 * u) & 1) << u;
    }
    return bad;
  };
  // where slot nu, the wavefront's first of tile `it`, lies in K and V
  struct Source {
    const char *k, *v;
  };
  auto locate = [&](int it, int nu) {
    Source x;
    if (paged) {
      const uint32_t page = (uint32_t)__builtin_amdgcn_readlane((int)entry, entry_of(it, wid * RPW));
      const uint32_t at = (uint32_t)nu & pmask;
      x.k = Kb + (page * kpage + (int64_t)at * kstep), x.v = Vb + (page * vpage + (int64_t)at * vstep);
    } else {
      x.k = Kb + (int64_t)(uint32_t)nu * kstep, x.v = Vb + (int64_t)(uint32_t)nu * vstep;
    }
    x.k = reinterpret_cast<const char*>(uniform64(reinterpret_cast<uint64_t>(x.k)));
    x.v = reinterpret_cast<const char*>(uniform64(reinterpret_cast<uint64_t>(x.v)));
    return x;
  };
  const uint32_t wave_rows = wid * RPW * kRowBytes;
  auto copy_k = [&](const char* from, int it) {
    const uint32_t dk = ldsK + kbuf(it) + wave_rows;
#pragma unroll
    for (int i = 0; i < RPW / 4; ++i) dma16<false>(from, koff[i], dk + 4 * i * kRowBytes);
  };
  auto copy_v = [&](const char* from, int slot) {
    const uint32_t dv = ldsV + slot * kPairTile + wave_rows;
#pragma unroll
    for (int i = 0; i < RPW / 4; ++i) dma16<false>(from, voff[i], dv + 4 * i * kRowBytes);
  };
  auto issue = [&](int it, int slot) {
    const int nu = min(tile_key(it) + wid * RPW, khi - 1);
    const Source x = locate(it, nu);
    const int last = khi - 1 - nu;  // last row that may be read, from there on
    if (last >= RPW - 1) {
      copy_k(x.k, it), copy_v(x.v, slot);
    } else {
      const uint32_t dk = ldsK + kbuf(it) + wave_rows, dv = ldsV + slot * kPairTile + wave_rows;
#pragma unroll
      for (int i = 0; i < RPW / 4; ++i) {
        const uint32_t r = min(4 * i + r4, last);
        dma16<false>(x.k, r * kstep + chunk[i], dk + 4 * i * kRowBytes);
        dma16<false>(x.v, r * vstep + chunk[i], dv + 4 * i * kRowBytes);
      }
    }
  };

  if (paged) fetch_entries(it0), take_entries();

  // ---- this lane's row ------------------------------------------------------
  const int row = wg_row0 + wid * kBlockRows + col;
  const bool live = row < rows;
  const int t = live ? a.div_G.quotient(row) : 0, g = live ? row - t * G : 0;
  const int place = first + t;
  // rows past the last see everything: they never make a tile partial
  const int lo = !live ? INT32_MIN : a.window ? max(0, place - a.window + 1) : 0, hi = live ? place + 1 : INT32_MAX;
  const int all_lo = wave_max(lo), all_hi = wave_min(hi);
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
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (it0 + i < it1) issue(it0 + i, i);
#pragma unroll
  for (int s = 0; s < 8; ++s) asm volatile("" : "+v"(qf[s]));

  f32x16 o[4], acc[NB];
#pragma unroll
  for (int d = 0; d < 4; ++d) {
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  }
#pragma unroll
  for (int k = 0; k < NB; ++k) acc[k] = f32x16{};
  u32x4 pw[NB][2];
#pragma unroll
  for (int k = 0; k < NB; ++k) pw[k][0] = pw[k][1] = u32x4{0, 0, 0, 0};
  // maximum, what a score has to exceed to move it, reference point (log2), sums
  float mrun = -INFINITY, limit = -INFINITY, mu = 0.f, lsum = 0.f, esum = 0.f;

  // operand s of a key block lies 2 s chunks on from kaddr, in exclusive or, and that
  // of 32 coordinates d of V 4 d chunks from vaddr, its second half 2 chunks from its first
  const uint32_t kaddr = ldsK + col * kRowBytes + (swz(col & 15) ^ half) * 16;
  const uint32_t i16 = lane & 15, vrow = 4 * half + (i16 >> 2);
  const uint32_t vaddr = ldsV + vrow * kRowBytes + ((2 * (r4 & 1) + ((i16 & 3) >> 1)) ^ swz(vrow)) * 16 + (i16 & 1) * 8;
  const float c1 = log2_units<CAP>(a.sm_scale), c8 = 8.f / c1;
  const float cap2 = a.softcap * kLog2e, capk = CAP ? 2.f * kLog2e * a.sm_scale / a.softcap : 0.f;
  auto visible = [&](int n, int sinks) { return (n >= lo || n < sinks) && n < hi; };

  // O^T += V^T P^T of the tile whose probabilities are in pw, 16 keys at a time
  bf16x8 operand[2][4];
  auto read_v = [&](int slot, int keys) {
    const uint32_t v0 = vaddr + slot * kPairTile, at = 16 * keys * kRowBytes;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const uint32_t x = opaque(v0 ^ 64u * d);
      operand[keys & 1][d] = __builtin_bit_cast(
          bf16x8, __builtin_shufflevector(lds_read_tr(x, at), lds_read_tr(x ^ 32u, at + 8 * kRowBytes), 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };
  auto product_v = [&](int keys) {
    const bf16x8 pf = __builtin_bit_cast(bf16x8, pw[keys / 2][keys % 2]);
#pragma unroll
    for (int d = 0; d < 4; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand[keys & 1][d], pf, o[d], 0, 0, 0);
  };
  auto product_k = [&](int it) {
    uint32_t ka[8];
    const uint32_t k0 = kaddr + kbuf(it);
#pragma unroll
    for (int i = 0; i < 8; ++i) ka[i] = opaque(k0 ^ 32u * i);
#pragma unroll
    for (int k = 0; k < NB; ++k) {
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const bf16x8 kf = __builtin_bit_cast(bf16x8, lds_read<u32x4>(ka[s], k * 32 * kRowBytes));
        acc[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], s ? acc[k] : f32x16{}, 0, 0, 0);
      }
    }
  };
  // values of V that clear_odd() took out of tile `it`
  auto add_odd = [&](int it, int slot) {
    const int n0 = tile_key(it);
    uint64_t odd = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) odd |= odd_rows[slot][w];
    odd = uniform64(odd);
    while (odd) {
      const int i = __ffsll((long long)odd) - 1, n = n0 + i;
      odd &= odd - 1;
      if (n >= khi) continue;
      const LateArgs la = late_args();
      const char* vr = Vb + n * la->sV_n * 2;
      if (paged) {
        const uint32_t pg = (uint32_t)uniform_load(la->table + b * la->st_b + (n >> la->page_shift));
        if (pg >= (uint32_t)la->num_pages) continue;
        vr = Vb + (pg * la->sV_b + (n & ((1 << la->page_shift) - 1)) * la->sV_n) * 2;
      }
      const bool see = visible(n, la->sinks);
#pragma unroll
      for (int c = 0; c < 16; ++c) {  // coordinates 8 c + 4 half + 0..3
        const u32x2 x = *reinterpret_cast<const u32x2*>(vr + 16 * c + 8 * half);
        const uint32_t w[4] = {x[0] << 16, x[0] & 0xFFFF0000u, x[1] << 16, x[1] & 0xFFFF0000u};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (see && (w[e] & 0x7F800000u) == 0x7F800000u) o[c / 4][4 * (c % 4) + e] += __uint_as_float(w[e]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  auto softmax = [&](int n0, uint32_t bad, bool plain) {
    // every row sees every key
    const bool full = plain || ((n0 >= all_lo || n0 + KT <= late_args()->sinks) && n0 + KT <= all_hi && !bad);
    const int nl = n0 + 4 * half;  // key of score e of block k: nl + 32 k + 8 (e / 4) + e % 4
    if (CAP || BIAS) {
      const float ahead = (float)(place - nl);
#pragma unroll
      for (int k = 0; k < NB; ++k) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float z = acc[k][e];
          // in units of log2: cap tanh(x) = cap - 2 cap / (1 + e^2x)
          if (CAP) z = fmaf(-2.f * cap2, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * capk)), cap2);
          if (BIAS) z = fmaf(-slope, fabsf(ahead - (float)(32 * k + 8 * (e / 4) + e % 4)), z);
          acc[k][e] = z;
        }
      }
    }
    if (!full) {
      // (two scores at a time: the compiler would hold all 32 masks at once, and
      // everything else in scratch registers)
      const int until = min(hi, khi), sinks = min(late_args()->sinks, until);
      const uint32_t span = (uint32_t)until - (uint32_t)lo;
#pragma unroll
      for (int k = 0; k < NB; ++k) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int n = nl + 32 * k + 8 * (e / 4) + e % 4;
          const float z = (uint32_t)n - (uint32_t)lo < span ? acc[k][e] : -INFINITY;
          acc[k][e] = n < sinks ? acc[k][e] : z;
          if (e & 1) __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (paged && bad) {
#pragma unroll
        for (int k = 0; k < NB; ++k) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            if (bad >> (2 * k + u) & 1) {
#pragma unroll
              for (int e = 0; e < 8; ++e) acc[k][8 * u + e] = -INFINITY;
            }
          }
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
    // as in attn_kernel: the reference point moves only when a score lies more than
    // 2^8 above it
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
  };

  // x, as a value that is computed where it is used: scalar registers are few in the loop
  auto here = [](int x) {
    asm volatile("" : "+s"(x));
    return x;
  };
  // Values of V that are not finite leave a tile that some row sees in part, as in
  // attn_kernel; a wavefront does this for the rows that it copied.
  auto clear_odd = [&](int slot) {
    uint64_t rows_odd = 0;
    const int w = here(wid);
#pragma unroll
    for (int i = 0; i < RPW / 4; ++i) {
      const uint32_t at = ldsV + slot * kPairTile + (w * RPW + 4 * i) * kRowBytes + 16 * lane;
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
          if ((lanes >> (16 * r)) & 0xFFFFu) rows_odd |= 1ull << (w * RPW + 4 * i + r);
      }
    }
    return rows_odd;
  };
  auto is_partial = [&](int n0, uint32_t bad) { return n0 + KT > wg_all_hi || (n0 < wg_all_lo && n0 + KT > late_args()->sinks) || bad; };
  // this wavefront's share of tile `it`, the last but one that it copied, there and cleared
  auto arrive = [&](int it, uint32_t bad, int slot) {
    if (it + 1 < it1) dma_wait<kShare>();
    else dma_wait<0>();
    if (it < it1 && is_partial(tile_key(it), bad)) {
      const uint64_t odd = clear_odd(slot);
      if ((lane ^ here(0)) == 0) odd_rows[slot][wid] = odd;
    }
  };
  auto meet = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" : : : "memory");
  };
  auto copy_ahead = [&](int it) {  // tile `it`, and the entries of the next; its bad pages
    if (paged && ((it - it0) & (ahead - 1)) == 0) take_entries();
    const uint32_t bad = bad_of(it);
    if (it < it1) issue(it, vslot(3));
    if (paged && ((it + 1 - it0) & (ahead - 1)) == 0) fetch_entries(it + 1);
    return bad;
  };
  // The end of the run of tiles from `it` on that all rows of the workgroup see
  // wholly, whose slots follow one another and whose entries are held.
  auto run_end = [&](int it) {
    int e;
    if (it < slots.near) {
      e = min(slots.near, min(late_args()->sinks, wg_all_hi) / KT);
    } else {
      e = (it + slots.gap) * KT >= wg_all_lo ? min(it1, wg_all_hi / KT - slots.gap) : it;
    }
    if (paged) e = entry_bad ? it : min(e, ((it - it0) | (ahead - 1)) + it0);
    return e;
  };

  // The tile before the first: probabilities and values of zero.
#pragma unroll
  for (int i = 0; i < RPW / 4; ++i)
    *(__attribute__((address_space(3))) u32x4*)(lds_char*)(ldsV + 4 * kPairTile + (wid * RPW + 4 * i) * kRowBytes + 16 * lane) = u32x4{0, 0, 0, 0};
  uint32_t bad[3] = {bad_of(it0), bad_of(it0 + 1), bad_of(it0 + 2)};  // of this tile and the next
  if (it0 + 2 < it1) dma_wait<2 * kShare>();
  else dma_wait<0>();
  if (is_partial(tile_key(it0), bad[0])) {
    const uint64_t odd = clear_odd(0);
    if (lane == 0) odd_rows[0][wid] = odd;
  }
  lds_done();
  meet();
  if (behind) meet();
  read_v(vslot(-1), 0);
  bool partial_last = false;  // of the tile before
  int run = it0;
  for (int it = it0; it < it1; ++it) {
    const int n0 = tile_key(it);
    // Tiles that need no masks, and three more behind them that need none, most of
    // them, go without the bookkeeping of the others.
    if (it >= run) run = run_end(it) - 3;
    const bool plain = it < run;
    // ---- products; the copies, and where from, beside them
    __builtin_amdgcn_s_setprio(1);
    read_v(vslot(-1), 1);
    product_v(0);
    const Source from = locate(it + 3, n0 + 3 * KT + wid * RPW);  // (used where this lies before khi)
    if (plain) copy_k(from.k, it + 3);
    read_v(vslot(-1), 2);
    product_v(1);
    if (plain) copy_v(from.v, vslot(3));
    read_v(vslot(-1), 3);
    product_v(2);
    product_v(3);
    product_k(it);
    // operands are read eight, then four products ahead
    __builtin_amdgcn_sched_group_barrier(kSchedLds, 8, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kSchedLds, 1, 0);
    }
#pragma unroll
    for (int i = 0; i < 12; ++i) {
      __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kSchedLds, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kSchedMfma, 8, 0);
    __builtin_amdgcn_s_setprio(0);
    if (partial_last) add_odd(it - 1, vslot(-1));
    if (plain) dma_wait<2 * kShare>();
    else arrive(it + 1, bad[1], vslot(1));
    lds_done();
    meet();
    // ---- softmax
    const uint32_t bad_here = bad[0];
    bad[0] = bad[1], bad[1] = bad[2];
    if (!plain) bad[2] = copy_ahead(it + 3);
    softmax(n0, bad_here, plain);
    partial_last = !plain && is_partial(n0, bad_here);
    read_v(v5, 0);
    v5 = vslot(1);
    meet();
  }
  if (!behind) meet();
#pragma unroll
  for (int keys = 0; keys < 4; ++keys) {
    if (keys) read_v(vslot(-1), keys);
    product_v(keys);
  }
  if (partial_last) add_odd(it1 - 1, vslot(-1));

  // ---- results ---------------------------------------------------------------
  lsum = sum_halves(lsum);
  if (LSE) esum = sum_halves(esum);
  // (where the workgroup is, found again: scalar registers are few in the loop)
  const LateArgs la = late_args();
  const PairItem end = pair_item(*la);
  const FastDiv by_G{la->div_G.mul, la->div_G.shift};
  const int end_first = uniform_load(la->lens + end.b), end_rows = chunk_tokens(*la, end.b, end_first) * la->G;
  const int end_row = end.rb * kPairRows + wid * kBlockRows + col;
  const bool joined = chunk_slots(*la, by_G, end_first, end_rows, end.rb * kPairRows, kPairRows, KT).tiles > la->unit;
  if (end_row >= end_rows) return;
  const int d0 = 4 * half;
  if (joined) {
    const int64_t at = ((int64_t)end.bh * (la->T * la->G) + end_row) * la->splits + end.split;
    if (d0 == 0) la->part_ml[at] = make_float2(mrun, lsum);
    if (LSE && d0 == 0) la->part_e[at] = esum;
    if (lsum == 0.f) return;
    float* po = la->part_o + at * kHeadDim + d0;
#pragma unroll
    for (int c = 0; c < 16; ++c)
      *reinterpret_cast<float4*>(po + 8 * c) = make_float4(o[c / 4][4 * (c % 4)], o[c / 4][4 * (c % 4) + 1], o[c / 4][4 * (c % 4) + 2], o[c / 4][4 * (c % 4) + 3]);
    return;
  }
  const float inv = lsum == 0.f ? 0.f : 1.f / lsum;  // a row that sees no key: zeros
  const int end_t = by_G.quotient(end_row), head = end.h * la->G + end_row - end_t * la->G;
  if (LSE && d0 == 0)
    la->lse[end.b * la->sl_b + head * la->sl_h + end_t] = log_of_sum<CAP>(mrun, esum, log2_units<CAP>(la->sm_scale));
  uint16_t* op = la->out + end.b * la->so_b + head * la->so_h + end_t * la->so_t + d0;
#pragma unroll
  for (int c = 0; c < 16; ++c)
    *reinterpret_cast<uint2*>(op + 8 * c) = make_uint2(cvt_pk_bf16(o[c / 4][4 * (c % 4)] * inv, o[c / 4][4 * (c % 4) + 1] * inv),
                                                       cvt_pk_bf16(o[c / 4][4 * (c % 4) + 2] * inv, o[c / 4][4 * (c % 4) + 3] * inv));
}

template <bool paged, bool LSE>
static hipError_t launch_chunk_rows(AttnArgs a) {
  const int nrb = (a.T * a.G + kPairRows - 1) / kPairRows, items = a.B * a.Hkv * nrb * a.splits;
  a.nrb = nrb, a.items = items, a.div_nrb = FastDiv::by(nrb);
  const int grid = a.rounds ? (items / nrb + 7) / 8 * 8 * nrb : (items + 7) / 8 * 8;
#define BPC_ROWS(CAP, BIAS)                                                                                          \
  {                                                                                                                  \
    auto* f = chunk_rows_kernel<paged, CAP, BIAS, LSE>;                                                              \
    static std::atomic<uint64_t> allowed{0};                                                                         \
    if (hipError_t e = allow_lds(reinterpret_cast<const void*>(f), kPairLds, allowed); e != hipSuccess) return e;    \
    f<<<grid, 512, kPairLds, a.stream>>>(a);                                                                         \
  }
  if (a.softcap > 0.f) {
    if (a.slopes) BPC_ROWS(true, true) else BPC_ROWS(true, false)
  } else {
    if (a.slopes) BPC_ROWS(false, true) else BPC_ROWS(false, false)
  }
#undef BPC_ROWS
  return hipGetLastError();
}

template <AttnKind KIND, bool LSE>
static hipError_t launch_chunk_lse(const AttnArgs& a, const AttnPlan& p) {
  if (p.rb == 1) return p.once ? launch_attn_shape<1, 4, 32, KIND, true, LSE>(a) : launch_attn_shape<1, 4, 32, KIND, false, LSE>(a);
  if (p.rb == 4) return launch_attn_shape<4, 1, 64, KIND, false, LSE>(a);
  return launch_chunk_rows<KIND == kPagedChunk, LSE>(a);
}

template <AttnKind KIND>
static hipError_t launch_chunk_as(const AttnArgs& a, const AttnPlan& p) {
  return a.lse ? launch_chunk_lse<KIND, true>(a, p) : launch_chunk_lse<KIND, false>(a, p);
}

}  // namespace bpc
