// Attention of new tokens over the paged 8-bit cache on gfx950: causal, grouped heads, optional window.
//
// With the codes k, v of a block and its scales sk, sv:  s = scale sk (q . k),  p = exp(s - m),
// out = (sum p sv v) / (sum p): codes go into the matrix instructions as they are, exact in the queries' type (keys) and
// bf16 (values), and the scales into the scores and the weights. One pass over the cache with the running maximum and sum of a
// softmax; statistics and sums in fp32.
//
// k_kv_rows keeps a whole 64-key tile in one wave's registers, without LDS: with S^T = K Q^T and
// O^T = V^T P^T, tile t = 0..3 of 16 keys takes the keys 16 (r / 4) + 4 t + r % 4 as its rows r, so that
// the lanes l / 16 = g end up with the weights of keys 16 g .. 16 g + 15 of their query l % 16: one block
// of the cache, in the order of V's [dim][16] codes, which are the other operand as they lie in memory.
#include <float.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "heads.h"
#include "kv_device.h"

namespace mebp {
namespace {

// Weights are 2^(s - m), m a row's largest score so far and kLift more, at most 1; it moves when a score passes it.
// Those below 2^-126 are 0.
constexpr float kLift = 6.f;
// A weight times its block's scale of values goes into the products as two bf16, the second what the first leaves out:
// 2^-17 of it at any size, so that many small ones beside a large one of small values are all there (in fp16 those
// below 2^-22 of the largest are not). fp32's range takes them and their sums as they are; a row whose scales so far are
// all below kSmall has them over kSmallRef, where theirs have their bits too. (The second products are what bounds
// k_kv_wide: 8 x 2048 tokens, 8 heads of 256, 261 us instead of 249, 12 of 128, 176 instead of 146, 14 of 64, 134 instead
// of 112; k_kv_rows reads in the time of both.)
constexpr float kSmall = 0x1p-20f, kSmallRef = 0x1p-100f;

// A block's scale, an infinite one as NaN: its numbers have none to go by.
DEV float usable(float scale) { return fabsf(scale) < INFINITY ? scale : NAN; }

// (as a scalar, so that what depends on it alone is one)
DEV int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// 16 bytes that are read once (1 GiB of codes in tiles: 6.9 TB/s, 6.0 with ordinary loads)
DEV uint4 stream16(const int8_t* p) {
  typedef uint32_t run __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load((const run*)p));
}

// 8 codes in 2 dwords -> 8 fp16: code + 128 below the bits of 1024, less 1152; exact.
DEV uint4 codes_f16(uint32_t lo, uint32_t hi) {
  const uint32_t a = lo ^ 0x80808080u, b = hi ^ 0x80808080u;
  const f16x2 off = {(f16)1152.0f, (f16)1152.0f};
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u)) - off);
  r.y = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u)) - off);
  r.z = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u)) - off);
  r.w = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)) - off);
  return r;
}

// The same as bf16, the upper halves of their fp32.
DEV uint32_t codes_bf16x2(uint32_t w, int j) {
  const float a = (float)(int8_t)(w >> 8 * j), b = (float)(int8_t)(w >> 8 * (j + 1));
  return perm_hi16(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}
DEV uint4 codes_bf16(uint32_t lo, uint32_t hi) {
  return make_uint4(codes_bf16x2(lo, 0), codes_bf16x2(lo, 2), codes_bf16x2(hi, 0), codes_bf16x2(hi, 2));
}
// Operands of a type T.
template <class T>
using OpOf = typename std::conditional<__is_same(T, f16), OpF16, OpBF16>::type;
template <class T>
DEV uint4 codes_as(uint32_t lo, uint32_t hi) {
  if constexpr (__is_same(T, f16))
    return codes_f16(lo, hi);
  else
    return codes_bf16(lo, hi);
}
// Two numbers as bf16, and what that leaves out of them.
struct TwoParts {
  uint32_t hi, lo;
};
DEV TwoParts two_parts(float a, float b) {
  const uint32_t hi = pack_bf16x2(a, b);
  return TwoParts{hi, pack_bf16x2(a - bf16_lo(hi), b - bf16_hi(hi))};
}

// 64-key tiles [t0, t1) that queries at positions [lo, hi] of a sequence of `len` tokens see
struct Tiles {
  int t0, t1;
};
DEV Tiles tiles_of(int lo, int hi, int window) {
  return Tiles{window ? max(lo - window + 1, 0) >> 6 : 0, (hi >> 6) + 1};
}

// Keys that the query at a position sees, as one unsigned comparison: key - lo <= span.
struct Seen {
  int lo;
  unsigned span;
};
DEV Seen keys_seen(int pos, int window) {
  const int lo = window ? max(pos - window + 1, 0) : 0;
  return Seen{lo, (unsigned)(pos - lo)};
}

// A row's queries as operands of their type, scaled by a power of two towards fp16's end (exact but for elements 2^-140 of
// a bf16 row's largest) and by the sign of `scale`, and what a score is to be multiplied by for it, not negative: NaN
// where the row has a NaN or an infinity.
// at(m): the lane's first element of operand m; LANES: of one row, this many apart.
template <class T>
struct Eight {
  typedef T run __attribute__((ext_vector_type(8)));
};
template <class T, int NF, class At>
DEV void load_queries(const T* p, bool vec, typename Eight<T>::run (&x)[NF], At&& at) {
#pragma unroll
  for (int m = 0; m < NF; ++m) {
    const T* e = p + at(m);
    if (vec) {
      x[m] = *(const typename Eight<T>::run*)e;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[m][i] = e[i];
    }
  }
}
template <class T, int NF, int LANES>
DEV float queries(const typename Eight<T>::run (&raw)[NF], float scale, uint4 (&f)[NF]) {
  float x[NF][8];
#pragma unroll
  for (int m = 0; m < NF; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[m][i] = (float)raw[m][i];
  // (bits of magnitudes are ordered as the magnitudes, infinities and NaN above all)
  uint32_t most = 0;
#pragma unroll
  for (int m = 0; m < NF; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __builtin_bit_cast(uint32_t, x[m][i]) & 0x7fffffffu);
#pragma unroll
  for (int o = LANES; o < 64; o *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, o, 64));
  const bool bad = most >= 0x7f800000u;
  // (by 2^100 at most, so that what takes it back has its bits)
  const int up = most && !bad ? min(15 - ilogbf(__builtin_bit_cast(float, most)), 100) : 0;
#pragma unroll
  for (int m = 0; m < NF; ++m) {
    typename Eight<T>::run r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (T)__builtin_amdgcn_ldexpf(scale < 0.f ? -x[m][i] : x[m][i], up);
    f[m] = __builtin_bit_cast(uint4, r);
  }
  return bad ? NAN : __builtin_amdgcn_ldexpf(fabsf(scale), -up);
}
template <class T, int NF>
DEV float row_queries(const T* p, bool vec, float scale, uint4 (&f)[NF], int g4) {
  typename Eight<T>::run x[NF];
  load_queries<T, NF>(p, vec, x, [&](int m) { return 64 * (m / 2) + 16 * g4 + 8 * (m & 1); });
  return queries<T, NF, 16>(x, scale, f);
}

// Where lengths differ the tiles of all sequences, heads and row tiles (the units) are dealt out in equal
// shares: workgroup w takes places w n .. of the units in their order, and units that more than one share
// has are joined by k_kv_join. (A grid of chunks up to the longest length took 1.5 times as long on 48
// sequences of 1 to 8192 tokens: which compute units get the workgroups that have nothing to do is chance.)
// A unit has kUnitCost places before those of its tiles, for what its start and end take.
constexpr int kUnitCost = 6;
struct KvShare {
  int64_t u0, u1;  // its places
  int64_t base;    // the first place of sequence s, the first that has some of them
  int s;
  KvSeq seq;
};
// Tiles that rows r0 .. r0 + R - 1 of a sequence see.
DEV Tiles row_tiles_of(const KvAttnArgs& a, const KvSeq& q, int r0, int R) {
  return tiles_of(q.past + r0 / a.group, q.past + (min(r0 + R, q.n * a.group) - 1) / a.group, a.window);
}
// Tiles that the rows of one sequence see, and places of its units. (Positions from max_len on have no result, and
// whatever `past` says no work.)
DEV Tiles seq_tiles(const KvAttnArgs& a, const KvSeq& q) {
  return q.n ? tiles_of(min(q.past, a.b.max_len - 1), min(q.past + q.n, a.b.max_len) - 1, a.window) : Tiles{0, 0};
}
DEV int64_t seq_places(const KvAttnArgs& a, const KvSeq& q) {
  const Tiles t = seq_tiles(a, q);
  return q.n ? (int64_t)a.c.heads * a.plan.row_tiles * (t.t1 - t.t0 + kUnitCost) : 0;
}
DEV int64_t share_size(int64_t places, int shares) {
  return max((places + shares - 1) / shares, (int64_t)(4 + kUnitCost));  // (a tile for each wave)
}
// The share of this workgroup, or false where there is none; the first also keeps where sequences begin, in
// a.first [seqs + 1].
DEV bool find_share(const KvAttnArgs& a, KvShare& out) {
  __shared__ int64_t wave_sum[4];
  const int tid = threadIdx.x, per = (a.b.seqs + 255) / 256, s0 = tid * per, s1 = min(s0 + per, a.b.seqs);
  int64_t mine = 0;
  KvSeq q{0, 0, 0};
  for (int s = s0; s < s1; ++s) mine += seq_places(a, q = kv_seq(a.b, s));
  int64_t sum = mine;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int64_t v = __shfl_up(sum, o, 64);
    if ((tid & 63) >= o) sum += v;
  }
  if ((tid & 63) == 63) wave_sum[tid >> 6] = sum;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    before += w < (tid >> 6) ? wave_sum[w] : 0;
    all += wave_sum[w];
  }
  const int64_t first = before + sum - mine, n = share_size(all, a.plan.shares), u0 = blockIdx.x * n;
  if (blockIdx.x == 0 || (u0 >= first && u0 < first + mine)) {
    int64_t at = first;
    for (int s = s0; s < s1; ++s) {
      if (per > 1) q = kv_seq(a.b, s);
      const int64_t c = seq_places(a, q);
      if (blockIdx.x == 0) a.first[s] = at;
      if (u0 >= at && u0 < at + c) out = KvShare{u0, min(u0 + n, all), at, s, q};
      at += c;
    }
  }
  if (blockIdx.x == 0 && tid == 0) a.first[a.b.seqs] = all;
  __syncthreads();
  return u0 < all;
}

// Few rows: one workgroup of 4 waves takes NR * 16 rows (token, head of the group) of one sequence and kv
// head over a chunk of its tiles, the waves one tile of KT keys in four each; their sums meet in LDS.
// D = 256 takes 32 keys at a time, so that two waves fit a SIMD's registers with a tile in flight each.
// Reading bounds it where there is much to read (48 sequences of up to 8192 tokens, 4 heads of 256: 77 us, 5.4 TB/s), else
// the way from the sequence's numbers over the page table to the codes and the scores (6 us for a tile a wave).
template <class T, int D, int NR>
__global__ __launch_bounds__(256, 2) void k_kv_rows(KvAttnArgs a, bool vec) {
  constexpr int NF = D / 32, NK = D / 16, R = 16 * NR;
  constexpr bool QL = D == 256;  // queries in LDS, in the order of the operand (no registers to spare)
  constexpr int KT = D == 256 ? 32 : 64, NT = KT / 16, KL = KT / 4, PT = 64 / KT;  // KL: keys of a lane's scores
  __shared__ float o_lds[4][R][D + 4];
  __shared__ float m_lds[4][R], l_lds[4][R], w_lds[4][R], ref_lds[4][R];
  __shared__ uint4 q_lds[QL ? NR * NF * 64 : 1];
  __shared__ KvShare share_lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id(), r16 = lane & 15, g4 = lane >> 4;
  const int units = a.c.heads * a.plan.row_tiles;
  KvShare sh;
  if (a.plan.shares) {
    if (!find_share(a, share_lds)) return;
    sh = share_lds;
  } else {
    // a chunk of one unit
    sh.s = blockIdx.x / (units * a.plan.splits);
    sh.seq = kv_seq(a.b, sh.s);
    sh.u0 = 0;
    sh.u1 = sh.seq.n ? 1 : 0;
  }
  for (int64_t at = sh.u0; at < sh.u1;) {
  const KvSeq sq = sh.seq;
  const int s = sh.s, rows = sq.n * a.group;
  Tiles range;
  int unit, off, len;
  if (a.plan.shares) {
    range = seq_tiles(a, sq);
    const int nt = range.t1 - range.t0;
    const int64_t rel = at - sh.base, per = nt + kUnitCost;
    if (!sq.n || rel >= units * per) {
      sh.base += seq_places(a, sq);
      if (++sh.s == a.b.seqs) return;
      sh.seq = kv_seq(a.b, sh.s);
      continue;
    }
    unit = (int)(rel / per);
    const int from = (int)(rel - unit * per), to = (int)min(per, from + sh.u1 - at);
    at += to - from;
    off = max(from - kUnitCost, 0);
    len = to - kUnitCost - off;
    if (len <= 0) continue;
  } else {
    unit = (int)(blockIdx.x / a.plan.splits % units);
    if (unit % a.plan.row_tiles * R >= rows) return;
    range = row_tiles_of(a, sq, unit % a.plan.row_tiles * R, R);
    off = blockIdx.x % a.plan.splits * a.plan.chunk;
    len = min(a.plan.chunk, range.t1 - range.t0 - off);
    if (len <= 0) return;
    at = sh.u1;
  }
  const int h = unit / a.plan.row_tiles, r0 = unit % a.plan.row_tiles * R, nt = range.t1 - range.t0;
  if (r0 >= rows) continue;
  // rows behind the last one repeat it
  const int last = min(r0 + R, rows) - 1;
  const int pos_lo = sq.past + r0 / a.group, pos_hi = sq.past + last / a.group;
  const int tb = range.t0 + off, te = tb + len;
  const int nblk = (sq.past + sq.n + 15) >> 4;
  const int k1 = te * PT;  // in tiles of KT keys

  // A tile's pages are looked up two of the wave's tiles ahead of its products, its keys loaded one ahead (into
  // the registers that the scores have just been made from), its values as its scores are made. Blocks: the
  // lane's as a row of the keys' operand (bk), and as a lane of the scores and the values (bv).
  const int kb = KL * (r16 >> 2), vb = KL * g4;
  typedef uint32_t vrun __attribute__((ext_vector_type(KL / 4)));
  int ek, ev, iv_page;
  uint32_t iv;
  uint4 kr[NT * (D / 64)];
  vrun vr[NK];
  auto look_up = [&](int tile) {
    tile = min(tile, k1 - 1) * (KT / 16);
    ek = kv_entry(a.c, a.b, s, min(tile + kb / 16, nblk - 1));
    ev = kv_entry(a.c, a.b, s, min(tile + vb / 16, nblk - 1));
  };
  auto load_keys = [&](int tile) {
    tile = min(tile, k1 - 1) * (KT / 16);
    const int bk = min(tile + kb / 16, nblk - 1), bv = min(tile + vb / 16, nblk - 1);
    const int8_t* kp = a.c.codes + (uint64_t)kv_block(a.c, max(kv_page_of(a.c, a.b, ek, bk), 0), h, bk) * (32 * D) + (kb % 16 + (r16 & 3)) * D + g4 * 16;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int j = 0; j < D / 64; ++j) kr[t * (D / 64) + j] = stream16(kp + t * 4 * D + j * 64);
    iv_page = kv_page_of(a.c, a.b, ev, bv);
    iv = kv_block(a.c, max(iv_page, 0), h, bv);
  };
  int tile = tb * PT + wave;
  look_up(tile);
  load_keys(tile);
  look_up(tile + 4);

  uint4 qf[NR][QL ? 1 : NF];
  float qs[NR];
  Seen see[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int r = min(r0 + n * 16 + r16, last), i = r / a.group, g = r - i * a.group;
    see[n] = keys_seen(sq.past + i, a.window);
    const T* p = (const T*)a.q.p + (int64_t)(sq.row + i) * a.q.ld + (int64_t)(h * a.group + g) * a.q.hld;
    if constexpr (QL) {
      uint4 f[NF];
      qs[n] = row_queries(p, vec, a.scale, f, g4);
      // (every wave has made the same ones)
      if (wave == 0) {
#pragma unroll
        for (int i = 0; i < NF; ++i) q_lds[(n * NF + i) * 64 + lane] = f[i];
      }
    } else {
      qs[n] = row_queries(p, vec, a.scale, qf[n], g4);
    }
  }
  if (QL) __syncthreads();
  auto query = [&](int n, int i) {
    if constexpr (QL)
      return q_lds[(n * NF + i) * 64 + lane];
    else
      return qf[n][i];
  };
  f32x4 acc[NR][NK];
  // As in k_kv_wide, the sums are scaled in an outer loop.
  float m[NR], l[NR], by[NR], ref[NR];  // (the row's sums of values are in units of ref)
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    m[n] = -FLT_MAX;
    l[n] = 0.f;
    by[n] = 1.f;
    ref[n] = kSmallRef;
#pragma unroll
    for (int d = 0; d < NK; ++d) acc[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bool fresh = true;  // (nothing to scale yet)
  bool moved = false;  // m or ref for this tile: once, whatever its numbers are
  while (tile < k1) {
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int d = 0; d < NK; ++d) acc[n][d] *= by[n];
    do {
      const int8_t* vp = a.c.codes + (uint64_t)iv * (32 * D) + 16 * D + r16 * 16 + vb % 16;
      const float2 sc = ((const float2*)a.c.scales)[iv];
#pragma unroll
      for (int d = 0; d < NK; ++d) vr[d] = __builtin_nontemporal_load((const vrun*)(vp + d * 256));
      __builtin_amdgcn_sched_barrier(0);  // (in flight while the scores are made)
      f32x4 sa[NR][NT];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int n = 0; n < NR; ++n) sa[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        uint4 q[NR][2];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          q[n][0] = query(n, 2 * j);
          q[n][1] = query(n, 2 * j + 1);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint4 c = kr[t * (D / 64) + j];
          const uint4 c0 = codes_as<T>(c.x, c.y), c1 = codes_as<T>(c.z, c.w);
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            sa[n][t] = mfma16_raw<OpOf<T>>(c0, q[n][0], sa[n][t]);
            sa[n][t] = mfma16_raw<OpOf<T>>(c1, q[n][1], sa[n][t]);
          }
        }
      }
      // a row's m and ref follow its scores, and the values' scales of the blocks that it sees
      const bool masked = tile * KT + KT - 1 > pos_lo || (a.window && tile * KT <= pos_hi - a.window);
      const float sx = iv_page < 0 ? NAN : usable(sc.x), sb = iv_page < 0 ? NAN : usable(sc.y);
      bool move = false;
      uint64_t large[NR];  // lanes whose block is too large for the row's ref
      float mx[NR], sv[NR];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const float f = sx * qs[n];
        const int k0 = tile * KT + vb - see[n].lo;
        mx[n] = -INFINITY;
        // (0 where the row sees none of the lane's keys)
        sv[n] = masked && (k0 + KL <= 0 || k0 > (int)see[n].span) ? 0.f : sb;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) sa[n][t][i] *= f;
        if (masked) {
#pragma unroll
          for (int k = 0; k < KL; ++k)
            sa[n][k >> 2][k & 3] = (unsigned)(k0 + k) <= see[n].span ? sa[n][k >> 2][k & 3] : -INFINITY;
        }
#pragma unroll
        for (int k = 0; k < KL; ++k) mx[n] = fmaxf(mx[n], sa[n][k >> 2][k & 3]);
        large[n] = __ballot(ref[n] < 1.f && fabsf(sv[n]) > kSmall);
        move |= large[n] || __ballot(mx[n] > m[n]) != 0;
      }
      if (move && !moved) {
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          float x = fmaxf(mx[n], __shfl_xor(mx[n], 16, 64));
          x = fmaxf(x, __shfl_xor(x, 32, 64));
          x = x > m[n] ? x + kLift : m[n];
          const float down = exp2_fast(m[n] - x);
          m[n] = x;
          l[n] *= down;
          const uint64_t l2 = large[n] | large[n] >> 32;  // (of the row's four lanes)
          const bool grow = (l2 | l2 >> 16) >> r16 & 1;
          by[n] = grow ? down * kSmallRef : down;
          ref[n] = grow ? 1.f : ref[n];
        }
        if (!fresh) {
          moved = true;
          break;
        }
      }
      fresh = moved = false;
      load_keys(tile + 4);
      look_up(tile + 8);
      __builtin_amdgcn_sched_barrier(0);
      TwoParts pw[NR][KL / 2];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        // (a scale of NaN: so are the weights of all its keys, in a row that sees one of them)
        const float svr = ref[n] < 1.f ? sv[n] * (1.f / kSmallRef) : sv[n];
#pragma unroll
        for (int k = 0; k < KL; k += 2) {
          const float p0 = exp2_fast(sa[n][k >> 2][k & 3] - m[n]), p1 = exp2_fast(sa[n][k >> 2][(k & 3) + 1] - m[n]);
          l[n] += p0 + p1;
          pw[n][k / 2] = two_parts(p0 * svr, p1 * svr);
        }
      }
#pragma unroll
      for (int d = 0; d < NK; ++d)
#pragma unroll
        for (int u = 0; u < KL / 8; ++u) {
          const uint4 v = codes_bf16(vr[d][2 * u], vr[d][2 * u + 1]);
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            const TwoParts* w = &pw[n][4 * u];
            acc[n][d] = mfma16_raw<OpBF16>(v, make_uint4(w[0].hi, w[1].hi, w[2].hi, w[3].hi), acc[n][d]);
            acc[n][d] = mfma16_raw<OpBF16>(v, make_uint4(w[0].lo, w[1].lo, w[2].lo, w[3].lo), acc[n][d]);
          }
        }
      tile += 4;
    } while (tile < k1);
  }
  // the waves' sums meet: lane holds dims 16 d + 4 g4 .. + 4 of its row
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    l[n] += __shfl_xor(l[n], 16, 64);
    l[n] += __shfl_xor(l[n], 32, 64);
#pragma unroll
    for (int d = 0; d < NK; ++d) *(f32x4*)&o_lds[wave][n * 16 + r16][d * 16 + g4 * 4] = acc[n][d];
    if (g4 == 0) {
      m_lds[wave][n * 16 + r16] = m[n];
      l_lds[wave][n * 16 + r16] = l[n];
      ref_lds[wave][n * 16 + r16] = ref[n];
    }
  }
  __syncthreads();
  if (tid < R) {
    float mm = m_lds[0][tid];
    for (int w = 1; w < 4; ++w) mm = fmaxf(mm, m_lds[w][tid]);
    float ll = 0.f;
    for (int w = 0; w < 4; ++w) {
      const float e = exp2_fast(m_lds[w][tid] - mm);
      ll += e * l_lds[w][tid];
      w_lds[w][tid] = e * ref_lds[w][tid];
    }
    m_lds[0][tid] = mm;
    l_lds[0][tid] = ll;
  }
  __syncthreads();
  // All of the unit's tiles: its rows are done. Else what there is of them is a part: a chunk's, or a share's
  // first or second, the one for a unit that began before it, the other for one that goes on behind it.
  const bool whole = a.plan.shares ? len == nt : a.plan.splits == 1;
  const int64_t part = (a.plan.shares ? (int64_t)blockIdx.x * 2 + (off ? 0 : 1) : (int64_t)blockIdx.x) * a.part_rows;
  for (int i = tid; i < R * (D / 4); i += 256) {
    const int r = i / (D / 4), e = (i % (D / 4)) * 4;
    if (r0 + r > last) continue;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) o += *(const f32x4*)&o_lds[w][r][e] * w_lds[w][r];
    if (!whole) {
      *(f32x4*)(a.part + (part + r) * (D + 4) + e) = o;
      if (e == 0) {
        a.part[(part + r) * (D + 4) + D] = m_lds[0][r];
        a.part[(part + r) * (D + 4) + D + 1] = l_lds[0][r];
      }
      continue;
    }
    const int i_tok = (r0 + r) / a.group, g = (r0 + r) - i_tok * a.group;
    const float ll = l_lds[0][r];
    const float inv = sq.past + i_tok >= a.b.max_len ? NAN : ll == 0.f ? 0.f : 1.f / ll;
    T* p = (T*)a.out.p + (int64_t)(sq.row + i_tok) * a.out.ld + (int64_t)(h * a.group + g) * a.out.hld + e;
    for (int k = 0; k < 4; ++k) p[k] = (T)(o[k] * inv);
    if (e == 0 && a.lse)
      a.lse[(int64_t)(sq.row + i_tok) * a.q_heads + h * a.group + g] =
          sq.past + i_tok >= a.b.max_len ? NAN : (m_lds[0][r] + log2f(ll)) * 0.6931471805599453f;
  }
  __syncthreads();  // (before the next one's sums)
  }
}

// Many rows: one workgroup of 4 waves takes 128 rows, 32 a wave, whose queries and sums stay in registers; the
// waves share tiles of KT keys [KT][D] in the queries' type and values [D][KT] in bf16 in LDS, turned to them once. Products on
// 32x32x16: S^T = K Q^T with row r of 32 as key r with bits 2 and 3 exchanged, so that a lane's 8 results
// are 8 successive keys, the other operand of O^T += V^T P^T. A wave's products and its other work follow one
// another unless they are of different tiles: the scores of tile t + 1 are made beside the weights of t, and
// tile t + 2 is turned to 16 bits beside the output's products of t, with three copies of the tile in LDS.
// 2 x 8192 tokens, 12 heads of 128: 640 TFLOP/s, and 960 with the weights' second products; 8 of 256, whose sums and
// queries leave room for one wave on a SIMD: 620, 1.7 us for 32 keys, of which loading the next tile is a fifth and turning
// it a sixth; before its first tile 5 us; 14 of 64: 520.
DEV int bits23(int r) { return (r & ~12) | (r & 4) << 1 | (r & 8) >> 1; }

template <int D>
struct WideTile {
  static constexpr int KT = D == 64 ? 64 : 32;  // (two sets of scores beside the sums)
  // in 16 bytes: a row of keys, and of values, and one more, an odd number, so that the same column of 16 rows
  // is in 16 bank groups
  static constexpr int KC = D / 8 + 1, VC = KT / 8 + 1;
  uint4 k[KT * KC], v[D * VC];
  float2 sc[KT / 16];
};

// N products in a row, their LDS operands read FA products ahead, and behind each a piece of other work, which
// runs beside it. (The order is held as it is written: left to itself the scheduler puts the products in one
// row, each behind the wait for its own operand, and the other work behind them.)
template <int N, class Read, class Mul, class Other>
DEV void streamed(Read&& read, Mul&& mul, Other&& other) {
  constexpr int FA = 4;
  uint4 f[FA];
#pragma unroll
  for (int i = 0; i < FA; ++i) f[i] = read(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint4 x = f[i % FA];
    mul(i, x);
    if (i + FA < N) f[i % FA] = read(i + FA);
    other(i);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// A wave's 32 rows of D, of which a lane holds four dims of row lane % 32 at a time, value(d, q) those at 32 d + 2 q +
// 4 (lane / 32): through LDS, so that stores are 256 bytes in a row. at(r): where row r goes.
template <class E, int D, class Value, class At>
DEV void rows_out(uint8_t* lds, int n, Value&& value, At&& at) {
  constexpr int RB = D * sizeof(E) < 256 ? D * sizeof(E) : 256, ND = RB / sizeof(E), LR = RB / 16, ST = RB + 16;
  static_assert(32 * ST * 4 <= 3 * sizeof(WideTile<D>), "a wave's rows in its part of the tiles");
  typedef E run __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int p = 0; p < D / ND; ++p) {
#pragma unroll
    for (int d = p * ND / 32; d < (p + 1) * ND / 32; ++d)
#pragma unroll
      for (int q = 0; q < 16; q += 4)
        *(run*)(lds + (lane & 31) * ST + (d * 32 - p * ND + 2 * q + (lane >> 5) * 4) * sizeof(E)) = value(d, q);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < 32 * LR / 64; ++i) {
      const int r = i * (64 / LR) + lane / LR, c = lane % LR * 16;
      uint8_t* to = (uint8_t*)at(r) + p * RB + c;
      const uint4 x = *(const uint4*)(lds + r * ST + c);
      if (r < n) *(uint4*)to = x;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

template <class T, int D>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void k_kv_wide(KvAttnArgs a, bool vec, bool vec_out) {
  using W = WideTile<D>;
  constexpr int KT = W::KT, NU = KT / 32, NB = KT / 16, NF = D / 16, NO = D / 32, NC = KT * D / 4096, R = 128;
  __shared__ W buf[3];
  // Sequences and heads first, so that (where they are a multiple of 8) all row tiles of one run on one XCD and
  // share its L2; the row tiles with the most keys begin. (With a head's row tiles behind one another, on one
  // XCD too, the last head's longest begin late: with one product a weight 2 x 8192 tokens, 12 heads of 128, took 730 us, so 566.)
  const int pairs = a.c.heads * a.b.seqs, pair = blockIdx.x % pairs, x_id = blockIdx.x / pairs;
  const int z = x_id % a.plan.splits, rt = a.plan.row_tiles - 1 - x_id / a.plan.splits, h = pair % a.c.heads, s = pair / a.c.heads;
  const KvSeq sq = kv_seq(a.b, s);
  const int rows = sq.n * a.group, r0 = rt * R;
  if (r0 >= rows) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id(), c32 = lane & 31, hi = lane >> 5;
  const int last = min(r0 + R, rows) - 1;
  const int pos_lo = sq.past + r0 / a.group, pos_hi = sq.past + last / a.group;
  const Tiles range = tiles_of(pos_lo, pos_hi, a.window);
  const int tb = range.t0 + z * a.plan.chunk, te = min(tb + a.plan.chunk, range.t1);
  if (tb >= te) return;
  const int nblk = (sq.past + sq.n + 15) >> 4;
  // in tiles of KT keys
  const int k0 = tb * (64 / KT), k1 = min(te * (64 / KT), pos_hi / KT + 1);

  const int row = min(r0 + wave * 32 + c32, last), tok = row / a.group, pos = sq.past + tok;
  const int w_lo = sq.past + min(r0 + wave * 32, last) / a.group, w_hi = sq.past + min(r0 + wave * 32 + 31, last) / a.group;
  // A tile goes through three stages: its pages looked up, its codes and scales loaded, both turned and
  // written to LDS; a tile's products run beside all three of those behind it.
  // Chunk i of this thread: 16 dims of a key, and 16 keys of a dim of values, of block (tid + 256 i) / D, which is
  // the same for a wave. The scales of a block are written by the first lane of one wave that has it.
  auto block_of = [&](int tile, int i) { return min(tile * NB + (wave * 64 + 256 * i) / D, nblk - 1); };
  const int sc_i = NC > 1 ? wave & 1 : 0, sc_b = NC > 1 ? wave & 1 : wave * 64 / D;
  const bool sc_mine = lane == 0 && (NC > 1 ? wave < 2 : wave * 64 % D == 0);
  struct Raw {
    uint4 k[NC], v[NC];
    float2 sc;
    bool ok;
  } raw;
  struct Entries {
    int e[NC];
  } next_pages;
  auto look_up = [&](int tile) {
    Entries pg;
#pragma unroll
    for (int i = 0; i < NC; ++i) pg.e[i] = kv_entry(a.c, a.b, s, block_of(tile, i));
    return pg;
  };
  auto load = [&](Raw& r, const Entries& pg, int tile) {
    uint32_t at = 0;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int blk = block_of(tile, i), page = kv_page_of(a.c, a.b, __builtin_amdgcn_readfirstlane(pg.e[i]), blk);
      const uint32_t x = kv_block(a.c, max(page, 0), h, blk);
      const int8_t* p = a.c.codes + (uint64_t)x * (32 * D) + (uint32_t)((tid + 256 * i) % D * 16);
      r.k[i] = *(const uint4*)p;
      r.v[i] = *(const uint4*)(p + 16 * D);
      if (i == sc_i) {
        at = x;
        r.ok = page >= 0;
      }
    }
    r.sc = ((const float2*)a.c.scales)[at];
  };
  // piece j of 4 NC
  auto store = [&](W& t, const Raw& r, int j) {
    const int i = j >> 2, key = (tid + 256 * i) / (D / 16), c = (tid + 256 * i) % (D / 16) * 2;
    const int dim = (tid + 256 * i) % D, b = (tid + 256 * i) / D * 2;
    uint4* to = j & 2 ? &t.v[dim * W::VC + b] : &t.k[key * W::KC + c];
    const uint4 x = j & 2 ? r.v[i] : r.k[i];
    const uint32_t y = j & 1 ? x.z : x.x, z = j & 1 ? x.w : x.y;
    to[j & 1] = j & 2 ? codes_bf16(y, z) : codes_as<T>(y, z);
  };
  auto store_scales = [&](W& t, const Raw& r) {
    if (sc_mine) t.sc[sc_b] = r.ok ? make_float2(usable(r.sc.x), usable(r.sc.y)) : make_float2(NAN, NAN);
  };
  auto store_all = [&](W& t, const Raw& r) {
#pragma unroll
    for (int j = 0; j < 4 * NC; ++j) store(t, r, j);
    store_scales(t, r);
  };
  // (behind the last tile: that one again, for nobody)
  auto tile_at = [&](int t) { return min(t, k1 - 1); };
  // (the first three at once, and the queries' own loads beside their pages)
  const Entries e0 = look_up(k0), e1 = look_up(tile_at(k0 + 1)), e2 = look_up(tile_at(k0 + 2));
  next_pages = look_up(tile_at(k0 + 3));
  typename Eight<T>::run qr[NF];
  load_queries<T, NF>((const T*)a.q.p + (int64_t)(sq.row + tok) * a.q.ld + (int64_t)(h * a.group + row - tok * a.group) * a.q.hld,
                      vec, qr, [&](int m) { return 16 * m + 8 * hi; });
  __builtin_amdgcn_sched_barrier(0);
  Raw first, second;
  load(first, e0, k0);
  load(second, e1, tile_at(k0 + 1));
  load(raw, e2, tile_at(k0 + 2));
  uint4 qf[NF];
  const float qs = queries<T, NF, 32>(qr, a.scale, qf);
  store_all(buf[0], first);
  store_all(buf[1], second);
  f32x16 acc[NO];
#pragma unroll
  for (int d = 0; d < NO; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
  const Seen see = keys_seen(pos, a.window);
  float m = -FLT_MAX, l = 0.f, ref = kSmallRef;  // (the row's sums of values are in units of ref)

  auto scores = [&](const W& t, f32x16 (&sa)[NU], auto&& other) {
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) sa[u][i] = 0.f;
    streamed<NU * NF>(
        [&](int i) { return t.k[(i % NU * 32 + bits23(c32)) * W::KC + 2 * (i / NU) + hi]; },
        [&](int i, uint4 x) { sa[i % NU] = mfma32<OpOf<T>>(x, qf[i / NU], sa[i % NU]); }, other);
  };
  f32x16 sn[NU];
  __syncthreads();
  scores(buf[0], sn, [](int) {});
  // The sums are scaled in the outer loop, which a tile whose references have to move falls back to: inside the
  // inner one nothing but the products touches them, so that they stay in the registers of the products
  // (moving 128 of them there and back takes a third of a tile's time).
  float by = 1.f;
  bool moved = false;
  int tile = k0, at = 0;
  float x[NU][16], f[NB], sv[NB];
  bool masked;
  // scores and scales of the tile, and whether m or ref has to move for it
  auto look = [&] {
    const W& t = buf[at];
    float most = 0.f;
    masked = tile * KT + KT - 1 > w_lo || (a.window && tile * KT <= w_hi - a.window);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const float2 sc = t.sc[b];
      f[b] = sc.x * qs;
      // (0 where the row sees none of the block's keys; NaN else makes the weights of all of them NaN)
      const int first = tile * KT + 16 * b - see.lo;
      sv[b] = masked && (first + 16 <= 0 || first > (int)see.span) ? 0.f : sc.y;
      most = fmaxf(most, fabsf(sv[b]));
    }
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[u][i] = sn[u][i] * f[2 * u + (i >> 3)];
    if (masked) {
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = tile * KT + hi * 8 + u * 32 + (i >> 3) * 16 + (i & 7);
          x[u][i] = (unsigned)(key - see.lo) <= see.span ? x[u][i] : -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, x[u][i]);
    const bool grow = ref < 1.f && most > kSmall;
    if (!__ballot(mx > m || grow)) return false;
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float nm = mx > m ? mx + kLift : m, down = exp2_fast(m - nm);
    m = nm;
    l *= down;
    by = grow ? down * kSmallRef : down;
    ref = grow ? 1.f : ref;
    return true;
  };
  look();
  while (tile < k1) {
#pragma unroll
    for (int d = 0; d < NO; ++d) acc[d] *= by;
    do {
      const int at1 = at == 2 ? 0 : at + 1, at2 = at == 0 ? 2 : at - 1;
      TwoParts pw[NU * 8];
      float up[NB], p0;
#pragma unroll
      for (int b = 0; b < NB; ++b) up[b] = ref < 1.f ? sv[b] * (1.f / kSmallRef) : sv[b];
      constexpr int PS = 16 / NF > 1 ? 16 / NF : 1;  // weights to a product
      scores(buf[at1], sn, [&](int j) {
#pragma unroll
        for (int i = j * PS; i < min((j + 1) * PS, NU * 16); ++i) {
          const float p = exp2_fast(x[i >> 4][i & 15] - m);
          l += p;
          if (i & 1)
            pw[i >> 1] = two_parts(p0 * up[i >> 3], p * up[i >> 3]);
          else
            p0 = p;
        }
      });
      const W& t = buf[at];
      constexpr int EV = NO * NB / (4 * NC);  // products to a piece of the tile after the next
      streamed<NO * NB>(
          [&](int i) { return t.v[(i % NO * 32 + c32) * W::VC + 2 * (i / NO) + hi]; },
          [&](int i, uint4 v) {
            const TwoParts* w = &pw[4 * (i / NO)];
            acc[i % NO] = mfma32<OpBF16>(v, make_uint4(w[0].hi, w[1].hi, w[2].hi, w[3].hi), acc[i % NO]);
            acc[i % NO] = mfma32<OpBF16>(v, make_uint4(w[0].lo, w[1].lo, w[2].lo, w[3].lo), acc[i % NO]);
          },
          [&](int i) {
            if (i % EV == 0) store(buf[at2], raw, i / EV);
            if (i == NO * NB - 1) {
              store_scales(buf[at2], raw);
              load(raw, next_pages, tile_at(tile + 3));
              next_pages = look_up(tile_at(tile + 4));
            }
          });
      __syncthreads();
      at = at1;
      if (++tile == k1) break;
      moved = look();
    } while (!moved);
  }
  l += __shfl_xor(l, 32, 64);
  const int n_rows = last + 1 - (r0 + wave * 32);  // (may be none)
  const bool mine = c32 < n_rows;
  uint8_t* lds = (uint8_t*)buf + wave * (sizeof(buf) / 64 * 16);
  if (a.plan.splits > 1) {
    float* p = a.part + (((((int64_t)s * a.c.heads + h) * a.plan.row_tiles + rt) * a.plan.splits + z) * a.part_rows + wave * 32) * (D + 4);
    rows_out<float, D>(
        lds, n_rows, [&](int d, int q) { return f32x4{acc[d][q], acc[d][q + 1], acc[d][q + 2], acc[d][q + 3]} * ref; },
        [&](int r) { return p + r * (D + 4); });
    if (mine && hi == 0) *(float2*)(p + c32 * (D + 4) + D) = make_float2(m, l);
    return;
  }
  const bool beyond = pos >= a.b.max_len;
  const float inv = beyond ? NAN : l == 0.f ? 0.f : ref / l;
  const int hq = h * a.group + row - tok * a.group;
  const int64_t off = (int64_t)(sq.row + tok) * a.out.ld + (int64_t)hq * a.out.hld;
  typedef T run __attribute__((ext_vector_type(4)));
  auto value = [&](int d, int q) { return run{(T)(acc[d][q] * inv), (T)(acc[d][q + 1] * inv), (T)(acc[d][q + 2] * inv), (T)(acc[d][q + 3] * inv)}; };
  if (vec_out) {
    rows_out<T, D>(lds, n_rows, value, [&](int r) { return (T*)a.out.p + __shfl(off, r, 64); });
  } else if (mine) {
#pragma unroll
    for (int d = 0; d < NO; ++d)
#pragma unroll
      for (int q = 0; q < 16; q += 4) {
        const run v = value(d, q);
#pragma unroll
        for (int i = 0; i < 4; ++i) ((T*)a.out.p)[off + d * 32 + 2 * q + 4 * hi + i] = v[i];
      }
  }
  if (mine && hi == 0 && a.lse)
    a.lse[(int64_t)(sq.row + tok) * a.q_heads + hq] = beyond ? NAN : (m + log2f(l)) * 0.6931471805599453f;
}

// Joins the parts of each row with W waves a row, 4 or 1: D / 4 lanes a part, the lanes of the others meeting by
// shuffles and (4) through LDS. Latency bounds it: 128 parts of 12 rows take 5.1 us by four waves a row and 16.8 by
// one, 16 parts 4.1 and 3.8; of the many rows that k_kv_wide splits, 6660 in 4 parts, 5.8 by one and 11.4 by a
// workgroup a row.
template <class T, int D, int W>
__global__ __launch_bounds__(256) void k_kv_join(KvAttnArgs a, bool vec) {
  constexpr int LP = D / 4, G = 64 / LP * W;
  __shared__ float o_lds[W == 4 ? 4 : 1][D];
  __shared__ float2 ml_lds[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int R = a.plan.rows, r = W == 4 ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave, h = blockIdx.y, s = blockIdx.z;
  const KvSeq sq = kv_seq(a.b, s);
  const int rows = sq.n * a.group;
  if (r >= rows) return;
  const int rt = r / R, r0 = rt * R;
  const int64_t step = (int64_t)a.part_rows * (D + 4);
  const float *p, *p0;  // parts 1 .. and part 0
  int nz;
  if (a.plan.shares) {
    const Tiles range = seq_tiles(a, sq);
    const int nt = range.t1 - range.t0;
    const int64_t n = share_size(a.first[a.b.seqs], a.plan.shares),
                  u = a.first[s] + (int64_t)(h * a.plan.row_tiles + rt) * (nt + kUnitCost) + kUnitCost, w0 = u / n;
    nz = (int)((u + nt - 1) / n - w0) + 1;
    if (nz == 1) return;  // (one share has all of it, and has written it)
    p = a.part + w0 * 2 * step + (int64_t)(r - r0) * (D + 4);
    p0 = p + step;
  } else {
    const Tiles range = row_tiles_of(a, sq, r0, R);
    nz = min((range.t1 - range.t0 + a.plan.chunk - 1) / a.plan.chunk, a.plan.splits);
    p0 = p = a.part + ((((int64_t)s * a.c.heads + h) * a.plan.row_tiles + rt) * a.plan.splits) * step + (int64_t)(r - r0) * (D + 4);
  }
  const int64_t stride = a.plan.shares ? 2 * step : step;
  auto at = [&](int z) { return z ? p + z * stride : p0; };
  const int e = lane % LP * 4, zg = lane / LP + (W == 4 ? wave * (64 / LP) : 0);
  constexpr int U = W == 4 ? 8 : 4;  // parts in flight
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -FLT_MAX, l = 0.f;
  for (int z0 = zg; z0 < nz; z0 += G * U) {
    f32x4 x[U];
    float2 ml[U];
    float most = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* c = at(min(z0 + u * G, nz - 1));
      x[u] = *(const f32x4*)(c + e);
      ml[u] = *(const float2*)(c + D);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) most = fmaxf(most, ml[u].x);
    const float down = exp2_fast(m - most);
    m = most;
    o *= down;
    l *= down;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (z0 + u * G >= nz) break;
      const float w = exp2_fast(ml[u].x - m);
      o += x[u] * w;
      l += w * ml[u].y;
    }
  }
#pragma unroll
  for (int d = LP; d < 64; d *= 2) {
    const float mo = __shfl_xor(m, d, 64), most = fmaxf(m, mo), w = exp2_fast(m - most), wo = exp2_fast(mo - most);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = o[i] * w + __shfl_xor(o[i], d, 64) * wo;
    l = l * w + __shfl_xor(l, d, 64) * wo;
    m = most;
  }
  if constexpr (W == 4) {
    if (lane < LP) *(f32x4*)&o_lds[wave][e] = o;
    if (lane == 0) ml_lds[wave] = make_float2(m, l);
    __syncthreads();
    if (tid >= LP) return;
    float most = ml_lds[0].x;
#pragma unroll
    for (int w = 1; w < 4; ++w) most = fmaxf(most, ml_lds[w].x);
    m = most;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
    l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = exp2_fast(ml_lds[w].x - most);
      o += *(const f32x4*)&o_lds[w][e] * f;
      l += ml_lds[w].y * f;
    }
  }
  if (lane >= LP) return;
  const int i = r / a.group, g = r - i * a.group;
  const bool beyond = sq.past + i >= a.b.max_len;
  const float inv = beyond ? NAN : l == 0.f ? 0.f : 1.f / l;
  const float x[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  T* to = (T*)a.out.p + (int64_t)(sq.row + i) * a.out.ld + (int64_t)(h * a.group + g) * a.out.hld + e;
  typedef T run __attribute__((ext_vector_type(4)));
  if (vec) {
    *(run*)to = run{(T)x[0], (T)x[1], (T)x[2], (T)x[3]};
  } else {
#pragma unroll
    for (int d = 0; d < 4; ++d) to[d] = (T)x[d];
  }
  if (lane == 0 && a.lse)
    a.lse[(int64_t)(sq.row + i) * a.q_heads + h * a.group + g] = beyond ? NAN : (m + log2f(l)) * 0.6931471805599453f;
}

template <class T, int D>
hipError_t kv_attention(const KvAttnArgs& a, hipStream_t st) {
  const bool vec = vectors(a.q, 2), vec_out = vectors(a.out, 2);
  // (what it reads depends on lengths that are on the device)
  const double most = (double)a.b.seqs * a.b.max_len * a.c.heads * 2 * D;
  if (a.plan.wide) {
    const dim3 grid((unsigned)a.plan.row_tiles * a.plan.splits * a.c.heads * a.b.seqs);
    MEBP_TIMED(st, "kv_wide", 0.0, most, hipLaunchKernelGGL((k_kv_wide<T, D>), grid, dim3(256), 0, st, a, vec, vec_out));
  } else {
    const dim3 grid(a.plan.shares ? (unsigned)a.plan.shares : (unsigned)(a.b.seqs * a.c.heads * a.plan.row_tiles * a.plan.splits));
    if (a.plan.rows == 16)
      MEBP_TIMED(st, "kv_rows", 0.0, most, hipLaunchKernelGGL((k_kv_rows<T, D, 1>), grid, dim3(256), 0, st, a, vec));
    else if constexpr (D == 64)
      MEBP_TIMED(st, "kv_rows", 0.0, most, hipLaunchKernelGGL((k_kv_rows<T, D, 2>), grid, dim3(256), 0, st, a, vec));
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || (a.plan.splits == 1 && !a.plan.shares)) return e;
  const unsigned rows = (unsigned)a.b.max_new * a.group, heads = (unsigned)a.c.heads, seqs = (unsigned)a.b.seqs;
  if (a.plan.shares || a.plan.splits > 8)
    MEBP_TIMED(st, "kv_join", 0.0, 0.0, hipLaunchKernelGGL((k_kv_join<T, D, 4>), dim3(rows, heads, seqs), dim3(256), 0, st, a, vec_out));
  else
    MEBP_TIMED(st, "kv_join", 0.0, 0.0, hipLaunchKernelGGL((k_kv_join<T, D, 1>), dim3((rows + 3) / 4, heads, seqs), dim3(256), 0, st, a, vec_out));
  return hipGetLastError();
}
}  // namespace

KvPlan kv_plan(int seqs, int max_new, int max_len, int q_heads, int heads, int dim, int window) {
  KvPlan p{};
  const int group = q_heads / heads;
  const int64_t rows = (int64_t)max_new * group, pairs = (int64_t)heads * std::max(seqs, 1);
  // tiles that a row tile's queries see at most
  auto tiles_seen = [&] {
    const int64_t tokens = std::min<int64_t>(max_new, p.rows / group + 2);
    return ((window ? std::min<int64_t>((int64_t)window + tokens + 126, max_len) : max_len) + 63) / 64;
  };
  auto shape = [&](int r) {
    p.rows = r;
    p.row_tiles = (int)((rows + r - 1) / r);
  };
  // Few rows by k_kv_rows, and as many as it has workgroups for in a round and a half of the chip, with up to 1536
  // times four tiles to do: it starts sooner than k_kv_wide, but each row tile reads the cache again. (Of heads of 128,
  // groups of 6, in us: one sequence of 1256 tokens, 256 of them new, 192 workgroups of 20 tiles, 18 and 30; of 8064,
  // 64 new, 1536 fours, 29 and 32; of 8128, 128 new, twice as many, 41 and 38; 4 sequences of 256 new tokens, 768
  // workgroups, 18 and 18; 40 of 68, 60 new, 1840 workgroups, 35 and 13.)
  // The longest sequences decide for all: a single token beside a prompt of 2048 walks all its keys in one workgroup (7
  // behind 8192, 12 heads of 128: 417 us, the prompt alone 66 and they 16; behind 65536, 8 of 256: 3580, 85 and 160).
  shape(rows <= 16 || dim > 64 ? 16 : 32);
  const int64_t groups = p.row_tiles * pairs, fours = groups * ((tiles_seen() + 3) / 4);
  p.wide = p.row_tiles > 2 && (groups > 768 || fours > 1536);
  if (p.wide) shape(128);
  p.splits = 1;
  // One or two row tiles of several long sequences that are more than two workgroups a compute unit: equal shares. (48
  // sequences of up to 8192 tokens, 4 heads of 256: 85 us, by chunks 137; 106 in a window of 1024, 2 heads of 128, 15
  // fours at most: 31 and 20.)
  if (!p.wide && p.row_tiles <= 2 && seqs > 1 && fours > 512 && fours > 16 * groups) {
    p.shares = 512;
    return p;
  }
  const int64_t tiles = tiles_seen(), units = p.row_tiles * pairs;
  // (large tiles go two to a compute unit at up to 128 dims, which pays for a join where the parts are long: 4 x 512
  // tokens behind 4000, 12 heads of 128, 158 us in one part, 133 in two)
  int64_t want = std::max<int64_t>(1, 256 / units);
  if (p.wide && dim < 256) want = std::max(want, std::min(384 / units, tiles / 16));
  // (a part of fewer tiles costs more to join than it saves: 3 x 344 tokens, 12 heads of 128, 30 us by 2, 21 by 6)
  int64_t chunk = std::max<int64_t>(p.wide ? 6 : 4, (tiles + want - 1) / want);
  if (!p.wide) chunk = (chunk + 3) / 4 * 4;
  p.chunk = (int)chunk;
  p.splits = (int)((tiles + chunk - 1) / chunk);
  return p;
}

// the parts, and behind them (shares) the places of the sequences' first tiles
size_t kv_part_floats(const KvPlan& p, int seqs, int max_new, int q_heads, int heads, int dim) {
  const size_t part_rows = std::min<int64_t>(p.rows, (int64_t)max_new * (q_heads / heads)), row = part_rows * (dim + 4);
  if (p.shares) return (size_t)p.shares * 2 * row + ((size_t)seqs + 1) * 2;
  return p.splits <= 1 ? 0 : (size_t)seqs * heads * p.row_tiles * p.splits * row;
}

hipError_t launch_kv_attention(KvAttnArgs a, int dtype, hipStream_t st) {
  a.part_rows = (int)std::min<int64_t>(a.plan.rows, (int64_t)a.b.max_new * a.group);
  a.first = (int64_t*)(a.part + (size_t)a.plan.shares * 2 * a.part_rows * (a.c.dim + 4));
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    return dtype == LOGIT_F16 ? kv_attention<f16, D>(a, st) : kv_attention<bf16, D>(a, st);
  };
  return a.c.dim == 64 ? go(IC<64>{}) : a.c.dim == 128 ? go(IC<128>{}) : go(IC<256>{});
}

}  // namespace mebp
