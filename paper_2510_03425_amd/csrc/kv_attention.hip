// Attention of new tokens over the paged 8-bit cache on gfx950: causal, grouped heads, optional window.
//
// With the codes k, v of a block and its scales sk, sv:  s = scale sk (q . k),  p = exp(s - m),
// out = (sum p sv v) / (sum p): codes go into the matrix instructions as they are, exact in fp16, and the
// scales into the scores and the weights. One pass over the cache with the running maximum and sum of a
// softmax; statistics and sums in fp32.
//
// k_kv_rows keeps a whole 64-key tile in one wave's registers, without LDS: with S^T = K Q^T and
// O^T = V^T P^T, tile t = 0..3 of 16 keys takes the keys 16 (r / 4) + 4 t + r % 4 as its rows r, so that
// the lanes l / 16 = g end up with the weights of keys 16 g .. 16 g + 15 of their query l % 16: one block
// of the cache, in the order of V's [dim][16] codes, which are the other operand as they lie in memory.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "device_common.h"
#include "heads.h"
#include "kv_device.h"

namespace mebp {
namespace {

// Weights are 2^(s - m + kBias), m following a row's largest score in steps of more than kLift: at most
// 2^11, and 2^15 with the scale of the values, relative to a reference within 2^4 above: in fp16's range,
// 2^-14 below which it loses bits being 2^-19 of the row's largest weight or less.
constexpr float kBias = 5.f, kLift = 6.f, kRefUp = 16.f, kRefDown = 1.f / 256.f;

// 8 codes in 2 dwords -> 8 fp16: code + 128 below the bits of 1024, less 1152; exact.
DEV f16x8 codes_f16(uint32_t lo, uint32_t hi) {
  const uint32_t a = lo ^ 0x80808080u, b = hi ^ 0x80808080u;
  const f16x2 off = {(f16)1152.0f, (f16)1152.0f};
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u)) - off);
  r.y = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u)) - off);
  r.z = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u)) - off);
  r.w = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)) - off);
  return __builtin_bit_cast(f16x8, r);
}

// 64-key tiles [t0, t1) that queries at positions [lo, hi] of a sequence of `len` tokens see
struct Tiles {
  int t0, t1;
};
DEV Tiles tiles_of(int lo, int hi, int window) {
  return Tiles{window ? max(lo - window + 1, 0) >> 6 : 0, (hi >> 6) + 1};
}

// A row's queries as fp16 operands, scaled by a power of two to just below fp16's end (exact but for
// elements 2^-28 of the largest), and what a score is to be multiplied by for it: NaN where the row has
// a NaN or an infinity.
template <class T, int NF>
DEV float row_queries(const T* p, bool vec, float scale, f16x8 (&f)[NF], int g4) {
  float x[NF][8], most = 0.f;
  int bad = 0;
#pragma unroll
  for (int m = 0; m < NF; ++m) {
    const T* e = p + 64 * (m / 2) + 16 * g4 + 8 * (m & 1);
    if (vec) {
      load8(e, x[m]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[m][i] = (float)e[i];
    }
  }
#pragma unroll
  for (int m = 0; m < NF; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      most = fmaxf(most, fabsf(x[m][i]));
      bad |= !(fabsf(x[m][i]) < INFINITY);
    }
#pragma unroll
  for (int o = 16; o < 64; o *= 2) {
    most = fmaxf(most, __shfl_xor(most, o, 64));
    bad |= __shfl_xor(bad, o, 64);
  }
  const int up = most > 0.f && !bad ? 14 - ilogbf(most) : 0;
#pragma unroll
  for (int m = 0; m < NF; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i) f[m][i] = (f16)ldexpf(x[m][i], up);
  return bad ? NAN : ldexpf(scale, -up);
}

// Few rows: one workgroup of 4 waves takes NR * 16 rows (token, head of the group) of one sequence and kv
// head over a chunk of its tiles, the waves one tile in four each; their sums meet in LDS.
template <class T, int D, int NR>
__global__ __launch_bounds__(256, D * NR > 256 ? 1 : 2) void k_kv_rows(KvAttnArgs a, bool vec) {
  constexpr int NF = D / 32, NK = D / 16, R = 16 * NR;
  __shared__ float o_lds[4][R][D + 4];
  __shared__ float m_lds[4][R], l_lds[4][R], w_lds[4][R], ref_lds[4];
  const int z = blockIdx.x % a.plan.splits, rt = blockIdx.x / a.plan.splits, h = blockIdx.y, s = blockIdx.z;
  const KvSeq sq = kv_seq(a.b, s);
  const int rows = sq.n * a.group, r0 = rt * R;
  if (r0 >= rows) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r16 = lane & 15, g4 = lane >> 4;
  // rows behind the last one repeat it
  const int last = min(r0 + R, rows) - 1;
  const int pos_lo = sq.past + r0 / a.group, pos_hi = sq.past + last / a.group;
  const Tiles range = tiles_of(pos_lo, pos_hi, a.window);
  const int tb = range.t0 + z * a.plan.chunk, te = min(tb + a.plan.chunk, range.t1);
  if (tb >= te) return;
  const int nblk = (sq.past + sq.n + 15) >> 4;

  f16x8 qf[NR][NF];
  float qs[NR];
  int pos[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int r = min(r0 + n * 16 + r16, last), i = r / a.group, g = r - i * a.group;
    pos[n] = sq.past + i;
    const T* p = (const T*)a.q.p + (int64_t)(sq.row + i) * a.q.ld + (int64_t)(h * a.group + g) * a.q.hld;
    qs[n] = row_queries(p, vec, a.scale, qf[n], g4);
  }
  f32x4 acc[NR][NK];
  float m[NR], l[NR], ref = 1.f;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    m[n] = -FLT_MAX;
    l[n] = 0.f;
#pragma unroll
    for (int d = 0; d < NK; ++d) acc[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  for (int tile = tb + wave; tile < te; tile += 4) {
    // the lane's block as a row of the keys' operand, and as a lane of the scores and the values
    const int bk = min(tile * 4 + (r16 >> 2), nblk - 1), bv = min(tile * 4 + g4, nblk - 1);
    const int pk = kv_page(a.c, a.b, s, bk), pv = kv_page(a.c, a.b, s, bv);
    const int64_t ik = kv_block(a.c, max(pk, 0), h, bk), iv = kv_block(a.c, max(pv, 0), h, bv);
    const int8_t* kp = a.c.codes + ik * (32 * D) + (r16 & 3) * D + g4 * 16;
    const int8_t* vp = a.c.codes + iv * (32 * D) + 16 * D + r16 * 16;
    float2 sc = ((const float2*)a.c.scales)[iv];
    uint4 kr[NK], vr[NK];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < D / 64; ++j) kr[t * (D / 64) + j] = *(const uint4*)(kp + t * 4 * D + j * 64);
#pragma unroll
    for (int d = 0; d < NK; ++d) vr[d] = *(const uint4*)(vp + d * 256);
    if (pv < 0) sc.x = sc.y = NAN;
    f32x4 sa[NR][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int n = 0; n < NR; ++n) sa[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        const uint4 c = kr[t * (D / 64) + j];
        const f16x8 c0 = codes_f16(c.x, c.y), c1 = codes_f16(c.z, c.w);
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          sa[n][t] = mfma16(c0, qf[n][2 * j], sa[n][t]);
          sa[n][t] = mfma16(c1, qf[n][2 * j + 1], sa[n][t]);
        }
      }
    }
    // the values' reference follows their scales
    const bool masked = tile * 64 + 63 > pos_lo || (a.window && tile * 64 <= pos_hi - a.window);
    const float sv = masked && !(tile * 64 + 16 * g4 <= pos_hi) ? 0.f : sc.y;
    if (__ballot(sv > ref * kRefUp) || (!__ballot(sv > ref * kRefDown) && __ballot(sv > 0.f))) {
      float mv = sv < INFINITY ? sv : 0.f;  // (NaN: no reference)
      mv = fmaxf(mv, __shfl_xor(mv, 16, 64));
      mv = fmaxf(mv, __shfl_xor(mv, 32, 64));
      const float next = mv > 0.f ? ldexpf(1.f, ilogbf(mv)) : ref, by = ref / next;
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int d = 0; d < NK; ++d) acc[n][d] *= by;
      ref = next;
    }
    const float svr = sv / ref;
    uint32_t pw[NR][8];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      float x[16];
      const float f = sc.x * qs[n];
      float mx = -INFINITY;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        x[k] = sa[n][k >> 2][k & 3] * f;
        if (masked) {
          const int key = tile * 64 + 16 * g4 + k;
          if (key > pos[n] || (a.window && key <= pos[n] - a.window)) x[k] = -INFINITY;
        }
        mx = fmaxf(mx, x[k]);
      }
      if (__ballot(mx > m[n] + kLift)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float next = fmaxf(m[n], mx), by = exp2_fast(m[n] - next);
        m[n] = next;
        l[n] *= by;
#pragma unroll
        for (int d = 0; d < NK; ++d) acc[n][d] *= by;
      }
      const float lift = kBias - m[n];
#pragma unroll
      for (int k = 0; k < 16; k += 2) {
        const float p0 = exp2_fast(x[k] + lift), p1 = exp2_fast(x[k + 1] + lift);
        l[n] += p0 + p1;
        float w0 = p0 * svr, w1 = p1 * svr;
        if (masked) {
          // (the scale of a block that the row does not see may be NaN)
          if (x[k] == -INFINITY) w0 = 0.f;
          if (x[k + 1] == -INFINITY) w1 = 0.f;
        }
        pw[n][k / 2] = pack_f16x2(w0, w1);
      }
    }
#pragma unroll
    for (int d = 0; d < NK; ++d) {
      const f16x8 v0 = codes_f16(vr[d].x, vr[d].y), v1 = codes_f16(vr[d].z, vr[d].w);
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        acc[n][d] = mfma16(v0, __builtin_bit_cast(f16x8, make_uint4(pw[n][0], pw[n][1], pw[n][2], pw[n][3])), acc[n][d]);
        acc[n][d] = mfma16(v1, __builtin_bit_cast(f16x8, make_uint4(pw[n][4], pw[n][5], pw[n][6], pw[n][7])), acc[n][d]);
      }
    }
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
    }
  }
  if (lane == 0) ref_lds[wave] = ref;
  __syncthreads();
  if (tid < R) {
    float mm = m_lds[0][tid];
    for (int w = 1; w < 4; ++w) mm = fmaxf(mm, m_lds[w][tid]);
    float ll = 0.f;
    for (int w = 0; w < 4; ++w) {
      const float e = exp2_fast(m_lds[w][tid] - mm);
      ll += e * l_lds[w][tid];
      w_lds[w][tid] = e * ref_lds[w];
    }
    m_lds[0][tid] = mm;
    l_lds[0][tid] = ll;
  }
  __syncthreads();
  const int64_t part = ((((int64_t)s * a.c.heads + h) * a.plan.row_tiles + rt) * a.plan.splits + z) * a.part_rows;
  for (int i = tid; i < R * (D / 4); i += 256) {
    const int r = i / (D / 4), e = (i % (D / 4)) * 4;
    if (r0 + r > last) continue;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) o += *(const f32x4*)&o_lds[w][r][e] * w_lds[w][r];
    if (a.plan.splits > 1) {
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
          sq.past + i_tok >= a.b.max_len ? NAN : (m_lds[0][r] - kBias + log2f(ll)) * 0.6931471805599453f;
  }
}

// Joins the chunks of each row: one workgroup a row.
template <class T, int D, int R>
__global__ __launch_bounds__(256) void k_kv_join(KvAttnArgs a) {
  __shared__ float o_lds[256 / (D / 4)][D];
  const int r = blockIdx.x, h = blockIdx.y, s = blockIdx.z;
  const KvSeq sq = kv_seq(a.b, s);
  const int rows = sq.n * a.group;
  if (r >= rows) return;
  const int rt = r / R, r0 = rt * R, last = min(r0 + R, rows) - 1;
  const Tiles range = tiles_of(sq.past + r0 / a.group, sq.past + last / a.group, a.window);
  const int nz = min((range.t1 - range.t0 + a.plan.chunk - 1) / a.plan.chunk, a.plan.splits);
  const float* p = a.part + (((((int64_t)s * a.c.heads + h) * a.plan.row_tiles + rt) * a.plan.splits) * a.part_rows + r - r0) * (D + 4);
  const int64_t step = (int64_t)a.part_rows * (D + 4);
  constexpr int G = 256 / (D / 4);
  const int e = (threadIdx.x % (D / 4)) * 4, zg = threadIdx.x / (D / 4);
  float mm = -FLT_MAX;
  for (int z = threadIdx.x & 63; z < nz; z += 64) mm = fmaxf(mm, p[z * step + D]);
  mm = wave_max(mm);
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  float ll = 0.f;
  for (int z = zg; z < nz; z += G) {
    const float w = exp2_fast(p[z * step + D] - mm);
    o += *(const f32x4*)(p + z * step + e) * w;
    ll += w * p[z * step + D + 1];
  }
  *(f32x4*)&o_lds[zg][e] = o;
  __shared__ float lz[G];
  if (e == 0) lz[zg] = ll;
  __syncthreads();
  if (threadIdx.x >= D) return;
  float sum = 0.f, tot = 0.f;
  for (int g = 0; g < G; ++g) {
    sum += o_lds[g][threadIdx.x];
    tot += lz[g];
  }
  const int i = r / a.group, g = r - i * a.group;
  const bool beyond = sq.past + i >= a.b.max_len;
  const float inv = beyond ? NAN : tot == 0.f ? 0.f : 1.f / tot;
  ((T*)a.out.p)[(int64_t)(sq.row + i) * a.out.ld + (int64_t)(h * a.group + g) * a.out.hld + threadIdx.x] = (T)(sum * inv);
  if (threadIdx.x == 0 && a.lse)
    a.lse[(int64_t)(sq.row + i) * a.q_heads + h * a.group + g] = beyond ? NAN : (mm - kBias + log2f(tot)) * 0.6931471805599453f;
}

template <class T, int D>
hipError_t kv_attention(const KvAttnArgs& a, hipStream_t st) {
  const bool vec = vectors(a.q, 2);
  const dim3 grid((unsigned)a.plan.row_tiles * a.plan.splits, (unsigned)a.c.heads, (unsigned)a.b.seqs);
  // (what it reads depends on lengths that are on the device)
  const double most = (double)a.b.seqs * a.b.max_len * a.c.heads * 2 * D;
  if (a.plan.rows == 16)
    MEBP_TIMED(st, "kv_rows", 0.0, most, hipLaunchKernelGGL((k_kv_rows<T, D, 1>), grid, dim3(256), 0, st, a, vec));
  else
    MEBP_TIMED(st, "kv_rows", 0.0, most, hipLaunchKernelGGL((k_kv_rows<T, D, 2>), grid, dim3(256), 0, st, a, vec));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.plan.splits == 1) return e;
  const dim3 rows((unsigned)a.b.max_new * a.group, (unsigned)a.c.heads, (unsigned)a.b.seqs);
  if (a.plan.rows == 16)
    MEBP_TIMED(st, "kv_join", 0.0, 0.0, hipLaunchKernelGGL((k_kv_join<T, D, 16>), rows, dim3(256), 0, st, a));
  else
    MEBP_TIMED(st, "kv_join", 0.0, 0.0, hipLaunchKernelGGL((k_kv_join<T, D, 32>), rows, dim3(256), 0, st, a));
  return hipGetLastError();
}
}  // namespace

KvPlan kv_plan(int seqs, int max_new, int max_len, int q_heads, int heads, int dim, int window) {
  KvPlan p{};
  const int64_t rows = (int64_t)max_new * (q_heads / heads);
  p.rows = rows <= 16 ? 16 : 32;
  p.row_tiles = (int)((rows + p.rows - 1) / p.rows);
  // tiles that a row tile's queries see at most
  const int64_t span = window ? std::min<int64_t>((int64_t)window + p.rows + 126, max_len) : max_len;
  const int64_t tiles = (span + 63) / 64;
  const int64_t groups = (int64_t)p.row_tiles * heads * std::max(seqs, 1);
  // about 1024 workgroups, a tile to each wave at least
  const int64_t want = std::max<int64_t>(1, 1024 / groups);
  int64_t chunk = (tiles + want - 1) / want;
  chunk = std::max<int64_t>(4, (chunk + 3) / 4 * 4);
  p.chunk = (int)chunk;
  p.splits = (int)((tiles + chunk - 1) / chunk);
  return p;
}

size_t kv_part_floats(const KvPlan& p, int seqs, int max_new, int q_heads, int heads, int dim) {
  if (p.splits <= 1) return 0;
  const size_t part_rows = std::min<int64_t>(p.rows, (int64_t)max_new * (q_heads / heads));
  return (size_t)seqs * heads * p.row_tiles * p.splits * part_rows * (dim + 4);
}

hipError_t launch_kv_attention(KvAttnArgs a, int dtype, hipStream_t st) {
  a.part_rows = (int)std::min<int64_t>(a.plan.rows, (int64_t)a.b.max_new * a.group);
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    return dtype == LOGIT_F16 ? kv_attention<f16, D>(a, st) : kv_attention<bf16, D>(a, st);
  };
  return a.c.dim == 64 ? go(IC<64>{}) : a.c.dim == 128 ? go(IC<128>{}) : go(IC<256>{});
}

}  // namespace mebp
