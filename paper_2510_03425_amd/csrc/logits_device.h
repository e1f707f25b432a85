// Device code shared by the operators on logits (logits.hip, distill.hip): loads of rows at any
// alignment, softmax statistics in one pass, and their join over lanes, waves and parts of a row.
//
// Every row is a softmax over tens of thousands of logits, and all that a row gives besides its
// gradient is a few numbers: the floor is the logits read once and the gradient written once.
// One pass keeps, per lane, a reference m, s = sum exp((z - m) / tau) and w = sum exp(..) (z - m);
// lanes, waves and parts of a row are joined by rescaling to the largest reference. The order of
// all sums is fixed by the shape alone.
#pragma once
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "mebp_internal.h"

namespace mebp {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNone = -FLT_MAX;  // reference of a lane that has seen no logit above -inf

typedef unsigned long long u64;

template <class T>
constexpr int kVec = 16 / (int)sizeof(T);

DEV float cvt(float x) { return x; }
DEV float cvt(f16 x) { return (float)x; }
DEV float cvt(bf16 x) { return (float)x; }

template <class T>
DEV void unpack(uint4 v, float (&x)[kVec<T>]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      x[i] = __builtin_bit_cast(float, w[i]);
    } else if constexpr (__is_same(T, f16)) {
      x[2 * i] = f16_lo(w[i]);
      x[2 * i + 1] = f16_hi(w[i]);
    } else {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    }
  }
}

// 16 bytes at an address that is a multiple of the element size alone: rows of an odd pitch start
// anywhere, and the memory pipeline takes such accesses as they are.
typedef uint32_t u32x4_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_2 __attribute__((ext_vector_type(2), aligned(2)));

// ONCE: the logits are read by this pass alone. Non-temporal loads read 7.0 .. 7.2 TB/s where
// ordinary ones read 6.2 (2 GiB, 4 loads of each lane in flight).
template <bool ONCE, class T>
DEV uint4 load16(const T* p) {
  const u32x4_2* q = (const u32x4_2*)p;
  const u32x4_2 v = ONCE ? __builtin_nontemporal_load(q) : *q;
  return make_uint4(v.x, v.y, v.z, v.w);
}

// Logits i .. i + kVec of a row, -inf at and behind `end`.
template <class T>
DEV void load_tail(const T* row, int i, int end, float (&x)[kVec<T>]) {
#pragma unroll
  for (int j = 0; j < kVec<T>; ++j) x[j] = i + j < end ? cvt(row[i + j]) : -INFINITY;
}

template <class G, int N>
DEV void store_vec(G* p, const float (&g)[N]) {
  constexpr int W = N * (int)sizeof(G) / 4;
  uint32_t w[W];
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if constexpr (sizeof(G) == 4)
      w[i] = __builtin_bit_cast(uint32_t, g[i]);
    else if constexpr (__is_same(G, f16))
      w[i] = pack_f16x2(g[2 * i], g[2 * i + 1]);
    else
      w[i] = pack_bf16x2(g[2 * i], g[2 * i + 1]);
  }
  if constexpr (W == 2) {
    __builtin_nontemporal_store(u32x2_2{w[0], w[1]}, (u32x2_2*)p);
  } else {
#pragma unroll
    for (int i = 0; i < W; i += 4)
      __builtin_nontemporal_store(u32x4_2{w[i], w[i + 1], w[i + 2], w[i + 3]}, (u32x4_2*)p + i / 4);
  }
}

template <class G>
DEV G to_out(float g) {
  return (G)g;
}

// what a workgroup wrote is in order before what follows the barrier writes to the same places
DEV void stores_done() {
  wait_vmcnt<0>();
  __syncthreads();
}

// ------------------------------------------------------------------ softmax statistics
struct Acc {
  float m, s, w, s1;  // reference, sum at c, sum weighted by z - m, sum at c1
};

DEV Acc acc_empty() { return Acc{kNone, 0.f, 0.f, 0.f}; }

// moves an accumulator to the reference M >= m
template <bool ENT, bool TWO>
DEV void acc_move(Acc& a, float M, float c, float c1) {
  const float f = exp2_fast((a.m - M) * c);
  // (from no reference at all f is 0, and m - M times s may overflow)
  if (ENT) a.w = f > 0.f ? f * (a.w + (a.m - M) * a.s) : 0.f;
  a.s *= f;
  if (TWO) a.s1 *= exp2_fast((a.m - M) * c1);
  a.m = M;
}

// The logits that scan() hands over at a time: `n` (all lanes alike) of U vectors, vector u of this
// lane at columns col + u * step ..
template <int U, int N>
struct Group {
  float x[U][N], top;  // top: the largest of them (NaN left out)
  int n, col, step;
};

// Adds a group. The reference only follows where a logit lies more than `lift` above it, 2^6 times
// its weight: fp32 holds the sums nearly as well with a stale one (the entropy's error grows with
// the distance to the largest logit), and few groups move it. A vector is summed by itself first,
// which leaves a lane an 8th (4th) of the additions in a row. NaN and +inf logits make s NaN:
// exp(NaN), and exp(inf - inf).
template <bool ENT, bool TWO, int U, int N>
DEV void acc_add(Acc& a, const Group<U, N>& g, float c, float c1, float lift) {
  if (g.top > a.m + lift) acc_move<ENT, TWO>(a, g.top, c, c1);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u >= g.n) break;
    float s = 0.f, w = 0.f, s1 = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float d = g.x[u][j] - a.m;
      const float e = exp2_fast(d * c);
      s = j ? s + e : e;
      // (a logit of -inf has weight 0, and 0 times -inf is not)
      const float dw = fmaxf(d, -1e30f);
      if (ENT) w = j ? fmaf(e, dw, w) : e * dw;
      const float e1 = TWO ? exp2_fast(d * c1) : 0.f;
      s1 = j ? s1 + e1 : e1;
    }
    a.s += s;
    if (ENT) a.w += w;
    if (TWO) a.s1 += s1;
  }
}

template <bool ENT, bool TWO>
DEV void acc_wave(Acc& a, float c, float c1) {
  acc_move<ENT, TWO>(a, wave_max(a.m), c, c1);
  a.s = wave_sum(a.s);
  if (ENT) a.w = wave_sum(a.w);
  if (TWO) a.s1 = wave_sum(a.s1);
}

// joined over the workgroup, for every thread
template <int NT, bool ENT, bool TWO>
DEV void acc_block(Acc& a, float c, float c1, Acc* lds) {
  constexpr int NW = NT / 64;
  acc_wave<ENT, TWO>(a, c, c1);
  if (lane_id() == 0) lds[threadIdx.x >> 6] = a;
  __syncthreads();
  float M = kNone;
#pragma unroll
  for (int i = 0; i < NW; ++i) M = fmaxf(M, lds[i].m);
  Acc t{M, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    Acc b = lds[i];
    acc_move<ENT, TWO>(b, M, c, c1);
    t.s += b.s;
    t.w += b.w;
    t.s1 += b.s1;
  }
  a = t;
}

// the statistics of a row's parts, for every lane of the wave
template <bool ENT, bool TWO>
DEV Acc join_parts(const LogitSplit& sp, size_t row, float c, float c1) {
  const int l = lane_id();
  Acc a = acc_empty();
  if (l < sp.n) {
    const float4 v = sp.stats[row * sp.n + l];
    a = Acc{v.x, v.y, v.z, v.w};
  }
  acc_wave<ENT, TWO>(a, c, c1);
  return a;
}

// Hands columns v0 .. v1 of a row to add(group), -inf in the place of columns behind the end; columns
// rise from vector to vector and from group to group. The loads of one group are in flight while
// the one before it is worked on.
template <class T, int NT, int U, bool ONCE, class F>
DEV void scan(const T* row, int v0, int v1, F&& add) {
  constexpr int N = kVec<T>, step = NT * N;
  int i = v0 + (int)threadIdx.x * N, b = v0;
  uint4 next[U];
  Group<U, N> g;
  g.n = U;
  g.step = step;
  auto top = [&](int n) {
    g.top = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u >= n) break;
#pragma unroll
      for (int j = 0; j < N; ++j) g.top = fmaxf(g.top, g.x[u][j]);
    }
  };
  if (b + U * step <= v1) {
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = load16<ONCE>(row + i + u * step);
    for (; b + U * step <= v1; b += U * step, i += U * step) {
#pragma unroll
      for (int u = 0; u < U; ++u) unpack<T>(next[u], g.x[u]);
      if (b + 2 * U * step <= v1) {
#pragma unroll
        for (int u = 0; u < U; ++u) next[u] = load16<ONCE>(row + i + (U + u) * step);
      }
      g.col = i;
      top(U);
      add(g);
    }
  }
  if (b >= v1) return;
  // fewer than U vectors of each lane are left
  g.n = (v1 - b + step - 1) / step;
  g.col = i;
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (i + u * step + N <= v1) next[u] = load16<ONCE>(row + i + u * step);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u >= g.n) break;
    if (i + u * step + N <= v1)
      unpack<T>(next[u], g.x[u]);
    else
      load_tail<T>(row, i + u * step, v1, g.x[u]);
  }
  top(g.n);
  add(g);
}

// Writes f(z) over columns v0 .. v1 of a row. Every element is read before it is written, by the
// thread that writes it: the output may be the input.
template <class T, class G, int NT, int U, bool ONCE, class F>
DEV void map_row(const T* z, G* dz, int v0, int v1, F&& f) {
  constexpr int N = kVec<T>, step = NT * N;
  int i = v0 + (int)threadIdx.x * N;
  for (; i + (U - 1) * step + N <= v1; i += U * step) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load16<ONCE>(z + i + u * step);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[N];
      unpack<T>(v[u], x);
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = f(x[j]);
      store_vec<G, N>(dz + i + u * step, x);
    }
  }
  for (; i + N <= v1; i += step) {
    float x[N];
    unpack<T>(load16<ONCE>(z + i), x);
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = f(x[j]);
    store_vec<G, N>(dz + i, x);
  }
  for (int j = 0; j < N; ++j)
    if (i + j < v1) dz[i + j] = to_out<G>(f(cvt(z[i + j])));
}

// zeros over columns v0 .. v1 of a row
template <class G, int NT>
DEV void zero_row(G* dz, int v0, int v1) {
  constexpr int N = kVec<G>;
  int i = v0 + (int)threadIdx.x * N;
  const float none[N] = {};
  for (; i + N <= v1; i += NT * N) store_vec<G, N>(dz + i, none);
  for (int j = 0; j < N; ++j)
    if (i + j < v1) dz[i + j] = to_out<G>(0.f);
}

template <class F>
hipError_t by_type(int dtype, F&& f) {
  switch (dtype) {
    case LOGIT_F32: return f((float*)nullptr);
    case LOGIT_F16: return f((f16*)nullptr);
    default: return f((bf16*)nullptr);
  }
}
inline double type_bytes(int dtype) { return dtype == LOGIT_F32 ? 4.0 : 2.0; }

}  // namespace
}  // namespace mebp
