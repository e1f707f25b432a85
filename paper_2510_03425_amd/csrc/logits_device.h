// Device code shared by the operators on logits (logits.hip, distill.hip): loads of rows at any
// alignment, softmax statistics in one pass, and their join over lanes, waves and parts of a row.
//
// Every row is a softmax over tens of thousands of logits, and all that a row gives besides its
// gradient is a few numbers: the floor is the logits read once and the gradient written once.
// One pass keeps a reference m, s = sum exp((z - m) / tau) and w = sum exp(..) (z - m); sums at several
// references are joined by rescaling to the largest. The order of all sums is fixed by the shape
// alone.
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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <class T>
DEV void unpack(u32x4 w, float (&x)[kVec<T>]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      x[i] = __builtin_bit_cast(float, (uint32_t)w[i]);
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
DEV u32x4 load16(const T* p) {
  const u32x4_2* q = (const u32x4_2*)p;
  return ONCE ? __builtin_nontemporal_load(q) : *q;
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

// ------------------------------------------------------------------ exchange between lanes
// the value of lane l ^ J: moves inside rows of 16 lanes, swaps of rows and of halves
template <int CTRL>
DEV uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
template <int J>
DEV uint32_t lane_xor(uint32_t x) {
  if constexpr (J == 1) return dpp<0xB1>(x);                 // quad [1,0,3,2]
  else if constexpr (J == 2) return dpp<0x4E>(x);            // quad [2,3,0,1]
  else if constexpr (J == 3) return dpp<0x1B>(x);            // quad [3,2,1,0]
  else if constexpr (J == 4) return dpp<0x1B>(dpp<0x141>(x));  // 7 ^ 3
  else if constexpr (J == 7) return dpp<0x141>(x);           // mirror of 8
  else if constexpr (J == 8) return dpp<0x128>(x);           // rotation by 8 of 16
  else if constexpr (J == 15) return dpp<0x140>(x);          // mirror of 16
  else if constexpr (J == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  } else if constexpr (J == 31) return lane_xor<16>(lane_xor<15>(x));
  else if constexpr (J == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  } else {
    static_assert(J == 63, "lane_xor");
    return lane_xor<32>(lane_xor<31>(x));
  }
}
// sums and maxima over a wave, in every lane
template <int J>
DEV float lane_xor_f(float x) {
  return __builtin_bit_cast(float, lane_xor<J>(__builtin_bit_cast(uint32_t, x)));
}
DEV float sum64(float v) {
  v += lane_xor_f<1>(v);
  v += lane_xor_f<2>(v);
  v += lane_xor_f<7>(v);  // (quads are alike by now, and so on)
  v += lane_xor_f<15>(v);
  v += lane_xor_f<16>(v);
  return v + lane_xor_f<32>(v);
}
DEV float max64(float v) {
  v = fmaxf(v, lane_xor_f<1>(v));
  v = fmaxf(v, lane_xor_f<2>(v));
  v = fmaxf(v, lane_xor_f<7>(v));
  v = fmaxf(v, lane_xor_f<15>(v));
  v = fmaxf(v, lane_xor_f<16>(v));
  return fmaxf(v, lane_xor_f<32>(v));
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
  float x[U][N];
  int n, col, step;

  __device__ __forceinline__ float top() const {  // the largest of them (NaN left out)
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u >= n) break;
#pragma unroll
      for (int j = 0; j < N; ++j) m = fmaxf(m, x[u][j]);
    }
    return m;
  }
};

// Adds a group, one lane's reference following its own largest logit. NaN and +inf logits make s NaN:
// exp(NaN), and exp(inf - inf).
template <bool ENT, bool TWO, int U, int N>
DEV void acc_add(Acc& a, const Group<U, N>& g, float c, float c1) {
  const float top = g.top();
  if (top > a.m) acc_move<ENT, TWO>(a, top, c, c1);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u >= g.n) break;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float d = g.x[u][j] - a.m;
      const float e = exp2_fast(d * c);
      a.s += e;
      // (a logit of -inf has weight 0, and 0 times -inf is not)
      if (ENT) a.w = fmaf(e, fmaxf(d, -1e30f), a.w);
      if (TWO) a.s1 += exp2_fast(d * c1);
    }
  }
}

template <int N>
DEV float max_of(const float (&x)[N]) {
  float m = x[0];
#pragma unroll
  for (int j = 1; j < N; ++j) m = fmaxf(m, x[j]);
  return m;
}

template <bool ENT, bool TWO>
DEV void acc_wave(Acc& a, float c, float c1) {
  acc_move<ENT, TWO>(a, max64(a.m), c, c1);
  a.s = sum64(a.s);
  if (ENT) a.w = sum64(a.w);
  if (TWO) a.s1 = sum64(a.s1);
}

// joined over the workgroup, for every thread
template <int NT, bool ENT, bool TWO>
DEV void acc_block(Acc& a, float c, float c1, Acc* lds) {
  constexpr int NW = NT / 64;
  acc_wave<ENT, TWO>(a, c, c1);
  if (lane_id() == 0) lds[threadIdx.x >> 6] = a;
  __syncthreads();
  a = lane_id() < NW ? lds[lane_id()] : acc_empty();
  acc_wave<ENT, TWO>(a, c, c1);
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

// ------------------------------------------------------------------ sums at a wave's reference
// The sums of a wave at one reference, 2^k: a weight is then exp2(z c - k), two instructions, and k, a
// whole number, costs no bits, as the difference is rounded once and a move to another k is a scaling by a
// power of two. k follows the wave's largest logit: it moves where one lies above the last by `lift`, twice
// its weight, so that no weight is above 2^1.5 and the largest are the most precise. That happens a few times
// in a row (for logits in no order, as often as the logarithm of the number of steps).
//
// What leaves the wave is relative to its largest logit itself, whose weight is divided out as it was added:
// s >= 1, w <= 0, so that no log probability is above 0 and no entropy below. k = inf, which makes all
// weights 0, where no logit was above -inf yet and where k would have no whole numbers left (logits of 2^23
// temperatures and more, of the size of the type's lowest value among them, and +inf). A wave that ends there
// has s NaN, as one with a NaN logit, and the caller sums again with acc_add: served().
enum Softmaxes { ONE, TWO_EXP, TWO_SQUARE };  // at tau alone; also at 1; the same where tau is 2:
                                              // exp(z) is then exp(z / 2)^2
// the reference of a largest logit m
DEV float whole_exponent(float m, float c) {
  const float k = rintf(m * c);
  return fabsf(k) < 0x1p23f ? k : INFINITY;
}
// what the weights at one reference are at another
DEV float rescaling(float from, float to) { return from == INFINITY ? 0.f : exp2_fast(from - to); }

template <bool ENT, Softmaxes SM>
struct Sums {
  float c, lift;
  float k, k1;      // the references at tau and at 1 (TWO_EXP)
  float over;       // a logit above it moves them
  float most;       // this lane's largest logit
  float s, w, s1;   // w: weighted by z c - k

  __device__ __forceinline__ void start(float scale, float rise) {
    c = scale;
    lift = rise;
    s = w = s1 = 0.f;
    k = k1 = INFINITY;
    over = most = -INFINITY;
  }
  // top: this lane's largest logit among those that are added next
  __device__ __forceinline__ void meet(float top) {
    most = fmaxf(most, top);
    if (!__any(top > over)) return;
    const float m = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, max64(most))));
    const float to = whole_exponent(m, c), f = rescaling(k, to);
    // (f = 0 leaves nothing, and k - to times s may be far beyond)
    if (ENT) w = f > 0.f ? f * fmaf(k - to, s, w) : 0.f;
    s *= f;
    if (SM == TWO_SQUARE) s1 *= f * f;
    if (SM == TWO_EXP) {
      const float to1 = whole_exponent(m, kLog2e);
      s1 *= rescaling(k1, to1);
      k1 = to1;
    }
    k = to;
    over = m + lift;
  }
  template <int N>
  __device__ __forceinline__ void add_met(const float (&x)[N]) {
    // a vector by itself first, which leaves a lane an 8th (4th) of the additions in a row
    float vs = 0.f, vw = 0.f, v1 = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float a = fmaf(x[j], c, -k), e = exp2_fast(a);
      vs = j ? vs + e : e;
      // (a logit of -inf has weight 0, and 0 times -inf is not)
      if (ENT) vw = j ? fmaf(e, fmaxf(a, -1e30f), vw) : e * fmaxf(a, -1e30f);
      if (SM == TWO_SQUARE) v1 = j ? fmaf(e, e, v1) : e * e;
      if (SM == TWO_EXP) {
        const float e1 = exp2_fast(fmaf(x[j], kLog2e, -k1));
        v1 = j ? v1 + e1 : e1;
      }
    }
    s += vs;
    if (ENT) w += vw;
    if (SM != ONE) s1 += v1;
  }
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N]) {
    meet(max_of(x));
    add_met(x);
  }
  // STEP vectors at a time, which groups of other sizes then give the same bits. Returns this lane's largest
  // logit of them all (NaN where all are).
  template <int STEP, int U, int N>
  __device__ __forceinline__ float add(const Group<U, N>& g) {
    float all = 0.f;
#pragma unroll
    for (int u0 = 0; u0 < U; u0 += STEP) {
      if (u0 >= g.n) break;
      float top = max_of(g.x[u0]);
#pragma unroll
      for (int u = u0 + 1; u < u0 + STEP; ++u)
        if (u < g.n) top = fmaxf(top, max_of(g.x[u]));
      meet(top);
#pragma unroll
      for (int u = u0; u < u0 + STEP; ++u)
        if (u < g.n) add_met(g.x[u]);
      all = u0 ? fmaxf(all, top) : top;
    }
    return all;
  }
  // over the workgroup, for every thread
  template <int NT>
  __device__ __forceinline__ Acc join(Acc* lds) const {
    Acc a = acc_empty();
    if (over > -INFINITY) {  // (alike in all lanes; else all logits were -inf or NaN)
      a.m = max64(most);
      const float at = fmaf(a.m, c, -k), e = exp2_fast(at), sum = sum64(s);
      a.s = sum / e;
      if (ENT) a.w = fminf(fmaf(-at, sum, sum64(w)) / (e * c), 0.f);
      if (SM == TWO_SQUARE) a.s1 = sum64(s1) / (e * e);
      if (SM == TWO_EXP) a.s1 = sum64(s1) / exp2_fast(fmaf(a.m, kLog2e, -k1));
    } else {
      a.s = sum64(s);
    }
    if (lane_id() == 0) lds[threadIdx.x >> 6] = a;
    __syncthreads();
    a = lane_id() < NT / 64 ? lds[lane_id()] : acc_empty();
    acc_wave<ENT, SM != ONE>(a, c, kLog2e);
    return a;
  }
};
template <bool TWO>
DEV bool served(const Acc& a) {
  return a.s == a.s && (!TWO || a.s1 == a.s1);
}

// Hands columns v0 .. v1 of a row to add(group), -inf in the place of columns behind the end; columns
// rise from vector to vector and from group to group. The loads of one group are in flight while
// the one before it is worked on.
template <class T, int NT, int U, bool ONCE, class F>
DEV void scan(const T* row, int v0, int v1, F&& add) {
  constexpr int N = kVec<T>, step = NT * N;
  int i = v0 + (int)threadIdx.x * N, b = v0;
  u32x4 next[U];
  // (of the last group a lane loads the vectors that are whole)
  auto load = [&](int from, int at) {
    if (from + U * step <= v1) {
#pragma unroll
      for (int u = 0; u < U; ++u) next[u] = load16<ONCE>(row + at + u * step);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at + u * step + N <= v1) next[u] = load16<ONCE>(row + at + u * step);
    }
  };
  Group<U, N> g;
  g.step = step;
  load(b, i);
  for (; b + U * step <= v1; b += U * step, i += U * step) {
#pragma unroll
    for (int u = 0; u < U; ++u) unpack<T>(next[u], g.x[u]);
    if (b + U * step < v1) load(b + U * step, i + U * step);
    g.n = U;
    g.col = i;
    add(g);
  }
  if (b >= v1) return;
  g.n = (v1 - b + step - 1) / step;
  g.col = i;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u >= g.n) break;
    if (i + u * step + N <= v1)
      unpack<T>(next[u], g.x[u]);
    else
      load_tail<T>(row, i + u * step, v1, g.x[u]);
  }
  add(g);
}

// Writes f(z) over columns v0 .. v1 of a row, BACK: the last ones first. Every element is read before
// it is written, by the thread that writes it: the output may be the input.
template <class T, class G, int NT, int U, bool ONCE, bool BACK = false, class F>
DEV void map_row(const T* z, G* dz, int v0, int v1, F&& f) {
  constexpr int N = kVec<T>, step = NT * N;
  const int i0 = v0 + (int)threadIdx.x * N, groups = (v1 - v0) / (U * step);
  auto rest = [&] {  // fewer than U steps
    int i = i0 + groups * U * step;
    for (; i + N <= v1; i += step) {
      float x[N];
      unpack<T>(load16<ONCE>(z + i), x);
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = f(x[j]);
      store_vec<G, N>(dz + i, x);
    }
    for (int j = 0; j < N; ++j)
      if (i + j < v1) dz[i + j] = to_out<G>(f(cvt(z[i + j])));
  };
  if (BACK) rest();
  for (int n = 0; n < groups; ++n) {
    const int i = i0 + (BACK ? groups - 1 - n : n) * U * step;
    u32x4 v[U];
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
  if (!BACK) rest();
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
