// Operators on a matrix of logits [rows][vocab]: log probabilities of given tokens with the
// entropy and the top alternatives, their gradient, and distillation from a teacher's top logits
// with its gradient.
//
// Every row is a softmax over tens of thousands of logits, and all that a row gives besides its
// gradient is a few numbers: the floor is the logits read once and the gradient written once.
// One pass keeps, per lane, a reference m, s = sum exp((z - m) / tau) and w = sum exp(..) (z - m);
// lanes, waves and parts of a row are joined by rescaling to the largest reference. Sums are fp32
// over at most a few thousand terms per lane. The order of all sums is fixed by the shape alone.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "mebp_internal.h"

namespace mebp {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNone = -FLT_MAX;  // reference of a lane that has seen no logit above -inf
constexpr int NT = 256, NW = NT / 64;

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

// 16 bytes from an address that is a multiple of the element size alone: rows of an odd pitch
// start anywhere, and the memory pipeline takes such accesses as they are.
template <class T>
DEV uint4 load16(const T* p) {
  uint4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
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
  __builtin_memcpy(p, w, sizeof w);
}

template <class G>
DEV G to_out(float g) {
  return (G)g;
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

// Adds N logits whose largest is vmax. The reference only follows where a logit lies more than
// `lift` above it, 2^32 times its weight: fp32 holds the sums as well with a stale one, and nearly
// no vector moves it. NaN and +inf logits make s NaN: exp(NaN), and exp(inf - inf).
template <bool ENT, bool TWO, int N>
DEV void acc_add(Acc& a, const float (&x)[N], float vmax, float c, float c1, float lift) {
  if (vmax > a.m + lift) acc_move<ENT, TWO>(a, vmax, c, c1);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float d = x[j] - a.m;
    const float e = exp2_fast(d * c);
    a.s += e;
    // (a logit of -inf has weight 0, and 0 times -inf is not)
    if (ENT) a.w = fmaf(e, fmaxf(d, -1e30f), a.w);
    if (TWO) a.s1 += exp2_fast(d * c1);
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
template <bool ENT, bool TWO>
DEV void acc_block(Acc& a, float c, float c1, Acc* lds) {
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

// ------------------------------------------------------------------ top alternatives
// A logit's place in a row's order is one 64-bit key: the value's bits in their numerical order
// above the complement of its column, so that equal logits rank by the lower column and no two
// keys are alike. 0 is below every logit's key. Each wave keeps its 64 largest keys sorted, one
// per lane, and appends the logits above the k-th to a buffer, which is sorted and merged in
// batches of 64: about k ln(n / 512) of n logits get that far.
DEV uint32_t order_bits(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);  // -0 ranks as +0
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
DEV float order_value(uint32_t o) {
  return __builtin_bit_cast(float, o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
DEV u64 order_key(float x, int col) { return (u64)order_bits(x) << 32 | (uint32_t)~col; }

DEV u64 keep(u64 a, u64 b, bool larger) { return (a > b) == larger ? a : b; }

DEV u64 sort64(u64 key) {
  const int l = lane_id();
#pragma unroll
  for (int k = 2; k <= 64; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) key = keep(key, __shfl_xor(key, j, 64), ((l & k) == 0) == ((l & j) == 0));
  return key;
}
// the 64 largest of two sorted lists, sorted
DEV u64 merge64(u64 a, u64 b) {
  const int l = lane_id();
  const u64 r = __shfl(b, 63 - l, 64);
  u64 key = a > r ? a : r;
#pragma unroll
  for (int j = 32; j > 0; j >>= 1) key = keep(key, __shfl_xor(key, j, 64), (l & j) == 0);
  return key;
}

struct Top {
  u64 list;    // this lane's key of the sorted list
  float thr;   // only logits above it can be among the first k
  int cnt, k;  // buffered keys, k (both the same in all lanes)
};

DEV void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// merges the last `n` keys of the buffer
DEV void top_flush(Top& t, u64* buf, int n) {
  wave_lds_fence();
  const int l = lane_id();
  t.cnt -= n;
  const u64 key = l < n ? buf[t.cnt + l] : 0ull;
  wave_lds_fence();
  t.list = merge64(t.list, sort64(key));
}
DEV float top_threshold(const Top& t) {
  const u64 key = __shfl(t.list, t.k - 1, 64);
  return key ? order_value((uint32_t)(key >> 32)) : -INFINITY;
}

// Columns rise from one vector of a wave to the next, so a logit that equals the k-th one of the
// earlier vectors ranks behind it and the comparison may be strict; within a vector lanes and
// elements do not rise together, hence one threshold for all of it. `buf`: 128 keys.
template <int N>
DEV void top_add(Top& t, u64* buf, const float (&x)[N], float vmax, int col) {
  if (!__any(vmax > t.thr)) return;
  bool flushed = false;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const bool p = x[j] > t.thr;
    const u64 mask = __ballot(p);
    if (!mask) continue;
    if (p) buf[t.cnt + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = order_key(x[j], col + j);
    t.cnt += __popcll(mask);
    if (t.cnt >= 64) {
      top_flush(t, buf, 64);
      flushed = true;
    }
  }
  if (flushed) t.thr = top_threshold(t);
}

// ------------------------------------------------------------------ one pass over part of a row
template <class T, bool ENT, bool TWO, bool TOP>
DEV void scan(const T* row, int v0, int v1, float c, float c1, float lift, Acc& a, Top& t, u64* buf) {
  constexpr int N = kVec<T>;
  const int step = NT * N;
  auto add = [&](const float(&x)[N], int col) {
    float vmax = x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) vmax = fmaxf(vmax, x[j]);
    acc_add<ENT, TWO, N>(a, x, vmax, c, c1, lift);
    if constexpr (TOP) top_add<N>(t, buf, x, vmax, col);
  };
  int i = v0 + (int)threadIdx.x * N;
  int b = v0;
  for (; b + step <= v1; b += step, i += step) {
    float x[N];
    unpack<T>(load16(row + i), x);
    add(x, i);
  }
  if (b < v1) {
    float x[N];
    load_tail<T>(row, i, v1, x);
    add(x, i);
  }
}

// joins the waves' lists into the first wave's
DEV void top_block(Top& t, u64* buf, u64* lists) {
  if (t.cnt > 0) top_flush(t, buf, t.cnt);
  const int wave = threadIdx.x >> 6, l = lane_id();
  if (wave > 0) lists[(wave - 1) * 64 + l] = t.list;
  __syncthreads();
  if (wave == 0)
    for (int i = 0; i < NW - 1; ++i) t.list = merge64(t.list, lists[i * 64 + l]);
}

// ------------------------------------------------------------------ log probabilities
// A row with no logit above -inf has lse -inf, entropy 0 and no alternatives; a NaN or +inf logit
// makes its numbers NaN.
DEV void write_scores(const ScoreArgs& p, size_t row, const Acc& a, float zt, u64 list) {
  const bool empty = a.s == 0.f;
  const float log_s = logf(a.s), base = a.m * p.inv_tau;
  const int l = lane_id();
  if (l == 0) {
    if (p.lse) p.lse[row] = empty ? -INFINITY : base + log_s;
    if (p.entropy) p.entropy[row] = empty ? 0.f : log_s - a.w / a.s * p.inv_tau;
    if (p.logp) {
      const int t = p.targets[row];
      p.logp[row] = t < 0 ? 0.f : t >= p.vocab ? NAN : empty ? -INFINITY : (zt - a.m) * p.inv_tau - log_s;
    }
  }
  if (l < p.top_k) {
    if (p.top_ids) p.top_ids[row * p.top_k + l] = list ? (int)~(uint32_t)list : -1;
    if (p.top_logp)
      p.top_logp[row * p.top_k + l] =
          list ? (order_value((uint32_t)(list >> 32)) - a.m) * p.inv_tau - log_s : -INFINITY;
  }
}

template <class T>
DEV float target_logit(const ScoreArgs& p, const T* z, size_t row) {
  if (!p.logp) return 0.f;
  const int t = p.targets[row];
  return t >= 0 && t < p.vocab ? cvt(z[t]) : 0.f;
}

// One workgroup per part of a row; the only part of a row writes its scores, others their
// statistics and lists for k_scores_join.
template <class T, bool TOP>
__global__ __launch_bounds__(NT) void k_scores(ScoreArgs p) {
  __shared__ Acc red[NW];
  __shared__ u64 buf[TOP ? NW * 128 : 1], lists[TOP ? (NW - 1) * 64 : 1];
  const size_t row = blockIdx.x / p.split.n;
  const int part = (int)(blockIdx.x % p.split.n);
  const T* z = (const T*)p.z + row * p.ld;
  const int v0 = part * p.split.cols, v1 = min(p.vocab, v0 + p.split.cols);
  Acc a = acc_empty();
  Top t{0ull, -INFINITY, 0, p.top_k};
  u64* mine = buf + (TOP ? (threadIdx.x >> 6) * 128 : 0);
  scan<T, true, false, TOP>(z, v0, v1, p.c, 0.f, p.lift, a, t, mine);
  acc_block<true, false>(a, p.c, 0.f, red);
  if constexpr (TOP) top_block(t, mine, lists);
  if (threadIdx.x >= 64) return;
  if (p.split.n == 1) {
    write_scores(p, row, a, target_logit<T>(p, z, row), t.list);
  } else {
    if (lane_id() == 0) p.split.stats[blockIdx.x] = make_float4(a.m, a.s, a.w, 0.f);
    if (TOP && lane_id() < p.top_k) p.split.keys[(size_t)blockIdx.x * p.top_k + lane_id()] = t.list;
  }
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

// one wave per row
template <class T>
__global__ __launch_bounds__(64) void k_scores_join(ScoreArgs p) {
  const size_t row = blockIdx.x;
  const int l = lane_id();
  const Acc a = join_parts<true, false>(p.split, row, p.c, 0.f);
  u64 list = 0;
  if (p.top_k)
    for (int i = 0; i < p.split.n; ++i)
      list = merge64(list, l < p.top_k ? p.split.keys[(row * p.split.n + i) * p.top_k + l] : 0ull);
  write_scores(p, row, a, target_logit<T>(p, (const T*)p.z + row * p.ld, row), list);
}

// ------------------------------------------------------------------ gradients
// Writes g(z) over columns v0 .. v1 of a row. Every element is read before it is written, by the
// thread that writes it: the output may be the input.
template <class T, class G, class F>
DEV void map_row(const T* z, G* dz, int v0, int v1, F&& f) {
  constexpr int N = kVec<T>;
  const int step = NT * N;
  int i = v0 + (int)threadIdx.x * N, b = v0;
  for (; b + step <= v1; b += step, i += step) {
    float x[N];
    unpack<T>(load16(z + i), x);
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = f(x[j]);
    store_vec<G, N>(dz + i, x);
  }
  if (b < v1)
    for (int j = 0; j < N; ++j)
      if (i + j < v1) dz[i + j] = to_out<G>(f(cvt(z[i + j])));
}

// what a workgroup wrote is in order before what follows the barrier writes to the same places
DEV void stores_done() {
  wait_vmcnt<0>();
  __syncthreads();
}

// d logp_t / dz = (1[t] - q) / tau and dH / dz = -q (ln q + H) / tau, weighted by the gradients of
// the two; the target's column is written again with its 1.
template <class T, class G>
__global__ __launch_bounds__(NT) void k_scores_grad(ScoreGradArgs p) {
  const size_t row = blockIdx.x / p.split.n;
  const int part = (int)(blockIdx.x % p.split.n);
  const T* z = (const T*)p.z + row * p.ld;
  G* dz = (G*)p.dz + row * p.ldd;
  const int v0 = part * p.split.cols, v1 = min(p.vocab, v0 + p.split.cols);
  const int t = p.targets && p.d_logp ? p.targets[row] : -1;
  const float lse = p.lse[row];
  float A = t < 0 ? 0.f : p.d_logp[row] * p.inv_tau;
  if (t >= p.vocab) A = NAN;
  const float B = p.d_entropy ? p.d_entropy[row] * p.inv_tau : 0.f;
  const float H = p.d_entropy ? p.entropy[row] : 0.f;
  const bool here = t >= v0 && t < v1, empty = lse == -INFINITY;
  const float zt = here && threadIdx.x == 0 ? cvt(z[t]) : 0.f;
  const float AB = A + B * H;
  auto f = [&](float x) {
    const float lq = x * p.inv_tau - lse;
    // (q = 0 at logits of -inf)
    return -exp2_fast(lq * kLog2e) * fmaf(B, fmaxf(lq, -1e30f), AB);
  };
  if (empty) {
    map_row<T, G>(z, dz, v0, v1, [](float) { return 0.f; });
    return;
  }
  if (here) __syncthreads();  // zt is read before any thread writes (the output may be the input)
  map_row<T, G>(z, dz, v0, v1, f);
  if (!here) return;
  stores_done();
  if (threadIdx.x == 0) dz[t] = to_out<G>(f(zt) + A);
}

// ------------------------------------------------------------------ distillation
// With p = softmax(teacher / tau) over the K entries, q = softmax(z / tau) and q1 = softmax(z) over
// the vocabulary, a row's loss is w (alpha tau^2 KL(p, q) + (1 - alpha) CE(z, target)) and its
// gradient w (alpha tau (q - p) + (1 - alpha) (q1 - 1[target])).
//
// The teacher's entries and the target, held by the first wave.
struct Teacher {
  int id;       // this lane's entry, -1 if it has none
  float p, lp;  // its probability and the logarithm
  bool any;     // the row has an entry
};

DEV Teacher teacher_row(const DistillArgs& a, size_t row) {
  const int l = lane_id();
  Teacher t{-1, 0.f, 0.f, false};
  float v = -INFINITY;
  if (l < a.k && a.alpha > 0.f) {
    t.id = a.ids[row * a.k + l];
    v = a.logits[row * a.k + l] * a.inv_tau;
    if (t.id < 0 || v == -INFINITY) {
      t.id = -1;
      v = -INFINITY;
    }
  }
  t.any = __any(t.id >= 0);
  if (!t.any) return t;
  float M = wave_max(v);
  const float e = v == -INFINITY ? 0.f : exp2_fast((v - M) * kLog2e);
  const float S = wave_sum(e);
  t.p = e / S;
  t.lp = (v - M) - logf(S);
  if (t.id >= a.vocab) t.p = NAN;
  return t;
}

// the target of the hard label's term: -1 if the row or the call has none
DEV int hard_target(const DistillArgs& a, size_t row) { return a.alpha < 1.f ? a.targets[row] : -1; }

// the row's loss without its weight (all lanes of a wave; zk, zt: the student's logits of this
// lane's entry and of the target)
DEV float distill_loss(const DistillArgs& a, const Acc& st, const Teacher& t, float zk, int target, float zt, bool two) {
  const bool empty = st.s == 0.f;
  float loss = 0.f;
  if (t.any) {
    // an entry whose probability rounds to 0 adds nothing
    const float term = t.id < 0 || t.p == 0.f ? 0.f : t.p * (t.lp - (zk - st.m) * a.inv_tau);
    const float mass = wave_sum(t.id < 0 ? 0.f : t.p);
    loss = empty ? INFINITY : a.alpha * a.tau * a.tau * (wave_sum(term) + mass * logf(st.s));
  }
  if (target >= 0) {
    const float ce = target >= a.vocab ? NAN : empty ? INFINITY : logf(two ? st.s1 : st.s) - (zt - st.m);
    loss += (1.f - a.alpha) * ce;
  }
  return loss;
}

DEV float row_weight(const DistillArgs& a, size_t row) { return a.weight ? a.weight[row] : 1.f; }

// Statistics of a part of a row (TWO: of both softmaxes); the only part of a row that needs no
// gradient writes the loss. The first part keeps the student's logits at the entries: a gradient
// that overwrites the logits reads them from there.
template <class T, bool TWO>
__global__ __launch_bounds__(NT) void k_distill_stats(DistillArgs p) {
  __shared__ Acc red[NW];
  const size_t row = blockIdx.x / p.split.n;
  const int part = (int)(blockIdx.x % p.split.n);
  const float w = row_weight(p, row);
  if (w == 0.f) {
    if (!p.dz && part == 0 && threadIdx.x == 0) p.loss[row] = 0.f;
    return;
  }
  const T* z = (const T*)p.z + row * p.ld;
  const int v0 = part * p.split.cols, v1 = min(p.vocab, v0 + p.split.cols);
  Acc a = acc_empty();
  Top none{};
  scan<T, false, TWO, false>(z, v0, v1, p.c, kLog2e, p.lift, a, none, nullptr);
  acc_block<false, TWO>(a, p.c, kLog2e, red);
  if (threadIdx.x >= 64) return;
  const int l = lane_id();
  if (p.split.n > 1 || p.dz) {
    if (l == 0) p.split.stats[blockIdx.x] = make_float4(a.m, a.s, 0.f, a.s1);
    if (part > 0) return;
  }
  const Teacher t = teacher_row(p, row);
  const int target = hard_target(p, row);
  const float zk = t.id >= 0 && t.id < p.vocab ? cvt(z[t.id]) : 0.f;
  const float zt = target >= 0 && target < p.vocab ? cvt(z[target]) : 0.f;
  if (p.split.n > 1 || p.dz) {
    float* keep = p.split.picked + row * 65;
    keep[l] = zk;
    if (l == 0) keep[64] = zt;
  } else {
    const float loss = w * distill_loss(p, a, t, zk, target, zt, TWO);
    if (l == 0) p.loss[row] = loss;
  }
}

template <bool TWO>
__global__ __launch_bounds__(64) void k_distill_join(DistillArgs p) {
  const size_t row = blockIdx.x;
  const float w = row_weight(p, row);
  if (w == 0.f) return;
  const Acc a = join_parts<false, TWO>(p.split, row, p.c, kLog2e);
  const float* keep = p.split.picked + row * 65;
  const float loss = w * distill_loss(p, a, teacher_row(p, row), keep[lane_id()], hard_target(p, row), keep[64], TWO);
  if (lane_id() == 0) p.loss[row] = loss;
}

// The gradient of a part of a row: the dense terms everywhere, then the entries' and the target's
// columns once more with the sparse ones.
template <class T, class G, bool TWO>
__global__ __launch_bounds__(NT) void k_distill_grad(DistillArgs p) {
  __shared__ float s_p[64];
  __shared__ int s_id[64];
  __shared__ float s_row[4];
  const size_t row = blockIdx.x / p.split.n;
  const int part = (int)(blockIdx.x % p.split.n);
  const T* z = (const T*)p.z + row * p.ld;
  G* dz = (G*)p.dz + row * p.ldd;
  const int v0 = part * p.split.cols, v1 = min(p.vocab, v0 + p.split.cols);
  const float w = row_weight(p, row);
  if (w == 0.f) {
    if (part == 0 && threadIdx.x == 0) p.loss[row] = 0.f;
    map_row<T, G>(z, dz, v0, v1, [](float) { return 0.f; });
    return;
  }
  const int target = hard_target(p, row);
  float zt = 0.f;
  if (threadIdx.x < 64) {
    const Acc a = join_parts<false, TWO>(p.split, row, p.c, kLog2e);
    const Teacher t = teacher_row(p, row);
    const float* keep = p.split.picked + row * 65;
    const float zk = keep[lane_id()];
    zt = keep[64];
    const float loss = w * distill_loss(p, a, t, zk, target, zt, TWO);
    if (part == 0 && lane_id() == 0) p.loss[row] = loss;
    s_p[lane_id()] = t.p;
    s_id[lane_id()] = t.id;
    // the coefficients of exp(.. - m): of the softmax at tau and of the one at 1
    const float mass = t.any ? wave_sum(t.id < 0 ? 0.f : t.p) : 0.f;
    const float soft = w * p.alpha * p.tau * mass, hard = target >= p.vocab ? NAN : target >= 0 ? w * (1.f - p.alpha) : 0.f;
    if (lane_id() == 0) {
      s_row[0] = a.m;
      s_row[1] = a.s == 0.f ? 0.f : (TWO ? soft : soft + hard) / a.s;
      s_row[2] = TWO && a.s1 > 0.f ? hard / a.s1 : 0.f;
      s_row[3] = a.s == 0.f;
    }
  }
  __syncthreads();
  const float m = s_row[0], c0 = s_row[1], c1 = s_row[2];
  const bool empty = s_row[3] != 0.f;
  if (empty) {
    map_row<T, G>(z, dz, v0, v1, [](float) { return 0.f; });
    return;
  }
  auto f = [&](float x) {
    const float d = x - m;
    float g = c0 * exp2_fast(d * p.c);
    if (TWO) g = fmaf(c1, exp2_fast(d * kLog2e), g);
    return g;
  };
  map_row<T, G>(z, dz, v0, v1, f);
  stores_done();
  if (threadIdx.x >= 64) return;
  // the first of entries with the same column writes it, with the sum of their probabilities
  const int l = lane_id(), id = s_id[l];
  float P = 0.f;
  bool first = true, seen = false;
  for (int j = 0; j < p.k; ++j) {
    const int o = s_id[j];
    seen |= o == target;
    if (o != id) continue;
    P += s_p[j];
    first &= j >= l;
  }
  const float hard = w * (1.f - p.alpha);
  if (id >= v0 && id < v1 && first) {
    const float zk = p.split.picked[row * 65 + l];
    dz[id] = to_out<G>(f(zk) - w * p.alpha * p.tau * P - (id == target ? hard : 0.f));
  }
  if (l == 0 && !seen && target >= v0 && target < v1) dz[target] = to_out<G>(f(zt) - hard);
}

// ------------------------------------------------------------------ launches
template <class F>
hipError_t by_type(int dtype, F&& f) {
  switch (dtype) {
    case LOGIT_F32: return f((float*)nullptr);
    case LOGIT_F16: return f((f16*)nullptr);
    default: return f((bf16*)nullptr);
  }
}
double type_bytes(int dtype) { return dtype == LOGIT_F32 ? 4.0 : 2.0; }

}  // namespace

// Parts of a row: enough workgroups for the chip where there are few rows, of no fewer than 4096
// columns each.
LogitSplit logit_split(int rows, int vocab) {
  LogitSplit s{};
  const int want = std::min(kLogitParts, (1024 + rows - 1) / std::max(rows, 1));
  const int most = (vocab + 4095) / 4096;
  const int n = std::max(1, std::min(want, most));
  s.cols = ((vocab + n - 1) / n + 2047) / 2048 * 2048;
  s.n = (vocab + s.cols - 1) / s.cols;
  return s;
}

hipError_t launch_scores(ScoreArgs a, int dtype, hipStream_t st) {
  const unsigned grid = (unsigned)((size_t)a.rows * a.split.n);
  hipError_t e = by_type(dtype, [&](auto* tp) {
    using T = std::remove_pointer_t<decltype(tp)>;
    const double bytes = (double)a.rows * a.vocab * sizeof(T);
    if (a.top_k)
      MEBP_TIMED(st, "token_scores_top", 0.0, bytes, hipLaunchKernelGGL((k_scores<T, true>), dim3(grid), dim3(NT), 0, st, a));
    else
      MEBP_TIMED(st, "token_scores", 0.0, bytes, hipLaunchKernelGGL((k_scores<T, false>), dim3(grid), dim3(NT), 0, st, a));
    if (a.split.n > 1)
      MEBP_TIMED(st, "token_scores_join", 0.0, (double)grid * (16 + 8 * a.top_k),
                 hipLaunchKernelGGL((k_scores_join<T>), dim3(a.rows), dim3(64), 0, st, a));
    return hipGetLastError();
  });
  return e;
}

hipError_t launch_scores_grad(ScoreGradArgs a, int dtype, int gtype, hipStream_t st) {
  const unsigned grid = (unsigned)((size_t)a.rows * a.split.n);
  const double bytes = (double)a.rows * a.vocab * (type_bytes(dtype) + type_bytes(gtype));
  return by_type(dtype, [&](auto* tp) {
    return by_type(gtype, [&](auto* gp) {
      using T = std::remove_pointer_t<decltype(tp)>;
      using G = std::remove_pointer_t<decltype(gp)>;
      MEBP_TIMED(st, a.z == a.dz ? "token_scores_grad_inplace" : "token_scores_grad", 0.0, bytes,
                 hipLaunchKernelGGL((k_scores_grad<T, G>), dim3(grid), dim3(NT), 0, st, a));
      return hipGetLastError();
    });
  });
}

hipError_t launch_distill(DistillArgs a, int dtype, int gtype, hipStream_t st) {
  const unsigned grid = (unsigned)((size_t)a.rows * a.split.n);
  const double read = (double)a.rows * a.vocab * type_bytes(dtype);
  const bool two = a.alpha < 1.f && a.tau != 1.f;
  auto run = [&](auto* tp, auto tw) {
    using T = std::remove_pointer_t<decltype(tp)>;
    constexpr bool TWO = decltype(tw)::value;
    MEBP_TIMED(st, "distill_stats", 0.0, read,
               hipLaunchKernelGGL((k_distill_stats<T, TWO>), dim3(grid), dim3(NT), 0, st, a));
    if (!a.dz) {
      if (a.split.n > 1)
        MEBP_TIMED(st, "distill_join", 0.0, (double)grid * 16,
                   hipLaunchKernelGGL((k_distill_join<TWO>), dim3(a.rows), dim3(64), 0, st, a));
      return hipGetLastError();
    }
    return by_type(gtype, [&](auto* gp) {
      using G = std::remove_pointer_t<decltype(gp)>;
      MEBP_TIMED(st, a.z == a.dz ? "distill_grad_inplace" : "distill_grad", 0.0,
                 read + (double)a.rows * a.vocab * type_bytes(gtype),
                 hipLaunchKernelGGL((k_distill_grad<T, G, TWO>), dim3(grid), dim3(NT), 0, st, a));
      return hipGetLastError();
    });
  };
  return by_type(dtype, [&](auto* tp) {
    return two ? run(tp, std::true_type()) : run(tp, std::false_type());
  });
}

}  // namespace mebp
