// Distillation from a teacher's top logits: row losses and the gradient w.r.t. the student's logits.
#include <utility>

#include "logits_device.h"

namespace mebp {
namespace {

constexpr int NT = 256;

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
    v = a.logits[row * a.k + l];
    if (t.id < 0 || v == -INFINITY) {
      t.id = -1;
      v = -INFINITY;
    }
  }
  t.any = __any(t.id >= 0);
  if (!t.any) return t;
  // (the difference first: a quotient by tau may leave fp32, and has fewer bits below its point)
  const float d = (v - max64(v)) * a.inv_tau;
  const float e = v == -INFINITY ? 0.f : exp2_fast(d * kLog2e);
  const float S = sum64(e);
  t.p = e / S;
  t.lp = d - logf(S);
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
    // tau times the term (a distance of the size of the type's lowest value may be no number in
    // temperatures, and is one times p); an entry whose probability rounds to 0 adds nothing
    const float term = t.id < 0 || t.p == 0.f ? 0.f : t.p * (t.lp * a.tau) - t.p * (zk - st.m);
    const float mass = sum64(t.id < 0 ? 0.f : t.p);
    loss = empty ? INFINITY : a.alpha * a.tau * (sum64(term) + mass * logf(st.s) * a.tau);
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
// ONCE: no gradient reads the logits again.
template <class T, Softmaxes SM, bool ONCE, int NT>
__global__ __launch_bounds__(NT) void k_distill_stats(DistillArgs p) {
  constexpr bool TWO = SM != ONE;
  __shared__ Acc red[NT / 64];
  const size_t row = blockIdx.x / p.split.n;
  const int part = (int)(blockIdx.x % p.split.n);
  const float w = row_weight(p, row);
  if (w == 0.f) {
    if (!p.dz && part == 0 && threadIdx.x == 0) p.loss[row] = 0.f;
    return;
  }
  const T* z = (const T*)p.z + row * p.ld;
  const int v0 = part * p.split.cols, v1 = min(p.vocab, v0 + p.split.cols);
  Sums<false, SM> sums;
  sums.start(p.c, p.lift);
  scan<T, NT, 4, ONCE>(z, v0, v1, [&](const auto& g) { sums.template add<4>(g); });
  Acc a = sums.template join<NT>(red);
  if (!served<TWO>(a)) {
    a = acc_empty();
    scan<T, NT, 1, false>(z, v0, v1, [&](const auto& g) { acc_add<false, TWO>(a, g, p.c, kLog2e); });
    __syncthreads();
    acc_block<NT, false, TWO>(a, p.c, kLog2e, red);
  }
  if (threadIdx.x >= 64) return;
  const int l = lane_id();
  if (p.split.n > 1) {
    if (l == 0) p.split.stats[blockIdx.x] = make_float4(a.m, a.s, 0.f, a.s1);
    if (part > 0) return;
  }
  const Teacher t = teacher_row(p, row);
  const int target = hard_target(p, row);
  const float zk = t.id >= 0 && t.id < p.vocab ? cvt(z[t.id]) : 0.f;
  const float zt = target >= 0 && target < p.vocab ? cvt(z[target]) : 0.f;
  if (p.split.n > 1) {
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

// What a row's gradient is made of (LDS, by the first wave).
struct RowTerms {
  float m, c0, c1;  // reference, coefficients of exp((z - m) / tau) and of exp(z - m)
  bool empty;       // no logit above -inf, or no term: no gradient
  // the columns that have a sparse term, -1: none, and the whole gradient there; the target is the last
  int col[65];
  float g[65];
};

template <bool TWO>
DEV float dense_grad(float x, float m, float c0, float c1, float c) {
  const float d = x - m;
  float g = c0 * exp2_fast(d * c);
  if (TWO) g = fmaf(c1, exp2_fast(d * kLog2e), g);
  return g;
}

// The sparse terms of a row without its statistics: the first of entries with the same column has it,
// with the sum of their probabilities; the target's column is one of its own where no entry has it.
struct Sparse {
  float P;
  bool first, seen;
};
DEV Sparse sparse_terms(const DistillArgs& p, const Teacher& t, int target) {
  Sparse r{0.f, true, false};
  for (int j = 0; j < p.k; ++j) {
    const int o = __builtin_amdgcn_readlane(t.id, j);
    const float q = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, t.p), j));
    r.seen |= o == target;
    if (o != t.id) continue;
    r.P += q;
    r.first &= j >= (int)lane_id();
  }
  return r;
}

template <bool TWO>
DEV void set_terms(const DistillArgs& p, const Acc& a, const Teacher& t, const Sparse& sp, float zk, int target, float zt,
                   float w, RowTerms& r) {
  const int l = lane_id();
  const float mass = t.any ? sum64(t.id < 0 ? 0.f : t.p) : 0.f;
  const float soft = w * p.alpha * p.tau * mass, one = w * (1.f - p.alpha);
  const float hard = target >= p.vocab ? NAN : target >= 0 ? one : 0.f;
  const bool empty = a.s == 0.f || (!t.any && target < 0);
  const float c0 = (TWO ? soft : soft + hard) / a.s, c1 = TWO ? hard / a.s1 : 0.f;
  r.col[l] = t.id < p.vocab && sp.first && !empty ? t.id : -1;
  r.g[l] = dense_grad<TWO>(zk, a.m, c0, c1, p.c) - w * p.alpha * p.tau * sp.P - (t.id == target ? one : 0.f);
  if (l == 0) {
    r.m = a.m;
    r.c0 = c0;
    r.c1 = c1;
    r.empty = empty;
    r.col[64] = sp.seen || empty || target >= p.vocab ? -1 : target;
    r.g[64] = dense_grad<TWO>(zt, a.m, c0, c1, p.c) - one;
  }
}

// Writes the columns with a sparse term among v0 .. v1, over their dense ones (the first wave, after
// every wave's stores of the row).
template <class G>
DEV void sparse_grad(const RowTerms& r, int v0, int v1, G* dz) {
  const int l = lane_id();
  if (r.col[l] >= v0 && r.col[l] < v1) dz[r.col[l]] = to_out<G>(r.g[l]);
  if (l == 0 && r.col[64] >= v0 && r.col[64] < v1) dz[r.col[64]] = to_out<G>(r.g[64]);
}

// The gradient of a part of a row: the dense terms everywhere, then the columns with sparse ones.
template <class T, class G, bool TWO>
__global__ __launch_bounds__(NT) void k_distill_grad(DistillArgs p) {
  __shared__ RowTerms terms;
  const size_t row = blockIdx.x / p.split.n;
  const int part = (int)(blockIdx.x % p.split.n);
  const T* z = (const T*)p.z + row * p.ld;
  G* dz = (G*)p.dz + row * p.ldd;
  const int v0 = part * p.split.cols, v1 = min(p.vocab, v0 + p.split.cols);
  const float w = row_weight(p, row);
  if (w == 0.f) {
    if (part == 0 && threadIdx.x == 0) p.loss[row] = 0.f;
    zero_row<G, NT>(dz, v0, v1);
    return;
  }
  if (threadIdx.x < 64) {
    const Acc a = join_parts<false, TWO>(p.split, row, p.c, kLog2e);
    const Teacher t = teacher_row(p, row);
    const int target = hard_target(p, row);
    const float* keep = p.split.picked + row * 65;
    const float zk = keep[lane_id()], zt = keep[64];
    const float loss = w * distill_loss(p, a, t, zk, target, zt, TWO);
    if (part == 0 && lane_id() == 0) p.loss[row] = loss;
    set_terms<TWO>(p, a, t, sparse_terms(p, t, target), zk, target, zt, w, terms);
  }
  __syncthreads();
  if (terms.empty) {
    zero_row<G, NT>(dz, v0, v1);
    return;
  }
  const float m = terms.m, c0 = terms.c0, c1 = terms.c1;
  auto f = [&](float x) { return dense_grad<TWO>(x, m, c0, c1, p.c); };
  map_row<T, G, NT, 4, true>(z, dz, v0, v1, f);
  stores_done();
  if (threadIdx.x < 64) sparse_grad(terms, v0, v1, dz);
}

// f(IC<0>()) .. f(IC<R - 1>()): a loop over registers, which only constants can index
template <class F, int... I>
DEV void each_of(std::integer_sequence<int, I...>, F&& f) {
  (f(IC<I>()), ...);
}
template <int R, class F>
DEV void each(F&& f) {
  each_of(std::make_integer_sequence<int, R>(), f);
}

// p + n as a scalar: each step's address is this and the same lane offset (else every step's lane
// offsets are kept in registers of their own)
template <class P>
DEV P* advance(P* p, int n) {
  p += n;
  asm volatile("" : "+s"(p));
  return p;
}

// Loss and gradient of a whole row by one workgroup, which holds up to R whole steps of it (16 bytes of
// each lane) in registers and L more in LDS from the statistics to the gradient: those logits are read
// once. What the row has beyond them is read a second time, the last of it first: that is still in the
// XCD's L2.
template <class T, class G, Softmaxes SM, int WG, int R, int L>
__global__ __launch_bounds__(WG, 4) void k_distill_row(DistillArgs p) {
  constexpr int N = kVec<T>, step = WG * N;
  constexpr bool TWO = SM != ONE;
  __shared__ RowTerms terms;
  __shared__ Acc red[WG / 64];
  const size_t row = blockIdx.x;
  const T* z = (const T*)p.z + row * p.ld;
  G* dz = (G*)p.dz + row * p.ldd;
  __shared__ u32x4 more[L ? L : 1][WG];
  const int V = p.vocab, steps = min(R, V / step), steps2 = L ? min(L, V / step - steps) : 0;
  const int held1 = steps * step, held = held1 + steps2 * step;
  const uint32_t lane = threadIdx.x * N;
  const float w = row_weight(p, row);
  if (w == 0.f) {
    if (threadIdx.x == 0) p.loss[row] = 0.f;
    zero_row<G, WG>(dz, 0, V);
    return;
  }
  u32x4 raw[R];
  {
    const T* at = z;
    each<R>([&](auto i) {
      constexpr int r = decltype(i)::value;
      if (r >= steps) return;
      raw[r] = load16<true>(at + lane);
      at = advance(at, step);
    });
  }
  // the first wave's sparse operands come with them
  Teacher t{};
  Sparse sp{};
  float zk = 0.f, zt = 0.f;
  int target = -1;
  if (threadIdx.x < 64) {
    t = teacher_row(p, row);
    target = hard_target(p, row);
    if (t.id >= 0 && t.id < V) zk = cvt(z[t.id]);
    if (target >= 0 && target < V) zt = cvt(z[target]);
    sp = sparse_terms(p, t, target);
  }
  Sums<false, SM> sums;
  sums.start(p.c, p.lift);
  each<R>([&](auto i) {
    constexpr int r = decltype(i)::value;
    if (r >= steps) return;
    asm volatile("" : "+v"(raw[r]));
    float x[N];
    unpack<T>(raw[r], x);
    sums.add(x);
  });
  if constexpr (L > 0) {
    const T* at = z + held1;
    for (int r = 0; r < steps2; r += 2, at += 2 * step) {
      u32x4 v[2];
      float x[N];
      v[0] = load16<true>(at + lane);
      if (r + 1 < steps2) v[1] = load16<true>(at + step + lane);
      more[r][threadIdx.x] = v[0];
      unpack<T>(v[0], x);
      sums.add(x);
      if (r + 1 == steps2) break;
      more[r + 1][threadIdx.x] = v[1];
      unpack<T>(v[1], x);
      sums.add(x);
    }
  }
  if (held < V) scan<T, WG, 2, false>(z, held, V, [&](const auto& h) { sums.template add<2>(h); });
  Acc a = sums.template join<WG>(red);
  const bool first_pass = served<TWO>(a);
  if (!first_pass) {
    a = acc_empty();
    scan<T, WG, 1, false>(z, 0, V, [&](const auto& g) { acc_add<false, TWO>(a, g, p.c, kLog2e); });
    __syncthreads();
    acc_block<WG, false, TWO>(a, p.c, kLog2e, red);
  }
  if (threadIdx.x < 64) {
    const float loss = w * distill_loss(p, a, t, zk, target, zt, TWO);
    if (threadIdx.x == 0) p.loss[row] = loss;
    set_terms<TWO>(p, a, t, sp, zk, target, zt, w, terms);
  }
  __syncthreads();
  if (terms.empty) {
    zero_row<G, WG>(dz, 0, V);
    return;
  }
  const float m = terms.m, c0 = terms.c0, c1 = terms.c1;
  if (!first_pass) {
    map_row<T, G, WG, 1, false>(z, dz, 0, V, [&](float x) { return dense_grad<TWO>(x, m, c0, c1, p.c); });
  } else {
    // weights at the row's own whole exponent, as Sums has them
    const float k = whole_exponent(m, p.c), k1 = whole_exponent(m, kLog2e), u = exp2_fast(-fmaf(m, p.c, -k));
    const float b0 = c0 * u, b1 = !TWO ? 0.f : c1 * (SM == TWO_SQUARE ? u * u : exp2_fast(-fmaf(m, kLog2e, -k1)));
    auto f = [&](float x) {
      const float e = exp2_fast(fmaf(x, p.c, -k));
      if (SM == ONE) return b0 * e;
      if (SM == TWO_SQUARE) return e * fmaf(b1, e, b0);
      return fmaf(b1, exp2_fast(fmaf(x, kLog2e, -k1)), b0 * e);
    };
    if (held < V) map_row<T, G, WG, 2, true, true>(z, dz, held, V, f);
    if constexpr (L > 0) {
      G* at = dz + held1;
      for (int r = 0; r < steps2; ++r, at += step) {
        float x[N];
        unpack<T>(more[r][threadIdx.x], x);
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = f(x[j]);
        store_vec<G, N>(at + lane, x);
      }
    }
    G* to = dz;
    each<R>([&](auto i) {
      constexpr int r = decltype(i)::value;
      if (r >= steps) return;
      // (unpacked again: the 32-bit values would not fit beside the others)
      asm volatile("" : "+v"(raw[r]));
      float x[N];
      unpack<T>(raw[r], x);
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = f(x[j]);
      store_vec<G, N>(to + lane, x);
      to = advance(to, step);
    });
  }
  stores_done();
  if (threadIdx.x < 64) sparse_grad(terms, 0, V, dz);
}

}  // namespace

hipError_t launch_distill(DistillArgs a, int dtype, int gtype, hipStream_t st) {
  const unsigned grid = (unsigned)((size_t)a.rows * a.split.n);
  const double read = (double)a.rows * a.vocab * type_bytes(dtype);
  const double both = read + (double)a.rows * a.vocab * type_bytes(gtype);
  const bool inplace = a.z == a.dz;
  auto stats = [&](auto* tp, auto sm, auto once, auto nt) {
    using T = std::remove_pointer_t<decltype(tp)>;
    constexpr int W = decltype(nt)::value;
    MEBP_TIMED(st, "distill_stats", 0.0, read,
               hipLaunchKernelGGL((k_distill_stats<T, (Softmaxes)decltype(sm)::value, decltype(once)::value, W>), dim3(grid),
                                  dim3(W), 0, st, a));
  };
  auto loss = [&](auto* tp, auto sm) {
    if (a.split.n == 1 && a.vocab > 16384) {
      stats(tp, sm, std::true_type(), IC<512>());
    } else {
      stats(tp, sm, std::true_type(), IC<NT>());
      if (a.split.n > 1)
        MEBP_TIMED(st, "distill_join", 0.0, (double)grid * 16,
                   hipLaunchKernelGGL((k_distill_join<decltype(sm)::value != ONE>), dim3(a.rows), dim3(64), 0, st, a));
    }
    return hipGetLastError();
  };
  auto grad = [&](auto* tp, auto* gp, auto sm) {
    using T = std::remove_pointer_t<decltype(tp)>;
    using G = std::remove_pointer_t<decltype(gp)>;
    constexpr Softmaxes SM = (Softmaxes)decltype(sm)::value;
    const size_t row = (size_t)a.vocab * sizeof(T);
    // as much of a row in registers as leaves none to spill: two exponentials' sums take more of them
    constexpr int R = SM == TWO_EXP ? 16 : 18;
    // few long rows go by parts, in two launches; from 96 of 151936 fp32 logits on a workgroup for each
    // row is faster (64 rows 23 us by rows and 19 by parts, 96: 24 and 27, 192: 31 and 49; bf16 22 and 17, 22
    // and 22, 25 and 37). Of 70000 .. 262144 fp32 and bf16 logits the two meet at 65 to 110 rows
    if (a.split.n > 1 && a.rows < 96 && row > R * 512 * 16) {
      stats(tp, sm, std::false_type(), IC<NT>());
      MEBP_TIMED(st, inplace ? "distill_grad_inplace" : "distill_grad", 0.0, both,
                 hipLaunchKernelGGL((k_distill_grad<T, G, SM != ONE>), dim3(grid), dim3(NT), 0, st, a));
      return hipGetLastError();
    }
    const char* name = inplace ? "distill_row_inplace" : "distill_row";
    auto run = [&](auto wg, auto lds) {
      constexpr int WG = decltype(wg)::value;
      MEBP_TIMED(st, name, 0.0, both,
                 hipLaunchKernelGGL((k_distill_row<T, G, SM, WG, R, decltype(lds)::value>), dim3(a.rows), dim3(WG), 0, st, a));
    };
    // the smallest workgroup whose registers hold the row, so that several share a compute unit; a row
    // beyond 144 KB has one to itself, and its LDS
    if (row <= R * 256 * 16)
      run(IC<256>(), IC<0>());
    else if (row <= R * 512 * 16)
      run(IC<512>(), IC<0>());
    else
      run(IC<1024>(), IC<9>());
    return hipGetLastError();
  };
  auto by_softmaxes = [&](auto&& f) {
    if (a.alpha == 1.f || a.tau == 1.f) return f(IC<ONE>());
    return a.tau == 2.f ? f(IC<TWO_SQUARE>()) : f(IC<TWO_EXP>());
  };
  return by_type(dtype, [&](auto* tp) {
    if (!a.dz) return by_softmaxes([&](auto sm) { return loss(tp, sm); });
    return by_type(gtype, [&](auto* gp) { return by_softmaxes([&](auto sm) { return grad(tp, gp, sm); }); });
  });
}

}  // namespace mebp
