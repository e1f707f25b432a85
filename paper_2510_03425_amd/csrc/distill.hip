// Distillation from a teacher's top logits: row losses and the gradient w.r.t. the student's logits.
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
  Acc a = acc_empty();
  scan<T, NT, 4, false>(z, v0, v1, [&](const auto& g) { acc_add<false, TWO>(a, g, p.c, kLog2e, p.lift); });
  acc_block<NT, false, TWO>(a, p.c, kLog2e, red);
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
    zero_row<G, NT>(dz, v0, v1);
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
    zero_row<G, NT>(dz, v0, v1);
    return;
  }
  auto f = [&](float x) {
    const float d = x - m;
    float g = c0 * exp2_fast(d * p.c);
    if (TWO) g = fmaf(c1, exp2_fast(d * kLog2e), g);
    return g;
  };
  map_row<T, G, NT, 4, true>(z, dz, v0, v1, f);
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

}  // namespace

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
