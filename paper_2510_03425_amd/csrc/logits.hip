// Log probabilities of given tokens with the entropy and the top alternatives, and their gradient,
// of a matrix of logits [rows][vocab].
#include "logits_device.h"

namespace mebp {
namespace {

// ------------------------------------------------------------------ top alternatives
// A logit's place in a row's order is one 64-bit key: the value's bits in their numerical order
// above the complement of its column, so that equal logits rank by the lower column and no two
// keys are alike. 0 is below every logit's key. Each wave keeps its 64 largest keys sorted, one
// per lane, and appends the logits above a threshold to a buffer, which is sorted and merged in
// batches of up to 64 (16 lanes do for 16 alternatives).
DEV uint32_t order_bits(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);  // -0 ranks as +0
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
DEV float order_value(uint32_t o) {
  return __builtin_bit_cast(float, o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
DEV u64 order_key(float x, int col) { return (u64)order_bits(x) << 32 | (uint32_t)~col; }

template <int J>
DEV u64 lane_xor64(u64 x) {
  return (u64)lane_xor<J>((uint32_t)(x >> 32)) << 32 | lane_xor<J>((uint32_t)x);
}
// of the lanes l and l ^ J the one without bit H keeps the larger key
template <int J, int H>
DEV u64 exchange(u64 key) {
  const u64 o = lane_xor64<J>(key);
  return (key > o) == ((threadIdx.x & H) == 0) ? key : o;
}
// sorted in falling order: blocks of K lanes from two sorted ones, mirrored, then halved
template <int J>
DEV u64 halve(u64 key) {
  key = exchange<J, J>(key);
  if constexpr (J > 1) key = halve<J / 2>(key);
  return key;
}
DEV u64 sort16(u64 key) {
  key = exchange<1, 1>(key);
  key = halve<1>(exchange<3, 2>(key));
  key = halve<2>(exchange<7, 4>(key));
  return halve<4>(exchange<15, 8>(key));
}
// n keys in the first lanes, 0 in the others
DEV u64 sort_keys(u64 key, int n) {
  key = sort16(key);
  if (n <= 16) return key;
  key = halve<8>(exchange<31, 16>(key));
  return halve<16>(exchange<63, 32>(key));
}
// the largest of two sorted lists, sorted: as many as k of them
DEV u64 merge_keys(u64 a, u64 b, int k) {
  if (k <= 16) {
    const u64 r = lane_xor64<15>(b);
    return halve<8>(a > r ? a : r);
  }
  const u64 r = lane_xor64<63>(b);
  return halve<32>(a > r ? a : r);
}

// the largest value, to 2^-7 of it, that at least n lanes' order bits reach
DEV uint32_t lanes_reach(uint32_t o, int n) {
  uint32_t t = 0;
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t up = t | 1u << bit;
    if (__popcll(__ballot(o >= up)) >= n) t = up;
  }
  return t;
}

constexpr int top_buffer(int n) { return 64 + 64 * n; }  // keys of a wave's buffer, vectors of n logits

// The threshold that a logit has to be above to be buffered comes from the lanes' largest logits so
// far: of each wave the ceil(k / waves)-th largest of its lanes' (to 2^-7 of it, by bisection), and
// of the waves the least. k lanes of the row at least have reached it, so it bounds the row's k-th
// logit from below; it is not far below, as the top logits are mostly in different lanes. `share`
// holds each wave's bound, which only rises: an older one is valid too. Taken anew whenever the
// groups seen have doubled (from four on), it lets about as many logits through between two of these
// times, some 16 of a wave for 64 alternatives on 8 waves.
//
// A wave whose list has filled up has its own k-th as a second threshold: columns rise from one
// vector of a wave to the next, so a logit that equals it ranks behind it. One that equals another
// wave's bound may rank before, so that one counts from the next value below it.
template <int NW>
struct Top {
  u64 list;    // this lane's key of the sorted list
  float thr;   // only logits above it can be among the first k
  int cnt, k;  // buffered keys, k (both the same in all lanes)
  int groups;  // seen
  u64* buf;
  uint32_t* share;  // [NW] order bits

  __device__ __forceinline__ void start(int top_k, u64* b, uint32_t* sh) {
    list = 0;
    thr = -INFINITY;
    cnt = groups = 0;
    k = top_k;
    buf = b;
    share = sh;
  }
  __device__ __forceinline__ void fence() const {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  // the next value below one (no logit has the bits of -0 here, which a comparison takes for +0)
  static __device__ __forceinline__ float below(uint32_t bits) {
    return bits > 0x00800000u ? order_value(bits - (bits == 0x80000000u ? 2 : 1)) : -INFINITY;
  }

  // merges the last n <= 64 keys of the buffer
  __device__ __forceinline__ void flush(int n) {
    fence();
    const int l = lane_id();
    cnt -= n;
    const u64 key = l < n ? buf[cnt + l] : 0ull;
    fence();
    list = merge_keys(list, sort_keys(key, n), k);
  }
  // appends the keys of the lanes with `in`; whether there is one
  __device__ __forceinline__ bool push(u64 key, bool in) {
    const u64 mask = __ballot(in);
    if (!mask) return false;
    if (in)
      buf[cnt + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = key;
    cnt += __popcll(mask);
    return true;
  }
  // most: this lane's largest logit so far
  __device__ __forceinline__ void publish(float most) {
    const uint32_t t = lanes_reach(order_bits(most), (k + NW - 1) / NW);
    if (lane_id() == 0) __hip_atomic_store(share + (threadIdx.x >> 6), t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  }
  __device__ __forceinline__ void shared_threshold() {
    uint32_t least = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < NW; ++i)
      least = min(least, __hip_atomic_load(share + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
    thr = fmaxf(thr, below(least));
  }

  // The first group's bounds are published before a barrier that every wave has to pass before it adds.
  template <int N>
  __device__ __forceinline__ void push(const float (&x)[N], int col) {
#pragma unroll
    for (int j = 0; j < N; ++j) push(order_key(x[j], col + j), x[j] > thr);
  }
  __device__ __forceinline__ void drain() {
    if (cnt < 64) return;
    do flush(64);
    while (cnt >= 64);
    const uint32_t kth = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(list >> 32), k - 1);
    if (kth) thr = fmaxf(thr, order_value(kth));
  }
  // a group (top: its largest logit), vector by vector: the buffer takes one more where it holds less than
  // 64 keys
  template <int U, int N>
  __device__ __forceinline__ void add(const Group<U, N>& g, float top, float most) {
    const int seen = ++groups;
    if (seen > 2 && (seen & (seen - 1)) == 0) publish(most);
    if (!__any(top > thr)) return;
    shared_threshold();
    if (!__any(top > thr)) return;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u >= g.n) break;
      push(g.x[u], g.col + u * g.step);
      drain();
    }
  }

  // joins the waves' lists into the first wave's; lists: [NW / 2][64]
  __device__ __forceinline__ void join(u64* lists) {
    if (cnt > 0) flush(cnt);
    __syncthreads();  // (the lists may lie in the buffers)
    const int wave = threadIdx.x >> 6, l = lane_id();
#pragma unroll
    for (int half = NW / 2; half > 0; half /= 2) {
      if (wave >= half && wave < 2 * half) lists[(wave - half) * 64 + l] = list;
      __syncthreads();
      if (wave < half) list = merge_keys(list, lists[wave * 64 + l], k);
      __syncthreads();
    }
  }
};

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
// statistics and lists for k_scores_join. U: loads of a lane in flight.
template <class T, bool TOP, int NT, int U>
__global__ __launch_bounds__(NT) void k_scores(ScoreArgs p) {
  constexpr int NW = NT / 64, B = TOP ? top_buffer(kVec<T>) : 1;
  __shared__ Acc red[NW];
  __shared__ u64 buf[NW * B];
  __shared__ uint32_t share[NW];
  const size_t row = blockIdx.x / p.split.n;
  const int part = (int)(blockIdx.x % p.split.n);
  const T* z = (const T*)p.z + row * p.ld;
  const int v0 = part * p.split.cols, v1 = min(p.vocab, v0 + p.split.cols);
  Top<NW> t;
  t.start(p.top_k, buf + (threadIdx.x >> 6) * B, share);
  Sums<true, ONE> sums;
  sums.start(p.c, p.lift);
  bool begun = false;
  scan<T, NT, U, true>(z, v0, v1, [&](const auto& g) {
    const float top = sums.template add<2>(g);
    if constexpr (TOP) {
      if (!begun) {  // (of every thread: each has a first group)
        t.publish(sums.most);
        __syncthreads();
        begun = true;
      }
      t.add(g, top, sums.most);
    }
  });
  Acc a = sums.template join<NT>(red);
  if (!served<false>(a)) {
    a = acc_empty();
    scan<T, NT, 1, false>(z, v0, v1, [&](const auto& g) { acc_add<true, false>(a, g, p.c, 0.f); });
    __syncthreads();
    acc_block<NT, true, false>(a, p.c, 0.f, red);
  }
  if constexpr (TOP) t.join(buf);
  if (threadIdx.x >= 64) return;
  if (p.split.n == 1) {
    write_scores(p, row, a, target_logit<T>(p, z, row), t.list);
  } else {
    if (lane_id() == 0) p.split.stats[blockIdx.x] = make_float4(a.m, a.s, a.w, 0.f);
    if (TOP && lane_id() < p.top_k) p.split.keys[(size_t)blockIdx.x * p.top_k + lane_id()] = t.list;
  }
}

// One workgroup per row. Where there are at least k parts, their largest logits (the heads of their
// lists) bound the row's k-th from below: each list gives the keys of its beginning that reach it, one
// of each list at a time, to one wave's buffer. Else the waves merge whole lists, and then theirs.
template <class T>
__global__ __launch_bounds__(256) void k_scores_join(ScoreArgs p) {
  __shared__ u64 keys[kLogitParts * 64], buf[128];
  const size_t row = blockIdx.x;
  const int l = lane_id(), n = p.split.n, k = p.top_k;
  for (int i = threadIdx.x; i < n * k; i += 256) keys[i] = p.split.keys[row * n * k + i];
  if (k) __syncthreads();
  Top<4> t;
  t.start(k, buf, nullptr);
  if (n < k) {
    for (int i = threadIdx.x >> 6; i < n; i += 4) t.list = merge_keys(t.list, l < k ? keys[i * k + l] : 0ull, k);
    t.join(buf);
  }
  if (threadIdx.x >= 64) return;
  const float zt = target_logit<T>(p, (const T*)p.z + row * p.ld, row);
  const Acc a = join_parts<true, false>(p.split, row, p.c, 0.f);
  if (k && n >= k) {
    const uint32_t bound = lanes_reach(l < n ? (uint32_t)(keys[l * k] >> 32) : 0u, k);
    for (int j = 0; j < k; ++j) {
      const u64 key = l < n ? keys[l * k + j] : 0ull;
      if (!t.push(key, key && (uint32_t)(key >> 32) >= bound)) break;
      if (t.cnt >= 64) t.flush(64);
    }
    t.flush(t.cnt);
  }
  write_scores(p, row, a, zt, t.list);
}

// ------------------------------------------------------------------ gradient
// d logp_t / dz = (1[t] - q) / tau and dH / dz = -q (ln q + H) / tau, weighted by the gradients of
// the two; the target's column is written again with its 1.
//
// ln q = z / tau - lse, and an fp32 lse is off by 2^-24 of itself: by 2^-18 at kWideLse, by all of ln s
// for a row of finite mask values such as -1e9. A row whose lse is larger is summed again, and written, by
// its first part alone (the output may be the input, which its other parts must not write meanwhile):
// ln q = (z - m) / tau - ln s then (1024 x 151936 bf16 227 us where all rows are such and 111 else; 8 x
// 151936 fp32 36 and 3.3; with 4 loads in flight 191 and 32, but the registers cost the others 3 %).
constexpr float kWideLse = 128.f;

template <class T, class G, int NT>
__global__ __launch_bounds__(NT) void k_scores_grad(ScoreGradArgs p) {
  __shared__ Acc red[NT / 64];
  const size_t row = blockIdx.x / p.split.n;
  const int part = (int)(blockIdx.x % p.split.n);
  const T* z = (const T*)p.z + row * p.ld;
  G* dz = (G*)p.dz + row * p.ldd;
  const float lse = p.lse[row];
  const bool wide = lse != -INFINITY && fabsf(lse) > kWideLse;
  if (wide && part > 0) return;
  const int v0 = part * p.split.cols, v1 = wide ? p.vocab : min(p.vocab, v0 + p.split.cols);
  const int t = p.targets && p.d_logp ? p.targets[row] : -1;
  Acc a = acc_empty();
  if (wide) {
    scan<T, NT, 2, false>(z, 0, p.vocab, [&](const auto& g) { acc_add<false, false>(a, g, p.c, 0.f); });
    acc_block<NT, false, false>(a, p.c, 0.f, red);
  }
  if (wide ? a.s == 0.f : lse == -INFINITY) {
    zero_row<G, NT>(dz, v0, v1);
    return;
  }
  float A = t < 0 ? 0.f : p.d_logp[row] * p.inv_tau;
  if (t >= p.vocab) A = NAN;
  const float B = p.d_entropy ? p.d_entropy[row] * p.inv_tau : 0.f;
  const float AB = A + B * (p.d_entropy ? p.entropy[row] : 0.f);
  const bool here = t >= v0 && t < v1;
  const float zt = here && threadIdx.x == 0 ? cvt(z[t]) : 0.f;
  // (q = 0 at logits of -inf, and 0 times -inf is not; the logarithm meets its weight before B, whose
  // product with it alone may be beyond fp32)
  auto grad = [&](float lq) {
    const float q = exp2_fast(lq * kLog2e);
    return -fmaf(B, q * fmaxf(lq, -1e30f), q * AB);
  };
  auto write = [&](auto&& lq) {
    if (here) __syncthreads();  // zt is read before any thread writes (the output may be the input)
    map_row<T, G, NT, 4, true>(z, dz, v0, v1, [&](float x) { return grad(lq(x)); });
    if (!here) return;
    stores_done();
    if (threadIdx.x == 0) dz[t] = to_out<G>(grad(lq(zt)) + A);
  };
  if (wide) {
    const float log_s = logf(a.s);
    write([&](float x) { return (x - a.m) * p.inv_tau - log_s; });
  } else {
    write([&](float x) { return x * p.inv_tau - lse; });
  }
}

}  // namespace

// Parts of a row: enough workgroups for the chip where there are few long rows, of no fewer than 4096
// columns each. The launch that joins them costs more than a workgroup's pass over a short row (call of
// 8 rows of 50257 fp32 logits 15.0 us by parts and 10.7 whole, with 20 alternatives 15.3 both; of 100000
// 15.3 and 12.9, 15.2 and 21.7), and so do the parts of many rows together (151936 fp32 logits: 128 rows
// 16 us by parts and 19 whole, 192 rows 23 and 21; with 20 alternatives 23 and 27, 29 and 29; bf16 128 rows 13
// and 14, 192 17 and 14). Of 70000 .. 262144 fp32 and bf16 logits the two meet at 110 to 160 rows, with
// alternatives at 110 to 260, and 160 costs no more than a fifth at any of them.
LogitSplit logit_split(int rows, int vocab) {
  LogitSplit s{};
  const int want = rows >= 160 || vocab <= 65536 ? 1 : std::min(kLogitParts, (1024 + rows - 1) / std::max(rows, 1));
  const int most = (vocab + 4095) / 4096;
  const int n = std::max(1, std::min(want, most));
  s.cols = ((vocab + n - 1) / n + 2047) / 2048 * 2048;
  s.n = (vocab + s.cols - 1) / s.cols;
  return s;
}

hipError_t launch_scores(ScoreArgs a, int dtype, hipStream_t st) {
  const unsigned grid = (unsigned)((size_t)a.rows * a.split.n);
  return by_type(dtype, [&](auto* tp) {
    using T = std::remove_pointer_t<decltype(tp)>;
    const double bytes = (double)a.rows * a.vocab * sizeof(T);
    auto run = [&](auto top, auto nt, auto loads) {
      constexpr int NT = decltype(nt)::value, U = decltype(loads)::value;
      MEBP_TIMED(st, a.top_k ? "token_scores_top" : "token_scores", 0.0, bytes,
                 hipLaunchKernelGGL((k_scores<T, decltype(top)::value, NT, U>), dim3(grid), dim3(NT), 0, st, a));
    };
    const bool wide = a.split.n == 1 && a.vocab > 16384;
    // 4 loads in flight read 151936 fp32 logits of 256 rows in 26 us, 2 in 31. Beside the alternatives'
    // work 2 are faster where several workgroups share a compute unit (64 of 2048 x 262144 bf16 199 us,
    // with 4 213; 5 of 800 x 50257 fp16 30 and 34, of 333 18 and 20), 4 where a row has one to itself (20 of
    // 256 x 151936 fp32 37 us with 2, 32 with 4; 262144 57 and 47)
    if (!a.top_k)
      wide ? run(std::false_type(), IC<512>(), IC<4>()) : run(std::false_type(), IC<256>(), IC<4>());
    else if (wide && a.rows <= 256)
      run(std::true_type(), IC<512>(), IC<4>());
    else
      wide ? run(std::true_type(), IC<512>(), IC<2>()) : run(std::true_type(), IC<256>(), IC<2>());
    if (a.split.n > 1)
      MEBP_TIMED(st, "token_scores_join", 0.0, (double)grid * (16 + 8 * a.top_k),
                 hipLaunchKernelGGL((k_scores_join<T>), dim3(a.rows), dim3(256), 0, st, a));
    return hipGetLastError();
  });
}

// The gradient goes by parts of 8192 columns: 4 loads of each lane of 256 in flight in 16 bits, and
// many small workgroups leave no part of the chip waiting (1024 x 151936 bf16 110 us, 5.6 TB/s; a
// workgroup per row 125 .. 130 us); by smaller ones where that makes fewer than four workgroups for
// each compute unit.
hipError_t launch_scores_grad(ScoreGradArgs a, int dtype, int gtype, hipStream_t st) {
  a.split.cols = 8192;
  while (a.split.cols > 2048 && (size_t)a.rows * ((a.vocab + a.split.cols - 1) / a.split.cols) < 1024) a.split.cols /= 2;
  // (a grid of 256-lane workgroups holds fewer than 2^24 of them)
  while ((size_t)a.rows * ((a.vocab + a.split.cols - 1) / a.split.cols) > (1u << 23)) a.split.cols *= 2;
  a.split.n = (a.vocab + a.split.cols - 1) / a.split.cols;
  const unsigned grid = (unsigned)((size_t)a.rows * a.split.n);
  const double bytes = (double)a.rows * a.vocab * (type_bytes(dtype) + type_bytes(gtype));
  return by_type(dtype, [&](auto* tp) {
    return by_type(gtype, [&](auto* gp) {
      using T = std::remove_pointer_t<decltype(tp)>;
      using G = std::remove_pointer_t<decltype(gp)>;
      MEBP_TIMED(st, a.z == a.dz ? "token_scores_grad_inplace" : "token_scores_grad", 0.0, bytes,
                 hipLaunchKernelGGL((k_scores_grad<T, G, 256>), dim3(grid), dim3(256), 0, st, a));
      return hipGetLastError();
    });
  });
}

}  // namespace mebp
