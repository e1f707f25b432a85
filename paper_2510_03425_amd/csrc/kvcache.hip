// Append to the paged 8-bit cache, with the rotation of keys and queries on the way, and its read back.
//
// A block of 16 tokens of one kv head has one fp32 scale for its keys and one for its values:
//   scale = max(|scale before|, fp32(max |x| / 127)),  code = rint(x / scale),
// "before" being 0 where the block's first token is new. A scale that changes has the block's earlier codes
// rounded again, rint(code before / after). Codes are the nearest ones of the definition in 64 bits (a
// rotated key rounded to 32 bits first would land on the other side of a border now and then, and a code
// is a whole step), so keys are turned, and their largest found, in 64 bits.
#include <math.h>

#include "device_common.h"
#include "heads.h"
#include "kv_device.h"

#define DEVM __device__ __forceinline__

namespace mebp {
namespace {

DEV double wave_max_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmax(v, __shfl_xor(v, o, 64));
  return v;
}

template <class T, int N>
DEV void load_n(const T* p, float* v, bool vec) {
  if (vec) {
    if constexpr (N % 8 == 0) {
#pragma unroll
      for (int i = 0; i < N; i += 8) load8(p + i, v + i);
      return;
    } else {
      typedef T run __attribute__((ext_vector_type(N)));
      const run r = *(const run*)p;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = (float)r[i];
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (float)p[i];
}
template <class T, int N>
DEV void store_n(T* p, const float* v, bool vec) {
  if (vec) {
    if constexpr (N % 8 == 0) {
#pragma unroll
      for (int i = 0; i < N; i += 8) store8(p + i, v + i);
      return;
    } else {
      typedef T run __attribute__((ext_vector_type(N)));
      run r;
#pragma unroll
      for (int i = 0; i < N; ++i) r[i] = (T)v[i];
      *(run*)p = r;
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = (T)v[i];
}

// the block's scale after max |x| = amax joined one of scale `old`; an amax that is not finite: NaN
DEV float raised(float old, double amax) {
  const float want = amax < INFINITY ? (float)(amax / 127.0) : NAN;
  return want != want || old != old ? NAN : fmaxf(old, want);
}
// The code of x at a scale by its definition: the quotient's nearest whole number, ties to even.
DEV int code_of(double x, double scale) { return (int)fmin(fmax(rint(x / scale), -127.0), 127.0); }
// The same from a quotient in 32 bits, x times a reciprocal: two roundings, within 127 2^-23 of the real one, so that
// a result further than 2^-15 from the border of two codes is the real one's; `near` is set by the others (one wave
// in 16 for heads of 256), which go by the definition, all of a thread's at once. (With a branch to the division at each
// element, 8 x 2048 tokens of 4 heads of 256 took 64 us instead of 49.) Adding 1.5 2^23 rounds to nearest even, and
// leaves the code in the low byte.
DEV uint32_t quick_code(float q, bool& near) {
  const float s = q + 12582912.f;
  near |= !(fabsf(q - (s - 12582912.f)) < 0.5f - 3.06e-5f);
  return __builtin_bit_cast(uint32_t, s);
}
DEV uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
// 4 x 4 bytes, transposed
DEV void transpose4(uint32_t (&x)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), b = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u),
                 c = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u), d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
  x[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  x[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  x[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  x[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// Which elements of a head a thread holds: E pairs c E + i of the head's D / 2, those that turn first. Pair P
// is (P, P + rot / 2), or (2 P, 2 P + 1) where they are interleaved; behind them the copied elements as pairs
// D / 2 apart (or neighbours). Runs of E (2 E) elements unless rot / 2 is no multiple of E.
template <int D>
struct Pairs {
  static constexpr int E = D / 32;
  int half, c;  // pairs that turn
  bool inter;
  DEVM Pairs(const RopeView* r, int c_) : half(r ? r->rot >> 1 : 0), c(c_), inter(r && r->interleaved) {}
  DEVM bool turns(int i) const { return c * E + i < half; }
  DEVM int a(int i) const {
    const int p = c * E + i;
    return inter ? 2 * p : p < half ? p : p + half;
  }
  DEVM int b(int i) const {
    const int p = c * E + i;
    return inter ? 2 * p + 1 : p < half ? p + half : p + D / 2;
  }
  DEVM bool runs() const { return inter || half % E == 0; }
  // the elements as they are in memory, and as numbers
  template <class T>
  struct Raw {
    typedef T run __attribute__((ext_vector_type(E)));
    run a, b;
  };
  template <class T>
  DEVM Raw<T> load(const T* p, bool vec) const {
    typedef typename Raw<T>::run run;
    Raw<T> r;
    if (vec && runs()) {
      // (of interleaved pairs the two runs follow one another, and are told apart below)
      r.a = *(const run*)(p + a(0));
      r.b = *(const run*)(p + (inter ? a(0) + E : b(0)));
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int j = inter ? a(0) + i : a(i), k = inter ? a(0) + E + i : b(i);
        r.a[i] = p[j];
        r.b[i] = p[k];
      }
    }
    return r;
  }
  template <class T>
  DEVM void numbers(const Raw<T>& r, float (&xa)[E], float (&xb)[E]) const {
    if (inter) {
      float x[2 * E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        x[i] = (float)r.a[i];
        x[E + i] = (float)r.b[i];
      }
#pragma unroll
      for (int i = 0; i < E; ++i) {
        xa[i] = x[2 * i];
        xb[i] = x[2 * i + 1];
      }
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        xa[i] = (float)r.a[i];
        xb[i] = (float)r.b[i];
      }
    }
  }
  template <class T>
  DEVM void store(T* p, const float (&xa)[E], const float (&xb)[E], bool vec) const {
    if (vec && runs()) {
      if (inter) {
        float x[2 * E];
#pragma unroll
        for (int i = 0; i < E; ++i) { x[2 * i] = xa[i]; x[2 * i + 1] = xb[i]; }
        store_n<T, 2 * E>(p + a(0), x, true);
      } else {
        store_n<T, E>(p + a(0), xa, true);
        store_n<T, E>(p + b(0), xb, true);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) { p[a(i)] = (T)xa[i]; p[b(i)] = (T)xb[i]; }
  }
};

// A block's scale from the largest of the workgroup's x, and x's codes as bytes a[..], b[..]: of the block's new tokens
// (`fresh`), or of earlier ones rounded again where the scale has changed. X: double for keys that are turned.
template <class X, int E>
struct Codes {
  float scale;
  uint8_t a[E], b[E];
  bool write;  // whether this thread's codes are new
  // code_at(i, b): an earlier code
  template <class At>
  DEVM Codes(const X (&xa)[E], const X (&xb)[E], bool fresh, bool earlier, float old, double* red, At&& code_at) {
    double m;
    if constexpr (sizeof(X) == 8) {
      double none = 0.0;  // (NaN where one is not finite, which a maximum may lose)
      m = 0.0;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        m = fmax(m, fabs(xa[i]));
        m = fmax(m, fabs(xb[i]));
        none = fma(xa[i], 0.0, none);
        none = fma(xb[i], 0.0, none);
      }
      if (none != none) m = INFINITY;
    } else {
      // (bits of magnitudes are ordered as the magnitudes, infinities and NaN above all)
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        most = max(most, __builtin_bit_cast(uint32_t, xa[i]) & 0x7fffffffu);
        most = max(most, __builtin_bit_cast(uint32_t, xb[i]) & 0x7fffffffu);
      }
      m = most < 0x7f800000u ? (double)__builtin_bit_cast(float, most) : (double)INFINITY;
    }
    m = wave_max_f64(fresh ? m : 0.0);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    m = fmax(fmax(red[0], red[1]), fmax(red[2], red[3]));
    scale = raised(fabsf(old), m);
    write = fresh || (earlier && scale != old);
    // (a scale too small for its reciprocal, or none: every code by its definition)
    bool near = fresh && !(scale > 1e-37f);
    const X inv = near ? (X)0 : (X)1 / (X)scale;
    uint32_t ca[E], cb[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      ca[i] = quick_code((float)(xa[i] * inv), near);
      cb[i] = quick_code((float)(xb[i] * inv), near);
    }
    if (near && fresh) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        ca[i] = scale > 0.f ? code_of(xa[i], scale) : 0;
        cb[i] = scale > 0.f ? code_of(xb[i], scale) : 0;
      }
    }
    if (!fresh) {
      const double ratio = write && scale > 0.f ? (double)old / (double)scale : 0.0;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        ca[i] = earlier ? code_at(i, false) : 0;
        cb[i] = earlier ? code_at(i, true) : 0;
        if (write) {
          ca[i] = (int)rint((double)(int)ca[i] * ratio);
          cb[i] = (int)rint((double)(int)cb[i] * ratio);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      a[i] = (uint8_t)ca[i];
      b[i] = (uint8_t)cb[i];
    }
  }
};

// One workgroup: a 16-token block of one kv head (its keys or its values), or the queries of those tokens and Q
// heads. Thread: token tid / 16, 1/16 of the head. Bytes bound it where there are many tokens, and the way from the
// sequence's numbers to the row and the page, three loads after one another, where there are few. 8 x 2048 tokens,
// 4 heads of 256 and 8 of queries: 69 us, 3.4 TB/s; 57 with its inputs in the cache behind the L2s. (Four blocks
// after one another in a workgroup, the next one's numbers on their way: 77 instead of 57.)
template <class T, int D, int Q>
__global__ __launch_bounds__(256) void k_kv_append(KvAppendArgs a, bool vk, bool vv, bool vq) {
  constexpr int E = D / 32;
  __shared__ double red[4];
  __shared__ __attribute__((aligned(16))) uint8_t turned[(D + 4) * 16];
  const int roles = 2 * a.c.heads + a.q_groups;
  const int role = blockIdx.x % roles, nb = blockIdx.x / roles, s = blockIdx.y;
  if (s == a.b.seqs) {
    // (one more than the sequences where rows that none has are to be cleared: around all of them, and behind the
    // max_new of one)
    auto clear = [&](int64_t r, int64_t end, int step) {
      for (; r < end; r += step)
        for (int e = threadIdx.x; e < a.rest_cols / 8; e += 256) ((uint4*)(a.rest + r * a.rest_cols))[e] = make_uint4(0, 0, 0, 0);
    };
    clear(blockIdx.x, min(a.b.start[0], a.b.rows), gridDim.x);
    clear(max(a.b.start[s], 0) + (int64_t)blockIdx.x, a.b.rows, gridDim.x);
    for (int i = blockIdx.x; i < a.b.seqs; i += gridDim.x) {
      const KvSeq q = kv_seq(a.b, i);
      clear(q.row + q.n, min(a.b.start[i + 1], a.b.rows), 1);
    }
    return;
  }
  const KvSeq q = kv_seq(a.b, s);
  const int end = q.past + q.n, blk = (q.past >> 4) + nb;
  if (q.n == 0 || blk * 16 >= end) return;
  const int tid = threadIdx.x, t = tid >> 4, c = tid & 15;
  const bool turn = a.rope.table && (role < a.c.heads || role >= 2 * a.c.heads), key = role < a.c.heads;
  const Pairs<D> at(turn ? &a.rope : nullptr, c);
  const int pos = blk * 16 + t, t_lo = max(q.past - blk * 16, 0);
  const bool fresh = pos >= q.past && pos < end;
  const int64_t row = (int64_t)q.row + (pos - q.past);
  auto angles = [&](float2 (&cs)[E]) {
    const bool ok = pos < a.rope.n_pos;
    const float2* tab = a.rope.table + (int64_t)(ok ? pos : 0) * at.half;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (at.turns(i)) cs[i] = ok ? tab[c * E + i] : make_float2(NAN, NAN);
  };
  if (role >= 2 * a.c.heads) {
    const int h0 = (role - 2 * a.c.heads) * Q, hn = min(Q, a.q_heads - h0);
    if (!fresh) return;
    const T* p = (const T*)a.q.p + row * a.q.ld + h0 * a.q.hld;
    T* o = (T*)a.q_out.p + row * a.q_out.ld + h0 * a.q_out.hld;
    typename Pairs<D>::template Raw<T> raw[Q];
    float2 cs[E];
#pragma unroll
    for (int h = 0; h < Q; ++h)
      if (h < hn) raw[h] = at.load(p + h * a.q.hld, vq);
    angles(cs);
#pragma unroll
    for (int h = 0; h < Q; ++h) {
      if (h >= hn) break;
      float xa[E], xb[E];
      at.numbers(raw[h], xa, xb);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float u = xa[i], w = xb[i];
        if (at.turns(i)) {
          xa[i] = u * cs[i].x - w * cs[i].y;
          xb[i] = w * cs[i].x + u * cs[i].y;
        }
      }
      at.store(o + h * a.q_out.hld, xa, xb, vq);
    }
    return;
  }
  const int h = key ? role : role - a.c.heads;
  const HeadsView& v = key ? a.k : a.v;
  typename Pairs<D>::template Raw<T> raw{};
  float2 cs[E];
  if (fresh) {
    raw = at.load((const T*)v.p + row * v.ld + h * v.hld, key ? vk : vv);
    if (turn) angles(cs);
  }
  const int page = kv_page(a.c, a.b, s, blk);
  if (page < 0) return;
  float fa[E], fb[E];
  at.numbers(raw, fa, fb);
  double xa[E], xb[E];
  if (key) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const double u = fa[i], w = fb[i];
      xa[i] = u;
      xb[i] = w;
      if (at.turns(i)) {
        const double co = cs[i].x, si = cs[i].y;
        xa[i] = u * co - w * si;
        xb[i] = w * co + u * si;
      }
    }
  }
  const uint64_t block = kv_block(a.c, page, h, blk);
  int8_t* out = a.c.codes + block * (2 * 16 * D) + (key ? 0 : 16 * D);
  float* scale_at = a.c.scales + block * 2 + (key ? 0 : 1);
  const float old = t_lo > 0 ? *scale_at : 0.f;
  float scale;
  if (key) {
    int8_t* o = out + t * D;
    const Codes<double, E> x(xa, xb, fresh, t < t_lo, old, red, [&](int i, bool b) { return (int)o[b ? at.b(i) : at.a(i)]; });
    scale = x.scale;
    if (x.write) {
      if (at.runs() && !at.inter) {
        __builtin_memcpy(__builtin_assume_aligned(o + at.a(0), E), x.a, E);
        __builtin_memcpy(__builtin_assume_aligned(o + at.b(0), E), x.b, E);
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          o[at.a(i)] = (int8_t)x.a[i];
          o[at.b(i)] = (int8_t)x.b[i];
        }
      }
    }
  } else {
    const Codes<float, E> x(fa, fb, fresh, t < t_lo, old, red, [&](int i, bool b) { return (int)out[(b ? at.b(i) : at.a(i)) * 16 + t]; });
    scale = x.scale;
    // Values lie transposed, [D][16]: through LDS as [16][D] (a word more a row), four tokens of four dims at a
    // time. (Codes of tokens that are still to come are 0.)
    __builtin_memcpy(__builtin_assume_aligned(turned + t * (D + 4) + at.a(0), E < 4 ? E : 4), x.a, E);
    __builtin_memcpy(__builtin_assume_aligned(turned + t * (D + 4) + at.b(0), E < 4 ? E : 4), x.b, E);
    __syncthreads();
    if (tid < D) {
      const int d4 = tid >> 2, t4 = tid & 3;
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = *(const uint32_t*)(turned + (t4 * 4 + i) * (D + 4) + d4 * 4);
      transpose4(w);
#pragma unroll
      for (int i = 0; i < 4; ++i) *(uint32_t*)(out + (d4 * 4 + i) * 16 + t4 * 4) = w[i];
    }
  }
  if (tid == 0 && (t_lo == 0 || scale != old)) *scale_at = scale;
}

// One workgroup: the tokens of one block that the call has, of one head. A thread of keys takes four dims at a
// time, one of values all its tokens of a dim, so that a wave's stores are whole lines. Bytes bound it: 16384 tokens, 4
// heads of 256, to fp32: 27 us, 6.3 TB/s.
template <class T, int D>
__global__ __launch_bounds__(256) void k_kv_read(KvReadArgs a, bool vk) {
  const int h = blockIdx.x % a.c.heads, nb = blockIdx.x / a.c.heads, s = blockIdx.y;
  const KvSeq q = kv_seq(a.b, s);
  const int blk = (q.past >> 4) + nb, base = blk << 4;
  const int t_lo = max(q.past - base, 0), t_hi = min(q.past + q.n - base, 16);
  if (q.n == 0 || t_hi <= t_lo) return;
  const int page = kv_page(a.c, a.b, s, blk);
  const uint64_t at = kv_block(a.c, max(page, 0), h, blk);
  const int8_t* in = a.c.codes + at * (2 * 16 * D);
  float2 sc = ((const float2*)a.c.scales)[at];
  constexpr int VT = D / 16, KI = D / 64;  // tokens of a thread of values, and its four dims of keys
  const int e = threadIdx.x % D, t0 = threadIdx.x / D * VT;
  int kc[KI];
  int8_t vc[VT];
#pragma unroll
  for (int i = 0; i < KI; ++i) kc[i] = ((const int*)in)[threadIdx.x + 256 * i];
  __builtin_memcpy(vc, __builtin_assume_aligned(in + 16 * D + e * 16 + t0, VT), VT);
  if (page < 0) sc = make_float2(NAN, NAN);
  const int64_t row = (int64_t)q.row + base - q.past;
  if (a.k.p) {
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      const int t = (threadIdx.x + 256 * i) / (D / 4), d = (threadIdx.x + 256 * i) % (D / 4) * 4;
      if (t < t_lo || t >= t_hi) continue;
      float x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = (float)(int8_t)(kc[i] >> 8 * j) * sc.x;
      store_n<T, 4>((T*)a.k.p + (row + t) * a.k.ld + h * a.k.hld + d, x, vk);
    }
  }
  if (a.v.p) {
#pragma unroll
    for (int i = 0; i < VT; ++i) {
      const int t = t0 + i;
      if (t >= t_lo && t < t_hi) ((T*)a.v.p)[(row + t) * a.v.ld + h * a.v.hld + e] = (T)((float)vc[i] * sc.y);
    }
  }
}

template <class T>
hipError_t kv_append(KvAppendArgs a, hipStream_t st) {
  // vectors of the E elements that a thread takes: 16 bytes' alignment covers every E
  const bool vk = vectors(a.k, sizeof(T)), vv = vectors(a.v, sizeof(T)),
             vq = a.q.p && vectors(a.q, sizeof(T)) && vectors(a.q_out, sizeof(T));
  constexpr int Q = 4;
  a.q_groups = a.q.p ? (a.q_heads + Q - 1) / Q : 0;
  const dim3 grid((unsigned)a.nblk * (2 * a.c.heads + a.q_groups), (unsigned)a.b.seqs + (a.rest ? 1 : 0));
  const double bytes = (double)a.b.rows * a.c.dim * (2.0 * a.c.heads * (sizeof(T) + 1) + (a.q.p ? 2.0 * a.q_heads * sizeof(T) : 0.0));
  const char* name = a.q.p && a.q.p == a.q_out.p ? "kv_append_inplace" : "kv_append";
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    MEBP_TIMED(st, name, 0.0, bytes, hipLaunchKernelGGL((k_kv_append<T, D, Q>), grid, dim3(256), 0, st, a, vk, vv, vq));
    return hipGetLastError();
  };
  return a.c.dim == 64 ? go(IC<64>{}) : a.c.dim == 128 ? go(IC<128>{}) : go(IC<256>{});
}

template <class T>
hipError_t kv_read(const KvReadArgs& a, hipStream_t st) {
  const bool vk = vectors(a.k, sizeof(T));
  const dim3 grid((unsigned)a.nblk * a.c.heads, (unsigned)a.b.seqs);
  const double bytes = (double)a.b.rows * a.c.dim * a.c.heads * 2.0 * (sizeof(T) + 1);
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    MEBP_TIMED(st, "kv_read", 0.0, bytes, hipLaunchKernelGGL((k_kv_read<T, D>), grid, dim3(256), 0, st, a, vk));
    return hipGetLastError();
  };
  return a.c.dim == 64 ? go(IC<64>{}) : a.c.dim == 128 ? go(IC<128>{}) : go(IC<256>{});
}
}  // namespace

hipError_t launch_kv_append(KvAppendArgs a, int dtype, hipStream_t st) {
  if (dtype == LOGIT_F32) return kv_append<float>(a, st);
  return dtype == LOGIT_F16 ? kv_append<f16>(a, st) : kv_append<bf16>(a, st);
}

hipError_t launch_kv_read(const KvReadArgs& a, int dtype, hipStream_t st) {
  if (dtype == LOGIT_F32) return kv_read<float>(a, st);
  return dtype == LOGIT_F16 ? kv_read<f16>(a, st) : kv_read<bf16>(a, st);
}

}  // namespace mebp
