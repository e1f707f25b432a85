// Append to the paged 8-bit cache, with the rotation of keys and queries on the way, and its read back.
//
// A block of 16 tokens of one kv head has one fp32 scale for its keys and one for its values:
//   scale = max(scale before, fp32(max |x| / 127)),  code = rint(x / scale),
// "before" being 0 where the block's first token is new. A scale that rises has the block's earlier codes
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

DEV unsigned long long wave_max_bits(unsigned long long v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const unsigned long long w = __shfl_xor(v, o, 64);
    v = w > v ? w : v;
  }
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

// the block's scale after max |x| = amax joined one of scale `old`; NaN or infinite amax: NaN
DEV float raised(float old, double amax) {
  const float want = amax < INFINITY ? (float)(amax / 127.0) : NAN;
  return want != want || old != old ? NAN : fmaxf(old, want);
}
DEV int code_of(double x, double scale) {
  const double c = scale > 0.0 ? rint(x / scale) : 0.0;  // (NaN scale: 0)
  return (int)fmin(fmax(c, -127.0), 127.0);
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
  template <class T>
  DEVM void load(const T* p, float (&xa)[E], float (&xb)[E], bool vec) const {
    if (vec && runs()) {
      float x[2 * E];
      if (inter) {
        load_n<T, 2 * E>(p + a(0), x, true);
#pragma unroll
        for (int i = 0; i < E; ++i) { xa[i] = x[2 * i]; xb[i] = x[2 * i + 1]; }
      } else {
        load_n<T, E>(p + a(0), xa, true);
        load_n<T, E>(p + b(0), xb, true);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) { xa[i] = (float)p[a(i)]; xb[i] = (float)p[b(i)]; }
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

// One workgroup: one 16-token block of one kv head (its keys or its values), or the queries of a block's
// tokens and q_per heads. Thread: token tid / 16, 1/16 of the head.
template <class T, int D>
__global__ __launch_bounds__(256) void k_kv_append(KvAppendArgs a, bool vk, bool vv, bool vq) {
  constexpr int E = D / 32;
  __shared__ unsigned long long red[4];
  __shared__ __attribute__((aligned(16))) uint8_t turned[D * 16];
  const int roles = 2 * a.c.heads + a.q_groups;
  const int role = blockIdx.x % roles, b = blockIdx.x / roles, s = blockIdx.y;
  if (s == a.b.seqs) {
    // (one more than the sequences where there is something to clear)
    for (int64_t r = max(a.b.start[s], 0) + (int64_t)blockIdx.x; r < a.b.rows; r += gridDim.x)
      for (int e = threadIdx.x; e < a.rest_cols / 8; e += 256) ((uint4*)(a.rest + r * a.rest_cols))[e] = make_uint4(0, 0, 0, 0);
    return;
  }
  const KvSeq q = kv_seq(a.b, s);
  const int blk = (q.past >> 4) + b, base = blk << 4;
  const int t_lo = max(q.past - base, 0), t_hi = min(q.past + q.n - base, 16);
  if (q.n == 0 || t_hi <= t_lo) return;
  const int tid = threadIdx.x, t = tid >> 4, c = tid & 15;
  const bool fresh = t >= t_lo && t < t_hi;
  const int64_t row = (int64_t)q.row + (base + t - q.past);
  const bool turn = a.rope.table && (role < a.c.heads || role >= 2 * a.c.heads);
  const Pairs<D> at(turn ? &a.rope : nullptr, c);
  float2 cs[E];
  if (turn && fresh) {
    const bool ok = base + t < a.rope.n_pos;
    const float2* tab = a.rope.table + (int64_t)(ok ? base + t : 0) * at.half;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (at.turns(i)) cs[i] = ok ? tab[c * E + i] : make_float2(NAN, NAN);
  }
  if (role >= 2 * a.c.heads) {
    if (!fresh) return;
    const int h0 = (role - 2 * a.c.heads) * a.q_per;
    for (int h = h0; h < min(h0 + a.q_per, a.q_heads); ++h) {
      float xa[E], xb[E];
      at.load((const T*)a.q.p + row * a.q.ld + h * a.q.hld, xa, xb, vq);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float u = xa[i], w = xb[i];
        if (at.turns(i)) {
          xa[i] = u * cs[i].x - w * cs[i].y;
          xb[i] = w * cs[i].x + u * cs[i].y;
        }
      }
      at.store((T*)a.q_out.p + row * a.q_out.ld + h * a.q_out.hld, xa, xb, vq);
    }
    return;
  }
  const bool key = role < a.c.heads;
  const int h = key ? role : role - a.c.heads;
  const int page = kv_page(a.c, a.b, s, blk);
  if (page < 0) return;
  const uint64_t block = kv_block(a.c, page, h, blk);
  int8_t* out = a.c.codes + block * (2 * 16 * D) + (key ? 0 : 16 * D);
  float* scale_at = a.c.scales + block * 2 + (key ? 0 : 1);
  const float old = t_lo > 0 ? *scale_at : 0.f;
  double xa[E], xb[E];
  unsigned long long most = 0;
  if (fresh) {
    const HeadsView& v = key ? a.k : a.v;
    float fa[E], fb[E];
    at.load((const T*)v.p + row * v.ld + h * v.hld, fa, fb, key ? vk : vv);
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
    // (bits of magnitudes are ordered as the magnitudes, infinities and NaN above all)
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const unsigned long long m = __double_as_longlong(xa[i]) & 0x7fffffffffffffffull,
                               n = __double_as_longlong(xb[i]) & 0x7fffffffffffffffull;
      most = max(most, max(m, n));
    }
  }
  most = wave_max_bits(most);
  if ((tid & 63) == 0) red[tid >> 6] = most;
  __syncthreads();
  most = max(max(red[0], red[1]), max(red[2], red[3]));
  const float scale = raised(old, __longlong_as_double((long long)most));
  const double sc = scale, ratio = scale > 0.f ? (double)old / sc : 0.0;
  const bool earlier = t < t_lo && scale != old;  // codes to be rounded again
  if (key) {
    int8_t* o = out + t * D;
    if (fresh || earlier) {
      int8_t ra[E], rb[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        ra[i] = (int8_t)(fresh ? code_of(xa[i], sc) : (int)rint((double)o[at.a(i)] * ratio));
        rb[i] = (int8_t)(fresh ? code_of(xb[i], sc) : (int)rint((double)o[at.b(i)] * ratio));
      }
      if (at.runs() && !at.inter) {
        __builtin_memcpy(__builtin_assume_aligned(o + at.a(0), E), ra, E);
        __builtin_memcpy(__builtin_assume_aligned(o + at.b(0), E), rb, E);
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          o[at.a(i)] = ra[i];
          o[at.b(i)] = rb[i];
        }
      }
    }
  } else {
    // values lie transposed, [D][16]: through LDS, out in runs of D / 16 bytes. (Codes of tokens that are
    // still to come are 0.)
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int ea = at.a(i) * 16 + t, eb = at.b(i) * 16 + t;
      int ca = 0, cb = 0;
      if (fresh) {
        ca = code_of(xa[i], sc);
        cb = code_of(xb[i], sc);
      } else if (t < t_lo) {
        ca = out[ea];
        cb = out[eb];
        if (earlier) {
          ca = (int)rint((double)ca * ratio);
          cb = (int)rint((double)cb * ratio);
        }
      }
      turned[ea] = (uint8_t)ca;
      turned[eb] = (uint8_t)cb;
    }
    __syncthreads();
    __builtin_memcpy(__builtin_assume_aligned(out + tid * (D / 16), D / 16), __builtin_assume_aligned(turned + tid * (D / 16), D / 16),
                     D / 16);
  }
  if (tid == 0 && (t_lo == 0 || scale != old)) *scale_at = scale;
}

// One workgroup: the tokens of one block that the call has, of one head.
template <class T, int D>
__global__ __launch_bounds__(256) void k_kv_read(KvReadArgs a) {
  const int both = 2 * a.c.heads;
  const int role = blockIdx.x % both, b = blockIdx.x / both, s = blockIdx.y;
  const KvSeq q = kv_seq(a.b, s);
  const int blk = (q.past >> 4) + b, base = blk << 4;
  const int t_lo = max(q.past - base, 0), t_hi = min(q.past + q.n - base, 16);
  if (q.n == 0 || t_hi <= t_lo) return;
  const bool key = role < a.c.heads;
  const int h = key ? role : role - a.c.heads;
  const HeadsView& v = key ? a.k : a.v;
  if (!v.p) return;
  const int page = kv_page(a.c, a.b, s, blk);
  const uint64_t at = kv_block(a.c, max(page, 0), h, blk);
  const int8_t* in = a.c.codes + at * (2 * 16 * D) + (key ? 0 : 16 * D);
  const float scale = page < 0 ? NAN : a.c.scales[at * 2 + (key ? 0 : 1)];
  for (int i = threadIdx.x; i < 16 * D; i += 256) {
    const int t = i / D, e = i % D;
    if (t < t_lo || t >= t_hi) continue;
    const int code = key ? in[i] : in[e * 16 + t];
    ((T*)v.p)[((int64_t)q.row + base + t - q.past) * v.ld + h * v.hld + e] = (T)((float)code * scale);
  }
}

template <class T>
hipError_t kv_append(KvAppendArgs a, hipStream_t st) {
  // vectors of the E elements that a thread takes: 16 bytes' alignment covers every E
  const bool vk = vectors(a.k, sizeof(T)), vv = vectors(a.v, sizeof(T)),
             vq = a.q.p && vectors(a.q, sizeof(T)) && vectors(a.q_out, sizeof(T));
  a.q_per = 4;
  a.q_groups = a.q.p ? (a.q_heads + a.q_per - 1) / a.q_per : 0;
  const dim3 grid((unsigned)a.nblk * (2 * a.c.heads + a.q_groups), (unsigned)a.b.seqs + (a.rest ? 1 : 0));
  const double bytes = (double)a.b.rows * a.c.dim * (2.0 * a.c.heads * (sizeof(T) + 1) + (a.q.p ? 2.0 * a.q_heads * sizeof(T) : 0.0));
  const char* name = a.q.p && a.q.p == a.q_out.p ? "kv_append_inplace" : "kv_append";
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    MEBP_TIMED(st, name, 0.0, bytes, hipLaunchKernelGGL((k_kv_append<T, D>), grid, dim3(256), 0, st, a, vk, vv, vq));
    return hipGetLastError();
  };
  return a.c.dim == 64 ? go(IC<64>{}) : a.c.dim == 128 ? go(IC<128>{}) : go(IC<256>{});
}

template <class T>
hipError_t kv_read(const KvReadArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.nblk * 2 * a.c.heads, (unsigned)a.b.seqs);
  const double bytes = (double)a.b.rows * a.c.dim * a.c.heads * 2.0 * (sizeof(T) + 1);
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    MEBP_TIMED(st, "kv_read", 0.0, bytes, hipLaunchKernelGGL((k_kv_read<T, D>), grid, dim3(256), 0, st, a));
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
