// Rotary positions on gfx950: the table of (cos, sin) per position and pair, and the rotation of heads by
// it. Pair j of a head turns by the angle p f_j:
//   y_a = x_a cos - x_b sin,  y_b = x_b cos + x_a sin,
// with (a, b) = (j, j + rot / 2), or (2 j, 2 j + 1) where pairs are interleaved; elements from `rot` on
// are copied. The gradient w.r.t. x is the transposed rotation: the sign of sin turns.
#include <math.h>

#include "device_common.h"
#include "heads.h"
#include "mebp_internal.h"

namespace mebp {
namespace {

// A thread computes its pair's frequency once, for kTablePos positions; angles and their reduction in
// 64 bits (a position of 2^20 at frequency 1 has 2e-10 of a turn left there, 0.06 in 32 bits). The 64-bit functions bound
// it: 131072 positions of 64 pairs 31 us, 2.1 TB/s; a program makes its tables once.
constexpr int kTablePos = 16;
__global__ __launch_bounds__(256) void k_rope_positions(RopeTableArgs a) {
  const int half = a.rot >> 1;
  const int j = blockIdx.y * 64 + (threadIdx.x & 63);
  if (j >= half) return;
  double f = pow(a.theta, -2.0 * j / (double)a.rot);
  if (a.inv_span != 0.0) {
    // by parts: the more turns a pair makes over the original length, the less is it slowed
    const double keep = fmin(fmax((a.turns * f - a.low) * a.inv_span, 0.0), 1.0);
    f *= keep + (1.0 - keep) * a.inv_factor;
  } else {
    f *= a.inv_factor;
  }
  const int64_t p0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * kTablePos;
  for (int64_t p = p0; p < p0 + kTablePos && p < a.n_pos; ++p) {
    double s, c;
    sincos((double)p * f, &s, &c);
    a.table[p * half + j] = make_float2((float)(a.gain * c), (float)(a.gain * s));
  }
}

DEV void turn(float2 cs, float sign, float& xa, float& xb) {
  const float s = cs.y * sign, a = xa, b = xb;
  xa = a * cs.x - b * s;
  xb = b * cs.x + a * s;
}

// 8 pairs (or 16 copied elements) of one token and of up to HP heads per thread, whose (cos, sin) are
// loaded once. Bytes bound it: 5.4 to 6.2 TB/s at 134 MB.
template <class T, bool INTER, int HP, bool STREAM>
__global__ __launch_bounds__(256) void k_rope_vec(RopeArgs a, int chunks, int groups) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int c = (int)(i % chunks);
  const int64_t r = i / chunks;
  const int g = (int)(r % groups);
  const int64_t n = r / groups;
  if (n >= a.tokens) return;
  const int half = a.rope.rot >> 1, e0 = c * 8, turned = half / 8;
  // the two runs of 8 elements
  const int ea = c < turned ? (INTER ? 2 * e0 : e0) : a.rope.rot + (c - turned) * 16;
  const int eb = c < turned && !INTER ? e0 + half : ea + 8;
  const bool two = eb + 8 <= a.dim;  // (an odd run of 8 at the end of the copied elements)
  float2 cs[8];
  const float sign = a.backward ? -1.f : 1.f;
  if (c < turned) {
    const int p = a.pos[n];
    const bool ok = (unsigned)p < (unsigned)a.rope.n_pos;
    const float4* t = (const float4*)(a.rope.table + (int64_t)(ok ? p : 0) * half + e0);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 v = t[k];
      cs[2 * k] = ok ? make_float2(v.x, v.y) : make_float2(NAN, NAN);
      cs[2 * k + 1] = ok ? make_float2(v.z, v.w) : make_float2(NAN, NAN);
    }
  }
  const T* x = (const T*)a.x.p + n * a.x.ld;
  T* y = (T*)a.y.p + n * a.y.ld;
  float va[HP][8], vb[HP][8];
#pragma unroll
  for (int k = 0; k < HP; ++k) {
    const int h = g * HP + k;
    if (h >= a.heads) break;
    load8(x + h * a.x.hld + ea, va[k]);
    if (two) load8(x + h * a.x.hld + eb, vb[k]);
  }
#pragma unroll
  for (int k = 0; k < HP; ++k) {
    const int h = g * HP + k;
    if (h >= a.heads) break;
    if (c < turned) {
#pragma unroll
      for (int m = 0; m < 8; ++m) {
        if constexpr (INTER) {
          if (m < 4)
            turn(cs[m], sign, va[k][2 * m], va[k][2 * m + 1]);
          else
            turn(cs[m], sign, vb[k][2 * m - 8], vb[k][2 * m - 7]);
        } else {
          turn(cs[m], sign, va[k][m], vb[k][m]);
        }
      }
    }
    if constexpr (STREAM) {
      stream8(y + h * a.y.hld + ea, va[k]);
      if (two) stream8(y + h * a.y.hld + eb, vb[k]);
    } else {
      store8(y + h * a.y.hld + ea, va[k]);
      if (two) store8(y + h * a.y.hld + eb, vb[k]);
    }
  }
}

// any size and alignment: a pair, or a copied element, of one head per thread. Small accesses and the indices' divisions
// bound it: 16384 x 8 x 256 bf16 62 us, 2.2 TB/s, 4096 x 12 x 128 fp32 19 us, 2.7.
template <class T>
__global__ __launch_bounds__(256) void k_rope_any(RopeArgs a) {
  const int half = a.rope.rot >> 1, per = half + a.dim - a.rope.rot;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int c = (int)(i % per);
  const int64_t r = i / per;
  const int h = (int)(r % a.heads);
  const int64_t n = r / a.heads;
  if (n >= a.tokens) return;
  const T* x = (const T*)a.x.p + n * a.x.ld + h * a.x.hld;
  T* y = (T*)a.y.p + n * a.y.ld + h * a.y.hld;
  if (c >= half) {
    const int e = a.rope.rot + c - half;
    y[e] = x[e];
    return;
  }
  const int ea = a.rope.interleaved ? 2 * c : c, eb = a.rope.interleaved ? 2 * c + 1 : c + half;
  const int p = a.pos[n];
  float2 cs = make_float2(NAN, NAN);
  if ((unsigned)p < (unsigned)a.rope.n_pos) cs = a.rope.table[(int64_t)p * half + c];
  float va = (float)x[ea], vb = (float)x[eb];
  turn(cs, a.backward ? -1.f : 1.f, va, vb);
  y[ea] = (T)va;
  y[eb] = (T)vb;
}

template <class T>
hipError_t rope_apply(const RopeArgs& a, hipStream_t st) {
  const double bytes = (double)a.tokens * a.heads * a.dim * 2 * sizeof(T);
  const char* name = a.x.p == a.y.p ? "rope_apply_inplace" : "rope_apply";
  const int half = a.rope.rot / 2;
  if (half % 8 == 0 && a.dim % 8 == 0 && vectors(a.x, sizeof(T)) && vectors(a.y, sizeof(T)) && aligned16(a.rope.table)) {
    const int chunks = half / 8 + (a.dim - a.rope.rot + 15) / 16;
    // One head a thread where four would leave compute units without a workgroup: 1111 x 12 x 128 fp32, half of it
    // turned, 5.9 us, by four 7.6; 4096 x 12 x 128 11.5 and 10.4. What the L2s cannot hold until it is read goes past
    // them: 16384 x 8 x 256 bf16, 67 MB, 24.8 us, else 29.1; 21.5 and 22.3 with inputs in the cache behind the L2s.
    auto blocks_by = [&](int hp) { return ((int64_t)a.tokens * ((a.heads + hp - 1) / hp) * chunks + 255) / 256; };
    auto go = [&](auto hp, auto stream, auto inter) {
      constexpr int HP = decltype(hp)::value;
      MEBP_TIMED(st, name, 0.0, bytes,
                 hipLaunchKernelGGL((k_rope_vec<T, decltype(inter)::value != 0, HP, decltype(stream)::value != 0>), dim3((unsigned)blocks_by(HP)),
                                    dim3(256), 0, st, a, chunks, (a.heads + HP - 1) / HP));
    };
    auto by = [&](auto hp, auto stream) { a.rope.interleaved ? go(hp, stream, IC<1>{}) : go(hp, stream, IC<0>{}); };
    blocks_by(4) < 256 ? by(IC<1>{}, IC<0>{}) : bytes / 2 > 32 << 20 ? by(IC<4>{}, IC<1>{}) : by(IC<4>{}, IC<0>{});
    return hipGetLastError();
  }
  const int64_t blocks = ((int64_t)a.tokens * a.heads * (a.dim - half) + 255) / 256;
  MEBP_TIMED(st, name, 0.0, bytes, hipLaunchKernelGGL(k_rope_any<T>, dim3((unsigned)blocks), dim3(256), 0, st, a));
  return hipGetLastError();
}
}  // namespace

hipError_t launch_rope_positions(const RopeTableArgs& a, hipStream_t st) {
  const int half = a.rot / 2;
  MEBP_TIMED(st, "rope_positions", 0.0, (double)a.n_pos * a.rot * 4,
             hipLaunchKernelGGL(k_rope_positions, dim3((unsigned)((a.n_pos + 4 * kTablePos - 1) / (4 * kTablePos)), (half + 63) / 64),
                                dim3(256), 0, st, a));
  return hipGetLastError();
}

hipError_t launch_rope_apply(const RopeArgs& a, int dtype, hipStream_t st) {
  if (dtype == LOGIT_F32) return rope_apply<float>(a, st);
  return dtype == LOGIT_F16 ? rope_apply<f16>(a, st) : rope_apply<bf16>(a, st);
}

}  // namespace mebp
