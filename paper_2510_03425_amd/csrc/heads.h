// Rows of heads in fp32, fp16 or bf16: loads and stores of 8 elements, and which views take them.
#pragma once
#include "device_common.h"
#include "mebp_internal.h"

// 8 elements of 16 aligned bytes each 4 (fp32) or 8 (16 bits)
DEV void load8(const float* p, float* v) {
  const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
DEV void load8(const f16* p, float* v) {
  const f16x8 a = *(const f16x8*)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
}
DEV void load8(const bf16* p, float* v) {
  const bf16x8 a = *(const bf16x8*)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
}
DEV void store8(float* p, const float* v) {
  ((float4*)p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  ((float4*)p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
DEV void store8(f16* p, const float* v) {
  f16x8 a;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = (f16)v[i];
  *(f16x8*)p = a;
}
DEV void store8(bf16* p, const float* v) {
  bf16x8 a;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = (bf16)v[i];
  *(bf16x8*)p = a;
}
// the same past the L2s, for what they would not hold until it is read
template <class T>
DEV void stream8(T* p, const float* v) {
  typedef uint32_t run __attribute__((ext_vector_type(4)));
  T t[8];
  run a[sizeof(T) / 2];
  store8(t, v);
  __builtin_memcpy(a, t, sizeof(t));
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) __builtin_nontemporal_store(a[i], (run*)p + i);
}

namespace mebp {
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// whether every run of 16 bytes of a view's rows starts at an aligned address
inline bool vectors(const HeadsView& v, size_t size) {
  return aligned16(v.p) && (size_t)v.ld * size % 16 == 0 && (size_t)v.hld * size % 16 == 0;
}
}  // namespace mebp
