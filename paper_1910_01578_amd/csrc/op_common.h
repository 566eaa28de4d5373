// What the layer operators (norm.hip, fc.hip, rel_attention.hip) share.
#pragma once

#include "device_common.h"
#include "train_planes.h"

namespace gdp {
namespace op {

// 16 bytes at any element address: global vector loads and stores have no alignment
// rule on gfx950, so odd widths and row strides take the same path as even ones.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

template <typename T>
__device__ __forceinline__ Vec16<T> load16_any(const T* p) {
  const u32x4_any t = *reinterpret_cast<const u32x4_any*>(p);
  Vec16<T> r;
  *reinterpret_cast<uint4*>(&r) = make_uint4(t.x, t.y, t.z, t.w);
  return r;
}
template <typename T>
__device__ __forceinline__ void store16_any(T* p, const Vec16<T>& r) {
  const uint4 t = *reinterpret_cast<const uint4*>(&r);
  *reinterpret_cast<u32x4_any*>(p) = u32x4_any{t.x, t.y, t.z, t.w};
}
// The first `left` (1 .. N) of a vector's elements; the rest of a load are zero.
template <typename T>
__device__ __forceinline__ Vec16<T> load16_part(const T* p, int left) {
  if (left >= Vec16<T>::N) return load16_any(p);
  Vec16<T> r;
#pragma unroll
  for (int i = 0; i < Vec16<T>::N; ++i) r.v[i] = i < left ? p[i] : (T)0.f;
  return r;
}
template <typename T>
__device__ __forceinline__ void store16_part(T* p, const Vec16<T>& r, int left) {
  if (left >= Vec16<T>::N) {
    store16_any(p, r);
    return;
  }
#pragma unroll
  for (int i = 0; i < Vec16<T>::N; ++i)
    if (i < left) p[i] = r.v[i];
}

__device__ __forceinline__ bf16x8 as_bf16x8(const Vec16<bf16>& r) { return __builtin_bit_cast(bf16x8, r); }

// Matrix-core operand: eight values as one bf16 (bf16 data, exact) or three (fp32 data).
template <int NP>
struct Operand {
  bf16x8 p[NP];
};
__device__ __forceinline__ Operand<1> operand(const bf16x8& v) { return {{v}}; }
__device__ __forceinline__ Operand<3> operand(const float (&v)[8]) {
  const tr::Planes s = tr::split8(v);
  return {{s.p[0], s.p[1], s.p[2]}};
}
// Eight fp32 values rounded to one bf16 plane, or as three.
template <int NP>
__device__ __forceinline__ Operand<NP> operand_of(const float (&v)[8]) {
  if constexpr (NP == 3) {
    return operand(v);
  } else {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
    union {
      bf16x2 h[4];
      bf16x8 q;
    } o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.h[i] = __builtin_convertvector(f32x2{v[2 * i], v[2 * i + 1]}, bf16x2);
    return {{o.q}};
  }
}

__device__ __forceinline__ f32x4 mma16(const bf16x8& a, const bf16x8& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// top += a b of the first planes; low += the five plane pairs of weight 2^-16 and above
// below them, smallest first, on a sum of their own (an instruction drops the low bits
// of what is small beside its sum).
template <int NP>
__device__ __forceinline__ void mma_planes(const Operand<NP>& a, const Operand<NP>& b, f32x4& top, f32x4& low) {
  if constexpr (NP == 3) {
    low = mma16(a.p[2], b.p[0], low);
    low = mma16(a.p[1], b.p[1], low);
    low = mma16(a.p[0], b.p[2], low);
    low = mma16(a.p[1], b.p[0], low);
    low = mma16(a.p[0], b.p[1], low);
  }
  top = mma16(a.p[0], b.p[0], top);
}

// Four 8-byte words of a 16-lane group, transposed: destination lane 4 q + p receives
// in slot e element p of the word that source lane 4 e + q addresses.
__device__ __forceinline__ uint2 read_tr16(const char* p) {
  typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4_t;
  const bf16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
      (__attribute__((address_space(3))) bf16x4_t*)((__attribute__((address_space(3))) char*)p));
  return __builtin_bit_cast(uint2, v);
}
__device__ __forceinline__ bf16x8 join8(uint2 lo, uint2 hi) {
  return __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y));
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) v += xor_shfl(v, m);
  return v;
}

}  // namespace op
}  // namespace gdp
