// Values into 8 bits: what the kernels of the projections share.
#pragma once
#include "fkv_proj.h"

namespace fkv {

// fp32 -> T, rounded once
template <int DT> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<0>(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)b) << 16;
}
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <> __device__ __forceinline__ uint32_t pack2<1>(float a, float b) {
  bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
template <int DT>
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(pack2<DT>(f[0], f[1]), pack2<DT>(f[2], f[3]), pack2<DT>(f[4], f[5]), pack2<DT>(f[6], f[7]));
}

struct OpMaxU32 {
  static __device__ __forceinline__ uint32_t identity() { return 0u; }
  __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};
// the largest of the bits of |v|: as whole numbers they are in the values' order, infinities and NaN behind them
__device__ __forceinline__ uint32_t top_bits(const float* v) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
    m = b > m ? b : m;
  }
  return m;
}
// over a row of 16 lanes, for all of them
__device__ __forceinline__ uint32_t top_of_16(uint32_t m) { return class_reduce_row<1>(m, OpMaxU32()); }

// What a block's values are divided by.  Quotients are fp32's nearest: one step of Newton's from the nearest reciprocal, whose remainder is
// exact.  For the scale, top / 448 = (top 2^-e / 0.875) 2^(e - 9) with top 2^-e in [1, 2), so nothing leaves fp32's normal range; scales of
// less than 2^-90 are taken with the values times 2^64, for the same reason.
struct Quant {
  float scale, inv;              // (of values times 2^64 where `small`)
  bool bad, small;
};
__device__ __forceinline__ float nearest_inverse(float m) {
  float y = __builtin_amdgcn_rcpf(m);
  y = fmaf(fmaf(-m, y, 1.f), y, y);
  return fmaf(fmaf(-m, y, 1.f), y, y);
}
__device__ __forceinline__ Quant quant_of(uint32_t top) {
  Quant q;
  q.bad = top >= 0x7f800000u;
  const uint32_t e = top & 0x7f800000u;
  const float a = __uint_as_float((top & 0x7fffffu) | 0x3f800000u), inv = 0x1.24924ap+0f, t = a * inv;
  const float m = fmaf(fmaf(-t, 0.875f, a), inv, t);
  // 2^(e - 9); a top below 2^-117 has the least scale (or next to it, which its half gives)
  const float scale = e >= (10u << 23) ? m * __uint_as_float(e - (9u << 23)) : m * __uint_as_float(e >= (9u << 23) ? 0x00400000u : 0u);
  q.scale = q.bad ? 1.f : fmaxf(scale, 0x1p-126f);
  q.small = q.scale < 0x1p-90f;
  if (q.small) q.scale *= 0x1p64f;
  q.inv = nearest_inverse(q.scale);
  return q;
}
__device__ __forceinline__ float scale_of(const Quant& q) { return q.bad ? __builtin_nanf("") : q.small ? q.scale * 0x1p-64f : q.scale; }
__device__ __forceinline__ float quotient(const Quant& q, float x) {
  const float t = x * q.inv;
  return fmaf(fmaf(-t, q.scale, x), q.inv, t);
}
// eight codes; a quotient is at most a step of fp32 above 448 and rounds to it
__device__ __forceinline__ uint2 codes_of(const Quant& q, const float* v) {
  float t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = v[i];
  if (q.small)
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] *= 0x1p64f;
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = quotient(q, t[i]);
  int a = 0, b = 0;
  a = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], a, false);
  a = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], a, true);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(t[4], t[5], b, false);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(t[6], t[7], b, true);
  return q.bad ? make_uint2(0u, 0u) : make_uint2((uint32_t)a, (uint32_t)b);
}

}  // namespace fkv
