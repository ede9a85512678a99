// Shared by the 8-bit operators (agcn_quant.hip, agcn_qlinear.hip): element
// types, blocks, and the power-of-two scale of a block.
#pragma once

#include <hip/hip_runtime.h>

#include <cfloat>
#include <cstdint>
#include <cstring>

#include "agcn_internal.hpp"

namespace agcn {

// Columns that share a scale (and rows, for a weight).
constexpr int kQBlock = 128;

using bf16_t = __bf16;
using f16_t = _Float16;

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16_t v) { return (float)v; }
__device__ __forceinline__ float to_float(f16_t v) { return (float)v; }

// v < 0 becomes 0 (NaN and -0 stay), as in the aggregation's epilogue.
__device__ __forceinline__ float q_act(float v, int32_t act) { return act != 0 && v < 0.0f ? 0.0f : v; }

// sizeof(V) bytes at any alignment; gfx950 loads and stores them in one
// instruction wherever they start.
template <class V, class P>
__device__ __forceinline__ V load_any(const P* p) {
  V v;
  __builtin_memcpy(&v, p, sizeof(V));
  return v;
}
template <class V, class P>
__device__ __forceinline__ void store_any(P* p, const V& v) {
  __builtin_memcpy(p, &v, sizeof(V));
}

// Lane i's value combined with lane i ^ ... of its 16 lanes by rotations: after
// the four steps every lane of the 16 holds the result of all of them.
template <int ROR>
__device__ __forceinline__ float dpp_ror(float v) {
  const int b = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, 0x120 + ROR, 0xf, 0xf, false));
}
__device__ __forceinline__ float sum16(float v) {
  v += dpp_ror<8>(v);
  v += dpp_ror<4>(v);
  v += dpp_ror<2>(v);
  return v + dpp_ror<1>(v);
}
__device__ __forceinline__ float max16(float v) {
  v = fmaxf(v, dpp_ror<8>(v));
  v = fmaxf(v, dpp_ror<4>(v));
  v = fmaxf(v, dpp_ror<2>(v));
  return fmaxf(v, dpp_ror<1>(v));
}

// The code (exponent + 127) of a block's scale: the least e >= -126 with
// amax <= 448 * 2^e, amax finite. 448 = 1.75 * 2^8, so e is amax's exponent
// less 8, and one more where its mantissa is past 1.75.
__device__ __forceinline__ int scale_code(float amax) {
  const uint32_t b = __builtin_bit_cast(uint32_t, amax);
  const int code = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return code < 1 ? 1 : code;
}
// 2^-e of a code in [1, 247], exactly.
__device__ __forceinline__ float inverse_scale(int code) {
  return __builtin_bit_cast(float, (uint32_t)(254 - code) << 23);
}
// |v| where it is finite, else 0: infinities and NaN do not set a block's scale.
__device__ __forceinline__ float finite_abs(float v) {
  const float a = fabsf(v);
  return a < __builtin_inff() ? a : 0.0f;
}
// Four values as e4m3, rounded to nearest even. |v| <= 448 after the scale;
// infinities and NaN become NaN (e4m3 has no infinity).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
  return (uint32_t)v;
}

}  // namespace agcn
