// Rows of a cache in eight bits: codes of one type with one fp32 scale a row.
//   scale = fl32(max |x| / top);  code = the type's value nearest to fl32(x / scale), ties to even
#pragma once

#include "common.h"

namespace adt {

// An element of a cache: float, uint16_t (bf16 bits) or one of these.
struct E4M3 {
  uint8_t bits;
  static constexpr float TOP = 448.f;
};
struct I8 {
  int8_t bits;
  static constexpr float TOP = 127.f;
};
template <typename C>
constexpr bool EIGHT = std::is_same_v<C, E4M3> || std::is_same_v<C, I8>;

// The scale of a row whose largest size is `top_value` (NaN or infinite: NaN), and what its values are
// multiplied by.  The division is done in double: the quotient by the reciprocal then rounds to the
// same fp32 value as x / scale, halfway cases included, whose quotients fp32 holds exactly.
template <typename C>
__device__ __forceinline__ float row_scale(float largest, double& inverse) {
  if (!(largest <= 3.402823466e38f)) {
    inverse = 0.0;
    return __uint_as_float(0x7fc00000u);
  }
  const float s = (float)((double)largest / (double)C::TOP);
  inverse = s > 0.f ? 1.0 / (double)s : 0.0;
  return s;
}

// Codes of four quotients, in four bytes.  A scale near the smallest fp32 is off by more than the
// quotient's rounding, so quotients are held within the type.
template <typename C>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  auto within = [](float x) { return fminf(fmaxf(x, -C::TOP), C::TOP); };
  a = within(a), b = within(b), c = within(c), d = within(d);
  if constexpr (std::is_same_v<C, E4M3>) {
    int r = 0;
    r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    return (uint32_t)r;
  } else {
    auto byte = [](float x) { return (uint32_t)(int)rintf(x) & 0xffu; };
    return byte(a) | byte(b) << 8 | byte(c) << 16 | byte(d) << 24;
  }
}

// Values of the codes in four bytes.
template <typename C>
__device__ __forceinline__ float4 decode4(uint32_t x) {
  if constexpr (std::is_same_v<C, E4M3>) {
    return make_float4(__builtin_amdgcn_cvt_f32_fp8((int)x, 0), __builtin_amdgcn_cvt_f32_fp8((int)x, 1),
                       __builtin_amdgcn_cvt_f32_fp8((int)x, 2), __builtin_amdgcn_cvt_f32_fp8((int)x, 3));
  } else {
    // (bit fields of 32 bits: the conversions take their bytes themselves; casts to int8_t go by way of 16 bits)
    auto code = [&](uint32_t at) { return (float)(int)__builtin_amdgcn_sbfe(x, at, 8); };
    return make_float4(code(0), code(8), code(16), code(24));
  }
}
// The same as bf16, which holds every code exactly.
template <typename C>
__device__ __forceinline__ u16x4 decode4_bf16(uint32_t x) {
  if constexpr (std::is_same_v<C, E4M3>) {
    struct Two {
      bf16x2 a, b;
    };
    return __builtin_bit_cast(u16x4, Two{__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false),
                                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true)});
  } else {
    const float4 f = decode4<C>(x);
    return u16x4{f2bf(f.x), f2bf(f.y), f2bf(f.z), f2bf(f.w)};
  }
}

}  // namespace adt
