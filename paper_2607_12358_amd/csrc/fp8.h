// 8-bit floating point (e4m3, OCP: finite up to 448, no infinities) with a scale
// for each group of 128 inputs: what the kernels that make such rows share.
#pragma once

#include "common.h"

namespace acid {

constexpr int kFp8Group = 128;
constexpr float kFp8Most = 448.0f;
constexpr float kFp8Least = 0x1p-126f;  // smallest scale: its reciprocal is finite

inline int64_t fp8_groups(int64_t k) { return (k + kFp8Group - 1) / kFp8Group; }

// |x| as bits: they order like the values, with infinity and then every NaN
// above all numbers, so a group's largest tells of both.
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Largest over the 16 lanes of a row of the wave, in each of them.
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
#define MAX_DPP(ctrl) \
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, false))
  MAX_DPP(0x128);  // rotated by 8 lanes, 4, 2, 1
  MAX_DPP(0x124);
  MAX_DPP(0x122);
  MAX_DPP(0x121);
#undef MAX_DPP
  return v;
}

// A group's scale, largest |x| / 448, and the factor that its values are
// multiplied with.  A group with an infinity or a NaN has scale NaN, and codes that
// mean nothing.
struct Fp8Scale {
  float scale, inv;
  __device__ __forceinline__ explicit Fp8Scale(uint32_t most) {
    const bool finite = most < 0x7f800000u;
    scale = finite ? fmaxf(__uint_as_float(most) / kFp8Most, kFp8Least) : __builtin_nanf("");
    inv = finite ? 1.0f / scale : 0.f;
  }
};

// Four values as e4m3, to nearest even, in one word from the lowest byte up.  The
// largest of a group may come out just over 448, and is that.
__device__ __forceinline__ uint32_t to_fp8(float a, float b, float c, float d) {
  a = __builtin_amdgcn_fmed3f(a, -kFp8Most, kFp8Most);
  b = __builtin_amdgcn_fmed3f(b, -kFp8Most, kFp8Most);
  c = __builtin_amdgcn_fmed3f(c, -kFp8Most, kFp8Most);
  d = __builtin_amdgcn_fmed3f(d, -kFp8Most, kFp8Most);
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return (uint32_t)w;
}

}  // namespace acid
