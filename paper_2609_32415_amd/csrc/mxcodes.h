// Codes of the quantised reference cache: e2m1 (two a byte, the first in the low half) and e4m3, and the
// scale bytes (exponent + 127, 255 for NaN) of their blocks of 32. Device code only; the definitions have
// internal linkage in every source that includes this header.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace refadapt {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

// Eight neighbouring elements of a row, in fp32 (bf16 widens exactly).
struct Oct {
  float f[8];
};

// The same as loaded.
template <bool BF16>
struct RawOct {
  u32x4 w[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const char* p) {
    w[0] = reinterpret_cast<const u32x4*>(p)[0];
    if constexpr (!BF16) w[1] = reinterpret_cast<const u32x4*>(p)[1];
  }
  __device__ __forceinline__ Oct widen() const {
    Oct x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        x.f[2 * i] = __uint_as_float(w[0][i] << 16);
        x.f[2 * i + 1] = __uint_as_float(w[0][i] & 0xffff0000u);
      } else {
        x.f[i] = __uint_as_float(w[0][i]);
        x.f[4 + i] = __uint_as_float(w[1][i]);
      }
    }
    return x;
  }
};

// bf16 bits of x, rounded to nearest even.
__device__ __forceinline__ uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
// The same of an fp64 value, in one rounding: by way of fp32 cut towards zero, whose last bit is set where something
// was cut off (a nearest fp32 value may lie halfway between two bf16 values where x does not).
__device__ __forceinline__ uint16_t bf16_bits(double x) {
  const float f = (float)x;
  uint32_t u = __float_as_uint(f);
  if ((double)f != x) {
    if (fabs((double)f) > fabs(x)) --u;
    u |= 1u;
  }
  return bf16_bits(__uint_as_float(u));
}

// Stores eight bf16 values (pairs, the first in the low half), widened for fp32.
template <bool BF16>
__device__ __forceinline__ void store_oct(char* p, u32x4 w) {
  if constexpr (BF16) {
    *reinterpret_cast<u32x4*>(p) = w;
  } else {
    reinterpret_cast<u32x4*>(p)[0] = u32x4{w[0] << 16, w[0] & 0xffff0000u, w[1] << 16, w[1] & 0xffff0000u};
    reinterpret_cast<u32x4*>(p)[1] = u32x4{w[2] << 16, w[2] & 0xffff0000u, w[3] << 16, w[3] & 0xffff0000u};
  }
}

// Bits of max|x_i|: for magnitudes the order of the bits is that of the values, with infinity and NaN on top.
__device__ __forceinline__ uint32_t max_bits(const Oct& x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x.f[i]) & 0x7fffffffu);
  return m;
}

// Scale byte of a block from the bits of its largest magnitude. Subnormals have exponent field 0, which
// the lowest exponent covers: their bits never reach e > lowest.
template <bool FP4>
__device__ __forceinline__ uint32_t scale_byte(uint32_t m) {
  constexpr int emax = FP4 ? 2 : 8, lowest = FP4 ? 0 : 3;
  constexpr uint32_t cut = FP4 ? 0x600000u : 0x680000u;  // fractions of 1.75 and 1.8125
  const int e = (int)(m >> 23) - emax + ((m & 0x7fffffu) > cut ? 1 : 0);
  return m >= 0x7f800000u ? 255u : (uint32_t)min(max(e, lowest), 254 - emax);
}

// The scale as the conversion instructions take it: the exponent field of a float.
__device__ __forceinline__ float scale_bits(uint32_t e) { return __uint_as_float(e << 23); }

// Rounds x * 2^-e to codes and stores them (4 or 8 bytes).
template <bool FP4>
__device__ __forceinline__ void store_codes(uint8_t* p, const Oct& x, uint32_t e) {
  const bool bad = e == 255;
  const float s = scale_bits(bad ? 127u : e);
  if constexpr (FP4) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.f[0], x.f[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.f[2], x.f[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.f[4], x.f[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.f[6], x.f[7], s, 3);
    *reinterpret_cast<uint32_t*>(p) = bad ? 0u : c;
  } else {
    // The conversion to e4m3 makes NaN of what rounds past 448. Only at the highest scale are there such
    // values, those above 448 * 2^119.
    constexpr float most = 1.75f * 0x1p127f;
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = fminf(fmaxf(x.f[i], -most), most);
    i16x2 a = {0, 0}, b = {0, 0};
    a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, f[0], f[1], s, false);
    a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, f[2], f[3], s, true);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, f[4], f[5], s, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, f[6], f[7], s, true);
    const u32x2 c = {__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
    *reinterpret_cast<u32x2*>(p) = bad ? u32x2{0u, 0u} : c;
  }
}

// Codes of eight elements (e2m1: in the first word).
template <bool FP4>
__device__ __forceinline__ u32x2 load_codes(const uint8_t* p) {
  if constexpr (FP4) return u32x2{*reinterpret_cast<const uint32_t*>(p), 0u};
  return *reinterpret_cast<const u32x2*>(p);
}

// Eight values as bf16 pairs: one conversion instruction a pair, exact; NaN under scale byte 255. Of the scale it reads
// the exponent field alone.
template <bool FP4>
__device__ __forceinline__ u32x4 decode_oct(u32x2 c, float s) {
  bf16x2 v[4];
  if constexpr (FP4) {
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], s, 0);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], s, 1);
    v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], s, 2);
    v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], s, 3);
  } else {
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[0], s, false);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[0], s, true);
    v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[1], s, false);
    v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[1], s, true);
  }
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, v[i]);
  return w;
}

}  // namespace
}  // namespace refadapt
