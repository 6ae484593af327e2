// What the sources of the network operators share: vectors of eight values, 8-bit blocks, reductions, errors.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/bbo_net.h"

__attribute__((visibility("hidden"))) int net_fail(int code, const char* msg);          // keeps the message, returns code
__attribute__((visibility("hidden"))) int net_launched(void);                           // BBO_OK, or the launch's error
__attribute__((visibility("hidden"))) void net_begin(void);                             // drops an old message

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
// Vectors at the alignment of one element: the memory pipe takes 16 bytes at any address.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));

typedef uint16_t bf16;  // as bits

// (by value: a bit cast of a vector's element reads its first)
__device__ inline float as_f32(uint32_t x) { return __builtin_bit_cast(float, x); }
__device__ inline uint32_t as_u32(float x) { return __builtin_bit_cast(uint32_t, x); }

__device__ inline float to_f32(float x) { return x; }
__device__ inline float to_f32(bf16 x) { return as_f32((uint32_t)x << 16); }
template <typename T>
__device__ inline T from_f32(float x);
template <>
__device__ inline float from_f32<float>(float x) {
  return x;
}
template <>
__device__ inline bf16 from_f32<bf16>(float x) {  // round to nearest, ties to even
  return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// Eight values from p, of which the first `here` exist; zeros for the others.
__device__ inline void load8(const float* p, int here, float (&v)[8]) {
  if (here >= 8) {
    const u32x4_any a = *(const u32x4_any*)p, b = *(const u32x4_any*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = as_f32(a[i]), v[4 + i] = as_f32(b[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = i < here ? p[i] : 0.f;
  }
}
__device__ inline void load8(const bf16* p, int here, float (&v)[8]) {
  if (here >= 8) {
    const u32x4_any a = *(const u32x4_any*)p;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      v[2 * i] = as_f32(a[i] << 16);
      v[2 * i + 1] = as_f32(a[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = i < here ? to_f32(p[i]) : 0.f;
  }
}
__device__ inline void store8(float* p, int here, const float (&v)[8]) {
  if (here >= 8) {
    u32x4_any a, b;
#pragma unroll
    for (int i = 0; i < 4; i++) a[i] = as_u32(v[i]), b[i] = as_u32(v[4 + i]);
    *(u32x4_any*)p = a;
    *(u32x4_any*)(p + 4) = b;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (i < here) p[i] = v[i];
  }
}
__device__ inline void store8(bf16* p, int here, const float (&v)[8]) {
  if (here >= 8) {
    u32x4_any a;
#pragma unroll
    for (int i = 0; i < 4; i++) a[i] = (uint32_t)from_f32<bf16>(v[2 * i]) | (uint32_t)from_f32<bf16>(v[2 * i + 1]) << 16;
    *(u32x4_any*)p = a;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (i < here) p[i] = from_f32<bf16>(v[i]);
  }
}
// Eight bytes, lowest first.
__device__ inline void store8_bytes(uint8_t* p, int here, uint32_t lo, uint32_t hi) {
  if (here >= 8) {
    u32x2_any a;
    a[0] = lo;
    a[1] = hi;
    *(u32x2_any*)p = a;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (i < here) p[i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
  }
}

// --- rows of 16 lanes and waves --------------------------------------------
template <int N>
__device__ inline float ror16(float x) {  // the value N lanes further round the row of 16
  return as_f32((uint32_t)__builtin_amdgcn_update_dpp(0, (int)as_u32(x), 0x120 + N, 0xf, 0xf, false));
}
__device__ inline float max16(float x) {
  x = fmaxf(x, ror16<8>(x));
  x = fmaxf(x, ror16<4>(x));
  x = fmaxf(x, ror16<2>(x));
  return fmaxf(x, ror16<1>(x));
}
__device__ inline float wave_sum(float x) {
  x += ror16<8>(x);
  x += ror16<4>(x);
  x += ror16<2>(x);
  x += ror16<1>(x);
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// --- 8-bit blocks ----------------------------------------------------------
__device__ inline float finite_abs(float x) {  // 0 for infinities and NaN
  const float a = __builtin_fabsf(x);
  return a < __builtin_inff() ? a : 0.f;
}
// The scale's byte for a block whose largest magnitude is `top`: top / 2^(byte - 127) is in (224, 448], 448 = 1.75 * 2^8 being e4m3's largest.
__device__ inline int scale_byte(float top) {
  const uint32_t b = as_u32(top);
  const int e = (int)(b >> 23) - 8 + ((b & 0x7fffff) > 0x600000);
  return e < 0 ? 0 : e;  // (at most 247: top is finite)
}
__device__ inline float inverse_scale(int byte) { return as_f32((uint32_t)(254 - byte) << 23); }  // 2^(127 - byte)
__device__ inline float e4m3_input(float x, float inv) {  // what the conversion is given: NaN stays, an infinity becomes NaN
  return __builtin_fabsf(x) < __builtin_inff() ? x * inv : __builtin_nanf("");
}
__device__ inline uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ inline void pack8_e4m3(const float (&v)[8], float inv, uint32_t& lo, uint32_t& hi) {
  float t[8];
#pragma unroll
  for (int i = 0; i < 8; i++) t[i] = e4m3_input(v[i], inv);
  lo = pack_e4m3(t[0], t[1], t[2], t[3]);
  hi = pack_e4m3(t[4], t[5], t[6], t[7]);
}

inline bool float_type(int dtype) { return dtype == BBO_F32 || dtype == BBO_BF16; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
__device__ inline int64_t ceil_div_d(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace
