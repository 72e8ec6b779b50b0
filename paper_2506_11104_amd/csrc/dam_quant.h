// Codes of 8 bits and their scales, as the cache kernels write them and the decode kernels read them.
//
// The rows [block i, block (i + 1)) of one (sequence, KV head) share a scale byte s for K and one for V; a code c stands for
// c 2^(s - 127), and for 0 where s is 0. Scales are powers of two: dividing by one is exact, so a value is rounded once, to
// the same code on every machine; a block whose scale has to grow shifts the codes it holds; and every value of the cache is a
// bf16 number (e4m3 has 4 significant bits, int8 7), so the matrix cores take it without another rounding.
// A row that held a value that is not finite is stored as the code kNan in every place and reads as NaN.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dam.h"

namespace dam {

inline bool quant_format_ok(int format, int block) {
  return (format == DAM_KV_E4M3 || format == DAM_KV_INT8) && (block == 16 || block == 32 || block == 64 || block == 128);
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

#ifdef __HIPCC__
// 2^(s - 127) for s from 1 to 254, 0 for s = 0
__device__ __forceinline__ float scale_value(unsigned s) { return __uint_as_float(s << 23); }

template <int FORMAT>
struct Code;

template <>
struct Code<DAM_KV_E4M3> {
  static constexpr unsigned kNan = 0x7Fu;
  // from this scale on not all codes are fp32 numbers: the largest that is there
  static constexpr unsigned kHuge = 247;
  static constexpr float kMostHuge = 240.0f;
  __device__ static bool is_nan(unsigned byte) { return (byte & 0x7Fu) == 0x7Fu; }
  // The smallest scale >= 1 that holds the magnitude with these fp32 bits (finite): the largest code is 1.75 2^8, and the
  // addition carries into the exponent exactly where the significand is above 1.75.
  __device__ static unsigned need(unsigned bits) {
    return bits == 0 ? 0u : (unsigned)max(1, (int)((bits + 0x1FFFFFu) >> 23) - 8);
  }
  // four codes, lowest byte first
  __device__ static void unpack4(unsigned w, float *v) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1];
  }
  // rounded to nearest, ties to even; magnitudes of at most 448
  __device__ static unsigned pack4(const float *v) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
    return (unsigned)w;
  }
};

template <>
struct Code<DAM_KV_INT8> {
  static constexpr unsigned kNan = 0x80u;
  static constexpr unsigned kHuge = 249;
  static constexpr float kMostHuge = 63.0f;
  __device__ static bool is_nan(unsigned byte) { return (byte & 0xFFu) == 0x80u; }
  // the largest code is 127 = 1.984375 2^6
  __device__ static unsigned need(unsigned bits) {
    return bits == 0 ? 0u : (unsigned)max(1, (int)((bits + 0x1FFFFu) >> 23) - 6);
  }
  __device__ static void unpack4(unsigned w, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)(int8_t)(w >> (8 * i));
  }
  __device__ static unsigned pack4(const float *v) {
    unsigned w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= ((unsigned)(int)rintf(v[i]) & 0xFFu) << (8 * i);
    return w;
  }
};

// Eight values, already divided by their scale s, as codes. (Rounding may carry a value of nearly 2^128 to 2^128, which is
// no fp32 number: such a value goes to the code below.)
template <int FORMAT>
__device__ __forceinline__ uint2 pack8(float (&v)[8], unsigned s) {
  using C = Code<FORMAT>;
  if (s >= C::kHuge)  // (the whole block)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = fminf(fmaxf(v[e], -C::kMostHuge), C::kMostHuge);
  return make_uint2(C::pack4(v), C::pack4(v + 4));
}
#endif

}  // namespace dam
