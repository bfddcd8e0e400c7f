// Pages of 8 bits (QUEST_FLAG_E4M3_PAGES): e4m3 numbers, a power-of-two scale for each (page, KV head) of keys and of values.
//
// With e >= -15 the smallest step of a stored number, 2^-9 2^e, is a step of fp16, and with magnitudes up to 61440 = 240 * 2^8 none
// passes the largest fp16 number: codes become fp16 numbers exactly.  The other way the hardware rounds to the nearest, ties to even,
// subnormal results included: tested for every e from -15 to 8 and all finite fp16 numbers that a scale of 2^e holds, and with the codes
// that come of them the way back.
#pragma once

#include "quest_common.h"

namespace quest {

constexpr int kRowBytes8 = kHeadDim;             // one token's key (or value) of one head
constexpr int kLeastExponent = -15;
constexpr uint32_t kMostHalf = 0x7b80;           // 61440

#if defined(__HIPCC__)

typedef short short2v_t __attribute__((ext_vector_type(2)));

// Two of the four codes of a dword, times the scale.
template <bool kHigh>
__device__ __forceinline__ uint32_t halves_of(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)codes, scale, kHigh));
}
// Eight codes.
__device__ __forceinline__ uint4 halves_of(uint2 codes, float scale) {
  return make_uint4(halves_of<false>(codes.x, scale), halves_of<true>(codes.x, scale), halves_of<false>(codes.y, scale),
                    halves_of<true>(codes.y, scale));
}
// Eight fp16 numbers of magnitude up to 448 times the scale, rounded.
__device__ __forceinline__ uint2 codes_of(uint4 h, float scale) {
  auto four = [&](uint32_t a, uint32_t b) {
    short2v_t r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(half2_t, a), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(half2_t, b), scale, true);
    return __builtin_bit_cast(uint32_t, r);
  };
  return make_uint2(four(h.x, h.y), four(h.z, h.w));
}

// Magnitudes of fp16 numbers as integers, those above 61440 as that (NaN is above all).
__device__ __forceinline__ uint32_t magnitude2(uint32_t h2) { return h2 & 0x7fff7fffu; }
// The number itself; NaN stays.
__device__ __forceinline__ uint32_t at_most2(uint32_t h2) {
  const half2_t most = {(_Float16)61440.f, (_Float16)61440.f};
  const half2_t v = __builtin_bit_cast(half2_t, h2);
  const half2_t c = __builtin_elementwise_minimum(__builtin_elementwise_maximum(v, -most), most);
  return __builtin_bit_cast(uint32_t, c);
}
__device__ __forceinline__ uint4 at_most8(uint4 v) {
  return make_uint4(at_most2(v.x), at_most2(v.y), at_most2(v.z), at_most2(v.w));
}

// e of the scale for a largest magnitude, given as the bits of an fp16 number: 448 is 1.75 * 2^8, so a
// magnitude with a mantissa above that of 1.75 carries into the exponent.
__device__ __forceinline__ int exponent_for(uint32_t bits) {
  const int e = (int)((min(bits, kMostHalf) + 0xff) >> 10) - 15 - 8;
  return max(e, kLeastExponent);
}
__device__ __forceinline__ float scale_of(int exponent) { return __builtin_bit_cast(float, (uint32_t)(exponent + 127) << 23); }
__device__ __forceinline__ int exponent_of(float scale) { return (int)(__builtin_bit_cast(uint32_t, scale) >> 23) - 127; }

// A buffer of the first `bytes` of a block of eight tokens: what lies behind them is not read, and zero.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const char* pool, uint32_t block, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(pool) + (size_t)block * (8 * kRowBytes8), 0, bytes, 0x00020000);
}
// kOnce: non-temporal, for what a launch reads once.
template <bool kOnce>
__device__ __forceinline__ uint4 row16(__amdgpu_buffer_rsrc_t rows, int lane) {
  const auto v = __builtin_amdgcn_raw_buffer_load_b128(rows, lane * 16, 0, kOnce ? 2 : 0);
  return make_uint4(v[0], v[1], v[2], v[3]);
}

#endif  // __HIPCC__

}  // namespace quest
