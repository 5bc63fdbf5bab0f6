// The 8-bit form of the KV cache: a token's row of 128 keys or values of one KV head is 128 e4m3 codes and one exponent e, and
// stands for code * 2^e.  e is the smallest power of two under which the row's largest finite magnitude is at most 448 (the largest
// e4m3 number), and at least -110: a power of two loses nothing to a finer scale, as e4m3 is itself a floating-point form, scaling by it is
// exact, and whatever is stored is a bf16 number again (4 significant bits, never subnormal).  Codes are rounded to nearest even; with
// the largest exponent, 120, they end at 240 (256 * 2^120 is past the largest bf16 number).
#ifndef MARL_KV_FP8_H
#define MARL_KV_FP8_H
#include "marl_internal.h"
#include "wave_ops.h"

namespace marl {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
constexpr int kMinExponent = -110, kMaxExponent = 120;

__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// Codes of the eight bf16 numbers `w` and the row's exponent.  The row's 128 numbers lie in the 16 neighbouring lanes of a DPP row.
// An infinity becomes the largest code and a NaN the code for it; neither counts for the exponent.  (Maxima and the tests are made on the bit patterns:
// a magnitude's order is that of its bits, and the compiler may take floating-point NaNs for impossible in some of the library's files.)
__device__ __forceinline__ u32x2 quantize_row(u32x4 w, int& e) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  auto row_max = [](u32x4 v) {
    u16x2 m = __builtin_bit_cast(u16x2, v[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu));
    uint32_t x = m[0] > m[1] ? m[0] : m[1];
    auto step = [&](auto ctrl_tag) {
      constexpr int ctrl = decltype(ctrl_tag)::value;
      const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, 0xf, 0xf, false);
      x = x > y ? x : y;
    };
    step(std::integral_constant<int, 0xB1>{});    // quad_perm [1, 0, 3, 2]
    step(std::integral_constant<int, 0x4E>{});    // quad_perm [2, 3, 0, 1]
    step(std::integral_constant<int, 0x141>{});   // row_half_mirror
    step(std::integral_constant<int, 0x140>{});   // row_mirror
    return x;
  };
  uint32_t top = row_max(w);
  constexpr uint32_t kLarge = 0x7f78u;   // 248 * 2^120, from where on the nearest code is 256
  const bool ordinary = __builtin_amdgcn_ballot_w64(top >= kLarge) == 0;   // wave-uniform
  if (!ordinary) {
    u32x4 finite = w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if ((finite[i] & 0x7fffu) >= 0x7f80u) finite[i] &= 0xffff0000u;
      if ((finite[i] & 0x7fff0000u) >= 0x7f800000u) finite[i] &= 0x0000ffffu;
    }
    top = row_max(finite);
  }
  // top = 1.f 2^(X - 127) with X its upper 8 bits: at most 448 2^e = 1.75 2^(e + 8)
  e = (int)(top >> 7) - 135 + ((top & 0x7fu) > 0x60u ? 1 : 0);
  e = e > kMinExponent ? e : kMinExponent;
  const float scale = pow2(-e);
  u32x2 codes;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int c = 0;
    c = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(w[2 * i] << 16) * scale, __uint_as_float(w[2 * i] & 0xffff0000u) * scale, c, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(w[2 * i + 1] << 16) * scale, __uint_as_float(w[2 * i + 1] & 0xffff0000u) * scale, c, true);
    codes[i] = (uint32_t)c;
  }
  if (!ordinary) {
    const uint32_t largest = e == kMaxExponent ? 0x77u : 0x7eu;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t x = (w[i >> 1] >> (16 * (i & 1))) & 0xffffu, at = 8 * (i & 3);
      if ((x & 0x7fffu) >= kLarge) {
        const uint32_t code = (x & 0x7fffu) > 0x7f80u ? 0x7fu : largest | (x >> 15) << 7;
        codes[i >> 2] = (codes[i >> 2] & ~(0xffu << at)) | code << at;
      }
    }
  }
  return codes;
}

// Two of the four codes of a word as packed bf16 numbers, times 2^e given as that number.
template <bool kUpper>
__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t w, float two_to_e) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, two_to_e, kUpper));
}

// The signed byte `i` of a word.
__device__ __forceinline__ int exponent_of(uint32_t w, int i) { return (int)(w << (24 - 8 * i)) >> 24; }

}  // namespace marl
#endif  // MARL_KV_FP8_H
