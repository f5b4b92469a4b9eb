// Reading the rows of the 4-bit cache: what the kernels that turn them into values share.
#pragma once

#include <type_traits>

#include "rbq_device.h"
#include "rbq_internal.h"

namespace rbq {
namespace {

// The place of dimension i of eight in a word of codes
template <int FMT>
constexpr int nibble_shift(int i) {
  return 4 * (FMT == RBQ_FP4 ? i : i / 2 + 4 * (i % 2));
}

// fp4's scale of a group, int4's step and base, from a row's word
template <int FMT>
__device__ __forceinline__ f32x2 row_scale(uint32_t word, int group) {
  if constexpr (FMT == RBQ_FP4) return f32x2{__uint_as_float((word >> (8 * group) & 255u) << 23), 0.f};
  return f32x2{__uint_as_float(word << 16), __uint_as_float(word & 0xFFFF0000u)};
}

// A code's value
template <int FMT>
__device__ __forceinline__ float code_value(uint32_t c, f32x2 sc) {
  if constexpr (FMT == RBQ_FP4) {
    // its exponent and mantissa as a float's, which is 2^-126 of it
    return __uint_as_float((c & 8u) << 28 | (c & 7u) << 22) * 0x1p126f * sc.x;
  } else {
    return fmaf(float(c), sc.x, sc.y);
  }
}

// Two whole numbers of 0 to 15 (bytes 2 HI, 2 HI + 1 of w) as a pair of bf16: as bytes they are e4m3
// codes of themselves times 2^-9 (that format's subnormals and its first octave are one linear range)
template <bool HI>
__device__ __forceinline__ uint32_t bytes_bf16(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 512.f, HI));
}
// The same less 7.5, so that sums over them do not grow beside their bases: 2 c - 15 by sign and magnitude
__device__ __forceinline__ uint32_t centred_bytes(uint32_t c) {   // four numbers of 0 to 15, as e4m3 of (2 c - 15) 2^-9
  const uint32_t low = ~c & 0x08080808u;                       // below 8: negative
  const uint32_t m = (c & 0x07070707u) ^ (low - (low >> 3));   // 7 - c there, c - 8 otherwise
  return m << 1 | 0x01010101u | low << 4;
}
template <bool HI>
__device__ __forceinline__ uint32_t centred_bf16(uint32_t bytes) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(bytes, 256.f, HI));
}
// int4's 8 codes of a word as bf16, in their order (CENTRED: less 7.5)
template <bool CENTRED = false>
__device__ __forceinline__ u32x4 word_whole(uint32_t w) {
  uint32_t even = w & 0x0F0F0F0Fu, odd = w >> 4 & 0x0F0F0F0Fu;   // dimensions 0 4 1 5, 2 6 3 7
  if constexpr (CENTRED) {
    even = centred_bytes(even);
    odd = centred_bytes(odd);
  }
  const uint32_t a = __builtin_amdgcn_perm(odd, even, 0x06040200u), b = __builtin_amdgcn_perm(odd, even, 0x07050301u);
  if constexpr (CENTRED) return u32x4{centred_bf16<false>(a), centred_bf16<true>(a), centred_bf16<false>(b), centred_bf16<true>(b)};
  return u32x4{bytes_bf16<false>(a), bytes_bf16<true>(a), bytes_bf16<false>(b), bytes_bf16<true>(b)};
}
// fp4's two codes of byte B of w, scaled, as a pair of bf16
template <int B>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}

// The 8 values of a word of codes as bf16, in their order
template <int FMT>
__device__ __forceinline__ u32x4 word_bf16(uint32_t w, f32x2 sc) {
  u32x4 r;
  if constexpr (FMT == RBQ_FP4) {
    r = u32x4{fp4_pair<0>(w, sc.x), fp4_pair<1>(w, sc.x), fp4_pair<2>(w, sc.x), fp4_pair<3>(w, sc.x)};
  } else {
    typedef float f32x2v __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const uint32_t even = w & 0x0F0F0F0Fu, odd = w >> 4 & 0x0F0F0F0Fu;   // nibbles 0 2 4 6 (dimensions 0 4 1 5), 1 3 5 7 (2 6 3 7)
    // (as bytes they are e4m3's codes of themselves times 2^-9)
    auto pair = [&](uint32_t v, auto high) {
      const f32x2v c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v, 512.f, decltype(high)::value);
      return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2v{fmaf(c.x, sc.x, sc.y), fmaf(c.y, sc.x, sc.y)}), bf16x2));
    };
    const uint32_t a = __builtin_amdgcn_perm(odd, even, 0x06040200u), b = __builtin_amdgcn_perm(odd, even, 0x07050301u);
    r = u32x4{pair(a, std::false_type{}), pair(a, std::true_type{}), pair(b, std::false_type{}), pair(b, std::true_type{})};
  }
  return r;
}

}  // namespace
}  // namespace rbq
