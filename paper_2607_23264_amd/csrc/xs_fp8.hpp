// E4M3 codes with one fp32 scale per block of 128, and the lanes' maxima that give the scale.
//
//   s = max(amax, 2^-60) / 448        code = E4M3(x / s), ties to even
//
// both quotients rounded to fp32, so that every implementation with these divisions has the same bits (a
// product with a rounded 1 / 448, as some take for a division by a constant, has other scales, and other codes
// where x / s is a tie). x / s comes without a division: with r = fl(1 / s) and q = fl(x r), q is within an fp32 unit of
// x / s, q s - x is exact in one fused multiply-add, and fl(q - (q s - x) r) is the rounded quotient
// (Markstein's theorem; it asks for r correctly rounded and for a remainder that does not
// underflow: at a code that is not zero q >= 2^-10 and s >= 2^-69, so its last bit is 2^-125 or more).
// A block with an infinity or a NaN has the scale NaN and zero codes: every product with it is NaN.
#pragma once
#include "xs_common.hpp"

namespace xs {
namespace f8 {

constexpr float kAmaxFloor = 0x1p-60f;

// A block's scale, its reciprocal, and ~0 or (a block without a finite maximum) 0, which the codes are
// masked with; such a block's scale is NaN.
struct Scale {
  float s, inv;
  uint32_t mask;
};
__device__ __forceinline__ Scale scale_from(float s, float inv) { return Scale{s, inv, s == s ? ~0u : 0u}; }

// From the bits of the block's largest magnitude as an fp32 value (sign cleared; a NaN's are above an
// infinity's, and magnitudes order as integers).
__device__ __forceinline__ Scale scale_of(uint32_t amax_bits) {
  const float s = amax_bits >= 0x7F800000u ? __builtin_nanf("") : fmaxf(__uint_as_float(amax_bits), kAmaxFloor) / 448.f;
  return scale_from(s, 1.f / s);
}

__device__ __forceinline__ float quotient(float x, const Scale& c) {
  const float q = x * c.inv;
  const float over = __builtin_fmaf(q, c.s, -x);   // the remainder negated: a zero keeps its sign
  return __builtin_fmaf(over, -c.inv, q);
}

// Four codes, the first in the low byte (round to nearest even in hardware; |x / s| <= 448 after
// its rounding, so nothing saturates).
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, const Scale& s) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(a, s), quotient(b, s), 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(c, s), quotient(d, s), v, true);
  return static_cast<uint32_t>(v) & s.mask;
}

// Eight bf16 of one 16-byte piece.
__device__ __forceinline__ uint2 codes8(u32x4 raw, const Scale& s) {
  return make_uint2(codes4(bf_lo(raw[0]), bf_hi(raw[0]), bf_lo(raw[1]), bf_hi(raw[1]), s),
                    codes4(bf_lo(raw[2]), bf_hi(raw[2]), bf_lo(raw[3]), bf_hi(raw[3]), s));
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {   // of two packed 16-bit magnitudes
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
__device__ __forceinline__ uint32_t mag2(uint32_t w) { return w & 0x7FFF7FFFu; }
// Largest magnitude of a piece, as two packed 16-bit halves; amax_f32 joins the halves.
__device__ __forceinline__ uint32_t amax8(u32x4 r) { return max2(max2(mag2(r[0]), mag2(r[1])), max2(mag2(r[2]), mag2(r[3]))); }
__device__ __forceinline__ uint32_t amax_f32(uint32_t packed) { return max(packed & 0xFFFFu, packed >> 16) << 16; }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xF, 0xF, false));
}
constexpr int kRor8 = 0x128, kRor4 = 0x124, kRor2 = 0x122, kRor1 = 0x121;
__device__ __forceinline__ uint32_t max16_packed(uint32_t v) {       // over the 16 lanes of a DPP row
  v = max2(v, dpp<kRor8>(v));
  v = max2(v, dpp<kRor4>(v));
  v = max2(v, dpp<kRor2>(v));
  return max2(v, dpp<kRor1>(v));
}
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, dpp<kRor8>(v));
  v = max(v, dpp<kRor4>(v));
  v = max(v, dpp<kRor2>(v));
  return max(v, dpp<kRor1>(v));
}

}  // namespace f8
}  // namespace xs
