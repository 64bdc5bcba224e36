// Rounding of eight values to 8-bit codes of a scale.
#pragma once

#include "dev_rows.cuh"

namespace archead {
namespace rows {

// The integers nearest to v[i] / s (the exact quotient, halves to even; |v| <=
// about 127 s) as eight bytes, zeros where the row is not finite.
//
// With inv about 1 / s, v * inv + 1.5 * 2^23 (one rounding) ends in the integer q
// nearest to v / s or next to it, in two's complement.  r = v - q s is exact (a
// multiple of the smaller of the two operands' units, and at most about s / 2),
// so comparing 2 r with s (s / 2 is no fp32 number where s is an odd multiple of
// 2^-149) says which integer is nearest, and which way a half goes.
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float s, float inv, bool finite) {
  constexpr float kBig = 0x1.8p23f;
  float t[8], r[8], far = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    t[i] = fmaf(v[i], inv, kBig);
    r[i] = fmaf(kBig - t[i], s, v[i]);
    far = fmaxf(far, fabsf(r[i]));
  }
  if (__builtin_expect(far + far >= s, 0)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool odd = __float_as_uint(t[i]) & 1;
      const float twice = r[i] + r[i];
      if (twice > s || (twice == s && odd)) t[i] += 1.f;
      else if (twice < -s || (twice == -s && odd)) t[i] -= 1.f;
    }
  }
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {   // the low bytes of four
    auto low = [&](int k) { return __float_as_uint(t[4 * i + k]); };
    const uint32_t a = __builtin_amdgcn_perm(low(1), low(0), 0x0c0c0400), b = __builtin_amdgcn_perm(low(3), low(2), 0x0c0c0400);
    w[i] = finite ? a | b << 16 : 0u;
  }
  return uint2{w[0], w[1]};
}

// eight codes from j on to a row of d, at any address
__device__ __forceinline__ void store_codes(int8_t* out, int64_t j, int64_t d, const uint2& w) {
  if (j + 8 <= d) {
    store_any(out + j, w);
  } else {
    const uint32_t v[2] = {w.x, w.y};
    for (int i = 0; j + i < d; ++i) out[j + i] = int8_t(v[i / 4] >> (8 * (i % 4)));
  }
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {   // another lane of the row of 16
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xF, 0xF, false));
}
// neighbours at 1 and 2, then the mirrors: after four steps every lane of a row has all 16
constexpr int kDpp1 = 0xB1, kDpp2 = 0x4E, kDpp4 = 0x141, kDpp8 = 0x140;

}  // namespace rows
}  // namespace archead
