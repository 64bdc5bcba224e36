// archead_matmul_i8: arguments of its kernels and their outputs.
//
// v_mfma_i32_16x16x64_i8 (32x32x32): lane l holds 16 consecutive k of row l % 16
// (l % 32) of an operand, from 16 (l / 16) (16 (l / 32)) on; of the result
// column l % 16 (l % 32) of the second operand, and of the first operand rows
// 4 (l / 16) + i (8 (i / 4) + 4 (l / 32) + i % 4).  The channels (b) go first, so
// a lane's results come as four neighbouring channels of one token.
#pragma once

#include "dev_rows.cuh"

namespace archead {
namespace i8 {

using namespace archead::rows;

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct I8Args {
  const int8_t* a;
  const int8_t* b;
  const float* sa;
  const float* sb;
  const float* bias;   // may be null
  uint8_t* out;
  int64_t lda, ldb, ldo;
  int64_t M, N;
  int K;
};

// four neighbouring outputs of a token
template <int DT>
__device__ __forceinline__ void store4(uint8_t* p, const float (&y)[4], int n) {
  if constexpr (DT == ARCHEAD_F32) {
    if (n == 4) {
      store_any(p, float4{y[0], y[1], y[2], y[3]});
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) reinterpret_cast<float*>(p)[i] = y[i];
  } else {
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == ARCHEAD_BF16) h[i] = bf16_rne(y[i]);
      else {
        const _Float16 f = _Float16(y[i]);
        __builtin_memcpy(&h[i], &f, 2);
      }
    }
    if (n == 4) {
      store_any(p, uint2{h[0] | uint32_t(h[1]) << 16, h[2] | uint32_t(h[3]) << 16});
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) reinterpret_cast<uint16_t*>(p)[i] = h[i];
  }
}

// the outputs of channels n .. n + 3 of token m
template <int DT>
__device__ __forceinline__ void finish4(const I8Args& g, int64_t m, int64_t n, const i32x4& acc) {
  if (m >= g.M || n >= g.N) return;
  const int cnt = g.N - n < 4 ? int(g.N - n) : 4;
  const float s = g.sa[m];
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t c = i < cnt ? n + i : n;
    y[i] = float(acc[i]) * s * g.sb[c];
    if (g.bias) y[i] += g.bias[c];
  }
  store4<DT>(g.out + (m * g.ldo + n) * (DT == ARCHEAD_F32 ? 4 : 2), y, cnt);
}


// kernel launchers, one translation unit each
template <int DT>
void launch_tiles(const I8Args& g, hipStream_t s);   // a, b aligned to 16, K, lda, ldb multiples of 16
bool tiles_take(const I8Args& g);

}  // namespace i8
}  // namespace archead
