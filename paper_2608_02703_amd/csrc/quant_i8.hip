// archead_quantize_i8: rows to int8 codes and one fp32 scale each.
#include "dev_rows.cuh"

namespace {

using namespace archead::rows;

constexpr int kQMost = 1024;     // threads of a workgroup
constexpr int kQShort = 512;     // longest row that 16 lanes take

// SHORT: 16 lanes to a row, four rows to a wave; else a workgroup to a row, as
// many threads as hold it in HELD groups of 8 elements each.  One pass over the row for the
// largest magnitude, compared as integers (so a NaN or an infinity is the
// largest), and one for the codes; what a thread holds stays in registers in
// between, longer rows are read again (from the caches).  151936 x 4096 bf16:
// 312 us (6.0 TB/s); a wave to a row, eight groups a lane: 443.
//
// With s the scale, x * (1 / s) + 1.5 * 2^23 (one rounding) ends in the integer
// q nearest to x / s or next to it, in two's complement.  r = x - q s is exact (a
// multiple of the smaller of the two operands' units, and at most about s / 2),
// so comparing 2 r with s (s / 2 is no fp32 number where s is an odd multiple of
// 2^-149) says which integer is nearest, and which way a half goes.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {   // another lane of the row of 16
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xF, 0xF, false));
}

template <int DT, bool SHORT, int HELD>
__global__ __launch_bounds__(SHORT ? 256 : kQMost) void k_quantize(const uint8_t* x, int64_t M, int64_t d, int64_t row_bytes,
                                                      int8_t* codes, int64_t ldc, float* scales) {
  using E = Eight<DT>;
  static_assert(!SHORT || HELD * 128 == kQShort, "a short row is held whole");
  const int TPR = SHORT ? 16 : int(blockDim.x), rows = SHORT ? int(blockDim.x) / 16 : 1;
  __shared__ uint32_t smax[2][kQMost / 64];
  const int tid = threadIdx.x, t = SHORT ? tid & 15 : tid;
  int turn = 0;
  for (int64_t m0 = int64_t(blockIdx.x) * rows; m0 < M; m0 += int64_t(gridDim.x) * rows, turn ^= 1) {
    const int64_t m = SHORT ? m0 + (tid >> 4) : m0;
    const bool live = m < M;
    const uint8_t* row = x + m * row_bytes;
    const int64_t n = live ? d : 0;
    E held[HELD];
    uint32_t top = 0;
    auto larger = [&](const E& e) {
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(e.at(i)) & 0x7fffffffu);
    };
#pragma unroll
    for (int g = 0; g < HELD; ++g) {
      const int64_t j = (int64_t(g) * TPR + t) * 8;
      if (j < n) held[g].load(row, j, n, 0);
    }
#pragma unroll
    for (int g = 0; g < HELD; ++g)
      if ((int64_t(g) * TPR + t) * 8 < n) larger(held[g]);
    for (int64_t j = (int64_t(HELD) * TPR + t) * 8; j < n; j += TPR * 8) {
      E e;
      e.load(row, j, n, 0);
      larger(e);
    }
    top = max(top, dpp<0xB1>(top));
    top = max(top, dpp<0x4E>(top));
    top = max(top, dpp<0x141>(top));
    top = max(top, dpp<0x140>(top));
    if constexpr (!SHORT) {
      auto of = [&](int l) { return uint32_t(__builtin_amdgcn_readlane(int(top), l)); };
      top = max(max(of(0), of(16)), max(of(32), of(48)));
    }
    if (!SHORT && TPR > 64) {
      if ((tid & 63) == 0) smax[turn][tid >> 6] = top;
      __syncthreads();   // (the other of the two is read no more)
      for (int w = 0; w < TPR / 64; ++w) top = max(top, smax[turn][w]);
    }
    if (!live) continue;
    const bool finite = top < 0x7f800000u;
    const float s = finite ? fmaxf(__uint_as_float(top) / 127.f, 0x1p-126f) : NAN;
    const float inv = finite ? 1.f / s : 0.f;
    if (t == 0) scales[m] = s;
    int8_t* out = codes + m * ldc;
    constexpr float kBig = 0x1.8p23f;
    auto write = [&](const E& e, int64_t j) {
      float t[8], r[8], far = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = e.at(i);
        t[i] = fmaf(v, inv, kBig);
        r[i] = fmaf(kBig - t[i], s, v);
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
      if (j + 8 <= d) {
        store_any(out + j, uint2{w[0], w[1]});
      } else {
        for (int i = 0; j + i < d; ++i) out[j + i] = int8_t(w[i / 4] >> (8 * (i % 4)));
      }
    };
#pragma unroll
    for (int g = 0; g < HELD; ++g) {
      const int64_t j = (int64_t(g) * TPR + t) * 8;
      if (j < d) write(held[g], j);
    }
    for (int64_t j = (int64_t(HELD) * TPR + t) * 8; j < d; j += TPR * 8) {
      E e;
      e.load(row, j, d, 0);
      write(e, j);
    }
  }
}

template <int DT, bool SHORT, int HELD>
hipError_t launch_rows(const uint8_t* x, int64_t M, int64_t d, int64_t row_bytes, int8_t* codes, int64_t ldc, float* scales,
                 hipStream_t s) {
  const int64_t groups = SHORT ? (M + 15) / 16 : M, waves = SHORT ? 4 : (d + 512 * HELD - 1) / (512 * HELD);
  const int64_t most = kQMost / 64;
  return launch_kernel(k_quantize<DT, SHORT, HELD>, dim3(unsigned(groups < (1 << 21) ? groups : 1 << 21)),
                       dim3(unsigned(64 * (waves < most ? waves : most))), 0, s, x, M, d, row_bytes, codes, ldc, scales);
}
template <int DT>
hipError_t launch_quantize(const uint8_t* x, int64_t M, int64_t d, int64_t row_bytes, int8_t* codes, int64_t ldc,
                     float* scales, hipStream_t s) {
  // Fewer waves with more in flight each where there are plenty: us with 2 / 4
  // groups 151936 x 4096 336 / 312, 16384 x 8192 88 / 74, 14709 x 4128 45 / 38,
  // 8192 x 4096 20.5 / 21.7, 4096 x 4096 12.2 / 13.1, 300 x 4096 4.5 / 5.8.
  if (d <= kQShort) return launch_rows<DT, true, 4>(x, M, d, row_bytes, codes, ldc, scales, s);
  if (M * d < (1 << 25)) return launch_rows<DT, false, 2>(x, M, d, row_bytes, codes, ldc, scales, s);
  return launch_rows<DT, false, 4>(x, M, d, row_bytes, codes, ldc, scales, s);
}

}  // namespace

extern "C" archead_status archead_quantize_i8(const void* x, archead_dtype x_dtype, int64_t M, int64_t d,
                                              int64_t ldx, int8_t* codes, int64_t ldc, float* scales,
                                              void* stream) {
  using archead::fail;
  archead::clear_error();
  if (!float_dtype(x_dtype)) return fail(ARCHEAD_E_INVALID_ARG, "x_dtype must be F32, BF16 or F16");
  if (M < 0 || M > INT32_MAX) return fail(ARCHEAD_E_INVALID_ARG, "M = %lld out of range", (long long)M);
  if (d < 1 || d > INT32_MAX) return fail(ARCHEAD_E_INVALID_ARG, "d = %lld out of range", (long long)d);
  if (M == 0) return ARCHEAD_OK;
  if (ldx < d || ldc < d) return fail(ARCHEAD_E_INVALID_ARG, "leading dimensions must be >= d");
  if (!x || !codes || !scales) return fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if (!aligned(x, dtype_bytes(x_dtype)) || !aligned(scales, 4))
    return fail(ARCHEAD_E_MISALIGNED, "x / scales misaligned");
  const uint8_t* xb = static_cast<const uint8_t*>(x);
  const int64_t row_bytes = ldx * dtype_bytes(x_dtype);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = x_dtype == ARCHEAD_F32    ? launch_quantize<ARCHEAD_F32>(xb, M, d, row_bytes, codes, ldc, scales, s)
                       : x_dtype == ARCHEAD_BF16 ? launch_quantize<ARCHEAD_BF16>(xb, M, d, row_bytes, codes, ldc, scales, s)
                                                 : launch_quantize<ARCHEAD_F16>(xb, M, d, row_bytes, codes, ldc, scales, s);
  return launch_status(e, "quantize launch");
}
