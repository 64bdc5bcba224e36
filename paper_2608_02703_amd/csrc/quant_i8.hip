// archead_quantize_i8: rows to int8 codes and one fp32 scale each.
#include "dev_rows.cuh"

namespace {

using namespace archead::rows;

constexpr int kQBlock = 256;
constexpr int kQHeld = 8;   // groups of 8 elements a thread keeps between its two passes

// TPR threads to a row (64: a wave each, 256: the workgroup).  One pass over
// the row for the largest magnitude, compared as integers (so a NaN or an
// infinity is the largest), and one for the codes; up to 64 TPR elements stay
// in registers in between, longer rows are read again (from the caches).
//
// With s the scale, q = rint(x * (1 / s)) is the nearest integer to x / s or
// next to it.  r = x - q s is exact (a multiple of the smaller of the two
// operands' units, and at most about s / 2), so comparing it with s / 2 (exact)
// says which integer is nearest, and which way a half goes.
template <int DT, int TPR>
__global__ __launch_bounds__(kQBlock) void k_quantize(const uint8_t* x, int64_t M, int64_t d, int64_t row_bytes,
                                                      int8_t* codes, int64_t ldc, float* scales) {
  using E = Eight<DT>;
  constexpr int kRows = kQBlock / TPR;
  __shared__ uint32_t smax[2][kQBlock / 64];
  const int tid = threadIdx.x, t = tid % TPR;
  int turn = 0;
  for (int64_t m0 = int64_t(blockIdx.x) * kRows; m0 < M; m0 += int64_t(gridDim.x) * kRows, turn ^= 1) {
    const int64_t m = m0 + tid / TPR;
    const bool live = m < M;   // (a wave's rows are its own: uniform)
    const uint8_t* row = x + m * row_bytes;
    const int64_t n = live ? d : 0;
    E held[kQHeld];
    uint32_t top = 0;
    auto larger = [&](const E& e) {
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(e.at(i)) & 0x7fffffffu);
    };
#pragma unroll
    for (int g = 0; g < kQHeld; ++g) {
      const int64_t j = (int64_t(g) * TPR + t) * 8;
      if (j < n) held[g].load(row, j, n, 0);
    }
#pragma unroll
    for (int g = 0; g < kQHeld; ++g)
      if ((int64_t(g) * TPR + t) * 8 < n) larger(held[g]);
    for (int64_t j = (int64_t(kQHeld) * TPR + t) * 8; j < n; j += TPR * 8) {
      E e;
      e.load(row, j, n, 0);
      larger(e);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, uint32_t(__shfl_xor(int(top), o, 64)));
    if constexpr (TPR > 64) {
      if ((tid & 63) == 0) smax[turn][tid >> 6] = top;
      __syncthreads();   // (the other of the two is read no more)
#pragma unroll
      for (int w = 0; w < kQBlock / 64; ++w) top = max(top, smax[turn][w]);
    }
    if (!live) continue;
    const bool finite = top < 0x7f800000u;
    const float s = finite ? fmaxf(__uint_as_float(top) / 127.f, 0x1p-126f) : NAN;
    const float inv = finite ? 1.f / s : 0.f, half = 0.5f * s;
    if (t == 0) scales[m] = s;
    int8_t* out = codes + m * ldc;
    auto write = [&](const E& e, int64_t j) {
      float q[8], r[8], far = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = finite ? e.at(i) : 0.f;
        q[i] = rintf(v * inv);
        r[i] = fmaf(-q[i], s, v);
        far = fmaxf(far, fabsf(r[i]));
      }
      if (__builtin_expect(far >= half, 0)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool odd = int(q[i]) & 1;
          if (r[i] > half || (r[i] == half && odd)) q[i] += 1.f;
          else if (r[i] < -half || (r[i] == -half && odd)) q[i] -= 1.f;
        }
      }
      uint32_t w[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i / 4] |= (uint32_t(int(q[i])) & 0xffu) << (8 * (i % 4));
      if (j + 8 <= d) {
        store_any(out + j, uint2{w[0], w[1]});
      } else {
        for (int i = 0; j + i < d; ++i) out[j + i] = int8_t(w[i / 4] >> (8 * (i % 4)));
      }
    };
#pragma unroll
    for (int g = 0; g < kQHeld; ++g) {
      const int64_t j = (int64_t(g) * TPR + t) * 8;
      if (j < d) write(held[g], j);
    }
    for (int64_t j = (int64_t(kQHeld) * TPR + t) * 8; j < d; j += TPR * 8) {
      E e;
      e.load(row, j, d, 0);
      write(e, j);
    }
  }
}

template <int DT>
void launch_quantize(const uint8_t* x, int64_t M, int64_t d, int64_t row_bytes, int8_t* codes, int64_t ldc,
                     float* scales, hipStream_t s) {
  const bool waves = d <= 64 * 8 * kQHeld && M >= 1024;
  const int64_t need = waves ? (M + 3) / 4 : M;
  const dim3 grid{unsigned(need < (1 << 22) ? need : 1 << 22)};
  if (waves) hipLaunchKernelGGL((k_quantize<DT, 64>), grid, dim3(kQBlock), 0, s, x, M, d, row_bytes, codes, ldc, scales);
  else hipLaunchKernelGGL((k_quantize<DT, 256>), grid, dim3(kQBlock), 0, s, x, M, d, row_bytes, codes, ldc, scales);
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
  if (x_dtype == ARCHEAD_F32) launch_quantize<ARCHEAD_F32>(xb, M, d, row_bytes, codes, ldc, scales, s);
  else if (x_dtype == ARCHEAD_BF16) launch_quantize<ARCHEAD_BF16>(xb, M, d, row_bytes, codes, ldc, scales, s);
  else launch_quantize<ARCHEAD_F16>(xb, M, d, row_bytes, codes, ldc, scales, s);
  return launch_status(hipGetLastError(), "quantize launch");
}
