// archead_matmul_i8: products of 8-bit integers with a scale per row of each
// operand.
#include <atomic>

#include "i8.cuh"

namespace {

using namespace archead::i8;

// ---------------------------------------------- any alignment, any K
// Tiles of 64 tokens x 64 channels, 128 of k at a time through registers into
// LDS, bytes past K as zeros.  Four waves of 32 x 32.
constexpr int kABlock = 256, kATile = 64, kAK = 128, kAStride = kAK + 16;

template <int DT>
__global__ __launch_bounds__(kABlock) void k_i8_any(I8Args g, int64_t m_tiles, int64_t tiles) {
  __shared__ __align__(16) int8_t lds[2][kATile * kAStride];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int wm = (wid & 1) * 32, wn = (wid >> 1) * 32;
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int64_t m0 = (t % m_tiles) * kATile, n0 = (t / m_tiles) * kATile;
    i32x4 acc[2][2] = {};
    for (int k0 = 0; k0 < g.K; k0 += kAK) {
      uint4 w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // two pieces of a's tile, two of b's
        const int piece = tid + (i & 1) * kABlock, row = piece / 8, k = k0 + (piece % 8) * 16;
        const int64_t r = (i < 2 ? m0 : n0) + row;
        const int8_t* p = i < 2 ? g.a + r * g.lda + k : g.b + r * g.ldb + k;
        w[i] = uint4{0, 0, 0, 0};
        if (r < (i < 2 ? g.M : g.N)) {
          if (k + 16 <= g.K) w[i] = load_any<uint4>(p);
          else {
            uint32_t d[4] = {};
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (k + j < g.K) d[j / 4] |= uint32_t(uint8_t(p[j])) << (8 * (j % 4));
            w[i] = uint4{d[0], d[1], d[2], d[3]};
          }
        }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int piece = tid + (i & 1) * kABlock;
        *reinterpret_cast<uint4*>(&lds[i / 2][(piece / 8) * kAStride + (piece % 8) * 16]) = w[i];
      }
      __syncthreads();
#pragma unroll
      for (int kk = 0; kk < kAK; kk += 64) {
        i32x4 fa[2], fb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int at = (lane & 15) * kAStride + kk + (lane >> 4) * 16;
          fa[i] = *reinterpret_cast<const i32x4*>(&lds[0][(wm + 16 * i) * kAStride + at]);
          fb[i] = *reinterpret_cast<const i32x4*>(&lds[1][(wn + 16 * i) * kAStride + at]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        finish4<DT>(g, m0 + wm + 16 * i + (lane & 15), n0 + wn + 16 * j + 4 * (lane >> 4), acc[i][j]);
  }
}

// compute units of the current device, asked for once
int compute_units() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  n = known[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) return 256;
    known[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

template <int DT>
hipError_t launch_matmul(const I8Args& g, hipStream_t s) {
  if (pieces(g)) {
    const int n_cu = compute_units();
    // From 9 tokens on the tiles' stores of 64 bytes and more of a token tell,
    // where there is a tile for every CU: us of the two M = 8 / 16 at N = 262144,
    // K = 2560 121 / 127 and 120 / 122; M = 8 at N = 16384, K = 4096 14 and 23.
    const bool few = few_take(g) && (g.M <= 8 || (g.N + 255) / 256 < n_cu || !tiles_take(g));
    if (few) return launch_few<DT>(g, n_cu, s);
    if (tiles_take(g)) return launch_tiles<DT>(g, n_cu, s);
  }
  const int64_t mt = (g.M + kATile - 1) / kATile, nt = (g.N + kATile - 1) / kATile, tiles = mt * nt;
  const dim3 grid{unsigned(tiles < (1 << 22) ? tiles : 1 << 22)};
  return launch_kernel(k_i8_any<DT>, grid, dim3(kABlock), 0, s, g, mt, tiles);
}

}  // namespace

extern "C" archead_status archead_matmul_i8(const int8_t* a, int64_t lda, const float* a_scales, const int8_t* b,
                                            int64_t ldb, const float* b_scales, const float* bias, int64_t M,
                                            int64_t N, int64_t K, void* out, archead_dtype out_dtype, int64_t ldo,
                                            void* stream) {
  using archead::fail;
  archead::clear_error();
  if (!float_dtype(out_dtype)) return fail(ARCHEAD_E_INVALID_ARG, "out_dtype must be F32, BF16 or F16");
  if (M < 0 || M > INT32_MAX || N < 0 || N > INT32_MAX || K < 0)
    return fail(ARCHEAD_E_INVALID_ARG, "M = %lld, N = %lld, K = %lld out of range", (long long)M, (long long)N,
                (long long)K);
  // 2^31 / 128^2: the largest sum of K products of codes stays below 2^31
  if (K > 131071) return fail(ARCHEAD_E_UNSUPPORTED, "K = %lld > 131071: the sum may pass 32 bits", (long long)K);
  if (M == 0 || N == 0) return ARCHEAD_OK;
  if (lda < K || ldb < K || ldo < N) return fail(ARCHEAD_E_INVALID_ARG, "leading dimensions must be >= K and N");
  if ((K && (!a || !b)) || !a_scales || !b_scales || !out) return fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if (!aligned(a_scales, 4) || !aligned(b_scales, 4) || !aligned(bias, 4) || !aligned(out, dtype_bytes(out_dtype)))
    return fail(ARCHEAD_E_MISALIGNED, "scales / bias / out misaligned");
  const I8Args g{a, b, a_scales, b_scales, bias, static_cast<uint8_t*>(out), lda, ldb, ldo, M, N, int(K)};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = out_dtype == ARCHEAD_F32    ? launch_matmul<ARCHEAD_F32>(g, s)
                       : out_dtype == ARCHEAD_BF16 ? launch_matmul<ARCHEAD_BF16>(g, s)
                                                   : launch_matmul<ARCHEAD_F16>(g, s);
  return launch_status(e, "int8 product launch");
}
