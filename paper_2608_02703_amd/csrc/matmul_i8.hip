// archead_matmul_i8: products of 8-bit integers with a scale per row of each
// operand.
#include <atomic>

#include "i8.cuh"

namespace {

using namespace archead::i8;

// ---------------------------------------------- any alignment, any K
// Tiles of T tokens x T channels, 128 k a stage, bytes past K as zeros, four
// waves of T/2 x T/2.  Rows that begin at any byte cannot be loaded to LDS
// directly: each thread loads its pieces of the next stage into registers while
// the waves multiply this one, and puts them into the other half of LDS after.
constexpr int kABlock = 256, kAK = 128, kARow = kAK + 16;   // (rows padded: no bank is hit twice as often)

template <int DT, int T>
__global__ __launch_bounds__(kABlock) void k_i8_any(I8Args g, int64_t m_tiles, int64_t tiles) {
  constexpr int F = T / 32, NP = T * 8 / kABlock;   // fragments of 16 rows a wave, pieces of 16 bytes a thread
  __shared__ __align__(16) int8_t la[2][T * kARow], lb[2][T * kARow];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, q = lane >> 4;
  const int wid = tid >> 6, wm = (wid & 1) * (T / 2), wn = (wid >> 1) * (T / 2);
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int64_t m0 = t % m_tiles * T, n0 = t / m_tiles * T;
    uint4 wa[NP], wb[NP];
    auto piece = [&](const int8_t* base, int64_t r, int64_t rows, int64_t ld, int k) {
      uint4 w{0, 0, 0, 0};
      if (r >= rows || k >= g.K) return w;
      const int8_t* const row = base + r * ld;
      if (__builtin_expect(g.K < 16, 0)) {
        uint32_t d[4] = {};
        for (int j = 0; j < g.K; ++j) d[j / 4] |= uint32_t(uint8_t(row[j])) << (8 * (j % 4));
        return uint4{d[0], d[1], d[2], d[3]};
      }
      // the row's last 16 bytes, moved down, where fewer are left
      const int over = max(k + 16 - g.K, 0);
      w = load_any<uint4>(row + k - over);
      if (over) {
        uint64_t lo = uint64_t(w.y) << 32 | w.x, hi = uint64_t(w.w) << 32 | w.z;
        const int bits = 8 * over;
        lo = bits < 64 ? lo >> bits | hi << (64 - bits) : hi >> (bits - 64);
        hi = bits < 64 ? hi >> bits : 0;
        w = uint4{uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32)};
      }
      return w;
    };
    auto fetch = [&](int k0) {
      const int k = k0 + tid % 8 * 16;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        wa[i] = piece(g.a, m0 + tid / 8 + 32 * i, g.M, g.lda, k);
        wb[i] = piece(g.b, n0 + tid / 8 + 32 * i, g.N, g.ldb, k);
      }
    };
    auto put = [&](int half) {
      const int at = tid / 8 * kARow + tid % 8 * 16;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        *reinterpret_cast<uint4*>(&la[half][at + 32 * i * kARow]) = wa[i];
        *reinterpret_cast<uint4*>(&lb[half][at + 32 * i * kARow]) = wb[i];
      }
    };
    i32x4 acc[F][F] = {};
    fetch(0);
    __syncthreads();   // the tile before this one has been read
    put(0);
    __syncthreads();
    int half = 0;
    for (int k0 = 0; k0 < g.K; k0 += kAK, half ^= 1) {
      const bool more = k0 + kAK < g.K;
      if (more) fetch(k0 + kAK);
#pragma unroll
      for (int kk = 0; kk < kAK; kk += 64) {
        i32x4 fa[F], fb[F];
        const int at = lr * kARow + kk + 16 * q;
#pragma unroll
        for (int i = 0; i < F; ++i) {
          fa[i] = *reinterpret_cast<const i32x4*>(&la[half][(wm + 16 * i) * kARow + at]);
          fb[i] = *reinterpret_cast<const i32x4*>(&lb[half][(wn + 16 * i) * kARow + at]);
        }
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
          for (int j = 0; j < F; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
      }
      if (more) put(half ^ 1);   // (read last in the stage before, behind a meeting)
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
      for (int j = 0; j < F; ++j) finish4<DT>(g, m0 + wm + 16 * i + lr, n0 + wn + 16 * j + 4 * q, acc[i][j]);
  }
}

template <int DT, int T>
hipError_t launch_any(const I8Args& g, hipStream_t s) {
  const int64_t mt = (g.M + T - 1) / T, tiles = mt * ((g.N + T - 1) / T);
  return launch_kernel(k_i8_any<DT, T>, dim3(unsigned(tiles < (1 << 22) ? tiles : 1 << 22)), dim3(kABlock), 0, s, g, mt,
                       tiles);
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
  // us with 128 / 64: 1172 x 43472 x 4229 451 / 727, 200 x 30000 x 1001 25 / 36,
  // 4096 x 4096 x 4095 116 / 203, but 3127 x 3460 x 141 25 / 21.
  const int64_t large = ((g.M + 127) / 128) * ((g.N + 127) / 128);
  return large >= 400 && g.K > 2 * kAK ? launch_any<DT, 128>(g, s) : launch_any<DT, 64>(g, s);
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
