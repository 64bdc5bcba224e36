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
// Bound by those loads' and their shifts' instructions: 4096 x 4096 x 4095 113 us (1.2
// POP/s; 4096 x 4096 x 4096 in tiles of aligned rows 63).
constexpr int kABlock = 256, kAK = 128, kARow = kAK + 16;   // (rows padded: no bank is hit twice as often)

template <int DT, int T>
__global__ __launch_bounds__(kABlock) void k_i8_any(I8Args g, int64_t m_tiles, int64_t tiles) {
  constexpr int F = T / 32, NP = T * 8 / kABlock;   // fragments of 16 rows a wave, pieces of 16 bytes a thread
  __shared__ __align__(16) int8_t la[2][T * kARow], lb[2][T * kARow];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, q = lane >> 4;
  const int wid = tid >> 6, wm = (wid & 1) * (T / 2), wn = (wid >> 1) * (T / 2);
  // workgroups go to the 8 XCDs in turn: a contiguous run of the tiles to each, so
  // that the tiles of the same channels find them in one L2 (1052 x 196069 x 126
  // 321 -> 263 us, 1696 x 67301 x 203 142 -> 124; 4000 x 9999 x 999 90 -> 95)
  const int64_t per_xcd = (tiles + 7) / 8, first = int64_t(blockIdx.x & 7) * per_xcd;
  const int64_t end = first + per_xcd < tiles ? first + per_xcd : tiles;
  for (int64_t t = first + (blockIdx.x >> 3); t < end; t += gridDim.x >> 3) {
    const int64_t m0 = t % m_tiles * T, n0 = t / m_tiles * T;
    uint4 wa[NP], wb[NP];
    auto piece = [&](int64_t r, int64_t rows, const int8_t* base, int64_t ld, int k) {
      return r < rows && k < g.K ? row_piece(base + r * ld, k, g.K) : uint4{0, 0, 0, 0};
    };
    auto fetch = [&](int k0) {
      const int k = k0 + tid % 8 * 16;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        wa[i] = piece(m0 + tid / 8 + 32 * i, g.M, g.a, g.lda, k);
        wb[i] = piece(n0 + tid / 8 + 32 * i, g.N, g.b, g.ldb, k);
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
    f32x4v sb[F], bi[F];
#pragma unroll
    for (int j = 0; j < F; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t n = n0 + wn + 16 * j + 4 * q + i, c = n < g.N ? n : g.N - 1;
        sb[j][i] = g.sb[c];
        bi[j][i] = g.bias ? g.bias[c] : 0.f;
      }
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
    // outputs: each wave turns 16 tokens at a time through its own part of the
    // LDS, so that neighbouring lanes store what lies together
    constexpr int EB = DT == ARCHEAD_F32 ? 4 : 2, OROW = T / 2 * EB + 16, LPR = T / 2 * EB / 16;   // lanes to a token
    static_assert(4 * 16 * OROW <= int(sizeof(la)), "the waves' parts fit");
    uint8_t* const buf = reinterpret_cast<uint8_t*>(&la[0][0]) + wid * 16 * OROW;
#pragma unroll
    for (int i = 0; i < F; ++i) {
      const int64_t m16 = m0 + wm + 16 * i;
      const float sa = g.sa[m16 + lr < g.M ? m16 + lr : g.M - 1];
#pragma unroll
      for (int j = 0; j < F; ++j) {
        float y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = scaled(acc[i][j][c], sa, sb[j][c], bi[j][c]);
        put4<DT>(buf + lr * OROW + (16 * j + 4 * q) * EB, y);
      }
      wave_lds_order();
#pragma unroll
      for (int r = lane / LPR; r < 16; r += 64 / LPR) {
        const int64_t m = m16 + r, n = n0 + wn + lane % LPR * (16 / EB);
        const uint4 v = *reinterpret_cast<const uint4*>(buf + r * OROW + lane % LPR * 16);
        if (m < g.M) store_part<EB>(g.out + (m * g.ldo + n) * EB, v, g.N - n);
      }
      wave_lds_order();
    }
  }
}

template <int DT, int T>
hipError_t launch_any(const I8Args& g, hipStream_t s) {
  const int64_t mt = (g.M + T - 1) / T, tiles = mt * ((g.N + T - 1) / T);
  const int64_t per_xcd = (tiles + 7) / 8;
  return launch_kernel(k_i8_any<DT, T>, dim3(unsigned(8 * (per_xcd < (1 << 19) ? per_xcd : 1 << 19))), dim3(kABlock), 0, s, g,
                       mt, tiles);
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

// A round of k_i8_split's tiles takes about as long to begin and end as this many
// k: us of it / tiles of 64 for 64 x 16384 x 256 9.1 / 7.1, 64 x 20000 x 128
// 10.8 / 7.1 (4 and 5 rounds).
constexpr int64_t kSplitStart = 1024;

// Rows of a and b that a CU loads with tiles of tm x tn: a round of tiles is
// bound by them, but for the tallest.
int64_t rows_loaded(const I8Args& g, int tm, int tn, int n_cu) {
  const int64_t tiles = (g.M + tm - 1) / tm * ((g.N + tn - 1) / tn);
  return (tiles + n_cu - 1) / n_cu * (tm + tn);
}

template <int DT>
hipError_t launch_matmul(const I8Args& g, hipStream_t s) {
  const int n_cu = compute_units();
  if (pieces(g)) {
    // Up to 16 tokens and above 4 units of channels to a CU, waves that stream
    // units rather than parts of them: us of split / few at K = 4096 for 1 x 8192
    // 7.5 / 9.3, 16 x 16384 13.5 / 16.1, 8 x 28672 24.1 / 23.1.  From 9 tokens on
    // the tiles' stores of 64 bytes and more of a token tell, where there is a
    // tile for every CU: us of few / tiles for M = 8 / 16 at N = 262144, K = 2560
    // 121 / 127 and 120 / 122.
    if (few_take(g) && (g.N + 15) / 16 > 4 * n_cu && (g.M <= 8 || (g.N + 255) / 256 < n_cu || !tiles_take(g)))
      return launch_few<DT>(g, n_cu, s);
    // Else the way that loads the fewest bytes a CU: us of split / tiles of 64 for
    // 64 x 8192 x 4096 10 / 19 (128 / 320 rows), 121 x 1325 x 8704 9 / 35 (64 / 320),
    // 256 x 4096 x 4096 18 / 19 (256 / 320), 64 x 28672 x 4096 48 / 32 (448 / 320);
    // of tiles of 64 / 128 / 192 / 256 for 64 x 151936 x 4096 127 / 140 / - / 167,
    // 333 x 50257 x 1536 63 / 53 / 48 / 51, 512 x 128256 x 8192 795 / 548 / 576 / 485.
    const int f = g.M <= 16 ? 1 : 2;
    int64_t best = split_take(g) ? rows_loaded(g, 16 * f, 16 * f, n_cu) * (g.K + kSplitStart) : INT64_MAX;
    int tm = 0;
    if (tiles_take(g))
      for (int t : {256, 192, 128, 64}) {
        const int64_t bytes = rows_loaded(g, t, 256, n_cu) * g.K;
        if (bytes < best) {
          best = bytes;
          tm = t;
        }
      }
    if (tm) return launch_tiles<DT>(g, tm, n_cu, s);
    if (best < INT64_MAX) return launch_split<DT>(g, f, s);
  }
  // K split over waves where there is not a tile for every CU: us of split / tiles
  // of 64 for 1 x 4096 x 4095 7.3 / 24, 120 x 1500 x 5001 12 / 36, 64 x 8192 x 2001
  // 11 / 17, 256 x 4096 x 4095 (256 tiles) 28 / 31, but 1 x 50000 x 1001 16 / 13,
  // 100 x 30000 x 1001 29 / 19.
  const auto tiles = [&](int t) { return (g.M + t - 1) / t * ((g.N + t - 1) / t); };
  if (g.K > 0 && tiles(64) <= n_cu) return launch_loose<DT>(g, g.M <= 16 ? 1 : 2, n_cu, s);
  // us with 128 / 64: 1172 x 43472 x 4229 440 / 721, 200 x 30000 x 1001 21 / 34,
  // 4096 x 4096 x 4095 113 / 197, 1696 x 67301 x 203 124 / 194, 3127 x 3460 x 141
  // 17 / 17, but 1000 x 20000 x 100 22 / 21.
  return tiles(128) >= 400 && g.K > kAK ? launch_any<DT, 128>(g, s) : launch_any<DT, 64>(g, s);
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
