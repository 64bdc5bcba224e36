// archead_matmul_i8 where there are few outputs and rows begin at any byte.
#include "i8.cuh"

namespace {

using namespace archead::i8;

constexpr int kLWaves = 8;

// Tiles of 16 F tokens x 16 F channels, K split over `share` waves of a workgroup
// (1, 2, 4 or 8; the others have tiles of their own), which add their int32 sums
// in LDS.  Rows at any byte do not go to LDS by themselves: a wave loads the next
// stage of its share into registers, 128 or 256 bytes of a row by neighbouring
// lanes, while it multiplies this one out of its own part of the LDS.  (Straight
// from memory to the products' registers, 64 bytes of a row: 11 us for 7.3, 32 for
// 12.5.)  1 x 4096 x 4095 7.3 us, 1 x 2000 x 16001 12.5 (2.6 TB/s).
template <int F>
struct Loose {
  static constexpr int T = 16 * F, K = F == 1 ? 256 : 128;     // rows of an operand, k of a stage
  static constexpr int LANES = K / 16, ROWS = 64 / LANES;      // of a load: lanes to a row, rows
  static constexpr int N = T / ROWS;                           // loads of an operand
  static constexpr int LROW = K + 16, WAVE = 2 * T * LROW;     // LDS bytes of a row (padded), of a wave
  static_assert(F * F * 1024 <= WAVE, "the sums fit");
};

template <int DT, int F>
__global__ __launch_bounds__(kLWaves * 64) void k_i8_loose(I8Args g, int64_t m_tiles, int64_t tiles, int64_t groups,
                                                           int share) {
  using G = Loose<F>;
  constexpr int T = G::T, FF = F * F;
  extern __shared__ __align__(16) uint8_t i8_lds[];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, q = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  // workgroups go to the 8 XCDs in turn: a contiguous run of the tiles to each
  const int64_t per_xcd = (groups + 7) / 8, wg = int64_t(blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if (int64_t(blockIdx.x >> 3) >= per_xcd || wg >= groups) return;
  const int64_t t = wg * (kLWaves / share) + wid / share;
  const bool live = t < tiles;
  const int part = wid % share;
  const int64_t m0 = (live ? t % m_tiles : 0) * T, n0 = (live ? t / m_tiles : 0) * T;
  const int stages = (g.K + G::K - 1) / G::K;
  const int s0 = int(int64_t(stages) * part / share);
  const int count = live ? int(int64_t(stages) * (part + 1) / share) - s0 : 0;
  const int row = lane / G::LANES, off = lane % G::LANES * 16;   // of a load: this lane's row and bytes
  const int rows_a = int(g.M - m0 < T ? g.M - m0 : T), rows_b = int(g.N - n0 < T ? g.N - n0 : T);
  uint8_t* const mine = i8_lds + wid * G::WAVE;
  uint4 wa[G::N], wb[G::N];
  auto fetch = [&](int s) {
    const int k = (s0 + s) * G::K + off;
    auto get = [&](uint4(&w)[G::N], const int8_t* base, int64_t ld, int rows) {
#pragma unroll
      for (int i = 0; i < G::N; ++i) {
        const int r = i * G::ROWS + row;
        w[i] = uint4{0, 0, 0, 0};
        if (r < rows && k < g.K) w[i] = row_piece(base + r * ld, k, g.K);
      }
    };
    get(wb, g.b + n0 * g.ldb, g.ldb, rows_b);
    get(wa, g.a + m0 * g.lda, g.lda, rows_a);
  };
  auto put = [&]() {
#pragma unroll
    for (int i = 0; i < G::N; ++i) {
      uint8_t* const to = mine + (i * G::ROWS + row) * G::LROW + off;
      *reinterpret_cast<uint4*>(to) = wa[i];
      *reinterpret_cast<uint4*>(to + T * G::LROW) = wb[i];
    }
  };
  i32x4 acc[F][F] = {};
  if (count > 0) fetch(0);
#pragma unroll 1
  for (int s = 0; s < count; ++s) {
    put();
    wave_lds_order();
    if (s + 1 < count) fetch(s + 1);
#pragma unroll
    for (int kk = 0; kk < G::K; kk += 64) {
      i32x4 fa[F], fb[F];
#pragma unroll
      for (int i = 0; i < F; ++i) {
        const uint8_t* const at = mine + (16 * i + lr) * G::LROW + kk + 16 * q;
        fa[i] = *reinterpret_cast<const i32x4*>(at);
        fb[i] = *reinterpret_cast<const i32x4*>(at + T * G::LROW);
      }
#pragma unroll
      for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
    wave_lds_order();
  }
  if (share == 1) {
    if (!live) return;
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
      for (int j = 0; j < F; ++j) finish4<DT>(g, m0 + 16 * i + lr, n0 + 16 * j + 4 * q, acc[i][j]);
    return;
  }
  auto sums = [&](int w) { return reinterpret_cast<i32x4*>(i8_lds + w * G::WAVE); };   // of a wave, in its own part
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j) sums(wid)[(i * F + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  if (!live) return;
  // the tile's fragments in turn to its waves
  for (int f = part; f < FF; f += share) {
    i32x4 all = sums(wid - part)[f * 64 + lane];
    for (int w = 1; w < share; ++w) {
      const i32x4 more = sums(wid - part + w)[f * 64 + lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) all[i] += more[i];
    }
    finish4<DT>(g, m0 + f / F * 16 + lr, n0 + f % F * 16 + 4 * q, all);
  }
}

template <int DT, int F>
hipError_t launch(const I8Args& g, int n_cu, hipStream_t s) {
  using G = Loose<F>;
  const int64_t m_tiles = (g.M + G::T - 1) / G::T, tiles = m_tiles * ((g.N + G::T - 1) / G::T);
  // no more waves to a tile than fill the CUs twice or have a stage each
  int share = 1;
  while (share < kLWaves && tiles * share < 2 * kLWaves * int64_t(n_cu) && 2 * share * G::K <= g.K) share *= 2;
  const int64_t groups = (tiles * share + kLWaves - 1) / kLWaves;
  return launch_kernel_lds(k_i8_loose<DT, F>, dim3(unsigned((groups + 7) / 8 * 8)), dim3(kLWaves * 64), kLWaves * G::WAVE, s, g,
                           m_tiles, tiles, groups, share);
}

}  // namespace

namespace archead {
namespace i8 {

template <int DT>
hipError_t launch_loose(const I8Args& g, int f, int n_cu, hipStream_t s) {
  return f == 1 ? launch<DT, 1>(g, n_cu, s) : launch<DT, 2>(g, n_cu, s);
}
template hipError_t launch_loose<ARCHEAD_F32>(const I8Args&, int, int, hipStream_t);
template hipError_t launch_loose<ARCHEAD_BF16>(const I8Args&, int, int, hipStream_t);
template hipError_t launch_loose<ARCHEAD_F16>(const I8Args&, int, int, hipStream_t);

}  // namespace i8
}  // namespace archead
