// archead_matmul_i8 where there are few outputs: workgroups that split a tile's K.
#include "dev_common.cuh"
#include "i8.cuh"

namespace {

using namespace archead::i8;

constexpr int kSWaves = 8;
constexpr int kSK = 128;          // k of a stage
constexpr int kSRing = 2;         // stages of a wave

__device__ __forceinline__ void load16(__amdgpu_buffer_rsrc_t r, lds_u8* dst, uint32_t off, int k0) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, reinterpret_cast<__attribute__((address_space(3))) void*>(dst), 16, off, k0,
                                           0, 0);
}
template <int LEFT>   // until at most LEFT of this wave's loads are under way
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}

// A workgroup to a tile of 16 F tokens x 16 F channels, an eighth of K to each
// wave: where there are fewer tiles than CUs could hold, time goes with the
// length of a wave's share, and this is the shortest.  Each wave streams its
// stages through a ring of its own (direct global-to-LDS loads, 16-byte units
// swizzled against bank conflicts); the waves meet once, to add their int32
// sums, which is exact in any order.  8 x 4096 x 14336 bf16: 10.4 us (5.6 TB/s; in
// tiles of 64 x 256 53), 121 x 1325 x 8704 9.0 (35), 256 x 1024 x 8192 8.5 (33).
template <int DT, int F>
__global__ __launch_bounds__(kSWaves * 64) void k_i8_split(I8Args g, int m_tiles, int n_tiles) {
  constexpr int T = 16 * F, kBytes = T * kSK, kStage = 2 * kBytes, kLoads = kBytes / 1024;   // of an operand: bytes, loads
  extern __shared__ __align__(16) uint8_t i8_lds[];
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, q = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  // workgroups go to the 8 XCDs in turn: the tiles of the same channels to one
  const int group = int(blockIdx.x >> 3), nt = group / m_tiles * 8 + int(blockIdx.x & 7);
  if (nt >= n_tiles) return;
  const int64_t m0 = int64_t(group % m_tiles) * T, n0 = int64_t(nt) * T;
  const int stages = (g.K + kSK - 1) / kSK;
  const int s0 = stages * wid / kSWaves, count = stages * (wid + 1) / kSWaves - s0;
  // neighbouring tiles begin at different k, so that rows of a power of two do
  // not all ask for the same memory channels
  const int turn = nt * 5 % stages;

  lds_u8* const ring = (lds_u8*)i8_lds + wid * kSRing * kStage;
  const int rows_a = int(g.M - m0 < T ? g.M - m0 : T), rows_b = int(g.N - n0 < T ? g.N - n0 : T);
  const int lda = int(g.lda), ldb = int(g.ldb);
  __amdgpu_buffer_rsrc_t ra, rb;
  ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(g.a + m0 * g.lda), 0, (rows_a - 1) * lda + g.K, kBufferWord3);
  rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(g.b + n0 * g.ldb), 0, (rows_b - 1) * ldb + g.K, kBufferWord3);
  // load i: row 8 i + lane / 8, unit lane % 8 of LDS, holding unit (lane % 8) ^
  // (row % 8); rows past the last repeat it
  const int unit = 16 * ((lane & 7) ^ (lane >> 3));
  uint32_t ao[kLoads], bo[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int r = 8 * i + (lane >> 3);
    ao[i] = uint32_t(min(r, rows_a - 1)) * lda + unit;
    bo[i] = uint32_t(min(r, rows_b - 1)) * ldb + unit;
  }
  auto k_of = [&](int s) {   // where the share's stage s begins
    const int at = s0 + s + turn;
    return (at < stages ? at : at - stages) * kSK;
  };
  auto issue = [&](int s, int slot) {
    const int k0 = k_of(s);
    const uint32_t back = k0 + unit < g.K ? 0 : unit;   // (past K: the row's piece at k0 instead)
    lds_u8* const to = ring + slot * kStage;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      load16(ra, to + i * 1024, ao[i] - back, k0);
      load16(rb, to + kBytes + i * 1024, bo[i] - back, k0);
    }
  };
#pragma unroll
  for (int i = 0; i < kSRing; ++i)
    if (i < count) issue(i, i);

  i32x4 acc[F][F] = {};
  int slot = 0;
#pragma unroll 1
  for (int s = 0; s < count; ++s) {
    // this stage has landed: the loads after it are kSRing - 1 stages', or fewer
    if (s + kSRing <= count) wait_loads<(kSRing - 1) * 2 * kLoads>();
    else wait_loads<0>();
    const lds_u8* const at = ring + slot * kStage + lr * kSK;
    i32x4 fa[2][F], fb[2][F];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < F; ++i) {
        const int u = 16 * ((4 * kk + q) ^ (lr & 7)) + 16 * i * kSK;
        fa[kk][i] = lds_load<i32x4>(at + u);
        fb[kk][i] = lds_load<i32x4>(at + kBytes + u);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (s + kSRing < count) issue(s + kSRing, slot);
    __builtin_amdgcn_sched_barrier(0);
    const int left = g.K - k_of(s);
    if (left < kSK)   // K ends in this stage
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < F; ++i)
          if (64 * kk + 16 * q >= left) fa[kk][i] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[kk][j], fa[kk][i], acc[i][j], 0, 0, 0);
    slot = slot + 1 == kSRing ? 0 : slot + 1;
  }

  // ---- the waves' sums, fragment by fragment: F * F of them to add, a wave each
  constexpr int FF = F * F;
  i32x4* const sums = reinterpret_cast<i32x4*>(i8_lds);
  static_assert(FF <= kSWaves && kSWaves * FF * 1024 <= kSWaves * kSRing * kStage, "the sums fit, a wave to each");
  __syncthreads();   // (every wave has waited for all its loads)
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j) sums[(wid * FF + i * F + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  if (wid >= FF) return;
  i32x4 all = sums[wid * 64 + lane];
#pragma unroll
  for (int w = 1; w < kSWaves; ++w) {
    const i32x4 one = sums[(w * FF + wid) * 64 + lane];
#pragma unroll
    for (int i = 0; i < 4; ++i) all[i] += one[i];
  }
  finish4<DT>(g, m0 + wid / F * 16 + lr, n0 + wid % F * 16 + 4 * q, all);
}

template <int DT, int F>
hipError_t launch(const I8Args& g, hipStream_t s) {
  constexpr int T = 16 * F;
  const int m_tiles = int((g.M + T - 1) / T), n_tiles = int((g.N + T - 1) / T);
  return launch_kernel_lds(k_i8_split<DT, F>, dim3(unsigned((n_tiles + 7) / 8 * 8 * m_tiles)), dim3(kSWaves * 64),
                           size_t(kSWaves) * kSRing * 2 * T * kSK, s, g, m_tiles, n_tiles);
}

}  // namespace

namespace archead {
namespace i8 {

bool split_take(const I8Args& g) {
  return g.K > 0 && g.lda <= kMaxLd && g.ldb <= kMaxLd && (g.M + 15) / 16 * ((g.N + 15) / 16) < (1 << 18);
}

template <int DT>
hipError_t launch_split(const I8Args& g, int f, hipStream_t s) {
  return f == 1 ? launch<DT, 1>(g, s) : launch<DT, 2>(g, s);
}
template hipError_t launch_split<ARCHEAD_F32>(const I8Args&, int, hipStream_t);
template hipError_t launch_split<ARCHEAD_BF16>(const I8Args&, int, hipStream_t);
template hipError_t launch_split<ARCHEAD_F16>(const I8Args&, int, hipStream_t);

}  // namespace i8
}  // namespace archead
