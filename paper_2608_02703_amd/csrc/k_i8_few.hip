// archead_matmul_i8 for up to 16 tokens: b is read once, by waves that work
// apart from each other.
#include "dev_common.cuh"
#include "i8.cuh"

namespace {

using namespace archead::i8;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kFWaves = 8;
constexpr int kFK = 256;                      // k of a stage
constexpr int kFRows = 16;                    // channels of a unit
constexpr int kFStage = kFRows * kFK;         // bytes of a wave's stage
constexpr int kFLoads = kFStage / 1024;       // loads of a stage
constexpr int kFLds = 160 * 1024;
// LDS of a wave: a ring of NS stages, and the scales and bias of the units that
// they may belong to (a load of 64 lanes x 4 bytes writes 256)
constexpr int scale_slots(int ns) { return ns + 1; }
constexpr int wave_lds(int ns) { return ns * kFStage + scale_slots(ns) * 256; }
__host__ __device__ constexpr int64_t a_row(int64_t K) { return (K + kFK - 1) / kFK * kFK + 16; }   // bytes of a row of a in LDS

// Every wave has a contiguous range of units of 16 channels and streams their
// rows through a ring of its own in LDS (direct global-to-LDS loads of 256
// contiguous bytes of a row), so no wave waits for another and 64 KB and more
// are in flight per CU.  a lies in LDS whole, zeros behind K (what a stage
// holds of b there does not matter), rows 16 bytes apart modulo 128 so that
// the rows' reads of one unit fall on different banks; the ring's 16-byte units
// are swizzled for the same.  Tokens past M repeat the last.  Bound by b's bytes:
// 1 x 151936 x 4096 in 109 us, 5.7 TB/s.
template <int DT, int NS>
__global__ __launch_bounds__(kFWaves * 64) void k_i8_few(I8Args g, int64_t units) {
  constexpr int kFWave = wave_lds(NS), kFRing = NS, kFScaleSlots = scale_slots(NS);
  extern __shared__ __align__(16) uint8_t i8_lds[];
  lds_u8* const L = (lds_u8*)i8_lds;
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, q = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int M = int(g.M), ar = int(a_row(g.K));
  lds_u8* const A = L + kFWaves * kFWave;
  for (int i = tid; i < M * (ar / 16); i += kFWaves * 64) {
    const int m = i / (ar / 16), u = i - m * (ar / 16);
    u32x4 v{0, 0, 0, 0};
    if (16 * u < g.K) v = *reinterpret_cast<const u32x4*>(g.a + m * g.lda + 16 * u);
    *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(A + m * ar + 16 * u) = v;
  }
  __syncthreads();

  // the workgroup's units in turn: what its waves write lies side by side at
  // about the same time
  const int64_t u0 = units * blockIdx.x / gridDim.x + wid, u1 = units * (blockIdx.x + 1) / gridDim.x;
  if (u0 >= u1) return;
  const int stages = (g.K + kFK - 1) / kFK;
  const int64_t total = (u1 - u0 + kFWaves - 1) / kFWaves * stages;
  // neighbouring waves begin at different k (the sum is exact in any order), so
  // that rows of a power of two do not all ask for the same memory channels
  const int k_first = int((u0 * 5) % stages);
  lds_u8* const ring = L + wid * kFWave;
  lds_u8* const scales = ring + kFRing * kFStage;

  // ---- loads
  int64_t l_unit = u0, l_done = 0;
  int l_stage = 0, l_slot = 0, l_sslot = 0;
  __amdgpu_buffer_rsrc_t rb;
  uint32_t bo[kFLoads];
  const int ldb = int(g.ldb);
  auto begin_unit = [&]() {
    const int64_t n0 = l_unit * kFRows;
    const int rows = int(g.N - n0 < kFRows ? g.N - n0 : kFRows);
    rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(g.b + n0 * g.ldb), 0, (rows - 1) * ldb + g.K,
                                           kBufferWord3);
#pragma unroll
    for (int i = 0; i < kFLoads; ++i) {   // row 4 i + q, unit lr of LDS, holding unit lr ^ row
      const int r = 4 * i + q;
      bo[i] = uint32_t(min(r, rows - 1)) * ldb + 16 * (lr ^ r);
    }
    // lanes 0-15 the scales, 16-31 the bias (the others the same again)
    const float* const from = (q & 1 && g.bias ? g.bias : g.sb) + n0 + min(lr, rows - 1);
    __builtin_amdgcn_global_load_lds(
        reinterpret_cast<const __attribute__((address_space(1))) void*>(reinterpret_cast<uintptr_t>(from)),
        reinterpret_cast<__attribute__((address_space(3))) void*>(scales + l_sslot * 256), 4, 0, 0);
    l_sslot = l_sslot + 1 == kFScaleSlots ? 0 : l_sslot + 1;
  };
  auto issue = [&]() {
    if (l_stage == 0) begin_unit();
    const int ks = l_stage + k_first, k0 = (ks < stages ? ks : ks - stages) * kFK;
    lds_u8* const to = ring + l_slot * kFStage;
#pragma unroll
    for (int i = 0; i < kFLoads; ++i) {
      uint32_t off = bo[i];
      if (k0 + kFK > g.K && k0 + 16 * (lr ^ (4 * i + q)) >= g.K) off -= 16 * (lr ^ (4 * i + q));   // the row's first bytes instead
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rb, reinterpret_cast<__attribute__((address_space(3))) void*>(to + i * 1024), 16, off,
          k0, 0, 0);
    }
    l_slot = l_slot + 1 == kFRing ? 0 : l_slot + 1;
    ++l_done;
    if (++l_stage == stages) {
      l_stage = 0;
      l_unit += kFWaves;
    }
  };
#pragma unroll
  for (int i = 0; i < kFRing; ++i)
    if (i < total) issue();

  // ---- products
  const int token = min(lr, M - 1);
  const float sa = g.sa[token];
  const lds_u8* const arow = A + token * ar + 16 * q;
  int slot = 0, sslot = 0;
  int64_t done = 0;
  for (int64_t u = u0; u < u1; u += kFWaves) {
    i32x4 acc = {0, 0, 0, 0};
#pragma unroll 1
    for (int s = 0; s < stages; ++s, ++done) {
      // this stage has landed: of the loads after it at most kFRing - 1 stages' are there
      if (done + kFRing <= total) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kFRing - 1) * kFLoads) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const int ks = s + k_first, k0 = (ks < stages ? ks : ks - stages) * kFK;
      const lds_u8* const at = ring + slot * kFStage + lr * kFK;
      i32x4 fb[4], fa[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        fb[i] = lds_load<i32x4>(at + 16 * ((4 * i + q) ^ lr));
        fa[i] = lds_load<i32x4>(arow + k0 + 64 * i);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      if (l_done < total) issue();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[i], fa[i], acc, 0, 0, 0);
      slot = slot + 1 == kFRing ? 0 : slot + 1;
    }
    // channels 16 u + 4 q .. + 3 of token lr
    const lds_u8* const sc = scales + sslot * 256 + 16 * q;
    const f32x4v sb = lds_load<f32x4v>(sc), bi = lds_load<f32x4v>(sc + 64);
    sslot = sslot + 1 == kFScaleSlots ? 0 : sslot + 1;
    const int64_t n = u * kFRows + 4 * q;
    if (lr < M && n < g.N) {
      constexpr int EB = DT == ARCHEAD_F32 ? 4 : 2;
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = scaled(acc[i], sa, sb[i], g.bias ? bi[i] : 0.f);
      __align__(16) uint32_t w[EB];
      put4<DT>(reinterpret_cast<uint8_t*>(w), y);
      if constexpr (EB == 4) store_part<EB>(g.out + (lr * g.ldo + n) * EB, u32x4{w[0], w[1], w[2], w[3]}, g.N - n);
      else store_part<EB>(g.out + (lr * g.ldo + n) * EB, uint2{w[0], w[1]}, g.N - n);
    }
  }
}

}  // namespace

namespace archead {
namespace i8 {

bool few_take(const I8Args& g) {
  return g.M <= 16 && g.K > 0 && g.ldb <= kMaxLd && g.M * a_row(g.K) + kFWaves * wave_lds(2) <= kFLds;
}

namespace {
template <int DT, int NS>
hipError_t launch_as(const I8Args& g, int n_cu, hipStream_t s) {
  const int64_t units = (g.N + kFRows - 1) / kFRows, need = (units + kFWaves - 1) / kFWaves;
  return launch_kernel_lds(k_i8_few<DT, NS>, dim3(unsigned(need < n_cu ? need : n_cu)), dim3(kFWaves * 64),
                           size_t(g.M * a_row(g.K)) + kFWaves * wave_lds(NS), s, g, units);
}
}  // namespace

template <int DT>
hipError_t launch_few(const I8Args& g, int n_cu, hipStream_t s) {
  // three stages a wave where a leaves them room
  if (g.M * a_row(g.K) + kFWaves * wave_lds(3) <= kFLds) return launch_as<DT, 3>(g, n_cu, s);
  return launch_as<DT, 2>(g, n_cu, s);
}
template hipError_t launch_few<ARCHEAD_F32>(const I8Args&, int, hipStream_t);
template hipError_t launch_few<ARCHEAD_BF16>(const I8Args&, int, hipStream_t);
template hipError_t launch_few<ARCHEAD_F16>(const I8Args&, int, hipStream_t);

}  // namespace i8
}  // namespace archead
