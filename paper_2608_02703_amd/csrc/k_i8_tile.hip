// archead_matmul_i8 for many tokens: tiles of TM tokens x 256 channels.
#include "dev_common.cuh"
#include "i8.cuh"

namespace {

using namespace archead::i8;

typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTK = 128;          // k of a stage
constexpr int kTileN = 256;       // channels of a tile
constexpr int kRaster = 8;        // token tiles of a raster group
constexpr int kMaxLd = 1 << 22;   // a tile's rows stay within 31-bit offsets

template <int TM, int WMW, int WNW>
struct Geom {
  static constexpr int NW = WMW * WNW;                     // waves
  static constexpr int WM = TM / WMW, WN = kTileN / WNW;   // a wave's tokens, channels
  static constexpr int MI = WM / 32, NI = WN / 32;
  static constexpr int ABYTES = TM * kTK, STAGE = ABYTES + kTileN * kTK;
  static constexpr int NA = ABYTES / 1024 / NW, NB = kTileN * kTK / 1024 / NW;   // loads of a wave and stage
  static constexpr int LDS = 2 * STAGE;
  static constexpr int OUT = WN + 4;                       // floats of a token in a wave's store buffer
  static_assert(NW * 32 * OUT * 4 <= LDS && LDS <= 160 * 1024, "LDS budget");
  static_assert(NA * 1024 * NW == ABYTES && NB * 1024 * NW == kTileN * kTK, "whole loads");
};

// Two stages of 128 k in LDS: one computed, one on its way.  Rows of 128 bytes
// with their 16-byte units swizzled, so eight rows' reads of one unit fall on
// eight different bank groups.  A wave reads the operands of a K-step (32 k)
// during the step before.  Before the last step of a stage all its reads are
// done, so there the waves meet, once a stage: the next stage has landed, its
// first operands are read and the loads of the one after it overwrite this
// one, all under the last step's products.
template <int DT, int TM, int WMW, int WNW>
__global__ __launch_bounds__(WMW* WNW * 64) __attribute__((amdgpu_waves_per_eu(2))) void k_i8_tile(
    I8Args g, int m_tiles, int n_tiles, int64_t per_xcd) {
  using G = Geom<TM, WMW, WNW>;
  constexpr int MI = G::MI, NI = G::NI;
  extern __shared__ __align__(16) uint8_t i8_lds[];
  lds_u8* const L = (lds_u8*)i8_lds;

  // workgroups go to the 8 XCDs in turn; each XCD takes a contiguous run of
  // the order that walks groups of kRaster token tiles along the channels
  const int64_t lin = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if (lin >= int64_t(m_tiles) * n_tiles) return;
  const int64_t gsz = int64_t(kRaster) * n_tiles, rg = lin / gsz;
  const int first = int(rg) * kRaster, gm = min(m_tiles - first, kRaster), within = int(lin - rg * gsz);
  const int64_t m0 = int64_t(first + within % gm) * TM, n0 = int64_t(within / gm) * kTileN;
  const int rows = int(g.M - m0 < TM ? g.M - m0 : TM), cols = int(g.N - n0 < kTileN ? g.N - n0 : kTileN);

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, h = lane >> 5;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wid / WNW, wn = wid % WNW;
  const int lda = int(g.lda), ldb = int(g.ldb);
  const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t*>(g.a + m0 * g.lda), 0, (rows - 1) * lda + g.K, kBufferWord3);
  const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t*>(g.b + n0 * g.ldb), 0, (cols - 1) * ldb + g.K, kBufferWord3);

  // this lane's unit of its wave's load i: row r, unit p of LDS, holding unit
  // p ^ swz of the row; rows past the last repeat it
  uint32_t ao[G::NA], bo[G::NB];
#pragma unroll
  for (int i = 0; i < G::NA; ++i) {
    const int off = (wid * G::NA + i) * 1024 + 16 * lane, r = off / kTK, p = off % kTK / 16;
    ao[i] = uint32_t(min(r, rows - 1)) * lda + 16 * (p ^ swz_x(r));
  }
#pragma unroll
  for (int i = 0; i < G::NB; ++i) {
    const int off = (wid * G::NB + i) * 1024 + 16 * lane, r = off / kTK, p = off % kTK / 16;
    bo[i] = uint32_t(min(r, cols - 1)) * ldb + 16 * (p ^ swz_x(r));
  }
  const int stages = (g.K + kTK - 1) / kTK;
  auto load = [&](__amdgpu_buffer_rsrc_t r, lds_u8* dst, uint32_t off, int k0) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, reinterpret_cast<__attribute__((address_space(3))) void*>(dst), 16, off,
                                             k0, 0, 0);
  };
  auto issue = [&](int s) {
    lds_u8* const base = L + (s & 1) * G::STAGE;
    const int k0 = s * kTK;
    if (__builtin_expect(k0 + kTK <= g.K, 1)) {
#pragma unroll
      for (int i = 0; i < G::NA; ++i) load(ra, base + (wid * G::NA + i) * 1024, ao[i], k0);
#pragma unroll
      for (int i = 0; i < G::NB; ++i) load(rb, base + G::ABYTES + (wid * G::NB + i) * 1024, bo[i], k0);
      return;
    }
    // the units past K: zeros in a; what is left of an earlier stage in b
#pragma unroll
    for (int i = 0; i < G::NA; ++i) {
      const int off = (wid * G::NA + i) * 1024 + 16 * lane, r = off / kTK, p = off % kTK / 16;
      if (k0 + 16 * (p ^ swz_x(r)) < g.K) load(ra, base + (wid * G::NA + i) * 1024, ao[i], k0);
      else *reinterpret_cast<__attribute__((address_space(3))) i32x4*>(base + off) = i32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < G::NB; ++i) {
      const int off = (wid * G::NB + i) * 1024 + 16 * lane, r = off / kTK, p = off % kTK / 16;
      if (k0 + 16 * (p ^ swz_x(r)) < g.K) load(rb, base + G::ABYTES + (wid * G::NB + i) * 1024, bo[i], k0);
    }
  };
  // operands of K-step ks: unit 2 ks + h of rows lr, lr + 32, ...
  uint32_t unit[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) unit[ks] = uint32_t(lr) * kTK + 16 * ((2 * ks + h) ^ swz_x(lr));
  auto read = [&](i32x4(&A)[MI], i32x4(&B)[NI], const lds_u8* base, int ks) {
#pragma unroll
    for (int i = 0; i < MI; ++i) A[i] = lds_load<i32x4>(base + unit[ks] + (wm * G::WM + 32 * i) * kTK);
#pragma unroll
    for (int i = 0; i < NI; ++i) B[i] = lds_load<i32x4>(base + G::ABYTES + unit[ks] + (wn * G::WN + 32 * i) * kTK);
  };
  i32x16 acc[MI][NI] = {};
  auto multiply = [&](const i32x4(&A)[MI], const i32x4(&B)[NI]) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(B[j], A[i], acc[i][j], 0, 0, 0);
  };

  if (stages > 0) {
    issue(0);
    if (stages > 1) issue(1);
    wait_loads_barrier<0>();
    i32x4 A[2][MI], B[2][NI];
    read(A[0], B[0], L, 0);
#pragma unroll 1
    for (int s = 0; s < stages; ++s) {
      const lds_u8* const base = L + (s & 1) * G::STAGE;
      read(A[1], B[1], base, 1);
      multiply(A[0], B[0]);
      read(A[0], B[0], base, 2);
      multiply(A[1], B[1]);
      read(A[1], B[1], base, 3);
      multiply(A[0], B[0]);
      wait_loads_barrier<0>();
      if (s + 2 < stages) issue(s + 2);
      if (s + 1 < stages) read(A[0], B[0], L + ((s + 1) & 1) * G::STAGE, 0);
      multiply(A[1], B[1]);
    }
  }
  __syncthreads();

  // Each wave turns 32 tokens at a time through its own part of the LDS: a
  // lane then holds the same channels of every token, and their scales.
  float* const buf = reinterpret_cast<float*>(i8_lds) + wid * 32 * G::OUT;
  constexpr int EB = DT == ARCHEAD_F32 ? 4 : 2, PER = 4, LPR = G::WN / PER;   // lanes to a token's channels
  const int cc = wn * G::WN + PER * (lane % LPR);
  float sb[PER], bi[PER];
  const int cnt = min(max(cols - cc, 0), PER);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    sb[i] = i < cnt ? g.sb[n0 + cc + i] : 0.f;
    bi[i] = g.bias && i < cnt ? g.bias[n0 + cc + i] : 0.f;
  }
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) {
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *reinterpret_cast<f32x4*>(buf + lr * G::OUT + 32 * ni + 8 * k + 4 * h) =
            f32x4{float(acc[mi][ni][4 * k]), float(acc[mi][ni][4 * k + 1]), float(acc[mi][ni][4 * k + 2]),
                  float(acc[mi][ni][4 * k + 3])};
    const int r0 = wm * G::WM + 32 * mi;
#pragma unroll
    for (int j = 0; j < 32 * LPR / 64; ++j) {
      const int rl = j * (64 / LPR) + lane / LPR;
      const f32x4 v = *reinterpret_cast<const f32x4*>(buf + rl * G::OUT + PER * (lane % LPR));
      if (r0 + rl >= rows || cnt == 0) continue;
      const float sa = g.sa[m0 + r0 + rl];
      float y[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        y[i] = v[i] * sa * sb[i];
        if (g.bias) y[i] += bi[i];
      }
      store4<DT>(g.out + ((m0 + r0 + rl) * g.ldo + n0 + cc) * EB, y, cnt);
    }
  }
}

template <int DT, int TM, int WMW, int WNW>
void launch(const I8Args& g, hipStream_t s) {
  using G = Geom<TM, WMW, WNW>;
  const int64_t mt = (g.M + TM - 1) / TM, nt = (g.N + kTileN - 1) / kTileN, per = (mt * nt + 7) / 8;
  const void* fn = reinterpret_cast<const void*>(k_i8_tile<DT, TM, WMW, WNW>);
  int m_tiles = int(mt), n_tiles = int(nt);
  int64_t per_xcd = per;
  void* args[] = {const_cast<I8Args*>(&g), &m_tiles, &n_tiles, &per_xcd};
  if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS) != hipSuccess) return;
  (void)hipLaunchKernel(fn, dim3(unsigned(8 * per)), dim3(G::NW * 64), args, G::LDS, s);
}

}  // namespace

namespace archead {
namespace i8 {

bool tiles_take(const I8Args& g) {
  const int64_t tiles = ((g.M + 255) / 256) * ((g.N + kTileN - 1) / kTileN);
  return aligned(g.a, 16) && aligned(g.b, 16) && g.K % 16 == 0 && g.lda % 16 == 0 && g.ldb % 16 == 0 && g.K > 0 &&
         g.lda <= kMaxLd && g.ldb <= kMaxLd && tiles < (1 << 22) && g.M > 64;
}

template <int DT>
void launch_tiles(const I8Args& g, hipStream_t s) {
  launch<DT, 256, 2, 4>(g, s);
}
template void launch_tiles<ARCHEAD_F32>(const I8Args&, hipStream_t);
template void launch_tiles<ARCHEAD_BF16>(const I8Args&, hipStream_t);
template void launch_tiles<ARCHEAD_F16>(const I8Args&, hipStream_t);

}  // namespace i8
}  // namespace archead
