// archead_matmul_i8 for several tokens: tiles of TM tokens x 256 channels.
#include "dev_common.cuh"
#include "i8.cuh"

namespace {

using namespace archead::i8;

typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTK = 128;          // k of a stage
constexpr int kTileN = 256;       // channels of a tile
constexpr int64_t kTurnMost = 2 << 20;   // bytes of a up to which tiles begin at different k
constexpr int kRaster = 8;        // token tiles of a raster group

// NSA stages of a and NSB of b in LDS, WMW x WNW waves
template <int TM, int WMW, int WNW, int NSA, int NSB>
struct Geom {
  static constexpr int NW = WMW * WNW;
  static constexpr int WM = TM / WMW, WN = kTileN / WNW;   // a wave's tokens, channels
  static constexpr int MI = WM / 32, NI = WN / 32;
  static constexpr int ABYTES = TM * kTK, BBYTES = kTileN * kTK, BAT = NSA * ABYTES;   // a stage of each; b's ring
  static constexpr int NA = ABYTES / 1024 / NW, NB = BBYTES / 1024 / NW;   // loads of a wave and stage
  static constexpr int NSC = TM + 2 * kTileN;
  // a wave's store buffer: 16 tokens of 128 bytes, or 64 where that is too much, padded
  static constexpr int OUT = BAT + NSB * BBYTES;
  static constexpr int OBYTES = OUT + NW * 16 * (128 + 16) + 2 * NSC * 4 <= 160 * 1024 ? 128 : 64, OROW = OBYTES + 16;
  static constexpr int SCALES = OUT + NW * 16 * OROW;      // fp32 [2][TM + 2 kTileN]: a_scales, b_scales, bias
  static constexpr int LDS = SCALES + 2 * NSC * 4;
  static_assert(LDS <= 160 * 1024, "LDS budget");
  static_assert(NA * 1024 * NW == ABYTES && NB * 1024 * NW == BBYTES, "whole loads");
};

// The order of a K-step of P products: after each of the first ones a share of
// R LDS reads, one or two, and of V loads to LDS.  Without it the compiler puts
// the next step's reads right before their use.
template <int R, int V, int P, int I = 0>
__device__ __forceinline__ void spread() {
  if constexpr (I < P) {
    constexpr int H = P * 3 / 4 > 0 ? P * 3 / 4 : 1;
    constexpr int r = I < H ? R * (I + 1) / H - R * I / H : 0, v = V * (I + 1) / P - V * I / P;
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);   // products
    if constexpr (r > 0) __builtin_amdgcn_sched_group_barrier(0x100, r, 0);
    if constexpr (v > 0) __builtin_amdgcn_sched_group_barrier(0x10, v, 0);
    spread<R, V, P, I + 1>();
  } else {
    __builtin_amdgcn_sched_barrier(0);
  }
}

// A persistent workgroup per CU takes its XCD's tiles in turn, their stages as
// one sequence: the loads run NSA (of a) and NSB (of b) stages ahead of the
// products, across tiles, so the next tile's first stages are on their way while
// one tile is written.  b comes from HBM where a single row of tiles covers the
// tokens, a from the L2: where LDS has room for one stage more it is b's.
//
// LDS rows of 128 bytes have their 16-byte units swizzled, so eight rows' reads
// of one unit fall on eight different bank groups.  A wave reads the operands
// of a K-step (32 k) during the step before.  Before the last step of a stage
// all its reads are done, so there the waves meet, once a stage: the next stage
// has landed, its first operands are read and later loads overwrite this one,
// all under the last step's products.
//
// 4096 x 151936 x 4096: 2.20 to 2.30 ms, 2.2 to 2.3 POP/s; the matrix units are busy 63 %
// of the time at the 1.5 GHz that the power limit leaves.  64 x 151936 x 4096: 127 us,
// 5.1 TB/s of b and the outputs.
template <int DT, int TM, int WMW, int WNW, int NSA, int NSB>
__global__ __launch_bounds__(WMW* WNW * 64) __attribute__((amdgpu_waves_per_eu(WMW * WNW / 4))) void k_i8_tile(
    I8Args g, int m_tiles, int n_tiles, int per_xcd, int turn) {
  using G = Geom<TM, WMW, WNW, NSA, NSB>;
  constexpr int MI = G::MI, NI = G::NI;
  extern __shared__ __align__(16) uint8_t i8_lds[];
  lds_u8* const L = (lds_u8*)i8_lds;
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, h = lane >> 5;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wid / WNW, wn = wid % WNW;
  const int lda = int(g.lda), ldb = int(g.ldb);
  const int stages = (g.K + kTK - 1) / kTK;

  // workgroups go to the 8 XCDs in turn; each XCD takes a contiguous run of
  // the order that walks groups of kRaster token tiles along the channels
  const int n_all = m_tiles * n_tiles, x0 = int(blockIdx.x & 7) * per_xcd;
  const int end = min(per_xcd, n_all - x0), step = int(gridDim.x >> 3);
  int cur = int(blockIdx.x >> 3);
  if (cur >= end) return;
  auto tile_at = [&](int t, int& m0, int& n0) {
    const int lin = x0 + t, gsz = kRaster * n_tiles, rg = lin / gsz, first = rg * kRaster;
    const int gm = min(m_tiles - first, kRaster), within = lin - rg * gsz;
    m0 = (first + within % gm) * TM;
    n0 = within / gm * kTileN;
  };

  // ---- loads of a and of b: the tile and stage they have come to
  struct Cursor {
    int tile, stage, slot, first;   // first: the stage of k that the tile begins with
  };
  Cursor ca{cur, 0, 0, 0}, cb{cur, 0, 0, 0};
  __amdgpu_buffer_rsrc_t ra, rb;
  uint32_t ao[G::NA], bo[G::NB];
  // This lane's unit of its wave's load i: row r, unit p of LDS, holding unit
  // p ^ swz of the row; rows past the last repeat it.
  auto unit_of = [&](int i, int n_loads, int& r) {
    const int off = (wid * n_loads + i) * 1024 + 16 * lane;
    r = off / kTK;
    return 16 * ((off % kTK / 16) ^ swz_x(r));
  };
  auto begin = [&](auto is_b) {
    constexpr bool B = decltype(is_b)::value;
    Cursor& c = B ? cb : ca;
    int m0, n0;
    tile_at(c.tile, m0, n0);
    c.first = turn ? n0 / kTileN * turn % stages : 0;
    const int64_t r0 = B ? n0 : m0, all = B ? g.N : g.M;
    constexpr int most = B ? kTileN : TM, n_loads = B ? G::NB : G::NA;
    const int rows = int(all - r0 < most ? all - r0 : most), ld = B ? ldb : lda;
    (B ? rb : ra) = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(B ? g.b + r0 * g.ldb : g.a + r0 * g.lda), 0,
                                               (rows - 1) * ld + g.K, kBufferWord3);
#pragma unroll
    for (int i = 0; i < n_loads; ++i) {
      int r;
      const int u = unit_of(i, n_loads, r);
      (B ? bo[i] : ao[i]) = uint32_t(min(r, rows - 1)) * ld + u;
    }
  };
  using IsA = std::false_type;
  using IsB = std::true_type;
  auto load = [&](__amdgpu_buffer_rsrc_t r, lds_u8* dst, uint32_t off, int k0) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, reinterpret_cast<__attribute__((address_space(3))) void*>(dst), 16, off,
                                             k0, 0, 0);
  };
  auto a_at = [&](int slot) { return L + slot * G::ABYTES; };
  auto b_at = [&](int slot) { return L + G::BAT + slot * G::BBYTES; };
  auto k_of = [&](const Cursor& c) {
    const int ks = c.stage + c.first;
    return (ks < stages ? ks : ks - stages) * kTK;
  };
  auto pass = [&](Cursor& c, int slots) {
    ++c.stage;
    c.slot = c.slot + 1 == slots ? 0 : c.slot + 1;
  };
  // a whole stage that is not its tile's last
  auto issue_whole = [&](auto is_b) {
    constexpr bool B = decltype(is_b)::value;
    constexpr int n_loads = B ? G::NB : G::NA;
    Cursor& c = B ? cb : ca;
    lds_u8* const to = B ? b_at(c.slot) : a_at(c.slot);
    const int k0 = k_of(c);
#pragma unroll
    for (int i = 0; i < n_loads; ++i)
      load(B ? rb : ra, to + (wid * n_loads + i) * 1024, B ? bo[i] : ao[i], k0);
    pass(c, B ? NSB : NSA);
  };
  // any next stage of the sequence, if there is one; of the units past K a's are
  // zeros, b's what is left of an earlier stage
  auto issue_next = [&](auto is_b) {
    constexpr bool B = decltype(is_b)::value;
    Cursor& c = B ? cb : ca;
    constexpr int n_loads = B ? G::NB : G::NA;
    if (c.tile >= end) return;
    lds_u8* const to = B ? b_at(c.slot) : a_at(c.slot);
    const int k0 = k_of(c);
    if (k0 + kTK <= g.K) {
#pragma unroll
      for (int i = 0; i < n_loads; ++i) load(B ? rb : ra, to + (wid * n_loads + i) * 1024, B ? bo[i] : ao[i], k0);
    } else {
#pragma unroll
      for (int i = 0; i < n_loads; ++i) {
        int r;
        lds_u8* const at = to + (wid * n_loads + i) * 1024;
        if (k0 + unit_of(i, n_loads, r) < g.K) load(B ? rb : ra, at, B ? bo[i] : ao[i], k0);
        else if (!B) *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(at + 16 * lane) = u32x4{0, 0, 0, 0};
      }
    }
    pass(c, B ? NSB : NSA);
    if (c.stage == stages) {
      c.stage = 0;
      c.tile += step;
      if (c.tile < end) begin(is_b);
    }
  };
  // a tile's scales and bias: read into registers, later put into LDS
  constexpr int kPer = (G::NSC + G::NW * 64 - 1) / (G::NW * 64);
  float held[kPer];
  auto fetch_scales = [&](int t) {
    int m0, n0;
    tile_at(t, m0, n0);
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int i = tid + u * G::NW * 64, j = i < TM ? i : (i - TM) % kTileN;
      held[u] = 0.f;
      if (i < TM) held[u] = m0 + j < g.M ? g.sa[m0 + j] : 0.f;
      else if (i < G::NSC && n0 + j < g.N) held[u] = i < TM + kTileN ? g.sb[n0 + j] : g.bias ? g.bias[n0 + j] : 0.f;
    }
  };
  auto put_scales = [&](int half) {
    float* const to = reinterpret_cast<float*>(i8_lds + G::SCALES) + half * G::NSC;
#pragma unroll
    for (int u = 0; u < kPer; ++u)
      if (tid + u * G::NW * 64 < G::NSC) to[tid + u * G::NW * 64] = held[u];
  };

  // ---- products
  uint32_t unit[4];   // operands of K-step ks: unit 2 ks + h of rows lr, lr + 32, ...
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) unit[ks] = uint32_t(lr) * kTK + 16 * ((2 * ks + h) ^ swz_x(lr));
  i32x4 A[2][MI], B[2][NI];
  int sa_slot = 0, sb_slot = 0;   // of the stage being computed
  auto read = [&](int to, int ks) {
    const lds_u8 *const pa = a_at(sa_slot) + unit[ks], *const pb = b_at(sb_slot) + unit[ks];
#pragma unroll
    for (int i = 0; i < MI; ++i) A[to][i] = lds_load<i32x4>(pa + (wm * G::WM + 32 * i) * kTK);
#pragma unroll
    for (int i = 0; i < NI; ++i) B[to][i] = lds_load<i32x4>(pb + (wn * G::WN + 32 * i) * kTK);
  };
  auto next_stage = [&]() {
    sa_slot = sa_slot + 1 == NSA ? 0 : sa_slot + 1;
    sb_slot = sb_slot + 1 == NSB ? 0 : sb_slot + 1;
  };
  i32x16 acc[MI][NI];
  auto multiply = [&](int at) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(B[at][j], A[at][i], acc[i][j], 0, 0, 0);
  };
  constexpr int kReads = MI + NI;
  // Where b runs a stage further ahead than a, its loads are issued a step
  // later, in the next stage's first.  Loads younger than the next stage's where
  // the waves meet: those of NSA - 2 stages, or this one's of b.
  constexpr bool kLateB = NSB > NSA;
  constexpr int kAhead = kLateB ? G::NB : (NSA - 2) * (G::NA + G::NB);
  static_assert(NSB == NSA || (NSA == 2 && NSB == 3), "what the counted wait assumes");
  // the steps of a stage but its last
  auto steps = [&](auto late_b) {
    constexpr bool LATE = decltype(late_b)::value;
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (LATE) issue_whole(IsB{});
    read(1, 1);
    multiply(0);
    spread<kReads, LATE ? G::NB : 0, MI * NI>();
    read(0, 2);
    multiply(1);
    spread<kReads, 0, MI * NI>();
    read(1, 3);
    multiply(0);
    spread<kReads, 0, MI * NI>();
  };

  begin(IsA{});
  begin(IsB{});
#pragma unroll
  for (int i = 0; i < NSA; ++i) {   // (of b one more, where there is room, in the first stage)
    issue_next(IsA{});
    issue_next(IsB{});
  }
  fetch_scales(cur);
  put_scales(0);
  wait_loads_barrier<0>();
  read(0, 0);
  int half = 0;
  for (; cur < end; cur += step, half ^= 1) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
    if (cur + step < end) fetch_scales(cur + step);
    int s = 0;
    const int full = stages - 1 - NSA;   // stages whose loads are of this tile, and not its last: whole
#pragma unroll 1
    for (; s < full; ++s) {
      steps(std::integral_constant<bool, kLateB>{});
      wait_loads_barrier<kAhead>();
      __builtin_amdgcn_sched_barrier(0);
      issue_whole(IsA{});
      if constexpr (!kLateB) issue_whole(IsB{});
      next_stage();
      read(0, 0);
      multiply(1);
      spread<kReads, G::NA + (kLateB ? 0 : G::NB), MI * NI>();
    }
#pragma unroll 1
    for (; s < stages; ++s) {
      if constexpr (kLateB) issue_next(IsB{});
      steps(std::false_type{});
      wait_loads_barrier<0>();
      issue_next(IsA{});
      if constexpr (!kLateB) issue_next(IsB{});
      next_stage();
      read(0, 0);   // (behind the last stage: values that nothing uses)
      multiply(1);
    }
    put_scales(half ^ 1);   // (read in the epilogue before this one, by waves that have met since)

    // ---- outputs: each wave turns 16 tokens of 128 (64) bytes at a time through
    // its own part of the LDS, so that eight (four) lanes store what lies together
    // (4096 x 151936 x 4096 bf16 2.23 ms; 32 tokens of 64 bytes at a time: 2.29)
    int m0, n0;
    tile_at(cur, m0, n0);
    const float* const sc = reinterpret_cast<const float*>(i8_lds + G::SCALES) + half * G::NSC;
    constexpr int EB = DT == ARCHEAD_F32 ? 4 : 2;
    constexpr int CP = G::OBYTES / EB < G::WN ? G::OBYTES / EB : G::WN;   // channels of a turn
    constexpr int KP = CP / 8, LPR = CP * EB / 16;                        // a lane's fours; lanes to a token
    uint8_t* const buf = i8_lds + G::OUT + wid * 16 * G::OROW;
    const bool whole = m0 + TM <= g.M && n0 + kTileN <= g.N;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const float sa = sc[wm * G::WM + 32 * mi + lr];
#pragma unroll
      for (int c0 = 0; c0 < G::WN; c0 += CP) {
        alignas(16) uint32_t pk[KP][EB];
#pragma unroll
        for (int k = 0; k < KP; ++k) {
          const int c = c0 + 8 * k, at = wn * G::WN + c + 4 * h;   // (of the wave's channels; of the tile's)
          const f32x4 sb = *reinterpret_cast<const f32x4*>(sc + TM + at);
          const f32x4 bi = *reinterpret_cast<const f32x4*>(sc + TM + kTileN + at);
          float y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = scaled(acc[mi][c / 32][c % 32 / 2 + i], sa, sb[i], bi[i]);
          put4<DT>(reinterpret_cast<uint8_t*>(pk[k]), y);
        }
#pragma unroll
        for (int t0 = 0; t0 < 32; t0 += 16) {
          if ((lr & 16) == t0)
#pragma unroll
            for (int k = 0; k < KP; ++k)
              __builtin_memcpy(__builtin_assume_aligned(buf + (lr & 15) * G::OROW + (8 * k + 4 * h) * EB, 4 * EB), pk[k],
                               4 * EB);
          wave_lds_order();
#pragma unroll
          for (int j = 0; j < 16; j += 64 / LPR) {
            const int rl = j + lane / LPR, q = lane % LPR;
            const u32x4 v = *reinterpret_cast<const u32x4*>(buf + rl * G::OROW + 16 * q);
            const int64_t m = m0 + wm * G::WM + 32 * mi + t0 + rl, n = n0 + wn * G::WN + c0 + q * (16 / EB);
            uint8_t* const p = g.out + (m * g.ldo + n) * EB;
            if (whole) store_any(p, v);
            else if (m < g.M) store_part<EB>(p, v, g.N - n);
          }
          wave_lds_order();
        }
      }
    }
  }
}

template <int DT, int TM, int WMW, int WNW, int NSA, int NSB>
hipError_t launch(const I8Args& g, int n_cu, hipStream_t s) {
  using G = Geom<TM, WMW, WNW, NSA, NSB>;
  const int m_tiles = int((g.M + TM - 1) / TM), n_tiles = int((g.N + kTileN - 1) / kTileN);
  const int per_xcd = (m_tiles * n_tiles + 7) / 8, wgs = 8 * std::min(per_xcd, std::max(n_cu / 8, 1));
  // Tiles of neighbouring channels begin at different k (the sums are exact in
  // any order) where a stays in the L2s all the same: else rows of a power of
  // two all ask for the same memory channels at once (64 x 151936 x 4096:
  // 158 -> 127 us).
  const int turn = g.K % kTK == 0 && g.M * g.K <= kTurnMost ? 5 : 0;
  return launch_kernel_lds(k_i8_tile<DT, TM, WMW, WNW, NSA, NSB>, dim3(unsigned(wgs)), dim3(G::NW * 64), G::LDS, s, g, m_tiles,
                           n_tiles, per_xcd, turn);
}

}  // namespace

namespace archead {
namespace i8 {

bool tiles_take(const I8Args& g) {
  const int64_t tiles = ((g.M + 63) / 64) * ((g.N + kTileN - 1) / kTileN);
  return g.K > 0 && g.lda <= kMaxLd && g.ldb <= kMaxLd && tiles < (1 << 22);
}

template <int DT>
hipError_t launch_tiles(const I8Args& g, int tm, int n_cu, hipStream_t s) {
  return tm == 256   ? launch<DT, 256, 2, 4, 2, 2>(g, n_cu, s)
         : tm == 192 ? launch<DT, 192, 2, 4, 2, 3>(g, n_cu, s)
         : tm == 128 ? launch<DT, 128, 2, 4, 3, 3>(g, n_cu, s)
                     : launch<DT, 64, 1, 8, 3, 3>(g, n_cu, s);
}
template hipError_t launch_tiles<ARCHEAD_F32>(const I8Args&, int, int, hipStream_t);
template hipError_t launch_tiles<ARCHEAD_BF16>(const I8Args&, int, int, hipStream_t);
template hipError_t launch_tiles<ARCHEAD_F16>(const I8Args&, int, int, hipStream_t);

}  // namespace i8
}  // namespace archead
