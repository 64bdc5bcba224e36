// Tiles of the dense head's products: logits and their statistics, the logits'
// gradient, and the gradients of hidden states and head.
#include <algorithm>

#include "dev_common.cuh"
#include "dev_rows.cuh"
#include "head_loss.h"

namespace {

using namespace archead::rows;
using namespace archead::loss;

typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kRasterI = 8;        // tiles of i in a raster group

template <int OP, int TI>
struct Geom {
  static constexpr bool AT = OP == kHead, BT = OP == kHidden || OP == kHead;   // operands whose rows are k
  static constexpr int WI = TI >= 128 ? 2 : 1, WJ = 8 / WI, NW = 8;             // waves along i, j
  static constexpr int NI = TI / WI / 32, NJ = kTileJ / WJ / 32;                // blocks of 32 x 32 of a wave
  static constexpr int NS = TI == 64 ? 3 : 2;                                   // stages in LDS (of 64 tokens: 64 x 151936 x 4096 logits 271 us, two 301)
  static constexpr int ABYTES = TI * kStageK * 2, BBYTES = kTileJ * kStageK * 2, STAGE = ABYTES + BBYTES;
  static constexpr int LA = ABYTES / 1024 / NW, LB = BBYTES / 1024 / NW;        // loads of a wave and stage
  // behind the stages: what the waves exchange (kStats), or their rows of 16-bit outputs: 16
  // rows of their columns each, padded
  static constexpr int OUT = NS * STAGE, OROW = NJ * 64 + 16;
  static constexpr int LDS = OUT + (OP == kStats ? WJ * TI * 8 : OP == kHidden ? 0 : NW * 16 * OROW);
  static_assert(LDS <= 160 * 1024, "LDS budget");
  static_assert(!AT || TI >= 128, "rows of k have four parts of 64 bytes to swizzle");
};

// After each of the first products of a K-step a share of its R LDS reads; of V
// loads to LDS after all of them.  Without it the compiler puts the reads right
// before their use.
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

// 16 bytes a lane, at voff + soff of a buffer, to LDS
__device__ __forceinline__ void load_lds(__amdgpu_buffer_rsrc_t r, lds_u8* to, uint32_t voff, int soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, reinterpret_cast<__attribute__((address_space(3))) void*>(to), 16, voff, soff, 0, 0);
}

// A transposing read of LDS.  (Of its own function, its argument restrict: the read then
// carries the alias information without which the compiler waits, before each such read,
// for every load to LDS that is on its way: the gradients 4.7 and 5.0 ms instead of
// 4.1 and 4.2.)
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
__device__ __forceinline__ s16x4 read_tr(lds_s16x4* __restrict p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p); }

// One operand's way to LDS and into registers.  T false: rows of the operand, 64 k =
// 128 bytes each, their 16-byte units swizzled so that eight rows' reads of one unit
// fall on eight different bank groups.  T true: rows of k, ROWS columns (128 at least)
// each; a group of 16 lanes reads four rows of 16 columns and gets them transposed,
// so a lane has four k of its column.  There the 64-byte parts of a row are swizzled
// by its place among four: the four rows of a read then lie in different banks.
template <bool T, int ROWS, int LOADS, int BLOCKS>
struct Operand {
  const uint16_t* next;    // the next stage's first element
  int64_t ld, left;        // T: rows of k from there on
  int there;               // rows of the tile, or T: columns
  int bytes;               // that a whole stage reaches over
  uint32_t off[LOADS];
  uint32_t at[4];          // of a lane's reads

  // a load's place in LDS of this lane: row and 16-byte unit of the source
  static __device__ __forceinline__ void place(int i, int wid, int lane, int& r, int& u) {
    const int o = (wid * LOADS + i) * 1024 + 16 * lane;
    if constexpr (T) {
      r = o / (ROWS * 2);
      u = (o % (ROWS * 2) / 16) ^ (4 * (r & 3));
    } else {
      r = o / 128;
      u = (o % 128 / 16) ^ swz_x(r);
    }
  }
  // T false: `first` row of `all`; T true: `first` column of `all`, krows rows of k there are;
  // and the stage that it begins with
  __device__ __forceinline__ void begin(const uint16_t* p, int64_t ld_, int64_t first, int64_t all, int64_t krows, int stage, int wid,
                                        int lane) {
    ld = ld_;
    there = int(all - first < ROWS ? all - first : ROWS);
    const int64_t k0 = int64_t(stage) * kStageK;
    if constexpr (T) {
      next = p + k0 * ld + first;
      left = krows - k0;
      bytes = int(((kStageK - 1) * ld + ((there + 7) & ~7)) * 2);
    } else {
      next = p + first * ld + k0;
      bytes = int(((there - 1) * ld + kStageK) * 2);
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      int r, u;
      place(i, wid, lane, r, u);
      off[i] = T ? uint32_t(r * ld * 2) + 2 * min(8 * u, (there - 1) & ~7) : uint32_t(min(r, there - 1) * ld * 2) + 16 * u;
    }
  }
  // a stage whose k are all there
  __device__ __forceinline__ void issue_whole(lds_u8* to, int wid) {
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(next), 0, bytes, kBufferWord3);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_lds(rsrc, to + (wid * LOADS + i) * 1024, off[i], 0);
    next += T ? kStageK * ld : kStageK;
    if constexpr (T) left -= kStageK;
  }
  __device__ __forceinline__ void issue(lds_u8* to, int wid, int lane) {
    if (!T || left >= kStageK) {
      issue_whole(to, wid);
      return;
    }
    // rows past the last repeat it (the other operand has zeros there)
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(next), 0, int(((left - 1) * ld + ((there + 7) & ~7)) * 2),
                                                        kBufferWord3);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      int r, u;
      place(i, wid, lane, r, u);
      load_lds(rsrc, to + (wid * LOADS + i) * 1024, uint32_t(min(r, int(left) - 1) * ld * 2) + 2 * min(8 * u, (there - 1) & ~7), 0);
    }
  }
  // this wave's reads begin at row (column) `first` of the tile
  __device__ __forceinline__ void aim(int first, int lane) {
    const int lr = lane & 31, h = lane >> 5;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (T) {   // of block i
        const int row = (lane >> 2) & 3, unit = (first + 32 * i) / 8 + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        at[i] = (8 * h + row) * (ROWS * 2) + 16 * (unit ^ (4 * row)) + 8 * (lane & 1);
      } else {             // of K-step i
        at[i] = (first + lr) * 128 + 16 * ((2 * i + h) ^ swz_x(lr));
      }
    }
  }
  __device__ __forceinline__ void read(b16x8 (&to)[BLOCKS], const lds_u8* from, int ks) const {
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
      if constexpr (T) {
        const lds_u8* const p = from + at[i] + 16 * ks * (ROWS * 2);
        const s16x4 lo = read_tr(reinterpret_cast<lds_s16x4*>(const_cast<lds_u8*>(p)));
        const s16x4 hi = read_tr(reinterpret_cast<lds_s16x4*>(const_cast<lds_u8*>(p + 4 * (ROWS * 2))));
        to[i] = __builtin_bit_cast(b16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      } else {
        to[i] = lds_load<b16x8>(from + at[ks] + 32 * i * 128);
      }
    }
  }
  static constexpr int kReads = BLOCKS * (T ? 2 : 1);
};

// LDS accesses of one wave stay in this order (the hardware keeps it; lanes read
// what other lanes wrote, which the compiler does not see).
__device__ __forceinline__ void wave_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}
// All waves' LDS accesses are done; loads to LDS may go on.
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int OP, int TI>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void k_ce_tile(TileArgs g) {
  using G = Geom<OP, TI>;
  constexpr int NI = G::NI, NJ = G::NJ, NS = G::NS;
  extern __shared__ __align__(16) uint8_t ce_lds[];
  lds_u8* const L = (lds_u8*)ce_lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wi = wid / G::WJ, wj = wid % G::WJ;
  const int live = *g.count;
  const int64_t rows = OP == kHead ? g.rows : int64_t(live);
  const int64_t depth = OP == kHead ? (int64_t(live) + kStageK - 1) / kStageK * kStageK : g.depth;

  // workgroups go to the 8 XCDs in turn; each XCD takes a contiguous run of the
  // order that walks groups of kRasterI tiles of i along j, its workgroups in turn
  const int i_tiles = int((rows + TI - 1) / TI), j_tiles = int((g.cols + kTileJ - 1) / kTileJ), ij = i_tiles * j_tiles;
  const int all_stages = int((depth + kStageK - 1) / kStageK);
  const int splits =
      OP == kHidden ? min(splits_for(ij, live, g.sum_rows, g.first_stages), max(1, all_stages / kPartStages)) : 1;
  const int n_all = ij * splits, per_xcd = (n_all + 7) / 8, x0 = int(blockIdx.x & 7) * per_xcd;
  const int end = min(per_xcd, n_all - x0), step = int(gridDim.x >> 3);
  int cur = int(blockIdx.x >> 3);
  if (cur >= end) return;
  struct At {
    int64_t i0, j0;
    int split, s0, stages;
  };
  auto tile_at = [&](int t) {
    const int lin = x0 + t, split = lin / ij, tile = lin - split * ij;
    const int gsz = kRasterI * j_tiles, rg = tile / gsz, first = rg * kRasterI;
    const int gi = min(i_tiles - first, kRasterI), within = tile - rg * gsz;
    At r;
    // (32 tiles later, where a workgroup goes on, another i: the last one may be cheaper)
    const int turn = 32 % gi == 0 ? tile / 32 : 0;
    r.i0 = int64_t(first + (within + turn) % gi) * TI;
    r.j0 = int64_t(within / gi) * kTileJ;
    r.split = split;
    r.s0 = int(int64_t(all_stages) * split / splits);
    r.stages = int(int64_t(all_stages) * (split + 1) / splits) - r.s0;
    return r;
  };

  // ---- loads: the tile and stage they have come to
  Operand<G::AT, TI, G::LA, NI> a;
  Operand<G::BT, kTileJ, G::LB, NJ> b;
  a.aim(wi * NI * 32, lane);
  b.aim(wj * NJ * 32, lane);
  int l_tile = cur, l_stage = 0, l_slot = 0, l_stages = 0;
  auto begin = [&]() {
    const At r = tile_at(l_tile);
    l_stages = r.stages, l_stage = 0;
    a.begin(g.a, g.a_ld, r.i0, OP == kHead ? (rows + 255) / 256 * 256 : rows, depth, r.s0, wid, lane);
    b.begin(g.b, g.b_ld, r.j0, g.cols, depth, r.s0, wid, lane);
  };
  // a stage that is not its tile's last
  auto issue_whole = [&]() {
    lds_u8* const to = L + l_slot * G::STAGE;
    a.issue_whole(to, wid);
    b.issue_whole(to + G::ABYTES, wid);
    l_slot = l_slot + 1 == NS ? 0 : l_slot + 1;
    ++l_stage;
  };
  // any next stage of the sequence, if there is one
  auto issue_next = [&]() {
    if (l_tile >= end) return;
    lds_u8* const to = L + l_slot * G::STAGE;
    a.issue(to, wid, lane);
    b.issue(to + G::ABYTES, wid, lane);
    l_slot = l_slot + 1 == NS ? 0 : l_slot + 1;
    if (++l_stage == l_stages) {
      l_tile += step;
      if (l_tile < end) begin();
    }
  };
  b16x8 A[2][NI], B[2][NJ];
  f32x16 acc[NI][NJ];
  int slot = 0;   // of the stage being computed
  auto read = [&](int to, int ks) {
    const lds_u8* const from = L + slot * G::STAGE;
    a.read(A[to], from, ks);
    b.read(B[to], from + G::ABYTES, ks);
  };
  auto multiply = [&](int of) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(B[of][j], A[of][i], acc[i][j], 0, 0, 0);
  };
  constexpr int kReads = decltype(a)::kReads + decltype(b)::kReads, P = NI * NJ;
  // A persistent workgroup per CU takes tiles in turn, their stages as one sequence: the
  // loads run NS stages ahead of the products, across tiles, so the next tile's first
  // stages are on their way while one is written.  A wave reads the operands of a K-step
  // (16 k) during the step before.  Before the last step of a stage all its reads are
  // done, so there the waves meet, once a stage: the next stage has landed, its first
  // operands are read and the loads of the one after overwrite this one, all under
  // the last step's products.
  //
  // 4096 x 151936 x 4096 (5.1 Tflop each): logits 3.74 to 4.0 ms over cards (1.36 to 1.27
  // Pflop/s; the matrix units are busy 69 % of the time at the 1.74 GHz that the power limit
  // leaves), G 4.3 to 4.6, hidden states 3.8 to 4.0, head 4.1 to 4.3.
  if (all_stages > 0) {
    begin();
#pragma unroll
    for (int i = 0; i < NS; ++i) issue_next();
    wait_loads_barrier<0>();
  }
  auto next_slot = [&]() { slot = slot + 1 == NS ? 0 : slot + 1; };
  // The steps of a stage but its last, and the meeting: with the loads of all stages but the next
  // one in flight where whole ones follow it, else with none.
  auto steps = [&](auto whole) {
    constexpr int AHEAD = decltype(whole)::value ? (NS - 2) * (G::LA + G::LB) : 0;
    __builtin_amdgcn_sched_barrier(0);
    read(1, 1);
    multiply(0);
    spread<kReads, 0, P>();
    read(0, 2);
    multiply(1);
    spread<kReads, 0, P>();
    read(1, 3);
    multiply(0);
    spread<kReads, 0, P>();
    wait_loads_barrier<AHEAD>();
    __builtin_amdgcn_sched_barrier(0);
    next_slot();
  };
  for (; cur < end; cur += step) {
  const At tile = tile_at(cur);
  const int64_t i0 = tile.i0, j0 = tile.j0;
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
  int s = 0;
  // A wave whose rows are all past the last loads and meets the others only: the other
  // wave of its SIMD has the matrix unit to itself, so a tile of half as many rows takes half
  // the time.
  if (i0 + wi * NI * 32 >= rows) {
#pragma unroll 1
    for (; s < tile.stages; ++s) {
      wait_loads_barrier<0>();
      next_slot();
      issue_next();
    }
  }
  if (s < tile.stages) read(0, 0);
  // stages whose loads are of this tile and not its last: no branches, the loads among the
  // products (behind a branch, before them: logits of 4096 x 151936 x 4096 3.83 ms, so 3.74)
#pragma unroll 1
  for (; s < tile.stages - NS - 1; ++s) {
    steps(std::true_type{});
    issue_whole();
    read(0, 0);
    multiply(1);
    spread<kReads, G::LA + G::LB, P>();
  }
#pragma unroll 1
  for (; s < tile.stages; ++s) {
    steps(std::false_type{});
    issue_next();
    if (s + 1 < tile.stages) read(0, 0);   // (beside the outputs they would not fit)
    multiply(1);
  }

  // ---- outputs.  A lane's results: row i = lr of a block, columns 8 (r / 4) + 4 h + r % 4
  const int64_t jw = j0 + wj * NJ * 32;   // this wave's first column
  int lane_here = lane;   // (its multiples are formed anew for each tile: kept over the stages they would not fit)
  asm volatile("" : "+v"(lane_here));
  const int lr = lane_here & 31, h = lane_here >> 5;
  if constexpr (OP == kStats) {
    float2* const red = reinterpret_cast<float2*>(ce_lds + G::OUT);   // [WJ][TI]
    const bool whole = j0 + kTileJ <= g.cols;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int row = wi * NI * 32 + 32 * i + lr;
      const int64_t token = i0 + row;
      if (!whole) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (jw + 32 * j + 8 * (r / 4) + 4 * h + r % 4 >= g.cols) acc[i][j][r] = -INFINITY;
      }
      float top = -INFINITY, sum = 0;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, acc[i][j][r]);
      top = fmaxf(top, __shfl_xor(top, 32));
      if (top > -INFINITY) {
        // (subtracted before it is scaled: the largest's exponential is 1 whatever its size, and
        // finite logits of any size have finite sums)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f((acc[i][j][r] - top) * kLog2e);
      } else {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) sum = acc[i][j][r] != acc[i][j][r] ? NAN : sum;
      }
      sum += __shfl_xor(sum, 32);
      if (h == 0) red[wj * TI + row] = float2{top, sum};
      const int64_t y = token < live ? g.target[token] - g.v0 - jw : -1;   // of this wave's columns
      const bool mine = y >= 0 && y < NJ * 32 && (int(y) >> 2 & 1) == h;
      if (__ballot(mine) != 0) {
        float hit = 0;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) hit = (int(y) & ~4) == 32 * j + 8 * (r / 4) + r % 4 ? acc[i][j][r] : hit;
        if (mine) g.at_target[token] = hit;
      }
      __builtin_amdgcn_sched_barrier(0);   // (one token's values at a time in registers)
    }
    meet();
    if (tid < TI && i0 + tid < live) {
      float top = -INFINITY, sum = 0;
#pragma unroll
      for (int w = 0; w < G::WJ; ++w) top = fmaxf(top, red[w * TI + tid].x);
#pragma unroll
      for (int w = 0; w < G::WJ; ++w) {
        const float2 p = red[w * TI + tid];
        sum += p.x == top ? p.y : p.y * __builtin_amdgcn_exp2f((p.x - top) * kLog2e);
      }
      g.part[(i0 + tid) * g.n_part + g.part0 + j0 / kTileJ] = float2{top, sum};
    }
    meet();   // (red has been read)
  } else if constexpr (OP == kHidden) {
    float* const base = g.sums + tile.split * padded_rows(live) * g.sum_ld;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      float* const row = base + (i0 + wi * NI * 32 + 32 * i + lr) * g.sum_ld;   // (rows are padded to whole tiles)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int64_t c = jw + 32 * j + 2 * r + 4 * h;
          if (c >= g.sum_ld) continue;   // (a multiple of 64)
          f32x4v v{acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]};
          f32x4v* const p = reinterpret_cast<f32x4v*>(row + c);
          if (g.add) v += *p;
          *p = v;
        }
    }
  } else {
    // 16-bit rows: each wave turns 16 at a time through its own part of the LDS, so
    // that neighbouring lanes store what lies together
    constexpr int LPR = NJ * 4;   // lanes to a row
    uint8_t* const buf = ce_lds + G::OUT + wid * 16 * G::OROW;
    const int64_t cols = g.cols;
    const bool whole = j0 + kTileJ <= cols;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int64_t row0 = i0 + wi * NI * 32 + 32 * i, token = row0 + lr;
      float lse = 0, gr = 0;
      int y = -1;
      const float unit = OP == kHead ? *g.unit : 1.f;
      if constexpr (OP == kGrad) {
        if (token < live) {
          lse = g.lse[token];
          gr = g.g[token];
          const int64_t at = g.target[token] - g.v0 - jw;
          y = at >= 0 && at < NJ * 32 ? int(at) : -1;
        }
      }
      b16x4 out[NJ][4];
      const bool some = token < live;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          f32x4v v;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[e] = acc[i][j][4 * k + e];
            if constexpr (OP == kHead) v[e] *= unit;
            if constexpr (OP == kGrad) {
              const int c = 32 * j + 8 * k + 4 * h + e;
              float p = __builtin_amdgcn_exp2f((v[e] - lse) * kLog2e);   // (scaled first it would leave fp32)
              if (y == c) p -= 1.f;
              v[e] = some && (whole || jw + c < cols) ? p * gr : 0.f;
            }
          }
          out[j][k] = __builtin_convertvector(v, b16x4);
        }
#pragma unroll
      for (int t = 0; t < 32; t += 16) {
        if ((lr & 16) == t) {
#pragma unroll
          for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              *reinterpret_cast<b16x4*>(buf + (lr & 15) * G::OROW + (32 * j + 8 * k + 4 * h) * 2) = out[j][k];
        }
        wave_order();
#pragma unroll
        for (int r = lane_here / LPR; r < 16; r += 64 / LPR) {
          const u32x4 v = *reinterpret_cast<const u32x4*>(buf + r * G::OROW + 16 * (lane_here % LPR));
          const int64_t row = row0 + t + r, j = jw + 8 * (lane_here % LPR);
          uint16_t* const p = g.out + row * g.out_ld + j;
          if constexpr (OP == kGrad) {   // (G has whole tiles)
            *reinterpret_cast<u32x4*>(p) = v;
          } else if (row < rows && j < cols) {
            if (j + 8 <= cols) {
              store_any(p, v);
            } else {
              const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (j + e < cols) p[e] = uint16_t(w[e / 2] >> (16 * (e & 1)));
            }
          }
        }
        wave_order();
      }
      __builtin_amdgcn_sched_barrier(0);   // (one row's values at a time in registers)
    }
  }
  }
}

template <int OP, int TI>
hipError_t launch(const TileArgs& g, hipStream_t s) {
  const int64_t i_tiles = (g.rows + TI - 1) / TI, j_tiles = (g.cols + kTileJ - 1) / kTileJ;
  // (of fewer tokens than there may be, more parts: as many tiles as there may be)
  const int64_t n = OP == kHidden ? kTargetTiles : i_tiles * j_tiles;
  const int64_t per_xcd = std::max((n + 7) / 8, OP == kHidden ? (i_tiles * j_tiles + 7) / 8 : 0);
  return launch_kernel_lds(k_ce_tile<OP, TI>, dim3(unsigned(8 * std::min<int64_t>(per_xcd, 32))), dim3(512), Geom<OP, TI>::LDS, s, g);
}

template <int OP>
hipError_t launch_op(int ti, const TileArgs& g, hipStream_t s) {
  return ti == 256 ? launch<OP, 256>(g, s) : ti == 128 ? launch<OP, 128>(g, s) : launch<OP, 64>(g, s);
}

}  // namespace

namespace archead {
namespace loss {

hipError_t launch_tiles(Op op, int ti, const TileArgs& g, hipStream_t s) {
  switch (op) {
    case kStats: return launch_op<kStats>(ti, g, s);
    case kGrad: return launch_op<kGrad>(ti, g, s);
    case kHidden: return launch_op<kHidden>(ti, g, s);
    default: return ti == 256 ? launch<kHead, 256>(g, s) : launch<kHead, 128>(g, s);
  }
}

}  // namespace loss
}  // namespace archead
