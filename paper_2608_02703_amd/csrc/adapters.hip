// archead_adapters_add: low-rank adapters of many requests at once.
#include <algorithm>
#include <type_traits>

#include "dev_rows.cuh"

namespace {

using namespace archead::rows;

constexpr int kUBlock = 256, kUWaves = kUBlock / 64;   // threads and waves of the outer products' workgroups
constexpr int64_t kMaxRank = 256;
constexpr int64_t kMaxM = int64_t(1) << 23;
constexpr float kMostBf16 = 0x1.fep127f;   // the largest finite bf16

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct AdaptArgs {
  const uint8_t* y;
  const uint8_t* x;
  const uint8_t* a;
  const uint8_t* b;
  const void* ids;
  const float* scales;     // may be null
  const int32_t* ranks;    // may be null
  uint8_t* out;
  uint4* t;                // operands [block][tile][32 ranks][part][64 lanes]
  float* back;             // fp16: powers of two [block][tile][32 ranks][16 tokens], or -1: t is in fp32
  uint8_t* table;          // Groups of the blocks
  int64_t M, N, K, n;
  int64_t y_row, x_row, a_ad, a_row, b_ad, b_row, o_row;   // bytes
  int R, kcs;              // operands of 32 ranks
  int spread;              // workgroups that share a block's tiles
  int per_block;           // tiles that a block may hold
  bool ids64, in_place;
};

__device__ __forceinline__ int rank_of(const AdaptArgs& p, int64_t id) {
  return p.ranks ? min(max(p.ranks[id], 0), p.R) : p.R;
}

// The TOK tokens of a block in the order of their adapters, and tiles of up to 16
// tokens of one adapter.
template <int TOK>
struct alignas(16) Groups {
  int32_t adapter[TOK], rank[TOK];   // of a tile; -1: none
  uint8_t first[TOK], len[TOK];      // of a tile: its first place, its tokens
  uint8_t token[TOK];                // of a place
  int32_t tiles, pad[3];
};
static_assert(sizeof(Groups<64>) % 16 == 0 && sizeof(Groups<256>) % 16 == 0, "copied by 16 bytes");

// Every thread counts the tokens whose (adapter, token) comes before its own.  Tokens
// without an adapter come last, and are left out where `none` is false.
template <int TOK>
__device__ __forceinline__ void group_tokens(Groups<TOK>& g, const AdaptArgs& p, int64_t m0, bool none) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  constexpr int W = TOK / 64;
  __shared__ u32x4 keys[TOK / 4];
  __shared__ int32_t ids[TOK];
  __shared__ uint64_t begins[W], starts[W];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int64_t id = -1;
  uint32_t key = 0;
  if (tid < TOK) {
    const bool there = m0 + tid < p.M;
    if (there) {
      id = p.ids64 ? static_cast<const int64_t*>(p.ids)[m0 + tid] : static_cast<const int32_t*>(p.ids)[m0 + tid];
      if (id < 0 || id >= p.n) id = -1;
    }
    // (adapters are fewer than 2^22: the numbers are different, and no number passes 32 bits)
    key = uint32_t(id >= 0 ? int(id) : there ? (1 << 22) : (1 << 22) + 1) * TOK + tid;
    reinterpret_cast<uint32_t*>(keys)[tid] = key;
  }
  __syncthreads();
  int place = 0;
  if (tid < TOK) {
#pragma unroll 8
    for (int l = 0; l < TOK / 4; ++l) {
      const u32x4 k = keys[l];
      place += int(k.x < key) + int(k.y < key) + int(k.z < key) + int(k.w < key);
    }
    g.token[place] = uint8_t(tid);
    ids[place] = m0 + tid < p.M ? int(id) : -2;
  }
  __syncthreads();
  int mine = -2;
  if (tid < TOK) {   // now of a place
    mine = ids[tid];
    const uint64_t mask = __ballot(tid == 0 || ids[tid - 1] != mine);
    if (lane == 0) begins[wave] = mask;
  }
  __syncthreads();
  bool start = false;
  int len = 0;
  if (tid < TOK) {
    // the places where this one's adapter begins and the next one does
    int from = 0, to = TOK;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const uint64_t upto = w < wave ? ~uint64_t(0) : w == wave ? ~uint64_t(0) >> (63 - lane) : 0;
      const uint64_t b = begins[w] & upto, n = begins[w] & ~upto;
      if (b) from = 64 * w + 63 - __builtin_clzll(b);
      if (n && to == TOK) to = 64 * w + __builtin_ctzll(n);
    }
    start = (mine >= 0 || (mine == -1 && none)) && (tid - from) % 16 == 0;
    len = min(16, to - tid);
    const uint64_t mask = __ballot(start);
    if (lane == 0) starts[wave] = mask;
  }
  __syncthreads();
  int at = 0, all = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int n = __popcll(starts[w]);
    at += w < wave ? n : w == wave ? __popcll(starts[w] & ((uint64_t(1) << lane) - 1)) : 0;
    all += n;
  }
  if (start) {
    g.first[at] = uint8_t(tid);
    g.len[at] = uint8_t(len);
    g.adapter[at] = mine;
    g.rank[at] = mine < 0 ? 0 : rank_of(p, mine);
  }
  if (tid == 0) g.tiles = all;
  __syncthreads();
}

template <int DT>
__device__ __forceinline__ f32x4 mma(const uint4& a, const uint4& b, const f32x4& c) {
  if constexpr (DT == ARCHEAD_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// t[m, j] = scale sum_k x[m, k] a[j, k] in fp32, written as the second operands of
// k_adapt_up's products.  A workgroup takes a tile of up to 16 tokens of one adapter (TT
// neighbouring ones of it, which share the loads of a) and RC x 16 ranks, its WAVES waves
// pieces of K in turn, whose sums meet in LDS.  Both operands come straight from memory
// (16 rows of 64 bytes a load), the ranks as the first.  Lanes past the tile's tokens or the
// adapter's ranks repeat the first: their results are not used, and no load hangs on a branch.  8192 x 4096, 64
// ranks of 8 adapters: 63 us, 10 of them grouping, most of the rest a's way through the L2s;
// 256 x 4096, up to 32 ranks of 32: 14 us, latency.
//
// t goes through the matrix units in PARTS parts of the operands' type: two hold 17
// bits of it in bf16 and 22 in fp16 (there after a power of two that brings a token's
// largest of 32 ranks to 2^14), three 25.  fp16's two have 22 bits of sums from 2^-3 on, 2^-17 of
// the largest.  Where one of a tile's is less, and not 0 (of normally distributed sums in a tile of
// some two hundred), its 32 ranks go on in fp32, in the place of two parts.
template <int DT, int RC, int TOK, int PARTS, int WAVES, int TT>
__global__ __launch_bounds__(64 * WAVES, 4) void k_adapt_down(AdaptArgs p) {
  constexpr int STEPS = TT == 2 ? 2 : RC == 4 ? 4 : 8, PIECE = 32 * STEPS, ROW = RC * 16 + 4;
  __shared__ Groups<TOK> g;
  __shared__ f32x4 part[WAVES][RC][64];
  __shared__ float ts[16 * ROW];
  const int64_t m0 = int64_t(blockIdx.x) * TOK;
  group_tokens(g, p, m0, !p.in_place);
  if (blockIdx.y == 0 && blockIdx.z == 0)   // for k_adapt_up
    for (int i = threadIdx.x; i < int(sizeof(g) / 16); i += 64 * WAVES)
      reinterpret_cast<uint4*>(p.table + blockIdx.x * sizeof(g))[i] = reinterpret_cast<const uint4*>(&g)[i];
  const int lane = threadIdx.x & 63, lr = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;
  const int j0 = int(blockIdx.y) * 16 * RC, K = int(p.K);
  // pieces of K to the waves in turn (shares one behind another would have rows of a
  // power of two all ask for the same memory channels), then 32 at a time of the rest
  const int pieces = K / PIECE;
  for (int t0 = int(blockIdx.z) * TT; t0 < g.tiles; t0 += p.spread * TT)
  for (int t1 = t0, run; t1 < min(t0 + TT, g.tiles); t1 += run) {   // tiles of one adapter
    const int64_t id = g.adapter[t1];
    const int rank = g.rank[t1];
    run = 1;
    while (run < TT - (t1 - t0) && t1 + run < g.tiles && g.adapter[t1 + run] == id) ++run;
    if (id < 0 || (j0 >= rank && j0 % 32 == 0)) continue;   // (operands are of 32 ranks: the second half of one is written)
    const uint8_t* x[TT];
#pragma unroll
    for (int u = 0; u < TT; ++u) {
      const int ti = t1 + min(u, run - 1);
      x[u] = p.x + (m0 + g.token[g.first[ti] + (lr < g.len[ti] ? lr : 0)]) * p.x_row;
    }
    const uint8_t* a[RC];
#pragma unroll
    for (int c = 0; c < RC; ++c) {
      const int j = j0 + 16 * c + lr;
      a[c] = p.a + id * p.a_ad + (j < rank ? j : 0) * p.a_row;
    }
    f32x4 acc[TT][RC] = {};
    for (int i = wave; i < pieces; i += WAVES) {   // all loads of a piece, then its products
      uint4 xv[STEPS][TT], av[STEPS][RC];
#pragma unroll
      for (int j = 0; j < STEPS; ++j) {
        const int at = 2 * (i * PIECE + 32 * j + 8 * q);
#pragma unroll
        for (int u = 0; u < TT; ++u) xv[j][u] = load_any<uint4>(x[u] + at);
#pragma unroll
        for (int c = 0; c < RC; ++c) av[j][c] = load_any<uint4>(a[c] + at);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < STEPS; ++j)
#pragma unroll
        for (int u = 0; u < TT; ++u)
#pragma unroll
          for (int c = 0; c < RC; ++c) acc[u][c] = mma<DT>(av[j][c], xv[j][u], acc[u][c]);
    }
    for (int last = pieces * PIECE + 32 * wave; last < K; last += 32 * WAVES) {   // zeros past K
      Eight<ARCHEAD_BF16> e;
      uint4 xv[TT];
#pragma unroll
      for (int u = 0; u < TT; ++u) {
        e.load(x[u], last + 8 * q, K, 0);
        xv[u] = e.w[0];
      }
#pragma unroll
      for (int c = 0; c < RC; ++c) {
        e.load(a[c], last + 8 * q, K, 0);
#pragma unroll
        for (int u = 0; u < TT; ++u) acc[u][c] = mma<DT>(e.w[0], xv[u], acc[u][c]);
      }
    }
    const float scale = p.scales ? p.scales[id] : 1.f;
#pragma unroll
    for (int u = 0; u < TT; ++u) {
    if (u >= run) break;
    const int ti = t1 + u;
#pragma unroll
    for (int c = 0; c < RC; ++c) part[wave][c][lane] = acc[u][c];
    __syncthreads();
    if (wave < RC) {
      f32x4 sum = part[0][wave][lane];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) sum += part[w][wave][lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] = j0 + 16 * wave + 4 * q + i < rank ? sum[i] * scale : 0.f;
      *reinterpret_cast<f32x4*>(&ts[lr * ROW + 16 * wave + 4 * q]) = sum;
    }
    __syncthreads();
    // operands of 32 ranks (RC = 1: half of one), a lane eight ranks of a token
    constexpr int LANES = RC == 1 ? 32 : RC * 32;
    const int w = threadIdx.x, jl = w / 16 * 8, kc = (j0 + jl) / 32, ql = (j0 + jl) % 32 / 8;
    if (w < LANES && kc < p.kcs) {
      float v[8], top = 0, pre = 1;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = ts[(w & 15) * ROW + jl + i];
        top = fmaxf(top, fabsf(v[i]));
      }
      bool full = false;   // of a tile's 32 ranks, which a wave has
      if constexpr (DT == ARCHEAD_F16) {
        static_assert(RC >= 2, "a wave has 32 ranks");
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        int e = 15;
        if (top > 0 && top < INFINITY) frexpf(top, &e);
        e = min(126, 15 - e);   // (no less than -113; 2^-126 is the least that back holds)
        pre = ldexpf(1.f, e);
        bool small = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) small |= v[i] != 0 && fabsf(v[i] * pre) < 0x1p-3f;
        full = __ballot(small) != 0;
        if (ql == 0) p.back[((int64_t(blockIdx.x) * p.per_block + ti) * p.kcs + kc) * 16 + (w & 15)] = full ? -1.f : ldexpf(1.f, -e);
      }
      uint32_t bits4[PARTS][4] = {};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float rest = v[i] * pre;
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
          uint16_t bits;
          float now;
          if constexpr (DT == ARCHEAD_BF16) {
            // (finite ones that would round to an infinity leave more to the next part)
            const __bf16 h = __bf16(fabsf(rest) < INFINITY ? fminf(fmaxf(rest, -kMostBf16), kMostBf16) : rest);
            now = float(h);
            __builtin_memcpy(&bits, &h, 2);
          } else {
            const _Float16 h = _Float16(rest);
            now = float(h);
            __builtin_memcpy(&bits, &h, 2);
          }
          bits4[k][i / 2] |= uint32_t(bits) << (16 * (i & 1));
          rest = fabsf(now) < INFINITY ? rest - now : 0.f;   // (an infinity or NaN has no rest)
        }
      }
      if (DT == ARCHEAD_F16 && full) {
        static_assert(DT != ARCHEAD_F16 || PARTS == 2, "eight fp32 take two parts' place");
#pragma unroll
        for (int i = 0; i < 8; ++i) bits4[i / 4][i % 4] = __float_as_uint(v[i]);
      }
#pragma unroll
      for (int k = 0; k < PARTS; ++k) {
        uint4* const to = p.t + (((int64_t(blockIdx.x) * p.per_block + ti) * p.kcs + kc) * PARTS + k) * 64 + ql * 16 + (w & 15);
        *to = uint4{bits4[k][0], bits4[k][1], bits4[k][2], bits4[k][3]};
        if (RC == 1 && j0 % 32 == 0 && p.R <= j0 + 16) to[32] = uint4{0, 0, 0, 0};   // (no other workgroup has that half)
      }
    }
    // (part is written again when all have read it, ts behind the next meeting)
    }
  }
}

// How rows of b lie: of whole eights; of eight elements at least; of fewer.
enum BRows { kEights, kOver, kShort };

// elements j .. j + 7 of a row of R, what lies past the row's end undefined
template <int BR>
__device__ __forceinline__ uint4 load_row(const uint8_t* row, int j, int R) {
  if constexpr (BR == kEights) {
    return load_any<uint4>(row + 2 * min(j, R - 8));
  } else if constexpr (BR == kOver) {   // the row's last eight, moved down, where fewer are left
    const int from = min(j, R - 8), bits = 16 * min(j - from, 7);
    const uint4 w = load_any<uint4>(row + 2 * from);
    const uint64_t lo = uint64_t(w.y) << 32 | w.x, hi = uint64_t(w.w) << 32 | w.z;
    const uint64_t down = lo >> (bits & 63) | (bits & 63 ? hi << (64 - (bits & 63)) : 0), top = hi >> (bits & 63);
    const uint64_t l = bits < 64 ? down : top, h = bits < 64 ? top : 0;
    return uint4{uint32_t(l), uint32_t(l >> 32), uint32_t(h), uint32_t(h >> 32)};
  } else {
    uint32_t d[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] = *reinterpret_cast<const uint16_t*>(row + 2 * min(i, R - 1));
    return uint4{d[0] | d[1] << 16, d[2] | d[3] << 16, d[4] | d[5] << 16, d[6] | d[7] << 16};
  }
}

// out[m, n] = y[m, n] + sum_j t[m, j] b[n, j].  A wave takes up to TILES tiles and 64
// outputs, once: all of their y and b's rows are asked for at the start, and the many
// waves of a CU keep the memory busy (waves that walked along n with the next outputs'
// loads ahead took 164 to 218 us for 8192 tokens).  b's rows are the first operand in
// an order that leaves 16 bytes of a token to a lane and 64 to four; t comes from LDS
// (from memory, each wave for itself: 37 us more).  No load hangs
// on a branch: lanes past a tile's tokens and ranks past the adapter's repeat others,
// and are masked where they are used.  The last outputs of a row that is no multiple of
// 64 go one by one.  Bound by y and out: 8192 x 14336 bf16 132 us (3.6 TB/s of the two),
// 333 x 50257 fp32 30 (4.5 TB/s).  The way of t in fp32 costs fp16 up to 4 % in registers (both
// launches, 8192 x 14336 of 8 x 64 ranks 201 and 208 us); with up to 32 ranks and four tiles, three waves
// of a SIMD hold what four spill (12 ranks 176 us, so 167).
template <int DT, int DY, int R32, int TOK, int PARTS, int BR, int TILES>
__global__ __launch_bounds__(kUBlock, R32 == 1 && DT == ARCHEAD_F16 && TILES > 1 ? 3 : R32 <= 2 ? 4 : R32 == 4 ? 2 : 1) void k_adapt_up(AdaptArgs p) {
  constexpr int YB = Eight<DY>::kBytes;
  const int lane = threadIdx.x & 63, lr = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t m0 = int64_t(blockIdx.z) * TOK;
  const Groups<TOK>& g = reinterpret_cast<const Groups<TOK>*>(p.table)[blockIdx.z];
  extern __shared__ __align__(16) uint4 adapt_t[];   // [TILES][kcs][PARTS][64]
  const int64_t n0 = (int64_t(blockIdx.x) * kUWaves + wave) * 64;
  const int tiles = g.tiles, t0 = int(blockIdx.y) * TILES;
  if (t0 >= tiles) return;
  const bool whole = n0 + 64 <= p.N;
  // A lane's results of the four products: 16 c + 4 q .. + 3 for fp32 outputs, and for
  // 16-bit ones eight neighbours of two, so that 16 bytes a lane are 64 of a token.
  constexpr bool F32 = DY == ARCHEAD_F32;
  auto b_row = [&](int c) { return F32 ? 16 * c + lr : 32 * (c >> 1) + 8 * (lr >> 2) + 4 * (c & 1) + (lr & 3); };
  auto n_of = [&](int i) { return F32 ? 16 * (i / 4) + 4 * q + i % 4 : 32 * (i / 8) + 8 * q + i % 8; };
  int64_t at[TILES];
  int id[TILES];
#pragma unroll
  for (int u = 0; u < TILES; ++u) {
    const int ti = min(t0 + u, tiles - 1), len = t0 + u < tiles ? g.len[ti] : 0;
    at[u] = m0 + g.token[g.first[ti] + (lr < len ? lr : 0)];
    id[u] = g.adapter[ti];
  }
  constexpr int NY = F32 ? 4 : 2;   // 16 bytes a lane
  uint4 yv[TILES][NY], bv[4][R32];
  auto fetch_b = [&](int id) {
    const uint8_t* const b = p.b + std::max(id, 0) * p.b_ad;   // (a tile without an adapter does not use it)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint8_t* const row = b + std::min(n0 + b_row(c), p.N - 1) * p.b_row;
#pragma unroll
      for (int kc = 0; kc < R32; ++kc) bv[c][kc] = load_row<BR>(row, 32 * kc + 8 * q, p.R);
    }
  };
  const int n_t = std::min(TILES, tiles - t0) * p.kcs * PARTS * 64;
  const uint4* const t = p.t + (int64_t(blockIdx.z) * p.per_block + t0) * p.kcs * PARTS * 64;
  for (int i = threadIdx.x; i < n_t; i += kUBlock) adapt_t[i] = t[i];
  if (whole)
#pragma unroll
    for (int u = 0; u < TILES; ++u)
#pragma unroll
      for (int i = 0; i < NY; ++i) yv[u][i] = load_any<uint4>(p.y + at[u] * p.y_row + (n0 + n_of(i * (16 / NY))) * YB);
  fetch_b(id[0]);
  __syncthreads();
  if (n0 >= p.N) return;
#pragma unroll
  for (int u = 0; u < TILES; ++u) {
    if (t0 + u >= tiles) break;
    const int ti = t0 + u, rank = g.rank[ti];
    if (u > 0 && id[u] != id[u > 0 ? u - 1 : 0]) fetch_b(id[u]);
    f32x4 sum[4] = {};
#pragma unroll
    for (int kc = 0; kc < R32; ++kc) {
      if (32 * kc >= rank) break;
      f32x4 acc[4] = {};
      const int64_t op = (int64_t(blockIdx.z) * p.per_block + ti) * p.kcs + kc;
      uint4 tv[PARTS];
#pragma unroll
      for (int k = 0; k < PARTS; ++k) tv[k] = adapt_t[((u * p.kcs + kc) * PARTS + k) * 64 + lane];
      if (rank < 32 * kc + 32) {   // b past the adapter's rank is not looked at
        const int j = 32 * kc + 8 * q;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint4& w = bv[c][kc];
          uint32_t d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) d[i] = j + 2 * i + 1 < rank ? d[i] : j + 2 * i < rank ? d[i] & 0xffffu : 0u;
          w = uint4{d[0], d[1], d[2], d[3]};
        }
      }
      float by = 1;
      if constexpr (DT == ARCHEAD_F16) by = p.back[op * 16 + lr];
      if (DT == ARCHEAD_F16 && __builtin_expect(int(__builtin_amdgcn_readfirstlane(__float_as_uint(by))) < 0, 0)) {
        // t in fp32: products of fp32, of the ranks 8 q + i in turn
        by = 1;
        Eight<ARCHEAD_F32> t;
        t.w[0] = tv[0], t.w[1] = tv[1];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          Eight<ARCHEAD_F16> e;
          e.w[0] = bv[c][kc];
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(e.at(i), t.at(i), acc[c], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);   // (one row's numbers at a time in registers: without it 231 us for 208 below)
        }
      } else {
#pragma unroll
        for (int k = 0; k < PARTS; ++k)
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[c] = mma<DT>(bv[c][kc], tv[k], acc[c]);
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) sum[c] += DT == ARCHEAD_F16 ? acc[c] * by : acc[c];
    }
    if (lr >= g.len[ti]) continue;
    uint8_t* const out = p.out + at[u] * p.o_row;
    if (whole) {
#pragma unroll
      for (int i = 0; i < NY; ++i) {
        if (id[u] >= 0) {   // (else y itself: y + 0 loses the sign of a zero)
          if constexpr (F32) {
            yv[u][i] = __builtin_bit_cast(uint4, __builtin_bit_cast(f32x4, yv[u][i]) + sum[i]);
          } else {
            Eight<DY> was;
            was.w[0] = yv[u][i];
            f32x8 v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = was.at(e) + sum[2 * i + e / 4][e % 4];
            if constexpr (DY == ARCHEAD_BF16) yv[u][i] = __builtin_bit_cast(uint4, __builtin_convertvector(v, bf16x8));
            else yv[u][i] = __builtin_bit_cast(uint4, __builtin_convertvector(v, f16x8));
          }
        }
        store_any(out + (n0 + n_of(i * (16 / NY))) * YB, yv[u][i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int64_t n = n0 + n_of(i);
        if (n >= p.N) continue;
        auto go = [&](auto* type) {
          typedef std::remove_pointer_t<decltype(type)> T;
          const T was = reinterpret_cast<const T*>(p.y + at[u] * p.y_row)[n];
          reinterpret_cast<T*>(out)[n] = id[u] >= 0 ? T(float(was) + sum[i / 4][i % 4]) : was;
        };
        if constexpr (DY == ARCHEAD_F32) go(static_cast<float*>(nullptr));
        else if constexpr (DY == ARCHEAD_BF16) go(static_cast<__bf16*>(nullptr));
        else go(static_cast<_Float16*>(nullptr));
      }
    }
  }
}

// rows of y where there is nothing to add
__global__ __launch_bounds__(kUBlock) void k_adapt_copy(const uint8_t* y, int64_t y_row, uint8_t* out, int64_t o_row, int64_t bytes) {
  const uint8_t* const from = y + int64_t(blockIdx.x) * y_row;
  uint8_t* const to = out + int64_t(blockIdx.x) * o_row;
  for (int64_t j = threadIdx.x * 2; j < bytes; j += kUBlock * 2)
    *reinterpret_cast<uint16_t*>(to + j) = *reinterpret_cast<const uint16_t*>(from + j);
}

// Sizes of a call's launches.
struct Shape {
  int tok;                 // tokens of a block
  int64_t blocks, in_block;   // tiles of 16 tokens of one adapter that a block may hold
  int kcs;                 // operands of 32 ranks
};
Shape shape(int64_t M, int64_t R, int64_t n) {
  Shape s{};
  // (of 16 tokens both launches took 13.0 us in a block of 64, 15.1 in one of 256; of 256 in four
  // blocks 26.7, in one 23.3)
  s.tok = M <= 64 ? 64 : 256;
  s.blocks = (M + s.tok - 1) / s.tok;
  const int64_t in = std::min<int64_t>(s.tok, M);
  s.in_block = std::min(in, n + 1 + in / 16);
  s.kcs = int((R + 31) / 32);
  return s;
}
constexpr int parts_of(int x_dtype, int y_dtype) { return y_dtype == ARCHEAD_F32 && x_dtype == ARCHEAD_BF16 ? 3 : 2; }

template <int DT, int TOK, int PARTS>
hipError_t down(AdaptArgs p, const Shape& sh, hipStream_t s) {
  // As many ranks to a workgroup as leave one for every CU, by the tiles that there may be, so
  // that fewer load each x (4096 wide, both launches at N = 1024, 16 / 32 / 64 ranks a workgroup:
  // 1024 tokens, 8 adapters of 64 ranks 29 / 29 / 35 us; 2048, 64 of 64 77 / 67 / 61; 8192, 64 of
  // 64 230 / 172 / 155; 1024, 8 of 32 23 / 26).  Two tiles, which then share the loads of a, where
  // most have a neighbour of their adapter (8192 tokens of 64 ranks, one tile and two: 1 adapter
  // 61 and 47 us, 8 adapters in any order 60 and 72, in runs of tokens 63 and 60 alone).  fp16's
  // powers of two are of 32 ranks.
  const int r16 = (p.R + 15) / 16;
  const auto go = [&](auto k, int rc, int waves, int tt) {
    p.spread = int((sh.in_block + tt - 1) / tt);
    return launch_kernel(k, dim3(unsigned(sh.blocks), unsigned((r16 + rc - 1) / rc), unsigned(p.spread)), dim3(64 * waves), 0, s, p);
  };
  const int64_t most = sh.blocks * sh.in_block;   // tiles
  if constexpr (TOK == 256)
    if (r16 >= 3 && p.n <= 4 && most * ((r16 + 3) / 4) >= 512) return go(k_adapt_down<DT, 4, TOK, PARTS, 8, 2>, 4, 8, 2);
  if (r16 >= 3 && most * ((r16 + 3) / 4) >= 250) return go(k_adapt_down<DT, 4, TOK, PARTS, 8, 1>, 4, 8, 1);
  if constexpr (DT == ARCHEAD_F16) return go(k_adapt_down<DT, 2, TOK, PARTS, 8, 1>, 2, 8, 1);
  else if (r16 >= 2 && most * r16 / 2 >= 200) return go(k_adapt_down<DT, 2, TOK, PARTS, 8, 1>, 2, 8, 1);
  else return go(k_adapt_down<DT, 1, TOK, PARTS, 8, 1>, 1, 8, 1);
}

template <int DT, int DY, int R32, int TOK, int BR, int TILES>
hipError_t up(const AdaptArgs& p, const Shape& sh, hipStream_t s) {
  const dim3 grid(unsigned((p.N + 64 * kUWaves - 1) / (64 * kUWaves)), unsigned((sh.in_block + TILES - 1) / TILES), unsigned(sh.blocks));
  return launch_kernel(k_adapt_up<DT, DY, R32, TOK, parts_of(DT, DY), BR, TILES>, grid, dim3(kUBlock), size_t(TILES) * sh.kcs * parts_of(DT, DY) * 1024, s, p);
}
// Four tiles to a wave (fp32 outputs two), which share b's rows where they are of one adapter,
// where a block of 256 tokens may have whole tiles of each and the waves are plenty (one tile and
// four: 8192 x 14336, 8 adapters of 64 ranks 257 and 219 us, 32 393 and 403, 128 1021 and 1088;
// 2048 x 14336, 8 of 16 40.7 and 43.6; 4096 x 14336, 8 of 16 77 and 76).
template <int DT, int DY, int R32, int TOK, int BR>
hipError_t up_tiles(const AdaptArgs& p, const Shape& sh, hipStream_t s) {
  constexpr int MANY = R32 <= 2 && DY != ARCHEAD_F32 ? 4 : 2;
  if constexpr (TOK == 256)
    if (p.n <= 16 && p.M * p.N >= (1 << 25)) return up<DT, DY, R32, TOK, BR, MANY>(p, sh, s);
  return up<DT, DY, R32, TOK, BR, 1>(p, sh, s);
}
template <int DT, int DY, int TOK, int BR>
hipError_t up_rank(const AdaptArgs& p, const Shape& sh, hipStream_t s) {
  if (p.R <= 32) return up_tiles<DT, DY, 1, TOK, BR>(p, sh, s);
  if constexpr (BR == kShort) return hipErrorInvalidValue;   // (of fewer than eight ranks)
  else if (p.R <= 64) return up_tiles<DT, DY, 2, TOK, BR>(p, sh, s);
  else if (p.R <= 128) return up_tiles<DT, DY, 4, TOK, BR>(p, sh, s);
  else return up_tiles<DT, DY, 8, TOK, BR>(p, sh, s);
}
template <int DT, int TOK, int BR>
hipError_t up_type(const AdaptArgs& p, archead_dtype y, const Shape& sh, hipStream_t s) {
  return y == ARCHEAD_F32    ? up_rank<DT, ARCHEAD_F32, TOK, BR>(p, sh, s)
         : y == ARCHEAD_BF16 ? up_rank<DT, ARCHEAD_BF16, TOK, BR>(p, sh, s)
                             : up_rank<DT, ARCHEAD_F16, TOK, BR>(p, sh, s);
}

template <int DT, int TOK>
hipError_t launch_tok(const AdaptArgs& p, archead_dtype y, const Shape& sh, hipStream_t s) {
  hipError_t e;
  if constexpr (DT == ARCHEAD_BF16)
    e = parts_of(DT, y) == 3 ? down<DT, TOK, 3>(p, sh, s) : down<DT, TOK, 2>(p, sh, s);
  else
    e = down<DT, TOK, 2>(p, sh, s);
  if (e != hipSuccess) return e;
  return p.R % 8 == 0 ? up_type<DT, TOK, kEights>(p, y, sh, s)
         : p.R > 8    ? up_type<DT, TOK, kOver>(p, y, sh, s)
                      : up_type<DT, TOK, kShort>(p, y, sh, s);
}

// What a call keeps in its workspace, offsets in bytes.
struct Space {
  size_t t, back, total;   // (the blocks' groups first)
};
Space space(const Shape& s) {
  const size_t tiles = size_t(s.blocks) * s.in_block;
  auto up256 = [](size_t v) { return (v + 255) / 256 * 256; };
  Space w{};
  w.t = up256(s.blocks * (s.tok == 64 ? sizeof(Groups<64>) : sizeof(Groups<256>)));
  w.back = w.t + tiles * s.kcs * 3 * 1024;
  w.total = w.back + up256(tiles * s.kcs * 64);
  return w;
}

}  // namespace

extern "C" size_t archead_adapters_workspace_bytes(int64_t M, int64_t K, int64_t R, int64_t n) {
  if (M < 1 || K < 1 || R < 1 || n < 1 || M > kMaxM || K > (1 << 24) || R > kMaxRank) return 0;
  return space(shape(M, R, n)).total;
}

extern "C" archead_status archead_adapters_add(const void* y, archead_dtype y_dtype, int64_t ldy, const void* x,
                                               archead_dtype x_dtype, int64_t ldx, const archead_adapters* ad,
                                               const void* ids, archead_dtype ids_dtype, int64_t M, int64_t N,
                                               int64_t K, void* out, int64_t ldo, void* ws, size_t ws_bytes,
                                               void* stream) {
  using archead::fail;
  archead::clear_error();
  if (!float_dtype(y_dtype)) return fail(ARCHEAD_E_INVALID_ARG, "y_dtype must be F32, BF16 or F16");
  if (x_dtype != ARCHEAD_BF16 && x_dtype != ARCHEAD_F16) return fail(ARCHEAD_E_INVALID_ARG, "x_dtype must be BF16 or F16");
  if (ids_dtype != ARCHEAD_I32 && ids_dtype != ARCHEAD_I64) return fail(ARCHEAD_E_INVALID_ARG, "ids_dtype must be I32 or I64");
  if (M < 0 || M > kMaxM || N < 0 || N > (1 << 23) || K < 0 || K > (1 << 24))
    return fail(ARCHEAD_E_INVALID_ARG, "M = %lld, N = %lld, K = %lld out of range", (long long)M, (long long)N, (long long)K);
  if (!ad) return fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if (ad->n < 0 || ad->n >= (1 << 22) || ad->R < 0) return fail(ARCHEAD_E_INVALID_ARG, "n or R out of range");
  if (ad->R > kMaxRank) return fail(ARCHEAD_E_UNSUPPORTED, "R = %lld > %lld", (long long)ad->R, (long long)kMaxRank);
  if (M == 0 || N == 0) return ARCHEAD_OK;
  const bool any = ad->n > 0 && ad->R > 0 && K > 0;
  if (ldy < N || ldo < N || (any && ldx < K)) return fail(ARCHEAD_E_INVALID_ARG, "leading dimensions must be >= N, N and K");
  const int64_t most = int64_t(1) << 40;
  if (any && (ad->a_adapter < 0 || ad->b_adapter < 0 || ad->a_row < K || ad->b_row < ad->R || ad->a_adapter > most ||
              ad->b_adapter > most || ad->a_row > most || ad->b_row > most))
    return fail(ARCHEAD_E_INVALID_ARG, "strides of a or b out of range");
  if (!y || !out || !ids || (any && (!x || !ad->a || !ad->b))) return fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if (out == y && ldo != ldy) return fail(ARCHEAD_E_INVALID_ARG, "in place, ldo must be ldy");
  const int yb = dtype_bytes(y_dtype);
  if (!aligned(y, yb) || !aligned(out, yb) || !aligned(x, 2) || !aligned(ad->a, 2) || !aligned(ad->b, 2) ||
      !aligned(ad->scales, 4) || !aligned(ad->ranks, 4) || !aligned(ids, ids_dtype == ARCHEAD_I64 ? 8 : 4))
    return fail(ARCHEAD_E_MISALIGNED, "a pointer is misaligned");
  if (any) {
    if (!ws) return fail(ARCHEAD_E_INVALID_ARG, "null workspace");
    if (!aligned(ws, 256)) return fail(ARCHEAD_E_MISALIGNED, "workspace must be 256-byte aligned");
    if (ws_bytes < archead_adapters_workspace_bytes(M, K, ad->R, ad->n))
      return fail(ARCHEAD_E_WORKSPACE, "workspace of %zu bytes is too small", ws_bytes);
  } else if (out == y) {
    return ARCHEAD_OK;
  }
  AdaptArgs p{};
  p.y = static_cast<const uint8_t*>(y);
  p.x = static_cast<const uint8_t*>(x);
  p.a = static_cast<const uint8_t*>(ad->a);
  p.b = static_cast<const uint8_t*>(ad->b);
  p.ids = ids;
  p.scales = ad->scales;
  p.ranks = ad->ranks;
  p.out = static_cast<uint8_t*>(out);
  p.M = M, p.N = N, p.K = K, p.n = any ? ad->n : 0;
  p.y_row = ldy * yb, p.x_row = ldx * 2, p.o_row = ldo * yb;
  p.a_ad = ad->a_adapter * 2, p.a_row = ad->a_row * 2, p.b_ad = ad->b_adapter * 2, p.b_row = ad->b_row * 2;
  p.R = int(ad->R);
  p.ids64 = ids_dtype == ARCHEAD_I64, p.in_place = out == y;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!any)
    return launch_status(launch_kernel(k_adapt_copy, dim3(unsigned(M)), dim3(kUBlock), 0, s, p.y, p.y_row, p.out, p.o_row, N * yb),
                         "adapters launch");
  const Shape sh = shape(M, ad->R, ad->n);
  const Space w = space(sh);
  p.kcs = sh.kcs, p.per_block = int(sh.in_block);
  p.table = static_cast<uint8_t*>(ws);
  p.t = reinterpret_cast<uint4*>(p.table + w.t);
  p.back = reinterpret_cast<float*>(p.table + w.back);
  const bool bf = x_dtype == ARCHEAD_BF16, few = sh.tok == 64;
  return launch_status(bf ? (few ? launch_tok<ARCHEAD_BF16, 64>(p, y_dtype, sh, s) : launch_tok<ARCHEAD_BF16, 256>(p, y_dtype, sh, s))
                          : (few ? launch_tok<ARCHEAD_F16, 64>(p, y_dtype, sh, s) : launch_tok<ARCHEAD_F16, 256>(p, y_dtype, sh, s)),
                       "adapters launch");
}
