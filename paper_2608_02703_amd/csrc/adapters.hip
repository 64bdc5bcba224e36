// archead_adapters_add: low-rank adapters of many requests at once.
#include <algorithm>
#include <type_traits>

#include "dev_rows.cuh"

namespace {

using namespace archead::rows;

constexpr int kUBlock = 256, kUWaves = kUBlock / 64;   // threads and waves of the outer products' workgroups
constexpr int kDBlock = 512, kDWaves = kDBlock / 64;   // of the inner ones'
constexpr int64_t kMaxRank = 256;
constexpr int kMaxSplit = 4;             // parts of K over workgroups at most
constexpr size_t kTileLds = 40 * 1024;   // of a workgroup's tokens in LDS

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
  float* t;                // [splits][M][rank16]
  uint8_t* table;          // Groups of the blocks
  int64_t M, N, K, n;
  int64_t y_row, x_row, a_ad, a_row, b_ad, b_row, o_row;   // bytes
  int R, rank16;
  int splits, k_split;     // parts of K, elements of each
  int spread;              // workgroups that share a block's tiles
  int n_wg;                // outputs of a token per workgroup
  int tiles_most;          // tiles of a workgroup of the outer products at most
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

// t[m, j] = sum_k x[m, k] a[j, k] over one part of K, fp32.  A workgroup takes a tile
// of up to 16 tokens of one adapter and RC x 16 ranks, its waves shares of the
// part of K, whose sums meet in LDS.  Both operands come straight from memory (16
// rows of 64 bytes a load), the ranks as the first, so a lane's results are four
// neighbouring ones of a token.  Lanes past the tile's tokens or the adapter's ranks
// repeat the first: their results are not stored, and no load hangs on a branch.
template <int DT, int RC, int TOK>
__global__ __launch_bounds__(kDBlock, 4) void k_adapt_down(AdaptArgs p) {
  __shared__ Groups<TOK> g;
  constexpr int STEPS = RC == 4 ? 4 : 8;
  __shared__ f32x4 part[kDWaves][RC][64];
  const int64_t m0 = int64_t(blockIdx.x) * TOK;
  group_tokens(g, p, m0, !p.in_place);
  if (blockIdx.y == 0 && blockIdx.z == 0)   // for k_adapt_up
    for (int i = threadIdx.x; i < int(sizeof(g) / 16); i += kDBlock)
      reinterpret_cast<uint4*>(p.table + blockIdx.x * sizeof(g))[i] = reinterpret_cast<const uint4*>(&g)[i];
  const int lane = threadIdx.x & 63, lr = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;
  const int split = int(blockIdx.y) % p.splits, j0 = int(blockIdx.y) / p.splits * 16 * RC;
  // the waves take pieces of the part in turn (rows of a power of two would have them
  // all ask for the same memory channels with shares one behind another), then 32 at a time of the rest
  constexpr int PIECE = 32 * STEPS;
  const int K = int(p.K), begin = split * p.k_split, end = min(K, begin + p.k_split);
  const int pieces = (end - begin) / PIECE, rest = begin + pieces * PIECE;
  for (int ti = int(blockIdx.z); ti < g.tiles; ti += p.spread) {
    const int64_t id = g.adapter[ti];
    const int rank = g.rank[ti];
    if (j0 >= rank) continue;
    const bool there = lr < g.len[ti];
    const int64_t m = m0 + g.token[g.first[ti] + (there ? lr : 0)];
    const uint8_t* const x = p.x + m * p.x_row;
    const uint8_t* a[RC];
#pragma unroll
    for (int c = 0; c < RC; ++c) {
      const int j = j0 + 16 * c + lr;
      a[c] = p.a + id * p.a_ad + (j < rank ? j : 0) * p.a_row;
    }
    f32x4 acc[RC] = {};
    for (int i = wave; i < pieces; i += kDWaves) {   // all loads of a piece, then its products
      uint4 xv[STEPS], av[STEPS][RC];
#pragma unroll
      for (int j = 0; j < STEPS; ++j) {
        const int at = 2 * (begin + i * PIECE + 32 * j + 8 * q);
        xv[j] = load_any<uint4>(x + at);
#pragma unroll
        for (int c = 0; c < RC; ++c) av[j][c] = load_any<uint4>(a[c] + at);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < STEPS; ++j)
#pragma unroll
        for (int c = 0; c < RC; ++c) acc[c] = mma<DT>(av[j][c], xv[j], acc[c]);
    }
    const int last = rest + 32 * wave;   // (a piece is at most eight times 32)
    if (last < end) {                    // zeros past K
      Eight<ARCHEAD_BF16> e;
      e.load(x, last + 8 * q, K, 0);
      const uint4 xv = e.w[0];
#pragma unroll
      for (int c = 0; c < RC; ++c) {
        e.load(a[c], last + 8 * q, K, 0);
        acc[c] = mma<DT>(e.w[0], xv, acc[c]);
      }
    }
#pragma unroll
    for (int c = 0; c < RC; ++c) part[wave][c][lane] = acc[c];
    __syncthreads();
    if (wave < RC) {
      f32x4 sum = part[0][wave][lane];
#pragma unroll
      for (int w = 1; w < kDWaves; ++w) sum += part[w][wave][lane];
      if (there && j0 + 16 * wave < rank)
        *reinterpret_cast<f32x4*>(p.t + (int64_t(split) * p.M + m) * p.rank16 + j0 + 16 * wave + 4 * q) = sum;
    }
    __syncthreads();
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

// out[m, n] = y[m, n] + sum_j t[m, j] b[n, j], t = scale times the sum of its parts.
// t goes through the matrix units in PARTS parts of the operands' type: two hold 17
// bits of it in bf16 and 22 in fp16 (there after a power of two that brings a
// token's largest to 2^14, so that no part is below the normal numbers), three 25.
// The workgroup holds the parts of its tokens in LDS; a wave takes 64 outputs of
// a tile at a time, the rows of b as the first operand in an order that leaves a lane
// with eight neighbouring outputs of a token twice.
//
// The loads of the next tile are on their way while one is computed, so none of them
// may hang on a branch: lanes past a tile's tokens, items past the last and ranks
// past the adapter's repeat others, and are masked where they are used.  HOLD: b's
// rows stay in registers over the tiles of one adapter; else every tile loads its
// own.  Only the last outputs of a row that is no multiple of 64 go one by one.
// Bound by y and out.
template <int DT, int DY, int R32, int TOK, int PARTS, int BR, bool HOLD>
__global__ __launch_bounds__(kUBlock, R32 <= 2 ? 4 : R32 == 4 ? 2 : 1) void k_adapt_up(AdaptArgs p) {
  constexpr int YB = Eight<DY>::kBytes, ROW = R32 * 32 + 8;   // elements of a token's row in LDS
  __shared__ Groups<TOK> g;
  __shared__ float back[TOK];    // fp16: the power of two to take out again
  extern __shared__ __align__(16) uint16_t adapt_t[];          // [PARTS][16 tiles_most][ROW]
  const int64_t m0 = int64_t(blockIdx.x) * TOK;
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, q = lane >> 4, wave = tid >> 6;
  for (int i = tid; i < int(sizeof(g) / 16); i += kUBlock)
    reinterpret_cast<uint4*>(&g)[i] = reinterpret_cast<const uint4*>(p.table + blockIdx.x * sizeof(g))[i];
  __syncthreads();
  const int z = int(blockIdx.z), tiles = g.tiles > z ? (g.tiles - z + p.spread - 1) / p.spread : 0;   // of this workgroup
  if (tiles == 0) return;
  auto adapter_of = [&](int u) { return __builtin_amdgcn_readfirstlane(g.adapter[z + u * p.spread]); };
  auto token_of = [&](int u) {
    const int ti = z + u * p.spread;
    return m0 + g.token[g.first[ti] + (lr < g.len[ti] ? lr : 0)];
  };
  int b_row[4];   // this lane's rows of b, from an item's first one on
#pragma unroll
  for (int c = 0; c < 4; ++c) b_row[c] = 32 * (c >> 1) + 8 * (lr >> 2) + 4 * (c & 1) + (lr & 3);
  // eight outputs of a lane, twice: y's and where they lie
  struct Held {
    Eight<DY> y[2];
    uint4 b[HOLD ? 1 : 4][R32];
  };
  constexpr int BATCH = !HOLD ? 2 : R32 <= 2 && DY != ARCHEAD_F32 ? 4 : 2;
  uint4 bh[4][R32];
  Held held[BATCH];
  auto fetch_y = [&](Held& h, int u, int64_t n0) {
    const uint8_t* const y = p.y + token_of(u) * p.y_row;
#pragma unroll
    for (int i = 0; i < 2; ++i) h.y[i].load(y, n0 + 32 * i + 8 * q, INT64_MAX, 0);
  };
  auto fetch_b = [&](uint4 (&b)[4][R32], int u, int64_t n0) {
    const int64_t id = max(adapter_of(u), 0);   // (a tile without one does not use them)
    const uint8_t* const rows = p.b + id * p.b_ad;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint8_t* const row = rows + std::min(n0 + b_row[c], p.N - 1) * p.b_row;
#pragma unroll
      for (int kc = 0; kc < R32; ++kc) b[c][kc] = load_row<BR>(row, 32 * kc + 8 * q, p.R);
    }
  };
  auto products = [&](f32x4 (&acc)[4], uint4 (&b)[4][R32], int u) {
    const int rank = __builtin_amdgcn_readfirstlane(g.rank[z + u * p.spread]);
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[c] = f32x4{0, 0, 0, 0};
    if (rank == 0) return;
#pragma unroll
    for (int kc = 0; kc < R32; ++kc) {
      if (rank < 32 * kc + 32) {   // b past the adapter's rank is not looked at
        const int j = 32 * kc + 8 * q;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint4& w = b[c][kc];
          uint32_t d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) d[i] = j + 2 * i + 1 < rank ? d[i] : j + 2 * i < rank ? d[i] & 0xffffu : 0u;
          w = uint4{d[0], d[1], d[2], d[3]};
        }
      }
#pragma unroll
      for (int k = 0; k < PARTS; ++k) {
        const uint4 tv = *reinterpret_cast<const uint4*>(&adapt_t[((k * p.tiles_most + u) * 16 + lr) * ROW + 32 * kc + 8 * q]);
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = mma<DT>(b[c][kc], tv, acc[c]);
      }
    }
    if constexpr (DT == ARCHEAD_F16) {
      const float by = back[16 * u + lr];
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] *= by;
    }
  };
  auto is_there = [&](int u) { return lr < g.len[z + u * p.spread]; };
  // (where a tile has no adapter, y + 0: the same but for the sign of a zero, so it is not formed)
  auto finish = [&](const Held& h, uint4 (&b)[4][R32], int u, int64_t n0) {
    f32x4 acc[4];
    products(acc, b, u);
    const bool some = adapter_of(u) >= 0;
    uint8_t* const out = p.out + token_of(u) * p.o_row;
    if (!is_there(u)) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f32x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = some ? h.y[i].at(e) + acc[2 * i + e / 4][e % 4] : h.y[i].at(e);
      uint8_t* const to = out + (n0 + 32 * i + 8 * q) * YB;
      if constexpr (DY == ARCHEAD_F32) store_any(to, v);
      else if constexpr (DY == ARCHEAD_BF16) store_any(to, __builtin_convertvector(v, bf16x8));
      else store_any(to, __builtin_convertvector(v, f16x8));
    }
  };
  auto finish_last = [&](int u, int64_t n0) {   // outputs up to N, one by one
    f32x4 acc[4];
    fetch_b(bh, u, n0);
    products(acc, bh, u);
    const bool some = adapter_of(u) >= 0;
    const int64_t m = token_of(u);
    if (!is_there(u)) return;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int64_t n = n0 + 32 * i + 8 * q + e;
        if (n >= p.N) continue;
        const float more = some ? acc[2 * i + e / 4][e % 4] : 0.f;
        auto go = [&](auto* type) {
          typedef std::remove_pointer_t<decltype(type)> T;
          const T v = *reinterpret_cast<const T*>(p.y + m * p.y_row + n * YB);
          *reinterpret_cast<T*>(p.out + m * p.o_row + n * YB) = some ? T(float(v) + more) : v;
        };
        if constexpr (DY == ARCHEAD_F32) go(static_cast<float*>(nullptr));
        else if constexpr (DY == ARCHEAD_BF16) go(static_cast<__bf16*>(nullptr));
        else go(static_cast<_Float16*>(nullptr));
      }
  };

  // t of this workgroup's tiles: 16 lanes a token
  auto stage = [&]() {
#pragma unroll 2
  for (int u = 0; u < tiles; ++u) {
    const int ti = z + u * p.spread, i = tid >> 4, id = max(g.adapter[ti], 0), rank = g.rank[ti];
    const bool there = i < g.len[ti];
    const int64_t m = m0 + g.token[g.first[ti] + (there ? i : 0)];
    const float scale = p.scales ? p.scales[id] : 1.f;
    float v[R32 * 2], top = 0;
#pragma unroll
    for (int c = 0; c < R32 * 2; ++c) {
      const int j = lr + 16 * c;
      const float* const from = p.t + m * p.rank16 + min(j, p.rank16 - 1);
      float sum = from[0];
#pragma unroll
      for (int s = 1; s < kMaxSplit; ++s) {
        const float more = from[int64_t(min(s, p.splits - 1)) * p.M * p.rank16];
        sum += s < p.splits ? more : 0.f;
      }
      v[c] = j < rank ? sum * scale : 0.f;
      top = fmaxf(top, fabsf(v[c]));
    }
    float pre = 1;
    if constexpr (DT == ARCHEAD_F16) {
#pragma unroll
      for (int s = 1; s < 16; s *= 2) top = fmaxf(top, __shfl_xor(top, s));
      int e = 15;
      if (top > 0 && top < INFINITY) frexpf(top, &e);
      e = max(-100, min(100, 15 - e));
      pre = ldexpf(1.f, e);
      if (lr == 0) back[16 * u + i] = ldexpf(1.f, -e);
    }
#pragma unroll
    for (int c = 0; c < R32 * 2; ++c) {
      float rest = v[c] * pre;
#pragma unroll
      for (int k = 0; k < PARTS; ++k) {
        uint16_t bits;
        float part;
        if constexpr (DT == ARCHEAD_BF16) {
          const __bf16 h = __bf16(rest);
          part = float(h);
          __builtin_memcpy(&bits, &h, 2);
        } else {
          const _Float16 h = _Float16(rest);
          part = float(h);
          __builtin_memcpy(&bits, &h, 2);
        }
        adapt_t[((k * p.tiles_most + u) * 16 + i) * ROW + lr + 16 * c] = bits;
        rest = fabsf(part) < INFINITY ? rest - part : 0.f;   // (an infinity or NaN has no rest)
      }
    }
  }
  __syncthreads();
  };

  const int64_t n_begin = int64_t(blockIdx.y) * p.n_wg + 64 * wave, n_end = std::min(p.N, (int64_t(blockIdx.y) + 1) * p.n_wg);
  const int64_t n_whole = std::min(n_end, p.N / 64 * 64);
  constexpr int STEP = 64 * kUWaves;
  const int chunks = n_begin < n_whole ? int((n_whole - n_begin + STEP - 1) / STEP) : 0;   // of 64 outputs, of this wave
  if constexpr (HOLD) {
    stage();
    for (int c = 0; c < chunks; ++c) {
      const int64_t n0 = n_begin + int64_t(c) * STEP;
      for (int u = 0; u < tiles;) {
        const int id = adapter_of(u);
        int end = u + 1;
        while (end < tiles && adapter_of(end) == id) ++end;
        fetch_b(bh, u, n0);
        for (; u < end; u += BATCH) {
#pragma unroll
          for (int i = 0; i < BATCH; ++i) fetch_y(held[i], min(u + i, end - 1), n0);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = 0; i < BATCH; ++i)
            if (u + i < end) finish(held[i], bh, u + i, n0);
        }
        u = end;
      }
    }
  } else {
    const int items = chunks * tiles;
    auto fetch = [&](Held& h, int i) {
      const int at = min(i, items - 1), c = at / tiles, u = at - c * tiles;
      fetch_y(h, u, n_begin + int64_t(c) * STEP);
      fetch_b(h.b, u, n_begin + int64_t(c) * STEP);
    };
    auto end = [&](Held& h, int i) {
      const int c = i / tiles, u = i - c * tiles;
      finish(h, h.b, u, n_begin + int64_t(c) * STEP);
    };
    if (items > 0) fetch(held[0], 0);
    stage();
    for (int i = 0; i < items; i += 2) {
      fetch(held[1], i + 1);
      end(held[0], i);
      fetch(held[0], i + 2);
      if (i + 1 < items) end(held[1], i + 1);
    }
  }
  const int64_t n_last = p.N / 64 * 64;   // (at most one wave of a block has it)
  if (n_last < p.N && n_last >= n_begin && n_last < n_end && (n_last - n_begin) % STEP == 0)
    for (int u = 0; u < tiles; ++u) finish_last(u, n_last);
}

// rows of y where there is nothing to add
__global__ __launch_bounds__(kUBlock) void k_adapt_copy(const uint8_t* y, int64_t y_row, uint8_t* out, int64_t o_row, int64_t bytes) {
  const uint8_t* const from = y + int64_t(blockIdx.x) * y_row;
  uint8_t* const to = out + int64_t(blockIdx.x) * o_row;
  for (int64_t j = threadIdx.x * 2; j < bytes; j += kUBlock * 2)
    *reinterpret_cast<uint16_t*>(to + j) = *reinterpret_cast<const uint16_t*>(from + j);
}

// Sizes of a call's launches, from its sizes alone, so that its sums have one order.
struct Shape {
  int tok;                 // tokens of a block
  int64_t tiles, in_block; // of 16 tokens of one adapter, in all and in a block: about as many as there may be
  int rc, groups;          // ranks of a workgroup in sixteens, groups of them
  int splits;
};
Shape shape(int64_t M, int64_t K, int64_t R, int64_t n) {
  Shape s{};
  s.tok = M <= 64 ? 64 : 256;
  const int64_t blocks = (M + s.tok - 1) / s.tok, in = std::min<int64_t>(s.tok, M);
  s.in_block = std::min(in, n + 1 + in / 16);
  s.tiles = blocks * s.in_block;
  const int r16 = int((R + 15) / 16);
  s.rc = r16 >= 3 ? 4 : r16 == 2 ? 2 : 1;
  while (s.rc > 1 && s.tiles * ((r16 + s.rc - 1) / s.rc) < 256) s.rc /= 2;
  s.groups = (r16 + s.rc - 1) / s.rc;
  s.splits = 1;
  while (s.splits < kMaxSplit && s.tiles * s.groups * s.splits < 128 && K / s.splits >= 4096) s.splits *= 2;
  return s;
}

size_t table_bytes(int64_t M, const Shape& s) {
  return (size_t((M + s.tok - 1) / s.tok) * (s.tok == 64 ? sizeof(Groups<64>) : sizeof(Groups<256>)) + 255) / 256 * 256;
}

template <int DT, int TOK>
hipError_t down(const AdaptArgs& p, int rc, dim3 grid, hipStream_t s) {
  const auto go = [&](auto k) { return launch_kernel(k, grid, dim3(kDBlock), 0, s, p); };
  return rc == 1 ? go(k_adapt_down<DT, 1, TOK>) : rc == 2 ? go(k_adapt_down<DT, 2, TOK>) : go(k_adapt_down<DT, 4, TOK>);
}

template <int DT, int DY, int R32, int TOK, int BR, bool HOLD>
hipError_t up(AdaptArgs p, const Shape& sh, hipStream_t s) {
  constexpr int PARTS = DY == ARCHEAD_F32 && DT == ARCHEAD_BF16 ? 3 : 2;
  constexpr size_t TILE = size_t(PARTS) * 16 * (R32 * 32 + 8) * 2;
  const int64_t blocks = (p.M + TOK - 1) / TOK;
  // Up to eight tiles to a workgroup (they share b's rows where they are of one
  // adapter), and as many outputs as leave about four workgroups to a CU (they share t).
  const int64_t chunks = (p.N + 63) / 64, each = (sh.tiles * chunks + 4095) / 4096;
  const int64_t per = each >= 32 ? 8 : each >= 8 ? 4 : each >= 2 ? 2 : 1;
  p.spread = int((sh.in_block + per - 1) / per);
  constexpr int64_t STEP = 64 * kUWaves;
  const int64_t steps = (p.N + STEP - 1) / STEP, wide = std::max<int64_t>(1, std::min(steps, 1024 / (blocks * p.spread)));
  p.n_wg = int(STEP * ((steps + wide - 1) / wide));
  // (a block may hold a tile for each of its tokens, or, of few adapters, fewer)
  const int64_t most = std::min<int64_t>(TOK, p.n + 1 + TOK / 16);
  p.tiles_most = int((most + p.spread - 1) / p.spread);
  while (TILE * p.tiles_most > kTileLds && p.tiles_most > 1) {
    ++p.spread;
    p.tiles_most = int((most + p.spread - 1) / p.spread);
  }
  const dim3 grid(static_cast<unsigned>(blocks), unsigned((p.N + p.n_wg - 1) / p.n_wg), unsigned(p.spread));
  return launch_kernel(k_adapt_up<DT, DY, R32, TOK, PARTS, BR, HOLD>, grid, dim3(kUBlock), TILE * p.tiles_most, s, p);
}
// Ranks up to 64: b held where an adapter has 16 tokens of a block or more; the widest always
// (two tiles' rows would not fit the registers).
template <int DT, int DY, int TOK, int BR>
hipError_t up_rank(const AdaptArgs& p, const Shape& sh, hipStream_t s) {
  const bool hold = std::min<int64_t>(TOK, p.M) >= 16 * p.n;
  if (p.R <= 32) return hold ? up<DT, DY, 1, TOK, BR, true>(p, sh, s) : up<DT, DY, 1, TOK, BR, false>(p, sh, s);
  if constexpr (BR == kShort) return hipErrorInvalidValue;   // (of fewer than eight ranks)
  else if (p.R <= 64) return hold ? up<DT, DY, 2, TOK, BR, true>(p, sh, s) : up<DT, DY, 2, TOK, BR, false>(p, sh, s);
  else if (p.R <= 128) return up<DT, DY, 4, TOK, BR, true>(p, sh, s);
  else return up<DT, DY, 8, TOK, BR, true>(p, sh, s);
}
template <int DT, int TOK, int BR>
hipError_t up_type(const AdaptArgs& p, archead_dtype y, const Shape& sh, hipStream_t s) {
  return y == ARCHEAD_F32    ? up_rank<DT, ARCHEAD_F32, TOK, BR>(p, sh, s)
         : y == ARCHEAD_BF16 ? up_rank<DT, ARCHEAD_BF16, TOK, BR>(p, sh, s)
                             : up_rank<DT, ARCHEAD_F16, TOK, BR>(p, sh, s);
}

template <int DT, int TOK>
hipError_t launch_tok(AdaptArgs p, archead_dtype y, const Shape& sh, hipStream_t s) {
  const int64_t blocks = (p.M + TOK - 1) / TOK;
  p.k_split = int(((p.K + sh.splits - 1) / sh.splits + 255) / 256 * 256);
  p.splits = int((p.K + p.k_split - 1) / p.k_split);
  p.spread = int(std::max<int64_t>(1, std::min(sh.in_block, 4096 / (blocks * p.splits * sh.groups))));
  const hipError_t e =
      down<DT, TOK>(p, sh.rc, dim3(static_cast<unsigned>(blocks), unsigned(p.splits * sh.groups), unsigned(p.spread)), s);
  if (e != hipSuccess) return e;
  return p.R % 8 == 0 ? up_type<DT, TOK, kEights>(p, y, sh, s)
         : p.R > 8    ? up_type<DT, TOK, kOver>(p, y, sh, s)
                      : up_type<DT, TOK, kShort>(p, y, sh, s);
}
template <int DT>
hipError_t launch(const AdaptArgs& p, archead_dtype y, hipStream_t s) {
  const Shape sh = shape(p.M, p.K, p.R, p.n);
  return sh.tok == 64 ? launch_tok<DT, 64>(p, y, sh, s) : launch_tok<DT, 256>(p, y, sh, s);
}

}  // namespace

extern "C" size_t archead_adapters_workspace_bytes(int64_t M, int64_t K, int64_t R, int64_t n) {
  if (M < 1 || K < 1 || R < 1 || n < 1 || M > INT32_MAX || K > (1 << 24) || R > kMaxRank) return 0;
  const Shape s = shape(M, K, R, n);
  return table_bytes(M, s) + (size_t(s.splits) * M * ((R + 15) / 16 * 16) * 4 + 255) / 256 * 256;
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
  if (M < 0 || M > INT32_MAX || N < 0 || N > (1 << 23) || K < 0 || K > (1 << 24))
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
  p.table = static_cast<uint8_t*>(ws);
  p.t = any ? reinterpret_cast<float*>(p.table + table_bytes(M, shape(M, K, ad->R, ad->n))) : nullptr;
  p.M = M, p.N = N, p.K = K, p.n = any ? ad->n : 0;
  p.y_row = ldy * yb, p.x_row = ldx * 2, p.o_row = ldo * yb;
  p.a_ad = ad->a_adapter * 2, p.a_row = ad->a_row * 2, p.b_ad = ad->b_adapter * 2, p.b_row = ad->b_row * 2;
  p.R = int(ad->R), p.rank16 = int((ad->R + 15) / 16 * 16);
  p.ids64 = ids_dtype == ARCHEAD_I64, p.in_place = out == y;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!any)
    return launch_status(launch_kernel(k_adapt_copy, dim3(unsigned(M)), dim3(kUBlock), 0, s, p.y, p.y_row, p.out, p.o_row, N * yb),
                         "adapters launch");
  return launch_status(x_dtype == ARCHEAD_BF16 ? launch<ARCHEAD_BF16>(p, y_dtype, s) : launch<ARCHEAD_F16>(p, y_dtype, s),
                       "adapters launch");
}
