// archead_adapters_add: low-rank adapters of many requests at once.
#include <algorithm>
#include <atomic>

#include "dev_rows.cuh"

namespace {

using namespace archead::rows;

constexpr int kABlock = 256, kWaves = kABlock / 64;
constexpr int kTok = 64;                 // tokens of a block, grouped by adapter
constexpr int64_t kMaxRank = 256;
constexpr int kMaxSplit = 16;            // parts of K at most

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
  int64_t M, N, K, n;
  int64_t y_row, x_row, a_ad, a_row, b_ad, b_row, o_row;   // bytes
  int R, rank16;
  int splits, k_split;     // parts of K, elements of each
  int spread;              // workgroups that share a block's tiles
  int n_wg;                // outputs of a token per workgroup
  bool ids64, in_place;
};

// The tokens of a block in the order of their adapters, and tiles of up to 16
// tokens of one adapter.
struct Groups {
  int16_t token[kTok];       // place -> token of the block
  int32_t first[kTok];       // of tile: its first place
  int32_t len[kTok];
  int64_t adapter[kTok];     // -1: none
  int tiles;
};

// Sorted by one wave: every lane counts the tokens that come before its own.
// Tokens without an adapter come last, and are left out where `none` is false.
__device__ __forceinline__ void group_tokens(Groups& g, const AdaptArgs& p, int64_t m0, bool none) {
  const int lane = threadIdx.x & 63;
  if (threadIdx.x < 64) {
    const bool there = m0 + lane < p.M;
    int64_t id = -1;
    if (there) id = p.ids64 ? static_cast<const int64_t*>(p.ids)[m0 + lane] : static_cast<const int32_t*>(p.ids)[m0 + lane];
    if (id < 0 || id >= p.n) id = -1;
    // adapters are fewer than 2^30: tokens without one, then lanes without a token, after all others
    const int key = !there ? INT32_MAX : id < 0 ? INT32_MAX - 1 : int(id);
    int place = 0, within = 0, same = 0;
#pragma unroll 8
    for (int l = 0; l < 64; ++l) {
      const int k = __builtin_amdgcn_readlane(key, l);
      place += k < key || (k == key && l < lane);
      within += k == key && l < lane;
      same += k == key;
    }
    const bool start = there && within % 16 == 0 && (id >= 0 || none);
    // tiles in the order of their first places: those of smaller keys, and of the same before this one
    g.token[place] = int16_t(lane);
    int before = 0;
#pragma unroll 8
    for (int l = 0; l < 64; ++l) {
      const int k = __builtin_amdgcn_readlane(place, l), s = __builtin_amdgcn_readlane(int(start), l);
      before += s && k < place;
    }
    if (start) {
      g.first[before] = place;
      g.len[before] = min(16, same - within);
      g.adapter[before] = id;
    }
    const int tiles = __popcll(__ballot(start));
    if (lane == 0) g.tiles = tiles;
  }
  __syncthreads();
}

// eight elements of a 16-bit type as they lie, zeros from element `end` on; ODD:
// rows may end inside the eight
template <bool ODD>
__device__ __forceinline__ uint4 load8(const uint8_t* row, int64_t j, int64_t end) {
  if constexpr (ODD) {
    Eight<ARCHEAD_BF16> e;
    e.load(row, j < end ? j : 0, j < end ? end : 0, 0);
    return e.w[0];
  } else {
    return j < end ? load_any<uint4>(row + 2 * j) : uint4{0, 0, 0, 0};
  }
}

template <int DT>
__device__ __forceinline__ f32x4 mma(const uint4& a, const uint4& b, const f32x4& c) {
  if constexpr (DT == ARCHEAD_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ int rank_of(const AdaptArgs& p, int64_t id) {
  return p.ranks ? min(max(p.ranks[id], 0), p.R) : p.R;
}

// t[m, j] = sum_k x[m, k] a[j, k] over one part of K, fp32.  A wave takes a tile of
// up to 16 tokens of one adapter and RC x 16 ranks at a time; both operands come
// straight from memory (16 rows of 64 bytes a load), the ranks as the first, so a
// lane's results are four neighbouring ones of a token.
template <int DT, int RC, bool ODD>
__global__ __launch_bounds__(kABlock) void k_adapt_down(AdaptArgs p) {
  __shared__ Groups g;
  const int64_t m0 = int64_t(blockIdx.x) * kTok;
  group_tokens(g, p, m0, false);
  const int lane = threadIdx.x & 63, lr = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;
  const int64_t k0 = int64_t(blockIdx.y) * p.k_split, k1 = std::min(p.K, k0 + p.k_split);
  for (int ti = int(blockIdx.z) * kWaves + wave; ti < g.tiles; ti += p.spread * kWaves) {
    const int64_t id = g.adapter[ti];
    const bool there = lr < g.len[ti];
    const int64_t m = m0 + (there ? g.token[g.first[ti] + lr] : 0);
    const uint8_t* const x = p.x + m * p.x_row;
    const int rank = rank_of(p, id);
    for (int j0 = 0; j0 < rank; j0 += 16 * RC) {
      f32x4 acc[RC] = {};
#pragma unroll 4
      for (int64_t k = k0 + 8 * q; k - 8 * q < k1; k += 32) {
        const uint4 xv = load8<ODD>(x, k, there ? k1 : 0);
#pragma unroll
        for (int c = 0; c < RC; ++c) {
          const int j = j0 + 16 * c + lr;
          const uint4 av = load8<ODD>(p.a + id * p.a_ad + (j < rank ? j : 0) * p.a_row, k, j < rank ? k1 : 0);
          acc[c] = mma<DT>(av, xv, acc[c]);
        }
      }
      float* const t = p.t + (int64_t(blockIdx.y) * p.M + m) * p.rank16 + j0 + 4 * q;
#pragma unroll
      for (int c = 0; c < RC; ++c)
        if (there && j0 + 16 * c < rank) *reinterpret_cast<f32x4*>(t + 16 * c) = acc[c];
    }
  }
}

// out[m, n] = y[m, n] + sum_j t[m, j] b[n, j], t = scale times the sum of its parts.
// t goes through the matrix units in PARTS parts of the operands' type: two hold 17
// bits of it in bf16 and 22 in fp16 (there after a power of two that brings a
// token's largest to 2^14, so that no part is below the normal numbers), three 25.
// The workgroup holds the parts of its tokens in LDS; a wave takes 64 outputs of
// every tile, the rows of b as the first operand in an order that leaves a lane with
// eight neighbouring outputs of a token twice.  b's rows stay in registers over
// tiles of one adapter.  Bound by y and out.
template <int DT, int DY, int R32, int PARTS, bool ODD>
__global__ __launch_bounds__(kABlock) void k_adapt_up(AdaptArgs p) {
  constexpr int YB = Eight<DY>::kBytes, ROW = R32 * 32 + 8;   // elements of a token's row in LDS
  __shared__ Groups g;
  __shared__ float back[kTok];   // fp16: the power of two to take out again
  extern __shared__ __align__(16) uint16_t adapt_t[];          // [PARTS][kTok places][ROW]
  const int64_t m0 = int64_t(blockIdx.x) * kTok;
  group_tokens(g, p, m0, !p.in_place);
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, q = lane >> 4, wave = tid >> 6;
  // ---- t of this workgroup's tiles: four lanes a token
  for (int ti = blockIdx.z; ti < g.tiles; ti += p.spread) {
    const int64_t id = g.adapter[ti];
    if (id < 0) continue;
    const int rank = rank_of(p, id);
    const float scale = p.scales ? p.scales[id] : 1.f;
    const int i = tid >> 4;   // 16 lanes a token
    if (i < g.len[ti]) {
      const int place = g.first[ti] + i;
      const int64_t m = m0 + g.token[place];
      float v[R32 * 2];
      float top = 0;
#pragma unroll
      for (int c = 0; c < R32 * 2; ++c) {
        const int j = lr + 16 * c;
        float sum = 0;
        if (j < rank)
          for (int s = 0; s < p.splits; ++s) sum += p.t[(int64_t(s) * p.M + m) * p.rank16 + j];
        v[c] = sum * scale;
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
        if (lr == 0) back[place] = ldexpf(1.f, -e);
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
          adapt_t[(k * kTok + place) * ROW + lr + 16 * c] = bits;
          rest = fabsf(part) < INFINITY ? rest - part : 0.f;   // (an infinity or NaN has no rest)
        }
      }
    }
  }
  __syncthreads();
  const int64_t n_end = std::min(p.N, (int64_t(blockIdx.y) + 1) * p.n_wg);
  for (int64_t n0 = int64_t(blockIdx.y) * p.n_wg + 64 * wave; n0 < n_end; n0 += 64 * kWaves) {
    int64_t held = -1;
    uint4 bv[4][R32];
    for (int ti = blockIdx.z; ti < g.tiles; ti += p.spread) {
      const int64_t id = g.adapter[ti];
      const bool there = lr < g.len[ti];
      const int place = g.first[ti] + (there ? lr : 0);
      const int64_t m = m0 + g.token[place];
      Eight<DY> yv[2];
      const uint8_t* const y = p.y + m * p.y_row;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t at = n0 + 32 * h + 8 * q;
        if (there && at < p.N) yv[h].load(y, at, p.N, 0);
      }
      f32x4 acc[4] = {};
      if (id >= 0) {
        if (id != held) {
          const int rank = rank_of(p, id);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int64_t nr = n0 + 32 * (c >> 1) + 8 * (lr >> 2) + 4 * (c & 1) + (lr & 3);
            const bool in = nr < p.N;
            const uint8_t* const row = p.b + id * p.b_ad + (in ? nr : 0) * p.b_row;
#pragma unroll
            for (int kc = 0; kc < R32; ++kc) {
              const int j = 32 * kc + 8 * q;
              uint4 w = load8<ODD>(row, j, in ? (ODD ? rank : p.R) : 0);
              if constexpr (!ODD) {   // b past the adapter's rank is not looked at
                uint32_t d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  d[i] = j + 2 * i + 1 < rank ? d[i] : j + 2 * i < rank ? d[i] & 0xffffu : 0u;
                w = uint4{d[0], d[1], d[2], d[3]};
              }
              bv[c][kc] = w;
            }
          }
          held = id;
        }
#pragma unroll
        for (int kc = 0; kc < R32; ++kc)
#pragma unroll
          for (int k = 0; k < PARTS; ++k) {
            const uint4 tv = *reinterpret_cast<const uint4*>(&adapt_t[(k * kTok + place) * ROW + 32 * kc + 8 * q]);
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[c] = mma<DT>(bv[c][kc], tv, acc[c]);
          }
      }
      if (!there) continue;
      const float by = DT == ARCHEAD_F16 && id >= 0 ? back[place] : 1.f;
      uint8_t* const out = p.out + m * p.o_row;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t at = n0 + 32 * h + 8 * q;
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = yv[h].at(i) + (id >= 0 ? acc[2 * h + i / 4][i % 4] * by : 0.f);
        if (at + 8 <= p.N) {
          f32x8 v;
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = z[i];
          if constexpr (DY == ARCHEAD_F32) store_any(out + at * YB, v);
          else if constexpr (DY == ARCHEAD_BF16) store_any(out + at * YB, __builtin_convertvector(v, bf16x8));
          else store_any(out + at * YB, __builtin_convertvector(v, f16x8));
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (at + i >= p.N) continue;
            if constexpr (DY == ARCHEAD_F32) reinterpret_cast<float*>(out)[at + i] = z[i];
            else if constexpr (DY == ARCHEAD_BF16) reinterpret_cast<__bf16*>(out)[at + i] = __bf16(z[i]);
            else reinterpret_cast<_Float16*>(out)[at + i] = _Float16(z[i]);
          }
        }
      }
    }
  }
}

// Parts of K: by sizes alone, so that a call's sums have one order.
int k_splits(int64_t M, int64_t K, int64_t n) {
  const int64_t tiles = std::min(M, n + (M + 15) / 16);   // about
  const int64_t most = std::min<int64_t>(kMaxSplit, (K + 255) / 256);
  int64_t s = 1;
  while (s * 2 <= most && tiles * s < 1024) s *= 2;
  return int(s);
}

template <int DT, int RC, bool ODD>
hipError_t down(const AdaptArgs& p, dim3 grid, hipStream_t s) {
  return launch_kernel(k_adapt_down<DT, RC, ODD>, grid, dim3(kABlock), 0, s, p);
}
template <int DT, bool ODD>
hipError_t down_rank(const AdaptArgs& p, dim3 grid, hipStream_t s) {
  return p.R <= 16 ? down<DT, 1, ODD>(p, grid, s) : p.R <= 32 ? down<DT, 2, ODD>(p, grid, s) : down<DT, 4, ODD>(p, grid, s);
}

template <int DT, int DY, int R32, bool ODD>
hipError_t up(const AdaptArgs& p, dim3 grid, hipStream_t s) {
  constexpr int PARTS = DY == ARCHEAD_F32 && DT == ARCHEAD_BF16 ? 3 : 2;
  return launch_kernel_lds(k_adapt_up<DT, DY, R32, PARTS, ODD>, grid, dim3(kABlock), size_t(PARTS) * kTok * (R32 * 32 + 8) * 2,
                           s, p);
}
template <int DT, int DY, bool ODD>
hipError_t up_rank(const AdaptArgs& p, dim3 grid, hipStream_t s) {
  return p.R <= 32    ? up<DT, DY, 1, ODD>(p, grid, s)
         : p.R <= 64  ? up<DT, DY, 2, ODD>(p, grid, s)
         : p.R <= 128 ? up<DT, DY, 4, ODD>(p, grid, s)
                      : up<DT, DY, 8, ODD>(p, grid, s);
}
template <int DT, bool ODD>
hipError_t up_type(const AdaptArgs& p, archead_dtype y, dim3 grid, hipStream_t s) {
  return y == ARCHEAD_F32    ? up_rank<DT, ARCHEAD_F32, ODD>(p, grid, s)
         : y == ARCHEAD_BF16 ? up_rank<DT, ARCHEAD_BF16, ODD>(p, grid, s)
                             : up_rank<DT, ARCHEAD_F16, ODD>(p, grid, s);
}

template <int DT>
hipError_t launch(AdaptArgs p, archead_dtype y, hipStream_t s) {
  const int64_t blocks = (p.M + kTok - 1) / kTok;
  const int64_t in_block = std::min<int64_t>(std::min<int64_t>(kTok, p.M), p.n + 4);   // tiles of a block, at most about
  if (p.R > 0 && p.K > 0 && p.n > 0) {
    p.spread = int((in_block + kWaves - 1) / kWaves);
    const dim3 grid(static_cast<unsigned>(blocks), unsigned(p.splits), unsigned(p.spread));
    const hipError_t e = p.K % 8 ? down_rank<DT, true>(p, grid, s) : down_rank<DT, false>(p, grid, s);
    if (e != hipSuccess) return e;
  }
  // outputs of a workgroup: fewer, and then a block's tiles to several workgroups, where there are few blocks
  p.n_wg = 1024;
  const auto wgs = [&] { return blocks * ((p.N + p.n_wg - 1) / p.n_wg); };
  while (p.n_wg > 256 && wgs() < 1024) p.n_wg /= 2;
  p.spread = int(std::min<int64_t>(in_block, std::max<int64_t>(1, 512 / wgs())));
  const dim3 grid(static_cast<unsigned>(blocks), unsigned((p.N + p.n_wg - 1) / p.n_wg), unsigned(p.spread));
  return p.R % 8 ? up_type<DT, true>(p, y, grid, s) : up_type<DT, false>(p, y, grid, s);
}

}  // namespace

extern "C" size_t archead_adapters_workspace_bytes(int64_t M, int64_t K, int64_t R, int64_t n) {
  if (M < 1 || K < 1 || R < 1 || n < 1 || M > INT32_MAX || K > INT32_MAX || R > kMaxRank) return 0;
  return (size_t(k_splits(M, K, n)) * M * ((R + 15) / 16 * 16) * 4 + 255) / 256 * 256;
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
  if (M < 0 || M > INT32_MAX || N < 0 || N > (1 << 23) || K < 0 || K > INT32_MAX)
    return fail(ARCHEAD_E_INVALID_ARG, "M = %lld, N = %lld, K = %lld out of range", (long long)M, (long long)N, (long long)K);
  if (!ad) return fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if (ad->n < 0 || ad->n >= (1 << 30) || ad->R < 0) return fail(ARCHEAD_E_INVALID_ARG, "n or R out of range");
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
  p.t = static_cast<float*>(ws);
  p.M = M, p.N = N, p.K = K, p.n = any ? ad->n : 0;
  p.y_row = ldy * yb, p.x_row = ldx * 2, p.o_row = ldo * yb;
  p.a_ad = ad->a_adapter * 2, p.a_row = ad->a_row * 2, p.b_ad = ad->b_adapter * 2, p.b_row = ad->b_row * 2;
  p.R = int(ad->R), p.rank16 = int((ad->R + 15) / 16 * 16);
  if (any) {
    const int s = k_splits(M, K, ad->n);
    p.k_split = int(((K + s - 1) / s + 31) / 32 * 32);
    p.splits = int((K + p.k_split - 1) / p.k_split);
  }
  p.ids64 = ids_dtype == ARCHEAD_I64, p.in_place = out == y;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return launch_status(x_dtype == ARCHEAD_BF16 ? launch<ARCHEAD_BF16>(p, y_dtype, s) : launch<ARCHEAD_F16>(p, y_dtype, s),
                       "adapters launch");
}
