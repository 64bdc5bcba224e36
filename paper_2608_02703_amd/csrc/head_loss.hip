// archead_head_loss, archead_head_loss_grad: softmax cross entropy of a dense
// bf16 head, and its gradients, a piece of the vocabulary at a time.
#include "head_loss.h"

#include <algorithm>

#include "dev_rows.cuh"

namespace {

using namespace archead::rows;
using namespace archead::loss;

constexpr int64_t kMaxM = int64_t(1) << 20, kMaxV = int64_t(1) << 22, kMaxD = 16384;
constexpr int64_t kMaxLdw = int64_t(1) << 20;           // a tile's rows stay within 31-bit offsets
// Of G, and of a copy of the head's rows: some thousand tiles, so that a last round of 256 that
// is not full costs little, and few additions to the hidden states' sums (64 / 128 / 256 MiB: G and the
// gradients of 4096 tokens, 151936 x 4096 13.1 / 12.7 / 12.6 ms, of 614, 262144 x 2560 3.21 / 2.99 / 2.89).
constexpr int64_t kPieceBytes = int64_t(256) << 20;
constexpr int kRBlock = 256;

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

struct RowArgs {
  const uint8_t* x;
  const void* target;
  const float* lse;        // by token, may be null
  const float* g;
  int64_t M, V, d, dp, x_row, x_ld;   // dp: d padded to whole stages; bytes between rows of x, elements between those of `rows`
  int per_block;
  bool t64;
  int32_t* count;
  int32_t* pos;            // [M] place among the live tokens, or -1
  int32_t* y;              // [Mp] by place
  float* lse_out;
  float* g_out;            // in units of *unit
  float* unit;             // the largest finite |g| of a live token
  uint16_t* rows;          // [Mp][x_ld]
};

__device__ __forceinline__ int64_t target_of(const RowArgs& a, int64_t m) {
  const int64_t y = a.t64 ? static_cast<const int64_t*>(a.target)[m] : static_cast<const int32_t*>(a.target)[m];
  return y >= 0 && y < a.V ? y : -1;
}

// The live tokens (those with a target in the vocabulary) back to back, in their
// order, with zeros behind each row up to whole stages and behind the last token's
// for sums over tokens: tokens without a target cost no products, and nothing that
// their rows hold can reach a sum.  Each workgroup counts the live tokens before its own, in all
// the targets (and g): one launch, the least for some thousand tokens (4096 x 64: 8 us in the loss, 11 in the
// gradients), but the targets are read up to 1024 times (2^16 x 64: 95 and 160 us, 2^20 x 64: 2.1 and 3.2 ms).
// g goes on in units of the largest, which the gradients get back in fp32: the entries of G
// that weigh most, g (p - 1) at the targets, are then -1 + p for tokens that count alike, and
// lose next to nothing in bf16 (g itself, say 1 / 87, would lose up to 2^-8 in each of them).
__global__ __launch_bounds__(kRBlock) void k_ce_rows(RowArgs a) {
  __shared__ int32_t sums[2][kRBlock / 64], place[kRBlock];
  __shared__ float tops[kRBlock / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t first = int64_t(blockIdx.x) * a.per_block, end = std::min(a.M, first + a.per_block);
  int before = 0, all = 0;
  float unit = 0;
  for (int64_t m = tid; m < a.M; m += kRBlock) {
    const bool live = target_of(a, m) >= 0;
    all += live;
    before += live && m < first;
    if (live && a.lse) {
      const float g = fabsf(a.g[m]);
      if (g < INFINITY) unit = fmaxf(unit, g);
    }
  }
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    before += __shfl_xor(before, s);
    all += __shfl_xor(all, s);
    unit = fmaxf(unit, __shfl_xor(unit, s));
  }
  if (lane == 0) {
    sums[0][wave] = before;
    sums[1][wave] = all;
    tops[wave] = unit;
  }
  __syncthreads();
  before = all = 0;
  for (int w = 0; w < kRBlock / 64; ++w) {
    before += sums[0][w];
    all += sums[1][w];
    unit = fmaxf(unit, tops[w]);
  }
  if (unit == 0) unit = 1;
  if (blockIdx.x == 0 && tid == 0) {
    *a.count = all;
    *a.unit = unit;
  }
  const int groups = int(a.dp / 8);
  for (int64_t m0 = first; m0 < end; m0 += kRBlock) {
    const int64_t m = m0 + tid;
    const int64_t y = m < end ? target_of(a, m) : -1;
    const uint64_t mask = __ballot(y >= 0);
    __syncthreads();   // (sums and place have been read)
    if (lane == 0) sums[0][wave] = __popcll(mask);
    __syncthreads();
    int at = before + __popcll(mask & ((uint64_t(1) << lane) - 1));
    for (int w = 0; w < kRBlock / 64; ++w) {
      if (w < wave) at += sums[0][w];
      before += sums[0][w];
    }
    place[tid] = y >= 0 ? at : -1;
    if (m < end) a.pos[m] = y >= 0 ? at : -1;
    if (y >= 0) {
      a.y[at] = int32_t(y);
      if (a.lse) {
        a.lse_out[at] = a.lse[m];
        a.g_out[at] = a.g[m] / unit;
      }
    }
    __syncthreads();
    const int here = int(std::min<int64_t>(kRBlock, end - m0));
    for (int i = wave; i < here; i += kRBlock / 64) {
      const int to = place[i];
      if (to < 0) continue;
      const uint8_t* const row = a.x + (m0 + i) * a.x_row;
      uint16_t* const out = a.rows + int64_t(to) * a.x_ld;
      int j = lane;
      for (; (j - lane + 256) * 8 <= a.d; j += 256) {
        uint4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = load_any<uint4>(row + (j + 64 * k) * 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(out + (j + 64 * k) * 8) = v[k];
      }
      for (; j < groups; j += 64) {
        Eight<ARCHEAD_BF16> e;
        e.load(row, int64_t(j) * 8, a.d, 0);
        *reinterpret_cast<uint4*>(out + j * 8) = e.w[0];
      }
    }
  }
  if (!a.lse) return;   // (sums over tokens are the gradient's)
  for (int64_t r = all + blockIdx.x; r < (int64_t(all) + kStageK - 1) / kStageK * kStageK; r += gridDim.x)
    for (int j = tid; j < groups; j += kRBlock)
      *reinterpret_cast<uint4*>(a.rows + r * a.x_ld + j * 8) = uint4{0, 0, 0, 0};
}

// rows of the head padded with zeros to whole stages
__global__ __launch_bounds__(kRBlock) void k_ce_pad(const uint8_t* w, int64_t w_row, int64_t d, int64_t dp, uint16_t* to) {
  const uint8_t* const row = w + int64_t(blockIdx.x) * w_row;
  for (int64_t j = threadIdx.x * 8; j < dp; j += kRBlock * 8) {
    Eight<ARCHEAD_BF16> e;
    e.load(row, j, d, 0);
    *reinterpret_cast<uint4*>(to + int64_t(blockIdx.x) * dp + j) = e.w[0];
  }
}

// A token's loss from its tiles' statistics, a wave to a token.
__global__ __launch_bounds__(kRBlock) void k_ce_merge(const float2* part, int64_t n_part, const float* at_target,
                                                      const int32_t* pos, int64_t M, float* loss, float* lse) {
  const int lane = threadIdx.x & 63;
  const int64_t m = int64_t(blockIdx.x) * (kRBlock / 64) + (threadIdx.x >> 6);
  if (m >= M) return;
  const int p = pos[m];
  float top = -INFINITY, sum = 0;
  if (p >= 0) {
    const float2* const mine = part + p * n_part;
    for (int64_t i = lane; i < n_part; i += 64) {   // (a NaN is in a tile's sum, never in its largest)
      const float2 v = mine[i];
      const float both = fmaxf(top, v.x);
      if (both > -INFINITY) sum = sum * expf(top - both) + v.y * expf(v.x - both);
      else sum += v.y;
      top = both;
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const float ot = __shfl_xor(top, s), os = __shfl_xor(sum, s), both = fmaxf(top, ot);
      if (both > -INFINITY) sum = sum * expf(top - both) + os * expf(ot - both);
      else sum += os;
      top = both;
    }
  }
  if (lane == 0) {
    const float log_sum = logf(sum);
    lse[m] = p >= 0 ? top + log_sum : 0.f;
    loss[m] = p >= 0 ? top - at_target[p] + log_sum : 0.f;   // (lse's rounding would be most of a small loss's error)
  }
}

// The gradient of a token's hidden state from the parts of its sums, zeros for a
// token without a target.
__global__ __launch_bounds__(kRBlock) void k_ce_hidden(const float* sums, int64_t sum_rows, int64_t first_stages, int ti, int64_t dp,
                                                       const int32_t* count, const float* unit, const int32_t* pos, int64_t d, uint16_t* dx, int64_t ld) {
  const int64_t m = blockIdx.x;
  const int p = pos[m], live = *count;
  const int splits = splits_for((live + ti - 1) / ti * ((d + kTileJ - 1) / kTileJ), live, sum_rows, first_stages);
  const int64_t split_step = padded_rows(live) * dp;
  typedef float f32x8 __attribute__((ext_vector_type(8)));
  typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
  const float c = *unit;
  for (int64_t j = 8 * threadIdx.x; j < d; j += 8 * kRBlock) {
    f32x8 v = {};
    if (p >= 0) {
      const float* const from = sums + p * dp + j;
#pragma unroll 4
      for (int s = 0; s < splits; ++s) v += *reinterpret_cast<const f32x8*>(from + s * split_step);
    }
    const bf16x8 o = __builtin_convertvector(v * c, bf16x8);
    uint16_t* const to = dx + m * ld + j;
    if (j + 8 <= d) {
      store_any(to, o);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (j + i < d) reinterpret_cast<__bf16*>(to)[i] = o[i];
    }
  }
}

__global__ __launch_bounds__(kRBlock) void k_ce_zero(uint16_t* w, int64_t d, int64_t ld) {
  for (int64_t j = threadIdx.x; j < d; j += kRBlock) w[int64_t(blockIdx.x) * ld + j] = 0;
}

// What a call keeps in its workspace (offsets in bytes, multiples of 256).
struct Plan {
  int64_t M, V, d, dp, Mp;
  int ti, ti_x, ti_w;      // rows of the tiles of logits, of the hidden states' and of the head's gradient
  bool direct;             // the head's rows are read where they are
  int64_t piece;           // vocabulary rows at a time
  int64_t n_part;
  int64_t sum_rows;        // of the hidden states' gradient, in its parts
  int64_t first_stages;    // of k in the first piece, the longest
  int64_t x_ld, g_ld;      // elements between rows of the tokens and of G
  size_t count, pos, y, tgt, part, lse, g, rows, copy, G, sums, total;
};

bool is_direct(const void* w, int64_t d, int64_t ldw) {
  return d % kStageK == 0 && ldw % 8 == 0 && ldw <= kMaxLdw && aligned(w, 16);
}

// Rows of the tiles of `rows` x `cols` tiles of columns: those of the least time, in rounds of
// 256 tiles of which one of 128 (64) rows takes 0.62 (0.49) of one of 256's (256 x 65536 x 4096: one,
// two and four rounds 156, 194 and 306 us).
int rows_of_tiles(int64_t rows, int64_t cols, int least) {
  int best = 256;
  double time = 0;
  for (const int t : {256, 128, 64}) {
    if (t < least) continue;
    const int64_t tiles = (rows + t - 1) / t * cols;
    const double now = double((tiles + 255) / 256) * (t == 256 ? 1.0 : t == 128 ? 0.62 : 0.49);
    if (t == 256 || now < 0.9 * time) {   // (near ties: the taller, whose last tile may be half empty)
      best = t;
      time = now;
    }
  }
  return best;
}

Plan plan(int64_t M, int64_t V, int64_t d, bool direct, bool grad) {
  Plan p{};
  p.M = M, p.V = V, p.d = d, p.dp = up(d, kStageK), p.Mp = up(M, kRowPad);
  p.direct = direct;
  p.piece = up(V, kTileJ);
  if (!direct) p.piece = std::min(p.piece, std::max<int64_t>(kTileJ, kPieceBytes / (p.dp * 2) / kTileJ * kTileJ));
  if (grad) p.piece = std::min(p.piece, std::max<int64_t>(16 * kTileJ, kPieceBytes / (p.Mp * 2) / kTileJ * kTileJ));
  p.ti = rows_of_tiles(M, up(p.piece, kTileJ) / kTileJ, 64);
  p.ti_x = rows_of_tiles(M, 1 << 20, 64);   // (its parts of k fill the CUs)
  p.ti_w = rows_of_tiles(std::min(V, p.piece), up(d, kTileJ) / kTileJ, 128);
  p.n_part = up(V, kTileJ) / kTileJ;
  const int64_t tiles = (M + p.ti_x - 1) / p.ti_x * (up(d, kTileJ) / kTileJ);
  p.first_stages = (std::min(V, p.piece) + kStageK - 1) / kStageK;
  p.sum_rows = p.Mp * std::max<int64_t>(1, std::min<int64_t>(p.first_stages / kPartStages, kTargetTiles / tiles));
  // rows of a power of two would all ask for the same memory channels at once
  p.x_ld = p.dp + kStageK, p.g_ld = p.piece + kStageK;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) / 256 * 256;
    return o;
  };
  p.count = take(8);   // and the unit of g
  p.pos = take(M * 4);
  p.y = take(p.Mp * 4);
  p.rows = take(p.Mp * p.x_ld * 2);
  if (!direct) p.copy = take(p.piece * p.dp * 2);
  if (grad) {
    p.lse = take(p.Mp * 4);
    p.g = take(p.Mp * 4);
    p.G = take(p.Mp * p.g_ld * 2);
    p.sums = take(p.sum_rows * p.dp * 4);
  } else {
    p.tgt = take(p.Mp * 4);
    p.part = take(p.Mp * p.n_part * 8);
  }
  p.total = at;
  return p;
}

bool in_range(int64_t M, int64_t V, int64_t d) { return M >= 0 && M <= kMaxM && V >= 1 && V <= kMaxV && d >= 1 && d <= kMaxD; }

archead_status check(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* targets, archead_dtype tdt, int64_t M,
                     int64_t V, int64_t d) {
  using archead::fail;
  if (tdt != ARCHEAD_I32 && tdt != ARCHEAD_I64) return fail(ARCHEAD_E_INVALID_ARG, "tgt_dtype must be I32 or I64");
  if (M < 0 || V < 1 || d < 1)
    return fail(ARCHEAD_E_INVALID_ARG, "M = %lld, V = %lld, d = %lld out of range", (long long)M, (long long)V, (long long)d);
  if (!in_range(M, V, d))
    return fail(ARCHEAD_E_UNSUPPORTED, "M = %lld, V = %lld, d = %lld beyond 2^20, 2^22, 16384", (long long)M, (long long)V,
                (long long)d);
  if (M == 0) return ARCHEAD_OK;
  if (ldx < d || ldw < d) return fail(ARCHEAD_E_INVALID_ARG, "leading dimensions must be >= d");
  if (!x || !w || !targets) return fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if (!aligned(x, 2) || !aligned(w, 2) || !aligned(targets, tdt == ARCHEAD_I64 ? 8 : 4))
    return fail(ARCHEAD_E_MISALIGNED, "x / w / targets misaligned");
  return ARCHEAD_OK;
}
archead_status check_ws(const void* ws, size_t bytes, size_t need) {
  using archead::fail;
  if (!ws) return fail(ARCHEAD_E_INVALID_ARG, "null workspace");
  if (!aligned(ws, 256)) return fail(ARCHEAD_E_MISALIGNED, "workspace must be 256-byte aligned");
  if (bytes < need) return fail(ARCHEAD_E_WORKSPACE, "workspace of %zu bytes, %zu needed", bytes, need);
  return ARCHEAD_OK;
}

hipError_t gather(const Plan& p, char* ws, const void* x, int64_t ldx, const void* targets, archead_dtype tdt,
                  const float* lse, const float* g, hipStream_t s) {
  RowArgs a{};
  a.x = static_cast<const uint8_t*>(x), a.target = targets, a.lse = lse, a.g = g;
  a.M = p.M, a.V = p.V, a.d = p.d, a.dp = p.dp, a.x_row = ldx * 2, a.x_ld = p.x_ld;
  a.per_block = int(std::max<int64_t>(4, (p.M + 1023) / 1024));
  a.t64 = tdt == ARCHEAD_I64;
  a.count = reinterpret_cast<int32_t*>(ws + p.count);
  a.unit = reinterpret_cast<float*>(a.count + 1);
  a.pos = reinterpret_cast<int32_t*>(ws + p.pos);
  a.y = reinterpret_cast<int32_t*>(ws + p.y);
  a.lse_out = reinterpret_cast<float*>(ws + p.lse);
  a.g_out = reinterpret_cast<float*>(ws + p.g);
  a.rows = reinterpret_cast<uint16_t*>(ws + p.rows);
  return launch_kernel(k_ce_rows, dim3(unsigned((p.M + a.per_block - 1) / a.per_block)), dim3(kRBlock), 0, s, a);
}

// the arguments that the pieces' products share, and the piece's rows of the head
// (copied where they cannot be read in place)
hipError_t piece_of(const Plan& p, char* ws, const void* w, int64_t ldw, int64_t v0, TileArgs& t, hipStream_t s) {
  t = TileArgs{};
  t.a = reinterpret_cast<const uint16_t*>(ws + p.rows);
  t.a_ld = p.x_ld;
  t.rows = p.M;
  t.cols = std::min(p.piece, p.V - v0);
  t.depth = p.dp;
  t.count = reinterpret_cast<const int32_t*>(ws + p.count);
  t.target = reinterpret_cast<const int32_t*>(ws + p.y);
  t.v0 = v0;
  t.b = static_cast<const uint16_t*>(w) + v0 * ldw;
  t.b_ld = ldw;
  if (p.direct) return hipSuccess;
  uint16_t* const copy = reinterpret_cast<uint16_t*>(ws + p.copy);
  const uint8_t* const from = reinterpret_cast<const uint8_t*>(t.b);
  t.b = copy;
  t.b_ld = p.dp;
  return launch_kernel(k_ce_pad, dim3(unsigned(t.cols)), dim3(kRBlock), 0, s, from, ldw * 2, p.d, p.dp, copy);
}

}  // namespace

extern "C" size_t archead_head_loss_workspace_bytes(int64_t M, int64_t V, int64_t d, const void* w, int64_t ldw, int grad) {
  return in_range(M, V, d) && M > 0 ? plan(M, V, d, is_direct(w, d, ldw), grad != 0).total : 0;
}

extern "C" archead_status archead_head_loss(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* targets,
                                            archead_dtype tgt_dtype, int64_t M, int64_t V, int64_t d, float* loss,
                                            float* lse, void* ws, size_t ws_bytes, void* stream) {
  using archead::fail;
  archead::clear_error();
  if (const archead_status st = check(x, ldx, w, ldw, targets, tgt_dtype, M, V, d)) return st;
  if (M == 0) return ARCHEAD_OK;
  if (!loss || !lse) return fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if (!aligned(loss, 4) || !aligned(lse, 4)) return fail(ARCHEAD_E_MISALIGNED, "loss / lse misaligned");
  const Plan p = plan(M, V, d, is_direct(w, d, ldw), false);
  if (const archead_status st = check_ws(ws, ws_bytes, p.total)) return st;
  char* const base = static_cast<char*>(ws);
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = gather(p, base, x, ldx, targets, tgt_dtype, nullptr, nullptr, s);
  float2* const part = reinterpret_cast<float2*>(base + p.part);
  float* const tgt = reinterpret_cast<float*>(base + p.tgt);
  for (int64_t v0 = 0; v0 < V && e == hipSuccess; v0 += p.piece) {
    TileArgs t;
    e = piece_of(p, base, w, ldw, v0, t, s);
    if (e != hipSuccess) break;
    t.part = part, t.n_part = p.n_part, t.part0 = v0 / kTileJ, t.at_target = tgt;
    e = launch_tiles(kStats, p.ti, t, s);
  }
  if (e == hipSuccess)
    e = launch_kernel(k_ce_merge, dim3(unsigned((M + kRBlock / 64 - 1) / (kRBlock / 64))), dim3(kRBlock), 0, s, part, p.n_part, tgt,
                      reinterpret_cast<const int32_t*>(base + p.pos), M, loss, lse);
  return launch_status(e, "head loss launch");
}

extern "C" archead_status archead_head_loss_grad(const void* x, int64_t ldx, const void* w, int64_t ldw,
                                                 const void* targets, archead_dtype tgt_dtype, const float* lse,
                                                 const float* grad, int64_t M, int64_t V, int64_t d, void* dx,
                                                 int64_t lddx, void* dw, int64_t lddw, void* ws, size_t ws_bytes,
                                                 void* stream) {
  using archead::fail;
  archead::clear_error();
  if (const archead_status st = check(x, ldx, w, ldw, targets, tgt_dtype, M, V, d)) return st;
  if (!dx && !dw) return M == 0 ? ARCHEAD_OK : fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if ((dx && lddx < d) || (dw && lddw < d)) return fail(ARCHEAD_E_INVALID_ARG, "leading dimensions must be >= d");
  if (!aligned(dx, 2) || !aligned(dw, 2)) return fail(ARCHEAD_E_MISALIGNED, "dx / dw misaligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (M == 0) {
    if (!dw) return ARCHEAD_OK;
    return launch_status(launch_kernel(k_ce_zero, dim3(unsigned(V)), dim3(kRBlock), 0, s, static_cast<uint16_t*>(dw), d, lddw),
                         "head gradient launch");
  }
  if (!lse || !grad) return fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if (!aligned(lse, 4) || !aligned(grad, 4)) return fail(ARCHEAD_E_MISALIGNED, "lse / grad misaligned");
  const Plan p = plan(M, V, d, is_direct(w, d, ldw), true);
  if (const archead_status st = check_ws(ws, ws_bytes, p.total)) return st;
  char* const base = static_cast<char*>(ws);
  hipError_t e = gather(p, base, x, ldx, targets, tgt_dtype, lse, grad, s);
  uint16_t* const G = reinterpret_cast<uint16_t*>(base + p.G);
  float* const sums = reinterpret_cast<float*>(base + p.sums);
  for (int64_t v0 = 0; v0 < V && e == hipSuccess; v0 += p.piece) {
    TileArgs t;
    e = piece_of(p, base, w, ldw, v0, t, s);
    if (e != hipSuccess) break;
    TileArgs q = t;
    q.lse = reinterpret_cast<const float*>(base + p.lse), q.g = reinterpret_cast<const float*>(base + p.g);
    q.out = G, q.out_ld = p.g_ld;
    e = launch_tiles(kGrad, p.ti, q, s);
    if (dx && e == hipSuccess) {
      q = t;
      q.a = G, q.a_ld = p.g_ld, q.cols = d, q.depth = t.cols;
      q.sums = sums, q.sum_ld = p.dp, q.sum_rows = p.sum_rows, q.first_stages = p.first_stages, q.add = v0 > 0;
      e = launch_tiles(kHidden, p.ti_x, q, s);
    }
    if (dw && e == hipSuccess) {
      q = t;
      q.unit = reinterpret_cast<const float*>(t.count + 1);
      q.a = G, q.a_ld = p.g_ld, q.b = t.a, q.b_ld = t.a_ld, q.rows = t.cols, q.cols = d;
      q.out = static_cast<uint16_t*>(dw) + v0 * lddw, q.out_ld = lddw;
      e = launch_tiles(kHead, p.ti_w, q, s);
    }
  }
  if (dx && e == hipSuccess)
    e = launch_kernel(k_ce_hidden, dim3(unsigned(M)), dim3(kRBlock), 0, s, sums, p.sum_rows, p.first_stages, p.ti_x, p.dp,
                      reinterpret_cast<const int32_t*>(base + p.count), reinterpret_cast<const float*>(base + p.count + 4),
                      reinterpret_cast<const int32_t*>(base + p.pos), d, static_cast<uint16_t*>(dx), lddx);
  return launch_status(e, "head gradient launch");
}
