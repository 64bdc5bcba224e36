// Beam search: the n best (beam, token) pairs of each sequence from rows of
// logits, and the reordering of the states they continue.
#include "beam.h"
#include "dev_rows.cuh"

namespace {

using namespace archead::rows;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------- selection
// Two launches.  k_beam_scan reads the logits once: of every chunk of a row
// its largest logit, and of every span of chunks (a wave's) the pair (maximum,
// sum of exponentials).  k_beam_pick, a workgroup per sequence, makes the rows'
// logsumexp of them and with it the chunks' largest scores.  If n chunks are
// ranked by (largest score, then position), every pair among the n best lies in
// one of the first n, so the logits of no more than those are read again.
constexpr int kScanBlock = 256;
constexpr int kSpanChunks = archead::kBeamSpan / archead::kBeamChunk;
static_assert(archead::kBeamChunk == 64 * 8, "a wave takes a chunk per step");

// fp64 values as integers of the same order; 0 for -inf and NaN
__device__ __forceinline__ uint64_t order_key(double v) {
  const uint64_t u = uint64_t(__double_as_longlong(v + 0.0));   // -0 becomes 0
  return v > -INFINITY ? (u >> 63 ? ~u : u | (uint64_t(1) << 63)) : 0;
}

template <int DT>
constexpr uint32_t neg_inf() {
  return DT == ARCHEAD_F32 ? 0xff800000u : DT == ARCHEAD_BF16 ? 0xff80u : 0xfc00u;
}

struct ScanArgs {
  const uint8_t* logits;
  int64_t V, row_bytes;
  int64_t n_span;          // spans of a row; kSpanChunks times as many chunks
  const float* scores;
  const uint8_t* finished;   // may be null
  float* cmax;               // [rows][n_span * kSpanChunks]
  archead::BeamSpanSum* span;   // [rows][n_span]
};

template <int DT>
__global__ __launch_bounds__(kScanBlock) void k_beam_scan(ScanArgs a) {
  const int lane = threadIdx.x & 63;
  const int wid = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int64_t r = blockIdx.y, sp = int64_t(blockIdx.x) * (kScanBlock / 64) + wid;
  if (sp >= a.n_span) return;
  if (!(fabsf(a.scores[r]) < INFINITY) || (a.finished && a.finished[r])) return;   // offers nothing by its logits
  const uint8_t* row = a.logits + r * a.row_bytes;
  Eight<DT> e[kSpanChunks];
#pragma unroll
  for (int c = 0; c < kSpanChunks; ++c)
    e[c].load(row, sp * archead::kBeamSpan + c * archead::kBeamChunk + lane * 8, a.V, neg_inf<DT>());
  float cm[kSpanChunks], top = -INFINITY;
#pragma unroll
  for (int c = 0; c < kSpanChunks; ++c) {
    float m = e[c].at(0);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = fmaxf(m, e[c].at(i));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    cm[c] = m;
    top = fmaxf(top, m);
  }
  // relative to 0 where nothing is above -inf: every term is then 0, or NaN
  const float ref = top > -INFINITY ? top : 0.f;
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < kSpanChunks; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) s += __builtin_amdgcn_exp2f((e[c].at(i) - ref) * 1.4426950408889634f);
  double sd = s;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sd += __shfl_xor(sd, o, 64);
  if (lane == 0) {
    a.span[r * a.n_span + sp] = archead::BeamSpanSum{sd, ref};
#pragma unroll
    for (int c = 0; c < kSpanChunks; ++c) a.cmax[(r * a.n_span + sp) * kSpanChunks + c] = cm[c];
  }
}

constexpr int kPickBlock = 1024, kPickWaves = kPickBlock / 64;
constexpr int kPickList = 512;   // chunks, and pairs, that are ranked one against all
static_assert(kPickList >= archead::kTopKMaxK + ARCHEAD_BEAM_MAX, "room for the n best and the ended beams");

struct PickArgs {
  ScanArgs in;
  int K, n;
  int64_t end_token;
  float* out_scores;
  int64_t *parents, *tokens;
  uint8_t* out_finished;   // may be null
};

// the order of pairs (position k * V + v) and of chunks (their number)
__device__ __forceinline__ bool before(double sa, int64_t ia, double sb, int64_t ib) {
  return sa > sb || (sa == sb && ia < ib);
}

template <int DT>
__global__ __launch_bounds__(kPickBlock) void k_beam_pick(PickArgs p) {
  __shared__ double lse[ARCHEAD_BEAM_MAX], cum[ARCHEAD_BEAM_MAX];   // lse: NaN where a row offers nothing by its logits
  __shared__ bool ended[ARCHEAD_BEAM_MAX];
  __shared__ uint32_t skey[kPickBlock];
  __shared__ double lscore[kPickList];
  __shared__ int64_t lat[kPickList];
  __shared__ int chunks[kPickList];
  __shared__ double wscore[kPickWaves];
  __shared__ int64_t wat[kPickWaves];
  __shared__ int n_list, n_pair;
  __shared__ uint32_t sfloor;
  const ScanArgs& a = p.in;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t b = blockIdx.x, r0 = b * p.K;
  const int n_chunk = int(a.n_span) * kSpanChunks, n_items = n_chunk * p.K;   // (K V / 512 < 2^27)
  if (tid == 0) n_list = n_pair = 0;
  for (int k = wid; k < p.K; k += kPickWaves) {
    const double c = a.scores[r0 + k];
    const bool f = a.finished && a.finished[r0 + k], alive = fabs(c) < INFINITY && !f;
    double m = -INFINITY, s = 0.0;
    if (alive) {
      const archead::BeamSpanSum* sp = a.span + (r0 + k) * a.n_span;
      // (a span with nothing above -inf has the sum 0, whatever its maximum)
      for (int64_t i = lane; i < a.n_span; i += 64)
        if (sp[i].sum != 0.0) m = fmax(m, double(sp[i].top));
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) m = fmax(m, __shfl_xor(m, o, 64));
      for (int64_t i = lane; i < a.n_span; i += 64)
        if (sp[i].sum != 0.0) s += sp[i].sum * exp(double(sp[i].top) - m);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    }
    if (lane == 0) {
      // +inf among the logits: a term inf - inf, so the sum is NaN
      lse[k] = alive && s > 0.0 ? m + log(s) : double(NAN);
      cum[k] = c;
      ended[k] = f;
    }
  }
  __syncthreads();
  auto score_of = [&](int k, float logit) { return cum[k] + (double(logit) - lse[k]); };
  auto chunk_score = [&](int item) {
    const int k = item / n_chunk;
    return lse[k] == lse[k] ? score_of(k, a.cmax[r0 * n_chunk + item]) : double(-INFINITY);
  };
  // ---- a floor: the n-th largest of the threads' best chunks (the order's
  // first 32 bits)
  uint32_t best = 0;
  for (int i = tid; i < n_items; i += kPickBlock) best = max(best, uint32_t(order_key(chunk_score(i)) >> 32));
  skey[tid] = best;
  __syncthreads();
  if (wid == 0) {
    uint32_t kk[kPickWaves];
#pragma unroll
    for (int i = 0; i < kPickWaves; ++i) kk[i] = skey[64 * i + lane];
    uint32_t f = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t t = f | (1u << bit);
      int c = 0;
#pragma unroll
      for (int i = 0; i < kPickWaves; ++i) c += __popcll(__ballot(kk[i] >= t));
      f = c >= p.n ? t : f;
    }
    if (lane == 0) sfloor = max(f, 1u);   // 1: every candidate
  }
  __syncthreads();
  const uint32_t floor = sfloor;
  // ---- the chunks that reach it
  for (int i = tid; i < n_items; i += kPickBlock) {
    const double s = chunk_score(i);
    if (uint32_t(order_key(s) >> 32) >= floor) {
      const int at = atomicAdd(&n_list, 1);
      if (at < kPickList) chunks[at] = i;
    }
  }
  __syncthreads();
  // The best of the threads' (s, i), in every thread.
  auto workgroup_best = [&](double& s, int64_t& i) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const double os = __shfl_xor(s, o, 64);
      const int64_t oi = __shfl_xor((long long)i, o, 64);
      if (before(os, oi, s, i)) {
        s = os;
        i = oi;
      }
    }
    if (lane == 0) {
      wscore[wid] = s;
      wat[wid] = i;
    }
    __syncthreads();
    s = wscore[0];
    i = wat[0];
#pragma unroll
    for (int w = 1; w < kPickWaves; ++w)
      if (before(wscore[w], wat[w], s, i)) {
        s = wscore[w];
        i = wat[w];
      }
    __syncthreads();
  };
  int n_ch = n_list;
  if (__builtin_expect(n_ch > kPickList, 0)) {
    // many that are equal or nearly so: the first n of the ranking, one a round
    double as = INFINITY;
    int64_t ai = -1;
    n_ch = 0;
    for (int j = 0; j < p.n; ++j) {
      double s = -INFINITY;
      int64_t at = INT64_MAX;
      for (int i = tid; i < n_items; i += kPickBlock) {
        const double si = chunk_score(i);
        if (si > -INFINITY && before(as, ai, si, i) && before(si, i, s, at)) {
          s = si;
          at = i;
        }
      }
      workgroup_best(s, at);
      if (!(s > -INFINITY)) break;
      if (tid == 0) chunks[j] = int(at);
      as = s;
      ai = at;
      n_ch = j + 1;
    }
    __syncthreads();
  }
  // ---- the pairs at or above the floor, and the ended beams'
  auto token_at = [&](int item, int i) {   // of element i of this lane in a chunk
    return int64_t(item % n_chunk) * archead::kBeamChunk + lane * 8 + i;
  };
  if (tid < p.K && ended[tid] && fabs(cum[tid]) < INFINITY) {
    const int at = atomicAdd(&n_pair, 1);
    if (at < kPickList) {
      lscore[at] = cum[tid];
      lat[at] = tid * a.V + p.end_token;
    }
  }
  for (int c = wid; c < n_ch; c += kPickWaves) {
    const int item = chunks[c], k = item / n_chunk;
    Eight<DT> e;
    e.load(a.logits + (r0 + k) * a.row_bytes, token_at(item, 0), a.V, neg_inf<DT>());
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double s = score_of(k, e.at(i));
      if (uint32_t(order_key(s) >> 32) >= floor) {
        const int at = atomicAdd(&n_pair, 1);
        if (at < kPickList) {
          lscore[at] = s;
          lat[at] = k * a.V + token_at(item, i);
        }
      }
    }
  }
  __syncthreads();
  const int np = n_pair;
  auto write = [&](int j, double s, int64_t at) {
    const int k = int(at / a.V);
    const int64_t v = at % a.V, o = b * p.n + j;
    p.out_scores[o] = float(s);
    p.parents[o] = k;
    p.tokens[o] = v;
    if (p.out_finished) p.out_finished[o] = ended[k] || v == p.end_token;
  };
  int filled = np < p.n ? np : p.n;
  if (__builtin_expect(np <= kPickList, 1)) {
    // rank each among all (distinct positions: distinct ranks)
    for (int t = tid; t < np; t += kPickBlock) {
      const double s = lscore[t];
      const int64_t at = lat[t];
      int rank = 0;
      for (int o = 0; o < np; ++o) rank += before(lscore[o], lat[o], s, at);
      if (rank < p.n) write(rank, s, at);
    }
  } else {
    double as = INFINITY;
    int64_t ai = -1;
    for (int j = 0; j < p.n; ++j) {
      double s = -INFINITY;
      int64_t at = INT64_MAX;
      auto offer = [&](double si, int64_t i) {
        if (si > -INFINITY && before(as, ai, si, i) && before(si, i, s, at)) {
          s = si;
          at = i;
        }
      };
      if (tid < p.K && ended[tid] && fabs(cum[tid]) < INFINITY) offer(cum[tid], tid * a.V + p.end_token);
      for (int c = wid; c < n_ch; c += kPickWaves) {
        const int item = chunks[c], k = item / n_chunk;
        Eight<DT> e;
        e.load(a.logits + (r0 + k) * a.row_bytes, token_at(item, 0), a.V, neg_inf<DT>());
#pragma unroll
        for (int i = 0; i < 8; ++i) offer(score_of(k, e.at(i)), k * a.V + token_at(item, i));
      }
      workgroup_best(s, at);
      if (!(s > -INFINITY)) {
        filled = j;
        break;
      }
      if (tid == 0) write(j, s, at);
      as = s;
      ai = at;
      filled = j + 1;
    }
  }
  if (tid >= filled && tid < p.n) {
    const int64_t o = b * p.n + tid;
    p.out_scores[o] = -INFINITY;
    p.parents[o] = -1;
    p.tokens[o] = -1;
    if (p.out_finished) p.out_finished[o] = 0;
  }
}

template <int DT>
void launch_select(const PickArgs& p, int64_t B, hipStream_t s) {
  const dim3 grid{unsigned((p.in.n_span + kScanBlock / 64 - 1) / (kScanBlock / 64)), unsigned(B * p.K)};
  hipLaunchKernelGGL(k_beam_scan<DT>, grid, dim3(kScanBlock), 0, s, p.in);
  if (hipPeekAtLastError() == hipSuccess)
    hipLaunchKernelGGL(k_beam_pick<DT>, dim3(unsigned(B)), dim3(kPickBlock), 0, s, p);
}

// ------------------------------------------------------------- reordering
// A workgroup takes a tile of one sequence's rows (the same bytes of each of
// its K beams) of one state.  A thread reads its units of every row that is
// continued elsewhere, then writes each to the rows that continue it: all reads
// of a unit come before all writes of it and no other thread touches it, so
// any parents may be applied in place, and a row is read once.
constexpr int kMoveBlock = 256;
constexpr int kMoveStates = 64;   // states of a launch

struct MoveArgs {
  archead_state_layout l;
  int B, K, n;
  const void* parents;
  const int32_t* lengths;
  int64_t units;      // units of a position
  int64_t most;       // units of an outer block with every position in use
  int n_states;
  bool wide_idx, in_place;
  const uint8_t* src[kMoveStates];
  uint8_t* dst[kMoveStates];
};

// U: the unit (16, 4 or 1 bytes); KM: the most rows of a sequence; FLAT:
// positions lie back to back in source and destination; NT: stores that are not
// kept in the caches
template <typename U, int KM, bool FLAT, bool NT>
__global__ __launch_bounds__(kMoveBlock) void k_beam_move(MoveArgs a) {
  const int lane = threadIdx.x & 63;
  for (int64_t z = blockIdx.z; z < int64_t(a.n_states) * a.B; z += gridDim.z) {
    const int st = int(z / a.B), b = int(z % a.B);
    int64_t len = a.l.positions;
    if (a.lengths) {
      const int64_t want = a.lengths[b];
      len = want < 0 ? 0 : want < len ? want : len;
    }
    const int64_t units = len * a.units;
    if (int64_t(blockIdx.x) * kMoveBlock >= units) continue;   // (uniform)
    int64_t parent = -1;
    if (lane < a.n) {
      parent = a.wide_idx ? static_cast<const int64_t*>(a.parents)[int64_t(b) * a.n + lane]
                          : static_cast<const int32_t*>(a.parents)[int64_t(b) * a.n + lane];
      if (a.in_place && parent == lane) parent = -1;   // stays where it is
    }
    uint64_t to[KM];   // the rows that continue row k
#pragma unroll
    for (int k = 0; k < KM; ++k) to[k] = k < a.K ? __ballot(parent == k) : 0;
    const uint8_t* const src_b = a.src[st] + int64_t(b) * a.K * a.l.src_row;
    uint8_t* const dst_b = a.dst[st] + int64_t(b) * a.n * a.l.dst_row;
    for (int64_t o = blockIdx.y; o < a.l.n_outer; o += gridDim.y) {
      for (int64_t u0 = int64_t(blockIdx.x) * kMoveBlock; u0 < units; u0 += int64_t(gridDim.x) * kMoveBlock) {
        const int64_t u = u0 + threadIdx.x;
        if (u >= units) continue;
        int64_t from = u * int64_t(sizeof(U)), at = from;
        if constexpr (!FLAT) {
          const int64_t pos = u / a.units, in = (u - pos * a.units) * int64_t(sizeof(U));
          from = pos * a.l.src_pos + in;
          at = pos * a.l.dst_pos + in;
        }
        const uint8_t* const src = src_b + o * a.l.src_outer + from;
        uint8_t* const dst = dst_b + o * a.l.dst_outer + at;
        U v[KM];
#pragma unroll
        for (int k = 0; k < KM; ++k)
          if (to[k]) v[k] = *reinterpret_cast<const U*>(src + k * a.l.src_row);
#pragma unroll
        for (int k = 0; k < KM; ++k)
          for (uint64_t m = to[k]; m; m &= m - 1) {
            U* const p = reinterpret_cast<U*>(dst + __builtin_ctzll(m) * a.l.dst_row);
            if constexpr (NT) __builtin_nontemporal_store(v[k], p);
            else *p = v[k];
          }
      }
    }
  }
}

template <typename U, int KM, bool FLAT, bool NT>
void launch_move_as(const MoveArgs& a, hipStream_t s) {
  const int64_t tiles = (a.most + kMoveBlock - 1) / kMoveBlock;
  auto upto = [](int64_t n, int64_t most) { return unsigned(n < most ? n : most); };
  hipLaunchKernelGGL((k_beam_move<U, KM, FLAT, NT>),
                     dim3(upto(tiles, 1 << 20), upto(a.l.n_outer, 65535), upto(int64_t(a.n_states) * a.B, 65535)),
                     dim3(kMoveBlock), 0, s, a);
}
template <typename U, bool FLAT, bool NT>
void launch_move_rows(const MoveArgs& a, hipStream_t s) {
  if (a.K <= 8) launch_move_as<U, 8, FLAT, NT>(a, s);
  else if (a.K <= 16) launch_move_as<U, 16, FLAT, NT>(a, s);
  else launch_move_as<U, ARCHEAD_BEAM_MAX, FLAT, NT>(a, s);
}
template <typename U, bool NT>
void launch_move(const MoveArgs& a, hipStream_t s) {
  const bool flat = a.l.positions == 1 || (a.l.src_pos == a.l.pos_bytes && a.l.dst_pos == a.l.pos_bytes);
  if (flat) launch_move_rows<U, true, NT>(a, s);
  else launch_move_rows<U, false, NT>(a, s);
}

}  // namespace

extern "C" {

size_t archead_beam_workspace_bytes(int64_t rows, int64_t V) {
  if (rows < 1 || V < 1 || rows > INT32_MAX || V > INT32_MAX) return 0;
  return archead::beam_layout(rows, V).total;
}

archead_status archead_beam_select(const void* logits, archead_dtype logits_dtype, int64_t B, int64_t K, int64_t V,
                                   int64_t ldl, const float* scores, const uint8_t* finished, int64_t end_token,
                                   int32_t n, float* out_scores, int64_t* parents, int64_t* tokens,
                                   uint8_t* out_finished, void* ws, size_t ws_bytes, void* stream) {
  using archead::fail;
  archead::clear_error();
  if (!float_dtype(logits_dtype)) return fail(ARCHEAD_E_INVALID_ARG, "logits_dtype must be F32, BF16 or F16");
  archead_status st = archead::beam_check(B, K, V, scores, finished, end_token, n, out_scores, parents, tokens);
  if (st != ARCHEAD_OK || B == 0) return st;
  if (ldl < V) return fail(ARCHEAD_E_INVALID_ARG, "ldl < V");
  if (!logits || !ws) return fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if (!aligned(logits, dtype_bytes(logits_dtype)) || !aligned(ws, 256))
    return fail(ARCHEAD_E_MISALIGNED, "logits / workspace misaligned");
  const archead::BeamLayout w = archead::beam_layout(B * K, V);
  if (ws_bytes < w.total) return fail(ARCHEAD_E_WORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, w.total);
  char* base = static_cast<char*>(ws);
  PickArgs p{};
  p.in = ScanArgs{static_cast<const uint8_t*>(logits), V, ldl * dtype_bytes(logits_dtype), w.n_span, scores, finished,
                  reinterpret_cast<float*>(base + w.cmax_off),
                  reinterpret_cast<archead::BeamSpanSum*>(base + w.span_off)};
  p.K = int(K);
  p.n = n;
  p.end_token = end_token;
  p.out_scores = out_scores;
  p.parents = parents;
  p.tokens = tokens;
  p.out_finished = out_finished;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (logits_dtype == ARCHEAD_F32) launch_select<ARCHEAD_F32>(p, B, s);
  else if (logits_dtype == ARCHEAD_BF16) launch_select<ARCHEAD_BF16>(p, B, s);
  else launch_select<ARCHEAD_F16>(p, B, s);
  return launch_status(hipGetLastError(), "beam selection launch");
}

archead_status archead_logits_beam(const archead_handle* h, const void* x, int64_t B, int64_t K, int64_t ldx,
                                   const float* scores, const uint8_t* finished, int64_t end_token, int32_t n,
                                   float* out_scores, int64_t* parents, int64_t* tokens, uint8_t* out_finished,
                                   void* ws, size_t ws_bytes, void* stream) {
  using archead::fail;
  archead::clear_error();
  if (!h) return fail(ARCHEAD_E_INVALID_ARG, "handle is NULL");
  const int64_t V = h->desc.V;
  archead_status st = archead::beam_check(B, K, V, scores, finished, end_token, n, out_scores, parents, tokens);
  if (st != ARCHEAD_OK || B == 0) return st;
  const int64_t M = B * K;
  const size_t need = archead_workspace_bytes(h, M, ARCHEAD_OP_BEAM);
  if (!ws) return fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if (!aligned(ws, 256)) return fail(ARCHEAD_E_MISALIGNED, "workspace misaligned");
  if (ws_bytes < need) return fail(ARCHEAD_E_WORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, need);
  // the logits, then the workspace of either of the two calls
  const size_t lg = archead::round256(size_t(M) * size_t(V) * 4);
  char* base = static_cast<char*>(ws);
  st = archead_logits(h, x, M, ldx, base, ARCHEAD_F32, V, base + lg, ws_bytes - lg, stream);
  if (st != ARCHEAD_OK) return st;
  return archead_beam_select(base, ARCHEAD_F32, B, K, V, V, scores, finished, end_token, n, out_scores, parents,
                             tokens, out_finished, base + lg, ws_bytes - lg, stream);
}

archead_status archead_beam_reorder(const archead_state_layout* layout, int64_t n_states, const void* const* src,
                                    void* const* dst, int64_t B, int64_t K, int64_t n, const void* parents,
                                    archead_dtype idx_dtype, const int32_t* lengths, void* stream) {
  using archead::fail;
  archead::clear_error();
  bool in_place = false;
  archead_status st = archead::reorder_check(layout, n_states, src, dst, B, K, n, parents, idx_dtype, lengths,
                                             &in_place);
  if (st != ARCHEAD_OK) return st;
  const archead_state_layout& l = *layout;
  if (n_states == 0 || B == 0 || l.n_outer == 0 || l.positions == 0 || l.pos_bytes == 0) return ARCHEAD_OK;
  uint64_t all = uint64_t(l.pos_bytes) | uint64_t(l.src_row) | uint64_t(l.dst_row);
  if (l.n_outer > 1) all |= uint64_t(l.src_outer) | uint64_t(l.dst_outer);
  if (l.positions > 1) all |= uint64_t(l.src_pos) | uint64_t(l.dst_pos);
  for (int64_t i = 0; i < n_states; ++i) all |= reinterpret_cast<uintptr_t>(src[i]) | reinterpret_cast<uintptr_t>(dst[i]);
  const int unit = all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 1;
  MoveArgs a{};
  a.l = l;
  a.B = int(B);
  a.K = int(K);
  a.n = int(n);
  a.parents = parents;
  a.lengths = lengths;
  a.wide_idx = idx_dtype == ARCHEAD_I64;
  a.in_place = in_place;
  a.units = l.pos_bytes / unit;
  a.most = l.positions * a.units;
  // Stores that are not kept in the caches, where the destinations do not fit
  // into the last one (256 MiB) in any case: 3.8 GB moved 699 -> 657 us, but
  // 0.9 MB 6.5 -> 7.5 us.
  const bool past_caches = double(n_states) * double(B * n) * double(l.n_outer) * double(l.positions) * double(l.pos_bytes) > 0x1p28;
  hipStream_t s = static_cast<hipStream_t>(stream);
  for (int64_t i0 = 0; i0 < n_states; i0 += kMoveStates) {
    a.n_states = int(n_states - i0 < kMoveStates ? n_states - i0 : kMoveStates);
    for (int i = 0; i < a.n_states; ++i) {
      a.src[i] = static_cast<const uint8_t*>(src[i0 + i]);
      a.dst[i] = static_cast<uint8_t*>(dst[i0 + i]);
    }
    if (unit == 16 && past_caches) launch_move<u32x4, true>(a, s);
    else if (unit == 16) launch_move<u32x4, false>(a, s);
    else if (unit == 4) launch_move<uint32_t, false>(a, s);
    else launch_move<uint8_t, false>(a, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return launch_status(e, "state reordering launch");
  }
  return ARCHEAD_OK;
}

}  // extern "C"
