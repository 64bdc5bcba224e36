// Beam search: the n best (beam, token) pairs of each sequence from rows of
// logits, and the reordering of the states they continue.
#include <float.h>

#include "beam.h"
#include "dev_rows.cuh"

namespace {

using namespace archead::rows;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------- selection
// Two launches.  k_beam_scan reads the logits once: of every chunk of a row
// its largest logit, and of every span of chunks (a wave's) the pair (maximum,
// sum of exponentials).  k_beam_pick, a workgroup per sequence, makes the rows'
// (maximum, sum) of them and with it the chunks' largest scores.  A score is
// (score of the beam - log sum) + (logit - maximum): the maximum and the log are
// not added up, since a row of the type's lowest value would lose the log.  If n chunks are
// ranked by (largest score, then position), every pair among the n best lies in
// one of the first n, so the logits of few more than those are read again.
// The scan is bound by the logits' bytes (256 rows x 262143 bf16: 134 MB in 26 us,
// 5.2 TB/s), the choice by its chain of reads and meetings (6 to 10 us).
// FINE: chunks of 128 logits (16 lanes' eight) instead of 512 (a wave's): fewer
// pairs above the floor that the chunks' maxima give, but four times as many
// chunks to look at.
constexpr int kScanBlock = 256;
constexpr int kSteps = archead::kBeamSpan / 512;   // a wave's loads of a span
__host__ __device__ constexpr int chunk_lanes(bool fine) { return fine ? 16 : 64; }
__host__ __device__ constexpr int chunk_logits(bool fine) { return 8 * chunk_lanes(fine); }
__host__ __device__ constexpr int span_chunks(bool fine) { return archead::kBeamSpan / chunk_logits(fine); }
static_assert(chunk_logits(true) == archead::kBeamChunk, "the workspace holds the smaller chunks' maxima");

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
  int64_t n_span;            // spans of a row
  const float* scores;
  const uint8_t* finished;   // may be null
  float* cmax;               // [rows][n_span][chunks of a span]
  archead::BeamSpanSum* span;   // [rows][n_span]
};

// The best of the lanes' values, in every lane: within rows of 16 lanes without
// LDS, then across the four rows.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u(uint32_t v) {
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float lane_f(float v, int l) {
  return __uint_as_float(uint32_t(__builtin_amdgcn_readlane(int(__float_as_uint(v)), l)));
}
template <int CTRL>
__device__ __forceinline__ float dpp_f(float v) {
  return __uint_as_float(dpp_u<CTRL>(__float_as_uint(v)));
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, dpp_f<0xB1>(v));
  v = fmaxf(v, dpp_f<0x4E>(v));
  v = fmaxf(v, dpp_f<0x141>(v));
  return fmaxf(v, dpp_f<0x140>(v));
}
__device__ __forceinline__ float rows_max(float v) {
  return fmaxf(fmaxf(lane_f(v, 0), lane_f(v, 16)), fmaxf(lane_f(v, 32), lane_f(v, 48)));
}
__device__ __forceinline__ float wave_max(float v) { return rows_max(row_max(v)); }
__device__ __forceinline__ double of_words(uint32_t lo, uint32_t hi) {
  return __longlong_as_double((long long)(uint64_t(hi) << 32 | lo));
}
template <int CTRL>
__device__ __forceinline__ double dpp_d(double v) {
  const uint64_t u = uint64_t(__double_as_longlong(v));
  return of_words(dpp_u<CTRL>(uint32_t(u)), dpp_u<CTRL>(uint32_t(u >> 32)));
}
__device__ __forceinline__ double lane_d(double v, int l) {
  const uint64_t u = uint64_t(__double_as_longlong(v));
  return of_words(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(u)), l)),
                  uint32_t(__builtin_amdgcn_readlane(int(uint32_t(u >> 32)), l)));
}
__device__ __forceinline__ double wave_sum(double v) {
  v += dpp_d<0xB1>(v);
  v += dpp_d<0x4E>(v);
  v += dpp_d<0x141>(v);
  v += dpp_d<0x140>(v);
  return (lane_d(v, 0) + lane_d(v, 16)) + (lane_d(v, 32) + lane_d(v, 48));
}

// whether a row's logits say anything
__device__ __forceinline__ bool row_counts(const ScanArgs& a, int64_t r) {
  return fabsf(a.scores[r]) < INFINITY && !(a.finished && a.finished[r]);
}

// Span sp of row r, by a wave: its logits, then its chunks' largest to cmax and its
// sum of exponentials to *span.
template <int DT>
__device__ __forceinline__ void load_span(Eight<DT> (&e)[kSteps], const ScanArgs& a, int64_t r, int64_t sp, int lane) {
  const uint8_t* row = a.logits + r * a.row_bytes;
#pragma unroll
  for (int c = 0; c < kSteps; ++c)
    e[c].load(row, sp * archead::kBeamSpan + c * 512 + lane * 8, a.V, neg_inf<DT>());
}
template <int DT, bool FINE>
__device__ __forceinline__ void scan_span(const Eight<DT> (&e)[kSteps], int lane, float* cmax, archead::BeamSpanSum* span) {
  float cm[kSteps], top = -INFINITY;   // cm: of 16 lanes
#pragma unroll
  for (int c = 0; c < kSteps; ++c) {
    float m = e[c].at(0);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = fmaxf(m, e[c].at(i));
    cm[c] = row_max(m);
    if constexpr (!FINE) cm[c] = rows_max(cm[c]);
    top = fmaxf(top, cm[c]);
  }
  if constexpr (FINE) top = rows_max(top);
  // relative to 0 where nothing is above -inf: every term is then 0, or NaN
  const float ref = top > -INFINITY ? top : 0.f;
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < kSteps; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) s += __builtin_amdgcn_exp2f((e[c].at(i) - ref) * 1.4426950408889634f);
  const double sd = wave_sum(double(s));
  if (lane == 0) *span = archead::BeamSpanSum{sd, ref};
  const int c = lane & 15;   // lane c of a row of 16 writes its maximum of step c
  if (c < kSteps && (FINE || lane < 16)) {
    float m = cm[0];
#pragma unroll
    for (int i = 1; i < kSteps; ++i) m = c == i ? cm[i] : m;
    cmax[FINE ? 4 * c + (lane >> 4) : c] = m;
  }
}

template <int DT, bool FINE>
__global__ __launch_bounds__(kScanBlock) void k_beam_scan(ScanArgs a) {
  const int lane = threadIdx.x & 63;
  const int wid = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int64_t r = blockIdx.y, sp = int64_t(blockIdx.x) * (kScanBlock / 64) + wid;
  if (sp >= a.n_span || !row_counts(a, r)) return;
  const int64_t i = r * a.n_span + sp;
  Eight<DT> e[kSteps];
  load_span<DT>(e, a, r, sp, lane);
  scan_span<DT, FINE>(e, lane, a.cmax + i * span_chunks(FINE), a.span + i);
}

constexpr int kPickBlock = 1024, kPickWaves = kPickBlock / 64;
constexpr int kPickHeld = 4;     // chunks whose largest logits a thread keeps
constexpr int kPickAhead = 2;    // listed chunks that a thread reads of at a time
constexpr int kPickSpans = 4;    // spans whose sums a lane keeps
constexpr int kPickGroups = kPickBlock / 16;   // groups of threads that share a maximum
constexpr int kPickList = 512;   // chunks, and pairs, that are ranked one against all
static_assert(kPickList >= archead::kTopKMaxK + ARCHEAD_BEAM_MAX, "room for the n best and the ended beams");
constexpr int kFewSpans = 2 * kPickWaves;   // spans of a sequence up to which there is no first launch
constexpr int kFineMost = 64;    // spans of a sequence up to which the chunks are the smaller ones
constexpr int kPickRank = 96;    // pairs up to which no second floor is looked for
static_assert(kPickGroups == 64, "a lane of a wave for each");

struct PickArgs {
  ScanArgs in;
  int K, n;
  int64_t end_token;
  float* out_scores;
  int64_t *parents, *tokens;
  uint8_t* out_finished;   // may be null
};

struct __align__(16) Ranked {
  double score;
  uint64_t at;
};
// the order of pairs (beam << 32 | token) and of chunks (their number)
__device__ __forceinline__ bool before(double sa, uint64_t ia, double sb, uint64_t ib) {
  return sa > sb || (sa == sb && ia < ib);
}

// FEW: few spans in a sequence, which the waves read here (no first launch)
template <int DT, bool FINE, bool FEW>
__global__ __launch_bounds__(kPickBlock) void k_beam_pick(PickArgs p) {
  __shared__ float few_cmax[FEW ? kFewSpans * span_chunks(FINE) : 1];
  __shared__ archead::BeamSpanSum few_span[FEW ? kFewSpans : 1];
  // of a beam: score, score less the log of its sum (NaN where the row offers
  // nothing by its logits), largest logit
  __shared__ double cum[ARCHEAD_BEAM_MAX], base[ARCHEAD_BEAM_MAX], most[ARCHEAD_BEAM_MAX];
  __shared__ bool ended[ARCHEAD_BEAM_MAX];
  __shared__ uint32_t skey[kPickGroups], lane_key[kPickBlock];
  __shared__ Ranked list[kPickList];
  __shared__ int chunks[kPickList];
  __shared__ double wscore[kPickWaves];
  __shared__ uint64_t wat[kPickWaves];
  __shared__ int n_list, n_pair;
  const ScanArgs& a = p.in;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t b = blockIdx.x, r0 = b * p.K;
  const int n_span = int(a.n_span), stored = n_span * span_chunks(FINE);   // a row's maxima in memory
  const int n_chunk = int((a.V + chunk_logits(FINE) - 1) / chunk_logits(FINE)), n_items = n_chunk * p.K;   // (K V / 512 < 2^27)
  if (tid == 0) n_list = n_pair = 0;
  if constexpr (FEW) {
    // the loads of a wave's two spans together
    Eight<DT> e[2][kSteps];
    bool use[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = wid + u * kPickWaves, k = i / n_span;
      use[u] = k < p.K && row_counts(a, r0 + k);
      if (use[u]) load_span<DT>(e[u], a, r0 + k, i - k * n_span, lane);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (use[u]) scan_span<DT, FINE>(e[u], lane, few_cmax + (wid + u * kPickWaves) * span_chunks(FINE), few_span + wid + u * kPickWaves);
    __syncthreads();
  }
  auto cmax_of = [&](int item) {
    const int k = item / n_chunk, c = item - k * n_chunk;
    if constexpr (FEW) return few_cmax[k * stored + c];
    else return a.cmax[(r0 + k) * stored + c];
  };
  auto span_of = [&](int k, int i) {
    if constexpr (FEW) return few_span[k * n_span + i];
    else return a.span[(r0 + k) * a.n_span + i];
  };
  // item i of u: chunk i % n_chunk of beam i / n_chunk; neighbouring items go
  // to different groups of 16 threads
  auto item_at = [&](int u) { return u * kPickBlock + (tid & 15) * kPickGroups + (tid >> 4); };
  float held[kPickHeld];   // (of rows that say nothing: whatever the workspace holds)
#pragma unroll
  for (int u = 0; u < kPickHeld; ++u) held[u] = item_at(u) < n_items ? cmax_of(item_at(u)) : -INFINITY;
  for (int k = wid; k < p.K; k += kPickWaves) {
    archead::BeamSpanSum first[kPickSpans];
#pragma unroll
    for (int u = 0; u < kPickSpans; ++u)
      first[u] = lane + 64 * u < n_span ? span_of(k, lane + 64 * u) : archead::BeamSpanSum{0.0, 0.f};
    const float c = a.scores[r0 + k];
    const bool f = a.finished && a.finished[r0 + k];
    double from = NAN;
    float top = -INFINITY;
    if (fabsf(c) < INFINITY && !f) {
      // (a span with nothing above -inf has the sum 0, whatever its maximum)
#pragma unroll
      for (int u = 0; u < kPickSpans; ++u) top = first[u].sum != 0.0 ? fmaxf(top, first[u].top) : top;
      for (int i = lane + 64 * kPickSpans; i < n_span; i += 64) {
        const archead::BeamSpanSum v = span_of(k, i);
        top = v.sum != 0.0 ? fmaxf(top, v.top) : top;
      }
      top = wave_max(top);
      double s = 0.0;
      auto add = [&](const archead::BeamSpanSum& v) {
        s += v.sum * exp(v.sum != 0.0 ? double(v.top) - double(top) : 0.0);
      };
#pragma unroll
      for (int u = 0; u < kPickSpans; ++u)
        if (64 * u < n_span) add(first[u]);
      for (int i = lane + 64 * kPickSpans; i < n_span; i += 64) add(span_of(k, i));
      s = wave_sum(s);
      // +inf among the logits: a term inf - inf, so the sum is NaN
      if (s > 0.0) from = c - log(s);
    }
    if (lane == 0) {
      cum[k] = c;
      base[k] = from;
      most[k] = top;
      ended[k] = f;
    }
  }
  __syncthreads();
  auto score_of = [&](int k, float logit) { return base[k] + (double(logit) - most[k]); };
  auto chunk_score = [&](int item, float top) {
    const int k = item / n_chunk;
    return base[k] == base[k] ? score_of(k, top) : double(-INFINITY);
  };
  auto score_again = [&](int item) { return chunk_score(item, cmax_of(item)); };
  // ---- a floor: about the n-th largest of the groups' best chunks, in the
  // order's first 32 bits
  double mine[kPickHeld];
  uint32_t best = 0;
#pragma unroll
  for (int u = 0; u < kPickHeld; ++u) {
    mine[u] = item_at(u) < n_items ? chunk_score(item_at(u), held[u]) : -INFINITY;
    best = max(best, uint32_t(order_key(mine[u]) >> 32));
  }
  for (int u = kPickHeld; u * kPickBlock < n_items; ++u)
    if (item_at(u) < n_items) best = max(best, uint32_t(order_key(score_again(item_at(u))) >> 32));
  best = max(best, dpp_u<0xB1>(best));
  best = max(best, dpp_u<0x4E>(best));
  best = max(best, dpp_u<0x141>(best));
  best = max(best, dpp_u<0x140>(best));
  if ((tid & 15) == 0) skey[tid >> 4] = best;
  __syncthreads();
  // (every wave finds it: no second meeting)
  uint32_t floor = 0;
  {
    const uint32_t key = skey[lane];
    int reach = kPickGroups;
    const int enough = p.n + p.n / 4;
    // the bits in which no two keys differ come first
    const uint32_t some = uint32_t(__builtin_amdgcn_readfirstlane(int(key)));
    uint32_t differ = key ^ some;
    differ |= dpp_u<0xB1>(differ);
    differ |= dpp_u<0x4E>(differ);
    differ |= dpp_u<0x141>(differ);
    differ |= dpp_u<0x140>(differ);
    auto row = [&](int l) { return uint32_t(__builtin_amdgcn_readlane(int(differ), l)); };
    const uint32_t all = row(0) | row(16) | row(32) | row(48);
    const int high = all ? 31 - __builtin_clz(all) : -1;
    floor = high == 31 ? 0u : some >> (high + 1) << (high + 1);
    for (int bit = high; bit >= 0 && reach > enough; --bit) {
      const uint32_t t = floor | (1u << bit);
      const int c = __popcll(__ballot(key >= t));
      if (c >= p.n) {
        floor = t;
        reach = c;
      }
    }
    floor = max(floor, 1u);   // 1: every candidate
  }
  // ---- the chunks that reach it
  auto list_chunk = [&](int i, double s) {
    if (uint32_t(order_key(s) >> 32) < floor) return;
    const int at = atomicAdd(&n_list, 1);
    if (at < kPickList) chunks[at] = i;
  };
#pragma unroll
  for (int u = 0; u < kPickHeld; ++u)
    if (u * kPickBlock < n_items) list_chunk(item_at(u), mine[u]);
  for (int u = kPickHeld; u * kPickBlock < n_items; ++u)
    if (item_at(u) < n_items) list_chunk(item_at(u), score_again(item_at(u)));
  __syncthreads();
  // the best of the threads' (s, i), in every thread
  auto workgroup_best = [&](double& s, uint64_t& i) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const double os = __shfl_xor(s, o, 64);
      const uint64_t oi = __shfl_xor((unsigned long long)i, o, 64);
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
    uint64_t ai = 0;
    n_ch = 0;
    for (int j = 0; j < p.n; ++j) {
      double s = -INFINITY;
      uint64_t at = UINT64_MAX;
      for (int i = tid; i < n_items; i += kPickBlock) {
        const double si = score_again(i);
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
  auto offers_end = [&](int k) { return k < p.K && ended[k] && fabs(cum[k]) < INFINITY; };
  auto pair = [&](int k, int64_t v) { return uint64_t(k) << 32 | uint64_t(v); };
  constexpr int kLanes = chunk_lanes(FINE), kAtOnce = kPickBlock / kLanes;   // chunks that the workgroup reads at once
  const int eight = tid % kLanes * 8;
  auto fetch = [&](Eight<DT>& e, int c) {   // this lane's eight logits of listed chunk c
    const int item = chunks[c], k = item / n_chunk;
    e.load(a.logits + (r0 + k) * a.row_bytes, int64_t(item - k * n_chunk) * chunk_logits(FINE) + eight, a.V, neg_inf<DT>());
  };
  auto each = [&](const Eight<DT>& e, int c, auto use) {   // use(score, pair) for them
    const int item = chunks[c], k = item / n_chunk;
    const int64_t v0 = int64_t(item - k * n_chunk) * chunk_logits(FINE) + eight;
#pragma unroll
    for (int i = 0; i < 8; ++i) use(score_of(k, e.at(i)), pair(k, v0 + i));
  };
  auto each_logit = [&](auto use) {   // of the listed chunks
    for (int c0 = tid / kLanes; c0 < n_ch; c0 += kPickAhead * kAtOnce) {
      Eight<DT> e[kPickAhead];
#pragma unroll
      for (int u = 0; u < kPickAhead; ++u)
        if (c0 + u * kAtOnce < n_ch) fetch(e[u], c0 + u * kAtOnce);
#pragma unroll
      for (int u = 0; u < kPickAhead; ++u)
        if (c0 + u * kAtOnce < n_ch) each(e[u], c0 + u * kAtOnce, use);
    }
  };
  auto put = [&](double s, uint64_t i) {
    const int at = atomicAdd(&n_pair, 1);
    if (at < kPickList) list[at] = Ranked{s, i};
  };
  // the least score whose order begins with f (below 1: -inf alone)
  auto score_at = [](uint32_t f) {
    const uint64_t k = uint64_t(f) << 32;
    return f > 1 ? __longlong_as_double((long long)(k >> 63 ? k ^ (uint64_t(1) << 63) : ~k)) : -DBL_MAX;
  };
  const double least = score_at(floor);
  double top = -INFINITY;   // this lane's best pair
  if (offers_end(tid)) {
    top = cum[tid];
    put(cum[tid], pair(tid, p.end_token));
  }
  each_logit([&](double s, uint64_t i) {
    if (s >= least) {
      top = fmax(top, s);
      put(s, i);
    }
  });
  __syncthreads();
  int np = n_pair;
  if (np > kPickRank) {
    // More than are ranked quickly (beams of unlike scores, few chunks, the best
    // logits side by side): a second floor, about the n-th largest of those
    // listed, or of the lanes' best where they are too many to list.
    const bool listed = np <= kPickList;
    Ranked r{-INFINITY, 0};
    if (listed && tid < np) r = list[tid];
    lane_key[tid] = uint32_t(order_key(listed ? r.score : top) >> 32);
    __syncthreads();
    if (wid == 0) {
      if (lane == 0) n_pair = 0;
      const int regs = listed ? kPickList / 64 : kPickWaves;
      uint32_t kk[kPickWaves];
#pragma unroll
      for (int i = 0; i < kPickWaves; ++i) kk[i] = i < regs ? lane_key[64 * i + lane] : 0u;
      uint32_t f = 0;
      int reach = kPickBlock;
      for (int bit = 31; bit >= 0 && reach > p.n + p.n / 4; --bit) {
        const uint32_t t = f | (1u << bit);
        int c = 0;
#pragma unroll
        for (int i = 0; i < kPickWaves; ++i)
          if (i < regs) c += __popcll(__ballot(kk[i] >= t));
        if (c >= p.n) {
          f = t;
          reach = c;
        }
      }
      if (lane == 0) skey[0] = max(f, 1u);
    }
    __syncthreads();
    const double least2 = score_at(skey[0]);
    if (listed) {
      if (tid < np && r.score >= least2) put(r.score, r.at);
    } else {
      if (offers_end(tid) && cum[tid] >= least2) put(cum[tid], pair(tid, p.end_token));
      each_logit([&](double s, uint64_t i) {
        if (s >= least2) put(s, i);
      });
    }
    __syncthreads();
    np = n_pair;
  }
  auto write = [&](int j, double s, uint64_t at) {
    const int k = int(at >> 32);
    const int64_t v = int64_t(at & 0xffffffffu), o = b * p.n + j;
    p.out_scores[o] = float(s);
    p.parents[o] = k;
    p.tokens[o] = v;
    if (p.out_finished) p.out_finished[o] = ended[k] || v == p.end_token;
  };
  int filled = np < p.n ? np : p.n;
  if (__builtin_expect(np <= kPickList, 1)) {
    // rank each among all (distinct positions: distinct ranks), 16 lanes to one
    for (int c = tid >> 4; c < np; c += kPickGroups) {
      const Ranked r = list[c];
      uint32_t rank = 0;
      for (int o = tid & 15; o < np; o += 16) {
        const Ranked x = list[o];
        rank += before(x.score, x.at, r.score, r.at);
      }
      rank += dpp_u<0xB1>(rank);
      rank += dpp_u<0x4E>(rank);
      rank += dpp_u<0x141>(rank);
      rank += dpp_u<0x140>(rank);
      if ((tid & 15) == 0 && rank < uint32_t(p.n)) write(int(rank), r.score, r.at);
    }
  } else {
    double as = INFINITY;
    uint64_t ai = 0;
    for (int j = 0; j < p.n; ++j) {
      double s = -INFINITY;
      uint64_t at = UINT64_MAX;
      auto offer = [&](double si, uint64_t i) {
        if (si > -INFINITY && before(as, ai, si, i) && before(si, i, s, at)) {
          s = si;
          at = i;
        }
      };
      if (offers_end(tid)) offer(cum[tid], pair(tid, p.end_token));
      each_logit(offer);
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

template <int DT, bool FINE>
hipError_t launch_select_as(const PickArgs& p, int64_t B, hipStream_t s) {
  const dim3 grid{unsigned((p.in.n_span + kScanBlock / 64 - 1) / (kScanBlock / 64)), unsigned(B * p.K)};
  const hipError_t e = launch_kernel(k_beam_scan<DT, FINE>, grid, dim3(kScanBlock), 0, s, p.in);
  if (e != hipSuccess) return e;
  return launch_kernel(k_beam_pick<DT, FINE, false>, dim3(unsigned(B)), dim3(kPickBlock), 0, s, p);
}

template <int DT>
hipError_t launch_select(const PickArgs& p, int64_t B, hipStream_t s) {
  // One launch where a wave has two spans of a sequence at most: us with two
  // launches / one in a loop of calls 15.7 / 12.6 (a launch takes the host 3), replayed
  // from a graph 9.3 / 9.3 at 20 spans and 9.9 / 11.3 at 30; at 64 in one 8.8 / 16.
  if (p.in.n_span * p.K <= kFewSpans)
    return launch_kernel(k_beam_pick<DT, true, true>, dim3(unsigned(B)), dim3(kPickBlock), 0, s, p);
  // us with chunks of 128 / 512: 12 x 16 beams over 4320 tokens 11.6 / 25, 4 over
  // 32000 (64 spans) 8.6 / 9.3, over 50257 (100) 9.2 / 8.6, 8 x 4 over 151936 15.3 / 13.1.
  return p.in.n_span * p.K <= kFineMost ? launch_select_as<DT, true>(p, B, s) : launch_select_as<DT, false>(p, B, s);
}

// ------------------------------------------------------------- reordering
// A workgroup takes a tile of one sequence's rows (the same bytes of each of
// its K beams) of one state.  A thread reads its units of every row that is
// continued elsewhere, then writes each to the rows that continue it: all reads
// of a unit come before all writes of it and no other thread touches it, so
// any parents may be applied in place, and a row is read once.  Bound by the
// bytes moved: 3.8 GB (reads and writes) in 658 us, 5.8 TB/s.
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
hipError_t launch_move_as(const MoveArgs& a, hipStream_t s) {
  const int64_t tiles = (a.most + kMoveBlock - 1) / kMoveBlock;
  auto upto = [](int64_t n, int64_t most) { return unsigned(n < most ? n : most); };
  return launch_kernel(k_beam_move<U, KM, FLAT, NT>,
                       dim3(upto(tiles, 1 << 20), upto(a.l.n_outer, 65535), upto(int64_t(a.n_states) * a.B, 65535)),
                       dim3(kMoveBlock), 0, s, a);
}
template <typename U, bool FLAT, bool NT>
hipError_t launch_move_rows(const MoveArgs& a, hipStream_t s) {
  if (a.K <= 8) return launch_move_as<U, 8, FLAT, NT>(a, s);
  if (a.K <= 16) return launch_move_as<U, 16, FLAT, NT>(a, s);
  return launch_move_as<U, ARCHEAD_BEAM_MAX, FLAT, NT>(a, s);
}
template <typename U, bool NT>
hipError_t launch_move(const MoveArgs& a, hipStream_t s) {
  const bool flat = a.l.positions == 1 || (a.l.src_pos == a.l.pos_bytes && a.l.dst_pos == a.l.pos_bytes);
  return flat ? launch_move_rows<U, true, NT>(a, s) : launch_move_rows<U, false, NT>(a, s);
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
  const archead::BeamLayout w = archead::beam_layout(B * K, V);
  if (!logits || !ws) return fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if (!aligned(logits, dtype_bytes(logits_dtype)) || !aligned(ws, 256))
    return fail(ARCHEAD_E_MISALIGNED, "logits / workspace misaligned");
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
  const hipError_t e = logits_dtype == ARCHEAD_F32    ? launch_select<ARCHEAD_F32>(p, B, s)
                       : logits_dtype == ARCHEAD_BF16 ? launch_select<ARCHEAD_BF16>(p, B, s)
                                                      : launch_select<ARCHEAD_F16>(p, B, s);
  return launch_status(e, "beam selection launch");
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
    const hipError_t e = unit == 16 && past_caches ? launch_move<u32x4, true>(a, s)
                         : unit == 16              ? launch_move<u32x4, false>(a, s)
                         : unit == 4               ? launch_move<uint32_t, false>(a, s)
                                                   : launch_move<uint8_t, false>(a, s);
    if (e != hipSuccess) return launch_status(e, "state reordering launch");
  }
  return ARCHEAD_OK;
}

}  // extern "C"
