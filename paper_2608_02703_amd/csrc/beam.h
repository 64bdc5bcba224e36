// Beam search: workspace layout and argument checks (host).
#pragma once

#include "internal.h"

namespace archead {

inline size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

constexpr int kBeamChunk = 128;    // logits of a chunk, the least
constexpr int kBeamSpan = 2048;    // logits of a span, a wave's share of a row

// of a span of a row: sum of exp(logit - top); top is its largest logit, or 0
// where nothing is above -inf
struct BeamSpanSum {
  double sum;
  float top;
};

struct BeamLayout {
  int64_t n_span = 0;
  size_t cmax_off = 0, span_off = 0, total = 0;
};
inline BeamLayout beam_layout(int64_t rows, int64_t V) {
  BeamLayout w;
  w.n_span = (V + kBeamSpan - 1) / kBeamSpan;
  w.span_off = round256(size_t(rows) * size_t(w.n_span) * (kBeamSpan / kBeamChunk) * sizeof(float));
  w.total = w.span_off + round256(size_t(rows) * size_t(w.n_span) * sizeof(BeamSpanSum));
  return w;
}

// the checks that archead_beam_select and archead_logits_beam share, and those of
// archead_beam_reorder; ARCHEAD_OK, or a status with its message set
archead_status beam_check(int64_t B, int64_t K, int64_t V, const float* scores, const uint8_t* finished,
                          int64_t end_token, int32_t n, const float* out_scores, const int64_t* parents,
                          const int64_t* tokens);
archead_status reorder_check(const archead_state_layout* l, int64_t n_states, const void* const* src,
                             void* const* dst, int64_t B, int64_t K, int64_t n, const void* parents,
                             archead_dtype idx_dtype, const int32_t* lengths, bool* in_place);

}  // namespace archead
