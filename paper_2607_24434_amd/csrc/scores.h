// Row operators over a vocabulary: token scores (log probabilities, entropy, best
// alternatives) and distillation from a teacher's top logits, with their gradients.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace de {

constexpr int kTopMax = 128;  // most alternatives, and most entries of a teacher's list, a row
constexpr int kStats = 4;     // floats a row of token scores keeps for its gradient
constexpr int kState = 4;     // floats a distillation row keeps beside one per entry

// The rows that every call reads, and the scale of their softmax: exp((l - max) / tau) is
// 2^d with d = (l - max) c, c = log2(e) / tau rounded.  The rounding moves every d the same
// way, and a loss is a small difference of sums of such terms; to first order, sum 2^d is
// right with corr * (sum 2^d d) added, a sum that the entropy takes anyway.
struct VocabRows {
  int rows, V;
  int bf16;            // 0: fp32 logits
  const void* logits;  // [rows, ld]
  int64_t ld;
  float tau, c, corr;
};

// Incoming gradients and where the logits' gradient goes (dlogits NULL: none).
struct RowGrad {
  const float* g;          // [rows] or NULL
  const float* g_entropy;  // [rows] or NULL
  void* dlogits;           // [rows, ldd], the logits' type
  int64_t ldd;
};

struct ScoresArgs {
  VocabRows x;
  const int32_t* tokens;  // [rows] or NULL
  float* logp;            // [rows] or NULL
  float* entropy;         // [rows] or NULL
  int m;
  int32_t* top_idx;       // [rows, m]
  float* top_logp;        // [rows, m]
  float* stats;           // [rows, kStats] or NULL
};

struct DistillArgs {
  VocabRows x;
  int m;
  const int32_t* ids;     // [rows, m]
  const float* values;    // [rows, m]
  int tail;
  float* loss;            // [rows]
  float* state;           // [rows, m + kState] or NULL
};

// Scratch of launch_scores and (m = 0) launch_distill, 16-byte aligned.
size_t scores_bytes(int rows, int V, int m);
// With g.dlogits the gradient too, for which a.stats (a.state) must not be NULL.
hipError_t launch_scores(const ScoresArgs& a, const RowGrad& g, void* ws, hipStream_t s);
hipError_t launch_scores_grad(const VocabRows& x, const int32_t* tokens, const float* stats,
                              const RowGrad& g, hipStream_t s);
hipError_t launch_distill(const DistillArgs& a, const RowGrad& g, void* ws, hipStream_t s);
hipError_t launch_distill_grad(const VocabRows& x, int m, const int32_t* ids, const float* state,
                               const RowGrad& g, hipStream_t s);

}  // namespace de
