// Token scores and distillation from a teacher's top logits, forward and backward.
//
// With z = l / tau, M = max l and S = sum_v exp((l_v - M) / tau):
//   log p_v = (l_v - M) / tau - log S,     H = log S - (sum_v e_v d_v) / S
// (e_v the summand, d_v = (l_v - M) / tau).  Differences to the maximum are taken before
// they are scaled, so that logits far from zero lose nothing.
#include "de_common.h"
#include "scores.h"

namespace de {
namespace {

constexpr int kRowThreads = 1024;
constexpr int kGradThreads = 256, kGradChunk = 4096;
constexpr int kMarkWords = 1024;  // marks of list entries: 32768 logits at a time
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float nan_f() { return __int_as_float(0x7fc00000); }

__device__ __forceinline__ float load1(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float load1(const uint16_t* p, int64_t i) {
  return __uint_as_float((uint32_t)p[i] << 16);
}
__device__ __forceinline__ void store1(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void store1(uint16_t* p, int64_t i, float v) {
  p[i] = __builtin_bit_cast(uint16_t, (__bf16)v);  // to nearest, ties to even; a NaN stays one
}

// log2 of exp((l - top) / tau), from a floor up: for -infinity, and for a NaN unless
// `nan` keeps it.
template <bool nan>
__device__ __forceinline__ float scaled(const VocabRows& x, float l, float top) {
  float d = l - top;
  d = nan ? (d < x.floor ? x.floor : d) : fmaxf(d, x.floor);
  return fmaf(d, x.c_lo, d * x.c_hi);
}

// log p of one logit (a NaN is -infinity).
__device__ __forceinline__ float log_p(float tau, float l, float top, float log_s) {
  return l == l ? (l - top) / tau - log_s : log_s == log_s ? -INFINITY : log_s;
}

// A whole number that orders values as their floats do (a NaN as -infinity, -0 as +0).
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v == v ? v + 0.f : -INFINITY);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
// ... and the lower index first.
__device__ __forceinline__ uint64_t order_key(float v, int i) {
  return (uint64_t)order_key(v) << 32 | (0xffffffffu - (uint32_t)i);
}

template <typename V, typename Op>
__device__ __forceinline__ V block_all(V v, V* red, Op op) {
  for (int o = 32; o > 0; o >>= 1) v = op(v, (V)__shfl_xor(v, o, kWave));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  V t = red[0];
  for (int w = 1; w < (int)blockDim.x / 64; ++w) t = op(t, red[w]);
  return t;
}
struct MaxOp {
  template <typename V>
  __device__ V operator()(V a, V b) const { return a > b ? a : b; }
};
struct SumOp {
  template <typename V>
  __device__ V operator()(V a, V b) const { return a + b; }
};

// One block per row.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void scores_kernel(ScoresArgs a) {
  __shared__ float red[kRowThreads / 64];
  __shared__ unsigned long long redk[kRowThreads / 64];
  const int r = blockIdx.x;
  const T* row = static_cast<const T*>(a.x.logits) + (int64_t)r * a.x.ld;
  float top = -INFINITY;
  for (int i = threadIdx.x; i < a.x.V; i += kRowThreads) top = fmaxf(top, load1(row, i));
  top = block_all(top, red, MaxOp{});
  float s = 0.f, w = 0.f;
  for (int i = threadIdx.x; i < a.x.V; i += kRowThreads) {
    const float d = scaled<false>(a.x, load1(row, i), top), e = exp2f(d);
    s += e;
    w += e * d;
  }
  s = block_all(s, red, SumOp{});
  w = block_all(w, red, SumOp{});
  // No distribution: nothing above -infinity, or an infinite logit.
  if (!(fabsf(top) < INFINITY)) s = w = nan_f();
  const float log_s = logf(s);
  if (threadIdx.x == 0) {
    const float h = log_s - w / s * kLn2;
    if (a.logp != nullptr) {
      const int t = a.tokens[r];
      a.logp[r] = t < 0 ? 0.f : t >= a.x.V ? nan_f() : log_p(a.x.tau, load1(row, t), top, log_s);
    }
    if (a.entropy != nullptr) a.entropy[r] = h;
    if (a.stats != nullptr) {
      float* st = a.stats + (int64_t)r * kStats;
      st[0] = top;
      st[1] = s;
      st[2] = h;
      st[3] = top / a.x.tau + log_s;
    }
  }
  unsigned long long last = ~0ull;
  for (int j = 0; j < a.m; ++j) {
    unsigned long long best = 0;
    for (int i = threadIdx.x; i < a.x.V; i += kRowThreads) {
      const unsigned long long k = order_key(load1(row, i), i);
      if (k < last && k > best) best = k;
    }
    last = block_all(best, redk, MaxOp{});
    if (threadIdx.x == 0) {
      const int i = (int)(0xffffffffu - (uint32_t)last);
      a.top_idx[(int64_t)r * a.m + j] = i;
      a.top_logp[(int64_t)r * a.m + j] = log_p(a.x.tau, load1(row, i), top, log_s);
    }
  }
}

// One block per row and kGradChunk logits.
template <typename T>
__global__ __launch_bounds__(kGradThreads) void scores_grad_kernel(VocabRows x, const int32_t* tokens,
                                                                   const float* stats, RowGrad g,
                                                                   int chunks) {
  const int r = blockIdx.x / chunks, i0 = blockIdx.x % chunks * kGradChunk;
  const T* row = static_cast<const T*>(x.logits) + (int64_t)r * x.ld;
  T* out = static_cast<T*>(g.dlogits) + (int64_t)r * g.ldd;
  const int t = tokens != nullptr ? tokens[r] : -1;
  float gl = g.g != nullptr && t >= 0 ? g.g[r] : 0.f;
  const float ge = g.g_entropy != nullptr ? g.g_entropy[r] : 0.f;
  const int end = min(x.V, i0 + kGradChunk);
  if (gl == 0.f && ge == 0.f) {  // a row without weight: zeros, whatever its logits hold
    for (int i = i0 + threadIdx.x; i < end; i += kGradThreads) store1(out, i, 0.f);
    return;
  }
  if (t >= x.V && gl != 0.f) gl = nan_f();
  const float* st = stats + (int64_t)r * kStats;
  const float top = st[0], inv = 1.f / st[1], b = st[2] - logf(st[1]), it = 1.f / x.tau;
  for (int i = i0 + threadIdx.x; i < end; i += kGradThreads) {
    const float d = scaled<false>(x, load1(row, i), top), p = exp2f(d) * inv;
    float v = -p * (gl + ge * fmaf(d, kLn2, b));
    if (i == t) v += gl;
    store1(out, i, v * it);
  }
}

// One block per row.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void distill_kernel(DistillArgs a) {
  __shared__ float red[kRowThreads / 64];
  __shared__ double redd[kRowThreads / 64];
  __shared__ uint32_t mark[kMarkWords];
  __shared__ int32_t ids[kTopMax];
  const int r = blockIdx.x, j = threadIdx.x;
  const T* row = static_cast<const T*>(a.x.logits) + (int64_t)r * a.x.ld;
  if (j < a.m) ids[j] = a.ids[(int64_t)r * a.m + j];
  __syncthreads();
  // The first slot of this thread's id, and whether this is it.
  const int id = j < a.m ? ids[j] : -1;
  const bool there = id >= 0 && id < a.x.V;
  int first = j;
  for (int i = j - 1; there && i >= 0; --i)
    if (ids[i] == id) first = i;
  const bool entry = there && first == j;
  // The logits outside the list: their maximum and sum.  A NaN makes the sum one.
  const auto sweep = [&](const auto& f) __attribute__((always_inline)) {
    for (int base = 0; base < a.x.V; base += kMarkWords * 32) {
      __syncthreads();
      for (int i = j; i < kMarkWords; i += kRowThreads) mark[i] = 0;
      __syncthreads();
      if (there && id >= base && id - base < kMarkWords * 32)
        atomicOr(&mark[(id - base) >> 5], 1u << ((id - base) & 31));
      __syncthreads();
      const int end = min(a.x.V - base, kMarkWords * 32);
      for (int i = j; i < end; i += kRowThreads)
        if (!(mark[i >> 5] >> (i & 31) & 1)) f(load1(row, base + i));
    }
  };
  float rest_top = -INFINITY;
  sweep([&](float l) { rest_top = fmaxf(rest_top, l); });
  rest_top = block_all(rest_top, red, MaxOp{});
  if (rest_top == -INFINITY) rest_top = 0.f;  // none: every term is 0
  float s = 0.f;
  sweep([&](float l) { s += exp2f(scaled<true>(a.x, l, rest_top)); });
  const double rest = block_all(s, red, SumOp{});
  // The list, in 64 bits: the loss is a small difference of its terms.
  const double l = there ? (double)load1(row, id) : -INFINITY, tau = a.x.tau;
  double top = block_all(entry ? l : -INFINITY, redd, MaxOp{});
  if (rest != 0. && rest_top > top) top = rest_top;
  const double e = entry ? exp((l - top) / tau) : 0.;
  const double tail_scale = rest != 0. ? exp((rest_top - top) / tau) : 0.;
  const double total = block_all(e, redd, SumOp{}) + rest * tail_scale;
  const double log_total = total > 0. ? log(total) : (double)nan_f();
  const double val = entry ? (double)a.values[(int64_t)r * a.m + j] : -INFINITY;
  double lp = val, pt = 0., sum;
  if (!a.tail) {
    const double vmax = block_all(val, redd, MaxOp{});
    sum = block_all(entry ? exp((val - vmax) / tau) : 0., redd, SumOp{});
    lp = entry ? (val - vmax) / tau - log(sum) : val;
  } else {
    sum = block_all(entry ? exp(lp) : 0., redd, SumOp{});
    pt = sum > 1. ? 0. : 1. - sum;
  }
  // A value that is a NaN or +infinity: no term of the row is a number.
  lp += sum - sum;
  pt += sum - sum;
  const double p = exp(lp), lq = (l - top) / tau - log_total;
  const bool none = block_all(entry ? 1.f : 0.f, red, MaxOp{}) == 0.f;
  double loss = block_all(entry && !(p == 0.) ? p * (lp - lq) : 0., redd, SumOp{});
  const double qt = rest * tail_scale / total;
  if (a.tail && !(pt == 0.) && !(rest == 0.))
    loss += pt * (log(pt) - (log(rest) + (rest_top - top) / tau - log_total));
  if (j == 0) a.loss[r] = none ? 0.f : (float)(tau * tau * loss);
  if (a.state == nullptr) return;
  float* st = a.state + (int64_t)r * (a.m + kState);
  if (j == 0) {
    st[0] = rest_top;
    st[1] = rest == 0. ? (total > 0. ? 0.f : nan_f()) : (float)(tau * (qt - pt) / rest);
    st[2] = none ? 1.f : 0.f;
    st[3] = 0.f;
  }
  // Each entry's own gradient; a repeated id has its first slot's.
  __shared__ float own[kTopMax];
  if (entry) own[j] = (float)(tau * (exp(lq) - p));
  __syncthreads();
  if (j < a.m) st[kState + j] = there ? own[first] : 0.f;
}

// One block per row and kGradChunk logits: what the logits outside the list get, then
// the list's entries of the chunk over it.
template <typename T>
__global__ __launch_bounds__(kGradThreads) void distill_grad_kernel(VocabRows x, int m,
                                                                    const int32_t* ids,
                                                                    const float* state, RowGrad g,
                                                                    int chunks) {
  const int r = blockIdx.x / chunks, i0 = blockIdx.x % chunks * kGradChunk;
  const T* row = static_cast<const T*>(x.logits) + (int64_t)r * x.ld;
  T* out = static_cast<T*>(g.dlogits) + (int64_t)r * g.ldd;
  const float* st = state + (int64_t)r * (m + kState);
  const float gr = g.g[r], top = st[0], k = st[1] * gr;
  const int end = min(x.V, i0 + kGradChunk);
  if (gr == 0.f || st[2] != 0.f) {
    for (int i = i0 + threadIdx.x; i < end; i += kGradThreads) store1(out, i, 0.f);
    return;
  }
  for (int i = i0 + threadIdx.x; i < end; i += kGradThreads)
    store1(out, i, exp2f(scaled<true>(x, load1(row, i), top)) * k);
  __threadfence_block();
  __syncthreads();
  for (int j = threadIdx.x; j < m; j += kGradThreads) {
    const int id = ids[(int64_t)r * m + j];
    if (id >= i0 && id < end) store1(out, id, st[kState + j] * gr);
  }
}

}  // namespace

hipError_t launch_scores(const ScoresArgs& a, hipStream_t s) {
  if (a.x.bf16)
    hipLaunchKernelGGL(scores_kernel<uint16_t>, dim3(a.x.rows), dim3(kRowThreads), 0, s, a);
  else
    hipLaunchKernelGGL(scores_kernel<float>, dim3(a.x.rows), dim3(kRowThreads), 0, s, a);
  return note_hip(hipGetLastError());
}

hipError_t launch_scores_grad(const VocabRows& x, const int32_t* tokens, const float* stats,
                              const RowGrad& g, hipStream_t s) {
  const int chunks = (x.V + kGradChunk - 1) / kGradChunk;
  const dim3 grid((unsigned)x.rows * chunks);
  if (x.bf16)
    hipLaunchKernelGGL(scores_grad_kernel<uint16_t>, grid, dim3(kGradThreads), 0, s, x, tokens,
                       stats, g, chunks);
  else
    hipLaunchKernelGGL(scores_grad_kernel<float>, grid, dim3(kGradThreads), 0, s, x, tokens, stats,
                       g, chunks);
  return note_hip(hipGetLastError());
}

hipError_t launch_distill(const DistillArgs& a, hipStream_t s) {
  if (a.x.bf16)
    hipLaunchKernelGGL(distill_kernel<uint16_t>, dim3(a.x.rows), dim3(kRowThreads), 0, s, a);
  else
    hipLaunchKernelGGL(distill_kernel<float>, dim3(a.x.rows), dim3(kRowThreads), 0, s, a);
  return note_hip(hipGetLastError());
}

hipError_t launch_distill_grad(const VocabRows& x, int m, const int32_t* ids, const float* state,
                               const RowGrad& g, hipStream_t s) {
  const int chunks = (x.V + kGradChunk - 1) / kGradChunk;
  const dim3 grid((unsigned)x.rows * chunks);
  if (x.bf16)
    hipLaunchKernelGGL(distill_grad_kernel<uint16_t>, grid, dim3(kGradThreads), 0, s, x, m, ids,
                       state, g, chunks);
  else
    hipLaunchKernelGGL(distill_grad_kernel<float>, grid, dim3(kGradThreads), 0, s, x, m, ids,
                       state, g, chunks);
  return note_hip(hipGetLastError());
}

}  // namespace de
