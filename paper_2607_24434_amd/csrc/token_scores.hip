// Token scores, forward and backward.
//
// With M = max l and S = sum_v exp((l_v - M) / tau):
//   log p_v = (l_v - M) / tau - log S,     H = log S - (sum_v e_v d_v) / S
// (e_v the summand, d_v = (l_v - M) / tau), and for the gradient
//   d (g log p_t + h H) / d l_v = (g (1[v = t] - p_v) - h p_v (log p_v + H)) / tau.
// Differences to the maximum are taken before they are scaled, so that logits far from zero
// lose nothing.  Memory bounds the long rows (2048 fp32 rows of 102400: parts 136 us, 6.2 TB/s;
// bf16 with the gradient from the same registers 159 us, 5.3 TB/s), the vector ALU bf16 parts (19
// instruction slots a logit), a chain of dependent steps the alternatives (7 us a row, 22
// for 2048).
#include "scores_core.h"

namespace de {
namespace {

// ---------------------------------------------------------------- the best m

constexpr int kGroupCap = 1024;         // groups looked at again
constexpr int kListCap = 4 * kThreads;  // logits: at least m and one of each thread (16 KB of both: 8 blocks a CU)
constexpr int kSlack = 16;              // how many more than m a threshold may let through
constexpr int kBatch = 8;               // slots a thread loads at once

struct TopShared {
  uint64_t groups[kGroupCap];
  alignas(16) uint64_t list[kListCap];
  uint64_t bound;
  int ngroups, n, through;
  int red[2][kThreads / 64];
};

// The m best of list[0, n), n > m: moved to its front in no order, n set to m; returns the
// least of them.  Keys differ, so that some bound lets exactly m through.
template <int CAP>
__device__ __attribute__((noinline)) uint64_t prune(uint64_t* list, int& n_shared, int m, TopShared& sh) {
  constexpr int Q = CAP / kThreads;
  __syncthreads();
  const int n = n_shared;
  uint64_t v[Q], hi = 0, lo = ~0ull;
#pragma unroll
  for (int i = 0; i < Q; ++i) {
    const int j = i * kThreads + threadIdx.x;
    v[i] = j < n ? list[j] : 0;
  }
  // 64 bits from the top: the largest bound with m or more at or over it.
  lo = 0;
  int it = 0;
  for (int b = 63; b >= 0; --b) {
    hi = lo | 1ull << b;
    int c = 0;
#pragma unroll
    for (int i = 0; i < Q; ++i) c += __popcll(__ballot(v[i] >= hi));
    if ((threadIdx.x & 63) == 0) sh.red[it & 1][threadIdx.x >> 6] = c;
    __syncthreads();
    c = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) c += sh.red[it & 1][w];
    ++it;
    if (c >= m) lo = hi;
    if (c == m) break;
  }
  __syncthreads();
  if (threadIdx.x == 0) n_shared = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < Q; ++i)
    if (v[i] >= lo && v[i] != 0) list[atomicAdd(&n_shared, 1)] = v[i];
  __syncthreads();
  return lo;
}

// The best m of a row in descending order, ties to the lower index, from its groups' maxima
// gm[0, G) (a block of kThreads threads).  `side` is run by the second wave's first thread while
// the first wave is busy alone.
//   1. Each thread's best group; a bound that m to m + kSlack of the threads reach, by
//      bisection in one wave.  At least m groups are at or over it.
//   2. Those groups' logits at or over the bound's value go to a list; both lists are
//      pruned to their best m whenever they could overflow (rows of many equal or sorted
//      logits).
//   3. Each logit's rank in the list is its place.
template <typename T, typename F>
__device__ void top_select(const Row& w, const uint32_t* gm, int G, int glog, int m, float tau, float top,
                           float log_s, int32_t* idx, float* logp, TopShared& sh, const F& side) {
  const int tid = threadIdx.x;
  // The first kBatch groups of a thread stay in registers.
  uint32_t v0[kBatch];
  each<kBatch>([&](auto i) __attribute__((always_inline)) {
    const int g = i * kThreads + tid;
    v0[i] = g < G ? gm[g] : 0;
  });
  const auto group_key = [&](uint32_t v, int g) { return g < G ? (uint64_t)v << 32 | (0xffffffffu - (uint32_t)g) : 0; };
  uint64_t best = 0;
  each<kBatch>([&](auto i) __attribute__((always_inline)) {
    const uint64_t k = group_key(v0[i], i * kThreads + tid);
    best = k > best ? k : best;
  });
  for (int g = kBatch * kThreads + tid; g < G; g += kThreads) {
    const uint64_t k = group_key(gm[g], g);
    best = k > best ? k : best;
  }
  sh.list[tid] = best;
  if (tid == 0) sh.ngroups = sh.n = 0;
  __syncthreads();
  if (tid < kWave) {
    constexpr int Q = kThreads / kWave;
    uint64_t v[Q];
    uint32_t h[Q], all = 0, any = ~0u;
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      v[i] = sh.list[i * kWave + tid];
      h[i] = (uint32_t)(v[i] >> 32);
      all |= h[i];
      any &= h[i];
    }
    // The bits in which the values differ at all.
    for (int o = 32; o > 0; o >>= 1) {
      all |= __shfl_xor(all, o, kWave);
      any &= __shfl_xor(any, o, kWave);
    }
    const auto count = [&](auto ge) __attribute__((always_inline)) {
      int c = 0;
#pragma unroll
      for (int i = 0; i < Q; ++i) c += __popcll(__ballot(ge(i)));
      return c;
    };
    uint32_t lo = any, differ = __builtin_amdgcn_readfirstlane(all ^ any);
    lo = __builtin_amdgcn_readfirstlane(lo);
    int c = count([&](int i) { return v[i] != 0; });
    uint64_t bound = 1;
    if (c > m + kSlack) {
      // The largest value with m or more at or over it, or the first with few enough.
      c = kThreads;
      while (differ != 0 && c > m + kSlack) {
        const uint32_t bit = 0x80000000u >> __builtin_clz(differ), mid = lo | bit;
        differ &= bit - 1;
        const int k = count([&](int i) { return h[i] >= mid; });
        if (k < m) continue;
        lo = mid;
        c = k;
      }
      bound = (uint64_t)lo << 32;
      // Equal values: the lower indices.
      for (uint32_t bit = 0x80000000u; bit != 0 && c > m + kSlack; bit >>= 1) {
        const uint64_t mid = bound | bit;
        const int k = count([&](int i) { return v[i] >= mid; });
        if (k < m) continue;
        bound = mid;
        c = k;
      }
    }
    if (tid == 0) {
      sh.bound = bound;
      sh.through = c;
    }
  }
  if (tid == kWave) side();
  __syncthreads();
  uint64_t bound = sh.bound;
  const int rounds = (G + kThreads - 1) / kThreads;
  if (rounds <= kBatch && sh.through * rounds <= kGroupCap) {
    each<kBatch>([&](auto i) __attribute__((always_inline)) {
      const uint64_t k = group_key(v0[i], i * kThreads + tid);
      if (k >= bound) sh.groups[atomicAdd(&sh.ngroups, 1)] = k;
    });
  } else {
    for (int i = 0; i < rounds; ++i) {
      __syncthreads();
      const bool full = sh.ngroups + kThreads > kGroupCap;
      __syncthreads();  // every thread has read it before one appends
      if (full) bound = prune<kGroupCap>(sh.groups, sh.ngroups, m, sh);
      const int g = i * kThreads + tid;
      const uint64_t k = g < G ? group_key(gm[g], g) : 0;
      if (k >= bound) sh.groups[atomicAdd(&sh.ngroups, 1)] = k;
    }
  }
  __syncthreads();
  const int work = sh.ngroups << glog;
  // A logit of the bound's value may beat the bound's group: only its value counts.
  bound = bound >> 32 << 32;
  const auto first_of = [&](int j) {  // the row's element that slot j of the work starts at
    return ((key_index(sh.groups[j >> glog]) << glog) + (j & ((1 << glog) - 1))) * kE<T> - w.o;
  };
  for (int j0 = 0; j0 < work; j0 += kBatch * kThreads) {
    const int n0 = sh.n;
    __syncthreads();  // every thread has read it before one appends
    u32x4 x[kBatch];
    int first[kBatch];
    each<kBatch>([&](auto b) __attribute__((always_inline)) {
      const int j = j0 + b * kThreads + tid;
      x[b] = all_dropped<T>();
      first[b] = w.V;
      if (j < work) {
        first[b] = first_of(j);
        if (first[b] < w.V) x[b] = load_edge<T>(w, (first[b] + w.o) / kE<T>);
      }
    });
    each<kBatch>([&](auto b) __attribute__((always_inline)) {
      if (j0 + b * kThreads >= work) return;
      float most = -INFINITY;
      each<kE<T>>([&](auto c) __attribute__((always_inline)) {
        most = fmaxf(most, __builtin_canonicalizef(get<T>(x[b], c)));
      });
      if ((uint64_t)order_key(most) << 32 < (bound >> 32 << 32)) return;
#pragma unroll 1
      for (int c = 0; c < kE<T>; ++c) {
        const float v = get_at<T>(x[b], c);
        const int i = first[b] + c;
        const uint64_t k = order_key(v, i);
        if (i < 0 || i >= w.V || k < bound) continue;
        const int at = atomicAdd(&sh.n, 1);
        if (at < kListCap) sh.list[at] = k;
      }
    });
    __syncthreads();
    if (sh.n <= kListCap) continue;
    // No room: what these slots added goes, and they are taken again, one logit of each at
    // a time.
    __syncthreads();
    if (tid == 0) sh.n = n0;
#pragma unroll 1
    for (int b = 0; b < kBatch; ++b)
#pragma unroll 1
      for (int c = 0; c < kE<T>; ++c) {
        __syncthreads();
        const bool full = sh.n + kThreads > kListCap;
        __syncthreads();
        if (full) bound = prune<kListCap>(sh.list, sh.n, m, sh);
        const int j = j0 + b * kThreads + tid, i = j < work ? first_of(j) + c : -1;
        if (i < 0 || i >= w.V) continue;
        const uint64_t k = order_key(load1(elem_at<T>(w, i)), i);
        if (k >= bound) sh.list[atomicAdd(&sh.n, 1)] = k;
      }
    __syncthreads();
  }
  if (sh.n > kThreads) prune<kListCap>(sh.list, sh.n, m, sh);
  const int n = sh.n;
  if (tid >= n) return;
  const uint64_t mine = sh.list[tid];
  int rank = 0;
#pragma unroll 4
  for (int i = 0; i + 1 < n; i += 2) {
    const ulonglong2 k = *reinterpret_cast<const ulonglong2*>(&sh.list[i]);
    rank += (k.x > mine) + (k.y > mine);
  }
  if (n & 1) rank += sh.list[n - 1] > mine;
  if (rank >= m) return;
  idx[rank] = key_index(mine);
  logp[rank] = log_p(tau, key_value(mine), top, log_s);
}

// ---------------------------------------------------------------- token scores

struct RowScore {
  float top, s, h, log_s;
};

__device__ __forceinline__ RowScore row_score(const VocabRows& x, const Part& p) {
  RowScore r;
  r.top = p.top;
  // No distribution: nothing above -infinity, or an infinite logit.
  r.s = fabsf(p.top) < INFINITY ? fmaf(x.corr, p.w, p.s) : nan_f();
  r.log_s = logf(r.s);
  r.h = r.log_s - p.w / r.s * kLn2;
  return r;
}

// The logit of a row's token (one thread); it may be overwritten once the block's gradients are.
template <typename T>
__device__ __forceinline__ float token_logit(const ScoresArgs& a, const Row& w, int r) {
  const int t = a.logp != nullptr ? a.tokens[r] : -1;
  return t >= 0 && t < w.V ? load1(elem_at<T>(w, t)) : 0.f;
}

// One thread: everything of a row but its alternatives and gradient.
__device__ __forceinline__ void write_scores(const ScoresArgs& a, int r, const RowScore& q, float l) {
  if (a.logp != nullptr) {
    const int t = a.tokens[r];
    a.logp[r] = t < 0 ? 0.f : t >= a.x.V ? nan_f() : log_p(a.x.tau, l, q.top, q.log_s);
  }
  if (a.entropy != nullptr) a.entropy[r] = q.h;
  if (a.stats != nullptr) {
    float* st = a.stats + (int64_t)r * kStats;
    st[0] = q.top;
    st[1] = q.s;
    st[2] = q.h;
    st[3] = q.top / a.x.tau + q.log_s;
  }
}

// Parts of rows, one block each: grid rows * chunks.
template <typename T, int U>
__global__ __launch_bounds__(kThreads, 6) void scores_part_kernel(ScoresArgs a, Split sp) {
  __shared__ float red[3][kThreads / 64];
  const int r = blockIdx.x / sp.chunks, slot0 = blockIdx.x % sp.chunks * sp.nu * kThreads;
  const Row w = until(row_at<T>(a.x.logits, a.x.ld, r, a.x.V), slot0 + sp.nu * kThreads);
  Tile<kThreads, U> x;
  load_tile<T>(x, w, slot0);
  uint32_t* gm = sp.gm + (int64_t)r * sp.gstride;
  const Part mine = tile_sums<T, false>(a.x, x, w, NoFix{}, [&](float v, int u) __attribute__((always_inline)) {
    if (a.m > 0) group_max(v, x.slot(u), w, sp.glog, gm);
  });
  const Part p = block_part<kThreads>(a.x, mine, red);
  if (threadIdx.x == 0) sp.parts[blockIdx.x] = make_float4(p.top, p.s, p.w, 0.f);
}

// A row's parts as one (a block of kThreads threads).
__device__ __forceinline__ Part merge_parts(const VocabRows& x, const float4* parts, int n, float (*red)[kThreads / 64]) {
  Part p{-INFINITY, 0.f, 0.f};
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const float4 q = parts[i];
    const float top = fmaxf(p.top, q.x);
    const Part b = rebased(x, Part{q.x, q.y, q.z}, top);
    p = rebased(x, p, top);
    p.s += b.s;
    p.w += b.w;
  }
  return block_part<kThreads>(x, p, red);
}

template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void scores_finish_kernel(ScoresArgs a, Split sp) {
  __shared__ float red[3][kThreads / 64];
  const int r = blockIdx.x;
  const Row w = row_at<T>(a.x.logits, a.x.ld, r, a.x.V);
  const float token = threadIdx.x == kWave ? token_logit<T>(a, w, r) : 0.f;
  const RowScore q = row_score(a.x, merge_parts(a.x, sp.parts + (int64_t)r * sp.chunks, sp.chunks, red));
  const auto rest = [&] { write_scores(a, r, q, token); };
  if constexpr (!TOP) {
    if (threadIdx.x == kWave) rest();
  } else {
    __shared__ TopShared sh;
    top_select<T>(w, sp.gm + (int64_t)r * sp.gstride, (w.slots + (1 << sp.glog) - 1) >> sp.glog, sp.glog, a.m,
                  a.x.tau, q.top, q.log_s, a.top_idx + (int64_t)r * a.m, a.top_logp + (int64_t)r * a.m, sh, rest);
  }
}

// Rows of one tile with alternatives, one block each.
template <typename T, int U>
__global__ __launch_bounds__(kThreads, 4) void scores_row_kernel(ScoresArgs a, int glog) {
  __shared__ float red[3][kThreads / 64];
  __shared__ uint32_t gm[U * kThreads];
  __shared__ TopShared sh;
  const int r = blockIdx.x;
  const Row w = row_at<T>(a.x.logits, a.x.ld, r, a.x.V);
  Tile<kThreads, U> x;
  load_tile<T>(x, w, 0);
  const float token = threadIdx.x == kWave ? token_logit<T>(a, w, r) : 0.f;
  const Part mine = tile_sums<T, false>(a.x, x, w, NoFix{}, [&](float v, int u) __attribute__((always_inline)) {
    group_max(v, x.slot(u), w, glog, gm);
  });
  const Part p = block_part<kThreads>(a.x, mine, red);
  const RowScore q = row_score(a.x, p);
  top_select<T>(w, gm, (w.slots + (1 << glog) - 1) >> glog, glog, a.m, a.x.tau, q.top, q.log_s,
                a.top_idx + (int64_t)r * a.m, a.top_logp + (int64_t)r * a.m, sh, [&] { write_scores(a, r, q, token); });
}

// What a logit's gradient is made of.
struct ScoreGrad {
  bool zero;          // a row without weight
  int token;
  float gl, ge;       // incoming gradients / tau
  float top, inv, b;  // p = inv 2^d, log p + H = d ln 2 + b
  float k;            // -gl inv
};

__device__ __forceinline__ ScoreGrad score_grad(const VocabRows& x, const int32_t* tokens, const RowGrad& g, int r,
                                                float top, float s, float h) {
  ScoreGrad q;
  q.token = tokens != nullptr ? tokens[r] : -1;
  q.gl = g.g != nullptr && q.token >= 0 ? g.g[r] : 0.f;
  q.ge = g.g_entropy != nullptr ? g.g_entropy[r] : 0.f;
  q.zero = q.gl == 0.f && q.ge == 0.f;
  if (q.token >= x.V && q.gl != 0.f) q.gl = nan_f();
  const float it = 1.f / x.tau;
  q.gl *= it;
  q.ge *= it;
  q.top = top;
  q.inv = 1.f / s;
  q.b = h - logf(s);
  q.k = -q.gl * q.inv;
  return q;
}

// A tile's gradients.  `entropy`: with its part.
template <typename T, bool entropy, int NTH, int U>
__device__ __forceinline__ void scores_grad_tile(const VocabRows& a, const ScoreGrad& q, Tile<NTH, U>& x, const Row& w,
                                                 const Row& out) {
  each_slot(x, [&](const u32x4& l, int u) __attribute__((always_inline)) {
    const int s = x.slot(u);
    if (s >= w.slots) return;
    float v[kE<T>];
    each<kE<T>>([&](auto c) __attribute__((always_inline)) {
      const float d = scaled_floor(a, get<T>(l, c), q.top), e = exp2_fast(d);
      if constexpr (entropy) v[c] = -e * q.inv * fmaf(q.ge, fmaf(d, kLn2, q.b), q.gl);
      else v[c] = e * q.k;
    });
    const int t = q.token + w.o - s * kE<T>;  // the token's place in the slot
    if (t >= 0 && t < kE<T>)
      each<kE<T>>([&](auto c) __attribute__((always_inline)) { v[c] += t == c ? q.gl : 0.f; });
    store_slot<T>(w, out, s, v);
  });
}

template <typename T, int U>
__global__ __launch_bounds__(kThreads) void scores_grad_kernel(VocabRows x, const int32_t* tokens, const float* stats,
                                                               RowGrad g, Split sp) {
  const int r = blockIdx.x / sp.chunks, slot0 = blockIdx.x % sp.chunks * sp.nu * kThreads;
  const Row w = until(row_at<T>(x.logits, x.ld, r, x.V), slot0 + sp.nu * kThreads), out = row_at<T>(g.dlogits, g.ldd, r, x.V);
  const float* st = stats + (int64_t)r * kStats;
  const ScoreGrad q = score_grad(x, tokens, g, r, st[0], st[1], st[2]);
  if (q.zero) return zero_tile<T, kThreads>(w, out, slot0);
  Tile<kThreads, U> l;
  static_assert(U <= kAhead * kRun, "every slot is loaded at once");
  load_tile<T>(l, w, slot0);
  load_first<T>(l, w);
  load_last<T>(l, w);
  if (q.ge == 0.f) scores_grad_tile<T, false>(x, q, l, w, out);
  else scores_grad_tile<T, true>(x, q, l, w, out);
}

// Whole rows without alternatives, one block each, and their gradient where one is asked for.
template <typename T, int NTH, int U>
__global__ __launch_bounds__(NTH, whole_waves(NTH, U)) void scores_whole_kernel(ScoresArgs a, RowGrad g) {
  __shared__ float red[3][NTH / 64];
  __shared__ float token;
  const int r = blockIdx.x;
  const Row w = row_at<T>(a.x.logits, a.x.ld, r, a.x.V);
  Tile<NTH, U> x;
  load_tile<T>(x, w, 0);
  if (threadIdx.x == 0) token = token_logit<T>(a, w, r);
  const Part p = block_part<NTH>(a.x, tile_sums<T, false>(a.x, x, w, NoFix{}, NoPeak{}), red);
  const RowScore q = row_score(a.x, p);
  if (threadIdx.x == 0) write_scores(a, r, q, token);
  if (g.dlogits == nullptr) return;
  const Row out = row_at<T>(g.dlogits, g.ldd, r, a.x.V);
  const ScoreGrad d = score_grad(a.x, a.tokens, g, r, q.top, q.s, q.h);
  if (d.zero) return zero_tile<T, NTH>(w, out, 0);
  if (d.ge == 0.f) scores_grad_tile<T, false>(a.x, d, x, w, out);
  else scores_grad_tile<T, true>(a.x, d, x, w, out);
}

template <typename T>
hipError_t scores_grad(const VocabRows& x, const int32_t* tokens, const float* stats, const RowGrad& g,
                       hipStream_t s) {
  const Split sp = split_of<T>(x, 0, nullptr);
  by_u(sp.nu, [&](auto u) {
    hipLaunchKernelGGL((scores_grad_kernel<T, u.value>), dim3((unsigned)x.rows * sp.chunks), dim3(kThreads), 0, s, x,
                       tokens, stats, g, sp);
  });
  return note_hip(hipGetLastError());
}

template <typename T>
hipError_t scores(const ScoresArgs& a, const RowGrad& g, void* ws, hipStream_t s) {
  const int slots = slots_most<T>(a.x);
  const dim3 rows(a.x.rows);
  if (a.m > 0 && slots <= kTileU * kThreads) {
    by_u((slots + kThreads - 1) / kThreads, [&](auto u) {
      hipLaunchKernelGGL((scores_row_kernel<T, u.value>), rows, dim3(kThreads), 0, s, a, group_log(slots));
    });
    return note_hip(hipGetLastError());
  }
  if (a.m == 0 && whole_pays<T>(a.x, g.dlogits != nullptr) && by_whole<T, 25>(a.x, [&](auto k) {
        hipLaunchKernelGGL((scores_whole_kernel<T, k.kNth, k.kU>), rows, dim3(k.kNth), 0, s, a, g);
      }))
    return note_hip(hipGetLastError());
  const Split sp = split_of<T>(a.x, a.m, ws);
  by_u(sp.nu, [&](auto u) {
    hipLaunchKernelGGL((scores_part_kernel<T, u.value>), dim3((unsigned)a.x.rows * sp.chunks), dim3(kThreads), 0, s,
                       a, sp);
  });
  if (a.m > 0)
    hipLaunchKernelGGL((scores_finish_kernel<T, true>), rows, dim3(kThreads), 0, s, a, sp);
  else
    hipLaunchKernelGGL((scores_finish_kernel<T, false>), rows, dim3(kThreads), 0, s, a, sp);
  const hipError_t e = note_hip(hipGetLastError());
  return e != hipSuccess || g.dlogits == nullptr ? e : scores_grad<T>(a.x, a.tokens, a.stats, g, s);
}

}  // namespace

size_t scores_bytes(int rows, int V, int m) {
  size_t most = 0;
  // Either type, rows at any element or at whole slots; never fewer bytes for more rows.
  const auto add = [&](int slots) {
    const size_t slabs = (slots + kThreads - 1) / kThreads, coarse = (slabs + kTileU - 1) / kTileU;
    size_t b = std::max(rows * coarse, std::min<size_t>(rows * slabs, kBlocks + rows)) * sizeof(float4);
    if (m > 0) b += (size_t)rows * ((slots >> group_log(slots)) + 1) * 4;
    most = std::max(most, b);
  };
  add((V + kE<float> - 1) / kE<float>);
  add((V + kE<uint16_t> - 1) / kE<uint16_t>);
  add(slots_most<float>(V));
  add(slots_most<uint16_t>(V));
  return most;
}

hipError_t launch_scores(const ScoresArgs& a, const RowGrad& g, void* ws, hipStream_t s) {
  return a.x.bf16 ? scores<uint16_t>(a, g, ws, s) : scores<float>(a, g, ws, s);
}
hipError_t launch_scores_grad(const VocabRows& x, const int32_t* tokens, const float* stats, const RowGrad& g,
                              hipStream_t s) {
  return x.bf16 ? scores_grad<uint16_t>(x, tokens, stats, g, s) : scores_grad<float>(x, tokens, stats, g, s);
}

}  // namespace de
