// Token scores and distillation from a teacher's top logits, forward and backward.
//
// With z = l / tau, M = max l and S = sum_v exp((l_v - M) / tau):
//   log p_v = (l_v - M) / tau - log S,     H = log S - (sum_v e_v d_v) / S
// (e_v the summand, d_v = (l_v - M) / tau).  Differences to the maximum are taken before
// they are scaled, so that logits far from zero lose nothing.
//
// A row is read in tiles: each thread of a block has up to U 16-byte slots of it in
// registers, all of their loads in flight together, and takes the maximum, the sums and
// (gradients) the results from there, so that logits are read once.  Slots lie at
// multiples of 16 bytes whatever element the row starts at; its first and last one may be
// partly outside it and are then loaded by the element.
#include "de_common.h"
#include "scores.h"

#include <algorithm>

namespace de {
namespace {

constexpr int kThreads = 256;
constexpr int kTileU = 8;  // slots a thread of a part of a row
constexpr float kLn2 = 0.6931471805599453f;

// Rows in parts: what each part leaves for the row's last step, in the caller's scratch.
struct Split {
  int chunks;      // parts of a row
  float4* parts;   // [rows, chunks]: maximum, sum e, sum e d
  float* gm;       // [rows, gstride]: groups' maxima
  int gstride, glog;
};

__device__ __forceinline__ float nan_f() { return __int_as_float(0x7fc00000); }

template <typename T>
constexpr int kE = 16 / (int)sizeof(T);  // logits of a slot

__device__ __forceinline__ float load1(const float* p) { return *gptr<float>(p); }
__device__ __forceinline__ float load1(const uint16_t* p) {
  return __uint_as_float((uint32_t)*gptr<uint16_t>(p) << 16);
}
__device__ __forceinline__ uint32_t bf16_bits(float v) {
  return __builtin_bit_cast(uint16_t, (__bf16)v);  // to nearest, ties to even; a NaN stays one
}
__device__ __forceinline__ void store1(float* p, float v) { *(DE_GLOBAL float*)p = v; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *(DE_GLOBAL uint16_t*)p = (uint16_t)bf16_bits(v); }

// Logit c of a slot.
template <typename T>
__device__ __forceinline__ float get(const u32x4& x, int c) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(x[c]);
  else return c & 1 ? bf16_hi(x[c >> 1]) : bf16_lo(x[c >> 1]);
}
// -infinity in its place.
template <typename T>
__device__ __forceinline__ void drop(u32x4& x, int c) {
  if constexpr (sizeof(T) == 4) x[c] = 0xff800000u;
  else x[c >> 1] = c & 1 ? (x[c >> 1] & 0xffffu) | 0xff800000u : (x[c >> 1] & 0xffff0000u) | 0xff80u;
}
template <typename T>
__device__ __forceinline__ u32x4 all_dropped() {
  const uint32_t v = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  return u32x4{v, v, v, v};
}
template <typename T>
__device__ __forceinline__ u32x4 packed(const float (&v)[kE<T>]) {
  u32x4 x;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if constexpr (sizeof(T) == 4) x[c] = __float_as_uint(v[c]);
    else x[c] = bf16_bits(v[2 * c]) | bf16_bits(v[2 * c + 1]) << 16;
  }
  return x;
}

// A row's slots: element i of the row is logit (i + o) % E of slot (i + o) / E.
struct Row {
  const char* base;  // slot 0
  int V, o;
  int f0, f1;        // slots wholly inside: [f0, f1)
  int slots;
};

template <typename T>
__device__ __forceinline__ Row row_at(const void* p, int64_t ld, int r, int V) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p) + (uintptr_t)((int64_t)r * ld) * sizeof(T);
  Row w;
  w.base = reinterpret_cast<const char*>(a & ~(uintptr_t)15);
  w.V = V;
  w.o = (int)(a & 15) / (int)sizeof(T);
  w.f0 = w.o > 0;
  w.f1 = (V + w.o) / kE<T>;
  w.slots = (V + w.o + kE<T> - 1) / kE<T>;
  return w;
}

template <typename T>
__device__ __forceinline__ const T* elem_at(const Row& w, int i) {
  return reinterpret_cast<const T*>(w.base) + w.o + i;
}

// One slot, any of whose elements may be outside the row (-infinity there).
template <typename T>
__device__ __forceinline__ u32x4 load_edge(const Row& w, int s) {
  if (s >= w.f0 && s < w.f1) return load_stream16(w.base + (int64_t)s * 16);
  u32x4 x = all_dropped<T>();
#pragma unroll
  for (int c = 0; c < kE<T>; ++c) {
    const int i = s * kE<T> + c - w.o;
    if (i >= 0 && i < w.V) {
      if constexpr (sizeof(T) == 4) {
        x[c] = __float_as_uint(load1(elem_at<T>(w, i)));
      } else {
        const uint32_t b = *gptr<uint16_t>(elem_at<T>(w, i));
        x[c >> 1] = c & 1 ? (x[c >> 1] & 0xffffu) | b << 16 : (x[c >> 1] & 0xffff0000u) | b;
      }
    }
  }
  return x;
}

// Slots slot0 + u * NTH + thread.  The whole ones first, so that an edge's wait holds
// none of them up.
template <typename T, int NTH, int U>
__device__ __forceinline__ void load_tile(u32x4 (&x)[U], const Row& w, int slot0) {
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int s0 = slot0 + u * NTH;
    if (s0 >= w.f0 && s0 + NTH <= w.f1)
      x[u] = load_stream16(w.base + (int64_t)s0 * 16 + threadIdx.x * 16);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int s0 = slot0 + u * NTH;
    if (s0 >= w.f0 && s0 + NTH <= w.f1) continue;
    x[u] = all_dropped<T>();
    if (s0 < w.slots) x[u] = load_edge<T>(w, s0 + threadIdx.x);
  }
}

// Writes a slot of results to the row `out`, whose slots are those of w (same offset) or not.
template <typename T>
__device__ __forceinline__ void store_slot(const Row& w, const Row& out, int s, const float (&v)[kE<T>]) {
  if (out.o == w.o && s >= w.f0 && s < w.f1) {
    *(DE_GLOBAL u32x4*)(out.base + (int64_t)s * 16) = packed<T>(v);
    return;
  }
#pragma unroll
  for (int c = 0; c < kE<T>; ++c) {
    const int i = s * kE<T> + c - w.o;
    if (i >= 0 && i < w.V) store1(const_cast<T*>(elem_at<T>(out, i)), v[c]);
  }
}

// log2 of exp(d / tau) for a difference d to the maximum.  c_lo is positive, so that a
// difference of -infinity gives -infinity.
__device__ __forceinline__ float scaled(const VocabRows& x, float d) {
  return fmaf(d, x.c_lo, d * x.c_hi);
}
__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

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
__device__ __forceinline__ int key_index(uint64_t k) { return (int)(0xffffffffu - (uint32_t)k); }

// ---------------------------------------------------------------- reductions

template <int ctrl, int rows>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), ctrl, rows, 0xF, false));
}
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, dpp<0xB1, 0xF>(v));     // quad_perm 1,0,3,2
  return fmaxf(v, dpp<0x4E, 0xF>(v));  // quad_perm 2,3,0,1
}
__device__ __forceinline__ float row16_max(float v) {
  v = quad_max(v);
  v = fmaxf(v, dpp<0x141, 0xF>(v));    // row_half_mirror
  return fmaxf(v, dpp<0x140, 0xF>(v)); // row_mirror
}
__device__ __forceinline__ float wave_max(float v) {
  v = row16_max(v);
  v = fmaxf(v, dpp<0x142, 0xA>(v));    // row_bcast:15
  v = fmaxf(v, dpp<0x143, 0xC>(v));    // row_bcast:31
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Over the block; every thread has the result.  `red` (a float for each wave) must not be
// in use by an earlier reduction that a thread may still read.
template <int NTH>
__device__ __forceinline__ float block_max(float v, float* red) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = red[0];
#pragma unroll
  for (int w = 1; w < NTH / 64; ++w) t = fmaxf(t, red[w]);
  return t;
}
template <int NTH>
__device__ __forceinline__ float block_sum(float v, float* red) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = red[0];
#pragma unroll
  for (int w = 1; w < NTH / 64; ++w) t += red[w];
  return t;
}

template <typename Op>
__device__ __forceinline__ double wave_all(double v, Op op) {
  for (int o = 32; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o, kWave));
  return v;
}
__device__ __forceinline__ double wave_sum64(double v) {
  return wave_all(v, [](double a, double b) { return a + b; });
}
__device__ __forceinline__ double wave_max64(double v) {
  return wave_all(v, [](double a, double b) { return a > b ? a : b; });
}

// ---------------------------------------------------------------- sums over a tile

// A part of a row: its maximum (a NaN left out) and, relative to it, sum e and sum e d (d in
// log2).  The maximum of a part without any is 0 for the differences.
struct Part {
  float top, s, w;
};

__device__ __forceinline__ float finite_top(float top) { return top == -INFINITY ? 0.f : top; }

template <typename T, int U>
__device__ __forceinline__ float tile_max(const u32x4 (&x)[U]) {
  float t = -INFINITY;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int c = 0; c < kE<T>; ++c) t = fmaxf(t, get<T>(x[u], c));
  return t;
}

// Scores: fmaxf with the floor makes a NaN, an infinity's difference to itself and -infinity
// terms of 0, whose product with their (finite) difference is 0.
template <typename T, int U>
__device__ __forceinline__ void tile_scores(const VocabRows& a, const u32x4 (&x)[U], float top, float& s,
                                            float& w) {
  s = w = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int c = 0; c < kE<T>; ++c) {
      const float d = scaled(a, fmaxf(get<T>(x[u], c) - top, a.floor)), e = exp2_fast(d);
      s += e;
      w = fmaf(e, d, w);
    }
}
// Distillation: a NaN makes the sum one.
template <typename T, int U>
__device__ __forceinline__ float tile_sum(const VocabRows& a, const u32x4 (&x)[U], float top) {
  float s = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int c = 0; c < kE<T>; ++c) s += exp2_fast(scaled(a, get<T>(x[u], c) - top));
  return s;
}

// The maxima of groups of 2^glog slots (0, 2 or 4) of a tile: the best m logits lie in the m
// groups whose (maximum, lower index) are best, so that only those are looked at again.
template <typename T, int NTH, int U>
__device__ __forceinline__ void tile_groups(const u32x4 (&x)[U], const Row& w, int slot0, int glog, float* gm) {
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int s = slot0 + u * NTH + threadIdx.x;
    if (slot0 + u * NTH >= w.slots) break;
    float v = -INFINITY;
#pragma unroll
    for (int c = 0; c < kE<T>; ++c) v = fmaxf(v, get<T>(x[u], c));
    if (glog == 4) v = row16_max(v);
    else if (glog == 2) v = quad_max(v);
    if ((s & ((1 << glog) - 1)) == 0 && s < w.slots) gm[s >> glog] = v;
  }
}

// Marks of a tile's list entries: a bit for each logit, and for each wave a bit for each of
// its slots that has one, so that the others cost a scalar test.
template <typename T, int NTH, int U>
struct Marks {
  uint32_t bits[U * NTH * kE<T> / 32];
  uint32_t slots[NTH / 64][(U + 31) / 32];
};

template <typename T, int NTH, int U>
__device__ __forceinline__ void clear_marks(Marks<T, NTH, U>& k) {
  for (int i = threadIdx.x; i < U * NTH * kE<T> / 32; i += NTH) k.bits[i] = 0;
  if (threadIdx.x < NTH / 64)
    for (int i = 0; i < (U + 31) / 32; ++i) k.slots[threadIdx.x][i] = 0;
}
template <typename T, int NTH, int U>
__device__ __forceinline__ void set_mark(Marks<T, NTH, U>& k, const Row& w, int slot0, int id) {
  if (id < 0 || id >= w.V) return;
  const int64_t e = (int64_t)id + w.o - (int64_t)slot0 * kE<T>;
  if (e < 0 || e >= (int64_t)U * NTH * kE<T>) return;
  const int i = (int)e, s = i / kE<T>, u = s / NTH, wave = s % NTH / 64;
  atomicOr(&k.bits[i >> 5], 1u << (i & 31));
  atomicOr(&k.slots[wave][u >> 5], 1u << (u & 31));
}
template <typename T, int NTH, int U>
__device__ __forceinline__ void drop_marked(u32x4 (&x)[U], const Marks<T, NTH, U>& k) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!(__builtin_amdgcn_readfirstlane(k.slots[wave][u >> 5]) >> (u & 31) & 1)) continue;
    const int i = (u * NTH + threadIdx.x) * kE<T>;
    const uint32_t b = k.bits[i >> 5] >> (i & 31);
#pragma unroll
    for (int c = 0; c < kE<T>; ++c)
      if (b >> c & 1) drop<T>(x[u], c);
  }
}

// ---------------------------------------------------------------- the best m

constexpr int kGroupCap = 1024;         // groups looked at again
constexpr int kListCap = 9 * kThreads;  // logits: at least m + one round's of a block
constexpr int kSlack = 16;              // how many more than m a threshold may let through
constexpr int kBatch = 8;               // slots a thread loads at once

struct TopShared {
  uint64_t groups[kGroupCap];
  uint64_t list[kListCap];
  uint64_t bound;
  int ngroups, n, need, through;
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
// gm[0, G) (a block of kThreads threads).
//   1. Each thread's best group; a bound that m to m + kSlack of the threads reach, by
//      bisection in one wave.  At least m groups are at or over it.
//   2. Those groups' logits at or over the bound's value go to a list; both lists are
//      pruned to their best m whenever they could overflow (rows of many equal or sorted
//      logits).
//   3. Each logit's rank in the list is its place.
template <typename T>
__device__ void top_select(const Row& w, const float* gm, int G, int glog, int m, float tau, float top,
                           float log_s, int32_t* idx, float* logp, TopShared& sh) {
  const int tid = threadIdx.x;
  uint64_t best = 0;
  for (int g = tid; g < G; g += kThreads) {
    const uint64_t k = order_key(gm[g], g);
    best = k > best ? k : best;
  }
  sh.list[tid] = best;
  if (tid == 0) sh.ngroups = sh.n = 0;
  __syncthreads();
  if (tid < kWave) {
    uint64_t v[kThreads / kWave];
#pragma unroll
    for (int i = 0; i < kThreads / kWave; ++i) v[i] = sh.list[i * kWave + tid];
    const auto count = [&](uint64_t b) {
      int c = 0;
#pragma unroll
      for (int i = 0; i < kThreads / kWave; ++i) c += __popcll(__ballot(v[i] >= b));
      return c;
    };
    uint64_t lo = 1;
    int c = count(lo);
    if (c > m + kSlack) {
      lo = 0;
      for (int b = 63; b >= 0; --b) {
        const uint64_t mid = lo | 1ull << b;
        const int k = count(mid);
        if (k < m) continue;
        lo = mid;
        c = k;
        if (k <= m + kSlack) break;
      }
    }
    if (tid == 0) {
      sh.bound = lo;
      sh.through = c;
    }
  }
  __syncthreads();
  uint64_t bound = sh.bound;
  const int rounds = (G + kThreads - 1) / kThreads;
  const bool fits = (int64_t)sh.through * rounds <= kGroupCap;
  for (int i = 0; i < rounds; ++i) {
    if (!fits) {
      __syncthreads();
      const bool full = sh.ngroups + kThreads > kGroupCap;
      __syncthreads();  // every thread has read it before one appends
      if (full) bound = prune<kGroupCap>(sh.groups, sh.ngroups, m, sh);
    }
    const int g = i * kThreads + tid;
    const uint64_t k = g < G ? order_key(gm[g], g) : 0;
    if (k >= bound) sh.groups[atomicAdd(&sh.ngroups, 1)] = k;
  }
  __syncthreads();
  const int work = sh.ngroups << glog;
  // A logit of the bound's value may beat the bound's group: only its value counts.
  bound = bound >> 32 << 32;
  for (int j0 = 0; j0 < work; j0 += kBatch * kThreads) {
    u32x4 x[kBatch];
    int first[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int j = j0 + b * kThreads + tid;
      x[b] = all_dropped<T>();
      first[b] = INT32_MIN / 2;
      if (j < work) {
        const int s = (key_index(sh.groups[j >> glog]) << glog) + (j & ((1 << glog) - 1));
        if (s < w.slots) {
          x[b] = load_edge<T>(w, s);
          first[b] = s * kE<T> - w.o;
        }
      }
    }
    // A bit for each logit at or over the bound.
    uint32_t take[kBatch];
    int mine = 0;
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      take[b] = 0;
#pragma unroll
      for (int c = 0; c < kE<T>; ++c) {
        const int i = first[b] + c;
        if (i >= 0 && i < w.V && order_key(get<T>(x[b], c), i) >= bound) take[b] |= 1u << c;
      }
      mine += __popc(take[b]);
    }
    if (tid == 0) sh.need = 0;
    __syncthreads();
    if (mine) atomicAdd(&sh.need, mine);
    __syncthreads();
    const bool room = sh.n + sh.need <= kListCap;
    __syncthreads();
    if (room) {
      int at = mine ? atomicAdd(&sh.n, mine) : 0;
#pragma unroll
      for (int b = 0; b < kBatch; ++b)
        if (take[b])
#pragma unroll
          for (int c = 0; c < kE<T>; ++c)
            if (take[b] >> c & 1) sh.list[at++] = order_key(get<T>(x[b], c), first[b] + c);
    } else {
      // One logit a thread at a time, read again.
#pragma unroll 1
      for (int b = 0; b < kBatch; ++b)
#pragma unroll 1
        for (int c = 0; c < kE<T>; ++c) {
          __syncthreads();
          const bool full = sh.n + kThreads > kListCap;
          __syncthreads();  // every thread has read it before one appends
          if (full) bound = prune<kListCap>(sh.list, sh.n, m, sh);
          const int j = j0 + b * kThreads + tid;
          if (j >= work) continue;
          const int i = ((key_index(sh.groups[j >> glog]) << glog) + (j & ((1 << glog) - 1))) * kE<T> - w.o + c;
          if (i < 0 || i >= w.V) continue;
          const uint64_t k = order_key(load1(elem_at<T>(w, i)), i);
          if (k >= bound) sh.list[atomicAdd(&sh.n, 1)] = k;
        }
    }
    __syncthreads();
  }
  if (sh.n > kThreads) prune<kListCap>(sh.list, sh.n, m, sh);
  const int n = sh.n;
  if (tid >= n) return;
  const uint64_t mine = sh.list[tid];
  int rank = 0;
  for (int i = 0; i < n; ++i) rank += sh.list[i] > mine;
  if (rank >= m) return;
  const int i = key_index(mine);
  idx[rank] = i;
  logp[rank] = log_p(tau, load1(elem_at<T>(w, i)), top, log_s);
}

// ---------------------------------------------------------------- token scores

struct RowScore {
  float top, s, h, log_s;
};

__device__ __forceinline__ RowScore row_score(const Part& p) {
  RowScore r;
  r.top = p.top;
  // No distribution: nothing above -infinity, or an infinite logit.
  r.s = fabsf(p.top) < INFINITY ? p.s : nan_f();
  r.log_s = logf(r.s);
  r.h = r.log_s - p.w / r.s * kLn2;
  return r;
}

// One thread: everything of a row but its alternatives.
template <typename T>
__device__ __forceinline__ void write_scores(const ScoresArgs& a, const Row& w, int r, const RowScore& q) {
  if (a.logp != nullptr) {
    const int t = a.tokens[r];
    a.logp[r] = t < 0 ? 0.f : t >= w.V ? nan_f() : log_p(a.x.tau, load1(elem_at<T>(w, t)), q.top, q.log_s);
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
__global__ __launch_bounds__(kThreads) void scores_part_kernel(ScoresArgs a, Split sp) {
  __shared__ float red[3][kThreads / 64];
  const int r = blockIdx.x / sp.chunks, ch = blockIdx.x % sp.chunks, slot0 = ch * U * kThreads;
  const Row w = row_at<T>(a.x.logits, a.x.ld, r, a.x.V);
  u32x4 x[U];
  load_tile<T, kThreads, U>(x, w, slot0);
  Part p;
  p.top = block_max<kThreads>(tile_max<T>(x), red[0]);
  tile_scores<T>(a.x, x, finite_top(p.top), p.s, p.w);
  if (a.m > 0) tile_groups<T, kThreads, U>(x, w, slot0, sp.glog, sp.gm + (int64_t)r * sp.gstride);
  p.s = block_sum<kThreads>(p.s, red[1]);
  p.w = block_sum<kThreads>(p.w, red[2]);
  if (threadIdx.x == 0) sp.parts[blockIdx.x] = make_float4(p.top, p.s, p.w, 0.f);
}

// A row's parts as one (a block of kThreads threads).
__device__ __forceinline__ Part merge_parts(const VocabRows& x, const float4* parts, int n, float (*red)[kThreads / 64]) {
  float top = -INFINITY;
  for (int i = threadIdx.x; i < n; i += kThreads) top = fmaxf(top, parts[i].x);
  top = block_max<kThreads>(top, red[0]);
  const float t = finite_top(top);
  float s = 0.f, w = 0.f;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const float4 q = parts[i];
    const float d = scaled(x, fmaxf(q.x - t, x.floor)), e = exp2_fast(d);
    s = fmaf(q.y, e, s);
    w = fmaf(fmaf(q.y, d, q.z), e, w);
  }
  return Part{top, block_sum<kThreads>(s, red[1]), block_sum<kThreads>(w, red[2])};
}

template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void scores_finish_kernel(ScoresArgs a, Split sp) {
  __shared__ float red[3][kThreads / 64];
  const int r = blockIdx.x;
  const Row w = row_at<T>(a.x.logits, a.x.ld, r, a.x.V);
  const RowScore q = row_score(merge_parts(a.x, sp.parts + (int64_t)r * sp.chunks, sp.chunks, red));
  if (threadIdx.x == 0) write_scores<T>(a, w, r, q);
  if constexpr (TOP) {
    __shared__ TopShared sh;
    top_select<T>(w, sp.gm + (int64_t)r * sp.gstride, (w.slots + (1 << sp.glog) - 1) >> sp.glog, sp.glog, a.m,
                  a.x.tau, q.top, q.log_s, a.top_idx + (int64_t)r * a.m, a.top_logp + (int64_t)r * a.m, sh);
  }
}

// Rows of one tile, one block each.
template <typename T, int U, bool TOP>
__global__ __launch_bounds__(kThreads) void scores_row_kernel(ScoresArgs a, Split sp) {
  __shared__ float red[3][kThreads / 64];
  __shared__ float gm[TOP ? U * kThreads : 1];
  const int r = blockIdx.x;
  const Row w = row_at<T>(a.x.logits, a.x.ld, r, a.x.V);
  u32x4 x[U];
  load_tile<T, kThreads, U>(x, w, 0);
  Part p;
  p.top = block_max<kThreads>(tile_max<T>(x), red[0]);
  tile_scores<T>(a.x, x, finite_top(p.top), p.s, p.w);
  if constexpr (TOP) tile_groups<T, kThreads, U>(x, w, 0, sp.glog, gm);
  p.s = block_sum<kThreads>(p.s, red[1]);
  p.w = block_sum<kThreads>(p.w, red[2]);
  const RowScore q = row_score(p);
  if (threadIdx.x == 0) write_scores<T>(a, w, r, q);
  if constexpr (TOP) {
    __shared__ TopShared sh;
    top_select<T>(w, gm, (w.slots + (1 << sp.glog) - 1) >> sp.glog, sp.glog, a.m, a.x.tau, q.top, q.log_s,
                  a.top_idx + (int64_t)r * a.m, a.top_logp + (int64_t)r * a.m, sh);
  }
}

// What a logit's gradient is made of.
struct ScoreGrad {
  bool zero;          // a row without weight
  int token;
  float gl, ge;       // incoming gradients / tau
  float top, inv, b;  // p = inv 2^d, log p + H = d ln 2 + b
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
  return q;
}

template <typename T>
__device__ __forceinline__ void scores_grad_slot(const VocabRows& a, const ScoreGrad& q, const Row& w,
                                                 const u32x4& x, int s, float (&v)[kE<T>]) {
  const int t = q.token + w.o - s * kE<T>;  // the token's place in the slot
#pragma unroll
  for (int c = 0; c < kE<T>; ++c) {
    const float d = scaled(a, fmaxf(get<T>(x, c) - q.top, a.floor)), p = exp2_fast(d) * q.inv;
    v[c] = -p * fmaf(q.ge, fmaf(d, kLn2, q.b), q.gl);
    if (c == t) v[c] += q.gl;
  }
}

template <typename T, int NTH, int U>
__device__ __forceinline__ void zero_tile(const Row& w, const Row& out, int slot0) {
  const float v[kE<T>] = {};
#pragma unroll 1
  for (int u = 0; u < U; ++u) {
    const int s = slot0 + u * NTH + threadIdx.x;
    if (s < w.slots) store_slot<T>(w, out, s, v);
  }
}

template <typename T, int U>
__global__ __launch_bounds__(kThreads) void scores_grad_kernel(VocabRows x, const int32_t* tokens, const float* stats,
                                                               RowGrad g, int chunks) {
  const int r = blockIdx.x / chunks, slot0 = blockIdx.x % chunks * U * kThreads;
  const Row w = row_at<T>(x.logits, x.ld, r, x.V), out = row_at<T>(g.dlogits, g.ldd, r, x.V);
  const float* st = stats + (int64_t)r * kStats;
  const ScoreGrad q = score_grad(x, tokens, g, r, st[0], st[1], st[2]);
  if (q.zero) return zero_tile<T, kThreads, U>(w, out, slot0);
  u32x4 l[U];
  load_tile<T, kThreads, U>(l, w, slot0);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int s = slot0 + u * kThreads + threadIdx.x;
    if (s >= w.slots) break;
    float v[kE<T>];
    scores_grad_slot<T>(x, q, w, l[u], s, v);
    store_slot<T>(w, out, s, v);
  }
}

// ---------------------------------------------------------------- distillation

// A teacher's list as one wave takes it, two slots a lane, in 64 bits: the loss is a small
// difference of its terms.
struct List {
  int id[2], first[2];  // -1: no entry; the first slot of a repeated id
  bool own[2];          // an entry, in its first slot
  double e[2], p[2];    // exp((l - em) / tau); the teacher's probability
  double em, se;        // the entries' largest logit; sum e
  double sp, pl;        // sum p; sum p (log p - (l - em) / tau)
  double P;             // the teacher's mass outside the list
  bool none;
};

template <typename T>
__device__ __forceinline__ List take_list(const DistillArgs& a, const Row& w, int r, int32_t* ids) {
  const int lane = threadIdx.x & 63;
  List q;
  double l[2], val[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int j = lane + 64 * k;
    const int id = j < a.m ? a.ids[(int64_t)r * a.m + j] : -1;
    q.id[k] = id >= 0 && id < w.V ? id : -1;
    q.first[k] = j;
    ids[j] = q.id[k];
    l[k] = q.id[k] >= 0 ? (double)load1(elem_at<T>(w, id)) : -INFINITY;
    val[k] = q.id[k] >= 0 ? (double)a.values[(int64_t)r * a.m + j] : -INFINITY;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (int i = min(a.m, kTopMax) - 1; i >= 0; --i) {
    const int id = ids[i];
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (id == q.id[k] && i < lane + 64 * k) q.first[k] = i;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    q.own[k] = q.id[k] >= 0 && q.first[k] == lane + 64 * k;
    if (!q.own[k]) val[k] = -INFINITY;
  }
  const double tau = a.x.tau;
  q.none = __ballot(q.own[0] || q.own[1]) == 0;
  q.em = wave_max64(l[0] > l[1] ? l[0] : l[1]);
  if (q.em == -INFINITY) q.em = 0.;
  const double vmax = a.tail ? 0. : wave_max64(val[0] > val[1] ? val[0] : val[1]);
  const double vt = a.tail ? 1. : tau;
  double lp[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    q.e[k] = q.id[k] >= 0 ? exp((l[k] - q.em) / tau) : 0.;
    lp[k] = q.own[k] ? (val[k] - vmax) / vt : -INFINITY;
    q.p[k] = q.own[k] ? exp(lp[k]) : 0.;
  }
  q.se = wave_sum64((q.own[0] ? q.e[0] : 0.) + (q.own[1] ? q.e[1] : 0.));
  q.sp = wave_sum64(q.p[0] + q.p[1]);
  // A value that is a NaN or +infinity: no term of the row is a number.
  const double bad = q.sp - q.sp, norm = a.tail ? 1. : q.sp, shift = a.tail ? 0. : log(q.sp);
  q.P = (a.tail && !(q.sp > 1.) ? 1. - q.sp : 0.) + bad;
  double pl = 0.;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    q.p[k] = q.own[k] ? q.p[k] / norm + bad : 0.;
    lp[k] = lp[k] - shift;
    if (q.own[k] && !(q.p[k] == 0.)) pl += q.p[k] * (lp[k] - (l[k] - q.em) / tau);
  }
  q.pl = wave_sum64(pl);
  if (!a.tail) q.sp = 1. + bad;
  return q;
}

// The row's numbers once the sum over the other logits is known: top and sum of exp((l - top) /
// tau) over them.
struct ListEnd {
  double loss;
  float k;       // tau (Q - P) / (sum outside): the others' gradient is k exp((l - top) / tau)
  double scale;  // q = scale e for the entries
};

__device__ __forceinline__ ListEnd end_list(const DistillArgs& a, const List& q, float top, double rest) {
  ListEnd z;
  const double tau = a.x.tau;
  // Sums relative to the larger maximum.
  const bool over = rest != 0. && (q.se == 0. || top > q.em);
  const double m = over ? (double)top : q.em;
  const double fr = rest != 0. ? exp((top - m) / tau) : 0., fe = exp((q.em - m) / tau);
  const double total = q.se * fe + rest * fr;
  const double log_total = total > 0. ? log(total) : (double)nan_f();
  z.scale = total > 0. ? fe / total : (double)nan_f();
  z.loss = q.pl + q.sp * (log_total + (m - q.em) / tau);
  if (!(rest == 0.) && !(q.P == 0.))
    z.loss += q.P * (log(q.P) - (log(rest) + (top - m) / tau - log_total));
  z.loss = q.none ? 0. : tau * tau * z.loss;
  z.k = rest == 0. ? (total > 0. ? 0.f : nan_f()) : (float)(tau * (fr / total - q.P / rest));
  return z;
}

// Each slot's own gradient tau (q - p) to st (a repeated id's is its first slot's; no
// entry's is not used).
__device__ __forceinline__ void list_grads(const DistillArgs& a, const List& q, const ListEnd& z, float* own) {
  const int lane = threadIdx.x & 63;
  const double tau = a.x.tau;
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (q.own[k]) own[lane + 64 * k] = (float)(tau * (q.e[k] * z.scale - q.p[k]));
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ void write_state(const DistillArgs& a, const List& q, const ListEnd& z, float top,
                                            const float* own, int r) {
  const int lane = threadIdx.x & 63;
  float* st = a.state + (int64_t)r * (a.m + kState);
  if (lane == 0) {
    st[0] = top;
    st[1] = z.k;
    st[2] = q.none ? 1.f : 0.f;
    st[3] = 0.f;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int j = lane + 64 * k;
    if (j < a.m) st[kState + j] = q.id[k] >= 0 ? own[q.first[k]] : 0.f;
  }
}

template <typename T, int U>
__global__ __launch_bounds__(kThreads) void distill_part_kernel(DistillArgs a, Split sp) {
  __shared__ float red[2][kThreads / 64];
  __shared__ Marks<T, kThreads, U> marks;
  const int r = blockIdx.x / sp.chunks, ch = blockIdx.x % sp.chunks, slot0 = ch * U * kThreads;
  const Row w = row_at<T>(a.x.logits, a.x.ld, r, a.x.V);
  const int id = (int)threadIdx.x < a.m ? a.ids[(int64_t)r * a.m + threadIdx.x] : -1;
  u32x4 x[U];
  load_tile<T, kThreads, U>(x, w, slot0);
  clear_marks(marks);
  __syncthreads();
  set_mark(marks, w, slot0, id);
  __syncthreads();
  drop_marked(x, marks);
  const float top = block_max<kThreads>(tile_max<T>(x), red[0]);
  const float s = block_sum<kThreads>(tile_sum<T>(a.x, x, finite_top(top)), red[1]);
  if (threadIdx.x == 0) sp.parts[blockIdx.x] = make_float4(top, s, 0.f, 0.f);
}

// One wave a row.
template <typename T>
__global__ __launch_bounds__(kWave) void distill_finish_kernel(DistillArgs a, Split sp) {
  __shared__ int32_t ids[kTopMax];
  __shared__ float own[kTopMax];
  const int r = blockIdx.x;
  const Row w = row_at<T>(a.x.logits, a.x.ld, r, a.x.V);
  const float4* parts = sp.parts + (int64_t)r * sp.chunks;
  float top = -INFINITY;
  for (int i = threadIdx.x; i < sp.chunks; i += kWave) top = fmaxf(top, parts[i].x);
  top = finite_top(wave_max(top));
  double s = 0.;
  for (int i = threadIdx.x; i < sp.chunks; i += kWave)
    s += (double)parts[i].y * (double)exp2_fast(scaled(a.x, parts[i].x - top));
  const double rest = wave_sum64(s);
  const List q = take_list<T>(a, w, r, ids);
  const ListEnd z = end_list(a, q, top, rest);
  if (threadIdx.x == 0) a.loss[r] = (float)z.loss;
  if (a.state == nullptr) return;
  list_grads(a, q, z, own);
  write_state(a, q, z, top, own, r);
}

template <typename T, int U>
__global__ __launch_bounds__(kThreads) void distill_grad_kernel(VocabRows x, int m, const int32_t* ids,
                                                                const float* state, RowGrad g, int chunks) {
  const int r = blockIdx.x / chunks, slot0 = blockIdx.x % chunks * U * kThreads;
  const Row w = row_at<T>(x.logits, x.ld, r, x.V), out = row_at<T>(g.dlogits, g.ldd, r, x.V);
  const float* st = state + (int64_t)r * (m + kState);
  const float gr = g.g[r], top = st[0], k = st[1] * gr;
  if (gr == 0.f || st[2] != 0.f) return zero_tile<T, kThreads, U>(w, out, slot0);
  u32x4 l[U];
  load_tile<T, kThreads, U>(l, w, slot0);
  const int j = threadIdx.x, id = j < m ? ids[(int64_t)r * m + j] : -1;
  const float own = j < m ? st[kState + j] * gr : 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int s = slot0 + u * kThreads + threadIdx.x;
    if (s >= w.slots) break;
    float v[kE<T>];
#pragma unroll
    for (int c = 0; c < kE<T>; ++c) v[c] = exp2_fast(scaled(x, get<T>(l[u], c) - top)) * k;
    store_slot<T>(w, out, s, v);
  }
  // The list's entries over what they got as the others; all of them are this block's.
  __syncthreads();
  const int s = (id + w.o) / kE<T>;
  if (id >= 0 && id < x.V && s >= slot0 && s - slot0 < U * kThreads)
    store1(const_cast<T*>(elem_at<T>(out, id)), own);
}

}  // namespace

namespace {

template <typename T>
int slots_most(int V) {
  return (V + 2 * (kE<T> - 1)) / kE<T>;  // of a row that starts at any element
}

// Slots a thread of a part: all kTileU where that gives every CU four blocks, else fewer,
// so that few rows spread over the chip.
template <typename T>
int split_u(int rows, int V) {
  int u = kTileU;
  while (u > 1 && (int64_t)rows * ((slots_most<T>(V) + u * kThreads - 1) / (u * kThreads)) < 1024) u /= 2;
  return u;
}

template <typename F>
void by_u(int u, const F& f) {
  if (u == 8) f(std::integral_constant<int, 8>{});
  else if (u == 4) f(std::integral_constant<int, 4>{});
  else if (u == 2) f(std::integral_constant<int, 2>{});
  else f(std::integral_constant<int, 1>{});
}

int group_log(int slots) { return slots <= 2048 ? 0 : slots <= 8192 ? 2 : 4; }

template <typename T>
Split split_of(int rows, int V, int m, void* ws, int u) {
  Split sp{};
  const int slots = slots_most<T>(V);
  sp.chunks = (slots + u * kThreads - 1) / (u * kThreads);
  sp.glog = group_log(slots);
  sp.gstride = m > 0 ? (slots >> sp.glog) + 1 : 0;
  sp.parts = static_cast<float4*>(ws);
  sp.gm = reinterpret_cast<float*>(sp.parts + (int64_t)rows * sp.chunks);
  return sp;
}

template <typename T>
hipError_t scores(const ScoresArgs& a, void* ws, hipStream_t s) {
  const int slots = slots_most<T>(a.x.V);
  if (slots <= kTileU * kThreads) {
    by_u(slots <= kThreads ? 1 : slots <= 2 * kThreads ? 2 : slots <= 4 * kThreads ? 4 : 8, [&](auto u) {
      const Split sp = split_of<T>(a.x.rows, a.x.V, a.m, ws, u.value);
      if (a.m > 0)
        hipLaunchKernelGGL((scores_row_kernel<T, u.value, true>), dim3(a.x.rows), dim3(kThreads), 0, s, a, sp);
      else
        hipLaunchKernelGGL((scores_row_kernel<T, u.value, false>), dim3(a.x.rows), dim3(kThreads), 0, s, a, sp);
    });
    return note_hip(hipGetLastError());
  }
  by_u(split_u<T>(a.x.rows, a.x.V), [&](auto u) {
    const Split sp = split_of<T>(a.x.rows, a.x.V, a.m, ws, u.value);
    hipLaunchKernelGGL((scores_part_kernel<T, u.value>), dim3((unsigned)a.x.rows * sp.chunks), dim3(kThreads), 0, s,
                       a, sp);
    if (a.m > 0)
      hipLaunchKernelGGL((scores_finish_kernel<T, true>), dim3(a.x.rows), dim3(kThreads), 0, s, a, sp);
    else
      hipLaunchKernelGGL((scores_finish_kernel<T, false>), dim3(a.x.rows), dim3(kThreads), 0, s, a, sp);
  });
  return note_hip(hipGetLastError());
}

template <typename T>
hipError_t scores_grad(const VocabRows& x, const int32_t* tokens, const float* stats, const RowGrad& g,
                       hipStream_t s) {
  by_u(split_u<T>(x.rows, x.V), [&](auto u) {
    const int chunks = (slots_most<T>(x.V) + u.value * kThreads - 1) / (u.value * kThreads);
    hipLaunchKernelGGL((scores_grad_kernel<T, u.value>), dim3((unsigned)x.rows * chunks), dim3(kThreads), 0, s, x,
                       tokens, stats, g, chunks);
  });
  return note_hip(hipGetLastError());
}

template <typename T>
hipError_t distill(const DistillArgs& a, void* ws, hipStream_t s) {
  by_u(split_u<T>(a.x.rows, a.x.V), [&](auto u) {
    const Split sp = split_of<T>(a.x.rows, a.x.V, 0, ws, u.value);
    hipLaunchKernelGGL((distill_part_kernel<T, u.value>), dim3((unsigned)a.x.rows * sp.chunks), dim3(kThreads), 0, s,
                       a, sp);
    hipLaunchKernelGGL(distill_finish_kernel<T>, dim3(a.x.rows), dim3(kWave), 0, s, a, sp);
  });
  return note_hip(hipGetLastError());
}

template <typename T>
hipError_t distill_grad(const VocabRows& x, int m, const int32_t* ids, const float* state, const RowGrad& g,
                        hipStream_t s) {
  by_u(split_u<T>(x.rows, x.V), [&](auto u) {
    const int chunks = (slots_most<T>(x.V) + u.value * kThreads - 1) / (u.value * kThreads);
    hipLaunchKernelGGL((distill_grad_kernel<T, u.value>), dim3((unsigned)x.rows * chunks), dim3(kThreads), 0, s, x,
                       m, ids, state, g, chunks);
  });
  return note_hip(hipGetLastError());
}

}  // namespace

size_t scores_bytes(int rows, int V, int m) {
  size_t most = 0;
  // Either type.  A split finer than kTileU has less than 2 * 1024 parts in all; never fewer
  // bytes for more rows.
  const auto add = [&](int slots) {
    const size_t coarse = (slots + kTileU * kThreads - 1) / (kTileU * kThreads), fine = (slots + kThreads - 1) / kThreads;
    size_t b = std::max(rows * coarse, std::min<size_t>(rows * fine, 2048)) * sizeof(float4);
    if (m > 0) b += (size_t)rows * ((slots >> group_log(slots)) + 1) * 4;
    most = std::max(most, b);
  };
  add(slots_most<float>(V));
  add(slots_most<uint16_t>(V));
  return most;
}

hipError_t launch_scores(const ScoresArgs& a, void* ws, hipStream_t s) {
  return a.x.bf16 ? scores<uint16_t>(a, ws, s) : scores<float>(a, ws, s);
}
hipError_t launch_scores_grad(const VocabRows& x, const int32_t* tokens, const float* stats, const RowGrad& g,
                              hipStream_t s) {
  return x.bf16 ? scores_grad<uint16_t>(x, tokens, stats, g, s) : scores_grad<float>(x, tokens, stats, g, s);
}
hipError_t launch_distill(const DistillArgs& a, void* ws, hipStream_t s) {
  return a.x.bf16 ? distill<uint16_t>(a, ws, s) : distill<float>(a, ws, s);
}
hipError_t launch_distill_grad(const VocabRows& x, int m, const int32_t* ids, const float* state, const RowGrad& g,
                               hipStream_t s) {
  return x.bf16 ? distill_grad<uint16_t>(x, m, ids, state, g, s) : distill_grad<float>(x, m, ids, state, g, s);
}

}  // namespace de
