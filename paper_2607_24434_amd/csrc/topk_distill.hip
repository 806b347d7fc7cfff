// Distillation from a teacher's top logits, forward and backward.
//
// With q = softmax(l / tau), p the teacher's probabilities of the list's entries S, P its mass
// outside them (0 unless asked for) and Q = sum_{v not in S} q_v:
//   loss = tau^2 (sum_S p (log p - log q) + P (log P - log Q))
//   d loss / d l_v = tau (W q_v - p_v) in S, tau q_v (W - P / Q) outside,
// W = sum_S p + P the weight of log sum exp(l / tau).  W is one unless the list's own masses
// are more than that (P = 0), or the student has no mass outside the list (P's term is left out).
// The logits outside the list are summed directly: one minus the entries' mass would lose a
// small Q.  Memory bounds it: a whole row is read once and its gradient written once from the
// same registers (1024 fp32 rows of 102400 with lists of 64: 166 us, 5.1 TB/s where a copy
// reaches 4.9; 2048 bf16 rows of 65537 with lists of 128: 117 us, 4.6 TB/s).
#include "scores_core.h"

namespace de {
namespace {

// A teacher's list, in 64 bits: the loss is a small difference of its terms.
struct List {
  alignas(16) int32_t id[kTopMax];  // -1: no entry
  float l[kTopMax];        // the student's logits, and
  float val[kTopMax];      // the teacher's values of the entries
  int32_t first[kTopMax];  // the first slot of the same id; an entry's own is itself
  double e[kTopMax];       // exp((l - em) / tau)
  double p[kTopMax];       // exp(value - vmax), 0 but in first slots
  float em, vmax;          // the entries' largest logit; the largest value (0 with tail)
  // Once the sum over the other logits is known:
  float own[kTopMax];      // an entry's gradient tau (W q - p), in its first slot
  float k;                 // tau (W Q - P) / (sum outside): the others' is k exp((l - top) / tau)
  int none;                // no entry at all
};

__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// What the list has in memory, before a gradient may be written over it (NTH threads).
template <typename T, int NTH>
__device__ __forceinline__ void fetch_list(const DistillArgs& a, const Row& w, int r, List& q) {
#pragma unroll
  for (int j = threadIdx.x; j < kTopMax; j += NTH) {
    const int at = j < a.m ? a.ids[(int64_t)r * a.m + j] : -1, id = at >= 0 && at < w.V ? at : -1;
    const float val = j < a.m ? a.values[(int64_t)r * a.m + j] : 0.f;
    q.id[j] = id;
    q.l[j] = id >= 0 ? load1(elem_at<T>(w, id)) : -INFINITY;
    q.val[j] = id >= 0 ? val : -INFINITY;
  }
}

// The entries' exponentials, by the first four of a block's waves (NTH threads): slot i's by
// thread i, its value's by thread kTopMax + i.  Each wave finds the repeated ids and the two
// maxima for itself, so that it waits for no other.
template <int NTH>
__device__ __forceinline__ void list_terms(const DistillArgs& a, List& q) {
  if (threadIdx.x >= 2 * kTopMax) return;
  const int lane = threadIdx.x & 63;
  const int id0 = q.id[lane], id1 = q.id[lane + 64];
  int f0 = lane, f1 = lane + 64;
  for (int i = (a.m - 1) / 4 * 4; i >= 0; i -= 4) {
    const int4 o = *reinterpret_cast<const int4*>(&q.id[i]);
    f0 = o.w == id0 && i + 3 < f0 ? i + 3 : f0;
    f0 = o.z == id0 && i + 2 < f0 ? i + 2 : f0;
    f0 = o.y == id0 && i + 1 < f0 ? i + 1 : f0;
    f0 = o.x == id0 && i < f0 ? i : f0;
    f1 = o.w == id1 && i + 3 < f1 ? i + 3 : f1;
    f1 = o.z == id1 && i + 2 < f1 ? i + 2 : f1;
    f1 = o.y == id1 && i + 1 < f1 ? i + 1 : f1;
    f1 = o.x == id1 && i < f1 ? i : f1;
  }
  const bool own0 = id0 >= 0 && f0 == lane, own1 = id1 >= 0 && f1 == lane + 64;
  const float em = finite_top(wave_max(fmaxf(q.l[lane], q.l[lane + 64])));  // a NaN shows in its own term
  const float vmax =
      a.tail ? 0.f : wave_max(fmaxf(own0 ? q.val[lane] : -INFINITY, own1 ? q.val[lane + 64] : -INFINITY));
  const double it = 1. / (double)a.x.tau;
#pragma unroll 1
  for (int t = threadIdx.x; t < 2 * kTopMax; t += NTH) {
    const bool value = t >= kTopMax;
    const int i = t & (kTopMax - 1);
    const bool entry = value ? (i < 64 ? own0 : own1) : q.id[i] >= 0;
    const double d = (value ? (double)q.val[i] - vmax : (double)q.l[i] - em) * (value && a.tail ? 1. : it);
    (value ? q.p : q.e)[i] = entry ? exp(d) : 0.;
    if (!value) q.first[i] = i < 64 ? f0 : f1;
  }
  if (threadIdx.x == 0) {
    q.em = em;
    q.vmax = vmax;
  }
}

// One wave, once the terms are there, with top and rest = sum exp((l - top) / tau) over the other
// logits: the loss, the gradients' numbers and the state.
__device__ __forceinline__ void end_list(const DistillArgs& a, List& q, float top, double rest, int r) {
  const int lane = threadIdx.x & 63;
  const double tau = a.x.tau, it = 1. / tau;
  double se = 0., sum = 0.;
  bool any = false;
#pragma unroll 1
  for (int j = lane; j < kTopMax; j += kWave) {
    const bool own = q.id[j] >= 0 && q.first[j] == j;
    any = any || own;
    se += own ? q.e[j] : 0.;
    sum += q.p[j];
  }
  se = wave_sum64(se);
  sum = wave_sum64(sum);
  const bool none = __ballot(any) == 0;
  // A value that is a NaN or +infinity: no term of the row is a number.
  const double bad = sum - sum, norm = a.tail ? 1. : 1. / sum;
  const double P = (a.tail && !(sum > 1.) ? 1. - sum : 0.) + bad;
  // The student's sums relative to the larger maximum; the first lane has the other logits'
  // part, the second lane the entries'; a side without any mass has no maximum, and none is taken.
  const bool over = rest != 0. && (se == 0. || top > q.em);
  const double m = over ? (double)top : q.em, far = ((lane == 0 ? (double)top : q.em) - m) * it;
  const double f = exp(far), fr = rest != 0. ? read_lane(f, 0) : 0., fe = se != 0. ? read_lane(f, 1) : 0.;
  const double total = se * fe + rest * fr, odd = total > 0. && total < INFINITY ? 0. : (double)nan_f();
  const double lg = log(lane == 0 ? rest : lane == 1 ? total : a.tail ? P : sum);
  const double log_total = read_lane(lg, 1) + odd, log_mass = read_lane(lg, 2), part = 1. / total + odd;
  const double shift = a.tail ? 0. : log_mass, vt = a.tail ? 1. : it;
  const double W = a.tail ? sum + (rest != 0. ? P : bad) : 1.;
  double pl = 0.;
#pragma unroll 1
  for (int j = lane; j < kTopMax; j += kWave) {
    if (q.id[j] < 0) continue;
    const bool own = q.first[j] == j;
    const double p = own ? q.p[j] * norm + bad : 0.;
    q.own[j] = (float)(tau * (W * (q.e[j] * fe * part) - p));
    if (own && !(p == 0.)) pl += p * (((double)q.val[j] - q.vmax) * vt - shift - ((double)q.l[j] - q.em) * it);
  }
  pl = wave_sum64(pl);
  if (lane == 0) {
    double loss = pl + ((a.tail ? sum : 1.) + bad) * (log_total + (m - q.em) * it);
    if (!(rest == 0.) && !(P == 0.)) loss += P * (log_mass - (lg + far - log_total));
    a.loss[r] = none ? 0.f : (float)(tau * tau * loss);
    q.k = rest == 0. ? (float)(odd + bad) : (float)(tau * (W * fr * part - P / rest));
    q.none = none;
  }
  wave_sync();
  if (a.state == nullptr) return;
  float* st = a.state + (int64_t)r * (a.m + kState);
  if (lane == 0) {
    st[0] = top;
    st[1] = q.k;
    st[2] = none ? 1.f : 0.f;
    st[3] = 0.f;
  }
#pragma unroll 1
  for (int j = lane; j < a.m; j += kWave) st[kState + j] = q.id[j] >= 0 ? q.own[q.first[j]] : 0.f;
}

template <typename T, int U>
__global__ __launch_bounds__(kThreads, 6) void distill_part_kernel(DistillArgs a, Split sp) {
  __shared__ float red[3][kThreads / 64];
  __shared__ Marks<T, kThreads, U> marks;
  const int r = blockIdx.x / sp.chunks, slot0 = blockIdx.x % sp.chunks * sp.nu * kThreads;
  const Row w = until(row_at<T>(a.x.logits, a.x.ld, r, a.x.V), slot0 + sp.nu * kThreads);
  const int id = (int)threadIdx.x < a.m ? a.ids[(int64_t)r * a.m + threadIdx.x] : -1;
  Tile<kThreads, U> x;
  load_tile<T>(x, w, slot0);
  clear_marks(marks);
  __syncthreads();
  set_mark(marks, w, slot0, id);
  __syncthreads();
  const auto unlisted = [&](u32x4& s, int u) __attribute__((always_inline)) { drop_marked(s, u, marks); };
  const Part p = block_part<kThreads>(a.x, tile_sums<T, true>(a.x, x, w, unlisted, NoPeak{}), red);
  if (threadIdx.x == 0) sp.parts[blockIdx.x] = make_float4(p.top, p.s, p.w, 0.f);
}

// One wave a row.
template <typename T>
__global__ __launch_bounds__(kWave) void distill_finish_kernel(DistillArgs a, Split sp) {
  __shared__ List q;
  const int r = blockIdx.x;
  const Row w = row_at<T>(a.x.logits, a.x.ld, r, a.x.V);
  fetch_list<T, kWave>(a, w, r, q);
  wave_sync();
  list_terms<kWave>(a, q);
  wave_sync();
  const float4* parts = sp.parts + (int64_t)r * sp.chunks;
  float top = -INFINITY;
  for (int i = threadIdx.x; i < sp.chunks; i += kWave) top = fmaxf(top, parts[i].x);
  top = finite_top(wave_max(top));
  double s = 0.;
  for (int i = threadIdx.x; i < sp.chunks; i += kWave) {
    const Part p = rebased(a.x, Part{parts[i].x, parts[i].y, parts[i].z}, top);
    s += (double)p.s + (double)a.x.corr * p.w;
  }
  end_list(a, q, top, wave_sum64(s), r);
}

template <typename T, int U>
__global__ __launch_bounds__(kThreads) void distill_grad_kernel(VocabRows x, int m, const int32_t* ids,
                                                                const float* state, RowGrad g, Split sp) {
  const int r = blockIdx.x / sp.chunks, slot0 = blockIdx.x % sp.chunks * sp.nu * kThreads;
  const Row w = until(row_at<T>(x.logits, x.ld, r, x.V), slot0 + sp.nu * kThreads), out = row_at<T>(g.dlogits, g.ldd, r, x.V);
  const float* st = state + (int64_t)r * (m + kState);
  const float gr = g.g[r], top = st[0], k = st[1] * gr;
  if (gr == 0.f || st[2] != 0.f) return zero_tile<T, kThreads>(w, out, slot0);
  Tile<kThreads, U> l;
  static_assert(U <= kAhead * kRun, "every slot is loaded at once");
  load_tile<T>(l, w, slot0);
  load_first<T>(l, w);
  load_last<T>(l, w);
  const int j = threadIdx.x, id = j < m ? ids[(int64_t)r * m + j] : -1;
  const float own = j < m ? st[kState + j] * gr : 0.f;
  each_slot(l, [&](const u32x4& s, int u) __attribute__((always_inline)) {
    if (l.slot(u) >= w.slots) return;
    float v[kE<T>];
    each<kE<T>>([&](auto c) __attribute__((always_inline)) {
      v[c] = exp2_fast(scaled(x, get<T>(s, c), top)) * k;
    });
    store_slot<T>(w, out, l.slot(u), v);
  });
  // The list's entries over what they got as the others; all of them are this block's.
  __syncthreads();
  const int s = (id + w.o) / kE<T>;
  if (id >= 0 && id < x.V && s >= slot0 && s < w.slots)
    store1(const_cast<T*>(elem_at<T>(out, id)), own);
}

// Whole rows, one block each, and their gradient where one is asked for.  The first waves
// fetch the list before their logits (a load that comes behind those takes as long as all of
// them: 12 of a row's 31 us at 2048 bf16 rows of 65537), and four of them take its
// exponentials while the logits come.
template <typename T, int NTH, int U>
__global__ __launch_bounds__(NTH, whole_waves(NTH, U)) void distill_whole_kernel(DistillArgs a, RowGrad g) {
  __shared__ float red[3][NTH / 64];
  __shared__ Marks<T, NTH, U> marks;
  __shared__ List q;
  const int r = blockIdx.x;
  const Row w = row_at<T>(a.x.logits, a.x.ld, r, a.x.V);
  clear_marks(marks);
  __syncthreads();
  Tile<NTH, U> x;
  if (threadIdx.x < kTopMax) {
    fetch_list<T, NTH>(a, w, r, q);
    set_mark(marks, w, 0, q.id[threadIdx.x]);
  } else {
    load_tile<T>(x, w, 0);
  }
  __syncthreads();
  if (threadIdx.x < kTopMax) load_tile<T>(x, w, 0);
  list_terms<NTH>(a, q);
  const auto unlisted = [&](u32x4& s, int u) __attribute__((always_inline)) { drop_marked(s, u, marks); };
  const Part p = block_part<NTH>(a.x, tile_sums<T, true>(a.x, x, w, unlisted, NoPeak{}), red);
  const float top = finite_top(p.top);
  if (threadIdx.x < kWave) end_list(a, q, top, (double)p.s + (double)a.x.corr * p.w, r);
  if (g.dlogits == nullptr) return;
  __syncthreads();
  const Row out = row_at<T>(g.dlogits, g.ldd, r, a.x.V);
  const float gr = g.g[r], k = q.k * gr;
  if (gr == 0.f || q.none) return zero_tile<T, NTH>(w, out, 0);
  each_slot(x, [&](const u32x4& s, int u) __attribute__((always_inline)) {
    if (x.slot(u) >= w.slots) return;
    float v[kE<T>];
    each<kE<T>>([&](auto c) __attribute__((always_inline)) {
      v[c] = exp2_fast(scaled(a.x, get<T>(s, c), top)) * k;
    });
    store_slot<T>(w, out, x.slot(u), v);
  });
  // The entries over what they got as the others.
  __syncthreads();
  const int j = threadIdx.x, id = j < kTopMax ? q.id[j] : -1;
  if (id >= 0 && q.first[j] == j) store1(const_cast<T*>(elem_at<T>(out, id)), q.own[j] * gr);
}

template <typename T>
hipError_t distill_grad(const VocabRows& x, int m, const int32_t* ids, const float* state, const RowGrad& g,
                        hipStream_t s) {
  const Split sp = split_of<T>(x, 0, nullptr);
  by_u(sp.nu, [&](auto u) {
    hipLaunchKernelGGL((distill_grad_kernel<T, u.value>), dim3((unsigned)x.rows * sp.chunks), dim3(kThreads), 0, s, x,
                       m, ids, state, g, sp);
  });
  return note_hip(hipGetLastError());
}

template <typename T>
hipError_t distill(const DistillArgs& a, const RowGrad& g, void* ws, hipStream_t s) {
  if (whole_pays<T>(a.x, g.dlogits != nullptr) && by_whole<T, 18>(a.x, [&](auto k) {
        hipLaunchKernelGGL((distill_whole_kernel<T, k.kNth, k.kU>), dim3(a.x.rows), dim3(k.kNth), 0, s, a, g);
      }))
    return note_hip(hipGetLastError());
  const Split sp = split_of<T>(a.x, 0, ws);
  by_u(sp.nu, [&](auto u) {
    hipLaunchKernelGGL((distill_part_kernel<T, u.value>), dim3((unsigned)a.x.rows * sp.chunks), dim3(kThreads), 0, s,
                       a, sp);
  });
  hipLaunchKernelGGL(distill_finish_kernel<T>, dim3(a.x.rows), dim3(kWave), 0, s, a, sp);
  const hipError_t e = note_hip(hipGetLastError());
  return e != hipSuccess || g.dlogits == nullptr ? e : distill_grad<T>(a.x, a.m, a.ids, a.state, g, s);
}

}  // namespace

hipError_t launch_distill(const DistillArgs& a, const RowGrad& g, void* ws, hipStream_t s) {
  return a.x.bf16 ? distill<uint16_t>(a, g, ws, s) : distill<float>(a, g, ws, s);
}
hipError_t launch_distill_grad(const VocabRows& x, int m, const int32_t* ids, const float* state, const RowGrad& g,
                               hipStream_t s) {
  return x.bf16 ? distill_grad<uint16_t>(x, m, ids, state, g, s) : distill_grad<float>(x, m, ids, state, g, s);
}

}  // namespace de
