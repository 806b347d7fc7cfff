// Distillation from a teacher's top logits, forward and backward.
#include "scores_core.h"

namespace de {
namespace {

// ---------------------------------------------------------------- distillation

// A teacher's list as one wave takes it, in 64 bits: the loss is a small difference of its
// terms.  Two slots a lane.
struct List {
  alignas(16) int32_t id[kTopMax];  // -1: no entry
  int32_t first[kTopMax];  // the first slot of the same id; an entry's own is itself
  double e[kTopMax];       // exp((l - em) / tau)
  double p[kTopMax];       // the teacher's probability (0 but in an entry's first slot)
  double em, se;           // the entries' largest logit; sum e
  double sp, pl;           // sum p; sum p (log p - (l - em) / tau)
  double P;                // the teacher's mass outside the list
  int none;                // no entry at all
  // Once the sum over the other logits is known:
  float own[kTopMax];      // an entry's gradient tau (q - p), in its first slot
  float k;                 // tau (Q - P) / (sum outside): the others' is k exp((l - top) / tau)
};

__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// One wave: everything that does not need the other logits.
template <typename T>
__device__ __forceinline__ void take_list(const DistillArgs& a, const Row& w, int r, List& q) {
  const int lane = threadIdx.x & 63;
  const double tau = a.x.tau;
  int ids[2], first[2];
  double l[2], val[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int j = lane + 64 * k;
    const int id = j < a.m ? a.ids[(int64_t)r * a.m + j] : -1;
    ids[k] = id >= 0 && id < w.V ? id : -1;
    first[k] = j;
    q.id[j] = ids[k];
    l[k] = ids[k] >= 0 ? (double)load1(elem_at<T>(w, id)) : -INFINITY;
    val[k] = ids[k] >= 0 ? (double)a.values[(int64_t)r * a.m + j] : -INFINITY;
  }
  wave_sync();
  for (int i = (a.m - 1) / 4 * 4; i >= 0; i -= 4) {
    const int4 id = *reinterpret_cast<const int4*>(&q.id[i]);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int j = lane + 64 * k;
      if (id.w == ids[k] && i + 3 < j) first[k] = i + 3;
      if (id.z == ids[k] && i + 2 < j) first[k] = i + 2;
      if (id.y == ids[k] && i + 1 < j) first[k] = i + 1;
      if (id.x == ids[k] && i < j) first[k] = i;
    }
  }
  bool own[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    own[k] = ids[k] >= 0 && first[k] == lane + 64 * k;
    if (!own[k]) val[k] = -INFINITY;
  }
  double em = wave_max64(l[0] > l[1] ? l[0] : l[1]);
  if (em == -INFINITY) em = 0.;
  const double vmax = a.tail ? 0. : wave_max64(val[0] > val[1] ? val[0] : val[1]);
  const double vt = a.tail ? 1. : tau;
  double e[2], p[2], lp[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    e[k] = ids[k] >= 0 ? exp((l[k] - em) / tau) : 0.;
    lp[k] = own[k] ? (val[k] - vmax) / vt : -INFINITY;
    p[k] = own[k] ? exp(lp[k]) : 0.;
  }
  const double se = wave_sum64((own[0] ? e[0] : 0.) + (own[1] ? e[1] : 0.));
  const double sum = wave_sum64(p[0] + p[1]);
  // A value that is a NaN or +infinity: no term of the row is a number.
  const double bad = sum - sum, norm = a.tail ? 1. : sum, shift = a.tail ? 0. : log(sum);
  double pl = 0.;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    p[k] = own[k] ? p[k] / norm + bad : 0.;
    if (own[k] && !(p[k] == 0.)) pl += p[k] * (lp[k] - shift - (l[k] - em) / tau);
    const int j = lane + 64 * k;
    q.first[j] = first[k];
    q.e[j] = e[k];
    q.p[j] = p[k];
  }
  pl = wave_sum64(pl);
  const bool none = __ballot(own[0] || own[1]) == 0;
  if (lane == 0) {
    q.em = em;
    q.se = se;
    q.sp = (a.tail ? sum : 1.) + bad;
    q.pl = pl;
    q.P = (a.tail && !(sum > 1.) ? 1. - sum : 0.) + bad;
    q.none = none;
  }
  wave_sync();
}

// The same wave, with top and rest = sum exp((l - top) / tau) over the other logits: the loss,
// the gradients' numbers and the state.
__device__ __forceinline__ void end_list(const DistillArgs& a, List& q, float top, double rest, int r) {
  const int lane = threadIdx.x & 63;
  const double tau = a.x.tau;
  // Sums relative to the larger maximum.
  const bool over = rest != 0. && (q.se == 0. || top > q.em);
  const double m = over ? (double)top : q.em;
  const double fr = rest != 0. ? exp((top - m) / tau) : 0., fe = exp((q.em - m) / tau);
  const double total = q.se * fe + rest * fr;
  const double log_total = total > 0. ? log(total) : (double)nan_f();
  const double scale = total > 0. ? fe / total : (double)nan_f();
  if (lane == 0) {
    double loss = q.pl + q.sp * (log_total + (m - q.em) / tau);
    if (!(rest == 0.) && !(q.P == 0.)) loss += q.P * (log(q.P) - (log(rest) + (top - m) / tau - log_total));
    a.loss[r] = q.none ? 0.f : (float)(tau * tau * loss);
    q.k = rest == 0. ? (total > 0. ? 0.f : nan_f()) : (float)(tau * (fr / total - q.P / rest));
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int j = lane + 64 * k;
    if (q.id[j] >= 0) q.own[j] = (float)(tau * (q.e[j] * scale - q.p[j]));
  }
  wave_sync();
  if (a.state == nullptr) return;
  float* st = a.state + (int64_t)r * (a.m + kState);
  if (lane == 0) {
    st[0] = top;
    st[1] = q.k;
    st[2] = q.none ? 1.f : 0.f;
    st[3] = 0.f;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int j = lane + 64 * k;
    if (j < a.m) st[kState + j] = q.id[j] >= 0 ? q.own[q.first[j]] : 0.f;
  }
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
  const Part p = block_part<kThreads>(a.x, tile_sums<T, true>(a.x, x, w, unlisted), red);
  if (threadIdx.x == 0) sp.parts[blockIdx.x] = make_float4(p.top, p.s, p.w, 0.f);
}

// One wave a row.
template <typename T>
__global__ __launch_bounds__(kWave) void distill_finish_kernel(DistillArgs a, Split sp) {
  __shared__ List q;
  const int r = blockIdx.x;
  const Row w = row_at<T>(a.x.logits, a.x.ld, r, a.x.V);
  take_list<T>(a, w, r, q);
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
  load_tile<T>(l, w, slot0);
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

// Whole rows, one block each, and their gradient where one is asked for.  The first wave
// takes the list (and the entries' logits, before any is overwritten) while the others load.
template <typename T, int NTH, int U>
__global__ __launch_bounds__(NTH, whole_waves(NTH, U)) void distill_whole_kernel(DistillArgs a, RowGrad g) {
  __shared__ float red[3][NTH / 64];
  __shared__ Marks<T, NTH, U> marks;
  __shared__ List q;
  const int r = blockIdx.x;
  const Row w = row_at<T>(a.x.logits, a.x.ld, r, a.x.V);
  if (threadIdx.x < kWave) take_list<T>(a, w, r, q);
  Tile<NTH, U> x;
  load_tile<T>(x, w, 0);
  clear_marks(marks);
  __syncthreads();
  if (threadIdx.x < kTopMax) set_mark(marks, w, 0, q.id[threadIdx.x]);
  __syncthreads();
  const auto unlisted = [&](u32x4& s, int u) __attribute__((always_inline)) { drop_marked(s, u, marks); };
  const Part p = block_part<NTH>(a.x, tile_sums<T, true>(a.x, x, w, unlisted), red);
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
  const int slots = slots_most<T>(a.x);
  if (slots <= kTileU * kThreads || (g.dlogits != nullptr && whole_row(a.x.rows, slots))) {
    by_whole(slots, [&](auto k) {
      hipLaunchKernelGGL((distill_whole_kernel<T, k.kNth, k.kU>), dim3(a.x.rows), dim3(k.kNth), 0, s, a, g);
    });
    return note_hip(hipGetLastError());
  }
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
