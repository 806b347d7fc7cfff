// What the row operators over a vocabulary are made of: a row as 16-byte slots, tiles of it in
// registers, reductions over a tile and the split of rows into parts.
//
// A row is read in tiles: each thread of a block has up to U 16-byte slots of it in
// registers, all of their loads in flight together, and takes the maximum, the sums and
// (gradients) the results from there, so that logits are read once.  Slots lie at
// multiples of 16 bytes whatever element the row starts at; its first and last one may be
// partly outside it and are then loaded by the element.
#pragma once

#include "de_common.h"
#include "scores.h"

#include <algorithm>
#include <type_traits>
#include <utility>

namespace de {
namespace {

constexpr int kThreads = 256;
constexpr int kTileU = 8;  // slots a thread of a part of a row
constexpr float kLn2 = 0.6931471805599453f;

// Rows in parts: what each part leaves for the row's last step, in the caller's scratch.
struct Split {
  int chunks;      // parts of a row
  int nu;          // slots a thread of a part, at most the kernel's U
  float4* parts;   // [rows, chunks]: maximum, sum e, sum e d
  uint32_t* gm;    // [rows, gstride]: groups' maxima
  int gstride, glog;
};

__device__ __forceinline__ float nan_f() { return __int_as_float(0x7fc00000); }

// f(0) ... f(U - 1), the numbers as types.  Not a loop: where f does nothing from some number on,
// the compiler shortens a loop before it unrolls it, and the tile becomes an array in memory.
template <int... u, typename F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, u...>, const F& f) {
  (f(std::integral_constant<int, u>{}), ...);
}
template <int U, typename F>
__device__ __forceinline__ void each(const F& f) {
  each_of(std::make_integer_sequence<int, U>{}, f);
}

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
// ... for any c, without an array in memory.
template <typename T>
__device__ __forceinline__ float get_at(const u32x4& x, int c) {
  const int d = sizeof(T) == 4 ? c : c >> 1;
  const uint32_t lo = d & 1 ? x[1] : x[0], hi = d & 1 ? x[3] : x[2], v = d & 2 ? hi : lo;
  if constexpr (sizeof(T) == 4) return __uint_as_float(v);
  else return c & 1 ? bf16_hi(v) : bf16_lo(v);
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
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <typename T>
__device__ __forceinline__ u32x4 packed(const float (&v)[kE<T>]) {
  u32x4 x;
  each<4>([&](auto c) __attribute__((always_inline)) {
    if constexpr (sizeof(T) == 4) x[c.value] = __float_as_uint(v[c]);
    else x[c.value] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v[2 * c], v[2 * c + 1]}), bf16x2));
  });
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

// The row up to slot `end`, for a tile of it.
__device__ __forceinline__ Row until(Row w, int end) {
  w.f1 = min(w.f1, end);
  w.slots = min(w.slots, end);
  return w;
}

template <typename T>
__device__ __forceinline__ const T* elem_at(const Row& w, int i) {
  return reinterpret_cast<const T*>(w.base) + w.o + i;
}

// One slot, any of whose elements may be outside the row (-infinity there).  Its elements
// are loaded whether inside or not, at the nearest place that is, so that their loads do
// not wait for each other.
template <typename T>
__device__ __forceinline__ u32x4 load_edge(const Row& w, int s) {
  if (s >= w.f0 && s < w.f1) return load_stream16(w.base + (int64_t)s * 16);
  uint32_t v[kE<T>];
  each<kE<T>>([&](auto c) __attribute__((always_inline)) {
    const T* p = elem_at<T>(w, min(max(s * kE<T> + c - w.o, 0), w.V - 1));
    if constexpr (sizeof(T) == 4) v[c] = __float_as_uint(load1(p));
    else v[c] = *gptr<uint16_t>(p);
  });
  u32x4 x;
  each<4>([&](auto c) __attribute__((always_inline)) {
    if constexpr (sizeof(T) == 4) x[c.value] = v[c];
    else x[c.value] = v[2 * c] | v[2 * c + 1] << 16;
  });
  each<kE<T>>([&](auto c) __attribute__((always_inline)) {
    const int i = s * kE<T> + c - w.o;
    if (i < 0 || i >= w.V) drop<T>(x, c);
  });
  return x;
}

// The slots slot0 + u * NTH + thread of a row, u < m in x; slot u = m, in `last`, where the row
// ends inside a slot: it is loaded by the element, once the others are taken.
template <int NTH, int U>
struct Tile {
  u32x4 x[U];
  u32x4 last;
  int slot0, m;
  bool ragged;

  __device__ __forceinline__ int slot(int u) const { return slot0 + u * NTH + threadIdx.x; }
};

// Slots are loaded and taken in batches of kRun, kAhead batches ahead of what is taken.  A wave issues
// its instructions in order: with all of a long tile's loads before its first term, or many
// batches ahead, the terms wait until the memory has room for those loads.  us, loss and
// gradient of 1024 fp32 rows of 102400 (50 slots): all loads first 188; batches of four, 6
// ahead 192, 2 ahead 182, 1 ahead 176; batches of eight, 1 ahead 176.
constexpr int kRun = 8, kAhead = 1;

// Batch b's loads.  Every thread loads every slot, without a branch, so that the wait for one
// does not wait for those after it; a slot that is not a whole one of the row is read at
// the nearest that is and replaced when it is taken (tile_sums) or not stored.
template <int b, int NTH, int U>
__device__ __forceinline__ void load_batch(Tile<NTH, U>& x, const Row& w) {
  if (w.f0 < w.f1)
    each<kRun>([&](auto i) __attribute__((always_inline)) {
      constexpr int u = b * kRun + i;
      if constexpr (u < U) x.x[u] = load_stream16(w.base + (uint32_t)min(max(x.slot(u), w.f0), w.f1 - 1) * 16u);
    });
}

// The first kAhead batches; the others are loaded by tile_sums.
template <typename T, int NTH, int U>
__device__ __forceinline__ void load_tile(Tile<NTH, U>& x, const Row& w, int slot0) {
  x.slot0 = slot0;
  x.ragged = w.f1 < w.slots && w.slots > slot0;
  x.m = (w.slots - slot0 + NTH - 1) / NTH - x.ragged;
  each<kAhead>([&](auto b) __attribute__((always_inline)) { load_batch<b>(x, w); });
}
// The row's first slot where the row starts inside it.
template <typename T, int NTH, int U>
__device__ __forceinline__ void load_first(Tile<NTH, U>& x, const Row& w) {
  if (x.m > 0 && x.slot0 < w.f0) {
    x.x[0] = load_edge<T>(w, x.slot(0));
    // Waited for here: a load that only some rows have in flight would make all of them wait
    // for everything at their first slot.
    asm volatile("" : "+v"(x.x[0]));
  }
}
template <typename T, int NTH, int U>
__device__ __forceinline__ void load_last(Tile<NTH, U>& x, const Row& w) {
  if (!x.ragged) return;
  x.last = all_dropped<T>();
  if (x.slot(x.m) < w.slots) x.last = load_edge<T>(w, x.slot(x.m));
}

// f(slot, u) for every slot of a thread.
template <int NTH, int U, typename F>
__device__ __forceinline__ void each_slot(Tile<NTH, U>& x, const F& f) {
  each<U>([&](auto u) __attribute__((always_inline)) {
    if (u < x.m) f(x.x[u], (int)u);
  });
  if (x.ragged) f(x.last, x.m);
}

// Writes a slot of results to the row `out`, whose slots are those of w (same offset) or not: then
// by the element, at twice the time (us, gradients of 2048 bf16 rows of 65537 in padded logits,
// padded alike and packed: token scores 106 and 213, distillation 113 and 227).
template <typename T>
__device__ __forceinline__ void store_slot(const Row& w, const Row& out, int s, const float (&v)[kE<T>]) {
  if (out.o == w.o && s >= w.f0 && s < w.f1) {
    // Past the caches: kept there, a large gradient pushes out the logits still to be read (us,
    // gradients of 1024 fp32 rows of 102400 175 and 166, of 2048 bf16 rows 173 and 167).
    __builtin_nontemporal_store(packed<T>(v), (DE_GLOBAL u32x4*)(out.base + (int64_t)s * 16));
    return;
  }
  each<kE<T>>([&](auto c) __attribute__((always_inline)) {
    const int i = s * kE<T> + c - w.o;
    if (i >= 0 && i < w.V) store1(const_cast<T*>(elem_at<T>(out, i)), v[c]);
  });
}

// Zeros to a row from slot0 on.
template <typename T, int NTH>
__device__ __forceinline__ void zero_tile(const Row& w, const Row& out, int slot0) {
  const float v[kE<T>] = {};
#pragma unroll 1
  for (int s = slot0 + threadIdx.x; s < w.slots; s += NTH) store_slot<T>(w, out, s, v);
}

// log2 of exp((l - top) / tau).  Differences are taken before they are scaled, so that logits
// far from zero, up to the type's lowest value, lose nothing.
__device__ __forceinline__ float scaled(const VocabRows& x, float l, float top) { return (l - top) * x.c; }
// ... not below a value whose power of two is 0 in fp32, and whose product with 0 is 0: also
// for -infinity, a NaN and an infinity's difference to itself.
__device__ __forceinline__ float scaled_floor(const VocabRows& x, float l, float top) {
  return fmaxf(scaled(x, l, top), -1000.f);
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
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t b = (uint32_t)(k >> 32);
  return __uint_as_float(b ^ (b >> 31 ? 0x80000000u : 0xffffffffu));
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

template <int ctrl, int rows>
__device__ __forceinline__ double dpp_add(double v) {  // lanes that take nothing add 0
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, ctrl, rows, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), ctrl, rows, 0xF, false);
  return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double read_lane(double v, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum64(double v) {
  v = dpp_add<0xB1, 0xF>(v);
  v = dpp_add<0x4E, 0xF>(v);
  v = dpp_add<0x141, 0xF>(v);
  v = dpp_add<0x140, 0xF>(v);
  v = dpp_add<0x142, 0xA>(v);
  v = dpp_add<0x143, 0xC>(v);
  return read_lane(v, 63);
}

// ---------------------------------------------------------------- sums over a tile

// Running sums of a part of a row: its maximum (a NaN left out) and, relative to it, sum e and
// sum e d (d in log2).  Without any logit above -infinity the differences are to 0.
struct Part {
  float top, s, w;
};

__device__ __forceinline__ float finite_top(float top) { return top == -INFINITY ? 0.f : top; }

// p relative to `top`, at least its own.
__device__ __forceinline__ Part rebased(const VocabRows& x, const Part& p, float top) {
  const float d = scaled_floor(x, p.top, finite_top(top)), e = exp2_fast(d);
  return Part{top, p.s * e, fmaf(p.s, d, p.w) * e};
}

// A thread's slots in batches, each as its loads arrive: waiting for all of them and the
// row's maximum first left the memory idle while the terms were computed.  `fix` may
// change a slot before it is taken.  With `nan` a NaN makes the sum one, else it counts
// as -infinity.
template <typename T, bool nan, int NTH, int U, typename F, typename P>
__device__ __forceinline__ Part tile_sums(const VocabRows& a, Tile<NTH, U>& x, const Row& w, const F& fix, const P& peak) {
  Part p{-INFINITY, 0.f, 0.f};
  const auto rise = [&](float& top, const u32x4& s, int u) __attribute__((always_inline)) {
    // A signalling NaN is quieted first: a maximum with one is a NaN, and the logits before it
    // are lost.  Where a NaN's sum shows it, that does not matter.
    float v = -INFINITY;
    each<kE<T>>([&](auto c) __attribute__((always_inline)) {
      v = fmaxf(v, nan ? get<T>(s, c) : __builtin_canonicalizef(get<T>(s, c)));
    });
    top = fmaxf(top, v);
    peak(v, u);
  };
  const auto add = [&](const u32x4& s) __attribute__((always_inline)) {
    const float t = finite_top(p.top);
    each<kE<T>>([&](auto c) __attribute__((always_inline)) {
      const float l = get<T>(s, c), d = scaled_floor(a, l, t), e = exp2_fast(nan ? scaled(a, l, t) : d);
      p.s += e;
      p.w = fmaf(e, d, p.w);
    });
  };
  each<(U + kRun - 1) / kRun>([&](auto b) __attribute__((always_inline)) {
    constexpr int u0 = b * kRun, k = U - u0 < kRun ? U - u0 : kRun;
    load_batch<b + kAhead>(x, w);
    if constexpr (u0 == 0) load_first<T>(x, w);
    if (u0 >= x.m) return;
    float top = p.top;
    each<k>([&](auto i) __attribute__((always_inline)) {
      if (u0 + i >= x.m) return;
      if (x.slot0 + (u0 + i + 1) * NTH > w.f1 && x.slot(u0 + i) >= w.slots) x.x[u0 + i] = all_dropped<T>();
      fix(x.x[u0 + i], u0 + i);
      rise(top, x.x[u0 + i], u0 + i);
    });
    p = rebased(a, p, top);
    each<k>([&](auto i) __attribute__((always_inline)) {
      if (u0 + i < x.m) add(x.x[u0 + i]);
    });
  });
  if (x.ragged) {
    load_last<T>(x, w);
    fix(x.last, x.m);
    float top = p.top;
    rise(top, x.last, x.m);
    p = rebased(a, p, top);
    add(x.last);
  }
  return p;
}
struct NoFix {
  __device__ __forceinline__ void operator()(u32x4&, int) const {}
};
struct NoPeak {
  __device__ __forceinline__ void operator()(float, int) const {}
};

// The parts of a block's threads as one.
template <int NTH>
__device__ __forceinline__ Part block_part(const VocabRows& a, Part p, float (*red)[NTH / 64]) {
  const float top = block_max<NTH>(p.top, red[0]);
  p = rebased(a, p, top);
  p.s = block_sum<NTH>(p.s, red[1]);
  p.w = block_sum<NTH>(p.w, red[2]);
  return p;
}

// The maxima of groups of 2^glog slots (0, 2 or 4) as whole numbers in their order, from a
// slot's v (no NaN): the best m logits lie in the m groups whose (maximum, lower index) are
// best, so that only those are looked at again.  All lanes of a wave.
template <int ctrl>
__device__ __forceinline__ uint32_t dpp_umax(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xF, 0xF, false));
}
__device__ __forceinline__ void group_max(float v, int s, const Row& w, int glog, uint32_t* gm) {
  const uint32_t b = __float_as_uint(v + 0.f);
  uint32_t k = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  if (glog > 0) {
    k = dpp_umax<0xB1>(k);
    k = dpp_umax<0x4E>(k);
  }
  if (glog == 4) {
    k = dpp_umax<0x141>(k);
    k = dpp_umax<0x140>(k);
  }
  if ((threadIdx.x & ((1 << glog) - 1)) == 0 && s < w.slots) gm[s >> glog] = k;
}

// Marks of a tile's list entries: a bit for each logit, and for each wave a bit for each of
// its slots that has one, so that the others cost a scalar test.
template <typename T, int NTH, int U>
struct Marks {
  static constexpr int kWords = (U + 1) * NTH * kE<T> / 32, kFlags = (U + 32) / 32;  // with Tile::last
  uint32_t bits[kWords];
  uint32_t slots[NTH / 64][kFlags];
};

template <typename T, int NTH, int U>
__device__ __forceinline__ void clear_marks(Marks<T, NTH, U>& k) {
  for (int i = threadIdx.x; i < k.kWords; i += NTH) k.bits[i] = 0;
  if (threadIdx.x < NTH / 64)
    for (int i = 0; i < k.kFlags; ++i) k.slots[threadIdx.x][i] = 0;
}
template <typename T, int NTH, int U>
__device__ __forceinline__ void set_mark(Marks<T, NTH, U>& k, const Row& w, int slot0, int id) {
  if (id < 0 || id >= w.V) return;
  const int64_t e = (int64_t)id + w.o - (int64_t)slot0 * kE<T>;
  if (e < 0 || e >= (int64_t)k.kWords * 32) return;
  const int i = (int)e, s = i / kE<T>, u = s / NTH, wave = s % NTH / 64;
  atomicOr(&k.bits[i >> 5], 1u << (i & 31));
  atomicOr(&k.slots[wave][u >> 5], 1u << (u & 31));
}
template <typename T, int NTH, int U>
__device__ __forceinline__ void drop_marked(u32x4& x, int u, const Marks<T, NTH, U>& k) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (!(__builtin_amdgcn_readfirstlane(k.slots[wave][u >> 5]) >> (u & 31) & 1)) return;
  const int i = (u * NTH + threadIdx.x) * kE<T>;
  const uint32_t b = k.bits[i >> 5] >> (i & 31);
  const auto all = [&](int at) { return (uint32_t)((int32_t)(b << (31 - at)) >> 31); };  // a bit in every place
  each<4>([&](auto c) __attribute__((always_inline)) {
    const uint32_t mask = sizeof(T) == 4 ? all(c) : (all(2 * c) & 0xffffu) | all(2 * c + 1) << 16;
    x[c.value] = (x[c.value] & ~mask) | (all_dropped<T>()[0] & mask);
  });
}

// ---------------------------------------------------------------- host side

// Slots of a row that starts at any element, and of the longest of these rows.
template <typename T>
inline int slots_most(int V) {
  return (V + 2 * (kE<T> - 1)) / kE<T>;
}
template <typename T>
inline bool at_slots(const VocabRows& x) {  // every row starts with a whole slot
  return (reinterpret_cast<uintptr_t>(x.logits) & 15u) == 0 && x.ld % kE<T> == 0;
}
template <typename T>
inline int slots_most(const VocabRows& x) {
  return at_slots<T>(x) ? (x.V + kE<T> - 1) / kE<T> : slots_most<T>(x.V);
}

// f with the smallest U that holds u slots a thread.
template <typename F>
inline void by_u(int u, const F& f) {
  if (u > 4) f(std::integral_constant<int, 8>{});
  else if (u > 2) f(std::integral_constant<int, 4>{});
  else if (u > 1) f(std::integral_constant<int, 2>{});
  else f(std::integral_constant<int, 1>{});
}

// Blocks that few rows are split into: four for each CU.
constexpr int kBlocks = 1024;

inline int group_log(int slots) { return slots <= 2048 ? 0 : slots <= 8192 ? 2 : 4; }

// Parts of kTileU slots a thread, or of fewer where that would leave CUs without one.
template <typename T>
inline Split split_of(const VocabRows& x, int m, void* ws) {
  Split sp{};
  const int rows = x.rows, slots = slots_most<T>(x), slabs = (slots + kThreads - 1) / kThreads;
  int chunks = (slabs + kTileU - 1) / kTileU;
  if (rows < kBlocks) chunks = std::max(chunks, std::min(slabs, (kBlocks + rows - 1) / rows));
  sp.nu = (slabs + chunks - 1) / chunks;
  sp.chunks = (slabs + sp.nu - 1) / sp.nu;
  sp.glog = group_log(slots);
  sp.gstride = m > 0 ? (slots >> sp.glog) + 1 : 0;
  sp.parts = static_cast<float4*>(ws);
  sp.gm = reinterpret_cast<uint32_t*>(sp.parts + (int64_t)rows * sp.chunks);
  return sp;
}

// Whole rows in one block's registers, which then write the gradient too: logits are read
// once and gradients written once.  Threads and slots a thread; at most 512 threads of 256
// registers, of which the distillation takes 250 with 50 slots (102400 fp32 logits; 52 spill).
// Token scores take 224 to 229 there and keep the same limit.
template <int NTH, int U>
struct Whole {
  static constexpr int kNth = NTH, kU = U;
};

// Whether a tile of u slots a thread holds any of the rows: a row that ends inside a slot has
// its last ones in Tile::last.
template <typename T>
inline bool holds(const VocabRows& x, int nth, int u) {
  for (int o = 0; o < (at_slots<T>(x) ? 1 : kE<T>); ++o) {
    const int64_t slots = ((int64_t)x.V + o + kE<T> - 1) / kE<T>, ragged = (x.V + o) % kE<T> != 0;
    if (slots > (int64_t)nth * (u + ragged)) return false;
  }
  return true;
}

// f with the smallest block that holds the rows; false if none does.  Pair: the most slots a
// thread with which a CU's registers hold two blocks, so that one computes while the other
// loads.
template <typename T, int Pair, typename F>
inline bool by_whole(const VocabRows& x, const F& f) {
  const auto take = [&](auto k) {
    if (!holds<T>(x, k.kNth, k.kU)) return false;
    f(k);
    return true;
  };
  return take(Whole<256, 1>{}) || take(Whole<256, 2>{}) || take(Whole<256, 4>{}) || take(Whole<256, 8>{}) ||
         take(Whole<256, 16>{}) || take(Whole<512, 16>{}) || take(Whole<512, Pair>{}) || take(Whole<512, 50>{});
}
// Waves of a SIMD that a block's registers leave room for.
constexpr int whole_waves(int nth, int u) { return u < 50 ? 4 : nth / 256; }

// Rows that a whole-row block serves better than parts (which read a gradient's logits twice, but
// put every CU on few long rows): a single tile's; with a gradient, rows short enough for one CU,
// or enough of them for all; without, where one launch saves more than the parts' finer
// grain does.  us, loss and gradient, whole and parts: 1 row of 50000 fp32 16
// and 17, 64 rows of 60000 bf16 17 and 17, of 102400 fp32 27 and 25, bf16 26 and 21, 128
// rows 28 and 37, 27 and 28, 256 rows 40 and 65, 30 and 39.
// Without a gradient, 64 rows of 50000 fp32 9.4 and 12, 256 12 and 12, 333 17 and 15: two blocks
// of 512 threads a CU.  Rows of other blocks (four of 256 threads a CU) take the same limit,
// where the crossing was not measured.
template <typename T>
inline bool whole_pays(const VocabRows& x, bool grad) {
  const int slots = slots_most<T>(x);
  if (slots <= kTileU * kThreads) return true;
  if (grad) return x.V <= 65536 || x.rows >= 100;
  return x.V <= 65536 && x.rows <= 256;
}

}  // namespace
}  // namespace de
