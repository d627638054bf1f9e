// Adjustment of logits (biases, penalties for repeated tokens, grammar masks) and the largest logits of
// each row with their log-sum-exp.
//
// An adjusted logit is fp32 and every operation that makes it is rounded by itself (no contraction), so
// that which tokens are the largest is well defined:
//   z1 = z + bias[v]
//   c  = occurrences of v in the row's history; where c > 0:
//   z1 = (z1 > 0 ? z1 / rep : z1 * rep) - (presence + frequency c)
//   z' = the row's mask allows v ? z1 : -inf
//
// Rows are read once, as the aligned 16-byte groups that cover them: a row may begin anywhere in a group
// (odd row lengths), so column c of a row is element c + a of its groups, a its first element's place in the
// first one.  The tokens of a history are counted in a hash table in shared memory (long ones by element, a few
// thousand elements at a time, the history read once for each such segment, and slow: see hashed): no sorting and no
// workspace.
//
// Measured (GB300; reading at the copy rate of 6.77 TB/s is the floor, beside the writing of the adjustment):
//   adjustment of 8192 x 50000 bf16: 259 us (floor 243, 6.3 TB/s); biases 271, masks 285, histories of 0 to 512 tokens
//     347, all three (of 0 to 1024) 448; with rows of 49999, which begin anywhere, 263, 335, 288, 348 and 472.  fp32: 505
//     (6.5 TB/s), 507, 515, 599, 675; rows of 49999 513, 516, 524, 610, 696.  In place within 9% of that, and less
//     where histories alone are asked for (bf16 130).  What histories add is scattered: a sector read and one written
//     in part for each token.
//   top 32 of 16383 x 50000 bf16: 371 us (floor 243), biases 459, masks 456, histories 526, all three 711; fp32 541
//     (6.1 TB/s; floor 485), 603, 573, 675, 875; top 1 306, top 128 678.  bf16 rows are bound by instructions and by
//     the latency of what comes one after the other in a row (issue slots 64%, fp32's unpacked rows hide it): 80
//     instructions a warp for 512 logits, 44 for the sum of exponentials, 37 for the biases, 55 for the bits.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "answer.h"
#include "kernels.h"
#include "tc_util.cuh"
#include "token.h"

namespace bg {

using tc::smem_u32;

namespace {

constexpr int kThreads = 256;     // of a block of the adjustment
constexpr int kSlots = 2048;      // of a hash table of a history's tokens, at most
constexpr int kEach = 16;         // elements of a thread at a time

// What an adjustment has (template flags): one without any costs nothing.
enum { kBias = 1, kMask = 2, kHistory = 4 };

struct Adjust {
  const float* bias;
  const uint32_t* mask;
  int words;  // of a mask
  int n_masks;
  const int32_t* mask_row;
  const int32_t* history;
  int64_t history_len;
  const int64_t* history_off;
  const float* penalty;
};

int flags_of(const bg_adjust& a) {
  return (a.bias ? kBias : 0) | (a.mask ? kMask : 0) | (a.history_off ? kHistory : 0);
}
Adjust make_adjust(const bg_adjust& a, int V) {
  return Adjust{a.bias, a.mask, (V + 31) / 32, a.n_masks, a.mask_row, a.history, a.history_len,
                a.history_off, a.penalty};
}

__device__ __forceinline__ void report(int* status, int site) {
  if (atomicCAS(status, 0, 2) == 0) atomicExch(status + 1, site);
}

// A row of logits and its part of the adjustment.
template <typename T>
struct Row {
  static constexpr int G = 16 / (int)sizeof(T);  // elements of a group
  const T* base;                                 // the group that holds column 0
  int a;                                         // column 0's place in it
  int V;
  const float* bias;
  const uint32_t* mask;  // NULL: everything is allowed
  int words;
  const int32_t* hist;
  int64_t hist_n;
  float rep, presence, frequency;
  __device__ int groups() const { return (V + a + G - 1) / G; }
};

template <typename T, int F>
__device__ __forceinline__ Row<T> make_row(const T* Z, int64_t ldz, int64_t i, int V, const Adjust& adj,
                                           int* status) {
  Row<T> r;
  const T* p = Z + i * ldz;
  r.a = (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
  r.base = p - r.a;
  r.V = V;
  r.bias = adj.bias;
  r.mask = nullptr;
  r.words = adj.words;
  r.hist = nullptr;
  r.hist_n = 0;
  if (F & kMask) {
    const int64_t m = adj.mask_row ? adj.mask_row[i] : adj.n_masks == 1 ? 0 : i;
    if (m >= adj.n_masks)
      report(status, kSiteMaskRow);
    else if (m >= 0)
      r.mask = adj.mask + m * adj.words;
  }
  if (F & kHistory) {
    const int64_t b = adj.history_off[i], e = adj.history_off[i + 1];
    if (b < 0 || e < b || e > adj.history_len) {
      report(status, kSiteHistoryOff);
    } else {
      r.hist = adj.history + b;
      r.hist_n = e - b;
    }
    r.rep = adj.penalty[3 * i];
    r.presence = adj.penalty[3 * i + 1];
    r.frequency = adj.penalty[3 * i + 2];
  }
  return r;
}

// Occurrences of the tokens of elements [first, first + segment) of a row (element = column + a).
template <int NT, typename T>
__device__ __forceinline__ void count_history(const Row<T>& r, int64_t first, int segment, uint32_t* counts,
                                              int* status) {
  __syncthreads();
  for (int i = threadIdx.x; i < segment / 4; i += NT)
    reinterpret_cast<uint4*>(counts)[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
  for (int64_t i = threadIdx.x; i < r.hist_n; i += NT) {
    const int id = r.hist[i];
    if (id >= r.V) report(status, kSiteHistoryId);
    const int64_t at = (int64_t)id + r.a - first;
    if (id >= 0 && id < r.V && at >= 0 && at < segment) atomicAdd(&counts[at], 1u);
  }
  __syncthreads();
}

__device__ __forceinline__ float penalised(float z, uint32_t count, float rep, float presence, float frequency) {
  z = z > 0.f ? __fdiv_rn(z, rep) : __fmul_rn(z, rep);
  return __fsub_rn(z, __fadd_rn(presence, __fmul_rn(frequency, (float)count)));
}

__device__ __forceinline__ void unpack(uint4 x, float* v, float) {
  v[0] = __uint_as_float(x.x);
  v[1] = __uint_as_float(x.y);
  v[2] = __uint_as_float(x.z);
  v[3] = __uint_as_float(x.w);
}
__device__ __forceinline__ void unpack(uint4 x, float* v, __nv_bfloat16) {
  const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(u[j] << 16);
    v[2 * j + 1] = __uint_as_float(u[j] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }

// The logits of group g (G of them) as they are; -inf past the row's ends.
template <typename T>
__device__ __forceinline__ void load_group(const Row<T>& r, int64_t g, float* v) {
  constexpr int G = Row<T>::G;
  const int64_t c0 = g * G - r.a;
  if (c0 >= 0 && c0 + G <= r.V) {
    unpack(__ldcs(reinterpret_cast<const uint4*>(r.base + g * G)), v, T());
  } else {
#pragma unroll
    for (int j = 0; j < G; ++j) v[j] = c0 + j >= 0 && c0 + j < r.V ? to_f32(r.base[g * G + j]) : -INFINITY;
  }
}

// Adjusts group g in place; counts: the occurrences of its elements.
template <typename T, int F>
__device__ __forceinline__ void adjust_group(const Row<T>& r, int64_t g, const uint32_t* counts, float* v) {
  constexpr int G = Row<T>::G;
  const int c0 = (int)(g * G - r.a);
  if (F & kBias) {
    if (r.a == 0 && c0 + G <= r.V) {
#pragma unroll
      for (int j = 0; j < G; j += 4) {
        const float4 b = __ldg(reinterpret_cast<const float4*>(r.bias + c0 + j));
        v[j] = __fadd_rn(v[j], b.x);
        v[j + 1] = __fadd_rn(v[j + 1], b.y);
        v[j + 2] = __fadd_rn(v[j + 2], b.z);
        v[j + 3] = __fadd_rn(v[j + 3], b.w);
      }
    } else if (c0 >= 0 && c0 + G <= r.V) {
#pragma unroll
      for (int j = 0; j < G; ++j) v[j] = __fadd_rn(v[j], __ldg(r.bias + c0 + j));
    } else {
#pragma unroll
      for (int j = 0; j < G; ++j)
        if (c0 + j >= 0 && c0 + j < r.V) v[j] = __fadd_rn(v[j], __ldg(r.bias + c0 + j));
    }
  }
  if ((F & kHistory) && r.hist_n > 0) {
#pragma unroll
    for (int k = 0; k < G; k += 4) {
      const uint4 c = *reinterpret_cast<const uint4*>(counts + k);
      if (c.x | c.y | c.z | c.w) {
        const uint32_t u[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (u[j]) v[k + j] = penalised(v[k + j], u[j], r.rep, r.presence, r.frequency);
      }
    }
  }
  if ((F & kMask) && r.mask) {
    // (c0 may lie up to G - 1 columns before the row)
    const int w = c0 >> 5, s = c0 & 31;
    const uint32_t lo = w >= 0 && w < r.words ? __ldg(r.mask + w) : 0u;
    const uint32_t hi = s > 32 - G && w + 1 < r.words ? __ldg(r.mask + w + 1) : 0u;
    const uint32_t bits = __funnelshift_r(lo, hi, s);
#pragma unroll
    for (int j = 0; j < G; ++j)
      if (!(bits >> j & 1u)) v[j] = -INFINITY;
  }
}

// A hash table of a history's tokens and their counts in shared memory: a slot holds a token plus
// one in its low `low` bits and its count above.  Only the part that the history needs is used: a small one is
// cleared and looked through quickly.
struct Hash {
  uint32_t* slot;
  int size;  // a power of two
  int low;
  __device__ int token(uint32_t x) const { return (int)(x & ((1u << low) - 1)) - 1; }
  __device__ uint32_t count(uint32_t x) const { return x >> low; }
};
// Whether a history goes there: it leaves a quarter of the slots free, and its length fits beside a token.  Longer
// ones are counted, as many elements at a time as there are slots.  That is the slow way: top 32 of 16383 x 49999 bf16
// with 1536 tokens a row 1110 us, with 1537 4920, with 4096 7060 (adjustment in place 580, 1250, 2070); one row of 2000
// among rows of 256 740 (572 without it); 300 rows of 1536 45 us, of 1537 270; one row of 256 19 us, of 4096 83.
template <typename R>
__device__ __forceinline__ bool hashed(const R& r, int slots) {
  return r.hist_n <= slots / 4 * 3 && r.V < 1 << 21;
}

// A token's place: a slot keeps the largest of the tokens that come to it and sends the smaller one on to the next.
// So where each ends up depends on which tokens there are and not on which came first, and with it the order in which
// their exponentials are added.  (By the order of arrival, lse differed in its last bits from run to run.)
__device__ __forceinline__ uint32_t hash_home(const Hash& h, uint32_t id) {
  return (id * 2654435761u) >> 7 & (h.size - 1);
}
__device__ __forceinline__ void hash_insert(const Hash& h, uint32_t id) {
  uint32_t at = hash_home(h, id), key = id + 1;
  for (int k = 0; k < h.size; ++k, at = (at + 1) & (h.size - 1)) {  // (a quarter of the slots stays empty)
    const uint32_t was = atomicMax(&h.slot[at], key);
    if (was == 0 || was == key) return;
    key = min(key, was);
  }
}
// One more of a token that is there; all are, behind a barrier.
__device__ __forceinline__ void hash_count(const Hash& h, uint32_t id) {
  const uint32_t mask = (1u << h.low) - 1;
  uint32_t at = hash_home(h, id);
  for (int k = 0; k < h.size; ++k, at = (at + 1) & (h.size - 1))
    if ((h.slot[at] & mask) == id + 1) {
      atomicAdd(&h.slot[at], 1u << h.low);
      return;
    }
}

// An empty table for the tokens of r's history (a barrier has to follow before it is filled).
template <int NT, typename T>
__device__ __forceinline__ Hash clear_hash(const Row<T>& r, uint32_t* table, int slots) {
  Hash h{table, 64, 32 - __clz(r.V)};  // (tokens plus one: 1 .. V)
  while (h.size < 2 * r.hist_n && h.size < slots) h.size *= 2;
  for (int i = threadIdx.x; i < h.size / 4; i += NT) reinterpret_cast<uint4*>(table)[i] = make_uint4(0, 0, 0, 0);
  return h;
}
// Adds the tokens whose elements (column + a) are in [first, last), calling seen(element) for each; the whole block
// calls it (a barrier has to follow before the table is read).  Two passes over the history, the second from the L1
// cache: counts can be added once no token moves any more.  U tokens of a thread are on their way in the first: one
// for the largest logits, whose kernel is bound by its code's length (top 32 of 16383 x 49999 bf16, all constraints
// and up to 512 tokens: 754 us, 773 with four), four for the adjustment (8192 x 49999 bf16, all constraints and up to
// 1024 tokens: 477 us, 493 with one).
template <int NT, int U, typename T, typename Fn>
__device__ __forceinline__ void fill_hash(const Hash& h, const Row<T>& r, int64_t first, int64_t last, int* status,
                                          Fn seen) {
  const int n = (int)r.hist_n;
  const uint32_t lo = (uint32_t)max((int64_t)0, first - r.a);
  const uint32_t span = (uint32_t)min((int64_t)r.V, last - r.a) - lo;
#pragma unroll 1
  for (int i0 = threadIdx.x; i0 < n; i0 += U * NT) {
    int id[U];
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = u == 0 || i0 + u * NT < n ? r.hist[i0 + u * NT] : -1;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (id[u] >= r.V) report(status, kSiteHistoryId);
      if ((uint32_t)id[u] - lo < span) {
        hash_insert(h, (uint32_t)id[u]);
        seen(id[u] + r.a);
      }
    }
  }
  __syncthreads();
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += NT) {
    const int id = r.hist[i];
    if ((uint32_t)id - lo < span) hash_count(h, (uint32_t)id);
  }
}

// ------------------------------------------------------------------------------ adjustment
__device__ __forceinline__ void store_group(float* p, const float* v) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
}
__device__ __forceinline__ void store_group(__nv_bfloat16* p, const float* v) {
  __nv_bfloat162 h[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
  __stcs(reinterpret_cast<uint4*>(p), *reinterpret_cast<const uint4*>(h));
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

template <typename T>
__device__ __forceinline__ void store_row_group(const Row<T>& r, T* o, bool vec, int64_t g, const float* v) {
  constexpr int G = Row<T>::G;
  const int64_t c0 = g * G - r.a;
  if (vec && c0 >= 0 && c0 + G <= r.V) {
    store_group(o + c0, v);
  } else {
#pragma unroll
    for (int j = 0; j < G; ++j)
      if (c0 + j >= 0 && c0 + j < r.V) store1(o + c0 + j, v[j]);
  }
}

// A row's groups [g0, g1).  Biases and masks are one pass over the elements (not where `tokens`: another launch has
// done that); the tokens of the history come after it, from a hash table, their logits read before it (out may be
// Z).  staged: the biases of the groups' elements, NULL: they are read where they lie.
template <typename T, int F>
__device__ __forceinline__ void adjust_run(const Row<T>& r, T* o, bool in_place, bool tokens, int64_t g0, int64_t g1,
                                           const float* staged, uint32_t* table, float* raw, int* status) {
  constexpr int G = Row<T>::G;
  // (rows of out at another place in 16 bytes than Z's are stored one by one: 8192 x 49999 into rows of 50000, bf16 970 us
  // instead of 268, fp32 534 instead of 518)
  const bool vec = (reinterpret_cast<uintptr_t>(o - r.a) & 15) == 0;
  // (short runs, of a few rows: occurrences by element are the shorter way)
  constexpr int SG = kSlots / G;
  if ((F & kHistory) && r.hist_n > 0 && (!hashed(r, kSlots) || (!tokens && g1 - g0 <= SG))) {
    for (int64_t s0 = g0; s0 < g1; s0 += SG) {
      count_history<kThreads>(r, s0 * G, kSlots, table, status);
      for (int64_t g = s0 + threadIdx.x; g < min(g1, s0 + SG); g += kThreads) {
        float v[G];
        load_group(r, g, v);
        adjust_group<T, F>(r, g, table + (g - s0) * G, v);
        store_row_group(r, o, vec, g, v);
      }
    }
    return;
  }
  Hash h{table, 0, 0};
  if ((F & kHistory) && r.hist_n > 0) {
    h = clear_hash<kThreads>(r, table, kSlots);
    __syncthreads();
    fill_hash<kThreads, 4>(h, r, g0 * G, g1 * G, status, [](int64_t) {});
    __syncthreads();
    for (int k = threadIdx.x; k < h.size; k += kThreads)
      if (const uint32_t x = h.slot[k]) raw[k] = to_f32(r.base[h.token(x) + r.a]);
    if (in_place) __syncthreads();
  }
  if (!tokens && ((F & (kBias | kMask)) || !in_place)) {
    auto finish = [&](int64_t g, float* v) {
      if ((F & kBias) && staged) {
#pragma unroll
        for (int j = 0; j < G; j += 4) {
          const float4 b = *reinterpret_cast<const float4*>(staged + (g - g0) * G + j);
          v[j] = __fadd_rn(v[j], b.x);
          v[j + 1] = __fadd_rn(v[j + 1], b.y);
          v[j + 2] = __fadd_rn(v[j + 2], b.z);
          v[j + 3] = __fadd_rn(v[j + 3], b.w);
        }
        adjust_group<T, F & kMask>(r, g, nullptr, v);
      } else {
        adjust_group<T, F & ~kHistory>(r, g, nullptr, v);
      }
      store_row_group(r, o, vec, g, v);
    };
    for (int64_t g = g0 + threadIdx.x; g < g1; g += kThreads) {
      float v[G];
      load_group(r, g, v);
      finish(g, v);
    }
  }
  if ((F & kHistory) && r.hist_n > 0) {
    __syncthreads();
    for (int k = threadIdx.x; k < h.size; k += kThreads) {
      const uint32_t x = h.slot[k];
      if (!x) continue;
      const int id = h.token(x);
      float v = raw[k];
      if (F & kBias) v = __fadd_rn(v, __ldg(r.bias + id));
      v = penalised(v, h.count(x), r.rep, r.presence, r.frequency);
      if ((F & kMask) && r.mask && !(__ldg(r.mask + (id >> 5)) >> (id & 31) & 1u)) v = -INFINITY;
      store1(o + id, v);
    }
  }
}

// Block (row, run of `per` groups).
template <typename T, int F>
__global__ void __launch_bounds__(kThreads)
    k_adjust(int V, int64_t ldz, const T* Z, Adjust adj, int64_t ldo, T* out, int per, int tokens, int* status) {
  __shared__ __align__(16) uint32_t table[F & kHistory ? kSlots : 4];
  __shared__ float raw[F & kHistory ? kSlots : 1];
  tc::grid_dep_launch();
  tc::grid_dep_wait();
  const int64_t i = blockIdx.x;
  const Row<T> r = make_row<T, F>(Z, ldz, i, V, adj, status);
  const int64_t g0 = (int64_t)blockIdx.y * per, g1 = min((int64_t)r.groups(), g0 + per);
  if (g0 >= g1) return;
  adjust_run<T, F>(r, out + i * ldo, out == Z, tokens, g0, g1, nullptr, table, raw, status);
}

// The same with biases where rows begin anywhere in 16 bytes: rows `step` apart begin at the same place, and kShare of
// them share a run of kRun biases, laid out in shared memory as their groups lie.  (Read one by one, a warp's biases
// are 16 bytes apart, 32 in bf16.)  Laying them out is worth it for many long bf16 rows at odd places alone: see
// shares_biases.
constexpr int kRun = 8192, kShare = 8;
template <typename T, int F>
__global__ void __launch_bounds__(kThreads)
    k_adjust_shared(int64_t n, int V, int64_t ldz, const T* Z, Adjust adj, int64_t ldo, T* out, int step, int* status) {
  constexpr int G = Row<T>::G, per = kRun / G;
  extern __shared__ __align__(16) uint8_t adjust_smem[];
  float* staged = reinterpret_cast<float*>(adjust_smem);
  tc::grid_dep_launch();
  tc::grid_dep_wait();
  const int64_t first = (int64_t)(blockIdx.x / step) * step * kShare + blockIdx.x % step;
  const int64_t g0 = (int64_t)blockIdx.y * per;
  // (what a row's own part of the adjustment is comes while the row before it is worked on)
  Row<T> next = make_row<T, F>(Z, ldz, min(first, n - 1), V, adj, status);
  for (int k = 0; k < kShare; ++k) {
    const int64_t i = first + (int64_t)k * step;
    if (i >= n) break;
    const Row<T> r = next;
    if (k + 1 < kShare && i + step < n) next = make_row<T, F>(Z, ldz, i + step, V, adj, status);
    const int64_t g1 = min((int64_t)r.groups(), g0 + per);
    if (g0 >= g1) break;
    if (k == 0) {
      const int c0 = (int)(g0 * G) - r.a;
#pragma unroll 8
      for (int e = threadIdx.x; e < kRun; e += kThreads) {
        const int c = c0 + e;
        staged[e] = c >= 0 && c < V ? __ldg(adj.bias + c) : 0.f;
      }
    }
    if (k == 0) __syncthreads();
    adjust_run<T, F>(r, out + i * ldo, out == Z, false, g0, g1, staged, nullptr, nullptr, status);
  }
}

// ------------------------------------------------------------------------------ largest logits
// One pass over a row notes which lanes' pieces of it (16 logits) may hold answers: those whose largest reaches a
// bound that at least K of the row's logits are known to reach, each warp's ceil(K / 4)-th largest of its
// lanes' maxima so far, the least over the warps.  The bound rises after 1, 2, 4, ... chunks; warps read each
// other's parts of it as they find them (an old part is a lower bound too), so that there is one barrier, after
// the first chunk.  Then the pieces noted, some 150 of 3100 for 49999 logits and K = 32, are read again, and their
// logits that reach the last bound, some 60, become candidates.  (Candidates taken as they were met, by the bound
// of the time, were a third of the kernel's instructions.)  Where pieces or candidates outgrow their room (ties
// without end, rows that rise), the block goes over the row again with exact bounds (rising_row, four to ten times
// slower).
//
// A block is a row's, of 128 threads where there are rows enough, eight blocks an SM: what one waits for (the
// history's offsets, its tokens, their logits; barriers) is hidden by the others (top 32 of 16383 x 50000 bf16 425 us
// with four blocks of 256 threads, 370 with eight of 128).  With few rows it has 512, and up to eight blocks of a
// cluster share a row, whose lists the first one joins.
//
// Masks and histories come as bits in shared memory, kBits elements at a time: a cleared bit leaves an element
// out.  The tokens of a history are cleared too, counted in a hash table, and added one by one after the
// others: c > 0 for a few hundred of 50000 tokens costs no element a test of its own.
constexpr int kBits = 65536;  // elements whose bits are in shared memory at a time
constexpr int kPass = 64;     // groups of a pass of rising_row
constexpr int kRoom = kPass * 8 + kMaxTop;  // candidates: those of a pass and the K before it
constexpr int kMaxCluster = 8;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNoLogit = -3.0e38f;  // reference of a sum without terms
constexpr float kLeast = -3.402823466e38f;

// What a block of NT threads has in shared memory, and after it, at the places of Room: the best candidates, a
// block's answers (in a cluster), the notes, the bits and the hash table.  The less there is of it, the more is left
// to the L1 cache, through which the logits and the biases come (with 26 KB a block, eight blocks an SM, fp32 rows
// take a quarter longer than with 15).
template <int NT>
struct TopShared {
  static constexpr int W = NT / 32;
  float m[W], l[W];
  float block_m, block_l;
  alignas(16) uint32_t part[W];  // of the bound, as orders
  int count, found, over, sum[64];  // over: pieces or candidates outgrew their room
  uint64_t* few;
  uint2* cand;  // rising_row's candidates: in the place of the notes and the bits, once those are done with
  int most;     // of few
};
struct Room {
  int few, notes, slots;                         // candidates, pieces a warp notes, slots
  int at_few, at_best, at_note, at_bits, at_table;  // in bytes
  int bytes;
};
template <int NT>
Room room_of(int flags, int V, int K, int64_t n, int64_t history_len, bool cluster) {
  Room r{};
  r.few = K <= 32 ? 256 : 512;
  r.notes = K <= 64 ? 128 : 256;
  // room for three histories of the average length
  r.slots = flags & kHistory ? 1024 : 0;
  while (r.slots && r.slots < kSlots && r.slots < 4 * history_len / std::max<int64_t>(n, 1)) r.slots *= 2;
  int at = ((int)sizeof(TopShared<NT>) + 15) / 16 * 16;
  auto take = [&](int bytes) {
    const int here = at;
    at += (bytes + 15) / 16 * 16;
    return here;
  };
  r.at_few = take(r.few * 8);
  r.at_best = take(cluster ? kMaxTop * 8 : 0);
  r.at_note = take(NT / 32 * r.notes * 4);
  // (whole chunks of the row)
  r.at_bits = take(flags & (kMask | kHistory) ? std::min(kBits, (V + 8 + NT * kEach - 1) / (NT * kEach) * NT * kEach) / 8 : 0);
  // (a cluster's lists come where the notes were)
  at = std::max(at, r.at_note + std::max(kRoom * 8, cluster ? kMaxCluster * kMaxTop * 8 : 0));
  r.at_table = take(r.slots * 4);
  r.bytes = at;
  return r;
}
// Order of logits as unsigned numbers (-0 counts as 0), and keys: the larger logit, then the lower token.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ ((int32_t)b < 0 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint64_t key_of(float v, int id) {
  return (uint64_t)order_of(v) << 32 | (uint32_t)~id;
}
// A candidate: a logit and its token (its key is made where it is wanted, of few of them).
__device__ __forceinline__ uint2 candidate(float v, int id) { return make_uint2(__float_as_uint(v), (uint32_t)id); }
__device__ __forceinline__ uint64_t key_of(uint2 c) { return key_of(__uint_as_float(c.x), (int)c.y); }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// two fp32 at a time
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t x, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// log of the sum l to the reference m (in base 2).  A sum of 0 with a reference: every term vanished beside
// the rounding of the reference, which then is the result to the last bit.
__device__ __forceinline__ float lse_of(float m, float l) {
  return (l == 0.f && m > kNoLogit ? m : m + log2f(l)) * 0.6931471805599453f;
}

// A thread's sum of exp2(c z) to the reference m, near the largest so far.
struct Sum {
  float m = kNoLogit, l = 0.f;
  // (rounded up: of logits beyond 2^31 the terms may vanish but not overflow)
  __device__ __forceinline__ void refer(float most) {
    const float mc = __fmul_ru(most, kLog2e);
    if (mc > m) {
      l *= ex2(m - mc);
      m = mc;
    }
  }
  template <int N>
  __device__ __forceinline__ void add(const float* v, float most) {
    refer(most);
    const uint64_t c2 = pack2(kLog2e, kLog2e), m2 = pack2(-m, -m);
    uint64_t s[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      float a, b;
      unpack2(fma2(pack2(v[j], v[j + 1]), c2, m2), a, b);
      s[(j >> 1) & 1] = add2(s[(j >> 1) & 1], pack2(ex2(a), ex2(b)));
    }
    float a, b;
    unpack2(add2(s[0], s[1]), a, b);
    l += a + b;
  }
};

template <int N>
__device__ __forceinline__ float max_of(const float* v) {
  static_assert(N % 4 == 0, "");
  float a = v[0], b = v[1];
#pragma unroll
  for (int j = 2; j < N - 2; j += 4) {
    a = max3(a, v[j], v[j + 1]);
    b = max3(b, v[j + 2], v[j + 3]);
  }
  return max3(fmaxf(a, b), v[N - 2], v[N - 1]);
}

// The K-th largest candidate's key (0 where there are fewer), a bit at a time; the whole block calls it.
template <int NT>
__device__ __noinline__ uint64_t kth_key(TopShared<NT>& s, int K) {
  __syncthreads();
  const int n = s.count;
  if (n < K) return 0;
  if (threadIdx.x < 64) s.sum[threadIdx.x] = 0;
  __syncthreads();
  uint64_t t = 0;
  for (int bit = 63; bit >= 0; --bit) {
    const uint64_t trial = t | (uint64_t)1 << bit;
    int c = 0;
    for (int i = threadIdx.x; i < n; i += NT) c += key_of(s.cand[i]) >= trial;
    c = __reduce_add_sync(0xffffffffu, c);
    if ((threadIdx.x & 31) == 0 && c) atomicAdd(&s.sum[bit], c);
    __syncthreads();
    if (s.sum[bit] >= K) t = trial;
  }
  return t;
}

// The candidates with keys of t or more to `few` (as many of them as it holds); the whole block calls it, with the
// candidates complete and `found` 0 behind a barrier.  Their number.
template <int NT>
__device__ __forceinline__ int pick(TopShared<NT>& s, uint64_t t) {
  const int n = s.count;
  for (int i = threadIdx.x; i < n; i += NT) {
    const uint64_t key = key_of(s.cand[i]);
    if (key >= t) {
      const int at = atomicAdd(&s.found, 1);
      if (at < s.most) s.few[at] = key;
    }
  }
  __syncthreads();
  return s.found;
}

// This warp's part of the bound: of its lanes' two largest pieces' maxima the one that is K-th over all warps at
// worst, ceil(K / W)-th here.
template <int NT>
__device__ __forceinline__ void raise(TopShared<NT>& s, float top, float second, int K) {
  constexpr int W = NT / 32;
  const int rounds = (K + W - 1) / W, lane = threadIdx.x & 31;
  uint32_t mine = order_of(top), then = order_of(second), t = 0;
  for (int k = 0; k < rounds; ++k) {
    t = __reduce_max_sync(0xffffffffu, mine);
    const unsigned holds = __ballot_sync(0xffffffffu, mine == t);
    if (lane == __ffs(holds) - 1) {
      mine = then;
      then = 0;
    }
  }
  if (lane == 0) *const_cast<volatile uint32_t*>(&s.part[threadIdx.x >> 5]) = t;
}
// The bound: the least of the parts, as they are found.
template <int NT>
__device__ __forceinline__ float bound(const TopShared<NT>& s) {
  uint32_t t = 0xFFFFFFFFu;
#pragma unroll
  for (int w = 0; w < NT / 32; w += 4) {
    uint32_t p[4];
    asm volatile("ld.volatile.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(p[0]), "=r"(p[1]), "=r"(p[2]), "=r"(p[3])
                 : "r"(smem_u32(s.part + w)));
    t = min(min(t, min(p[0], p[1])), min(p[2], p[3]));
  }
  return t == 0 ? kLeast : fmaxf(kLeast, value_of(t));
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_addr(const void* p, int rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ uint64_t cluster_ld64(const void* p, int rank) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(cluster_addr(p, rank)));
  return v;
}
__device__ __forceinline__ float cluster_ldf(const void* p, int rank) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr(p, rank)));
  return v;
}

// Groups [begin, end) of a row whatever they hold: a barrier and, where there is no more room, an exact
// bound before each pass.  The sum goes on only where `summing`.
template <int NT, typename T, int F>
__device__ __noinline__ void rising_row(TopShared<NT>& s, const Row<T>& r, int64_t begin, int64_t end, int K,
                                        uint32_t* counts, int segment, bool summing, Sum& sum, int* status) {
  constexpr int G = Row<T>::G;
  const int64_t SG = F & kHistory && r.hist_n > 0 ? segment / G : end - begin;
  __syncthreads();
  if (threadIdx.x == 0) s.count = 0;
  __syncthreads();
  float least = kLeast;
  uint64_t least_key = 0;
  int upper = 0;
  for (int64_t s0 = begin; s0 < end; s0 += SG) {
    if ((F & kHistory) && r.hist_n > 0) count_history<NT>(r, s0 * G, segment, counts, status);
    const int64_t s1 = min(end, s0 + SG);
    for (int64_t g0 = s0; g0 < s1; g0 += kPass) {
      const int64_t g = g0 + threadIdx.x;
      float v[G];
      if (threadIdx.x < kPass && g < s1) {
        load_group(r, g, v);
        adjust_group<T, F>(r, g, counts + (F & kHistory ? (g - s0) * G : 0), v);
      } else {
#pragma unroll
        for (int j = 0; j < G; ++j) v[j] = -INFINITY;
      }
      const float most = max_of<G>(v);
      if (summing) sum.add<G>(v, most);
      const int threads = __syncthreads_count(most >= least);
      upper += threads * G;
      if (upper > kRoom) {  // (nobody adds candidates between the barrier above and those below)
        if (s.count + threads * G > kRoom) {
          least_key = max(least_key, kth_key(s, K));
          least = fmaxf(least, value_of((uint32_t)(least_key >> 32)));
          if (threadIdx.x == 0) s.found = 0;
          __syncthreads();
          const int kept = pick(s, least_key);
          if (threadIdx.x < kept) {
            const uint64_t key = s.few[threadIdx.x];
            s.cand[threadIdx.x] = candidate(value_of((uint32_t)(key >> 32)), (int)~(uint32_t)key);
          }
          if (threadIdx.x == 0) s.count = kept;
          __syncthreads();
        }
        upper = s.count + threads * G;
        __syncthreads();
      }
#pragma unroll
      for (int j = 0; j < G; ++j)
        if (v[j] >= least) {
          const uint2 c = candidate(v[j], (int)(g * G - r.a) + j);
          if (key_of(c) >= least_key) s.cand[atomicAdd(&s.count, 1)] = c;
        }
    }
  }
  if (threadIdx.x == 0) s.found = 0;
  __syncthreads();
}

// Group g of a row as it lies in memory, -inf past the row's ends and from group `end` on.
template <typename T>
__device__ __forceinline__ uint4 load_raw(const Row<T>& r, int64_t g, int64_t end) {
  constexpr int G = Row<T>::G;
  constexpr uint32_t none = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
  if (g >= end) return make_uint4(none, none, none, none);
  const int64_t c0 = g * G - r.a;
  if (c0 >= 0 && c0 + G <= r.V) return __ldcs(reinterpret_cast<const uint4*>(r.base + g * G));
  uint32_t u[4] = {none, none, none, none};
#pragma unroll
  for (int j = 0; j < G; ++j)
    if (c0 + j >= 0 && c0 + j < r.V) {
      if (sizeof(T) == 4) {
        u[j & 3] = reinterpret_cast<const uint32_t*>(r.base)[g * G + j];
      } else {
        const uint32_t h = reinterpret_cast<const unsigned short*>(r.base)[g * G + j];
        u[j >> 1] = j & 1 ? (u[j >> 1] & 0xFFFFu) | h << 16 : (u[j >> 1] & 0xFFFF0000u) | h;
      }
    }
  return make_uint4(u[0], u[1], u[2], u[3]);
}

// A cluster of CL blocks a row, each with a run of its groups.
template <int NT, typename T, int F>
__global__ void __launch_bounds__(NT, (NT > 128 ? 2 : !(F & kBias) ? 8 : sizeof(T) == 4 ? 6 : 7))
    k_top(int V, int64_t ldz, const T* Z, Adjust adj, int K, int log_cl, float* top_logit, int32_t* top_id,
          float* lse, Room room, int* status) {
  constexpr int G = Row<T>::G, NV = kEach / G, CG = NT * NV, BG = kBits / G;
  extern __shared__ __align__(16) uint8_t top_smem[];
  TopShared<NT>& s = *reinterpret_cast<TopShared<NT>*>(top_smem);
  uint64_t* few = reinterpret_cast<uint64_t*>(top_smem + room.at_few);
  uint64_t* best = reinterpret_cast<uint64_t*>(top_smem + room.at_best);
  uint32_t* bits = reinterpret_cast<uint32_t*>(top_smem + room.at_bits);
  uint32_t* table = reinterpret_cast<uint32_t*>(top_smem + room.at_table);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int CL = 1 << log_cl, rank = CL > 1 ? (int)cluster_rank() : 0;
  const int64_t row = blockIdx.x >> log_cl;
  uint32_t* note = reinterpret_cast<uint32_t*>(top_smem + room.at_note) + (tid >> 5) * room.notes;
  if (tid == 0) {
    s.found = s.over = 0;
    s.few = few;
    s.cand = reinterpret_cast<uint2*>(top_smem + room.at_note);
    s.most = room.few;
  }
  if (tid < (NT / 32)) s.part[tid] = 0;
  __syncthreads();
  tc::grid_dep_launch();
  tc::grid_dep_wait();
  const Row<T> r = make_row<T, F>(Z, ldz, row, V, adj, status);
  const int NG = r.groups(), begin = (int)((int64_t)NG * rank >> log_cl),
            end = (int)((int64_t)NG * (rank + 1) >> log_cl);
  Sum sum;
  bool quick = !(F & kHistory) || hashed(r, room.slots);
  if (!quick) {
    rising_row<NT, T, F>(s, r, begin, end, K, table, room.slots, lse != nullptr, sum, status);
  } else {
    float top = -INFINITY, second = -INFINITY, least = kLeast;
    Hash h{table, 0, 0};
    auto offer = [&](float v, int id) {
      const int at = atomicAdd(&s.found, 1);
      if (at < room.few) few[at] = key_of(v, id);
    };
    int notes = 0;  // of this warp
    const uint4* lane_base = reinterpret_cast<const uint4*>(r.base) + tid;
    const uint8_t* lane_bits = reinterpret_cast<const uint8_t*>(bits) + tid * G / 8;
    int chunk = 0;
    for (int s0 = begin; s0 < end; s0 += BG) {
      const int s1 = min(end, s0 + BG), first = s0 * G;  // (first: a multiple of 8)
      // chunks with nothing past the row's or the run's ends are read without a look at each group
      auto inside = [&](int g0) { return g0 * G >= r.a && g0 + CG <= s1 && (g0 + CG) * G - r.a <= V; };
      uint4 raw[NV];
      auto fetch = [&](int g0) {
        if (inside(g0)) {
#pragma unroll
          for (int u = 0; u < NV; ++u) raw[u] = __ldcs(lane_base + g0 + u * NT);
        } else {
#pragma unroll
          for (int u = 0; u < NV; ++u) raw[u] = load_raw(r, g0 + u * NT + tid, s1);
        }
      };
      // biases ahead too, where rows begin with a group and they lie as the logits do
      constexpr bool ahead = (F & kBias) != 0;
      float4 soon[ahead ? kEach / 4 : 1];
      auto fetch_bias = [&](int g0) {
        const float4* b = reinterpret_cast<const float4*>(r.bias + (g0 + tid) * G);
#pragma unroll
        for (int j = 0; j < kEach; j += 4) soon[ahead ? j / 4 : 0] = __ldg(b + (j / G * NT * G + j % G) / 4);
      };
      fetch(s0);
      if (ahead && r.a == 0 && inside(s0)) fetch_bias(s0);
      if (F & (kMask | kHistory)) {
        const bool past = (F & kHistory) && r.hist_n > 0;
        if (s0 != begin) __syncthreads();
        // bit e is element first + e, column first + e - a
        const int words = ((s1 - s0) * G + 31) / 32;
        for (int w = tid; w < words; w += NT) {
          uint32_t b = 0xFFFFFFFFu;
          if ((F & kMask) && r.mask && (first - r.a) % 32 == 0) {
            const int q = (first - r.a) / 32 + w;
            b = q < r.words ? __ldg(r.mask + q) : 0u;
          } else if ((F & kMask) && r.mask) {
            const int c = first + w * 32 - r.a, q = c >> 5, sh = c & 31;  // c: the word's first column
            const uint32_t lo = q >= 0 && q < r.words ? __ldg(r.mask + q) : 0u;
            const uint32_t hi = sh && q + 1 < r.words ? __ldg(r.mask + q + 1) : 0u;
            b = __funnelshift_r(lo, hi, sh);
          }
          bits[w] = b;
        }
        auto leave_out = [&](int64_t element) {
          const int64_t e = element - first;
          if (e >= 0 && e < (s1 - s0) * G) atomicAnd(&bits[e >> 5], ~(1u << (e & 31)));
        };
        if (past && s0 == begin) h = clear_hash<NT>(r, table, room.slots);
        __syncthreads();
        if (past) {
          if (s0 == begin) {
            fill_hash<NT, 1>(h, r, begin * G, end * G, status, leave_out);
          } else {
            for (int i = tid; i < h.size; i += NT)
              if (const uint32_t x = h.slot[i]) leave_out(h.token(x) + r.a);
          }
          __syncthreads();
        }
      }
      for (int g0 = s0; g0 < s1; g0 += CG, ++chunk) {
        float v[kEach];
#pragma unroll
        for (int u = 0; u < NV; ++u) unpack(raw[u], v + u * G, T());
        if (g0 + CG < s1) fetch(g0 + CG);
        const int c0 = (g0 + tid) * G - r.a;  // column of v[0]
        if (F & kBias) {
          if (r.a == 0 && inside(g0)) {
            const float4* b = reinterpret_cast<const float4*>(r.bias + c0);
#pragma unroll
            for (int j = 0; j < kEach; j += 4) {
              const float4 x = ahead ? soon[ahead ? j / 4 : 0] : __ldg(b + (j / G * NT * G + j % G) / 4);
              v[j] = __fadd_rn(v[j], x.x);
              v[j + 1] = __fadd_rn(v[j + 1], x.y);
              v[j + 2] = __fadd_rn(v[j + 2], x.z);
              v[j + 3] = __fadd_rn(v[j + 3], x.w);
            }
          } else {
#pragma unroll
            for (int u = 0; u < NV; ++u)
              if (g0 + u * NT + tid < s1)
                adjust_group<T, F & kBias>(r, g0 + u * NT + tid, nullptr, v + u * G);
          }
        }
        if (ahead && r.a == 0 && g0 + CG < s1 && inside(g0 + CG)) fetch_bias(g0 + CG);
        if (F & (kMask | kHistory)) {
          const uint8_t* q = lane_bits + (g0 - s0) * G / 8;
#pragma unroll
          for (int u = 0; u < NV; ++u) {
            const uint32_t b = G == 8 ? q[u * NT] : q[u * NT / 2] >> (tid & 1) * 4;
#pragma unroll
            for (int j = 0; j < G; ++j)
              if (!(b & 1u << j)) v[u * G + j] = -INFINITY;
          }
        }
        // (a piece of nothing but NaN has no largest: as NaN it would make `second` the lane's own `top` again)
        const float most = fmaxf(max_of<kEach>(v), -INFINITY);
        if (lse) sum.add<kEach>(v, most);
        second = fmaxf(second, fminf(top, most));
        top = fmaxf(top, most);
        if ((chunk & (chunk + 1)) == 0) {
          raise(s, top, second, K);
          if (chunk == 0) __syncthreads();
        }
        least = fmaxf(least, bound(s));
        const unsigned pass = __ballot_sync(0xffffffffu, most >= least);
        if (pass) {
          const int at = notes + __popc(pass & ((1u << lane) - 1));
          uint32_t groups = 0;  // of the piece that reach it
#pragma unroll
          for (int u = 0; u < NV; ++u) groups |= max_of<G>(v + u * G) >= least ? 1u << (28 + u) : 0u;
          if (groups && at < room.notes) note[at] = groups | (uint32_t)(g0 + tid);
          notes += __popc(pass);
        }
      }
      // the pieces noted, by the last bound where this is the last run
      if (s1 == end) {
        raise(s, top, second, K);
        __syncthreads();
      } else {
        __syncwarp();
      }
      least = fmaxf(least, bound(s));
      if (notes > room.notes && lane == 0) s.over = 1;
      for (int i = lane; i < min(notes, room.notes); i += 32) {
        const uint32_t piece = note[i], p = piece & 0xFFFFFFFu;  // the piece's first group
#pragma unroll
        for (int u = 0; u < NV; ++u) {
          const int g = (int)p + u * NT;
          if (!(piece >> (28 + u) & 1u)) continue;
          float v[G];
          load_group(r, g, v);
          if (F & kBias) adjust_group<T, F & kBias>(r, g, nullptr, v);
          uint32_t b = 0xFFu;
          if (F & (kMask | kHistory))
            b = reinterpret_cast<const uint8_t*>(bits)[(g - s0) * G / 8] >> ((g - s0) * G & 7);
#pragma unroll
          for (int j = 0; j < G; ++j)
            if (v[j] >= least && (b >> j & 1u)) offer(v[j], g * G - r.a + j);
        }
      }
      notes = 0;
    }
    if ((F & kHistory) && r.hist_n > 0) {
      // the tokens of the history, the logits of several on their way
      constexpr int U = 8;
      for (int i0 = tid; i0 < h.size; i0 += U * NT) {
        uint32_t slot[U];
        int id[U];
        float v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + u * NT;
          slot[u] = i < h.size ? h.slot[i] : 0u;
          id[u] = h.token(slot[u]);
          if ((F & kMask) && r.mask && id[u] >= 0 && !(__ldg(r.mask + (id[u] >> 5)) >> (id[u] & 31) & 1u)) id[u] = -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          v[u] = id[u] >= 0 ? to_f32(r.base[id[u] + r.a]) : -INFINITY;
          if ((F & kBias) && id[u] >= 0) v[u] = __fadd_rn(v[u], __ldg(r.bias + id[u]));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (id[u] < 0) continue;
          v[u] = penalised(v[u], h.count(slot[u]), r.rep, r.presence, r.frequency);
          if (lse) {
            sum.refer(v[u]);
            sum.l += ex2(fmaf(v[u], kLog2e, -sum.m));
          }
          if (v[u] >= least) offer(v[u], id[u]);
        }
      }
    }
  }
  if (lse) {
    float top_m = sum.m, l = sum.l;
#pragma unroll
    for (int o = 16; o; o >>= 1) top_m = fmaxf(top_m, __shfl_xor_sync(0xffffffffu, top_m, o));
    l *= ex2(sum.m - top_m);
#pragma unroll
    for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (lane == 0) s.m[warp] = top_m, s.l[warp] = l;
  }
  __syncthreads();
  if (quick && (s.over || s.found > room.few)) {
    rising_row<NT, T, F>(s, r, begin, end, K, table, room.slots, false, sum, status);
    quick = false;
  }
  if (lse && tid == NT - 1) {
    float bm = s.m[0], bl = 0.f;
#pragma unroll
    for (int w = 1; w < (NT / 32); ++w) bm = fmaxf(bm, s.m[w]);
#pragma unroll
    for (int w = 0; w < (NT / 32); ++w) bl += s.l[w] * ex2(s.m[w] - bm);
    if (CL > 1)
      s.block_m = bm, s.block_l = bl;
    else
      lse[row] = lse_of(bm, bl);
  }
  // the block's largest in order: few candidates, each one's place counted, four threads a candidate
  int n = quick ? s.found : pick(s, 0);
  if (n > room.few) {
    const uint64_t t = kth_key(s, K);
    if (tid == 0) s.found = 0;
    __syncthreads();
    n = pick(s, t);
  }
  auto answer = [&](int place, uint64_t key) {
    top_logit[row * K + place] = key ? value_of((uint32_t)(key >> 32)) : -INFINITY;
    top_id[row * K + place] = key ? (int32_t) ~(uint32_t)key : -1;
  };
  for (int i0 = 0; i0 < n; i0 += NT / 4) {
    const int i = i0 + tid / 4;
    const uint64_t key = i < n ? few[i] : 0;
    int place = 0;
    for (int o = tid & 3; o < n; o += 4) place += few[o] > key;
    place += __shfl_xor_sync(0xffffffffu, place, 1);
    place += __shfl_xor_sync(0xffffffffu, place, 2);
    if ((tid & 3) == 0 && i < n && place < K) {
      if (CL > 1)
        best[place] = key;
      else
        answer(place, key);
    }
  }
  for (int k = n + tid; k < K; k += NT) {
    if (CL > 1)
      best[k] = 0;
    else
      answer(k, 0);
  }
  if (CL > 1) {
    cluster_sync();
    if (rank == 0) {
      uint64_t* lists = reinterpret_cast<uint64_t*>(top_smem + room.at_note);
      // the blocks' lists, each in order: a key's place is the number of larger ones in all lists
      for (int i = tid; i < CL * K; i += NT) lists[i] = cluster_ld64(best + i % K, i / K);
      __syncthreads();
      for (int i = tid; i < CL * K; i += NT) {
        const uint64_t key = lists[i];
        if (key == 0) continue;
        int place = 0;
        for (int b = 0; b < CL; ++b) {
          int lo = 0, hi = K;  // entries of list b larger than key
          while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (lists[b * K + mid] > key) lo = mid + 1; else hi = mid;
          }
          place += lo;
        }
        if (place < K) {
          top_logit[row * K + place] = value_of((uint32_t)(key >> 32));
          top_id[row * K + place] = (int32_t) ~(uint32_t)key;
        }
      }
      int have = 0;
      for (int b = 0; b < CL; ++b) {
        int lo = 0, hi = K;
        while (lo < hi) {
          const int mid = (lo + hi) / 2;
          if (lists[b * K + mid] != 0) lo = mid + 1; else hi = mid;
        }
        have += lo;
      }
      for (int k = have + tid; k < K; k += NT) {
        top_logit[row * K + k] = -INFINITY;
        top_id[row * K + k] = -1;
      }
      if (lse && tid == 0) {
        float bm = s.block_m;
        for (int b = 1; b < CL; ++b) bm = fmaxf(bm, cluster_ldf(&s.block_m, b));
        float bl = 0.f;
        for (int b = 0; b < CL; ++b) bl += cluster_ldf(&s.block_l, b) * ex2(cluster_ldf(&s.block_m, b) - bm);
        lse[row] = lse_of(bm, bl);
      }
    }
    __syncthreads();
    cluster_sync();  // (no block leaves while the first may still read its list)
  }
}

// ------------------------------------------------------------------------------ host
// Whether n bf16 rows with biases, each of which begins `lead` elements further on in a group than the one before,
// share them.  8192 x 49999 takes 355 us shared and 390 with the biases read one by one (masks too 370 and 414,
// histories too 498 and 523), 8192 x 32769 242 and 263; but 1024 x 20001 38 and 27, 32 x 49999 21 and 11, rows 4
// elements further on each (8192 x 50004) 355 and 324, and fp32 (8192 x 49999) 699 and 533.
bool shares_biases(int64_t n, int V, int lead) {
  return lead % 2 && V >= 4 * kRun && n * V >= (int64_t)1 << 27;
}

template <typename T, int F>
cudaError_t run_adjust(int64_t n, int V, int64_t ldz, const void* Z, const Adjust& adj, int64_t ldo, void* out,
                       int* status, cudaStream_t st) {
  constexpr int G = Row<T>::G;
  const T* z = static_cast<const T*>(Z);
  T* o = static_cast<T*>(out);
  const int64_t groups = ((int64_t)V + 2 * G - 2) / G;
  const int lead = (int)(ldz % G);  // rows begin so much further on than the one before
  int tokens = 0;
  if constexpr (sizeof(T) == 2 && (F & kBias) != 0) {
    // (in place, the tokens' logits would be gone after the first launch)
    if (shares_biases(n, V, lead) && !((F & kHistory) && out == Z)) {
      constexpr int D = F & ~kHistory;
      constexpr int step = G;  // (an odd lead)
      const int64_t sets = (n + step * kShare - 1) / (step * kShare) * step;
      const cudaError_t e =
          launch_pdl(k_adjust_shared<T, D>, dim3((unsigned)sets, (unsigned)((groups * G + kRun - 1) / kRun)),
                     dim3(kThreads), kRun * 4, st, n, V, ldz, z, adj, ldo, o, step, status);
      if (e != cudaSuccess) return e;
      note_launch();
      if (!(F & kHistory)) return e;
      tokens = 1;
    }
  }
  // runs of 8192 elements; with histories, which are read for each run, longer ones where there are blocks enough, and
  // shorter ones where there are few (49999 elements and 256 tokens a row, short and 8192: fp32 50 rows 5.6 and 8.4 us,
  // 100 8.7 and 11.5, 200 17 and 14; bf16 50 5.7 and 5.7, 100 8.3 and 7.3)
  int64_t per = 8192 / G;
  if ((F & kHistory) && n * V <= 152 * 8 * kSlots) per = kSlots / G;
  while ((F & kHistory) && per * G < 65536 && n * ((groups + 2 * per - 1) / (2 * per)) >= 152 * 16) per *= 2;
  const cudaError_t e = launch_pdl(k_adjust<T, F>, dim3((unsigned)n, (unsigned)((groups + per - 1) / per)),
                                   dim3(kThreads), 0, st, V, ldz, z, adj, ldo, o, (int)per, tokens, status);
  if (e == cudaSuccess) note_launch();
  return e;
}

// Blocks a row, as a power of two: one where rows fill the card, else as many as leave a block 1024 logits.
int cluster_of(int64_t n, int V) {
  int c = 0;
  while (1 << c < kMaxCluster && (n << (c + 1)) <= 152 * 2 && V >> (c + 1) >= 1024) ++c;
  return c;
}

template <int NT, typename T, int F>
cudaError_t launch_top(int64_t n, int V, int64_t ldz, const void* Z, const Adjust& adj, int K, int log_cl,
                       float* top_logit, int32_t* top_id, float* lse, int* status, cudaStream_t st) {
  const Room room = room_of<NT>(F, V, K, n, adj.history_len, log_cl > 0);
  static std::atomic<uint64_t> done{0};
  cudaError_t e = allow_smem(k_top<NT, T, F>, 65536, done);  // (more than it takes)
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(n << log_cl));
  cfg.blockDim = dim3(NT);
  cfg.dynamicSmemBytes = room.bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1u << log_cl;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = log_cl > 0 ? 2 : 1;
  e = cudaLaunchKernelEx(&cfg, k_top<NT, T, F>, V, ldz, static_cast<const T*>(Z), adj, K, log_cl, top_logit, top_id,
                         lse, room, status);
  if (e == cudaSuccess) note_launch();
  return e;
}

template <typename T, int F>
cudaError_t run_top(int64_t n, int V, int64_t ldz, const void* Z, const Adjust& adj, int K, float* top_logit,
                    int32_t* top_id, float* lse, int* status, cudaStream_t st) {
  const int log_cl = cluster_of(n, V);
  // Many rows: small blocks, so that one's latencies are another's work.  Few: a row's own work in one go.  (Top 32 of
  // 49999, 512 and 128 threads: bf16 456 rows 25 and 29 us, 608 28 and 26, 912 39 and 36; fp32 305 22 and 29, 608 32 and
  // 33, 912 47 and 41.  With biases and histories 128 would be ahead sooner: 305 rows 39 and 38, fp32 48 and 38.)
  if ((n << log_cl) <= 152 * 4)
    return launch_top<512, T, F>(n, V, ldz, Z, adj, K, log_cl, top_logit, top_id, lse, status, st);
  return launch_top<128, T, F>(n, V, ldz, Z, adj, K, log_cl, top_logit, top_id, lse, status, st);
}

// f with the adjustment's flags as a constant.
template <typename Fn>
cudaError_t with_flags(int flags, Fn f) {
  switch (flags) {
    case 0: return f(std::integral_constant<int, 0>());
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 3: return f(std::integral_constant<int, 3>());
    case 4: return f(std::integral_constant<int, 4>());
    case 5: return f(std::integral_constant<int, 5>());
    case 6: return f(std::integral_constant<int, 6>());
    default: return f(std::integral_constant<int, 7>());
  }
}

}  // namespace

cudaError_t logits_adjust(int bf16, int64_t n, int V, int64_t ldz, const void* Z, const bg_adjust& b, int64_t ldo,
                          void* out, int* status, cudaStream_t st) {
  if (n == 0) return cudaSuccess;
  const Adjust adj = make_adjust(b, V);
  return with_flags(flags_of(b), [&](auto f) {
    constexpr int F = decltype(f)::value;
    return bf16 ? run_adjust<__nv_bfloat16, F>(n, V, ldz, Z, adj, ldo, out, status, st)
                : run_adjust<float, F>(n, V, ldz, Z, adj, ldo, out, status, st);
  });
}

cudaError_t logits_top(int bf16, int64_t n, int V, int64_t ldz, const void* Z, const bg_adjust& b, int K,
                       float* top_logit, int32_t* top_id, float* lse, int* status, cudaStream_t st) {
  if (n == 0) return cudaSuccess;
  const Adjust adj = make_adjust(b, V);
  return with_flags(flags_of(b), [&](auto f) {
    constexpr int F = decltype(f)::value;
    return bf16 ? run_top<__nv_bfloat16, F>(n, V, ldz, Z, adj, K, top_logit, top_id, lse, status, st)
                : run_top<float, F>(n, V, ldz, Z, adj, K, top_logit, top_id, lse, status, st);
  });
}

}  // namespace bg
