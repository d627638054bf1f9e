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
// first one.  Occurrences are counted in shared memory, kSegment columns at a time, by reading the
// row's history once for each segment: no sorting and no workspace.
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

constexpr int kThreads = 256;
constexpr int kSegment = 8192;  // elements whose occurrences are counted at a time
constexpr int kEach = 16;       // elements of a thread at a time
constexpr int kChunk = kThreads * kEach;

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

// Occurrences of the tokens of elements [first, first + kSegment) of a row (element = column + a).
template <typename T>
__device__ __forceinline__ void count_history(const Row<T>& r, int64_t first, uint32_t* counts, int* status) {
  __syncthreads();
  for (int i = threadIdx.x; i < kSegment / 4; i += kThreads)
    reinterpret_cast<uint4*>(counts)[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
  for (int64_t i = threadIdx.x; i < r.hist_n; i += kThreads) {
    const int id = r.hist[i];
    if (id >= r.V) report(status, kSiteHistoryId);
    const int64_t at = (int64_t)id + r.a - first;
    if (id >= 0 && id < r.V && at >= 0 && at < kSegment) atomicAdd(&counts[at], 1u);
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
    if (c0 >= 0 && c0 + G <= r.V) {
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

// ------------------------------------------------------------------------------ adjustment
__device__ __forceinline__ void store_group(float* p, const float* v) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store_group(__nv_bfloat16* p, const float* v) {
  __nv_bfloat162 h[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(h);
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

// Block (segment, row).
template <typename T, int F>
__global__ void __launch_bounds__(kThreads)
    k_adjust(int64_t n, int V, int64_t ldz, const T* Z, Adjust adj, int64_t ldo, T* out, int* status) {
  constexpr int G = Row<T>::G, SG = kSegment / G;
  __shared__ __align__(16) uint32_t counts[F & kHistory ? kSegment : 4];
  tc::grid_dep_launch();
  tc::grid_dep_wait();
  const int64_t i = blockIdx.x;
  const Row<T> r = make_row<T, F>(Z, ldz, i, V, adj, status);
  T* o = out + i * ldo;
  const bool vec = (reinterpret_cast<uintptr_t>(o - r.a) & 15) == 0;
  for (int64_t g0 = (int64_t)blockIdx.y * SG; g0 < r.groups(); g0 += (int64_t)gridDim.y * SG) {
    if ((F & kHistory) && r.hist_n > 0) count_history(r, g0 * G, counts, status);
    const int64_t g1 = min((int64_t)r.groups(), g0 + SG);
    for (int64_t g = g0 + threadIdx.x; g < g1; g += kThreads) {
      float v[G];
      load_group(r, g, v);
      adjust_group<T, F>(r, g, counts + (F & kHistory ? (g - g0) * G : 0), v);
      const int64_t c0 = g * G - r.a;
      if (vec && c0 >= 0 && c0 + G <= V) {
        store_group(o + c0, v);
      } else {
#pragma unroll
        for (int j = 0; j < G; ++j)
          if (c0 + j >= 0 && c0 + j < V) store1(o + c0 + j, v[j]);
      }
    }
  }
}

// ------------------------------------------------------------------------------ largest logits
constexpr int kRoom = kChunk + 1024;  // candidates a block keeps
constexpr int kMaxCluster = 8;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNoLogit = -3.0e38f;  // reference of a sum without terms

struct TopShared {
  uint64_t cand[kRoom];
  uint64_t best[kMaxTop];
  float m[kThreads / 32], l[kThreads / 32];
  float block_m, block_l;
  uint32_t warp_t[kThreads / 32];
  int count, sum[64];
};

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

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// log of the sum l to the reference m (in base 2).  A sum of 0 with a reference: every term vanished beside
// the rounding of the reference, which then is the result to the last bit.
__device__ __forceinline__ float lse_of(float m, float l) {
  return (l == 0.f && m > kNoLogit ? m : m + log2f(l)) * 0.6931471805599453f;
}

// Keeps the candidates with keys of t or more; the whole block calls it.
__device__ __noinline__ void keep_from(TopShared& s, uint64_t t) {
  uint64_t mine[kRoom / kThreads];
  __syncthreads();
  const int n = s.count;
#pragma unroll
  for (int k = 0; k < kRoom / kThreads; ++k) {
    const int i = threadIdx.x + k * kThreads;
    mine[k] = i < n ? s.cand[i] : 0;
  }
  __syncthreads();
  if (threadIdx.x == 0) s.count = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kRoom / kThreads; ++k)
    if (mine[k] >= t && mine[k] != 0) s.cand[atomicAdd(&s.count, 1)] = mine[k];
  __syncthreads();
}

// The K-th largest candidate's key (0 where there are fewer), a bit at a time; the whole block calls it.
__device__ __noinline__ uint64_t kth_key(TopShared& s, int K) {
  __syncthreads();
  const int n = s.count;
  if (n < K) return 0;
  if (threadIdx.x < 64) s.sum[threadIdx.x] = 0;
  __syncthreads();
  uint64_t t = 0;
  for (int bit = 63; bit >= 0; --bit) {
    const uint64_t trial = t | (uint64_t)1 << bit;
    int c = 0;
    for (int i = threadIdx.x; i < n; i += kThreads) c += s.cand[i] >= trial;
    c = __reduce_add_sync(0xffffffffu, c);
    if ((threadIdx.x & 31) == 0 && c) atomicAdd(&s.sum[bit], c);
    __syncthreads();
    if (s.sum[bit] >= K) t = trial;
  }
  return t;
}

// A value that K of the row's logits reach at least, from a logit of each thread: each warp's
// ceil(K / 8)-th largest, the least of them.
__device__ __forceinline__ float reached(TopShared& s, float top, int K) {
  const int rounds = (K + kThreads / 32 - 1) / (kThreads / 32), lane = threadIdx.x & 31;
  uint32_t mine = order_of(top), t = 0;
  for (int k = 0; k < rounds; ++k) {
    t = __reduce_max_sync(0xffffffffu, mine);
    const unsigned holds = __ballot_sync(0xffffffffu, mine == t);
    if (lane == __ffs(holds) - 1) mine = 0;
  }
  if (lane == 0) s.warp_t[threadIdx.x >> 5] = t;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) t = min(t, s.warp_t[w]);
  return t == 0 ? -INFINITY : value_of(t);
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

// A cluster of CL blocks a row, each with a run of its groups.
template <typename T, int F>
__global__ void __launch_bounds__(kThreads)
    k_top(int V, int64_t ldz, const T* Z, Adjust adj, int K, int CL, float* top_logit, int32_t* top_id,
          float* lse, int* status) {
  constexpr int G = Row<T>::G, NV = kEach / G, SG = kSegment / G, CG = kThreads * NV;
  extern __shared__ __align__(16) uint8_t top_smem[];
  TopShared& s = *reinterpret_cast<TopShared*>(top_smem);
  uint32_t* counts = reinterpret_cast<uint32_t*>(top_smem + sizeof(TopShared));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = CL > 1 ? (int)cluster_rank() : 0;
  const int64_t row = blockIdx.x / CL;
  if (tid == 0) s.count = 0;
  tc::grid_dep_launch();
  tc::grid_dep_wait();
  const Row<T> r = make_row<T, F>(Z, ldz, row, V, adj, status);
  const int64_t NG = r.groups(), begin = NG * rank / CL, end = NG * (rank + 1) / CL;
  float m = kNoLogit, l = 0.f, top = -INFINITY;  // of this thread
  float least = -3.402823466e38f;                // candidates are at least this large
  uint64_t least_key = 0;
  int upper = 0, chunk = 0;  // candidates at most; chunks so far
  __syncthreads();
  for (int64_t s0 = begin; s0 < end; s0 += SG) {
    if ((F & kHistory) && r.hist_n > 0) count_history(r, s0 * G, counts, status);
    const int64_t s1 = min(end, s0 + SG);
    for (int64_t g0 = s0; g0 < s1; g0 += CG, ++chunk) {
      float v[kEach];
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int64_t g = g0 + u * kThreads + tid;
        if (g < s1) {
          load_group(r, g, v + u * G);
        } else {
#pragma unroll
          for (int j = 0; j < G; ++j) v[u * G + j] = -INFINITY;
        }
      }
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int64_t g = g0 + u * kThreads + tid;
        if (F && g < s1) adjust_group<T, F>(r, g, counts + (F & kHistory ? (g - s0) * G : 0), v + u * G);
      }
      float most = v[0];
#pragma unroll
      for (int j = 1; j < kEach; ++j) most = fmaxf(most, v[j]);
      if (lse) {
        // (rounded up: of logits beyond 2^31 the terms may vanish but not overflow)
        const float mc = __fmul_ru(most, kLog2e);
        if (mc > m) {
          l *= ex2(m - mc);
          m = mc;
        }
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kEach; ++j) sum[j & 1] += ex2(fmaf(v[j], kLog2e, -m));
        l += sum[0] + sum[1];
      }
      top = fmaxf(top, most);
      // after 1, 2, 4, ... chunks the bound rises
      if ((chunk & (chunk + 1)) == 0) {
        const float t = reached(s, top, K);
        if (t > least) {
          least = t;
          least_key = (uint64_t)order_of(t) << 32;
        }
      }
      const bool some = most >= least;
      const int threads = __syncthreads_count(some);
      if (threads == 0) continue;
      upper += threads * kEach;
      if (upper > kRoom) {  // (rare; nobody adds candidates between the barrier above and those below)
        if (s.count + threads * kEach > kRoom) {
          least_key = max(least_key, kth_key(s, K));
          least = fmaxf(least, value_of((uint32_t)(least_key >> 32)));
          keep_from(s, least_key);
        }
        upper = s.count + threads * kEach;
        __syncthreads();
      }
      if (some) {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
          if (v[j] >= least) {
            const int64_t g = g0 + j / G * kThreads + tid;
            const uint64_t key = key_of(v[j], (int)(g * G - r.a) + j % G);
            if (key >= least_key) s.cand[atomicAdd(&s.count, 1)] = key;
          }
      }
    }
  }
  // the block's largest in order: few candidates, each one's place counted
  {
    const float t = reached(s, top, K);  // (and a barrier)
    if (t > least) least_key = (uint64_t)order_of(t) << 32;
    if (s.count > 64) keep_from(s, least_key);
    if (s.count > kThreads) keep_from(s, kth_key(s, K));
    __syncthreads();
    const int n = s.count;
    if (tid < kMaxTop) s.best[tid] = 0;
    __syncthreads();
    if (tid < n) {
      const uint64_t key = s.cand[tid];
      int place = 0;
      for (int i = 0; i < n; ++i) place += s.cand[i] > key;
      if (place < K) s.best[place] = key;
    }
  }
  if (lse) {
    float top_m = m;
#pragma unroll
    for (int o = 16; o; o >>= 1) top_m = fmaxf(top_m, __shfl_xor_sync(0xffffffffu, top_m, o));
    l *= ex2(m - top_m);
#pragma unroll
    for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (lane == 0) s.m[warp] = top_m, s.l[warp] = l;
  }
  __syncthreads();
  if (lse && tid == 0) {
    float bm = s.m[0];
    for (int w = 1; w < kThreads / 32; ++w) bm = fmaxf(bm, s.m[w]);
    float bl = 0.f;
    for (int w = 0; w < kThreads / 32; ++w) bl += s.l[w] * ex2(s.m[w] - bm);
    s.block_m = bm;
    s.block_l = bl;
  }
  if (CL > 1) {
    cluster_sync();
    if (rank == 0) {
      // the blocks' lists, each in order: a key's place is the number of larger ones in all lists
      for (int i = tid; i < CL * K; i += kThreads) s.cand[i] = cluster_ld64(&s.best[i % K], i / K);
      __syncthreads();
      for (int i = tid; i < CL * K; i += kThreads) {
        const uint64_t key = s.cand[i];
        if (key == 0) continue;
        int place = 0;
        for (int b = 0; b < CL; ++b) {
          int lo = 0, hi = K;  // entries of list b larger than key
          while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (s.cand[b * K + mid] > key) lo = mid + 1; else hi = mid;
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
          if (s.cand[b * K + mid] != 0) lo = mid + 1; else hi = mid;
        }
        have += lo;
      }
      for (int k = have + tid; k < K; k += kThreads) {
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
  } else {
    __syncthreads();
    if (tid < K) {
      const uint64_t key = s.best[tid];
      top_logit[row * K + tid] = key ? value_of((uint32_t)(key >> 32)) : -INFINITY;
      top_id[row * K + tid] = key ? (int32_t) ~(uint32_t)key : -1;
    }
    if (lse && tid == 0) lse[row] = lse_of(s.block_m, s.block_l);
  }
}

// ------------------------------------------------------------------------------ host
template <typename T, int F>
cudaError_t run_adjust(int64_t n, int V, int64_t ldz, const void* Z, const Adjust& adj, int64_t ldo, void* out,
                       int* status, cudaStream_t st) {
  const int segments = (int)(((int64_t)V + 7 + kSegment - 1) / kSegment);
  const cudaError_t e =
      launch_pdl(k_adjust<T, F>, dim3((unsigned)n, (unsigned)segments), dim3(kThreads), 0, st, n, V, ldz,
                 static_cast<const T*>(Z), adj, ldo, static_cast<T*>(out), status);
  if (e == cudaSuccess) note_launch();
  return e;
}

// Blocks a row: one where rows fill the card, else as many as still leave a block a chunk.
int cluster_of(int64_t n, int V) {
  int c = 1;
  while (c < kMaxCluster && n * c * 2 <= 152 * 2 && V >= c * 2 * kChunk / 4) c *= 2;
  return c;
}

template <typename T, int F>
cudaError_t run_top(int64_t n, int V, int64_t ldz, const void* Z, const Adjust& adj, int K, float* top_logit,
                    int32_t* top_id, float* lse, int* status, cudaStream_t st) {
  const int CL = cluster_of(n, V);
  constexpr int smem = (int)sizeof(TopShared) + (F & kHistory ? kSegment * 4 : 0);
  static std::atomic<uint64_t> done{0};
  cudaError_t e = allow_smem(k_top<T, F>, smem, done);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(n * CL));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)CL;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CL > 1 ? 2 : 1;
  e = cudaLaunchKernelEx(&cfg, k_top<T, F>, V, ldz, static_cast<const T*>(Z), adj, K, CL, top_logit, top_id, lse,
                         status);
  if (e == cudaSuccess) note_launch();
  return e;
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
