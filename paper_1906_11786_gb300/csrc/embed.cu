// Dropout with a mask that is never stored, and the embedding lookup that makes initial node
// states with its gradient by sorted tokens.
//
// Every kernel here moves bytes and does little arithmetic; a thread works on 8 consecutive
// elements, the elements of one generator block (philox.h), as one 16-byte (bf16) or two 16-byte
// (fp32) accesses.  Measured (GB300; a fill of 67 MB takes 12.4 us there, of 134 MB 20.7): dropout of 33.5 M
// bf16 elements with residual 34 us (201 MB, 5.9 TB/s), of 25.6 M fp32 gradients 37 us (205 MB); lookup of
// 131072 x 256 bf16 states 23 us, with dropout 29 (67 MB written), of fp32 states 33-35 (134 MB written);
// table gradient of 131071 x 256 over 49999 tokens 75 us a pass (134 MB read, 51 written).  Its kernels one by
// one, caches cold (ncu): sorting 31 us, sums 34-37 (3.9 TB/s), joining 12.  No unit is full in the lookup
// (with dropout: issue slots 70%, ALU 57%): the way from an id to its row to the store is hidden by other
// warps alone.
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "tc_util.cuh"
#include "token.h"

namespace bg {

using tc::grid_dep_launch;
using tc::grid_dep_wait;

namespace {

// ------------------------------------------------------------------------------ 8 elements
__device__ __forceinline__ void load8(const float* p, float* v) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float* v) {
  const uint4 a = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(u[j] << 16);
    v[2 * j + 1] = __uint_as_float(u[j] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void store8(float* p, const float* v) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* v) {
  __nv_bfloat162 h[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(h);
}
// Past the caches' reach: the line is not kept in L2.
__device__ __forceinline__ void store8_stream(float* p, const float* v) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
  __stcs(reinterpret_cast<float4*>(p + 4), make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void store8_stream(__nv_bfloat16* p, const float* v) {
  __nv_bfloat162 h[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
  __stcs(reinterpret_cast<uint4*>(p), *reinterpret_cast<const uint4*>(h));
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

// ------------------------------------------------------------------------------ dropout
// y = add + drop(x), add = res (forward) or y's own values (a gradient that accumulates).  x, res
// and y may be the same array: a thread reads its elements before it writes them.
template <typename T>
__global__ void __launch_bounds__(256)
    k_dropout(int64_t n, Drop d, const T* x, const T* res, T* y, int stream) {
  const int64_t full = n / 8, step = (int64_t)gridDim.x * blockDim.x;
  int64_t b = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
  // 32 bytes of each array in flight a thread: at 64, or with more or fewer than 8 blocks an SM, both
  // types took up to 15% longer
  constexpr int kDropUnroll = 4 / (int)sizeof(T);
  auto blocks8 = [&](auto unroll) {
    constexpr int U = decltype(unroll)::value;
    float v[U][8], r[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      load8(x + (b + u * step) * 8, v[u]);
      if (res) load8(res + (b + u * step) * 8, r[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (d.thr) drop8(d, (uint64_t)(b + u * step), d.scale, v[u]);
      if (res) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[u][j] += r[u][j];
      }
      if (stream)
        store8_stream(y + (b + u * step) * 8, v[u]);
      else
        store8(y + (b + u * step) * 8, v[u]);
    }
  };
  for (; b + (kDropUnroll - 1) * step < full; b += kDropUnroll * step)
    blocks8(std::integral_constant<int, kDropUnroll>());
  for (; b < full; b += step) blocks8(std::integral_constant<int, 1>());
  if (b == full && full * 8 < n) {  // the last elements, fewer than 8: one thread's
    const int64_t i = full * 8;
    const int m = (int)(n - i);
    float v[8], r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = j < m ? load1(x + i + j) : 0.f;
      r[j] = j < m && res ? load1(res + i + j) : 0.f;
    }
    if (d.thr) drop8(d, (uint64_t)full, d.scale, v);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < m) store1(y + i + j, res ? v[j] + r[j] : v[j]);
  }
}

template <typename T>
cudaError_t run_dropout(int64_t n, const Drop& d, const void* x, const void* res, void* y,
                        cudaStream_t st) {
  if (n == 0) return cudaSuccess;
  const int64_t blocks = (n + 7) / 8;
  const int grid = (int)std::min<int64_t>((blocks + 255) / 256, 152 * 8);
  // a result that cannot stay in L2 (129 MB) beside the operands is not kept there: 37.0 -> 34.8 us at
  // 3 x 67 MB; a smaller one is its reader's
  const int stream = n * (int64_t)sizeof(T) * (res ? 3 : 2) > ((int64_t)128 << 20);
  k_dropout<T><<<grid, 256, 0, st>>>(n, d, static_cast<const T*>(x), static_cast<const T*>(res),
                                     static_cast<T*>(y), stream);
  note_launch();
  return cudaGetLastError();
}

// ------------------------------------------------------------------------------ embedding lookup
// A row is H / 8 threads; a thread takes the same place of kEmbedUnroll rows, whose ids, and then whose
// table rows, are in flight together.
constexpr int kEmbedUnroll = 2;

template <typename T>
__global__ void __launch_bounds__(256)
    k_embed_fwd(int64_t n, int H, int V, const int32_t* __restrict__ ids,
                const T* __restrict__ table, float scale, Drop d, T* __restrict__ out, int* status) {
  const int lanes = H / 8, rows = 256 / lanes;
  const int r = threadIdx.x / lanes, c = threadIdx.x % lanes;
  if (r >= rows) return;
  const int64_t i0 = (int64_t)blockIdx.x * rows * kEmbedUnroll + r;
  int id[kEmbedUnroll];
  float v[kEmbedUnroll][8];
#pragma unroll
  for (int u = 0; u < kEmbedUnroll; ++u) id[u] = i0 + u * rows < n ? ids[i0 + u * rows] : -1;
#pragma unroll
  for (int u = 0; u < kEmbedUnroll; ++u) {
    if (id[u] >= 0 && id[u] < V) {
      load8(table + (int64_t)id[u] * H + c * 8, v[u]);
    } else {
      if (id[u] >= V && c == 0 && atomicCAS(status, 0, 2) == 0) atomicExch(status + 1, kSiteEmbedId);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[u][j] = 0.f;
    }
  }
#pragma unroll
  for (int u = 0; u < kEmbedUnroll; ++u) {
    const int64_t i = i0 + u * rows;
    if (i >= n) break;
    if (d.thr) {
      drop8(d, (uint64_t)i * lanes + c, scale * d.scale, v[u]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[u][j] *= scale;
    }
    store8(out + i * H + c * 8, v[u]);
  }
}

// ------------------------------------------------------------------------------ embedding gradient
// The rows of dout are summed by token in three steps that give the same bits every time: a stable
// radix sort of (id, position), sums over pieces of sorted positions, and a join of the
// tokens that span pieces, in the order of the pieces.  An id that names no row sorts as V, after
// all others, and is not summed.
constexpr int kTile = 2048;  // keys a sorting block ranks at a time: 8 warps x 8 x 32

struct SortPlan {
  int passes, bits;  // digits of `bits` bits
  int D;             // 1 << bits
  int64_t T;         // keys of one block, a multiple of kTile
  int nb;            // blocks
};

SortPlan sort_plan(int64_t n, int V) {
  SortPlan s;
  int bits = 1;
  while (((int64_t)1 << bits) <= V) ++bits;  // keys 0 .. V
  s.passes = (bits + 8) / 9;
  s.bits = std::max(2, (bits + s.passes - 1) / s.passes);
  s.D = 1 << s.bits;
  s.T = kTile * std::max<int64_t>(1, (n + (int64_t)kTile * 152 - 1) / ((int64_t)kTile * 152));
  s.nb = (int)std::max<int64_t>(1, (n + s.T - 1) / s.T);
  return s;
}

// The blocks of k_embed_sum: a group of lanes (H / 8, rounded up to a power of two) sums a piece of sorted
// positions; a warp has a ring of kRing rows on their way for its groups.
constexpr int kMaxPiece = 64, kRing = 8;
struct SumPlan {
  int lanes, groups, piece;
  int64_t pieces, blocks;
  int smem;
};
SumPlan sum_plan(int64_t n, int H) {
  SumPlan p;
  p.lanes = H / 8 <= 4 ? 4 : H / 8 <= 8 ? 8 : H / 8 <= 16 ? 16 : 32;
  p.groups = 256 / p.lanes;
  // pieces of at most kMaxPiece that fill the SMs (two or three blocks each) a whole number of times
  const int most = p.groups * kMaxPiece * 8 + kRing * 8192 + 1024;
  const int64_t slots = 152LL * std::min(3, 232448 / most) * p.groups;
  const int64_t waves = std::max<int64_t>(1, (n + slots * kMaxPiece - 1) / (slots * kMaxPiece));
  const int64_t piece = (n + slots * waves - 1) / (slots * waves);
  p.piece = (int)std::min<int64_t>(kMaxPiece, std::max<int64_t>(8, (piece + 1) / 2 * 2));
  p.pieces = (n + p.piece - 1) / p.piece;
  p.blocks = (p.pieces + p.groups - 1) / p.groups;
  p.smem = kRing * 8192 + (2 * p.groups * p.piece + 4) * 4;
  return p;
}

inline size_t al(size_t x) { return (x + 255) & ~(size_t)255; }

struct BwdWs {
  size_t key[2], pos[2], hist, head, tail, total;
};
BwdWs bwd_ws(int64_t n, int H, int V) {
  const SortPlan s = sort_plan(n, V);
  BwdWs w;
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += al(bytes);
    return at;
  };
  const size_t pieces = (size_t)sum_plan(n, H).pieces;
  for (int i = 0; i < 2; ++i) {
    w.key[i] = take((size_t)n * 4);
    w.pos[i] = take((size_t)n * 4);
  }
  w.hist = take((size_t)s.passes * s.nb * s.D * 4);
  w.head = take(pieces * H * 4);
  w.tail = take(pieces * H * 4);
  w.total = std::max<size_t>(o, 256);
  return w;
}

__device__ __forceinline__ int sort_key(int id, int V) { return id < 0 || id >= V ? V : id; }

// Digit counts of each block's keys for the first pass; clears the counts of the later passes.
__global__ void __launch_bounds__(256)
    k_sort_count(int64_t n, int V, SortPlan s, const int32_t* __restrict__ ids,
                 int* __restrict__ hist, int* status) {
  __shared__ int cnt[512];
  grid_dep_launch();
  for (int i = threadIdx.x; i < s.D; i += 256) cnt[i] = 0;
  grid_dep_wait();
  const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  const int64_t per = (int64_t)s.nb * s.D;
  for (int64_t i = per + first; i < per * s.passes; i += step) hist[i] = 0;
  __syncthreads();
  const int64_t end = min(n, (blockIdx.x + 1) * s.T);
  for (int64_t i = blockIdx.x * s.T + threadIdx.x; i < end; i += 256) {
    const int id = ids[i];
    if (id >= V && atomicCAS(status, 0, 2) == 0) atomicExch(status + 1, kSiteEmbedId);
    atomicAdd(&cnt[sort_key(id, V) & (s.D - 1)], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < s.D; i += 256) hist[(int64_t)blockIdx.x * s.D + i] = cnt[i];
}

// Stable ranks of the keys of a warp (its rows of 32, in order) among its keys of equal digit; cnt
// [512], zero before, gets the digits' counts.  A negative key takes no part.
__device__ __forceinline__ void warp_ranks(const int* key, int shift, int D, int* cnt, int* rank,
                                           int rows = 8) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (k >= rows) break;
    const int dig = key[k] < 0 ? -1 : (key[k] >> shift) & (D - 1);
    const unsigned peers = __match_any_sync(0xffffffffu, dig);
    const int lower = __popc(peers & ((1u << lane) - 1));
    const int old = dig < 0 ? 0 : cnt[dig];
    __syncwarp();
    if (dig >= 0 && lower == 0) cnt[dig] = old + __popc(peers);
    __syncwarp();
    rank[k] = old + lower;
  }
}

// Exclusive prefix sum over the block of v, sums [warps] in shared memory.
__device__ __forceinline__ int block_prefix(int v, int* sums) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int run = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += up;
  }
  if (lane == 31) sums[warp] = run;
  __syncthreads();
  int base = run - v;
  for (int w = 0; w < warp; ++w) base += sums[w];
  return base;
}

// One stable counting pass.  A key's place is: the keys of smaller digits, the same digit's keys of
// earlier blocks, of earlier tiles, of earlier warps, of earlier rows of its warp, and of lower lanes.
__global__ void __launch_bounds__(256)
    k_sort_pass(int64_t n, int V, SortPlan s, int pass, const int32_t* __restrict__ ids,
                const int32_t* __restrict__ key_in, const int32_t* __restrict__ pos_in,
                int32_t* __restrict__ key_out, int32_t* __restrict__ pos_out,
                int* __restrict__ hist) {
  __shared__ int off[512];     // next place of each digit
  __shared__ int cnt[8][512];  // per warp: counts, then first places
  __shared__ int sums[8];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  grid_dep_launch();
  grid_dep_wait();
  const int shift = pass * s.bits, D = s.D;
  const int* mine = hist + (int64_t)pass * s.nb * D;
  // two neighbouring digits a thread: 4 <= D <= 512
  int before[2] = {0, 0}, total[2] = {0, 0};
  if (2 * tid < D) {
#pragma unroll 16
    for (int b = 0; b < s.nb; ++b) {
      const int2 h = *reinterpret_cast<const int2*>(mine + (int64_t)b * D + 2 * tid);
      total[0] += h.x;
      total[1] += h.y;
      if (b < (int)blockIdx.x) {
        before[0] += h.x;
        before[1] += h.y;
      }
    }
  }
  const int base = block_prefix(total[0] + total[1], sums);
  if (2 * tid < D) {
    off[2 * tid] = base + before[0];
    off[2 * tid + 1] = base + total[0] + before[1];
  }
  const int64_t begin = blockIdx.x * s.T, end = min(n, begin + s.T);
  int* next = pass + 1 < s.passes ? hist + (int64_t)(pass + 1) * s.nb * D : nullptr;
  for (int64_t t0 = begin; t0 < end; t0 += kTile) {
    for (int i = tid; i < 8 * 512; i += 256) (&cnt[0][0])[i] = 0;
    __syncthreads();
    int key[8], rank[8], place[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t i = t0 + warp * 256 + k * 32 + lane;
      key[k] = i < end ? (pass == 0 ? sort_key(ids[i], V) : key_in[i]) : -1;
    }
    warp_ranks(key, shift, D, cnt[warp], rank);
    __syncthreads();
    for (int dg = tid; dg < D; dg += 256) {
      int at = off[dg];
      for (int w = 0; w < 8; ++w) {
        const int c = cnt[w][dg];
        cnt[w][dg] = at;
        at += c;
      }
      off[dg] = at;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (key[k] < 0) continue;
      const int64_t i = t0 + warp * 256 + k * 32 + lane;
      const int at = cnt[warp][(key[k] >> shift) & (D - 1)] + rank[k];
      key_out[at] = key[k];
      pos_out[at] = pass == 0 ? (int32_t)i : pos_in[i];
      place[k] = at;
    }
    if (next) {
      // counts for the next pass, one atomic for the keys of a warp row that go to the same one
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int to = key[k] < 0 ? -1
                                  : (int)((uint32_t)place[k] / (uint32_t)s.T) * D +
                                        ((key[k] >> (shift + s.bits)) & (D - 1));
        const unsigned peers = __match_any_sync(0xffffffffu, to);
        if (to >= 0 && (peers & ((1u << lane) - 1)) == 0) atomicAdd(&next[to], __popc(peers));
      }
    }
    __syncthreads();
  }
}

// All of it for at most kCluster * kClusterTile ids, in one cluster of blocks: each has a tile of the keys
// in shared memory and writes a key to where it goes, in its own or another block's.
constexpr int kCluster = 8, kClusterThreads = 512, kClusterTile = 4096;  // 16 warps x at most 8 x 32
struct ClusterSort {
  int cnt[16][512];  // per warp: counts, then first places
  int total[512];    // of the block
  int sums[16];
  int key[2][kClusterTile], pos[2][kClusterTile];
};

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address in block `rank` of the cluster of what is at p here.
__device__ __forceinline__ uint32_t cluster_addr(const void* p, int rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tc::smem_u32(p)), "r"(rank));
  return a;
}

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kClusterThreads)
    k_sort_cluster(int n, int V, SortPlan s, const int32_t* __restrict__ ids,
                   int32_t* __restrict__ key_out, int32_t* __restrict__ pos_out, int* status) {
  extern __shared__ __align__(16) uint8_t sort_smem[];
  ClusterSort& b = *reinterpret_cast<ClusterSort*>(sort_smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = blockIdx.x;
  // rows of 32 keys a warp: the blocks' tiles are as even as that allows
  const int per = (n + kCluster * kClusterThreads - 1) / (kCluster * kClusterThreads);
  const int tile = per * kClusterThreads;
  grid_dep_launch();
  grid_dep_wait();
  for (int p = 0; p < s.passes; ++p) {
    const int shift = p * s.bits;
    for (int i = tid; i < 16 * s.D; i += kClusterThreads) b.cnt[i / s.D][i % s.D] = 0;
    __syncthreads();
    int key[8], pos[8], order[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int at = (warp * per + k) * 32 + lane, i = rank * tile + at;
      key[k] = -1;
      pos[k] = i;
      if (k >= per || i >= n) continue;
      if (p == 0) {
        const int id = ids[i];
        if (id >= V && atomicCAS(status, 0, 2) == 0) atomicExch(status + 1, kSiteEmbedId);
        key[k] = sort_key(id, V);
      } else {
        key[k] = b.key[p & 1][at];
        pos[k] = b.pos[p & 1][at];
      }
    }
    warp_ranks(key, shift, s.D, b.cnt[warp], order, per);
    __syncthreads();
    if (tid < s.D) {
      int t = 0;
      for (int w = 0; w < 16; ++w) t += b.cnt[w][tid];
      b.total[tid] = t;
    }
    cluster_sync();
    int before = 0, total = 0;
    if (tid < s.D) {
#pragma unroll
      for (int r = 0; r < kCluster; ++r) {
        int t;
        asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(t) : "r"(cluster_addr(&b.total[tid], r)));
        total += t;
        before += r < rank ? t : 0;
      }
    }
    int at = block_prefix(total, b.sums) + before;
    if (tid < s.D)
      for (int w = 0; w < 16; ++w) {
        const int c = b.cnt[w][tid];
        b.cnt[w][tid] = at;
        at += c;
      }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (key[k] < 0) continue;
      const int to = b.cnt[warp][(key[k] >> shift) & (s.D - 1)] + order[k];
      if (p + 1 == s.passes) {
        key_out[to] = key[k];
        pos_out[to] = pos[k];
      } else {
        const int r = to / tile, slot = to - r * tile, buf = (p + 1) & 1;
        asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(cluster_addr(&b.key[buf][slot], r)), "r"(key[k])
                     : "memory");
        asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(cluster_addr(&b.pos[buf][slot], r)), "r"(pos[k])
                     : "memory");
      }
    }
    cluster_sync();  // (also: no block leaves while another may still read its totals)
  }
}

// All of it for at most kTile ids, in one block.
__global__ void __launch_bounds__(256)
    k_sort_small(int n, int V, SortPlan s, const int32_t* __restrict__ ids,
                 int32_t* __restrict__ key_out, int32_t* __restrict__ pos_out,
                 int* status) {
  __shared__ int cnt[8][512];
  __shared__ int sums[8];
  __shared__ int keys[kTile], poss[kTile];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  grid_dep_launch();
  grid_dep_wait();
  int key[8], pos[8], rank[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int i = warp * 256 + k * 32 + lane;
    pos[k] = i;
    key[k] = -1;
    if (i < n) {
      const int id = ids[i];
      if (id >= V && atomicCAS(status, 0, 2) == 0) atomicExch(status + 1, kSiteEmbedId);
      key[k] = sort_key(id, V);
    }
  }
  for (int p = 0; p < s.passes; ++p) {
    const int shift = p * s.bits;
    for (int i = tid; i < 8 * 512; i += 256) (&cnt[0][0])[i] = 0;
    __syncthreads();
    warp_ranks(key, shift, s.D, cnt[warp], rank);
    __syncthreads();
    int total[2] = {0, 0};
    if (2 * tid < s.D)
      for (int w = 0; w < 8; ++w) {
        total[0] += cnt[w][2 * tid];
        total[1] += cnt[w][2 * tid + 1];
      }
    int at = block_prefix(total[0] + total[1], sums);
    if (2 * tid < s.D)
      for (int j = 0; j < 2; ++j)
        for (int w = 0; w < 8; ++w) {
          const int c = cnt[w][2 * tid + j];
          cnt[w][2 * tid + j] = at;
          at += c;
        }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (key[k] >= 0) {
        const int to = cnt[warp][(key[k] >> shift) & (s.D - 1)] + rank[k];
        keys[to] = key[k];
        poss[to] = pos[k];
      }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = warp * 256 + k * 32 + lane;
      if (i < n) {
        key[k] = keys[i];
        pos[k] = poss[i];
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int i = warp * 256 + k * 32 + lane;
    if (i >= n) continue;
    key_out[i] = key[k];
    pos_out[i] = pos[k];
  }
}

// A row's finished sum to the table (adding in L2 instead, without reading the row, took twice as long).
__device__ __forceinline__ void add_row(float* acc, float* row, int accumulate) {
  if (accumulate) {
    float old[8];
    load8(row, old);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += old[j];
  }
  store8(row, acc);
}

__device__ __forceinline__ void copy16_async(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::smem_u32(dst)), "l"(src) : "memory");
}

// Sums of the rows of each piece of sorted positions, a group of threads a piece.  A token that lies
// within the piece is finished here; the part of one that began in an earlier piece goes to head[piece],
// of one that begins here and goes on to tail[piece].  Every block also writes the zero rows of its share
// of the table, the tokens that do not occur.
//
// The rows of dout come through rings in shared memory, kRing - 1 rows a group ahead.  Held in registers
// instead, the same number ahead, uniform tokens took 69 us for 131071 x 256 over 49999 (63 now); deeper or
// shallower rings with fewer or more blocks an SM take up to 5% longer.
__global__ void __launch_bounds__(256)
    k_embed_sum(int64_t n, int H, int V, SumPlan sp, const int32_t* __restrict__ key,
                const int32_t* __restrict__ pos, const float* __restrict__ dout, float scale,
                Drop d, float* __restrict__ dtable, int accumulate, float* __restrict__ head,
                float* __restrict__ tail) {
  extern __shared__ __align__(16) uint8_t sum_smem[];
  __shared__ uint8_t occurs[256];
  int* keys = reinterpret_cast<int*>(sum_smem + kRing * 8192);  // [groups * piece + 2]
  int* rows = keys + sp.groups * sp.piece + 2;                  // [groups * piece]
  const int g = threadIdx.x / sp.lanes, c = threadIdx.x % sp.lanes, lanes = H / 8;
  grid_dep_launch();
  grid_dep_wait();
  // the block's pieces lie side by side: their keys and rows come in one go, one more key on either side
  const int64_t first = (int64_t)blockIdx.x * sp.groups * sp.piece;
  const int run = (int)max((int64_t)0, min((int64_t)sp.groups * sp.piece, n - first));
  if (run > 0)
    for (int i = threadIdx.x; i < run + 2; i += 256) {
      const int64_t e = first + i - 1;
      keys[i] = e >= 0 && e < n ? key[e] : -1;
      if (i < run) rows[i] = pos[first + i];
    }
  __syncthreads();
  const int e0 = g * sp.piece, m = max(0, min(sp.piece, run - e0));
  const int warp_m = __reduce_max_sync(0xffffffffu, m);
  if (warp_m > 0) {
    const int* k0 = keys + 1 + e0;
    const int64_t q = first / sp.piece + g;
    // the warp's ring: rows of 1 KB, 32 bytes a thread
    uint8_t* ring = sum_smem + (threadIdx.x >> 5) * (kRing * 1024) + (threadIdx.x & 31 & ~(sp.lanes - 1)) * 32;
    auto fetch = [&](int i) {
      if (i < m && c < lanes && k0[i] < V) {
        const float* src = dout + (int64_t)rows[e0 + i] * H;
        uint8_t* dst = ring + i % kRing * 1024;
        copy16_async(dst + c * 16, src + c * 4);
        copy16_async(dst + (c + lanes) * 16, src + (c + lanes) * 4);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int cur = m > 0 ? k0[0] : V;
    bool begun = m > 0 && k0[-1] == cur;  // the first token began in an earlier piece
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto finish = [&](bool goes_on) {
      if (cur >= V || c >= lanes) return;
      const float f = d.thr ? scale * d.scale : scale;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] *= f;
      if (begun || goes_on) {
        store8((begun ? head : tail) + q * H + c * 8, acc);
      } else {
        add_row(acc, dtable + (int64_t)cur * H + c * 8, accumulate);
      }
    };
    for (int i = 0; i < kRing - 1; ++i) fetch(i);
    for (int i = 0; i < warp_m; ++i) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 2) : "memory");
      __syncwarp();
      if (i < m) {
        const int k = k0[i];
        if (k != cur) {
          finish(false);
          begun = false;
          cur = k;
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] = 0.f;
        }
        if (k < V && c < lanes) {
          float v[8];
          load8(reinterpret_cast<const float*>(ring + i % kRing * 1024) + c * 8, v);
          if (d.thr) drop8(d, (uint64_t)rows[e0 + i] * lanes + c, 1.f, v);
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] += v[j];
        }
      }
      // the place that the row before this one had: every lane has read it before the barrier above
      fetch(i + kRing - 1);
    }
    if (m > 0) finish(k0[m] == cur);
  }
  if (accumulate) return;
  const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  // (tokens blockIdx.x, + gridDim.x, ...: a share of the frequent and of the rare ones)
  const int share = (int)(((int64_t)V - blockIdx.x + gridDim.x - 1) / gridDim.x);
  for (int s0 = 0; s0 < share; s0 += 256) {
    if (s0 + threadIdx.x < share) {  // looked up among the sorted keys: the first of `mine` or more
      const int mine = blockIdx.x + (s0 + threadIdx.x) * gridDim.x;
      int lo = 0, hi = (int)n;
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (key[mid] < mine) lo = mid + 1; else hi = mid;
      }
      occurs[threadIdx.x] = lo < n && key[lo] == mine;
    }
    __syncthreads();
    if (c < lanes)
      for (int k = g; k < 256 && s0 + k < share; k += sp.groups)
        if (!occurs[k])
          store8(dtable + (blockIdx.x + (int64_t)(s0 + k) * gridDim.x) * H + c * 8, zero);
    __syncthreads();
  }
}

// Tokens that begin in piece q and go on: tail[q] + head[q + 1] + ... , in an order that depends on their
// count alone.  A group of threads takes a piece; tokens of more than kJoinFew pieces more are left to
// the whole block, whose groups take a run of the pieces each.
constexpr int kJoinFew = 16;
__global__ void __launch_bounds__(256)
    k_embed_join(int64_t n, int H, int V, int piece, const int32_t* __restrict__ key,
                 float* __restrict__ dtable, int accumulate, const float* __restrict__ head,
                 const float* __restrict__ tail) {
  __shared__ float part[256 * 8];
  __shared__ uint8_t many[64];
  grid_dep_wait();
  const int lanes = H / 8, groups = 256 / lanes;
  const int g = threadIdx.x / lanes, c = threadIdx.x % lanes;
  const int64_t q0 = (int64_t)blockIdx.x * groups, q = q0 + g, e0 = q * piece, e1 = e0 + piece;
  if (threadIdx.x < 64) many[threadIdx.x] = 0;
  __syncthreads();
  if (g < groups && e1 < n) {
    const int cur = key[e1 - 1];
    const bool begins = !(key[e0] == cur && e0 > 0 && key[e0 - 1] == cur);
    if (cur < V && key[e1] == cur && begins) {
      int next[kJoinFew];
#pragma unroll
      for (int i = 0; i < kJoinFew; ++i) next[i] = e1 + (int64_t)i * piece < n ? key[e1 + (int64_t)i * piece] : -1;
      int count = 0;
#pragma unroll
      for (int i = 0; i < kJoinFew; ++i) count += count == i && next[i] == cur;
      if (count == kJoinFew) {
        many[g] = 1;
      } else {
        float acc[8];
        load8(tail + q * H + c * 8, acc);
        for (int i = 1; i <= count; ++i) {
          float v[8];
          load8(head + (q + i) * H + c * 8, v);
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] += v[j];
        }
        add_row(acc, dtable + (int64_t)cur * H + c * 8, accumulate);
      }
    }
  }
  __syncthreads();
  for (int b = 0; b < groups; ++b) {
    if (!many[b]) continue;
    const int64_t qb = q0 + b;
    const int cur = key[(qb + 1) * piece];
    int64_t count = 1;  // pieces qb .. qb + count - 1
    for (int more = 256; more == 256; count += more) {
      const int64_t e = (qb + count + threadIdx.x) * piece;
      more = __syncthreads_count(e < n && key[e] == cur);
    }
    const int64_t per = (count + groups - 1) / groups;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (g < groups) {
      const int64_t end = min(count, (g + 1) * per);
#pragma unroll 4
      for (int64_t i = g * per; i < end; ++i) {
        float v[8];
        load8((i == 0 ? tail : head) + (qb + i) * H + c * 8, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += v[j];
      }
      store8(part + threadIdx.x * 8, acc);
    }
    __syncthreads();
    if (g == 0) {
      for (int o = 1; o < groups; ++o) {
        float v[8];
        load8(part + (o * lanes + c) * 8, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += v[j];
      }
      add_row(acc, dtable + (int64_t)cur * H + c * 8, accumulate);
    }
    __syncthreads();
  }
}

}  // namespace

cudaError_t dropout_fwd(int bf16, int64_t n, const Drop& d, const void* x, const void* res, void* y,
                        cudaStream_t st) {
  return bf16 ? run_dropout<__nv_bfloat16>(n, d, x, res, y, st)
              : run_dropout<float>(n, d, x, res, y, st);
}

cudaError_t dropout_bwd(int64_t n, const Drop& d, const float* dy, float* dx, int accumulate,
                        cudaStream_t st) {
  return run_dropout<float>(n, d, dy, accumulate ? dx : nullptr, dx, st);
}

cudaError_t embed_fwd(int bf16, int64_t n, int H, int V, const int32_t* ids, const void* table,
                      float scale, const Drop& d, void* out, int* status, cudaStream_t st) {
  if (n == 0) return cudaSuccess;
  const int rows = 256 / (H / 8) * kEmbedUnroll;
  const unsigned grid = (unsigned)((n + rows - 1) / rows);
  if (bf16)
    k_embed_fwd<__nv_bfloat16><<<grid, 256, 0, st>>>(n, H, V, ids,
                                                     static_cast<const __nv_bfloat16*>(table), scale,
                                                     d, static_cast<__nv_bfloat16*>(out), status);
  else
    k_embed_fwd<float><<<grid, 256, 0, st>>>(n, H, V, ids, static_cast<const float*>(table), scale,
                                             d, static_cast<float*>(out), status);
  note_launch();
  return cudaGetLastError();
}

size_t embed_bwd_ws_bytes(int64_t n, int H, int V) { return bwd_ws(n, H, V).total; }

cudaError_t embed_bwd(int64_t n, int H, int V, const int32_t* ids, const float* dout, float scale,
                      const Drop& d, float* dtable, int accumulate, void* ws, int* status,
                      cudaStream_t st) {
  if (n == 0)
    return accumulate ? cudaSuccess : cudaMemsetAsync(dtable, 0, (size_t)V * H * sizeof(float), st);
  const SortPlan s = sort_plan(n, V);
  const BwdWs w = bwd_ws(n, H, V);
  char* base = static_cast<char*>(ws);
  int32_t* key[2] = {reinterpret_cast<int32_t*>(base + w.key[0]),
                     reinterpret_cast<int32_t*>(base + w.key[1])};
  int32_t* pos[2] = {reinterpret_cast<int32_t*>(base + w.pos[0]),
                     reinterpret_cast<int32_t*>(base + w.pos[1])};
  int* hist = reinterpret_cast<int*>(base + w.hist);
  float* head = reinterpret_cast<float*>(base + w.head);
  float* tail = reinterpret_cast<float*>(base + w.tail);
  cudaError_t e;
  // 20001 ids of 10000 tokens: 17 us in one cluster, 26 as a count and two passes of many blocks (cold)
  const bool small = n <= kCluster * kClusterTile;
  if (n > kTile && small) {
    static std::atomic<uint64_t> done{0};
    e = allow_smem(k_sort_cluster, (int)sizeof(ClusterSort), done);
    if (e != cudaSuccess) return e;
    e = launch_pdl(k_sort_cluster, dim3(kCluster), dim3(kClusterThreads), sizeof(ClusterSort), st, (int)n, V,
                   s, ids, key[(s.passes - 1) & 1], pos[(s.passes - 1) & 1], status);
  } else if (small)
    e = launch_pdl(k_sort_small, dim3(1), dim3(256), 0, st, (int)n, V, s, ids, key[(s.passes - 1) & 1],
                   pos[(s.passes - 1) & 1], status);
  else
    e = launch_pdl(k_sort_count, dim3(s.nb), dim3(256), 0, st, n, V, s, ids, hist, status);
  if (e != cudaSuccess) return e;
  note_launch();
  for (int p = 0; p < s.passes && !small; ++p) {
    e = launch_pdl(k_sort_pass, dim3(s.nb), dim3(256), 0, st, n, V, s, p, ids, key[(p + 1) & 1],
                   pos[(p + 1) & 1], key[p & 1], pos[p & 1], hist);
    if (e != cudaSuccess) return e;
    note_launch();
  }
  const int32_t* k = key[(s.passes - 1) & 1];
  const int32_t* at = pos[(s.passes - 1) & 1];
  const SumPlan sp = sum_plan(n, H);
  // with few rows, blocks for the table's zeros
  const int64_t blocks =
      accumulate ? sp.blocks : std::max<int64_t>(sp.blocks, std::min<int64_t>((V + 127) / 128, 152 * 2));
  static std::atomic<uint64_t> done{0};
  e = allow_smem(k_embed_sum, kRing * 8192 + (2 * 64 * kMaxPiece + 4) * 4, done);  // the most it takes
  if (e != cudaSuccess) return e;
  e = launch_pdl(k_embed_sum, dim3((unsigned)blocks), dim3(256), sp.smem, st, n, H, V, sp, k, at, dout,
                 scale, d, dtable, accumulate, head, tail);
  if (e != cudaSuccess) return e;
  note_launch();
  if (sp.pieces == 1) return cudaSuccess;
  const int groups = 256 / (H / 8);
  e = launch_pdl(k_embed_join, dim3((unsigned)((sp.pieces + groups - 1) / groups)), dim3(256), 0, st, n,
                 H, V, sp.piece, k, dtable, accumulate, head, tail);
  if (e != cudaSuccess) return e;
  note_launch();
  return cudaSuccess;
}

}  // namespace bg
