// Dropout with a mask that is never stored, and the embedding lookup that makes initial node
// states with its gradient by sorted tokens.
//
// Every kernel here moves bytes and does little arithmetic; a thread works on 8 consecutive
// elements, the elements of one generator block (philox.h), as one 16-byte (bf16) or two 16-byte
// (fp32) accesses.
#include <cuda_bf16.h>

#include <algorithm>

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
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

// ------------------------------------------------------------------------------ dropout
// y = add + drop(x), add = res (forward) or y's own values (a gradient that accumulates).  x, res
// and y may be the same array: a thread reads its elements before it writes them.
template <typename T>
__global__ void __launch_bounds__(256)
    k_dropout(int64_t n, Drop d, const T* x, const T* res, T* y) {
  const int64_t full = n / 8, blocks = (n + 7) / 8;
  for (int64_t b = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; b < blocks;
       b += (int64_t)gridDim.x * blockDim.x) {
    const int64_t i = b * 8;
    float v[8], r[8];
    if (b < full) {
      load8(x + i, v);
      if (res) load8(res + i, r);
      if (d.thr) drop8(d, (uint64_t)b, v);
      if (res) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += r[j];
      }
      store8(y + i, v);
    } else {
      const int m = (int)(n - i);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = j < m ? load1(x + i + j) : 0.f;
        r[j] = j < m && res ? load1(res + i + j) : 0.f;
      }
      if (d.thr) drop8(d, (uint64_t)b, v);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < m) store1(y + i + j, res ? v[j] + r[j] : v[j]);
    }
  }
}

template <typename T>
cudaError_t run_dropout(int64_t n, const Drop& d, const void* x, const void* res, void* y,
                        cudaStream_t st) {
  if (n == 0) return cudaSuccess;
  const int64_t blocks = (n + 7) / 8;
  const int grid = (int)std::min<int64_t>((blocks + 255) / 256, 152 * 8);
  k_dropout<T><<<grid, 256, 0, st>>>(n, d, static_cast<const T*>(x), static_cast<const T*>(res),
                                     static_cast<T*>(y));
  note_launch();
  return cudaGetLastError();
}

// ------------------------------------------------------------------------------ embedding lookup
// A row is H / 8 threads; a block takes 256 / (H / 8) rows at a time.
template <typename T>
__global__ void __launch_bounds__(256)
    k_embed_fwd(int64_t n, int H, int V, const int32_t* __restrict__ ids,
                const T* __restrict__ table, float scale, Drop d, T* __restrict__ out, int* status) {
  const int lanes = H / 8, rows = 256 / lanes;
  const int r = threadIdx.x / lanes, c = threadIdx.x % lanes;
  if (r >= rows) return;
  for (int64_t i = (int64_t)blockIdx.x * rows + r; i < n; i += (int64_t)gridDim.x * rows) {
    const int id = ids[i];
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (id >= V) {
      if (c == 0 && atomicCAS(status, 0, 2) == 0) atomicExch(status + 1, kSiteEmbedId);
    } else if (id >= 0) {
      load8(table + (int64_t)id * H + c * 8, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= scale;
      if (d.thr) drop8(d, (uint64_t)i * lanes + c, v);
    }
    store8(out + i * H + c * 8, v);
  }
}

// ------------------------------------------------------------------------------ embedding gradient
// The rows of dout are summed by token in three steps that give the same bits every time: a stable
// radix sort of (id, position), sums over pieces of kPiece sorted positions, and a join of the
// tokens that span pieces, in the order of the pieces.  An id that names no row sorts as V, after
// all others, and is not summed.
constexpr int kTile = 2048;  // keys a sorting block ranks at a time: 8 warps x 8 x 32
constexpr int kPiece = 32;

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
  s.bits = (bits + s.passes - 1) / s.passes;
  s.D = 1 << s.bits;
  s.T = kTile * std::max<int64_t>(1, (n + (int64_t)kTile * 152 - 1) / ((int64_t)kTile * 152));
  s.nb = (int)std::max<int64_t>(1, (n + s.T - 1) / s.T);
  return s;
}

inline size_t al(size_t x) { return (x + 255) & ~(size_t)255; }

struct BwdWs {
  size_t key[2], pos[2], hist, seen, head, tail, total;
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
  const size_t pieces = (size_t)((n + kPiece - 1) / kPiece);
  for (int i = 0; i < 2; ++i) {
    w.key[i] = take((size_t)n * 4);
    w.pos[i] = take((size_t)n * 4);
  }
  w.hist = take((size_t)s.passes * s.nb * s.D * 4);
  w.seen = take((size_t)V);
  w.head = take(pieces * H * 4);
  w.tail = take(pieces * H * 4);
  w.total = std::max<size_t>(o, 256);
  return w;
}

__device__ __forceinline__ int sort_key(int id, int V) { return id < 0 || id >= V ? V : id; }

// Digit counts of each block's keys for the first pass; clears the counts of the later passes and
// the marks of the tokens that occur.
__global__ void __launch_bounds__(256)
    k_sort_count(int64_t n, int V, SortPlan s, const int32_t* __restrict__ ids,
                 int* __restrict__ hist, uint8_t* __restrict__ seen, int* status) {
  __shared__ int cnt[512];
  grid_dep_launch();
  for (int i = threadIdx.x; i < s.D; i += 256) cnt[i] = 0;
  grid_dep_wait();
  const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  const int64_t per = (int64_t)s.nb * s.D;
  for (int64_t i = per + first; i < per * s.passes; i += step) hist[i] = 0;
  for (int64_t i = first; i < V; i += step) seen[i] = 0;
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

// One stable counting pass.  A key's place is: the keys of smaller digits, the same digit's keys of
// earlier blocks, of earlier tiles, of earlier warps, of earlier rows of its warp, and of lower lanes.
__global__ void __launch_bounds__(256)
    k_sort_pass(int64_t n, int V, SortPlan s, int pass, const int32_t* __restrict__ ids,
                const int32_t* __restrict__ key_in, const int32_t* __restrict__ pos_in,
                int32_t* __restrict__ key_out, int32_t* __restrict__ pos_out,
                int* __restrict__ hist, uint8_t* __restrict__ seen) {
  __shared__ int off[512];     // next place of each digit
  __shared__ int cnt[8][512];  // per warp: counts, then first places
  __shared__ int sums[8];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  grid_dep_launch();
  grid_dep_wait();
  const int shift = pass * s.bits, D = s.D;
  const int* mine = hist + (int64_t)pass * s.nb * D;
  // two neighbouring digits a thread: D <= 512
  int before[2] = {0, 0}, total[2] = {0, 0};
  for (int j = 0; j < 2; ++j) {
    const int d = 2 * tid + j;
    if (d < D)
      for (int b = 0; b < s.nb; ++b) {
        const int h = mine[(int64_t)b * D + d];
        total[j] += h;
        if (b < (int)blockIdx.x) before[j] += h;
      }
  }
  int run = total[0] + total[1];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += up;
  }
  if (lane == 31) sums[warp] = run;
  __syncthreads();
  int base = run - total[0] - total[1];
  for (int w = 0; w < warp; ++w) base += sums[w];
  if (2 * tid < D) off[2 * tid] = base + before[0];
  if (2 * tid + 1 < D) off[2 * tid + 1] = base + total[0] + before[1];
  const int64_t begin = blockIdx.x * s.T, end = min(n, begin + s.T);
  int* next = pass + 1 < s.passes ? hist + (int64_t)(pass + 1) * s.nb * D : nullptr;
  for (int64_t t0 = begin; t0 < end; t0 += kTile) {
    for (int i = tid; i < 8 * 512; i += 256) (&cnt[0][0])[i] = 0;
    __syncthreads();
    int key[8], rank[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t i = t0 + warp * 256 + k * 32 + lane;
      key[k] = i < end ? (pass == 0 ? sort_key(ids[i], V) : key_in[i]) : -1;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int dig = key[k] < 0 ? -1 : (key[k] >> shift) & (D - 1);
      const unsigned peers = __match_any_sync(0xffffffffu, dig);
      const int lower = __popc(peers & ((1u << lane) - 1));
      const int old = dig < 0 ? 0 : cnt[warp][dig];
      __syncwarp();
      if (dig >= 0 && lower == 0) cnt[warp][dig] = old + __popc(peers);
      __syncwarp();
      rank[k] = old + lower;
    }
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
      if (next) atomicAdd(&next[(int64_t)(at / s.T) * D + ((key[k] >> (shift + s.bits)) & (D - 1))], 1);
      if (pass == 0 && key[k] < V) seen[key[k]] = 1;
    }
    __syncthreads();
  }
}

// Sums of the rows of each piece of kPiece sorted positions, one group of H / 8 threads a piece.
// A token that lies within the piece is finished here; the part of one that began in an earlier
// piece goes to head[piece], of one that begins here and goes on to tail[piece].  The blocks from
// `sum_blocks` on write the zero rows of the tokens that do not occur.
__global__ void __launch_bounds__(256)
    k_embed_sum(int64_t n, int H, int V, const int32_t* __restrict__ key,
                const int32_t* __restrict__ pos, const float* __restrict__ dout, float scale,
                Drop d, float* __restrict__ dtable, int accumulate, float* __restrict__ head,
                float* __restrict__ tail, const uint8_t* __restrict__ seen, int sum_blocks) {
  const int lanes = H / 8, groups = 256 / lanes;
  const int g = threadIdx.x / lanes, c = threadIdx.x % lanes;
  grid_dep_launch();
  grid_dep_wait();
  if (g >= groups) return;
  if ((int)blockIdx.x >= sum_blocks) {
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int64_t v = (int64_t)(blockIdx.x - sum_blocks) * groups + g; v < V;
         v += (int64_t)(gridDim.x - sum_blocks) * groups)
      if (!seen[v]) store8(dtable + v * H + c * 8, zero);
    return;
  }
  const int64_t pieces = (n + kPiece - 1) / kPiece;
  for (int64_t q = (int64_t)blockIdx.x * groups + g; q < pieces; q += (int64_t)sum_blocks * groups) {
    const int64_t e0 = q * kPiece;
    const int m = (int)min((int64_t)kPiece, n - e0);
    int cur = key[e0];
    bool begun = e0 > 0 && key[e0 - 1] == cur;  // the first token began in an earlier piece
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto finish = [&](bool goes_on) {
      if (cur >= V) return;
      const float f = d.thr ? scale * d.scale : scale;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] *= f;
      if (begun || goes_on) {
        store8((begun ? head : tail) + q * H + c * 8, acc);
      } else {
        float* row = dtable + (int64_t)cur * H + c * 8;
        if (accumulate) {
          float old[8];
          load8(row, old);
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] += old[j];
        }
        store8(row, acc);
      }
    };
    for (int i0 = 0; i0 < m; i0 += 4) {
      float v[4][8];
      int k[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        k[u] = i0 + u < m ? key[e0 + i0 + u] : V;
        if (k[u] < V) {
          const int64_t i = pos[e0 + i0 + u];
          load8(dout + i * H + c * 8, v[u]);
          if (d.thr) {
            const uint4 w = philox_block(d, (uint64_t)i * lanes + c);
            const uint32_t b[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (((b[j / 2] >> (16 * (j & 1))) & 0xFFFFu) < d.thr) v[u][j] = 0.f;
          }
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (i0 + u >= m) break;
        if (k[u] != cur) {
          finish(false);
          begun = false;
          cur = k[u];
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] = 0.f;
        }
        if (cur < V) {
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] += v[u][j];
        }
      }
    }
    finish(e0 + m < n && key[e0 + m] == cur);
  }
}

// One block a piece in which a token begins that goes on: its sum is tail[piece] + head[piece + 1] +
// ... in that order of quarters; each group of threads takes one run of the pieces.
__global__ void __launch_bounds__(256)
    k_embed_join(int64_t n, int H, int V, const int32_t* __restrict__ key,
                 float* __restrict__ dtable, int accumulate, const float* __restrict__ head,
                 const float* __restrict__ tail) {
  __shared__ float part[256 * 8];
  grid_dep_wait();
  const int64_t q = blockIdx.x, e0 = q * kPiece, e1 = e0 + kPiece;
  if (e1 >= n) return;
  const int cur = key[e1 - 1];
  if (cur >= V || key[e1] != cur) return;
  if (key[e0] == cur && e0 > 0 && key[e0 - 1] == cur) return;  // began earlier
  // the last position of the token: the first of a larger key, less one
  int64_t lo = e1, hi = n;
  while (lo + 1 < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (key[mid] == cur) lo = mid; else hi = mid;
  }
  const int64_t last = lo / kPiece, count = last - q + 1;  // pieces q .. last
  const int lanes = H / 8, groups = 256 / lanes;
  const int g = threadIdx.x / lanes, c = threadIdx.x % lanes;
  const int64_t per = (count + groups - 1) / groups;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (g < groups) {
    const int64_t end = min(count, (g + 1) * per);
    for (int64_t i = g * per; i < end; ++i) {
      float v[8];
      load8((i == 0 ? tail : head) + (q + i) * H + c * 8, v);
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
    float* row = dtable + (int64_t)cur * H + c * 8;
    if (accumulate) {
      float old[8];
      load8(row, old);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += old[j];
    }
    store8(row, acc);
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
  const int rows = 256 / (H / 8);
  const int grid = (int)std::min<int64_t>((n + rows - 1) / rows, 152 * 8);
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
  uint8_t* seen = reinterpret_cast<uint8_t*>(base + w.seen);
  float* head = reinterpret_cast<float*>(base + w.head);
  float* tail = reinterpret_cast<float*>(base + w.tail);
  cudaError_t e = launch_pdl(k_sort_count, dim3(s.nb), dim3(256), 0, st, n, V, s, ids, hist, seen,
                             status);
  if (e != cudaSuccess) return e;
  note_launch();
  for (int p = 0; p < s.passes; ++p) {
    e = launch_pdl(k_sort_pass, dim3(s.nb), dim3(256), 0, st, n, V, s, p, ids, key[(p + 1) & 1],
                   pos[(p + 1) & 1], key[p & 1], pos[p & 1], hist, seen);
    if (e != cudaSuccess) return e;
    note_launch();
  }
  const int32_t* k = key[(s.passes - 1) & 1];
  const int32_t* at = pos[(s.passes - 1) & 1];
  const int groups = 256 / (H / 8);
  const int64_t pieces = (n + kPiece - 1) / kPiece;
  const int sum_blocks = (int)std::min<int64_t>((pieces + groups - 1) / groups, 152 * 16);
  const int zero_blocks =
      accumulate ? 0 : (int)std::min<int64_t>(((int64_t)V + 16 * groups - 1) / (16 * groups), 152 * 4);
  e = launch_pdl(k_embed_sum, dim3(sum_blocks + zero_blocks), dim3(256), 0, st, n, H, V, k, at, dout,
                 scale, d, dtable, accumulate, head, tail, seen, sum_blocks);
  if (e != cudaSuccess) return e;
  note_launch();
  e = launch_pdl(k_embed_join, dim3((unsigned)pieces), dim3(256), 0, st, n, H, V, k, dtable,
                 accumulate, head, tail);
  if (e != cudaSuccess) return e;
  note_launch();
  return cudaSuccess;
}

}  // namespace bg
