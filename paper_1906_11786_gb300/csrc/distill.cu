// Distillation from a teacher's largest logits: a row has up to K entries (token t_k, logit u_k), and
//   q = softmax(u / tau) over them,  z = X W^T,  lse_i = log sum_v exp(z_iv / tau)
//   loss_i = tau^2 (sum_k q_k (log q_k - z_{i,t_k} / tau) + lse_i)
//   d = g_i tau (softmax(z_i / tau) - q_i),  dX = d W,  dW = d^T X
//
// What runs over the whole vocabulary is the cross entropy's (xent.cu), with a temperature and without a
// target: lse, and the products with the probabilities P.  The teacher's side is sparse, and its own:
//   k_distill_rows   a warp a row; the rows of W that its entries name come from L2 (W is some tens of MB):
//                    sum_k q_k (log q_k - z_k / tau) forward, sum_k c_k w_k backward
//   token_sum        sum of c_k x_i by token (embed.cu: stable sort, pieces, joins; no float atomics)
// The sparse sums are written first, in fp32, and the dense kernels add to them: a bf16 gradient is rounded
// once.  The dense products take P rounded to bf16 there, which where P is near Q would be worse than the
// gradient's own rounding; so c_k also holds what that rounding took from the entry's own P (whose z is a
// product of H terms, computed again): the entries' coefficients P - Q are exact to fp32, and only tokens
// without an entry, whose whole coefficient is P, have it rounded.
//
// 65537 rows x 49999 x 256 bf16 with 32 entries: 5.8 ms forward and backward, of which the dense products take 4.6-4.9
// (xent.cu), the rows 0.12 and 0.19 (1.07 GB each from L2: 8.8 TB/s forward; backward also two more passes over the
// registers), the sort of 2.1 M entries 0.14 and their sums 0.31.  15% of 71969 rows x 10000 x 64, 16 entries, fp32
// gradients: 328 us, a chain of fifteen kernels.
#include <cuda_bf16.h>

#include <algorithm>

#include "answer.h"
#include "kernels.h"
#include "tc_util.cuh"
#include "token.h"

namespace bg {

using tc::grid_dep_launch;
using tc::grid_dep_wait;

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWarps = 8;
constexpr int kMaxEntries = kMaxTop;

enum { kForward, kBackward, kCorrected };  // kCorrected: bf16 gradients

struct RowArgs {
  int64_t n;
  int H, V, K, width;  // width: threads of an entry, H / 8 rounded up to a power of two
  const void* X;
  const void* W;
  const int32_t* top_id;
  const float* top_logit;
  float inv_tau, tau;
  int32_t* mark;  // [n] 0: the row has entries, -1: it has none
  float* inner;   // forward: sum_k q_k (log q_k - z_k / tau)
  // backward
  const float* lse;
  const float* dloss;
  float* dX;       // fp32 sums of the rows (NULL: not wanted)
  int accumulate;  // they are added to
  int32_t* id;     // [n][K] tokens of the entries, -1: none (NULL: no dW wanted)
  float* c;        // [n][K] their coefficients for dW
  int* status;
};

struct Entry {
  int id;
  float q, other;  // other: log q, then z (forward); bits: first of its token (corrected)
};

__device__ __forceinline__ void load8(const float* p, float* v) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float* v) {
  const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
  const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(u[j] << 16);
    v[2 * j + 1] = __uint_as_float(u[j] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <typename T, int MODE>
__global__ void __launch_bounds__(kWarps * 32) k_distill_rows(const __grid_constant__ RowArgs a) {
  __shared__ Entry entries[kWarps][kMaxEntries];
  const int lane = threadIdx.x & 31;
  const int64_t i = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  Entry* e = entries[threadIdx.x >> 5];
  grid_dep_launch();
  grid_dep_wait();
  if (i >= a.n) return;
  // the teacher's distribution, a lane an entry (four of them at most)
  constexpr int E = kMaxEntries / 32;
  float u[E];
  int id[E];
  float high = -INFINITY;
  bool some = false;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    const int k = j * 32 + lane;
    id[j] = -1;
    u[j] = -INFINITY;
    if (k >= a.K) continue;
    const int t = a.top_id[i * a.K + k];
    const float x = a.top_logit[i * a.K + k];
    if (t >= a.V && atomicCAS(a.status, 0, 2) == 0) atomicExch(a.status + 1, kSiteTeacherId);
    if (t < 0 || t >= a.V || x == -INFINITY) continue;
    id[j] = t;
    u[j] = x;
    some = true;
    high = fmaxf(high, u[j]);
  }
  some = __any_sync(0xffffffffu, some);
  if (lane == 0) a.mark[i] = some ? 0 : -1;
  const bool keep_dx = MODE != kForward && a.dX;
  const int q0 = lane & (a.width - 1), at = q0 * 8;  // the lane's 8 elements of a row
  const bool in = at < a.H;
  if (!some) {
    if (MODE != kForward) {
      if (keep_dx && !a.accumulate)
        for (int c = lane * 4; c < a.H; c += 128)
          *reinterpret_cast<float4*>(a.dX + i * a.H + c) = make_float4(0.f, 0.f, 0.f, 0.f);
      if (a.id)
        for (int k = lane; k < a.K; k += 32) a.id[i * a.K + k] = -1;
    }
    return;
  }
  high = warp_max(high);
  float sum = 0.f;
  // (the largest is taken off before tau divides: the type's lowest value stays an entry, with q = 0 beside larger ones)
#pragma unroll
  for (int j = 0; j < E; ++j) {
    u[j] = (u[j] - high) * a.inv_tau;
    sum += id[j] < 0 ? 0.f : expf(u[j]);
  }
  sum = warp_sum(sum);
  const float log_sum = logf(sum), inv = 1.f / sum;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    const int k = j * 32 + lane;
    if (k < a.K) e[k] = Entry{id[j], id[j] < 0 ? 0.f : expf(u[j]) * inv, u[j] - log_sum};
  }
  __syncwarp();
  if (MODE == kCorrected) {
    // an entry is the first of its token: what rounding took from P counts once
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const int k = j * 32 + lane;
      if (k >= a.K) continue;
      bool first = true;
      for (int p = 0; p < k; ++p) first &= e[p].id != id[j];
      e[k].other = first ? 1.f : 0.f;
    }
    __syncwarp();
  }
  float x[8], acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = acc[j] = 0.f;
  if (MODE != kBackward && in) load8(static_cast<const T*>(a.X) + i * a.H + at, x);
  const int groups = 32 / a.width, group = lane / a.width;
  const float g = MODE == kForward ? 0.f : a.dloss[i] * a.tau;
  const float nlse = MODE == kCorrected ? -safe_lse(a.lse[i]) * kLog2e : 0.f, l2e = kLog2e * a.inv_tau;
  const bool rows = MODE != kBackward || a.dX;  // rows of W are needed
  float inner = 0.f;
  // Four rows of W at a time: their products with x are added up over the row's threads so that thread t ends with
  // the product of entry t mod 4, makes that entry's coefficient, and hands it to the others.
  constexpr int U = 4;
  for (int k0 = 0; k0 < a.K; k0 += U * groups) {
    float w[U][8];
    bool there[U];
#pragma unroll
    for (int s = 0; s < U; ++s) {
      const int k = k0 + s * groups + group, t = k < a.K ? e[k].id : -1;
      there[s] = t >= 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) w[s][j] = 0.f;
      if (rows && t >= 0 && in) load8(static_cast<const T*>(a.W) + (int64_t)t * a.H + at, w[s]);
    }
    const int mine = k0 + (lane & 3) * groups + group;
    const Entry en = mine < a.K ? e[mine] : Entry{-1, 0.f, 0.f};
    float z = 0.f;
    if (MODE != kBackward) {
      float p[U];
#pragma unroll
      for (int s = 0; s < U; ++s) {
        p[s] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) p[s] = fmaf(x[j], w[s][j], p[s]);
      }
      const bool odd = lane & 1, high = lane & 2;
      const float x01 = (odd ? p[1] : p[0]) + __shfl_xor_sync(0xffffffffu, odd ? p[0] : p[1], 1);
      const float x23 = (odd ? p[3] : p[2]) + __shfl_xor_sync(0xffffffffu, odd ? p[2] : p[3], 1);
      z = (high ? x23 : x01) + __shfl_xor_sync(0xffffffffu, high ? x01 : x23, 2);
      for (int o = 4; o < a.width; o <<= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
    }
    if (MODE == kForward) {
      if (q0 < U && en.id >= 0 && en.q != 0.f) inner += en.q * (en.other - z * a.inv_tau);
      continue;
    }
    float cx = -en.q, cw = -g * en.q;
    if (MODE == kCorrected && en.other != 0.f) {
      // the dense kernels' P: bf16(p) for dX, bf16(g p) for dW
      const float p = ex2(fmaf(z, l2e, nlse)), gp = p * g;
      cx += p - __bfloat162float(__float2bfloat16(p));
      cw += gp - __bfloat162float(__float2bfloat16(gp));
    }
    if (q0 < U && mine < a.K && a.id) {
      a.id[i * a.K + mine] = en.id;
      a.c[i * a.K + mine] = cw;
    }
    if (!rows) continue;
#pragma unroll
    for (int s = 0; s < U; ++s) {
      const float c = __shfl_sync(0xffffffffu, cx, (lane & ~3) | s);
      if (there[s]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = fmaf(c, w[s][j], acc[j]);
      }
    }
  }
  if (MODE == kForward) {
    inner = warp_sum(inner);
    if (lane == 0) a.inner[i] = inner;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      for (int o = a.width; o < 32; o <<= 1) acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], o);
  }
  if (keep_dx && group == 0 && in) {
    float4* d = reinterpret_cast<float4*>(a.dX + i * a.H + at);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float4 v = make_float4(acc[4 * h] * g, acc[4 * h + 1] * g, acc[4 * h + 2] * g, acc[4 * h + 3] * g);
      if (a.accumulate) {
        const float4 old = d[h];
        v = make_float4(v.x + old.x, v.y + old.y, v.z + old.z, v.w + old.w);
      }
      d[h] = v;
    }
  }
}

inline size_t al(size_t x) { return (x + 255) & ~(size_t)255; }

struct Ws {
  size_t mark, inner, id, c, add_x, add_w, sum, xent, total;
};
Ws layout(int bf16, int64_t n, int H, int V, int K, int backward) {
  Ws w{};
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += al(bytes);
    return at;
  };
  w.mark = take((size_t)n * 4);
  if (backward) {
    w.id = take((size_t)n * K * 4);
    w.c = take((size_t)n * K * 4);
    w.add_x = take(bf16 ? (size_t)n * H * 4 : 0);
    w.add_w = take(bf16 ? (size_t)V * H * 4 : 0);
    w.sum = take(token_sum_ws_bytes(n * K, H, V));
  } else {
    w.inner = take((size_t)n * 4);
  }
  w.xent = take(xent_ws_bytes(bf16, n, H, V, backward));
  w.total = o;
  return w;
}

template <int MODE>
cudaError_t rows(const DistillArgs& d, RowArgs r, cudaStream_t st) {
  r.n = d.n;
  r.H = d.H;
  r.V = d.V;
  r.K = d.K;
  r.width = d.H / 8 <= 4 ? 4 : d.H / 8 <= 8 ? 8 : d.H / 8 <= 16 ? 16 : 32;
  r.X = d.X;
  r.W = d.W;
  r.top_id = d.top_id;
  r.top_logit = d.top_logit;
  r.inv_tau = 1.f / d.tau;
  r.tau = d.tau;
  r.status = d.status;
  const dim3 grid((unsigned)((d.n + kWarps - 1) / kWarps)), block(kWarps * 32);
  const cudaError_t e = d.bf16 ? launch_pdl(k_distill_rows<__nv_bfloat16, MODE>, grid, block, 0, st, r)
                               : launch_pdl(k_distill_rows<float, MODE>, grid, block, 0, st, r);
  if (e == cudaSuccess) note_launch();
  return e;
}

}  // namespace

size_t distill_ws_bytes(int bf16, int64_t n, int H, int V, int K, int backward) {
  return layout(bf16, n, H, V, K, backward).total;
}

cudaError_t distill_fwd(const DistillArgs& d, float* loss, float* lse, cudaStream_t st) {
  if (d.n == 0) return cudaSuccess;
  const Ws w = layout(d.bf16, d.n, d.H, d.V, d.K, 0);
  char* base = static_cast<char*>(d.ws);
  RowArgs r{};
  r.mark = reinterpret_cast<int32_t*>(base + w.mark);
  r.inner = reinterpret_cast<float*>(base + w.inner);
  const cudaError_t e = rows<kForward>(d, r, st);
  if (e != cudaSuccess) return e;
  const XentSoft soft{d.tau, r.inner, nullptr, nullptr};
  const XentArgs x{d.bf16, d.n, d.H, d.V, d.X, d.W, r.mark, base + w.xent, d.status, &soft};
  return xent_fwd(x, loss, lse, st);
}

cudaError_t distill_bwd(const DistillArgs& d, const float* lse, const float* dloss, int grad_bf16, void* dX,
                        void* dW, int accumulate, cudaStream_t st) {
  if (d.n == 0) {
    if (!dW || accumulate) return cudaSuccess;
    return cudaMemsetAsync(dW, 0, (size_t)d.V * d.H * (grad_bf16 ? 2 : 4), st);
  }
  const Ws w = layout(d.bf16, d.n, d.H, d.V, d.K, 1);
  char* base = static_cast<char*>(d.ws);
  // fp32 gradients: the sparse sums are written where the dense ones are added to them
  float* add_x = !dX ? nullptr : grad_bf16 ? reinterpret_cast<float*>(base + w.add_x) : static_cast<float*>(dX);
  float* add_w = !dW ? nullptr : grad_bf16 ? reinterpret_cast<float*>(base + w.add_w) : static_cast<float*>(dW);
  RowArgs r{};
  r.mark = reinterpret_cast<int32_t*>(base + w.mark);
  r.lse = lse;
  r.dloss = dloss;
  r.dX = add_x;
  r.accumulate = accumulate;
  r.id = dW ? reinterpret_cast<int32_t*>(base + w.id) : nullptr;
  r.c = reinterpret_cast<float*>(base + w.c);
  cudaError_t e = grad_bf16 ? rows<kCorrected>(d, r, st) : rows<kBackward>(d, r, st);
  if (e != cudaSuccess) return e;
  if (dW) {
    e = token_sum(d.n * d.K, d.H, d.V, r.id, d.bf16, d.X, d.K, r.c, add_w, accumulate, base + w.sum, d.status, st);
    if (e != cudaSuccess) return e;
  }
  const XentSoft soft{d.tau, nullptr, grad_bf16 ? add_x : nullptr, grad_bf16 ? add_w : nullptr};
  const XentArgs x{d.bf16, d.n, d.H, d.V, d.X, d.W, r.mark, base + w.xent, d.status, &soft};
  return xent_bwd(x, lse, dloss, grad_bf16, dX, dW, !grad_bf16, st);
}

}  // namespace bg
