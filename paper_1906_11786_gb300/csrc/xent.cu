// Softmax cross entropy of node states against a vocabulary, in pieces of the vocabulary, with its
// gradient; the [n, V] logits are never in memory:
//   z = X W^T,  lse_i = log sum_v exp(z_iv),  loss_i = lse_i - z_{i,t_i}
//   P = softmax(z) - onehot(t),  dX = diag(g) P W,  dW = P^T diag(g) X     (g: the loss's gradient)
// A block keeps 64 rows of one side (X for the loss and dX, W for dW), walks the other side 64 rows
// at a time and recomputes the 64 x 64 logits between them; the gradients take exp(z - lse) from the
// forward's lse.  Everything is fp32 in shared memory and registers.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "kernels.h"
#include "token.h"

namespace bg {

namespace {

enum Mode { kLoss = 0, kDX = 1, kDW = 2 };

struct XentKernel {
  int64_t n;
  int H, V;
  const void* X;
  const void* W;
  const int32_t* target;
  float* loss;
  float* lse;         // written by the loss, read by the gradients
  const float* dloss;
  void* grad;
  int grad_bf16, accumulate;
  int* status;
};

__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const __nv_bfloat16* p) { return __bfloat162float(*p); }

__device__ __forceinline__ int row_target(const XentKernel& k, int64_t i) {
  if (i >= k.n) return -1;
  const int t = k.target[i];
  if (t >= k.V) {
    if (atomicCAS(k.status, 0, 2) == 0) atomicExch(k.status + 1, kSiteXentTarget);
    return -1;
  }
  return t;
}

template <typename T, int MODE>
__global__ void __launch_bounds__(256) k_xent(XentKernel k) {
  extern __shared__ float sm[];
  const int H = k.H, ld_ = H + 1;
  float* A = sm;              // [64][H + 1]: the rows that stay
  float* B = A + 64 * ld_;    // [64][H + 1]: the rows that pass
  float* P = B + 64 * ld_;    // [64][65]
  float* top = P + 64 * 65;   // per staying row: running maximum and sum (kLoss)
  float* sum = top + 64;
  float* hit = sum + 64;      // the target's logit
  float* slse = hit + 64;     // of the X rows at hand
  float* sg = slse + 64;
  int* tgt = reinterpret_cast<int*>(sg + 64);
  const int tid = threadIdx.x;
  const T* X = static_cast<const T*>(k.X);
  const T* W = static_cast<const T*>(k.W);
  const int64_t a0 = (int64_t)blockIdx.x * 64;
  const int64_t na = MODE == kDW ? k.V : k.n, nb = MODE == kDW ? k.n : k.V;
  auto load_x = [&](float* dst, int64_t i0) {
    if (tid < 64) {
      const int t = row_target(k, i0 + tid);
      tgt[tid] = t;
      slse[tid] = MODE != kLoss && t >= 0 ? k.lse[i0 + tid] : 0.f;
      sg[tid] = MODE != kLoss && t >= 0 ? k.dloss[i0 + tid] : 0.f;
    }
    __syncthreads();
    for (int e = tid; e < 64 * H; e += 256) {
      const int r = e / H, h = e % H;
      dst[r * ld_ + h] = tgt[r] >= 0 ? ld(X + (i0 + r) * H + h) : 0.f;
    }
  };
  auto load_w = [&](float* dst, int64_t v0) {
    for (int e = tid; e < 64 * H; e += 256) {
      const int r = e / H, h = e % H;
      dst[r * ld_ + h] = v0 + r < k.V ? ld(W + (v0 + r) * H + h) : 0.f;
    }
  };
  if (MODE == kDW) load_w(A, a0); else load_x(A, a0);
  if (tid < 64) {
    top[tid] = -INFINITY;
    sum[tid] = 0.f;
    hit[tid] = 0.f;
  }
  float acc[64];
#pragma unroll
  for (int r = 0; r < 64; ++r) acc[r] = 0.f;
  const int tr = tid / 16 * 4, tc = tid % 16 * 4;
  for (int64_t b0 = 0; b0 < nb; b0 += 64) {
    __syncthreads();
    if (MODE == kDW) load_x(B, b0); else load_w(B, b0);
    __syncthreads();
    float z[4][4] = {};
    for (int h = 0; h < H; ++h) {
      float a[4], b[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        a[j] = A[(tr + j) * ld_ + h];
        b[j] = B[(tc + j) * ld_ + h];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) z[i][j] = fmaf(a[i], b[j], z[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int ar = tr + i, br = tc + j;
        float v = z[i][j];
        if (MODE != kLoss) {
          const int x = MODE == kDX ? ar : br;
          const int64_t voc = MODE == kDX ? b0 + br : a0 + ar;
          v = tgt[x] >= 0 && voc < k.V
                  ? sg[x] * (expf(v - slse[x]) - (voc == tgt[x] ? 1.f : 0.f))
                  : 0.f;
        }
        P[ar * 65 + br] = v;
      }
    __syncthreads();
    if (MODE == kLoss) {
      if (tid < 64 && tgt[tid] >= 0) {
        const int m = (int)min((int64_t)64, nb - b0);
        float mx = top[tid];
        for (int c = 0; c < m; ++c) mx = fmaxf(mx, P[tid * 65 + c]);
        float s = mx == -INFINITY ? 0.f : sum[tid] * expf(top[tid] - mx);
        if (mx != -INFINITY)
          for (int c = 0; c < m; ++c) s += expf(P[tid * 65 + c] - mx);
        top[tid] = mx;
        sum[tid] = s;
        if (tgt[tid] >= b0 && tgt[tid] < b0 + m) hit[tid] = P[tid * 65 + tgt[tid] - b0];
      }
    } else if (tid < H) {
      for (int c = 0; c < 64; ++c) {
        const float b = B[c * ld_ + tid];
#pragma unroll
        for (int r = 0; r < 64; ++r) acc[r] = fmaf(P[r * 65 + c], b, acc[r]);
      }
    }
  }
  if (MODE == kLoss) {
    if (tid < 64 && a0 + tid < k.n) {
      const float l = tgt[tid] >= 0 ? top[tid] + logf(sum[tid]) : 0.f;
      k.lse[a0 + tid] = l;
      k.loss[a0 + tid] = tgt[tid] >= 0 ? l - hit[tid] : 0.f;
    }
  } else if (tid < H) {
#pragma unroll
    for (int r = 0; r < 64; ++r) {
      if (a0 + r >= na) continue;
      const int64_t at = (a0 + r) * H + tid;
      if (k.grad_bf16) {
        static_cast<__nv_bfloat16*>(k.grad)[at] = __float2bfloat16(acc[r]);
      } else {
        float* g = static_cast<float*>(k.grad) + at;
        *g = k.accumulate ? *g + acc[r] : acc[r];
      }
    }
  }
}

template <typename T, int MODE>
cudaError_t launch(const XentKernel& k, cudaStream_t st) {
  const size_t smem = (2 * 64 * (size_t)(k.H + 1) + 64 * 65 + 6 * 64) * sizeof(float);
  cudaError_t e = cudaFuncSetAttribute(k_xent<T, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)smem);
  if (e != cudaSuccess) return e;
  const int64_t rows = MODE == kDW ? k.V : k.n;
  k_xent<T, MODE><<<(unsigned)((rows + 63) / 64), 256, smem, st>>>(k);
  note_launch();
  return cudaGetLastError();
}

XentKernel base(const XentArgs& a) {
  XentKernel k{};
  k.n = a.n;
  k.H = a.H;
  k.V = a.V;
  k.X = a.X;
  k.W = a.W;
  k.target = a.target;
  k.status = a.status;
  return k;
}

}  // namespace

size_t xent_ws_bytes(int, int64_t, int, int, int) { return 256; }

cudaError_t xent_fwd(const XentArgs& a, float* loss, float* lse, cudaStream_t st) {
  if (a.n == 0) return cudaSuccess;
  XentKernel k = base(a);
  k.loss = loss;
  k.lse = lse;
  return a.bf16 ? launch<__nv_bfloat16, kLoss>(k, st) : launch<float, kLoss>(k, st);
}

cudaError_t xent_bwd(const XentArgs& a, const float* lse, const float* dloss, int grad_bf16,
                     void* dX, void* dW, int accumulate, cudaStream_t st) {
  XentKernel k = base(a);
  k.lse = const_cast<float*>(lse);
  k.dloss = dloss;
  k.grad_bf16 = grad_bf16;
  k.accumulate = accumulate;
  cudaError_t e = cudaSuccess;
  if (dX && a.n > 0) {
    k.grad = dX;
    e = a.bf16 ? launch<__nv_bfloat16, kDX>(k, st) : launch<float, kDX>(k, st);
  }
  if (e == cudaSuccess && dW) {
    k.grad = dW;
    e = a.bf16 ? launch<__nv_bfloat16, kDW>(k, st) : launch<float, kDW>(k, st);
  }
  return e;
}

}  // namespace bg
