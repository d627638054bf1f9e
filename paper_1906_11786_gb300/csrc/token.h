// Launchers of the token operators: dropout, embedding (embed.cu) and vocabulary cross entropy
// (xent.cu).  All launch on `st` and return the first CUDA error.
#pragma once

#include <cuda_runtime.h>

#include <atomic>
#include <cstddef>
#include <cstdint>

#include "philox.h"

namespace bg {

// y[i] = res[i] + drop(x[i]) (res may be NULL); x, res, y of one type.
cudaError_t dropout_fwd(int bf16, int64_t n, const Drop& d, const void* x, const void* res, void* y,
                        cudaStream_t st);
// dx[i] (+)= drop(dy[i])
cudaError_t dropout_bwd(int64_t n, const Drop& d, const float* dy, float* dx, int accumulate,
                        cudaStream_t st);

// out[i] = drop(scale * table[ids[i]]), a zero row where ids[i] < 0.
cudaError_t embed_fwd(int bf16, int64_t n, int H, int V, const int32_t* ids, const void* table,
                      float scale, const Drop& d, void* out, int* status, cudaStream_t st);

size_t embed_bwd_ws_bytes(int64_t n, int H, int V);
// dtable[v] (+)= scale * sum over ids[i] == v of drop(dout[i])
cudaError_t embed_bwd(int64_t n, int H, int V, const int32_t* ids, const float* dout, float scale,
                      const Drop& d, float* dtable, int accumulate, void* ws, int* status,
                      cudaStream_t st);

// dtable[v] (+)= sum over ids[e] == v of weight[e] X[e / K] (X: rows of fp32 or bf16): embed_bwd's sum with
// weighted rows that K ids share.  ids outside [0, V) name no row.
size_t token_sum_ws_bytes(int64_t n, int H, int V);
cudaError_t token_sum(int64_t n, int H, int V, const int32_t* ids, int bf16, const void* X, int K,
                      const float* weight, float* dtable, int accumulate, void* ws, int* status,
                      cudaStream_t st);

// Blocks of an SM that the sum (embed_bwd's or the weighted one) cuts its rows for, and each one's shared memory.
int token_sum_resident(int64_t n, int H, int weighted, int* smem);

// Soft targets instead of one token a row (distill.cu): probabilities softmax(z / tau) without a target's
// one, a row counts where `target` is 0 or more; loss = tau^2 (inner + lse), gradients times tau.
struct XentSoft {
  float tau;
  const float* inner;  // [n] forward
  const float* add_x;  // bf16 gradients: what is added to dX and dW before they are rounded (or NULL)
  const float* add_w;
};
struct XentArgs {
  int bf16;  // type of X and W
  int64_t n;
  int H, V;
  const void* X;          // [n][H]
  const void* W;          // [V][H]
  const int32_t* target;  // [n], < 0: the row is left out
  void* ws;
  int* status;
  const XentSoft* soft = nullptr;
};
size_t xent_ws_bytes(int bf16, int64_t n, int H, int V, int backward);
// CTAs of a tile kernel on a device of so many SMs, and the workspace that a call takes there: never more
// than xent_ws_bytes.
int xent_ctas(int sms);
size_t xent_ws_used(int bf16, int64_t n, int H, int V, int backward, int grad_bf16, int sms);
cudaError_t xent_fwd(const XentArgs& a, float* loss, float* lse, cudaStream_t st);
// Gradients in the type grad_bf16 says; dX or dW may be NULL.
cudaError_t xent_bwd(const XentArgs& a, const float* lse, const float* dloss, int grad_bf16,
                     void* dX, void* dW, int accumulate, cudaStream_t st);

// The lse that probabilities exp(z - lse) are taken with.  Both z and lse are fp32: from |lse| of 2^20 on their
// own roundings (2^-19 of them at most) may make the largest probability more than 2, beyond fp16 with its
// scale, and from 2^26 on infinite, from where one row would spread to all of dW.  Such rows have it raised by
// as much as that, so that no probability passes 1 (and, far out, all of them are 0).  Cutting them to 1 in
// the epilogues instead took up to 17% longer.
__device__ __forceinline__ float safe_lse(float lse) {
  return lse + fmaxf(fabsf(lse) - 0x1p20f, 0.f) * 0x1p-18f;
}

// Lets a kernel use `bytes` of dynamic shared memory, once a device.
template <typename K>
cudaError_t allow_smem(K kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// Sites of BG_EDEVICE records (status word): an id or a target of V or more.
constexpr int kSiteEmbedId = 130;
constexpr int kSiteXentTarget = 131;

}  // namespace bg
