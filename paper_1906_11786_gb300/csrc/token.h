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

struct XentArgs {
  int bf16;  // type of X and W
  int64_t n;
  int H, V;
  const void* X;          // [n][H]
  const void* W;          // [V][H]
  const int32_t* target;  // [n], < 0: the row is left out
  void* ws;
  int* status;
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
