// Launchers of the operators that answer with a vocabulary and learn from such answers: logits
// (logits.cu), their adjustment and their largest entries (top.cu), distillation from a teacher's largest
// logits (distill.cu).  All launch on `st` and return the first CUDA error.
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "bandggnn.h"

namespace bg {

// Z[i][v] = X[i] . W[v], rows of Z ldz elements apart.
struct LogitsArgs {
  int bf16;  // type of X and W
  int out_bf16;
  int64_t n;
  int H, V;
  const void* X;  // [n][H]
  const void* W;  // [V][H]
  int64_t ldz;
  void* Z;
  void* ws;
  int* status;
};
size_t logits_ws_bytes(int bf16, int64_t n, int H, int V);
cudaError_t logits_fwd(const LogitsArgs& a, cudaStream_t st);

// out = adjusted Z; out may be Z (with ldo == ldz).
cudaError_t logits_adjust(int bf16, int64_t n, int V, int64_t ldz, const void* Z, const bg_adjust& adj,
                          int64_t ldo, void* out, int* status, cudaStream_t st);
// The K largest adjusted logits of each row; lse may be NULL.
constexpr int kMaxTop = 128;
cudaError_t logits_top(int bf16, int64_t n, int V, int64_t ldz, const void* Z, const bg_adjust& adj, int K,
                       float* top_logit, int32_t* top_id, float* lse, int* status, cudaStream_t st);

struct DistillArgs {
  int bf16;
  int64_t n;
  int H, V, K;
  const void* X;
  const void* W;
  const int32_t* top_id;   // [n][K], < 0: no entry
  const float* top_logit;  // [n][K]
  float tau;
  void* ws;
  int* status;
};
size_t distill_ws_bytes(int bf16, int64_t n, int H, int V, int K, int backward);
cudaError_t distill_fwd(const DistillArgs& a, float* loss, float* lse, cudaStream_t st);
cudaError_t distill_bwd(const DistillArgs& a, const float* lse, const float* dloss, int grad_bf16, void* dX,
                        void* dW, int accumulate, cudaStream_t st);

// Sites of BG_EDEVICE records: a token of a history or of a teacher's answer of V or more, a mask's number of
// n_masks or more, history offsets that fall or leave the array.
constexpr int kSiteHistoryId = 132;
constexpr int kSiteMaskRow = 133;
constexpr int kSiteHistoryOff = 134;
constexpr int kSiteTeacherId = 135;

}  // namespace bg
