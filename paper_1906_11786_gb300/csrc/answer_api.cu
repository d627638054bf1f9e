// C ABI of the operators that answer with a vocabulary: argument checks and hand-over to their launchers.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdlib>
#include <string>

#include "answer.h"
#include "internal.h"

namespace {

bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

#define ANS_PTR(p)                                                                \
  do {                                                                            \
    if (!(p)) return bg_fail(BG_EINVAL, #p " is NULL");                           \
    if (misaligned(p)) return bg_fail(BG_EINVAL, #p " not 16-byte aligned");      \
  } while (0)
#define ANS_OPT_PTR(p)                                                            \
  do {                                                                            \
    if ((p) && misaligned(p)) return bg_fail(BG_EINVAL, #p " not 16-byte aligned"); \
  } while (0)
#define ANS_TRY(call)             \
  do {                            \
    const int rc_ = (call);       \
    if (rc_ != BG_OK) return rc_; \
  } while (0)

int cuda_rc(cudaError_t e, const char* what) {
  if (e == cudaSuccess) return BG_OK;
  return bg_fail(BG_ECUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

bool is_dtype(bg_dtype dt) { return dt == BG_F32 || dt == BG_BF16; }
int check_dtype(bg_dtype dt) { return is_dtype(dt) ? BG_OK : bg_fail(BG_EINVAL, "unknown dtype"); }

constexpr int64_t kMaxRows = (int64_t)1 << 29;
constexpr int32_t kMaxVocab = 1 << 24;
constexpr int64_t kMaxStride = (int64_t)1 << 31;

bool valid_rows(int64_t n, int32_t V) { return n >= 0 && n <= kMaxRows && V >= 1 && V <= kMaxVocab; }
bool valid_h(int32_t H) { return H >= 32 && H <= 256 && H % 32 == 0; }

int check_rows(int64_t n, int32_t V) {
  if (n < 0 || n > kMaxRows) return bg_fail(BG_EINVAL, "n must be in [0, 2^29]");
  if (V < 1 || V > kMaxVocab) return bg_fail(BG_EINVAL, "V must be in [1, 2^24]");
  return BG_OK;
}
int check_h(int32_t H) {
  return valid_h(H) ? BG_OK : bg_fail(BG_EINVAL, "H must be a multiple of 32 in [32, 256]");
}
int check_stride(const char* name, int64_t ld, int32_t V) {
  return ld >= V && ld <= kMaxStride ? BG_OK
                                     : bg_fail(BG_EINVAL, std::string(name) + " must be in [V, 2^31]");
}

// Whether any of n rows of `width` bytes from a, lda bytes apart, shares a byte with one of those from b.
bool rows_meet(const void* pa, int64_t lda, const void* pb, int64_t ldb, int64_t n, int64_t width) {
  const int64_t a = (int64_t)(uintptr_t)pa, b = (int64_t)(uintptr_t)pb;
  if (a + (n - 1) * lda + width <= b || b + (n - 1) * ldb + width <= a) return false;
  if (lda == ldb) {  // rows i and j are b - a + (j - i) lda apart
    const int64_t d = b - a, k = d / lda;
    for (int64_t s = k - 1; s <= k + 1; ++s)
      if (s > -n && s < n && std::abs(d - s * lda) < width) return true;
    return false;
  }
  for (int64_t i = 0, j = 0; i < n && j < n;) {
    const int64_t x = a + i * lda, y = b + j * ldb;
    if (x < y + width && y < x + width) return true;
    ++(x < y ? i : j);
  }
  return false;
}

// The adjustment as the launchers take it (an empty one for NULL).
int check_adjust(const bg_adjust* in, int64_t n, bg_adjust* out) {
  *out = bg_adjust{};
  if (!in) return BG_OK;
  const bg_adjust& adjust = *in;
  ANS_OPT_PTR(adjust.bias);
  ANS_OPT_PTR(adjust.mask);
  ANS_OPT_PTR(adjust.mask_row);
  ANS_OPT_PTR(adjust.history);
  ANS_OPT_PTR(adjust.history_off);
  ANS_OPT_PTR(adjust.penalty);
  if (adjust.mask) {
    if (adjust.n_masks < 1) return bg_fail(BG_EINVAL, "adjust.n_masks must be 1 or more with a mask");
    if (!adjust.mask_row && adjust.n_masks != 1 && adjust.n_masks < n)
      return bg_fail(BG_EINVAL, "adjust.n_masks must be 1 or at least n without adjust.mask_row");
  } else if (adjust.mask_row || adjust.n_masks) {
    return bg_fail(BG_EINVAL, "adjust.mask_row or n_masks without adjust.mask");
  }
  if (adjust.history_len < 0) return bg_fail(BG_EINVAL, "adjust.history_len < 0");
  if (!adjust.history_off != !adjust.penalty)
    return bg_fail(BG_EINVAL, "adjust.history_off and adjust.penalty belong together");
  if (adjust.history_len > 0 && (!adjust.history || !adjust.history_off))
    return bg_fail(BG_EINVAL, "adjust.history_len without adjust.history and adjust.history_off");
  *out = adjust;
  return BG_OK;
}

}  // namespace

extern "C" size_t bg_logits_workspace_bytes(bg_dtype dt, int64_t n, int32_t H, int32_t V) {
  return is_dtype(dt) && valid_rows(n, V) && valid_h(H) ? bg::logits_ws_bytes(dt == BG_BF16, n, H, V) : 0;
}

extern "C" int bg_logits_fwd(bg_dtype dt, int64_t n, int32_t H, int32_t V, const void* X, const void* W,
                             bg_dtype out_dt, int64_t ldz, void* Z, void* ws, size_t ws_bytes, void* stream) {
  bg_clear_error();
  ANS_TRY(check_dtype(dt));
  ANS_TRY(check_dtype(out_dt));
  ANS_TRY(check_rows(n, V));
  ANS_TRY(check_h(H));
  ANS_TRY(check_stride("ldz", ldz, V));
  if (n == 0) return BG_OK;
  ANS_PTR(X); ANS_PTR(W); ANS_PTR(Z);
  const size_t need = bg::logits_ws_bytes(dt == BG_BF16, n, H, V);
  if (need > 0) {
    ANS_PTR(ws);
    if (ws_bytes < need) return bg_fail(BG_ECAPACITY, "workspace too small");
  }
  bg::LogitsArgs a{dt == BG_BF16, out_dt == BG_BF16, n, H, V, X, W, ldz, Z, ws, nullptr};
  ANS_TRY(bg_status_word(&a.status));
  return cuda_rc(bg::logits_fwd(a, (cudaStream_t)stream), "bg_logits_fwd");
}

extern "C" int bg_logits_adjust(bg_dtype dt, int64_t n, int32_t V, int64_t ldz, const void* Z,
                                const bg_adjust* adjust, int64_t ldo, void* out, void* stream) {
  bg_clear_error();
  bg_adjust adj;
  ANS_TRY(check_dtype(dt));
  ANS_TRY(check_rows(n, V));
  ANS_TRY(check_stride("ldz", ldz, V));
  ANS_TRY(check_stride("ldo", ldo, V));
  ANS_TRY(check_adjust(adjust, n, &adj));
  if (n == 0) return BG_OK;
  ANS_PTR(Z); ANS_PTR(out);
  if (out == Z && ldo != ldz) return bg_fail(BG_EINVAL, "in place, ldo must be ldz");
  const int64_t e = dt == BG_BF16 ? 2 : 4;
  if (out != Z && rows_meet(Z, ldz * e, out, ldo * e, n, V * e))
    return bg_fail(BG_EINVAL, "out overlaps Z and is not Z");
  int* status = nullptr;
  ANS_TRY(bg_status_word(&status));
  return cuda_rc(bg::logits_adjust(dt == BG_BF16, n, V, ldz, Z, adj, ldo, out, status, (cudaStream_t)stream),
                 "bg_logits_adjust");
}

extern "C" int bg_logits_top(bg_dtype dt, int64_t n, int32_t V, int64_t ldz, const void* Z,
                             const bg_adjust* adjust, int32_t K, float* top_logit, int32_t* top_id, float* lse,
                             void* stream) {
  bg_clear_error();
  bg_adjust adj;
  ANS_TRY(check_dtype(dt));
  ANS_TRY(check_rows(n, V));
  ANS_TRY(check_stride("ldz", ldz, V));
  if (K < 1 || K > bg::kMaxTop) return bg_fail(BG_EINVAL, "K must be in [1, 128]");
  ANS_TRY(check_adjust(adjust, n, &adj));
  if (n == 0) return BG_OK;
  ANS_PTR(Z); ANS_PTR(top_logit); ANS_PTR(top_id); ANS_OPT_PTR(lse);
  int* status = nullptr;
  ANS_TRY(bg_status_word(&status));
  return cuda_rc(bg::logits_top(dt == BG_BF16, n, V, ldz, Z, adj, K, top_logit, top_id, lse, status,
                                (cudaStream_t)stream),
                 "bg_logits_top");
}

extern "C" size_t bg_distill_workspace_bytes(bg_dtype dt, int64_t n, int32_t H, int32_t V, int32_t K,
                                             int32_t op) {
  if (!is_dtype(dt) || !valid_rows(n, V) || !valid_h(H) || K < 1 || K > bg::kMaxTop || n * K > kMaxRows ||
      (op != BG_OP_DISTILL_FWD && op != BG_OP_DISTILL_BWD))
    return 0;
  return bg::distill_ws_bytes(dt == BG_BF16, n, H, V, K, op == BG_OP_DISTILL_BWD);
}

static int distill_args(bg_dtype dt, int64_t n, int32_t H, int32_t V, int32_t K, const void* X, const void* W,
                        const int32_t* top_id, const float* top_logit, float tau, void* ws, size_t ws_bytes,
                        int backward, bg::DistillArgs* a) {
  ANS_TRY(check_dtype(dt));
  ANS_TRY(check_rows(n, V));
  ANS_TRY(check_h(H));
  if (K < 1 || K > bg::kMaxTop) return bg_fail(BG_EINVAL, "K must be in [1, 128]");
  if (n * K > kMaxRows) return bg_fail(BG_EINVAL, "n K must be at most 2^29");
  if (!(tau >= 1e-3f && tau <= 1e3f)) return bg_fail(BG_EINVAL, "tau must be in [0.001, 1000]");  // NaN fails too
  ANS_PTR(W);
  if (n > 0) {
    ANS_PTR(X); ANS_PTR(top_id); ANS_PTR(top_logit); ANS_PTR(ws);
    if (ws_bytes < bg::distill_ws_bytes(dt == BG_BF16, n, H, V, K, backward))
      return bg_fail(BG_ECAPACITY, "workspace too small");
  }
  *a = bg::DistillArgs{dt == BG_BF16, n, H, V, K, X, W, top_id, top_logit, tau, ws, nullptr};
  return BG_OK;
}

extern "C" int bg_distill_fwd(bg_dtype dt, int64_t n, int32_t H, int32_t V, int32_t K, const void* X,
                              const void* W, const int32_t* top_id, const float* top_logit, float tau,
                              float* loss, float* lse, void* ws, size_t ws_bytes, void* stream) {
  bg_clear_error();
  bg::DistillArgs a;
  ANS_TRY(distill_args(dt, n, H, V, K, X, W, top_id, top_logit, tau, ws, ws_bytes, 0, &a));
  if (n == 0) return BG_OK;
  ANS_PTR(loss); ANS_PTR(lse);
  ANS_TRY(bg_status_word(&a.status));
  return cuda_rc(bg::distill_fwd(a, loss, lse, (cudaStream_t)stream), "bg_distill_fwd");
}

extern "C" int bg_distill_bwd(bg_dtype dt, int64_t n, int32_t H, int32_t V, int32_t K, const void* X,
                              const void* W, const int32_t* top_id, const float* top_logit, float tau,
                              const float* lse, const float* dloss, bg_dtype grad_dt, void* dX, void* dW,
                              uint32_t flags, void* ws, size_t ws_bytes, void* stream) {
  bg_clear_error();
  bg::DistillArgs a;
  ANS_TRY(distill_args(dt, n, H, V, K, X, W, top_id, top_logit, tau, ws, ws_bytes, 1, &a));
  ANS_TRY(check_dtype(grad_dt));
  if (flags & ~BG_ACCUM) return bg_fail(BG_EINVAL, "unknown flags");
  if (dt == BG_F32 && grad_dt != BG_F32)
    return bg_fail(BG_EINVAL, "fp32 states and table have fp32 gradients");
  if ((flags & BG_ACCUM) && grad_dt != BG_F32) return bg_fail(BG_EINVAL, "BG_ACCUM needs fp32 gradients");
  // (without rows dX is empty and may be NULL all the same)
  if (n > 0 && !dX && !dW) return bg_fail(BG_EINVAL, "dX and dW are NULL");
  ANS_OPT_PTR(dX); ANS_OPT_PTR(dW);
  if (n > 0) {
    ANS_PTR(lse); ANS_PTR(dloss);
    ANS_TRY(bg_status_word(&a.status));
  }
  return cuda_rc(bg::distill_bwd(a, lse, dloss, grad_dt == BG_BF16, dX, dW, (flags & BG_ACCUM) != 0,
                                 (cudaStream_t)stream),
                 "bg_distill_bwd");
}
