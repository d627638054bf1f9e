// C ABI of the token operators: argument checks and hand-over to their launchers.
#include <cuda_runtime.h>

#include <string>

#include "internal.h"
#include "token.h"

namespace {

bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

#define TOK_PTR(p)                                                                \
  do {                                                                            \
    if (!(p)) return bg_fail(BG_EINVAL, #p " is NULL");                           \
    if (misaligned(p)) return bg_fail(BG_EINVAL, #p " not 16-byte aligned");      \
  } while (0)
#define TOK_OPT_PTR(p)                                                            \
  do {                                                                            \
    if ((p) && misaligned(p)) return bg_fail(BG_EINVAL, #p " not 16-byte aligned"); \
  } while (0)
#define TOK_TRY(call)             \
  do {                            \
    const int rc_ = (call);       \
    if (rc_ != BG_OK) return rc_; \
  } while (0)

int cuda_rc(cudaError_t e, const char* what) {
  if (e == cudaSuccess) return BG_OK;
  return bg_fail(BG_ECUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

int check_dtype(bg_dtype dt) {
  return dt == BG_F32 || dt == BG_BF16 ? BG_OK : bg_fail(BG_EINVAL, "unknown dtype");
}

constexpr int64_t kMaxRows = (int64_t)1 << 29;
constexpr int32_t kMaxVocab = 1 << 24;

int check_shape(int64_t n, int32_t H, int32_t V) {
  if (n < 0 || n > kMaxRows) return bg_fail(BG_EINVAL, "n must be in [0, 2^29]");
  if (H < 32 || H > 256 || H % 32) return bg_fail(BG_EINVAL, "H must be a multiple of 32 in [32, 256]");
  if (V < 1 || V > kMaxVocab) return bg_fail(BG_EINVAL, "V must be in [1, 2^24]");
  return BG_OK;
}

int check_p(float p) {
  return p >= 0.f && p <= 1.f ? BG_OK : bg_fail(BG_EINVAL, "p must be in [0, 1]");  // NaN fails too
}

int check_flags(uint32_t flags) {
  return flags & ~BG_ACCUM ? bg_fail(BG_EINVAL, "unknown flags") : BG_OK;
}

bool valid_shape(int64_t n, int32_t H, int32_t V) {
  return n >= 0 && n <= kMaxRows && H >= 32 && H <= 256 && H % 32 == 0 && V >= 1 && V <= kMaxVocab;
}

}  // namespace

extern "C" int bg_dropout_fwd(bg_dtype dt, int64_t n, float p, int64_t seed, int64_t call,
                              const void* x, const void* residual, void* y, void* stream) {
  bg_clear_error();
  TOK_TRY(check_dtype(dt));
  TOK_TRY(check_p(p));
  if (n < 0) return bg_fail(BG_EINVAL, "n < 0");
  if (n == 0) return BG_OK;
  TOK_PTR(x); TOK_OPT_PTR(residual); TOK_PTR(y);
  return cuda_rc(bg::dropout_fwd(dt == BG_BF16, n, bg::make_drop(p, seed, call), x, residual, y,
                                 (cudaStream_t)stream), "bg_dropout_fwd");
}

extern "C" int bg_dropout_bwd(int64_t n, float p, int64_t seed, int64_t call, const float* dy,
                              float* dx, uint32_t flags, void* stream) {
  bg_clear_error();
  TOK_TRY(check_p(p));
  TOK_TRY(check_flags(flags));
  if (n < 0) return bg_fail(BG_EINVAL, "n < 0");
  if (n == 0) return BG_OK;
  TOK_PTR(dy); TOK_PTR(dx);
  if ((flags & BG_ACCUM) && dy == dx) return bg_fail(BG_EINVAL, "dx is dy with BG_ACCUM");
  return cuda_rc(bg::dropout_bwd(n, bg::make_drop(p, seed, call), dy, dx, (flags & BG_ACCUM) != 0,
                                 (cudaStream_t)stream), "bg_dropout_bwd");
}

extern "C" int bg_embed_fwd(bg_dtype dt, int64_t n, int32_t H, int32_t V, const int32_t* ids,
                            const void* table, float scale, float p, int64_t seed, int64_t call,
                            void* out, void* stream) {
  bg_clear_error();
  TOK_TRY(check_dtype(dt));
  TOK_TRY(check_shape(n, H, V));
  TOK_TRY(check_p(p));
  if (n == 0) return BG_OK;
  TOK_PTR(ids); TOK_PTR(table); TOK_PTR(out);
  int* status = nullptr;
  TOK_TRY(bg_status_word(&status));
  return cuda_rc(bg::embed_fwd(dt == BG_BF16, n, H, V, ids, table, scale,
                               bg::make_drop(p, seed, call), out, status, (cudaStream_t)stream),
                 "bg_embed_fwd");
}

extern "C" size_t bg_embed_workspace_bytes(int64_t n, int32_t H, int32_t V) {
  return valid_shape(n, H, V) ? bg::embed_bwd_ws_bytes(n, H, V) : 0;
}

extern "C" int bg_embed_bwd(int64_t n, int32_t H, int32_t V, const int32_t* ids, const float* dout,
                            float scale, float p, int64_t seed, int64_t call, float* dtable,
                            uint32_t flags, void* ws, size_t ws_bytes, void* stream) {
  bg_clear_error();
  TOK_TRY(check_shape(n, H, V));
  TOK_TRY(check_p(p));
  TOK_TRY(check_flags(flags));
  TOK_PTR(dtable);
  if (n > 0) {
    TOK_PTR(ids); TOK_PTR(dout); TOK_PTR(ws);
    if (ws_bytes < bg::embed_bwd_ws_bytes(n, H, V))
      return bg_fail(BG_ECAPACITY, "workspace too small");
  }
  int* status = nullptr;
  if (n > 0) TOK_TRY(bg_status_word(&status));
  return cuda_rc(bg::embed_bwd(n, H, V, ids, dout, scale, bg::make_drop(p, seed, call), dtable,
                               (flags & BG_ACCUM) != 0, ws, status, (cudaStream_t)stream),
                 "bg_embed_bwd");
}

extern "C" size_t bg_xent_workspace_bytes(bg_dtype dt, int64_t n, int32_t H, int32_t V, int32_t op) {
  if ((dt != BG_F32 && dt != BG_BF16) || !valid_shape(n, H, V) ||
      (op != BG_OP_XENT_FWD && op != BG_OP_XENT_BWD))
    return 0;
  return bg::xent_ws_bytes(dt == BG_BF16, n, H, V, op == BG_OP_XENT_BWD);
}

static int xent_args(bg_dtype dt, int64_t n, int32_t H, int32_t V, const void* X, const void* W,
                     const int32_t* target, void* ws, size_t ws_bytes, int backward,
                     bg::XentArgs* a) {
  TOK_TRY(check_dtype(dt));
  TOK_TRY(check_shape(n, H, V));
  TOK_PTR(W);
  if (n > 0) {
    TOK_PTR(X); TOK_PTR(target); TOK_PTR(ws);
    if (ws_bytes < bg::xent_ws_bytes(dt == BG_BF16, n, H, V, backward))
      return bg_fail(BG_ECAPACITY, "workspace too small");
  }
  *a = bg::XentArgs{dt == BG_BF16, n, H, V, X, W, target, ws, nullptr};
  return BG_OK;
}

extern "C" int bg_xent_fwd(bg_dtype dt, int64_t n, int32_t H, int32_t V, const void* X,
                           const void* W, const int32_t* target, float* loss, float* lse, void* ws,
                           size_t ws_bytes, void* stream) {
  bg_clear_error();
  bg::XentArgs a;
  TOK_TRY(xent_args(dt, n, H, V, X, W, target, ws, ws_bytes, 0, &a));
  if (n == 0) return BG_OK;
  TOK_PTR(loss); TOK_PTR(lse);
  TOK_TRY(bg_status_word(&a.status));
  return cuda_rc(bg::xent_fwd(a, loss, lse, (cudaStream_t)stream), "bg_xent_fwd");
}

extern "C" int bg_xent_bwd(bg_dtype dt, int64_t n, int32_t H, int32_t V, const void* X,
                           const void* W, const int32_t* target, const float* lse,
                           const float* dloss, bg_dtype grad_dt, void* dX, void* dW, uint32_t flags,
                           void* ws, size_t ws_bytes, void* stream) {
  bg_clear_error();
  bg::XentArgs a;
  TOK_TRY(xent_args(dt, n, H, V, X, W, target, ws, ws_bytes, 1, &a));
  TOK_TRY(check_dtype(grad_dt));
  TOK_TRY(check_flags(flags));
  if (dt == BG_F32 && grad_dt != BG_F32)
    return bg_fail(BG_EINVAL, "fp32 states and table have fp32 gradients");
  if ((flags & BG_ACCUM) && grad_dt != BG_F32)
    return bg_fail(BG_EINVAL, "BG_ACCUM needs fp32 gradients");
  // (without rows dX is empty and may be NULL all the same)
  if (n > 0 && !dX && !dW) return bg_fail(BG_EINVAL, "dX and dW are NULL");
  TOK_OPT_PTR(dX); TOK_OPT_PTR(dW);
  if (n > 0) {
    TOK_PTR(lse); TOK_PTR(dloss);
    TOK_TRY(bg_status_word(&a.status));
  }
  return cuda_rc(bg::xent_bwd(a, lse, dloss, grad_dt == BG_BF16, dX, dW, (flags & BG_ACCUM) != 0,
                              (cudaStream_t)stream), "bg_xent_bwd");
}
