// C entry points of the operators at a language model's end (kmpath.h):
// argument checks, then one launcher each. Nothing is launched after an error,
// and none of them waits for the device.
#include <cmath>
#include <string>

#include "kmp_operators.h"

namespace kmp {
namespace {

int refuse(const char* name, const char* why, int code = KMP_EINVAL) {
  set_error(std::string(name) + ": " + why);
  return code;
}

// No C++ exception leaves a C entry point.
template <typename F>
int guarded(F&& f) noexcept {
  try {
    return f();
  } catch (...) {                       // (no memory for a message)
    return KMP_EHIP;
  }
}

constexpr int64_t kMost = INT32_MAX;              // rows, columns, tokens
constexpr int64_t kMostLd = (int64_t)1 << 40;     // elements between two rows

bool float_type(int32_t t) { return t == KMP_F32 || t == KMP_BF16 || t == KMP_F16; }
// The weights are of x's type or, for 16-bit x, 32-bit floats.
bool norm_types(int32_t x, int32_t w) {
  return (x >= KMP_F64 && x <= KMP_F16) && (w == x || (w == KMP_F32 && x != KMP_F64));
}
size_t acc_bytes(int32_t t) { return t == KMP_F64 ? 8 : 4; }

}  // namespace
}  // namespace kmp

using namespace kmp;

extern "C" {

int kmp_layer_norm(void* stream, int32_t xtype, const void* x, int64_t rows, int64_t d, int64_t ldx,
                   int32_t wtype, const void* gamma, const void* beta, double eps, int32_t ytype,
                   void* y, int64_t ldy, void* mean, void* rstd, float* scale) {
  return guarded([&]() -> int {
    const char* name = "kmp_layer_norm";
    if (!norm_types(xtype, wtype)) return refuse(name, "types of x and of the weights do not go together");
    if (ytype != xtype && !(ytype == KMP_I8 && xtype != KMP_F64))
      return refuse(name, "y has the type of x or, for x of at most 32 bits, 8 bits");
    if (rows < 0 || rows > kMost || d < 1 || d > kMost || ldx < d || ldy < d || ldx > kMostLd || ldy > kMostLd)
      return refuse(name, "rows, d or a leading dimension out of range");
    if (!(eps >= 0.0) || !std::isfinite(eps)) return refuse(name, "eps must be finite and not negative");
    if (rows == 0) return KMP_OK;
    if (!x || !y || (ytype == KMP_I8 && !scale)) return refuse(name, "null pointer");
    NormArgs a{xtype, wtype, x, rows, d, ldx, gamma, beta, eps, ytype == KMP_I8, false, y, ldy, mean, rstd, scale};
    return norm_forward((hipStream_t)stream, a);
  });
}

size_t kmp_layer_norm_workspace_bytes(int32_t xtype, int64_t rows, int64_t d) {
  if (xtype < KMP_F64 || xtype > KMP_F16 || rows < 0 || rows > kMost || d < 1 || d > kMost) return 0;
  // 256 bytes where there is nothing to keep, so that 0 means an error
  return std::max<size_t>(256, (size_t)norm_partials(xtype, rows, d) * 2 * (size_t)d * acc_bytes(xtype));
}

int kmp_layer_norm_backward(void* stream, int32_t xtype, const void* dy, int64_t lddy, const void* x,
                            int64_t ldx, int64_t rows, int64_t d, int32_t wtype, const void* gamma,
                            const void* mean, const void* rstd, void* dx, int64_t lddx, void* dgamma,
                            void* dbeta, void* workspace, size_t workspace_bytes) {
  return guarded([&]() -> int {
    const char* name = "kmp_layer_norm_backward";
    if (!norm_types(xtype, wtype)) return refuse(name, "types of x and of the weights do not go together");
    if (rows < 0 || rows > kMost || d < 1 || d > kMost || lddy < d || ldx < d || (dx && lddx < d) ||
        lddy > kMostLd || ldx > kMostLd || lddx > kMostLd)
      return refuse(name, "rows, d or a leading dimension out of range");
    if (rows > 0 && (!dy || !x || !mean || !rstd)) return refuse(name, "null pointer");
    if (!dx && !dgamma && !dbeta) return KMP_OK;
    if (dgamma || dbeta) {
      const size_t need = kmp_layer_norm_workspace_bytes(xtype, rows, d);
      if (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15))
        return refuse(name, "the workspace is missing, too small or not aligned to 16 bytes", KMP_EWORKSPACE);
    }
    NormBackArgs a{xtype, wtype, dy, lddy, x, ldx, rows, d, gamma, mean, rstd, dx, lddx, dgamma, dbeta, workspace};
    return norm_backward((hipStream_t)stream, a);
  });
}

int kmp_quantize_rows(void* stream, int32_t xtype, const void* x, int64_t rows, int64_t d, int64_t ldx,
                      int8_t* q, int64_t ldq, float* scale) {
  return guarded([&]() -> int {
    const char* name = "kmp_quantize_rows";
    if (!float_type(xtype)) return refuse(name, "x must be of type KMP_F32, KMP_BF16 or KMP_F16");
    if (rows < 0 || rows > kMost || d < 1 || d > kMost || ldx < d || ldq < d || ldx > kMostLd || ldq > kMostLd)
      return refuse(name, "rows, d or a leading dimension out of range");
    if (rows == 0) return KMP_OK;
    if (!x || !q || !scale) return refuse(name, "null pointer");
    NormArgs a{xtype, xtype, x, rows, d, ldx, nullptr, nullptr, 0.0, true, true, q, ldq, nullptr, nullptr, scale};
    return norm_forward((hipStream_t)stream, a);
  });
}

int kmp_quantized_product(void* stream, const int8_t* x, int64_t ldx, const float* xscale, int64_t M,
                          const int8_t* w, int64_t ldw, const float* wscale, int64_t N, int64_t K,
                          const float* bias, int32_t otype, void* out, int64_t ldo) {
  return guarded([&]() -> int {
    const char* name = "kmp_quantized_product";
    if (!float_type(otype)) return refuse(name, "the output must be of type KMP_F32, KMP_BF16 or KMP_F16");
    if (M < 0 || N < 0 || K < 0 || M > kMost || N > kMost || ldx < K || ldw < K || ldo < N || ldx > kMostLd ||
        ldw > kMostLd || ldo > kMostLd)
      return refuse(name, "a size or a leading dimension out of range");
    if (K > 131071) return refuse(name, "K above 131071: the 32-bit sums could overflow");
    if (M == 0 || N == 0) return KMP_OK;
    if (ceil_div(M, 64) * ceil_div(N, 64) > (int64_t)1 << 23) return refuse(name, "more than 2^23 tiles of 64 x 64");
    if ((K > 0 && (!x || !w)) || !xscale || !wscale || !out) return refuse(name, "null pointer");
    QProductArgs a{x, ldx, xscale, w, ldw, wscale, bias, M, N, K, otype, out, ldo};
    return quantized_product((hipStream_t)stream, a);
  });
}

size_t kmp_token_logprobs_workspace_bytes(int64_t T, int64_t V, int32_t top) {
  if (T < 0 || T > kMost || V < 1 || V > kMost || top < 0 || top > KMP_MAX_TOP || top > V) return 0;
  return logprob_workspace(T, V, top);
}

int kmp_token_logprobs(void* stream, int32_t type, const void* logits, int64_t T, int64_t V, int64_t ldl,
                       int32_t token_bits, const void* tokens, float* logp, float* entropy, float* stats,
                       int32_t top, int32_t* top_id, float* top_logp, void* workspace,
                       size_t workspace_bytes) {
  return guarded([&]() -> int {
    const char* name = "kmp_token_logprobs";
    if (!float_type(type)) return refuse(name, "logits must be of type KMP_F32, KMP_BF16 or KMP_F16");
    if (T < 0 || T > kMost || V < 1 || V > kMost || ldl < V || ldl > kMostLd)
      return refuse(name, "T, V or the leading dimension out of range");
    if (top < 0 || top > KMP_MAX_TOP || top > V) return refuse(name, "top must lie in 0 .. min(V, KMP_MAX_TOP)");
    if (token_bits != 32 && token_bits != 64) return refuse(name, "tokens have 32 or 64 bits");
    if (T == 0) return KMP_OK;
    if (!logits || (logp && !tokens)) return refuse(name, "null pointer");
    if (!workspace || workspace_bytes < logprob_workspace(T, V, top) || (reinterpret_cast<uintptr_t>(workspace) & 15))
      return refuse(name, "the workspace is missing, too small or not aligned to 16 bytes", KMP_EWORKSPACE);
    LogprobArgs a{type, logits, T, V, ldl, tokens, token_bits == 64, logp, entropy, stats, top, top_id, top_logp, workspace};
    return token_logprobs((hipStream_t)stream, a);
  });
}

int kmp_token_logprobs_backward(void* stream, int32_t type, const void* logits, int64_t T, int64_t V,
                                int64_t ldl, int32_t token_bits, const void* tokens, const float* stats,
                                const float* entropy, const float* dlogp, const float* dentropy,
                                void* dlogits, int64_t ldd) {
  return guarded([&]() -> int {
    const char* name = "kmp_token_logprobs_backward";
    if (!float_type(type)) return refuse(name, "logits must be of type KMP_F32, KMP_BF16 or KMP_F16");
    if (T < 0 || T > kMost || V < 1 || V > kMost || ldl < V || ldd < V || ldl > kMostLd || ldd > kMostLd)
      return refuse(name, "T, V or a leading dimension out of range");
    if (token_bits != 32 && token_bits != 64) return refuse(name, "tokens have 32 or 64 bits");
    if (T == 0) return KMP_OK;
    if (!logits || !stats || !dlogits || (dlogp && !tokens) || (dentropy && !entropy))
      return refuse(name, "null pointer");
    LogprobBackArgs a{type, logits, T, V, ldl, tokens, token_bits == 64, stats, entropy, dlogp, dentropy, dlogits, ldd};
    return token_logprobs_backward((hipStream_t)stream, a);
  });
}

}  // extern "C"
