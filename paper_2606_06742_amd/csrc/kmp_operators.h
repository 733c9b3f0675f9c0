// Internal interface of the operators at a language model's end: layer norm,
// products in 8-bit integers, log probabilities of tokens. Element types,
// 16-byte vectors of them, and the launchers (norm.hip, quantized.hip,
// logprobs.hip; arguments checked in operators_api.cpp).
#pragma once

#include <algorithm>

#include "kmp_common.h"

namespace kmp {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// Sums, statistics and products are formed in Acc: 32 bits, or 64 for doubles.
template <typename T> struct acc_of { typedef float type; };
template <> struct acc_of<double> { typedef double type; };

// Elements of one 16-byte access.
template <typename T> constexpr int vec_of() { return 16 / (int)sizeof(T); }

// N consecutive elements from any address that is aligned to one element (the
// hardware takes 16-byte accesses at such addresses, aligned ones are faster).
// Conversion to Acc is exact; to T it rounds to the nearest, ties to even.
template <typename T, int N, typename A>
__device__ __forceinline__ void load_n(const T* p, A (&v)[N]) {
  constexpr int B = N * (int)sizeof(T) < 16 ? N * (int)sizeof(T) : 16;   // bytes an access
  constexpr int E = B / (int)sizeof(T);
#pragma unroll
  for (int c = 0; c < N / E; ++c) {
    T t[E];
    __builtin_memcpy(t, p + c * E, B);
#pragma unroll
    for (int e = 0; e < E; ++e) v[c * E + e] = (A)t[e];
  }
}
template <typename T, int N, typename A>
__device__ __forceinline__ void store_n(T* p, const A (&v)[N]) {
  constexpr int B = N * (int)sizeof(T) < 16 ? N * (int)sizeof(T) : 16;
  constexpr int E = B / (int)sizeof(T);
#pragma unroll
  for (int c = 0; c < N / E; ++c) {
    T t[E];
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] = (T)v[c * E + e];
    __builtin_memcpy(p + c * E, t, B);
  }
}

// ---------------------------------------------------------------- layer norm
struct NormArgs {
  int xtype, wtype;                     // KMP_F64 .. KMP_F16
  const void* x; int64_t rows, d, ldx;
  const void* gamma; const void* beta;  // may be null (ones, zeros)
  double eps;
  bool bytes;                           // y in 8 bits with a scale per row
  bool plain;                           // x itself instead of its norm (bytes only)
  void* y; int64_t ldy;
  void* mean; void* rstd;               // may be null
  float* scale;
};
int norm_forward(hipStream_t s, const NormArgs& a);

struct NormBackArgs {
  int xtype, wtype;
  const void* dy; int64_t lddy;
  const void* x; int64_t ldx, rows, d;
  const void* gamma;                    // may be null (ones)
  const void* mean; const void* rstd;
  void* dx; int64_t lddx;               // may be null
  void* dgamma; void* dbeta;            // may be null
  void* partial;                        // norm_partials(..) x 2 x d of Acc
};
int64_t norm_partials(int xtype, int64_t rows, int64_t d);
int norm_backward(hipStream_t s, const NormBackArgs& a);

// ------------------------------------------------- products in 8-bit integers
struct QProductArgs {
  const int8_t* x; int64_t ldx; const float* xscale;   // M x K, a scale per row
  const int8_t* w; int64_t ldw; const float* wscale;   // N x K, a scale per row
  const float* bias;                                   // N, may be null
  int64_t M, N, K;
  int otype; void* out; int64_t ldo;
};
int quantized_product(hipStream_t s, const QProductArgs& a);

// ------------------------------------------------- log probabilities of tokens
constexpr int kMaxTop = KMP_MAX_TOP;
struct LogprobArgs {
  int type;
  const void* logits; int64_t T, V, ld;
  const void* tokens; bool wide;        // int64 tokens; may be null
  float* logp; float* entropy; float* stats; // each may be null
  int top; int32_t* top_id; float* top_logp; // each may be null
  void* workspace;
};
size_t logprob_workspace(int64_t T, int64_t V, int top);
int token_logprobs(hipStream_t s, const LogprobArgs& a);

struct LogprobBackArgs {
  int type;
  const void* logits; int64_t T, V, ld;
  const void* tokens; bool wide;
  const float* stats; const float* entropy; const float* dlogp; const float* dentropy;
  void* dlogits; int64_t ldd;
};
int token_logprobs_backward(hipStream_t s, const LogprobBackArgs& a);

}  // namespace kmp
