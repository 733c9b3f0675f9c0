// Internal interface of the operators at a language model's end: layer norm, the
// norms around a block, products in 8-bit integers and in 16 and 32 bits, log
// probabilities of tokens and their choice. Element types, 16-byte vectors of them, and
// the launchers (norm.hip, block.hip, quantized.hip, linear.hip, logprobs.hip,
// sample.hip; arguments checked in operators_api.cpp).
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

// A number as a type.
template <int N> struct Count { static constexpr int n = N; };

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

// ------------------------------------------- the norms around a model's block
struct BlockArgs {
  int xtype, wtype;
  bool rms, after;
  const void* b; int64_t ldb;
  const void* res; int64_t ldr;         // may be null
  int64_t rows, d;
  const void* gamma_after; const void* beta_after;  // may be null (ones, zeros)
  const void* gate; int64_t ldg;        // may be null (ones); ldg = 0: one for all rows
  float rscale;
  const void* gamma; const void* beta;  // may be null
  float eps;
  void* h; int64_t ldh;                 // may be null
  bool bytes;                           // y in 8 bits
  void* y; int64_t ldy;                 // may be null
  float* stats;                         // rows x 4, may be null
  float* scale;
};
int block_forward(hipStream_t s, const BlockArgs& a);

struct BlockBackArgs {
  int xtype, wtype;
  bool rms, after;
  const void* dy; int64_t lddy;         // may be null
  const void* dh; int64_t lddh;         // may be null
  const void* b; int64_t ldb;
  const void* h; int64_t ldh;
  int64_t rows, d;
  const void* gamma_after; const void* beta_after;
  const void* gate; int64_t ldg;
  float rscale;
  const void* gamma;
  const float* stats;
  void* db; int64_t lddb;               // each output may be null
  void* dres; int64_t lddres;
  void* dgate; int64_t lddg;
  void* dgamma_after; void* dbeta_after; void* dgamma; void* dbeta;
  float* partial;                       // block_partials(..) x 4 x d
  float* means;                         // rows x 2 (rows too long for the registers)
};
int64_t block_partials(int xtype, int64_t rows, int64_t d);
int block_backward(hipStream_t s, const BlockBackArgs& a);

// ------------------------------------------------- products in 8-bit integers
struct QProductArgs {
  const int8_t* x; int64_t ldx; const float* xscale;   // M x K, a scale per row
  const int8_t* w; int64_t ldw; const float* wscale;   // N x K, a scale per row
  const float* bias;                                   // N, may be null
  int64_t M, N, K;
  int otype; void* out; int64_t ldo;
};
int quantized_product(hipStream_t s, const QProductArgs& a);

// ------------------------------ products with bias, activation and residual
struct DenseArgs {
  int type;
  const void* x; int64_t ldx;           // M x K
  const void* w; int64_t ldw;           // N x K
  int64_t M, N, K;
  int btype; const void* bias;          // N, may be null
  int act, otype;
  const void* residual; int64_t ldr;    // may be null
  void* out; int64_t ldo;
  void* z; int64_t ldz;                 // may be null
};
int dense_product(hipStream_t s, const DenseArgs& a);

struct DenseBackArgs {
  int type;
  const void* dout; int64_t lddo;
  int64_t M, N, K;
  int act;
  const void* z; int64_t ldz;
  const void* x; int64_t ldx;
  const void* w; int64_t ldw;
  void* dx; int64_t lddx;               // each output may be null
  void* dw; int64_t lddw;
  int btype; void* dbias;
  void* workspace;
};
size_t dense_workspace(int type, int64_t M, int64_t N, int64_t K);
int dense_backward(hipStream_t s, const DenseBackArgs& a);

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

// ----------------------------------------------------------- choice of tokens
struct SampleArgs {
  int type;
  const void* logits; int64_t T, V, ld;
  const float* u;
  const float* temperature; const int32_t* top_k; const float* top_p; const float* min_p;  // each may be null
  bool wide; void* tokens;              // int64 tokens
  float* logp;                          // may be null
  void* workspace;
};
size_t sample_workspace(int64_t T, int64_t V);
int sample_tokens(hipStream_t s, const SampleArgs& a);

}  // namespace kmp
