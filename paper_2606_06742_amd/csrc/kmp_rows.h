// Rows over the threads of a workgroup: sums and largest values of a row, its
// vectors in registers, its elements in 8 bits (norm.hip, kmp_block.h).
#pragma once

#include "kmp_operators.h"

namespace kmp {

constexpr int BT = 256, BIG = 1024;    // threads of a workgroup; of one for a long row

// The larger, or NaN where either is NaN.
__device__ __forceinline__ float larger(float a, float b) { return b > a || b != b ? b : a; }

template <typename A>
__device__ __forceinline__ A block_total(A v, A* red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, kWave);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  A t = 0;
#pragma unroll
  for (int i = 0; i < BIG / 64; ++i) t += red[i];
  return t;
}
// Largest value, or NaN where any is NaN.
__device__ __forceinline__ float block_most(float v, float* red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = larger(v, __shfl_xor(v, off, kWave));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = red[0];
#pragma unroll
  for (int i = 1; i < BIG / 64; ++i) t = larger(t, red[i]);
  return t;
}
// f(j, N elements) over a row of d by a workgroup of BIG threads: whole vectors of
// 16 bytes, then single elements.
template <int VEC, typename F>
__device__ __forceinline__ void over_row(int64_t d, F f) {
  const int64_t whole = d / VEC;
#pragma unroll 2
  for (int64_t v = threadIdx.x; v < whole; v += BIG) f(v * VEC, Count<VEC>());
  if (whole * VEC + threadIdx.x < d) f(whole * VEC + threadIdx.x, Count<1>());
}

__device__ __forceinline__ float inv_sqrt(float v) { return 1.0f / sqrtf(v); }
__device__ __forceinline__ double inv_sqrt(double v) { return 1.0 / sqrt(v); }

// The factor (1 / a) 127 that takes a row into 8 bits, and its scale a / 127. Three
// roundings with the product by x: a result differs from the nearest to x 127 / a only
// where that lies within 127 * 3 * 2^-24 of a half (65 of 4e7 normal numbers in 32
// bits, 45 with the factor 127 / a). Below 2^-100 the factor would overflow: such rows
// are brought up by 2^100 first. A row with an infinity or NaN gets factor 0 and scale
// NaN.
struct ByteScale {
  float lift, factor, scale;
  __device__ explicit ByteScale(float a) {
    const bool tiny = a < 0x1p-100f, good = a < INFINITY;
    lift = tiny ? 0x1p100f : 1.0f;
    factor = good && a > 0.0f ? 1.0f / (a * lift) * 127.0f : 0.0f;
    scale = good ? a / 127.0f : __builtin_nanf("");
  }
  __device__ int8_t operator()(float v) const {
    const float q = rintf(v * lift * factor);
    return (int8_t)(int)(factor > 0.0f ? fminf(fmaxf(q, -127.0f), 127.0f) : 0.0f);
  }
};

// A row that fits the registers of TPR threads: a sum over it is a butterfly, then for
// TPR > 64 one exchange in LDS (slots alternate between the sums, so one barrier each
// is enough).
constexpr int threads_of(int tpr) { return tpr > BT ? tpr : BT; }
template <typename A, int TPR>
__device__ __forceinline__ A row_total(A v, A (*red)[threads_of(TPR) / 64], int& slot) {
#pragma unroll
  for (int off = (TPR < 64 ? TPR : 64) / 2; off >= 1; off >>= 1) v += __shfl_xor(v, off, kWave);
  if constexpr (TPR > 64) {
    A* r = red[slot];
    slot ^= 1;
    if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = v;
    __syncthreads();
    v = r[0];
#pragma unroll
    for (int i = 1; i < TPR / 64; ++i) v += r[i];
  }
  return v;
}
// Two sums at once.
template <typename A, int TPR>
__device__ __forceinline__ void row_totals(A& u, A& v, A (*red)[2 * (threads_of(TPR) / 64)], int& slot) {
#pragma unroll
  for (int off = (TPR < 64 ? TPR : 64) / 2; off >= 1; off >>= 1) {
    u += __shfl_xor(u, off, kWave);
    v += __shfl_xor(v, off, kWave);
  }
  if constexpr (TPR > 64) {
    A* r = red[slot];
    slot ^= 1;
    if ((threadIdx.x & 63) == 0) {
      r[2 * (threadIdx.x >> 6)] = u;
      r[2 * (threadIdx.x >> 6) + 1] = v;
    }
    __syncthreads();
    u = r[0];
    v = r[1];
#pragma unroll
    for (int i = 1; i < TPR / 64; ++i) u += r[2 * i], v += r[2 * i + 1];
  }
}
template <int TPR>
__device__ __forceinline__ float row_most(float v, float (*red)[threads_of(TPR) / 64], int& slot) {
#pragma unroll
  for (int off = (TPR < 64 ? TPR : 64) / 2; off >= 1; off >>= 1) v = larger(v, __shfl_xor(v, off, kWave));
  if constexpr (TPR > 64) {
    float* r = red[slot];
    slot ^= 1;
    if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = v;
    __syncthreads();
    v = r[0];
#pragma unroll
    for (int i = 1; i < TPR / 64; ++i) v = larger(v, r[i]);
  }
  return v;
}

// A thread's vector of N elements of a row of d >= N that would start at j: it is
// moved back to end with the row, so that every load is one access and no branch
// stands between the loads (a branch for the row's end made each wait for the one
// before). Its first `skip` elements are another vector's, all of them where j
// lies past the end: cleared, and not stored.
template <int N>
struct Place {
  int at, skip;
  __device__ Place(int j, int d) : at(min(j, d - N)), skip(j - at) {}
};
template <int N, typename A>
__device__ __forceinline__ void clear(const Place<N>& q, A (&v)[N]) {
  if (q.skip > 0) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = e < q.skip ? (A)0 : v[e];
  }
}
template <typename T, int N, typename A>
__device__ __forceinline__ void store_at(T* p, const Place<N>& q, const A (&v)[N]) {
  if (q.skip == 0) {
    store_n(p + q.at, v);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e >= q.skip) p[q.at + e] = (T)v[e];
  }
}

}  // namespace kmp
