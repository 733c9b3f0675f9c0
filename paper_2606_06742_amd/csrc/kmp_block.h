// The norms around a model's block (block.hip, block_back.hip), fused with the block's
// gate and the residual stream, forward and backward. With N(x) = (x - mu) r g + c (mu = 0 and r from the
// mean square for the norm by the root mean square):
//   n = N(b) or b,  h = rscale res + gate n,  y = N(h)
//   s = dh + r2 (w - mean(w) - xh2 mean(w xh2)),  w = dy g2,  xh2 = (h - mu2) r2
//   dres = rscale s,  t = gate s,  db = r1 (w1 - mean(w1) - xh1 mean(w1 xh1)) or t
// (w1 = t g1, xh1 = (b - mu1) r1; without the mean of w for the root mean square), and
// over the rows, with A = sum s xh1, B = sum s for a gate per column,
//   dgate = g1 A + c1 B,  dg1 = gate A,  dc1 = gate B,  dg2 = sum dy xh2,  dc2 = sum dy
// so that four sums a column serve five gradients (for a gate per row A and B are taken
// of t, and dgate = s n has no sum). Bound by memory: b and res are read, h and y
// written, and the backward pass reads dy, dh, h and b and writes db and dres, each
// once. y is formed from h in 32 bits; the backward pass reads h as it was rounded, as
// 32 bits of it would double that read: dg2 has that rounding beside its own, 1.4 (up to
// 1.53 seen) times the error of one.
#pragma once

#include "kmp_rows.h"

// No products and sums are joined but those written so: every kernel here gives the same
// bits, whichever outputs a call asks for.
#pragma clang fp contract(off)

namespace kmp {

typedef float float4v __attribute__((ext_vector_type(4)));

// N elements of a weight vector (ones or zeros where there is none) from j on.
template <typename W, int N>
__device__ __forceinline__ void load_weights(const void* p, int64_t j, float none, float (&v)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = none;
  if (p) load_n(static_cast<const W*>(p) + j, v);
}

// N elements as they come from memory, in the registers that their bytes take: half of
// what 32-bit ones would for 16-bit elements.
template <typename T, int N>
struct Kept {
  uint32_t u[N * sizeof(T) / 4];
  __device__ __forceinline__ void load(const void* p, int64_t j) {
    const char* q = static_cast<const char*>(p) + j * (int64_t)sizeof(T);
#pragma unroll
    for (int c = 0; c < N * (int)sizeof(T) / 16; ++c) __builtin_memcpy(u + 4 * c, q + 16 * c, 16);
  }
  __device__ __forceinline__ void fill(float v) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const T x = (T)v;
      if constexpr (sizeof(T) == 4) u[e] = __builtin_bit_cast(uint32_t, x);
      else u[e / 2] = (uint32_t)__builtin_bit_cast(uint16_t, x) * 0x10001u;
    }
  }
  __device__ __forceinline__ void load_or(const void* p, int64_t j, float none) {
    if (p) load(p, j);
    else fill(none);
  }
  // Keeps the compiler from converting what does not change once, ahead of a loop, into
  // twice the registers.
  __device__ __forceinline__ void pin() {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) asm volatile("" : "+v"(u[i]));
    }
  }
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, u[e]);
    else return (float)__builtin_bit_cast(T, (uint16_t)(u[e / 2] >> 16 * (e & 1)));
  }
};

// Values to be stored, each rounded to 32 bits before it is to its type (a product that
// the compiler rounds to 16 bits at once may differ from that).
template <typename A, int N> struct Values { A v[N]; };
template <int N>
__device__ __forceinline__ Values<float, N> values_of(const float (&v)[N]) {
  Values<float, N> r;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    r.v[e] = v[e];
    asm volatile("" : "+v"(r.v[e]));
  }
  return r;
}

// Which calls a kernel is for: any; or, by bits, those that have every operand. In the
// latter no load or store stands behind a branch, so that how many of them are under way
// is known where one is waited for; behind branches every row waited for the stores of
// the one before: 16384 x 4096 in 16 bits 113 / 102 us forward and 263 / 184 backward,
// 8192 x 8192 129 / 107 and 440 / 178. Vectors that were moved back from the row's end
// are then stored whole, and rows past the last one are that one again: the same values
// twice (not where h is res, whose elements must be read before they are overwritten).
enum { kAny = 0, kKnown = 1, kGates = 2, kRagged = 4, kOther = 8 };   // kOther: y in 8 bits; no dh

// 16-byte vectors of a row; rows shorter than a vector go with those too long for the
// registers.
inline int64_t vectors(int xtype, int64_t d) {
  const int vec = xtype == KMP_F32 ? 4 : 8;
  return d < vec ? INT32_MAX : ceil_div(d, vec);
}

// Threads for nv vectors, NV each: no more wavefronts than have any.
inline int threads_for(int tpr, int NV, int64_t nv) { return tpr <= 64 ? BT : (int)round_up(ceil_div(nv, NV), 64); }

// f(form as a constant)
template <bool APART, typename F>
void with_form(int form, F f) {
  if constexpr (APART) {
    switch (form) {
      case kKnown: return f(Count<kKnown>());
      case kKnown | kGates: return f(Count<kKnown | kGates>());
      case kKnown | kOther: return f(Count<kKnown | kOther>());
      case kKnown | kGates | kOther: return f(Count<kKnown | kGates | kOther>());
    }
  }
  switch (form) {
    case kKnown | kRagged: return f(Count<kKnown | kRagged>());
    case kKnown | kGates | kRagged: return f(Count<kKnown | kGates | kRagged>());
    case kKnown | kRagged | kOther: return f(Count<kKnown | kRagged | kOther>());
    case kKnown | kGates | kRagged | kOther: return f(Count<kKnown | kGates | kRagged | kOther>());
    default: return f(Count<kAny>());
  }
}

}  // namespace kmp
