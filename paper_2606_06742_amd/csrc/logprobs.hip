// Log probabilities of tokens under rows of logits x (T x V):
//   m = max_j x_j,  s = sum_j exp(x_j - m),  u = sum_j exp(x_j - m) (x_j - m)
//   log p_j = (x_j - m) - log s,  entropy H = -sum_j p_j log p_j = log s - u / s
// the top values in the order (value descending, index ascending), and the
// gradient of g logp + h H with respect to x:
//   dx_j = g (1[j = token] - p_j) - h p_j (log p_j + H).
// A logit of -inf has p = 0 and no term. A row of nothing but -inf has
// every log p = -inf, H = 0 and gradient 0. A row with NaN or +inf has
// NaN results (its alternatives are still in order: NaN, then +inf, first).
// A negative token stands for none: logp 0 and no g; a token from V on gives
// NaN in logp and in the row's gradient, and reads nothing.
#include "kmp_operators.h"

namespace kmp {
namespace {

constexpr int BT = 256;
constexpr float kLog2e = 1.44269504088896340736f;

// Largest value with NaN above all (so that it is never lost).
__device__ __forceinline__ float most(float a, float b) { return a > b || a != a ? a : b; }

// m = max, s and u of a part of a row (see above); s = 0 for an empty part or
// one of nothing but -inf.
struct Part { float m, s, u; };
__device__ __forceinline__ Part join(const Part& a, const Part& b) {
  Part r;
  r.m = most(a.m, b.m);
  if (!(r.m > -INFINITY)) {                 // both empty, or NaN
    r.s = r.m != r.m ? r.m : 0.0f;
    r.u = r.s;
    return r;
  }
  const float da = a.s != 0.0f ? a.m - r.m : 0.0f, db = b.s != 0.0f ? b.m - r.m : 0.0f;
  const float fa = a.s != 0.0f ? exp2f(da * kLog2e) : 0.0f, fb = b.s != 0.0f ? exp2f(db * kLog2e) : 0.0f;
  // a part far below the maximum: its factor is 0, its distance unbounded
  const float ua = fa > 0.0f ? fa * (a.u + da * a.s) : 0.0f, ub = fb > 0.0f ? fb * (b.u + db * b.s) : 0.0f;
  r.s = fa * a.s + fb * b.s;
  r.u = ua + ub;
  return r;
}
__device__ __forceinline__ Part shuffle_xor(const Part& p, int off) {
  return Part{__shfl_xor(p.m, off, kWave), __shfl_xor(p.s, off, kWave), __shfl_xor(p.u, off, kWave)};
}
__device__ __forceinline__ Part block_join(Part p, Part* red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) p = join(p, shuffle_xor(p, off));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = p;
  __syncthreads();
  Part t = red[0];
#pragma unroll
  for (int i = 1; i < BT / 64; ++i) t = join(t, red[i]);
  return t;
}

// Order of the alternatives as one unsigned number: the value's bits mapped to
// increasing order (NaN highest, -0 as 0) above the complemented index.
__device__ __forceinline__ uint32_t value_key(float v) {
  if (v != v) return 0xFFFFFFFFu;
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return k == 0xFFFFFFFFu ? __builtin_nanf("") : __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

__device__ __forceinline__ int64_t token_at(const LogprobArgs& a, int64_t t) {
  return a.wide ? static_cast<const int64_t*>(a.tokens)[t] : static_cast<const int32_t*>(a.tokens)[t];
}

// A row's results from m, s, u: log p_j = (x_j - m) - log s, which keeps its
// digits at any size of m (masks of the type's lowest value).
struct Row { float m, logs; };
template <typename T>
__device__ __forceinline__ Row finish_row(const LogprobArgs& a, int64_t t, const Part& p) {
  // s = 0 (all -inf): -inf; NaN or an infinite maximum: NaN
  const Row r{p.m == INFINITY ? __builtin_nanf("") : p.m, p.m == INFINITY ? __builtin_nanf("") : logf(p.s)};
  if (threadIdx.x == 0) {
    if (a.stats) {
      a.stats[2 * t] = r.m;
      a.stats[2 * t + 1] = r.logs;
    }
    if (a.entropy)
      a.entropy[t] = p.s == 0.0f ? 0.0f : r.logs != r.logs ? r.logs : fmaxf(r.logs - p.u / p.s, 0.0f);
    if (a.logp) {
      const int64_t id = token_at(a, t);
      float v = 0.0f;
      if (id >= a.V) v = __builtin_nanf("");
      else if (id >= 0)
        v = p.s == 0.0f ? -INFINITY : ((float)static_cast<const T*>(a.logits)[t * a.ld + id] - r.m) - r.logs;
      a.logp[t] = v;
    }
  }
  return r;
}

// One workgroup per row; the alternatives one after another, each the largest
// key below the last.
template <typename T>
__global__ __launch_bounds__(BT) void logprob_row_kernel(LogprobArgs a) {
  __shared__ Part red[BT / 64];
  __shared__ unsigned long long kred[BT / 64];
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const T* x = static_cast<const T*>(a.logits) + t * a.ld;
    Part p{-INFINITY, 0.0f, 0.0f};
    for (int64_t j = threadIdx.x; j < a.V; j += BT) {
      const float v = (float)x[j];
      p = join(p, Part{v, v > -INFINITY || v != v ? 1.0f : 0.0f, 0.0f});
    }
    p = block_join(p, red);
    const Row row = finish_row<T>(a, t, p);
    unsigned long long last = ~0ull;
    for (int k = 0; k < a.top; ++k) {
      unsigned long long best = 0;
      for (int64_t j = threadIdx.x; j < a.V; j += BT) {
        const unsigned long long key = (unsigned long long)value_key((float)x[j]) << 32 | (uint32_t)~(uint32_t)j;
        if (key < last && key > best) best = key;
      }
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) {
        const unsigned long long o = __shfl_xor(best, off, kWave);
        best = o > best ? o : best;
      }
      __syncthreads();
      if ((threadIdx.x & 63) == 0) kred[threadIdx.x >> 6] = best;
      __syncthreads();
      for (int i = 0; i < BT / 64; ++i) best = kred[i] > best ? kred[i] : best;
      last = best;
      if (threadIdx.x == 0) {
        if (a.top_id) a.top_id[t * a.top + k] = (int32_t)~(uint32_t)best;
        if (a.top_logp)
          a.top_logp[t * a.top + k] = p.s == 0.0f ? -INFINITY : (key_value((uint32_t)(best >> 32)) - row.m) - row.logs;
      }
    }
  }
}

// The gradient of one row, elements blockIdx.x .. of it.
template <typename T>
__global__ __launch_bounds__(BT) void logprob_back_kernel(LogprobBackArgs a) {
  for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y) {
    const T* x = static_cast<const T*>(a.logits) + t * a.ld;
    T* dx = static_cast<T*>(a.dlogits) + t * a.ldd;
    int64_t id = -1;
    if (a.tokens && a.dlogp)
      id = a.wide ? static_cast<const int64_t*>(a.tokens)[t] : static_cast<const int32_t*>(a.tokens)[t];
    const float m = a.stats[2 * t], logs = a.stats[2 * t + 1];
    const float g = id < 0 ? 0.0f : id >= a.V ? __builtin_nanf("") : a.dlogp[t];
    const float h = a.dentropy ? a.dentropy[t] : 0.0f;
    const float H = a.dentropy ? a.entropy[t] : 0.0f;
    const bool none = m == -INFINITY && g == g;
    for (int64_t j = (int64_t)blockIdx.x * BT + threadIdx.x; j < a.V; j += (int64_t)gridDim.x * BT) {
      const float v = (float)x[j];
      const float lp = (v - m) - logs;
      // -inf: no probability and no term (unless the row is NaN)
      float r = none || (v == -INFINITY && logs == logs) ? (g != g ? g : 0.0f) : -exp2f(lp * kLog2e) * (g + h * (lp + H));
      if (j == id && !none) r += g;
      dx[j] = (T)r;
    }
  }
}

template <typename T>
int forward_as(hipStream_t s, const LogprobArgs& a) {
  hipLaunchKernelGGL(logprob_row_kernel<T>, dim3((unsigned)std::min<int64_t>(a.T, 1 << 20)), dim3(BT), 0, s, a);
  KMP_LAUNCH_CHECK();
  return 0;
}
template <typename T>
int backward_as(hipStream_t s, const LogprobBackArgs& a) {
  hipLaunchKernelGGL(logprob_back_kernel<T>,
                     dim3((unsigned)std::min<int64_t>(ceil_div(a.V, BT), 1024), (unsigned)std::min<int64_t>(a.T, 65535)),
                     dim3(BT), 0, s, a);
  KMP_LAUNCH_CHECK();
  return 0;
}

}  // namespace

size_t logprob_workspace(int64_t, int64_t, int) { return 256; }

int token_logprobs(hipStream_t s, const LogprobArgs& a) {
  switch (a.type) {
    case KMP_F32: return forward_as<float>(s, a);
    case KMP_BF16: return forward_as<bf16_t>(s, a);
    default: return forward_as<f16_t>(s, a);
  }
}

int token_logprobs_backward(hipStream_t s, const LogprobBackArgs& a) {
  switch (a.type) {
    case KMP_F32: return backward_as<float>(s, a);
    case KMP_BF16: return backward_as<bf16_t>(s, a);
    default: return backward_as<f16_t>(s, a);
  }
}

}  // namespace kmp
