// Layer norm of rows, forward and backward.
//   y = (x - mu) r g + b,  mu = mean_j x_j,  r = 1 / sqrt(mean_j (x_j - mu)^2 + eps)
//   dx = r (w - mean(w) - xh mean(w xh)),  w = dy g,  xh = (x - mu) r
//   dg_j = sum over rows of dy xh,  db_j = sum over rows of dy
// The variance is the mean square of x - mu in a pass of its own (no
// cancellation of two large sums). The 8-bit form writes rint(y (1 / a) 127) with
// a = max_j |y_j| and the row's scale a / 127.
#include "kmp_operators.h"

namespace kmp {
namespace {

constexpr int BT = 256, BIG = 1024;    // threads of a workgroup; of one for a long row
// what is written: the norm in x's type or in 8 bits, or x itself in 8 bits
enum { kNorm, kNormBytes, kBytesOfX };

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
template <int N> struct Count { static constexpr int n = N; };
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

// One workgroup per row, any length (rows too long for the registers, or shorter
// than a vector): a pass for the mean, one for the variance, one for the largest
// |y| of the 8-bit form, one to write; all but the first find the row in the cache.
template <typename T, typename W, int MODE>
__global__ __launch_bounds__(BIG) void norm_row_kernel(NormArgs a) {
  typedef typename acc_of<T>::type A;
  constexpr bool BYTES = MODE != kNorm, PLAIN = MODE == kBytesOfX;
  constexpr int VEC = vec_of<T>();
  __shared__ A red[BIG / 64];
  __shared__ float fred[BIG / 64];
  const W* gamma = static_cast<const W*>(a.gamma);
  const W* beta = static_cast<const W*>(a.beta);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    A mu = 0, rs = 1;
    if constexpr (!PLAIN) {
      A s = 0;
      over_row<VEC>(a.d, [&](int64_t j, auto c) {
        A v[c.n];
        load_n(x + j, v);
#pragma unroll
        for (int e = 0; e < c.n; ++e) s += v[e];
      });
      mu = block_total(s, red) / (A)a.d;
      A q = 0;
      over_row<VEC>(a.d, [&](int64_t j, auto c) {
        A v[c.n];
        load_n(x + j, v);
#pragma unroll
        for (int e = 0; e < c.n; ++e) q += (v[e] - mu) * (v[e] - mu);
      });
      rs = inv_sqrt(block_total(q, red) / (A)a.d + (A)a.eps);
      if (threadIdx.x == 0) {
        if (a.mean) static_cast<A*>(a.mean)[r] = mu;
        if (a.rstd) static_cast<A*>(a.rstd)[r] = rs;
      }
    }
    const auto values = [&](int64_t j, auto& v) {
      constexpr int N = sizeof(v) / sizeof(A);
      load_n(x + j, v);
      if constexpr (!PLAIN) {
        A g[N], b[N];
#pragma unroll
        for (int e = 0; e < N; ++e) g[e] = 1, b[e] = 0;
        if (gamma) load_n(gamma + j, g);
        if (beta) load_n(beta + j, b);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (v[e] - mu) * rs * g[e] + b[e];
      }
    };
    if constexpr (BYTES) {
      float m = 0.0f;
      over_row<VEC>(a.d, [&](int64_t j, auto c) {
        A v[c.n];
        values(j, v);
#pragma unroll
        for (int e = 0; e < c.n; ++e) m = larger(m, fabsf((float)v[e]));
      });
      const ByteScale b(block_most(m, fred));
      int8_t* y = static_cast<int8_t*>(a.y) + r * a.ldy;
      over_row<VEC>(a.d, [&](int64_t j, auto c) {
        A v[c.n];
        int8_t q[c.n];
        values(j, v);
#pragma unroll
        for (int e = 0; e < c.n; ++e) q[e] = b((float)v[e]);
        store_n(y + j, q);
      });
      if (threadIdx.x == 0) a.scale[r] = b.scale;
    } else {
      T* y = static_cast<T*>(a.y) + r * a.ldy;
      over_row<VEC>(a.d, [&](int64_t j, auto c) {
        A v[c.n];
        values(j, v);
        store_n(y + j, v);
      });
    }
  }
}

// Rows that fit the registers of TPR threads, NV 16-byte vectors each: x is read
// once. A thread's vectors are TPR apart, so a wavefront reads whole lines. The
// sum over a row is a butterfly, then for TPR > 64 one exchange in LDS (slots
// alternate between the sums, so one barrier each is enough). gamma and beta
// stay in registers over the rows of a workgroup, and the next row is on its way
// while one is worked on (16384 x 4096 in 16 bits 54 us at 5.0 TB/s, the backward
// pass 77 us at 5.2).
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

template <typename T, typename W, int MODE, int TPR, int NV>   // MODE: below
__global__ __launch_bounds__(threads_of(TPR)) void norm_reg_kernel(NormArgs a) {
  typedef typename acc_of<T>::type A;
  constexpr int VEC = vec_of<T>(), RPB = threads_of(TPR) / TPR;
  __shared__ A red[2][threads_of(TPR) / 64];
  __shared__ float fred[2][threads_of(TPR) / 64];
  int slot = 0, fslot = 0;
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR, d = (int)a.d;
  A g[NV][VEC], b[NV][VEC];
  if constexpr (MODE != kBytesOfX) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Place<VEC> q((t + i * TPR) * VEC, d);
#pragma unroll
      for (int e = 0; e < VEC; ++e) g[i][e] = 1, b[i][e] = 0;
      if (a.gamma) load_n(static_cast<const W*>(a.gamma) + q.at, g[i]);
      if (a.beta) load_n(static_cast<const W*>(a.beta) + q.at, b[i]);
      clear(q, g[i]);
      clear(q, b[i]);
    }
  }
  T nx[NV][VEC];                                  // the next row, as it comes
  const auto next = [&](int64_t r) {
    const T* x = static_cast<const T*>(a.x) + min(r, a.rows - 1) * a.ldx;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      __builtin_memcpy(nx[i], x + Place<VEC>((t + i * TPR) * VEC, d).at, sizeof(nx[i]));
  };
  next((int64_t)blockIdx.x * RPB + sub);
  // a workgroup's rows: every thread takes part in every round (the barriers)
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB) {
    const bool live = r0 + sub < a.rows;
    const int64_t r = live ? r0 + sub : a.rows - 1;
    A v[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[i][e] = (A)nx[i][e];
      clear(Place<VEC>((t + i * TPR) * VEC, d), v[i]);
    }
    if (r0 + (int64_t)gridDim.x * RPB < a.rows) next(r + (int64_t)gridDim.x * RPB);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (MODE != kBytesOfX) {
      A s = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) s += v[i][e];
      const A mu = row_total<A, TPR>(s, red, slot) / (A)d;
      A q = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i][e] -= mu;
        clear(Place<VEC>((t + i * TPR) * VEC, d), v[i]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) q += v[i][e] * v[i][e];
      }
      const A rs = inv_sqrt(row_total<A, TPR>(q, red, slot) / (A)d + (A)a.eps);
      if (t == 0 && live) {
        if (a.mean) static_cast<A*>(a.mean)[r] = mu;
        if (a.rstd) static_cast<A*>(a.rstd)[r] = rs;
      }
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i][e] = v[i][e] * rs * g[i][e] + b[i][e];
    }
    if constexpr (MODE == kNorm) {
      T* y = static_cast<T*>(a.y) + r * a.ldy;
      if (live) {
#pragma unroll
        for (int i = 0; i < NV; ++i) store_at(y, Place<VEC>((t + i * TPR) * VEC, d), v[i]);
      }
    } else {
      float m = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) m = larger(m, fabsf((float)v[i][e]));
      const ByteScale bs(row_most<TPR>(m, fred, fslot));
      int8_t* y = static_cast<int8_t*>(a.y) + r * a.ldy;
      if (live) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          int8_t q[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) q[e] = bs((float)v[i][e]);
          store_at(y, Place<VEC>((t + i * TPR) * VEC, d), q);
        }
        if (t == 0) a.scale[r] = bs.scale;
      }
    }
  }
}

// dgamma and dbeta of columns j0 .. j0 + 15 over all rows by a workgroup of NT
// threads: 16 columns beside each other, every NT / 16-th row, then the row groups
// in order. `sums` holds 2 NT values.
template <typename T, typename W, int NT, typename A>
__device__ __forceinline__ void sum_columns(const NormBackArgs& a, int64_t j0, A* sums) {
  constexpr int G = NT / 16;
  const int c = threadIdx.x & 15, q = threadIdx.x >> 4;
  const int64_t j = min(j0 + c, a.d - 1);
  A dg = 0, db = 0;
#pragma unroll 8
  for (int64_t r = q; r < a.rows; r += G) {
    const A w = (A)static_cast<const T*>(a.dy)[r * a.lddy + j];
    const A xh = ((A)static_cast<const T*>(a.x)[r * a.ldx + j] - static_cast<const A*>(a.mean)[r]) *
                 static_cast<const A*>(a.rstd)[r];
    dg += w * xh;
    db += w;
  }
  sums[threadIdx.x] = dg;
  sums[NT + threadIdx.x] = db;
  __syncthreads();
  if (threadIdx.x >= 32) return;                  // 16 columns of the one, 16 of the other
  A v = 0;
  for (int i = 0; i < G; ++i) v += sums[(q ? NT : 0) + 16 * i + c];
  W* out = static_cast<W*>(q ? a.dbeta : a.dgamma);
  if (out && j0 + c < a.d) out[j0 + c] = (W)v;
}

// dx of one row per workgroup, any length: a pass for the two means, one to write.
// ONE: as in norm_back_reg_kernel.
template <typename T, typename W, bool ONE>
__global__ __launch_bounds__(BIG) void norm_back_row_kernel(NormBackArgs a, int rowblocks) {
  typedef typename acc_of<T>::type A;
  constexpr int VEC = vec_of<T>();
  __shared__ A red[BIG / 64];
  if constexpr (ONE) {
    __shared__ A sums[2 * BIG];
    if ((int)blockIdx.x >= rowblocks) {
      sum_columns<T, W, BIG>(a, (int64_t)((int)blockIdx.x - rowblocks) * 16, sums);
      return;
    }
  }
  const W* gamma = static_cast<const W*>(a.gamma);
  for (int64_t r = blockIdx.x; r < a.rows; r += rowblocks) {
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + r * a.lddy;
    const A mu = static_cast<const A*>(a.mean)[r], rs = static_cast<const A*>(a.rstd)[r];
    const auto values = [&](int64_t j, auto& xh, auto& w) {
      constexpr int N = sizeof(w) / sizeof(A);
      A g[N];
#pragma unroll
      for (int e = 0; e < N; ++e) g[e] = 1;
      load_n(x + j, xh);
      load_n(dy + j, w);
      if (gamma) load_n(gamma + j, g);
#pragma unroll
      for (int e = 0; e < N; ++e) xh[e] = (xh[e] - mu) * rs, w[e] *= g[e];
    };
    A s1 = 0, s2 = 0;
    over_row<VEC>(a.d, [&](int64_t j, auto c) {
      A xh[c.n], w[c.n];
      values(j, xh, w);
#pragma unroll
      for (int e = 0; e < c.n; ++e) s1 += w[e], s2 += w[e] * xh[e];
    });
    s1 = block_total(s1, red) / (A)a.d;
    s2 = block_total(s2, red) / (A)a.d;
    T* dx = static_cast<T*>(a.dx) + r * a.lddx;
    over_row<VEC>(a.d, [&](int64_t j, auto c) {
      A xh[c.n], w[c.n];
      values(j, xh, w);
#pragma unroll
      for (int e = 0; e < c.n; ++e) w[e] = rs * (w[e] - s1 - xh[e] * s2);
      store_n(dx + j, w);
    });
  }
}

// dx and the column sums in one pass over x and dy, rows in registers as in
// norm_reg_kernel: workgroup b takes rows b, b + gridDim.x, .. (RPB at a time),
// keeps its threads' columns of the two sums in registers, adds its RPB row
// groups in LDS and writes partial[b]. The next rows' loads are in flight
// during the current ones' sums.
// ONE: a single launch for few rows, whose time is launches: the first rowblocks
// workgroups form dx alone, the others the sums over all rows of 16 columns each,
// which need no more than the given mean and rstd.
template <typename T, typename W, int TPR, int NV, bool ONE>
__global__ __launch_bounds__(threads_of(TPR)) void norm_back_reg_kernel(NormBackArgs a, int rowblocks) {
  typedef typename acc_of<T>::type A;
  constexpr int VEC = vec_of<T>(), RPB = threads_of(TPR) / TPR;
  __shared__ A red[2][2 * (threads_of(TPR) / 64)];
  __shared__ A sums[ONE ? 2 * threads_of(TPR) : RPB > 1 ? TPR * NV * VEC : 1];
  if constexpr (ONE) {
    if ((int)blockIdx.x >= rowblocks) {
      sum_columns<T, W, threads_of(TPR)>(a, (int64_t)((int)blockIdx.x - rowblocks) * 16, sums);
      return;
    }
  }
  int slot = 0;
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR, d = (int)a.d;
  A g[NV][VEC], dg[NV][VEC], db[NV][VEC], x[NV][VEC], w[NV][VEC];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < VEC; ++e) g[i][e] = 1, dg[i][e] = 0, db[i][e] = 0;
  if (a.gamma) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      load_n(static_cast<const W*>(a.gamma) + Place<VEC>((t + i * TPR) * VEC, d).at, g[i]);
  }
  const int64_t step = (int64_t)rowblocks * RPB;
  T nx[NV][VEC], nd[NV][VEC];                     // the next row, as it comes
  A nmu, nrs;
  const auto next = [&](int64_t r) {
    r = min(r, a.rows - 1);
    const T* px = static_cast<const T*>(a.x) + r * a.ldx;
    const T* pd = static_cast<const T*>(a.dy) + r * a.lddy;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int at = Place<VEC>((t + i * TPR) * VEC, d).at;
      __builtin_memcpy(nx[i], px + at, sizeof(nx[i]));
      __builtin_memcpy(nd[i], pd + at, sizeof(nd[i]));
    }
    nmu = static_cast<const A*>(a.mean)[r];
    nrs = static_cast<const A*>(a.rstd)[r];
  };
  int64_t r0 = (int64_t)blockIdx.x * RPB;
  next(r0 + sub);
  for (; r0 < a.rows; r0 += step) {
    const int64_t r = r0 + sub;
    const bool live = r < a.rows;
    const A mu = nmu, rs = live ? nrs : (A)0;
    A s1 = 0, s2 = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        x[i][e] = ((A)nx[i][e] - mu) * rs;
        w[i][e] = live ? (A)nd[i][e] : (A)0;      // (a last round's missing rows add nothing)
      }
      clear(Place<VEC>((t + i * TPR) * VEC, d), w[i]);
    }
    next(r + step);                               // past the end: the last row again, unused
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if constexpr (!ONE) {
          dg[i][e] += w[i][e] * x[i][e];
          db[i][e] += w[i][e];
        }
        w[i][e] *= g[i][e];
        s1 += w[i][e];
        s2 += w[i][e] * x[i][e];
      }
    }
    if (a.dx) {
      row_totals<A, TPR>(s1, s2, red, slot);
      s1 /= (A)d;
      s2 /= (A)d;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[i][e] = rs * (w[i][e] - s1 - x[i][e] * s2);
      if (live) {
        T* dx = static_cast<T*>(a.dx) + r * a.lddx;
#pragma unroll
        for (int i = 0; i < NV; ++i) store_at(dx, Place<VEC>((t + i * TPR) * VEC, d), w[i]);
      }
    }
  }
  if (ONE || (!a.dgamma && !a.dbeta)) return;
  A* p = static_cast<A*>(a.partial) + (int64_t)blockIdx.x * 2 * a.d;
  const auto write = [&](A (&v)[NV][VEC], A* out) {
    if constexpr (RPB > 1) {
      for (int q = RPB - 1; q > 0; --q) {         // row group q adds to what those above it left
        if (sub == q) {
#pragma unroll
          for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              const int at = (i * VEC + e) * TPR + t;
              sums[at] = q == RPB - 1 ? v[i][e] : sums[at] + v[i][e];
            }
        }
        __syncthreads();
      }
      if (sub == 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < VEC; ++e) v[i][e] += sums[(i * VEC + e) * TPR + t];
      }
      __syncthreads();
    }
    if (sub == 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) store_at(out, Place<VEC>((t + i * TPR) * VEC, d), v[i]);
    }
  };
  write(dg, p);
  write(db, p + a.d);
}

// Column sums of dy xh and dy over the strip blockIdx.y of rows, a thread per
// column: partial[strip][0 or 1][column].
template <typename T>
__global__ __launch_bounds__(BT) void norm_back_columns_kernel(NormBackArgs a, int64_t strip) {
  typedef typename acc_of<T>::type A;
  const int64_t j = (int64_t)blockIdx.x * BT + threadIdx.x;
  if (j >= a.d) return;
  const int64_t r0 = (int64_t)blockIdx.y * strip, r1 = min(r0 + strip, a.rows);
  A dg = 0, db = 0;
#pragma unroll 4
  for (int64_t r = r0; r < r1; ++r) {
    const A g = (A)static_cast<const T*>(a.dy)[r * a.lddy + j];
    const A xh = ((A)static_cast<const T*>(a.x)[r * a.ldx + j] - static_cast<const A*>(a.mean)[r]) *
                 static_cast<const A*>(a.rstd)[r];
    dg += g * xh;
    db += g;
  }
  A* p = static_cast<A*>(a.partial) + (int64_t)blockIdx.y * 2 * a.d;
  p[j] = dg;
  p[a.d + j] = db;
}

// Adds the partial sums in a fixed order: 64 columns a workgroup at a time, each of
// its 16 wavefronts every sixteenth part, then the sixteen. At most 2^20 workgroups: a
// launch takes less than 2^32 threads.
template <typename A, typename W>
__global__ __launch_bounds__(1024) void norm_back_join_kernel(const A* partial, int64_t parts, int64_t d,
                                                              W* dgamma, W* dbeta) {
  __shared__ A red[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  W* out = blockIdx.y == 0 ? dgamma : dbeta;
  if (!out) return;
  for (int64_t j0 = (int64_t)blockIdx.x * 64; j0 < d; j0 += (int64_t)gridDim.x * 64) {
    const int64_t j = j0 + lane;
    A s = 0;
    if (j < d) {
#pragma unroll 8
      for (int64_t p = w; p < parts; p += 16) s += partial[(p * 2 + blockIdx.y) * d + j];
    }
    red[w][lane] = s;
    __syncthreads();
    if (w == 0 && j < d) {
#pragma unroll
      for (int i = 1; i < 16; ++i) s += red[i][lane];
      out[j] = (W)s;
    }
    __syncthreads();
  }
}

template <typename T, typename W, int MODE>
int forward_mode(hipStream_t s, const NormArgs& a) {
  // (rows shorter than a vector go with those too long for the registers)
  const int64_t nv = a.d < vec_of<T>() ? INT32_MAX : ceil_div(a.d, vec_of<T>());
  const auto grid = [&](int rpb) { return dim3((unsigned)std::min<int64_t>(ceil_div(a.rows, rpb), 2048)); };
#define KMP_NORM_CASE(TPR, NV)                                                                   \
  if (nv <= TPR * NV) {                                                                          \
    hipLaunchKernelGGL((norm_reg_kernel<T, W, MODE, TPR, NV>), grid(threads_of(TPR) / TPR),      \
                       dim3(threads_of(TPR)), 0, s, a);                                          \
    KMP_LAUNCH_CHECK();                                                                          \
    return 0;                                                                                    \
  }
  KMP_NORM_CASE(32, 1)
  KMP_NORM_CASE(64, 1)
  KMP_NORM_CASE(64, 2)
  KMP_NORM_CASE(256, 1)
  KMP_NORM_CASE(256, 2)
  KMP_NORM_CASE(256, 4)
  KMP_NORM_CASE(1024, 2)
  if constexpr (sizeof(T) >= 4) {                 // (more than 128 registers in 16 bits)
    KMP_NORM_CASE(1024, 4)
  }
#undef KMP_NORM_CASE
  hipLaunchKernelGGL((norm_row_kernel<T, W, MODE>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)),
                     dim3(BIG), 0, s, a);
  KMP_LAUNCH_CHECK();
  return 0;
}

template <typename T, typename W>
int forward_as(hipStream_t s, const NormArgs& a) {
  if (!a.bytes) return forward_mode<T, W, kNorm>(s, a);
  if constexpr (sizeof(T) <= 4) {
    if (!a.plain) return forward_mode<T, W, kNormBytes>(s, a);
    if constexpr (sizeof(T) == sizeof(W)) return forward_mode<T, W, kBytesOfX>(s, a);
  }
  return KMP_EINVAL;                              // refused before
}

template <typename T, typename W>
int backward_as(hipStream_t s, const NormBackArgs& a) {
  typedef typename acc_of<T>::type A;
  const int64_t parts = norm_partials(a.xtype, a.rows, a.d);
  const int64_t nv = a.d < vec_of<T>() ? INT32_MAX : ceil_div(a.d, vec_of<T>());
  const bool weights = a.dgamma || a.dbeta;
  // One launch where that is what the call costs; us of the kernels in one and in
  // two launches: 4 x 1024 in 16 bits 2.6 / 6.9, 300 x 512 4.4 / 8.1, 500 x 4096 8.8 /
  // 15.0, 200 x 8192 in 32 bits 9.1 / 15.6, 1003 x 1999 14.0 / 12.9, but 1000 x 4096
  // in 16 bits 21.8 / 17.2, 2000 x 512 12.4 / 10.7 (and 3 us of launch on the host). Rows
  // too long for the registers, in one and in three: 4 x 13134 in 16 bits 6.0 / 10.0,
  // 116 x 14770 10.1 / 17.9, 250 x 16384 19.6 / 23.7, 100 x 16384 in 32 bits 10.1 / 18.2.
  // Doubles: 300 x 512 4.4 / 7.2, 500 x 2000 11.5 / 13.9, 100 x 10000 11.5 / 19.2, but
  // slower between 513 and 2048 rows: 1000 x 500 13.9 / 10.5, 2000 x 250 20.2 / 10.9.
  const int64_t size = a.rows * a.d * (int64_t)sizeof(T);
  const bool small = a.rows <= 512 ? size <= 8 << 20 : a.rows <= 2048 && size <= 4 << 20;
  const bool one = weights && a.rows > 0 && small;
  const auto blocks = [&](int rpb) {              // of rows; with one launch 16 columns each beside them
    return one ? (a.dx ? (int)std::min<int64_t>(ceil_div(a.rows, rpb), 1024) : 0) : (int)parts;
  };
  const auto launch = [&](auto kernel, int rowblocks, int threads) {
    const int64_t grid = rowblocks + (one ? ceil_div(a.d, 16) : 0);
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(threads), 0, s, a, rowblocks);
  };
#define KMP_NORM_CASE(TPR, NV)                                                                       \
  if (nv <= TPR * NV) {                                                                              \
    const int rpb = threads_of(TPR) / TPR;                                                           \
    if (one) launch(norm_back_reg_kernel<T, W, TPR, NV, true>, blocks(rpb), threads_of(TPR));        \
    else launch(norm_back_reg_kernel<T, W, TPR, NV, false>, blocks(rpb), threads_of(TPR));           \
  } else
  if (a.rows > 0) {
    KMP_NORM_CASE(32, 1)
    KMP_NORM_CASE(64, 1)
    KMP_NORM_CASE(64, 2)
    KMP_NORM_CASE(256, 1)
    KMP_NORM_CASE(256, 2)
    // 512 threads with two vectors each take rows that 1024 threads with one were
    // slower on (8038 x 4228 in 16 bits 56 / 64 us, 8192 x 8192 87 / 94, 3000 x 4096 in
    // 32 bits 30 / 33)
    KMP_NORM_CASE(512, 2)
    // Longer rows in one launch without registers (with four vectors in them 116 x
    // 14770 in 16 bits 12.8 / 10.1 us, 250 x 16384 24.4 / 19.6). Else four vectors
    // against the passes for any length: 2000 x 16384 in 16 bits 79 / 97, 4000 x 9000
    // 97 / 109, 8000 x 16384 227 / 306, though 36 registers are spilled; eight vectors
    // of 32-bit elements spill 169, 2000 x 16384 226 / 158. (The choice is the same
    // without the weights, so that dx has the same bits.)
    if (one) {
      launch(norm_back_row_kernel<T, W, true>, blocks(1), BIG);
    } else if (nv <= 2048 && !small) {
      launch(norm_back_reg_kernel<T, W, 512, 4, false>, blocks(1), 512);
    } else {                                      // x and dy are read again for the weights
      if (a.dx)
        launch(norm_back_row_kernel<T, W, false>, (int)std::min<int64_t>(a.rows, 1 << 20), BIG);
      if (weights)
        hipLaunchKernelGGL((norm_back_columns_kernel<T>), dim3((unsigned)ceil_div(a.d, BT), (unsigned)parts),
                           dim3(BT), 0, s, a, ceil_div(a.rows, parts));
    }
    KMP_LAUNCH_CHECK();
  }
#undef KMP_NORM_CASE
  if (!weights || one) return 0;
  hipLaunchKernelGGL((norm_back_join_kernel<A, W>), dim3((unsigned)std::min<int64_t>(ceil_div(a.d, 64), 1 << 20), 2),
                     dim3(1024), 0, s, static_cast<const A*>(a.partial), a.rows > 0 ? parts : 0, a.d,
                     static_cast<W*>(a.dgamma), static_cast<W*>(a.dbeta));
  KMP_LAUNCH_CHECK();
  return 0;
}

}  // namespace

// Workgroups of the backward pass, each with its own column sums: two rounds of
// rows each up to 256 workgroups, at least four beyond, at most 512. us of the pass
// and of the join of the sums at rows x columns (16 bits but for the second):
//                      64 x 4096   1003 x 1999   16384 x 4096
//   two rounds, <= 512  5.7  2.7     11.4  5.3     77.1  5.4
//   two, <= 1024        5.8  2.8     11.4  5.5     92.3  6.8
//   four, <= 512        8.6  3.9      9.8  4.4     77.4  5.4
int64_t norm_partials(int xtype, int64_t rows, int64_t d) {
  const int64_t nv = ceil_div(d, 16 / (xtype == KMP_F64 ? 8 : xtype == KMP_F32 ? 4 : 2));
  const int64_t groups = ceil_div(rows, nv <= 32 ? 8 : nv <= 128 ? 4 : 1);
  return std::max<int64_t>({1, std::min<int64_t>(ceil_div(groups, 2), 256), std::min<int64_t>(ceil_div(groups, 4), 512)});
}

int norm_forward(hipStream_t s, const NormArgs& a) {
  switch (a.xtype * 8 + a.wtype) {
    case KMP_F64 * 8 + KMP_F64: return forward_as<double, double>(s, a);
    case KMP_F32 * 8 + KMP_F32: return forward_as<float, float>(s, a);
    case KMP_BF16 * 8 + KMP_BF16: return forward_as<bf16_t, bf16_t>(s, a);
    case KMP_BF16 * 8 + KMP_F32: return forward_as<bf16_t, float>(s, a);
    case KMP_F16 * 8 + KMP_F16: return forward_as<f16_t, f16_t>(s, a);
    default: return forward_as<f16_t, float>(s, a);
  }
}

int norm_backward(hipStream_t s, const NormBackArgs& a) {
  switch (a.xtype * 8 + a.wtype) {
    case KMP_F64 * 8 + KMP_F64: return backward_as<double, double>(s, a);
    case KMP_F32 * 8 + KMP_F32: return backward_as<float, float>(s, a);
    case KMP_BF16 * 8 + KMP_BF16: return backward_as<bf16_t, bf16_t>(s, a);
    case KMP_BF16 * 8 + KMP_F32: return backward_as<bf16_t, float>(s, a);
    case KMP_F16 * 8 + KMP_F16: return backward_as<f16_t, f16_t>(s, a);
    default: return backward_as<f16_t, float>(s, a);
  }
}

}  // namespace kmp
