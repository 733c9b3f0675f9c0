// Layer norm of rows, forward and backward.
//   y = (x - mu) r g + b,  mu = mean_j x_j,  r = 1 / sqrt(mean_j (x_j - mu)^2 + eps)
//   dx = r (w - mean(w) - xh mean(w xh)),  w = dy g,  xh = (x - mu) r
//   dg_j = sum over rows of dy xh,  db_j = sum over rows of dy
// The variance is the mean square of x - mu in a pass of its own (no
// cancellation of two large sums). The 8-bit form writes rint(y 127 / a) with
// a = max_j |y_j| and the row's scale a / 127.
#include "kmp_operators.h"

namespace kmp {
namespace {

constexpr int BT = 256;                // threads of a workgroup

template <typename A>
__device__ __forceinline__ A block_total(A v, A* red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, kWave);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  A t = 0;
#pragma unroll
  for (int i = 0; i < BT / 64; ++i) t += red[i];
  return t;
}
// Largest value, or NaN where any is NaN.
__device__ __forceinline__ float block_most(float v, float* red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const float o = __shfl_xor(v, off, kWave);
    v = o > v || o != o ? o : v;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = red[0];
#pragma unroll
  for (int i = 1; i < BT / 64; ++i) t = red[i] > t || red[i] != red[i] ? red[i] : t;
  return t;
}

__device__ __forceinline__ float inv_sqrt(float v) { return 1.0f / sqrtf(v); }
__device__ __forceinline__ double inv_sqrt(double v) { return 1.0 / sqrt(v); }

// The factor 127 / a that takes a row into 8 bits, and its scale a / 127.
// Below 2^-100 the factor would overflow: such rows are brought up by 2^100
// first. A row with an infinity or NaN gets factor 0 and scale NaN.
struct ByteScale {
  float lift, factor, scale;
  __device__ explicit ByteScale(float a) {
    const bool tiny = a < 0x1p-100f, good = a < INFINITY;
    lift = tiny ? 0x1p100f : 1.0f;
    factor = good && a > 0.0f ? 127.0f / (a * lift) : 0.0f;
    scale = good ? a / 127.0f : __builtin_nanf("");
  }
  __device__ int8_t operator()(float v) const {
    const float q = rintf(v * lift * factor);
    return (int8_t)(int)(factor > 0.0f ? fminf(fmaxf(q, -127.0f), 127.0f) : 0.0f);
  }
};

// One workgroup per row, any length: a pass for the mean, one for the
// variance, one for the largest |y| of the 8-bit form, one to write.
template <typename T, typename W, bool BYTES, bool PLAIN>
__global__ __launch_bounds__(BT) void norm_row_kernel(NormArgs a) {
  typedef typename acc_of<T>::type A;
  __shared__ A red[BT / 64];
  __shared__ float fred[BT / 64];
  const W* gamma = static_cast<const W*>(a.gamma);
  const W* beta = static_cast<const W*>(a.beta);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    A mu = 0, rs = 1;
    if constexpr (!PLAIN) {
      A s = 0;
      for (int64_t j = threadIdx.x; j < a.d; j += BT) s += (A)x[j];
      mu = block_total(s, red) / (A)a.d;
      A q = 0;
      for (int64_t j = threadIdx.x; j < a.d; j += BT) {
        const A t = (A)x[j] - mu;
        q += t * t;
      }
      rs = inv_sqrt(block_total(q, red) / (A)a.d + (A)a.eps);
      if (threadIdx.x == 0) {
        if (a.mean) static_cast<A*>(a.mean)[r] = mu;
        if (a.rstd) static_cast<A*>(a.rstd)[r] = rs;
      }
    }
    const auto value = [&](int64_t j) {
      if constexpr (PLAIN) return (A)x[j];
      A v = ((A)x[j] - mu) * rs;
      if (gamma) v *= (A)gamma[j];
      if (beta) v += (A)beta[j];
      return v;
    };
    if constexpr (BYTES) {
      float m = 0.0f;
      for (int64_t j = threadIdx.x; j < a.d; j += BT) {
        const float v = fabsf((float)value(j));
        m = v > m || v != v ? v : m;
      }
      const ByteScale b(block_most(m, fred));
      int8_t* y = static_cast<int8_t*>(a.y) + r * a.ldy;
      for (int64_t j = threadIdx.x; j < a.d; j += BT) y[j] = b((float)value(j));
      if (threadIdx.x == 0) a.scale[r] = b.scale;
    } else {
      T* y = static_cast<T*>(a.y) + r * a.ldy;
      for (int64_t j = threadIdx.x; j < a.d; j += BT) y[j] = (T)value(j);
    }
  }
}

// dx of one row per workgroup, any length.
template <typename T, typename W>
__global__ __launch_bounds__(BT) void norm_back_row_kernel(NormBackArgs a) {
  typedef typename acc_of<T>::type A;
  __shared__ A red[BT / 64];
  const W* gamma = static_cast<const W*>(a.gamma);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + r * a.lddy;
    const A mu = static_cast<const A*>(a.mean)[r], rs = static_cast<const A*>(a.rstd)[r];
    A s1 = 0, s2 = 0;
    for (int64_t j = threadIdx.x; j < a.d; j += BT) {
      const A w = (A)dy[j] * (gamma ? (A)gamma[j] : (A)1);
      s1 += w;
      s2 += w * (((A)x[j] - mu) * rs);
    }
    s1 = block_total(s1, red) / (A)a.d;
    s2 = block_total(s2, red) / (A)a.d;
    T* dx = static_cast<T*>(a.dx) + r * a.lddx;
    for (int64_t j = threadIdx.x; j < a.d; j += BT) {
      const A w = (A)dy[j] * (gamma ? (A)gamma[j] : (A)1);
      dx[j] = (T)(rs * (w - s1 - ((A)x[j] - mu) * rs * s2));
    }
  }
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

// Adds the partial sums in a fixed order: 64 columns a workgroup, each
// wavefront every fourth part, then the four.
template <typename A, typename W>
__global__ __launch_bounds__(BT) void norm_back_join_kernel(const A* partial, int64_t parts, int64_t d,
                                                            W* dgamma, W* dbeta) {
  __shared__ A red[BT];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t j = (int64_t)blockIdx.x * 64 + lane;
  W* out = blockIdx.y == 0 ? dgamma : dbeta;
  A s = 0;
  if (j < d)
    for (int64_t p = w; p < parts; p += BT / 64) s += partial[(p * 2 + blockIdx.y) * d + j];
  red[threadIdx.x] = s;
  __syncthreads();
  if (w == 0 && j < d && out) out[j] = (W)((red[lane] + red[64 + lane]) + (red[128 + lane] + red[192 + lane]));
}

template <typename T, typename W>
int forward_as(hipStream_t s, const NormArgs& a) {
  const dim3 grid((unsigned)std::min<int64_t>(a.rows, 1 << 20)), block(BT);
  if (!a.bytes)
    hipLaunchKernelGGL((norm_row_kernel<T, W, false, false>), grid, block, 0, s, a);
  else if (a.plain)
    hipLaunchKernelGGL((norm_row_kernel<T, W, true, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((norm_row_kernel<T, W, true, false>), grid, block, 0, s, a);
  KMP_LAUNCH_CHECK();
  return 0;
}

template <typename T, typename W>
int backward_as(hipStream_t s, const NormBackArgs& a) {
  typedef typename acc_of<T>::type A;
  const int64_t parts = norm_partials(a.xtype, a.rows, a.d);
  if (a.rows > 0 && a.dx) {
    hipLaunchKernelGGL((norm_back_row_kernel<T, W>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)),
                       dim3(BT), 0, s, a);
    KMP_LAUNCH_CHECK();
  }
  if (!a.dgamma && !a.dbeta) return 0;
  if (parts > 0) {
    hipLaunchKernelGGL((norm_back_columns_kernel<T>), dim3((unsigned)ceil_div(a.d, BT), (unsigned)parts),
                       dim3(BT), 0, s, a, ceil_div(a.rows, parts));
    KMP_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL((norm_back_join_kernel<A, W>), dim3((unsigned)ceil_div(a.d, 64), 2), dim3(BT), 0, s,
                     static_cast<const A*>(a.partial), parts, a.d, static_cast<W*>(a.dgamma),
                     static_cast<W*>(a.dbeta));
  KMP_LAUNCH_CHECK();
  return 0;
}

}  // namespace

// Strips of rows whose column sums are kept apart.
int64_t norm_partials(int, int64_t rows, int64_t) { return std::min<int64_t>(ceil_div(rows, 32), 512); }

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
