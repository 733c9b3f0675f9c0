// Products of 8-bit integers with a scale per token and per channel,
//   y[m][n] = xscale[m] wscale[n] sum_k x[m][k] w[n][k] + bias[n],
// x M x K and w N x K row-major. The sums are exact in 32-bit integers up to
// K = 131071, so their order does not matter; they are converted to 32-bit
// floats, scaled, and rounded once to the output's type.
#include "kmp_operators.h"

namespace kmp {
namespace {

typedef int int4v __attribute__((ext_vector_type(4)));

// The 16 bytes of row `p` from byte k on, zeros from byte K on. No byte past K
// is touched.
__device__ __forceinline__ int4v chunk16(const int8_t* p, int64_t k, int64_t K) {
  int4v v = {0, 0, 0, 0};
  if (k + 16 <= K) {
    __builtin_memcpy(&v, p + k, 16);
  } else if (k < K) {
    int8_t b[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) b[i] = k + i < K ? p[k + i] : (int8_t)0;
    __builtin_memcpy(&v, b, 16);
  }
  return v;
}

template <typename O>
__device__ __forceinline__ O scaled(int acc, float xs, float ws, float bias) {
  return (O)((float)acc * xs * ws + bias);
}

// Tiles of 64 x 64, four wavefronts in a 2 x 2 arrangement, slices of 64 bytes
// of k through LDS (rows 16 bytes apart from a power of two, against bank
// conflicts). v_mfma_i32_16x16x64_i8: lane l holds 16 bytes of row l % 16 of
// either operand from k = 16 (l / 16) on; register r of the result is D(row 4
// (l / 16) + r, column l % 16).
template <typename O>
__global__ __launch_bounds__(256) void qproduct_tile_kernel(QProductArgs a) {
  __shared__ int4v As[64][5], Bs[64][5];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int64_t m0 = (int64_t)blockIdx.y * 64, n0 = (int64_t)blockIdx.x * 64;
  const int row = t >> 2, c = t & 3;
  const int8_t* pa = a.x + min(m0 + row, a.M - 1) * a.ldx;
  const int8_t* pb = a.w + min(n0 + row, a.N - 1) * a.ldw;
  const int wm = (w & 1) * 32, wn = (w >> 1) * 32;
  int4v acc[2][2] = {};
  for (int64_t k = 0; k < a.K; k += 64) {
    const int4v va = chunk16(pa, k + 16 * c, a.K), vb = chunk16(pb, k + 16 * c, a.K);
    __syncthreads();
    As[row][c] = va;
    Bs[row][c] = vb;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(As[wm + 16 * i + (lane & 15)][lane >> 4],
                                                          Bs[wn + 16 * j + (lane & 15)][lane >> 4],
                                                          acc[i][j], 0, 0, 0);
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int64_t n = n0 + wn + 16 * j + (lane & 15);
    if (n >= a.N) continue;
    const float ws = a.wscale[n], bias = a.bias ? a.bias[n] : 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t m = m0 + wm + 16 * i + 4 * (lane >> 4) + r;
        if (m < a.M) static_cast<O*>(a.out)[m * a.ldo + n] = scaled<O>(acc[i][j][r], a.xscale[m], ws, bias);
      }
  }
}

template <typename O>
int product_as(hipStream_t s, const QProductArgs& a) {
  hipLaunchKernelGGL(qproduct_tile_kernel<O>, dim3((unsigned)ceil_div(a.N, 64), (unsigned)ceil_div(a.M, 64)),
                     dim3(256), 0, s, a);
  KMP_LAUNCH_CHECK();
  return 0;
}

}  // namespace

int quantized_product(hipStream_t s, const QProductArgs& a) {
  switch (a.otype) {
    case KMP_F32: return product_as<float>(s, a);
    case KMP_BF16: return product_as<bf16_t>(s, a);
    default: return product_as<f16_t>(s, a);
  }
}

}  // namespace kmp
