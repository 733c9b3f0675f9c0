// Products with bias, activation and residual,
//   z = x W' + b,  out = act(z) + residual   (x M x K, W N x K, both along k)
// and their gradients: with dz = dout act'(z)
//   dx = dz W,  dW = dz' x,  db_n = sum_m dz[m][n].
// The products are those of kmp_tiles.h: 32-bit sums of 16-bit products (or of 32-bit
// ones); bias, activation and residual are applied to the 32-bit sums on their way out.
#include "kmp_tiles.h"

namespace kmp {
namespace {

// act(z) and act'(z). The tanh form of gelu is z / (1 + exp(-2 t)), as (1 + tanh t) / 2
// = 1 / (1 + exp(-2 t)).
constexpr float kTanhScale = 0.79788456080286535588f, kTanhCube = 0.044715f;   // sqrt(2 / pi)
__device__ __forceinline__ float sigmoid(float v) { return 1.0f / (1.0f + expf(-v)); }
__device__ __forceinline__ float activate(int act, float z) {
  switch (act) {
    case KMP_ACT_RELU: return z > 0.0f || z != z ? z : 0.0f;
    case KMP_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678118654752440f));
    case KMP_ACT_GELU_TANH: return z * sigmoid(2.0f * kTanhScale * (z + kTanhCube * z * z * z));
    case KMP_ACT_SILU: return z * sigmoid(z);
    default: return z;
  }
}
// (From |z| = 256 on the slopes are 0 or 1 in 32 bits: z is held there, where no power of
// it overflows. NaN stays.)
__device__ __forceinline__ float slope(int act, float z) {
  z = __builtin_elementwise_maximum(__builtin_elementwise_minimum(z, 256.0f), -256.0f);
  switch (act) {
    case KMP_ACT_RELU: return z > 0.0f ? 1.0f : z != z ? z : 0.0f;
    case KMP_ACT_GELU:
      return 0.5f * (1.0f + erff(z * 0.70710678118654752440f)) + z * 0.39894228040143267794f * expf(-0.5f * z * z);
    case KMP_ACT_GELU_TANH: {
      const float p = sigmoid(2.0f * kTanhScale * (z + kTanhCube * z * z * z));
      return p + z * 2.0f * p * (1.0f - p) * kTanhScale * (1.0f + 3.0f * kTanhCube * z * z);
    }
    case KMP_ACT_SILU: {
      const float p = sigmoid(z);
      return p * (1.0f + z * (1.0f - p));
    }
    default: return 1.0f;
  }
}

// What becomes of the sums.
struct OutArgs {
  int64_t M, N;
  int act;
  bool wide_bias;                      // bias in 32 bits
  const void* bias;
  const void* residual; int64_t ldr;
  void* out; int64_t ldo;
  void* z; int64_t ldz;
};
// E: type of x, W, z and of a bias that is not wide; O: of out and residual.
template <typename E>
__device__ __forceinline__ float bias_at(const OutArgs& a, int64_t n) {
  return a.wide_bias ? static_cast<const float*>(a.bias)[n] : (float)static_cast<const E*>(a.bias)[n];
}

// A wavefront's MB x NB blocks of 32 x 32 from row m1, column n1 on. The blocks are
// transposed, so a lane has four neighbouring columns of one row; 32 rows at a time go
// through LDS (`region`, the wavefront's own) in 32 bits, and come back as whole
// 16-byte vectors of the output's rows, with which those of residual and z go.
template <typename E, typename O>
struct DenseTile {
  typedef OutArgs Args;
  template <int MB, int NB>
  static constexpr int region_bytes() { return 32 * (NB * 32 + 4) * 4; }
  template <int MB, int NB>
  static __device__ __forceinline__ void store(const OutArgs& a, const float16v (&acc)[MB][NB], int64_t m1, int64_t n1,
                                               int lane, int8_t* region) {
    constexpr int STRIDE = NB * 32 + 4, PER = 16 / (int)sizeof(O), CH = NB * 32 / PER, RPI = 64 / CH;
    float* rows = reinterpret_cast<float*>(region);
    const int row = lane & 31, half = lane >> 5, c = lane % CH * PER;
    const int64_t n = n1 + c;
    float bias[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) bias[e] = a.bias && n + e < a.N ? bias_at<E>(a, n + e) : 0.0f;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * g + e];
          __builtin_memcpy(__builtin_assume_aligned(rows + row * STRIDE + j * 32 + 8 * g + 4 * half, 16), v, 16);
        }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll 1
      for (int q = 0; q < 32 / RPI; ++q) {
        const int r = q * RPI + lane / CH;
        const int64_t m = m1 + i * 32 + r;
        if (m >= a.M || n >= a.N) continue;
        float v[PER];
        __builtin_memcpy(v, __builtin_assume_aligned(rows + r * STRIDE + c, 16), sizeof(v));
#pragma unroll
        for (int e = 0; e < PER; ++e) v[e] += bias[e];
        O* out = static_cast<O*>(a.out) + m * a.ldo + n;
        const O* res = static_cast<const O*>(a.residual) + (a.residual ? m * a.ldr + n : 0);
        E* z = static_cast<E*>(a.z) + (a.z ? m * a.ldz + n : 0);
        if (n + PER <= a.N) {
          if (a.z) store_n(z, v);
#pragma unroll
          for (int e = 0; e < PER; ++e) v[e] = activate(a.act, v[e]);
          if (a.residual) {
            float s[PER];
            load_n(res, s);
#pragma unroll
            for (int e = 0; e < PER; ++e) v[e] += s[e];
          }
          store_n(out, v);
        } else {
#pragma unroll
          for (int e = 0; e < PER; ++e) {
            if (n + e >= a.N) continue;
            if (a.z) z[e] = (E)v[e];
            v[e] = activate(a.act, v[e]) + (a.residual ? (float)res[e] : 0.0f);
            out[e] = (O)v[e];
          }
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
};

template <typename E, typename O>
int product_as(hipStream_t s, const TileArgs& a, const OutArgs& out) {
  typedef DenseTile<E, O> S;
  const auto tiles = [&](int tm, int tn) { return ceil_div(a.M, tm) * ceil_div(a.N, tn); };
  if (!aligned_rows(a)) {
    if (tiles(32, 64) <= 256) return tiles_as<E, S, 32, 64, 1, 2, 4, 2, false>(s, a, out);
    if (tiles(64, 64) <= 512) return tiles_as<E, S, 64, 64, 2, 2, 1, 2, false>(s, a, out);
    return tiles_as<E, S, 128, 128, 2, 4, 1, 2, false>(s, a, out);
  }
  if (tiles(32, 64) <= 256) return tiles_as<E, S, 32, 64, 1, 2, 4, 3, true>(s, a, out);
  if (tiles(64, 64) <= 512) return tiles_as<E, S, 64, 64, 2, 2, 2, 2, true>(s, a, out);
  if (tiles(256, 256) < 192) return ahead_as<E, S, 128, 128, 2, 4, 2>(s, a, out);
  return ahead_as<E, S, 256, 256, 2, 4, 2>(s, a, out);
}

// ------------------------------------------------------------------- gradients
// The transposes of what the products take along the other index, in tiles of 64 x 64
// through LDS, with dz = dout act'(z), its rounding and its column sums on the way:
// wide rows of 16 bytes are read and written.
struct TurnArgs {
  const void* in; int64_t ldi;         // rows x cols
  const void* z; int64_t ldz; int act; // dz instead of `in` itself
  int64_t rows, cols;
  void* out; int64_t ldo;              // the same, may be null
  void* turned; int64_t ldt;           // cols x rows, may be null
  float* partial;                      // [row tiles][cols], may be null
};
template <typename T>
__global__ __launch_bounds__(256) void turn_kernel(TurnArgs a) {
  constexpr int S = 64, VEC = vec_of<T>(), PER = S / VEC, RPI = 256 / PER;
  __shared__ T tile[S][S + 2];
  __shared__ float sums[RPI][S];
  const int lr = threadIdx.x / PER, c = threadIdx.x % PER * VEC;
  const int64_t across = ceil_div(a.cols, S), tiles = ceil_div(a.rows, S) * across;
  for (int64_t at = blockIdx.x; at < tiles; at += gridDim.x) {
    const int64_t r0 = at / across * S, c0 = at % across * S;
    float sum[VEC] = {};
#pragma unroll
    for (int q = 0; q < S / RPI; ++q) {
      const int r = q * RPI + lr;
      const int64_t m = r0 + r, n = c0 + c;
      float v[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = 0.0f;
      if (m < a.rows && n < a.cols) {
        const T* p = static_cast<const T*>(a.in) + m * a.ldi + n;
        const T* pz = static_cast<const T*>(a.z) + (a.z ? m * a.ldz + n : 0);
        T* o = static_cast<T*>(a.out) + (a.out ? m * a.ldo + n : 0);
        if (n + VEC <= a.cols) {
          load_n(p, v);
          if (a.z) {
            float z[VEC];
            load_n(pz, z);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] *= slope(a.act, z[e]);
          }
          if (a.out) store_n(o, v);
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            if (n + e >= a.cols) continue;
            v[e] = (float)p[e];
            if (a.z) v[e] *= slope(a.act, (float)pz[e]);
            if (a.out) o[e] = (T)v[e];
          }
        }
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        sum[e] += v[e];
        tile[r][c + e] = (T)v[e];
      }
    }
    if (a.partial) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) sums[lr][c + e] = sum[e];
    }
    __syncthreads();
    if (a.partial && threadIdx.x < S && c0 + threadIdx.x < a.cols) {
      float s = 0.0f;
      for (int i = 0; i < RPI; ++i) s += sums[i][threadIdx.x];
      a.partial[r0 / S * a.cols + c0 + threadIdx.x] = s;
    }
    if (a.turned) {
#pragma unroll
      for (int q = 0; q < S / RPI; ++q) {
        const int r = q * RPI + lr;               // a column of the tile
        const int64_t n = c0 + r, m = r0 + c;
        if (n >= a.cols || m >= a.rows) continue;
        T v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = tile[c + e][r];
        T* o = static_cast<T*>(a.turned) + n * a.ldt + m;
        if (m + VEC <= a.rows) {
          __builtin_memcpy(o, v, 16);
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (m + e < a.rows) o[e] = v[e];
        }
      }
    }
    __syncthreads();
  }
}

// Adds the row tiles' sums in a fixed order: 64 columns a workgroup, each of its 16
// wavefronts every sixteenth part, then the sixteen.
template <typename W>
__global__ __launch_bounds__(1024) void bias_join_kernel(const float* partial, int64_t parts, int64_t n, W* dbias) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  for (int64_t j0 = (int64_t)blockIdx.x * 64; j0 < n; j0 += (int64_t)gridDim.x * 64) {
    const int64_t j = j0 + lane;
    float s = 0.0f;
    if (j < n) {
#pragma unroll 4
      for (int64_t p = w; p < parts; p += 16) s += partial[p * n + j];
    }
    red[w][lane] = s;
    __syncthreads();
    if (w == 0 && j < n) {
#pragma unroll
      for (int i = 1; i < 16; ++i) s += red[i][lane];
      dbias[j] = (W)s;
    }
    __syncthreads();
  }
}

// What the workspace holds, each part's rows at multiples of 128 bytes.
struct Layout {
  int64_t dz, dz_turned, x_turned, w_turned, partial, bytes;   // first bytes
  int64_t pn, pm;                                              // pitches of rows of N and of M elements
  Layout(int size, int64_t M, int64_t N, int64_t K) {
    pn = round_up(N, 128 / size);
    pm = round_up(M, 128 / size);
    dz = 0;
    dz_turned = dz + M * pn * size;
    x_turned = dz_turned + N * pm * size;
    w_turned = x_turned + K * pm * size;
    partial = w_turned + K * pn * size;
    bytes = partial + round_up(ceil_div(M, 64) * N * 4, 256);
  }
};

template <typename T>
int turn(hipStream_t s, const TurnArgs& a) {
  const int64_t tiles = ceil_div(a.rows, 64) * ceil_div(a.cols, 64);
  hipLaunchKernelGGL(turn_kernel<T>, dim3((unsigned)std::min<int64_t>(tiles, 1 << 20)), dim3(256), 0, s, a);
  KMP_LAUNCH_CHECK();
  return 0;
}

template <typename T>
int backward_as(hipStream_t s, const DenseBackArgs& a) {
  constexpr int SIZE = (int)sizeof(T);
  const Layout at(SIZE, a.M, a.N, a.K);
  char* ws = static_cast<char*>(a.workspace);
  float* partial = reinterpret_cast<float*>(ws + at.partial);
  const bool some = a.M > 0 && a.N > 0;
  if (some) {
    TurnArgs t{a.dout, a.lddo, a.act == KMP_ACT_NONE ? nullptr : a.z, a.ldz, a.act, a.M, a.N, a.dx ? ws + at.dz : nullptr, at.pn,
               a.dw ? ws + at.dz_turned : nullptr, at.pm, a.dbias ? partial : nullptr};
    if (int e = turn<T>(s, t)) return e;
  }
  if (a.dbias && a.N > 0) {
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(a.N, 64), 1 << 20));
    const int64_t parts = ceil_div(a.M, 64);
    if (a.btype == KMP_F32)
      hipLaunchKernelGGL(bias_join_kernel<float>, grid, dim3(1024), 0, s, partial, parts, a.N, static_cast<float*>(a.dbias));
    else
      hipLaunchKernelGGL(bias_join_kernel<T>, grid, dim3(1024), 0, s, partial, parts, a.N, static_cast<T*>(a.dbias));
    KMP_LAUNCH_CHECK();
  }
  if (a.K == 0) return 0;
  const auto product = [&](int64_t x, int64_t ldx, int64_t w, int64_t ldw, int64_t M, int64_t N, int64_t depth, void* out, int64_t ldo) {
    const TileArgs t{reinterpret_cast<const int8_t*>(ws + x), ldx * SIZE, reinterpret_cast<const int8_t*>(ws + w), ldw * SIZE, M, N,
                     depth * SIZE};
    const OutArgs o{M, N, KMP_ACT_NONE, false, nullptr, nullptr, 0, out, ldo, nullptr, 0};
    return product_as<T, T>(s, t, o);
  };
  if (a.dx && a.M > 0) {
    if (some)
      if (int e = turn<T>(s, TurnArgs{a.w, a.ldw, nullptr, 0, 0, a.N, a.K, nullptr, 0, ws + at.w_turned, at.pn, nullptr})) return e;
    if (int e = product(at.dz, at.pn, at.w_turned, at.pn, a.M, a.K, a.N, a.dx, a.lddx)) return e;
  }
  if (a.dw && a.N > 0) {
    if (some)
      if (int e = turn<T>(s, TurnArgs{a.x, a.ldx, nullptr, 0, 0, a.M, a.K, nullptr, 0, ws + at.x_turned, at.pm, nullptr})) return e;
    if (int e = product(at.dz_turned, at.pm, at.x_turned, at.pm, a.N, a.K, a.M, a.dw, a.lddw)) return e;
  }
  return 0;
}

}  // namespace

int dense_product(hipStream_t s, const DenseArgs& a) {
  const int64_t size = a.type == KMP_F32 ? 4 : 2;
  const TileArgs t{static_cast<const int8_t*>(a.x), a.ldx * size, static_cast<const int8_t*>(a.w), a.ldw * size, a.M, a.N, a.K * size};
  const OutArgs o{a.M, a.N, a.act, a.btype == KMP_F32, a.bias, a.residual, a.ldr, a.out, a.ldo, a.z, a.ldz};
  switch (a.type * 8 + a.otype) {
    case KMP_F32 * 8 + KMP_F32: return product_as<float, float>(s, t, o);
    case KMP_BF16 * 8 + KMP_BF16: return product_as<bf16_t, bf16_t>(s, t, o);
    case KMP_BF16 * 8 + KMP_F32: return product_as<bf16_t, float>(s, t, o);
    case KMP_F16 * 8 + KMP_F16: return product_as<f16_t, f16_t>(s, t, o);
    default: return product_as<f16_t, float>(s, t, o);
  }
}

size_t dense_workspace(int type, int64_t M, int64_t N, int64_t K) {
  return std::max<int64_t>(256, Layout(type == KMP_F32 ? 4 : 2, M, N, K).bytes);
}

int dense_backward(hipStream_t s, const DenseBackArgs& a) {
  switch (a.type) {
    case KMP_F32: return backward_as<float>(s, a);
    case KMP_BF16: return backward_as<bf16_t>(s, a);
    default: return backward_as<f16_t>(s, a);
  }
}

}  // namespace kmp
