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

// Few tokens: a workgroup takes 16 channels and up to 16 tokens, its four wavefronts
// each a run of the 64-byte slices of k, both operands from memory to registers, DEEP
// slices in flight; the wavefronts' sums are added in LDS in their order. w is the first
// operand of a block of 16 x 16, so that a lane has four channels of one token. Rows past
// the end repeat the last one and are not stored. Bound by reading w once.
template <typename E, typename O>
__global__ __launch_bounds__(256) void dense_few_kernel(TileArgs a, OutArgs o) {
  constexpr int DEEP = 8;
  __shared__ float sums[4][4][64];
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int row = lane & 15, c = (lane >> 4) * 16;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int8_t* pw = a.w + min(n0 + row, a.N - 1) * a.ldw;
  const int8_t* px = a.x + min((int64_t)row, a.M - 1) * a.ldx;
  // whole slices, dealt to the wavefronts in runs of n from s0 on
  const int whole = (int)(a.K / 64), run = (whole + 3) / 4;
  const int s0 = min(w * run, whole), n = min(s0 + run, whole) - s0;
  typename Blocks<E>::acc16_t acc = {};
  int4v fw[DEEP], fx[DEEP];
  const auto fetch = [&](int i, int4v& vw, int4v& vx) {
    const int k = 64 * (s0 + min(i, n - 1)) + c;  // past the end: the last slice again, unused
    __builtin_memcpy(&vw, pw + k, 16);
    __builtin_memcpy(&vx, px + k, 16);
  };
  if (n > 0) {
#pragma unroll
    for (int p = 0; p < DEEP; ++p) fetch(p, fw[p], fx[p]);
    int i = 0;
    for (; i + DEEP < n; i += DEEP) {
#pragma unroll
      for (int p = 0; p < DEEP; ++p) {
        acc = Blocks<E>::multiply16(fw[p], fx[p], acc);
        fetch(i + DEEP + p, fw[p], fx[p]);
      }
    }
#pragma unroll
    for (int p = 0; p < DEEP; ++p)
      if (i + p < n) acc = Blocks<E>::multiply16(fw[p], fx[p], acc);
  }
  if (w == 3 && a.K % 64 != 0)                    // the rest of k, zeros past its end
    acc = Blocks<E>::multiply16(chunk16(pw, 64 * (int64_t)whole + c, a.K), chunk16(px, 64 * (int64_t)whole + c, a.K), acc);
#pragma unroll
  for (int r = 0; r < 4; ++r) sums[w][r][lane] = acc[r];
  __syncthreads();
  if (w > 0 || row >= a.M) return;
  const int64_t n1 = n0 + (lane >> 4) * 4;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (n1 + r >= a.N) continue;
    float v = ((sums[0][r][lane] + sums[1][r][lane]) + sums[2][r][lane]) + sums[3][r][lane];
    if (o.bias) v += bias_at<E>(o, n1 + r);
    if (o.z) static_cast<E*>(o.z)[row * o.ldz + n1 + r] = (E)v;
    v = activate(o.act, v);
    if (o.residual) v += (float)static_cast<const O*>(o.residual)[row * o.ldr + n1 + r];
    static_cast<O*>(o.out)[row * o.ldo + n1 + r] = (O)v;
  }
}
template <typename E, typename O>
int few_as(hipStream_t s, const TileArgs& a, const OutArgs& out) {
  hipLaunchKernelGGL((dense_few_kernel<E, O>), dim3((unsigned)ceil_div(a.N, 16)), dim3(256), 0, s, a, out);
  KMP_LAUNCH_CHECK();
  return 0;
}

// Which form, by what keeps the chip's 256 compute units busy. us per launch at M x N x
// K, in a recorded graph, the forms in turn, operands from HBM: few tokens; tiles of 32 x 64
// (four groups over k, ring of 3), 64 x 64 (two groups, ring of 3, or of 2; one group, ring
// of 2), operands ahead in tiles of 128 (ring of 4, or of 2), 256 x 128 and 256 x 256; the
// floor, the larger of the bytes at a copy's 4.93 TB/s and the products at the 1574 TFLOP/s
// (bf16; f32: 155) of the library's product of order 8192. In bf16:
//                        few  32x64  64,3  64,2  64,1 128,4 128,2 256,128  256  floor
//   1 x 4096 x 4096      8.9   15.7  18.5  30.4  47.4  31.2  56.2    65.8 83.6    6.8
//   1 x 16384 x 4096    24.6   29.7  30.7  35.9  51.4  37.8  61.4    70.7 89.4   27.2
//   16 x 8192 x 4096    20.4   18.4  20.3  31.5  48.3  31.8  57.6    67.3 85.3   13.7
//   16 x 32000 x 2048   38.6   31.1  31.6  29.2  32.2  33.4  36.8    42.4 51.2   26.8
//   64 x 4096 x 4096           18.6  23.5  33.1  48.5  35.6  60.2    71.1 89.7    7.0
//   64 x 12288 x 4096          35.5  26.5  34.9  49.3  37.7  60.7    71.8 90.1   20.8
//   256 x 4096 x 4096          32.7  22.7  32.1  48.4  40.7  60.2    84.2  108    7.7
//   512 x 4096 x 4096          62.5  41.6  36.3  47.9  40.3  58.2    81.2  106   10.9
//   600 x 4500 x 704           30.2  19.3  16.1  12.2  13.6  14.4    21.0 35.2    2.6
//   1000 x 3000 x 4096         86.3  58.8  64.7  52.9  39.9  58.2    78.2  105   15.6
//   1024 x 4096 x 4096          117  80.2  68.8  67.1  44.0  57.7    79.4  106   21.8
//   2048 x 2048 x 2048         63.8  44.7  36.4  34.3  26.1  32.3    41.6 58.3   10.9
//   1024 x 8192 x 4096          236   158   132   128  88.0  78.3    86.8  108   43.7
//   2048 x 4096 x 4096          210   155   130   125  86.2  77.8    84.1  105   43.7
//   3000 x 5000 x 1000          198   122  91.6  82.2  69.4  57.7    60.5 49.9   19.1
//   4096 x 4096 x 4096          394   288   239   233   168   151     159  121   87.3
//   4096 x 8192 x 4096          777   568   463   449   332   296     308  237  174.6
//   8192 x 8192 x 8192         2546  1949  1642  1673  1216  1119    1090  881  698.5
// Those of 256 x 128 are ahead of 128,2 where operands come from the last-level cache (2048 x
// 4096 x 4096 69.4 / 77.0, 1024 x 8192 x 4096 69.5 / 76.8, 1500 x 5000 x 8192 123 / 142),
// which the rule goes by, and behind it from HBM (84.1 / 77.8, 86.8 / 78.3, 145 / 142).
// In f32 (128: of four wavefronts, ring of 2):
//                        few  32x64  64,2   128  floor
//   1 x 4096 x 4096     16.1   44.3  77.2   253   13.6
//   128 x 4096 x 1000          19.6  25.8  74.5    6.8
//   1024 x 1024 x 1024         31.0  25.6  72.4   13.9
//   2048 x 2048 x 2048          189   154   138  110.8
//   4096 x 4096 x 1024          431   304   274  221.7
// Rows that are not aligned, f16: few tokens; tiles of 32 x 64 (four groups), 64 and 128:
//                      few  32x64    64   128  floor
//   16 x 4096 x 4097  11.5  17.8  22.1  36.3   6.9
//   77 x 2051 x 8191        23.9  31.6  59.4   7.1
//   128 x 4096 x 4097       20.9  24.5  45.4   7.2
//   512 x 4096 x 4097       75.2  45.8  45.6  11.4
//   1244 x 1824 x 5001       108  72.5  55.2  15.1
//   4096 x 4096 x 4097       573   329   206  91.4
template <typename E, typename O>
int product_as(hipStream_t s, const TileArgs& a, const OutArgs& out) {
  typedef DenseTile<E, O> S;
  const auto tiles = [&](int tm, int tn) { return ceil_div(a.M, tm) * ceil_div(a.N, tn); };
  // (a launch has fewer than 2^32 threads: few_as takes 256 for 16 channels)
  if (a.M <= 16 && (a.N <= 6144 || (a.M <= 4 && a.N <= ((int64_t)1 << 28) - 16))) return few_as<E, O>(s, a, out);
  // the fewest tiles: eight groups over k (32x64 above; us: 77 x 2051 x 8192 23.9 / 26.8,
  // 64 x 1000 x 8192 24.2 / 27.8, 128 x 2048 x 4096 15.2 / 17.2; f32 77 x 2051 x 4096 28.6
  // / 45.0; rows not aligned 77 x 2051 x 8191 29.9 / 39.2, 32 x 4096 x 4097 17.5 / 22.8)
  const bool least = tiles(32, 32) <= 256;
  if (!aligned_rows(a)) {
    if (least) return tiles_as<E, S, 32, 32, 1, 1, 8, 2, false>(s, a, out);
    if (tiles(32, 64) <= 256) return tiles_as<E, S, 32, 64, 1, 2, 4, 2, false>(s, a, out);
    if (tiles(64, 64) <= 512) return tiles_as<E, S, 64, 64, 2, 2, 1, 2, false>(s, a, out);
    return tiles_as<E, S, 128, 128, 2, 4, 1, 2, false>(s, a, out);
  }
  if (least) return tiles_as<E, S, 32, 32, 1, 1, 8, 2, true>(s, a, out);
  if (tiles(32, 64) <= 256) return tiles_as<E, S, 32, 64, 1, 2, 4, 3, true>(s, a, out);
  if constexpr (sizeof(E) == 4) {
    if (tiles(64, 64) <= 512) return tiles_as<E, S, 64, 64, 2, 2, 2, 2, true>(s, a, out);
    return ahead_as<E, S, 128, 128, 2, 2, 2>(s, a, out);
  } else {
    if (tiles(64, 64) <= 256) return tiles_as<E, S, 64, 64, 2, 2, 2, 3, true>(s, a, out);
    if (tiles(64, 64) <= 512) return tiles_as<E, S, 64, 64, 2, 2, 2, 2, true>(s, a, out);
    if (tiles(64, 64) <= 768 && (a.K < 4096 || tiles(128, 128) > 256)) return tiles_as<E, S, 64, 64, 2, 2, 1, 2, true>(s, a, out);
    if (tiles(128, 128) <= 256) return ahead_as<E, S, 128, 128, 2, 4, 4>(s, a, out);
    if (tiles(256, 256) < 192) return ahead_as<E, S, 256, 128, 4, 2, 2>(s, a, out);
    return ahead_as<E, S, 256, 256, 2, 4, 2>(s, a, out);
  }
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
struct TurnsArgs { TurnArgs each[3]; int64_t tiles[3]; };   // up to three in one launch
template <typename T>
__global__ __launch_bounds__(256) void turn_kernel(TurnsArgs all) {
  constexpr int S = 64, VEC = vec_of<T>(), PER = S / VEC, RPI = 256 / PER;
  __shared__ T tile[S][S + 2];
  __shared__ float sums[RPI][S];
  const int lr = threadIdx.x / PER, c = threadIdx.x % PER * VEC;
  for (int64_t job = blockIdx.x; job < all.tiles[0] + all.tiles[1] + all.tiles[2]; job += gridDim.x) {
    const int which = job < all.tiles[0] ? 0 : job < all.tiles[0] + all.tiles[1] ? 1 : 2;
    const TurnArgs a = all.each[which];
    const int64_t at = job - (which > 0 ? all.tiles[0] : 0) - (which > 1 ? all.tiles[1] : 0), across = ceil_div(a.cols, S);
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

// Few tokens (M <= MM <= kFew) take no part of the above: reading w once for dx and
// writing dw once is all that counts, and dz stays in 32 bits.
// dz [N][MM], zeros from M on, so that a channel's are one load for a whole wavefront;
// and its sums over the tokens. A thread per channel.
template <typename T, typename W, int MM>
__global__ __launch_bounds__(256) void few_dz_kernel(DenseBackArgs a, float* dz) {
  for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < a.N; n += (int64_t)gridDim.x * 256) {
    float sum = 0.0f;
#pragma unroll
    for (int m = 0; m < MM; ++m) {
      float v = 0.0f;
      if (m < a.M) {
        v = (float)static_cast<const T*>(a.dout)[m * a.lddo + n];
        if (a.act != KMP_ACT_NONE) v *= slope(a.act, (float)static_cast<const T*>(a.z)[m * a.ldz + n]);
        sum += v;
      }
      dz[n * MM + m] = v;
    }
    if (a.dbias) static_cast<W*>(a.dbias)[n] = (W)sum;
  }
}
// N elements from k on of a row of K (zeros past its end), as 32-bit floats.
template <typename T, int N>
__device__ __forceinline__ void load_part(const T* p, int64_t k, int64_t K, float (&v)[N]) {
  if (k + N <= K) {
    load_n(p + k, v);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = k + e < K ? (float)p[k + e] : 0.0f;
  }
}
// Sums over the run blockIdx.y of w's rows: a wavefront has 64 vectors of columns, the
// workgroup's four every fourth row; partial[run][m][k].
template <typename T, int MM>
__global__ __launch_bounds__(256) void few_dx_kernel(DenseBackArgs a, const float* dz, float* partial, int64_t run) {
  constexpr int VEC = vec_of<T>(), U = 4;
  __shared__ float sums[3][MM][VEC][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t k = ((int64_t)blockIdx.x * 64 + lane) * VEC, from = blockIdx.y * run, to = min(a.N, from + run);
  float acc[MM][VEC] = {};
  for (int64_t n0 = from + w; n0 < to; n0 += 4 * U) {
    float v[U][VEC], f[U][MM];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int64_t n = min(n0 + 4 * i, to - 1);
      load_part(static_cast<const T*>(a.w) + n * a.ldw, k, a.K, v[i]);
#pragma unroll
      for (int m = 0; m < MM; ++m) f[i][m] = dz[n * MM + m];
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (n0 + 4 * i >= to) continue;             // (not 0 times what may be infinite)
#pragma unroll
      for (int m = 0; m < MM; ++m)
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[m][e] += f[i][m] * v[i][e];
    }
  }
  if (w > 0) {
#pragma unroll
    for (int m = 0; m < MM; ++m)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sums[w - 1][m][e][lane] = acc[m][e];
  }
  __syncthreads();
  if (w > 0) return;
#pragma unroll
  for (int m = 0; m < MM; ++m) {
    if (m >= a.M) continue;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float s = ((acc[m][e] + sums[0][m][e][lane]) + sums[1][m][e][lane]) + sums[2][m][e][lane];
      if (k + e < a.K) partial[((int64_t)blockIdx.y * a.M + m) * a.K + k + e] = s;
    }
  }
}
template <typename T>
__global__ __launch_bounds__(256) void few_join_kernel(DenseBackArgs a, const float* partial, int runs) {
  const int64_t all = a.M * a.K;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    float s = 0.0f;
#pragma unroll 8
    for (int r = 0; r < runs; ++r) s += partial[r * all + i];
    static_cast<T*>(a.dx)[i / a.K * a.lddx + i % a.K] = (T)s;
  }
}
// dw: a wavefront keeps the tokens' 64 vectors of columns and goes along its rows.
template <typename T, int MM>
__global__ __launch_bounds__(256) void few_dw_kernel(DenseBackArgs a, const float* dz, int64_t run) {
  constexpr int VEC = vec_of<T>();
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t k = ((int64_t)blockIdx.x * 64 + lane) * VEC, from = blockIdx.y * run, to = min(a.N, from + run);
  float x[MM][VEC];
#pragma unroll
  for (int m = 0; m < MM; ++m) {
    load_part(static_cast<const T*>(a.x) + min((int64_t)m, a.M - 1) * a.ldx, k, a.K, x[m]);
    if (m >= a.M) {                               // (tokens that are not there: 0, not 0 times what may be infinite)
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[m][e] = 0.0f;
    }
  }
  if (k >= a.K) return;
#pragma unroll 2
  for (int64_t n = from + w; n < to; n += 4) {
    float v[VEC] = {};
#pragma unroll
    for (int m = 0; m < MM; ++m) {
      const float f = dz[n * MM + m];
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] += f * x[m][e];
    }
    T* p = static_cast<T*>(a.dw) + n * a.lddw + k;
    if (k + VEC <= a.K) {
      store_n(p, v);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (k + e < a.K) p[e] = (T)v[e];
    }
  }
}
// us of a call with all three gradients, N = K = 4096 in bf16: 1 token 29, 4 tokens 36, 8
// tokens 47; by the other way 17 tokens 54, and 16 tokens by this one 84.
constexpr int kFew = 8;
// Tiles of 128 x 128 from which on w or x is taken as it is (us of a call so / by
// transposes: 256 x 4096 x 4096 with 64 tiles of dx 72.8 / 69.2, 1024 x 2048 x 2048 with 128
// of either 50.9 / 52.4, 512 x 4096 x 4096 80.3 / 86.4, 4096 x 4096 x 4096 308 / 340, 8192 x
// 4096 x 1024 213 / 260).
constexpr int kLeastTurned = 128;
// Runs of w's rows, so that about 1024 workgroups read it, of 64 rows at least.
int64_t few_runs(int64_t N, int64_t K, int vec) {
  return std::max<int64_t>(1, std::min<int64_t>({ceil_div(N, 64), 1024 / ceil_div(std::max<int64_t>(K, 1), 64 * vec), 32768}));
}
int few_tokens(int64_t M) { return M <= 1 ? 1 : M <= 4 ? 4 : kFew; }   // MM of M
// Bytes of dz and of the runs' sums; never fewer for larger M, N or K.
int64_t few_bytes(int64_t M, int64_t N, int64_t K) {
  M = std::min<int64_t>(M, kFew);
  return round_up(few_tokens(M) * N * 4, 256) + M * std::min<int64_t>(ceil_div(std::max<int64_t>(N, 1), 64) * K, 1024 * 512 + K) * 4;
}
template <typename T, int MM>
int few_backward(hipStream_t s, const DenseBackArgs& a) {
  constexpr int VEC = vec_of<T>();
  float* dz = static_cast<float*>(a.workspace);
  float* partial = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + round_up(MM * a.N * 4, 256));
  const dim3 columns((unsigned)std::min<int64_t>(ceil_div(a.N, 256), 1 << 20));
  if (a.btype == KMP_F32) hipLaunchKernelGGL((few_dz_kernel<T, float, MM>), columns, dim3(256), 0, s, a, dz);
  else hipLaunchKernelGGL((few_dz_kernel<T, T, MM>), columns, dim3(256), 0, s, a, dz);
  const int64_t across = ceil_div(a.K, 64 * VEC), runs = few_runs(a.N, a.K, VEC);
  if (a.dx && a.K > 0) {
    hipLaunchKernelGGL((few_dx_kernel<T, MM>), dim3((unsigned)across, (unsigned)runs), dim3(256), 0, s, a, dz, partial, ceil_div(a.N, runs));
    hipLaunchKernelGGL(few_join_kernel<T>, dim3((unsigned)std::min<int64_t>(ceil_div(a.M * a.K, 256), 1 << 20)), dim3(256), 0, s, a,
                       partial, (int)runs);
  }
  if (a.dw && a.K > 0)
    hipLaunchKernelGGL((few_dw_kernel<T, MM>), dim3((unsigned)across, (unsigned)runs), dim3(256), 0, s, a, dz, ceil_div(a.N, runs));
  KMP_LAUNCH_CHECK();
  return 0;
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
    bytes = std::max(partial + round_up(ceil_div(M, 64) * N * 4, 256), few_bytes(M, N, K));
  }
};

// Products with operands given the other way round (kmp_tiles.h): w, or x and w.
template <typename T, bool XT>
int turned_product(hipStream_t s, const TileArgs& a, const OutArgs& out) {
  typedef DenseTile<T, T> S;
  const auto tiles = [&](int tm, int tn) { return ceil_div(a.M, tm) * ceil_div(a.N, tn); };
  if (tiles(128, 128) <= 256) return ahead_as<T, S, 128, 128, 2, 4, 4, XT, true>(s, a, out);
  if (tiles(256, 256) < 192) return ahead_as<T, S, 256, 128, 4, 2, 2, XT, true>(s, a, out);
  return ahead_as<T, S, 256, 256, 2, 4, 2, XT, true>(s, a, out);
}
// Whether such an operand is: rows of a whole number of 16 bytes, at multiples of them.
bool turnable(const void* p, int64_t ld, int64_t cols) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0 && cols % 8 == 0;
}

template <typename T>
int backward_as(hipStream_t s, const DenseBackArgs& a) {
  constexpr int SIZE = (int)sizeof(T);
  if (a.M > 0 && a.N > 0 && a.M <= kFew) {
    switch (few_tokens(a.M)) {
      case 1: return few_backward<T, 1>(s, a);
      case 4: return few_backward<T, 4>(s, a);
      default: return few_backward<T, kFew>(s, a);
    }
  }
  const Layout at(SIZE, a.M, a.N, a.K);
  char* ws = static_cast<char*>(a.workspace);
  float* partial = reinterpret_cast<float*>(ws + at.partial);
  const bool some = a.M > 0 && a.N > 0;
  // Where w or x can be taken as they are, and the product has tiles enough for that, they
  // are not transposed first.
  const bool dx_as_is = SIZE == 2 && some && a.dx && turnable(a.w, a.ldw, a.K) && ceil_div(a.M, 128) * ceil_div(a.K, 128) >= kLeastTurned;
  const bool dw_as_is = SIZE == 2 && some && a.dw && turnable(a.x, a.ldx, a.K) && ceil_div(a.N, 128) * ceil_div(a.K, 128) >= kLeastTurned;
  if (some) {
    TurnsArgs all{};
    int n = 0;
    const auto add = [&](const TurnArgs& t) {
      all.each[n] = t;
      all.tiles[n++] = ceil_div(t.rows, 64) * ceil_div(t.cols, 64);
    };
    add(TurnArgs{a.dout, a.lddo, a.act == KMP_ACT_NONE ? nullptr : a.z, a.ldz, a.act, a.M, a.N,
                 a.dx || dw_as_is ? ws + at.dz : nullptr, at.pn, a.dw && !dw_as_is ? ws + at.dz_turned : nullptr, at.pm,
                 a.dbias ? partial : nullptr});
    if (a.dx && a.K > 0 && !dx_as_is) add(TurnArgs{a.w, a.ldw, nullptr, 0, 0, a.N, a.K, nullptr, 0, ws + at.w_turned, at.pn, nullptr});
    if (a.dw && a.K > 0 && !dw_as_is) add(TurnArgs{a.x, a.ldx, nullptr, 0, 0, a.M, a.K, nullptr, 0, ws + at.x_turned, at.pm, nullptr});
    const int64_t jobs = all.tiles[0] + all.tiles[1] + all.tiles[2];
    hipLaunchKernelGGL(turn_kernel<T>, dim3((unsigned)std::min<int64_t>(jobs, 1 << 20)), dim3(256), 0, s, all);
    KMP_LAUNCH_CHECK();
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
  const auto bytes = [](const void* p) { return static_cast<const int8_t*>(p); };
  const auto plain = [](int64_t M, int64_t N, void* out, int64_t ldo) {
    return OutArgs{M, N, KMP_ACT_NONE, false, nullptr, nullptr, 0, out, ldo, nullptr, 0};
  };
  if (a.dx && a.M > 0) {
    const OutArgs o = plain(a.M, a.K, a.dx, a.lddx);
    if (dx_as_is) {
      if constexpr (SIZE == 2)
        if (int e = turned_product<T, false>(s, TileArgs{bytes(ws + at.dz), at.pn * SIZE, bytes(a.w), a.ldw * SIZE, a.M, a.K, a.N * SIZE}, o)) return e;
    } else {
      const TileArgs t{bytes(ws + at.dz), at.pn * SIZE, bytes(ws + at.w_turned), at.pn * SIZE, a.M, a.K, a.N * SIZE};
      if (int e = product_as<T, T>(s, t, o)) return e;
    }
  }
  if (a.dw && a.N > 0) {
    const OutArgs o = plain(a.N, a.K, a.dw, a.lddw);
    if (dw_as_is) {
      if constexpr (SIZE == 2)
        if (int e = turned_product<T, true>(s, TileArgs{bytes(ws + at.dz), at.pn * SIZE, bytes(a.x), a.ldx * SIZE, a.N, a.K, a.M * SIZE}, o)) return e;
    } else {
      const TileArgs t{bytes(ws + at.dz_turned), at.pm * SIZE, bytes(ws + at.x_turned), at.pm * SIZE, a.N, a.K, a.M * SIZE};
      if (int e = product_as<T, T>(s, t, o)) return e;
    }
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
