// Products of 8-bit integers with a scale per token and per channel,
//   y[m][n] = xscale[m] wscale[n] sum_k x[m][k] w[n][k] + bias[n],
// x M x K and w N x K row-major. The sums are exact in 32-bit integers up to
// K = 131071, so their order does not matter; they are converted to 32-bit
// floats, scaled, and rounded once to the output's type.
#include "kmp_tiles.h"

namespace kmp {
namespace {

template <typename O>
__device__ __forceinline__ O scaled(int acc, float xs, float ws, float bias) {
  return (O)((float)acc * xs * ws + bias);
}

// Few tokens: a workgroup takes 16 channels and up to 16 tokens, its four wavefronts
// each a run of the 64-byte slices of k, both operands from memory to registers,
// DEEP slices in flight; the wavefronts' sums are added in LDS (whole numbers: in
// any order). v_mfma_i32_16x16x64_i8: lane l holds 16 bytes of row l % 16 of either
// operand from k = 16 (l / 16) on; register r of the result is D(row 4 (l / 16) +
// r, column l % 16): w is the first operand, so a lane has four channels of one
// token. Rows past the end repeat the last one and are not stored. Bound by reading
// w once: 1 x 4096 x 4096 in 6.0 us, 2.8 TB/s (launch, one round of loads, sum).
template <typename O>
__global__ __launch_bounds__(256) void qproduct_few_kernel(QProductArgs a) {
  constexpr int DEEP = 8;
  __shared__ int sums[4][64];
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
  (&sums[0][0])[t] = 0;
  const int row = lane & 15, c = (lane >> 4) * 16;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int8_t* pw = a.w + min(n0 + row, a.N - 1) * a.ldw;
  const int8_t* px = a.x + min((int64_t)row, a.M - 1) * a.ldx;
  // whole slices, dealt to the wavefronts in runs of n from s0 on
  const int whole = (int)a.K / 64, run = (whole + 3) / 4;
  const int s0 = min(w * run, whole), n = min(s0 + run, whole) - s0;
  int4v acc = {}, fw[DEEP], fx[DEEP];
  const auto fetch = [&](int i, int4v& vw, int4v& vx) {
    const int k = 64 * (s0 + min(i, n - 1)) + c;  // past the end: the last slice again, unused
    __builtin_memcpy(&vw, pw + k, 16);
    __builtin_memcpy(&vx, px + k, 16);
  };
  const auto products = [&](const int4v& vw, const int4v& vx) {
    acc = Blocks<int8_t>::multiply16(vw, vx, acc);
  };
  if (n > 0) {
#pragma unroll
    for (int p = 0; p < DEEP; ++p) fetch(p, fw[p], fx[p]);
    int i = 0;
    for (; i + DEEP < n; i += DEEP) {
#pragma unroll
      for (int p = 0; p < DEEP; ++p) {
        products(fw[p], fx[p]);
        fetch(i + DEEP + p, fw[p], fx[p]);
      }
    }
#pragma unroll
    for (int p = 0; p < DEEP; ++p)
      if (i + p < n) products(fw[p], fx[p]);
  }
  if (w == 3 && a.K % 64 != 0)                    // the rest of k, zeros past its end
    products(chunk16(pw, 64 * whole + c, a.K), chunk16(px, 64 * whole + c, a.K));
  __syncthreads();
#pragma unroll
  for (int r = 0; r < 4; ++r) atomicAdd(&sums[r][lane], acc[r]);
  __syncthreads();
  if (w > 0 || row >= a.M) return;
  const int64_t n1 = n0 + (lane >> 4) * 4;
  const float xs = a.xscale[row];
  O* out = static_cast<O*>(a.out) + row * a.ldo + n1;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (n1 + r < a.N) out[r] = scaled<O>(sums[r][lane], xs, a.wscale[n1 + r], a.bias ? a.bias[n1 + r] : 0.0f);
}

// Scales and writes a wavefront's MB x NB blocks of 32 x 32 from row m1, column n1
// on; the blocks are transposed (w was the first operand), so a lane has four
// neighbouring columns of one row. They go through LDS (`region`, the wavefront's
// own) into whole rows of 16-byte stores; stored straight from the registers, two
// bytes a lane, a tile of 256 x 256 took 10 us for its 128 KB, as long as 500 of k.
template <typename O>
struct ScaledTile {
  typedef QProductArgs Args;
  template <int MB, int NB>
  static constexpr int region_bytes() { return 32 * (NB * 32 * (int)sizeof(O) + 16); }
  template <int MB, int NB>
  static __device__ __forceinline__ void store(const QProductArgs& a, const int16v (&acc)[MB][NB], int64_t m1, int64_t n1,
                                               int lane, int8_t* region) {
    constexpr int S = (int)sizeof(O), STRIDE = NB * 32 * S + 16, PER = 16 / S, CH = NB * 32 / PER, RPI = 64 / CH;
    const int row = lane & 31, half = lane >> 5;
    float ws[NB][4][4], bias[NB][4][4];
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int64_t n = n1 + j * 32 + 8 * g + 4 * half;
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[j][g][e] = 0.0f;
        if (n + 4 <= a.N) {
          load_n(a.wscale + n, ws[j][g]);
          if (a.bias) load_n(a.bias + n, bias[j][g]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            ws[j][g][e] = n + e < a.N ? a.wscale[n + e] : 0.0f;
            if (a.bias && n + e < a.N) bias[j][g][e] = a.bias[n + e];
          }
        }
      }
    float xs[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) xs[i] = a.xscale[min(m1 + i * 32 + row, a.M - 1)];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          O v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = scaled<O>(acc[i][j][4 * g + e], xs[i], ws[j][g][e], bias[j][g][e]);
          __builtin_memcpy(__builtin_assume_aligned(region + row * STRIDE + (j * 32 + 8 * g + 4 * half) * S, 4 * S), v, 4 * S);
        }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int q = 0; q < 32 / RPI; ++q) {
        const int r = q * RPI + lane / CH, c = lane % CH * PER;
        const int64_t m = m1 + i * 32 + r, n = n1 + c;
        O v[PER];
        __builtin_memcpy(v, __builtin_assume_aligned(region + r * STRIDE + c * S, 16), 16);
        O* out = static_cast<O*>(a.out) + m * a.ldo + n;
        if (m < a.M && n + PER <= a.N) {
          __builtin_memcpy(out, v, 16);
        } else if (m < a.M) {
#pragma unroll
          for (int e = 0; e < PER; ++e)
            if (n + e < a.N) out[e] = v[e];
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
};

// Which form, by what keeps the chip's 256 compute units busy. us per launch at M x
// N x K (here and up to the rows that are not aligned: in a recorded graph, the forms in
// turn, operands from HBM): few tokens; tiles of 32 x 64 (four groups over k, ring of 3), 64 x 64 (two groups, ring
// of 3, or of 2 and so two workgroups a compute unit); operands ahead in tiles of 128 and
// 256; the floor, the larger of the bytes at a copy's 4.93 TB/s and the products at the
// 2380 TOP/s that the 8-bit product of order 8192 has reached:
//                         few  32x64  64,3  64,2   128   256  floor
//   1 x 4096 x 4096       6.1    8.4  10.2  14.8  25.5  41.3    3.4
//   16 x 8192 x 4096     11.7   11.4  12.2  17.5  30.7  46.4    6.9
//   16 x 32000 x 2048    21.6   18.7  19.0  15.6  19.7  28.2   13.5
//   64 x 1000 x 8192            11.8  16.4  21.9  40.1  77.3    1.8
//   64 x 4096 x 4096            10.5  13.0  17.3  30.9  45.6    3.6
//   128 x 4096 x 4096           10.4  12.7  17.1  32.3  47.2    3.7
//   256 x 4096 x 4096           18.4  13.0  17.2  31.8  53.2    4.0
//   64 x 12288 x 4096           21.1  15.5  19.7  32.9  47.8   10.6
//   64 x 32000 x 2048           27.5  20.7  17.2  20.8  29.0   14.2
//   512 x 4096 x 4096           35.1  23.3  20.6  31.5  52.3    7.2
//   2048 x 2048 x 2048          37.4  25.8  19.8  16.6  28.6    7.2
//   1024 x 8192 x 4096           129  86.9  73.1  45.6  58.2   28.9
//   3000 x 5000 x 1000           149  84.6  59.7  37.0  31.7   12.6
//   4096 x 4096 x 4096           222   161   134  85.7  68.3   57.7
//   4096 x 16384 x 4096          859   658   521   331   262  231.0
//   8192 x 8192 x 8192          1428  1094   906   610   476  462.0
// Between 512 and 768 tiles of 64 those of 128 leave compute units idle: one group a
// tile of 64 and a ring of 2, up to five workgroups a compute unit (64,1):
//                        64,2  64,1   128  floor
//   600 x 4500 x 700     13.4  10.4  11.1    1.8
//   1500 x 1500 x 1500   18.2  14.7  15.1    2.8
//   1244 x 1824 x 10909  86.8  71.6  83.2   20.8
//   1000 x 3000 x 4096   33.3  28.8  30.4   10.3
//   768 x 4096 x 8192    55.8  52.0  56.8   21.7
//   1024 x 3584 x 4096   37.2  35.9  32.1   12.6
//   2048 x 2048 x 2048   19.8  19.6  16.6    7.2
// Up to 256 tiles of 128 have a compute unit each and room for a ring of 4 there,
// which hides more of the loads than a ring of 2 (128,4):
//                        64,1   128  128,4
//   600 x 4500 x 700     10.4  11.1   10.8
//   1500 x 1500 x 1500   14.7  15.1   13.5
//   1244 x 1824 x 10909  71.6  83.2   66.4
//   4138 x 534 x 7988    53.6  58.5   44.2
//   1000 x 3000 x 4096   28.8  30.4   23.1
//   768 x 4096 x 8192    52.0  56.8   40.2
//   1024 x 3584 x 4096   35.9  32.1   25.0
//   2000 x 2000 x 8192   65.2  58.8   45.0
//   2048 x 2048 x 2048   19.6  16.6   15.6
// Few tokens with more channels than the first table's have 192 tiles of 256 and take
// them, though smaller ones are ahead (reading alone is a little faster than the copy that
// the floor's rate is of):
//                         few  32x64  64,3  64,2  64,1   128   256  floor
//   1 x 50257 x 2048     18.4   27.4  27.8  24.2  21.0  26.5  30.9   20.9
//   64 x 50257 x 2048           42.2  33.3  28.4  27.2  29.9  32.8   22.2
//   16 x 128256 x 4096    140   98.5   103  98.1  95.1  97.3   126  107.5
//   64 x 128256 x 4096           159   122   116   113   113   132  110.0
//   1 x 151936 x 4096    98.6    126   133   135   148   151   174  126.4
//   64 x 151936 x 4096           192   159   153   153   165   186  130.4
// Rows that are not aligned: few tokens; tiles of 32 x 64 (four groups), 64 and 128
// (one; 128 with eight wavefronts, with four 97 for 87 at 1244 x 1824 x 10909):
//                        few  32x64    64   128  floor
//   16 x 4096 x 4097    17.3   17.6  21.6  38.1   3.5
//   7 x 6245 x 9579     42.7   38.9  47.5  87.5  12.4
//   16 x 32000 x 2047   60.5   21.7  20.1  20.6  13.8
//   64 x 1000 x 8191           24.6  28.4  54.7   1.8
//   128 x 4096 x 4097          17.1  21.8  40.6   3.8
//   512 x 4096 x 4097          61.5  36.1  37.1   8.4
//   957 x 5082 x 1874          79.9  31.1  28.3   8.9
//   1244 x 1824 x 10909         155   110  86.2  24.3
//   4426 x 1994 x 543           107  27.4  25.2   4.7
//   3000 x 5000 x 1001          189  63.2  42.4  14.7
//   4096 x 4096 x 4097          425   213   134  67.4
template <typename O>
int product_as(hipStream_t s, const QProductArgs& a) {
  const auto tiles = [&](int tm, int tn) { return ceil_div(a.M, tm) * ceil_div(a.N, tn); };
  if (a.M <= 16 && a.N <= 6144) {
    hipLaunchKernelGGL(qproduct_few_kernel<O>, dim3((unsigned)ceil_div(a.N, 16)), dim3(256), 0, s, a);
    KMP_LAUNCH_CHECK();
    return 0;
  }
  typedef ScaledTile<O> S;
  const TileArgs t{a.x, a.ldx, a.w, a.ldw, a.M, a.N, a.K};
  if (!aligned_rows(t)) {
    if (tiles(32, 64) <= 256) return tiles_as<int8_t, S, 32, 64, 1, 2, 4, 2, false>(s, t, a);
    if (tiles(64, 64) <= 512) return tiles_as<int8_t, S, 64, 64, 2, 2, 1, 2, false>(s, t, a);
    return tiles_as<int8_t, S, 128, 128, 2, 4, 1, 2, false>(s, t, a);
  }
  if (tiles(32, 64) <= 256) return tiles_as<int8_t, S, 32, 64, 1, 2, 4, 3, true>(s, t, a);
  if (tiles(64, 64) <= 256) return tiles_as<int8_t, S, 64, 64, 2, 2, 2, 3, true>(s, t, a);
  if (tiles(64, 64) <= 512) return tiles_as<int8_t, S, 64, 64, 2, 2, 2, 2, true>(s, t, a);
  if (tiles(64, 64) <= 768 && (a.K < 2048 || tiles(128, 128) > 256)) return tiles_as<int8_t, S, 64, 64, 2, 2, 1, 2, true>(s, t, a);
  if (tiles(128, 128) <= 256) return ahead_as<int8_t, S, 128, 128, 2, 4, 4>(s, t, a);
  if (tiles(256, 256) < 192) return ahead_as<int8_t, S, 128, 128, 2, 4, 2>(s, t, a);
  return ahead_as<int8_t, S, 256, 256, 2, 4, 2>(s, t, a);
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
