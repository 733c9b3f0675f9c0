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

typedef int int16v __attribute__((ext_vector_type(16)));

// 16 bytes per lane from memory straight into LDS, at `lds` + 16 lane (lds the
// same for the wavefront). The compiler does not count these loads: they are
// waited for by wait_loads.
__device__ __forceinline__ void load_to_lds(const int8_t* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Tiles of TM x TN, WR x WC wavefronts of 32 x 32 blocks of v_mfma_i32_32x32x32_i8
// each (lane l holds 16 bytes of row l % 32 of either operand from k = 16 (l / 32)
// on; register r of the result is D(row 8 (r / 4) + 4 (l / 32) + r % 4, column l %
// 32)), slices of 128 bytes of k through two LDS stages: while one is multiplied
// the next is on its way. A row of a slice is eight 16-byte chunks, chunk c kept
// at place c ^ (row % 8), so that eight lanes with eight rows and one c read all
// banks. Rows past the end repeat the last one and are not stored; a last slice
// that is not whole is brought up with zeros. ALIGNED: rows start at multiples of
// 16 bytes and go from memory to LDS without registers.
template <typename O, int TM, int TN, int WR, int WC, bool ALIGNED>
__global__ __launch_bounds__(64 * WR * WC, 2) void qproduct_tile_kernel(QProductArgs a, int tm, int tn) {
  constexpr int NW = WR * WC, QA = TM / 8 / NW, QB = TN / 8 / NW;   // loads a wavefront, 8 rows each
  constexpr int MB = TM / WR / 32, NB = TN / WC / 32;
  constexpr int STAGE = (TM + TN) * 128;
  __shared__ __align__(16) int8_t lds[2 * STAGE];
  // workgroups go round the 8 chiplets: each takes a run of tiles of its own, in
  // groups of four tile rows, for its cache
  const int per = (tm * tn + 7) / 8, id = (int)blockIdx.x / 8 + ((int)blockIdx.x % 8) * per;
  if ((int)blockIdx.x / 8 >= per || id >= tm * tn) return;
  const int group = id / (4 * tn), rows = min(4, tm - 4 * group), in = id - group * 4 * tn;
  const int64_t m0 = (int64_t)(4 * group + in % rows) * TM, n0 = (int64_t)(in / rows) * TN;
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wr = w / WC, wc = w % WC;
  const int lr = lane >> 3, lc = ((lane & 7) ^ lr) * 16;            // loads: row of 8, byte of the slice
  const int8_t* pa[QA];
  const int8_t* pb[QB];
#pragma unroll
  for (int q = 0; q < QA; ++q) pa[q] = a.x + min(m0 + (w * QA + q) * 8 + lr, a.M - 1) * a.ldx + lc;
#pragma unroll
  for (int q = 0; q < QB; ++q) pb[q] = a.w + min(n0 + (w * QB + q) * 8 + lr, a.N - 1) * a.ldw + lc;
  const uint32_t base = (uint32_t)(uintptr_t)lds;                   // LDS addresses have 32 bits
  const auto fetch = [&](int k, int st) {                           // ALIGNED: starts the loads of a whole slice
#pragma unroll
    for (int q = 0; q < QA; ++q) load_to_lds(pa[q] + k, base + st * STAGE + (w * QA + q) * 1024);
#pragma unroll
    for (int q = 0; q < QB; ++q) load_to_lds(pb[q] + k, base + st * STAGE + TM * 128 + (w * QB + q) * 1024);
  };
  int4v ra[QA], rb[QB];
  const auto pull = [&](int k) {                                    // a slice into registers, zeros past K
#pragma unroll
    for (int q = 0; q < QA; ++q) ra[q] = chunk16(pa[q] - lc, k + lc, a.K);
#pragma unroll
    for (int q = 0; q < QB; ++q) rb[q] = chunk16(pb[q] - lc, k + lc, a.K);
  };
  const auto push = [&](int st) {
#pragma unroll
    for (int q = 0; q < QA; ++q) *reinterpret_cast<int4v*>(lds + st * STAGE + (w * QA + q) * 1024 + lane * 16) = ra[q];
#pragma unroll
    for (int q = 0; q < QB; ++q)
      *reinterpret_cast<int4v*>(lds + st * STAGE + TM * 128 + (w * QB + q) * 1024 + lane * 16) = rb[q];
  };
  int16v acc[MB][NB] = {};
  const int row = lane & 31, half = lane >> 5;
  const int8_t* la = lds + (wr * MB * 32 + row) * 128;
  const int8_t* lb = lds + TM * 128 + (wc * NB * 32 + row) * 128;
  const auto multiply = [&](int st) {
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      const int c = ((2 * ks + half) ^ (row & 7)) * 16 + st * STAGE;
      int4v fa[MB], fb[NB];
#pragma unroll
      for (int i = 0; i < MB; ++i) fa[i] = *reinterpret_cast<const int4v*>(la + i * 32 * 128 + c);
#pragma unroll
      for (int j = 0; j < NB; ++j) fb[j] = *reinterpret_cast<const int4v*>(lb + j * 32 * 128 + c);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[i], fb[j], acc[i][j], 0, 0, 0);
    }
  };
  const int whole = (int)a.K / 128, tail = (int)a.K % 128;
  if constexpr (ALIGNED) {
    if (whole > 0) {
      fetch(0, 0);
      wait_loads();
      __syncthreads();
      for (int s = 0; s < whole; ++s) {
        if (s + 1 < whole) fetch((s + 1) * 128, (s + 1) & 1);
        multiply(s & 1);
        wait_loads();
        __syncthreads();
      }
    }
    if (tail > 0) {
      pull(whole * 128);
      push(0);
      __syncthreads();
      multiply(0);
    }
  } else {
    const int slices = whole + (tail > 0);
    if (slices > 0) pull(0);
    for (int s = 0; s < slices; ++s) {                              // (the stages alternate: one barrier each)
      push(s & 1);
      __syncthreads();
      if (s + 1 < slices) pull((s + 1) * 128);
      multiply(s & 1);
    }
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int64_t n = n0 + wc * NB * 32 + j * 32 + row;
    if (n >= a.N) continue;
    const float ws = a.wscale[n], bias = a.bias ? a.bias[n] : 0.0f;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int64_t m = m0 + wr * MB * 32 + i * 32 + 8 * (r / 4) + 4 * half + r % 4;
        if (m < a.M) static_cast<O*>(a.out)[m * a.ldo + n] = scaled<O>(acc[i][j][r], a.xscale[m], ws, bias);
      }
  }
}

template <typename O, int TM, int TN, int WR, int WC>
int tiles_as(hipStream_t s, const QProductArgs& a) {
  const int tm = (int)ceil_div(a.M, TM), tn = (int)ceil_div(a.N, TN);
  const bool aligned = ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w) | a.ldx | a.ldw) & 15) == 0;
  const dim3 grid((unsigned)round_up((int64_t)tm * tn, 8)), block(64 * WR * WC);
  if (aligned)
    hipLaunchKernelGGL((qproduct_tile_kernel<O, TM, TN, WR, WC, true>), grid, block, 0, s, a, tm, tn);
  else
    hipLaunchKernelGGL((qproduct_tile_kernel<O, TM, TN, WR, WC, false>), grid, block, 0, s, a, tm, tn);
  KMP_LAUNCH_CHECK();
  return 0;
}

template <typename O>
int product_as(hipStream_t s, const QProductArgs& a) {
  if (ceil_div(a.M, 256) * ceil_div(a.N, 256) >= 192) return tiles_as<O, 256, 256, 2, 4>(s, a);
  return tiles_as<O, 128, 128, 2, 2>(s, a);
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
