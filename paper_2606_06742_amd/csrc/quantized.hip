// Products of 8-bit integers with a scale per token and per channel,
//   y[m][n] = xscale[m] wscale[n] sum_k x[m][k] w[n][k] + bias[n],
// x M x K and w N x K row-major. The sums are exact in 32-bit integers up to
// K = 131071, so their order does not matter; they are converted to 32-bit
// floats, scaled, and rounded once to the output's type.
#include "kmp_operators.h"

namespace kmp {
namespace {

typedef int int4v __attribute__((ext_vector_type(4)));

// The 16 bytes of row `p` from byte k on, zeros from byte K on. No byte outside
// the row is touched: where the row ends within them, its last 16 bytes are read
// and moved down (one load; sixteen conditional ones took 3 us of a short product).
__device__ __forceinline__ int4v chunk16(const int8_t* p, int64_t k, int64_t K) {
  union { int4v v; uint64_t w[2]; int8_t b[16]; } u;
  u.v = int4v{0, 0, 0, 0};
  if (k >= K) return u.v;
  const int over = (int)max((int64_t)0, k + 16 - K);
  if (over <= k) {
    __builtin_memcpy(&u, p + k - over, 16);
    if (over >= 8) {
      u.w[0] = u.w[1] >> (8 * over - 64);
      u.w[1] = 0;
    } else if (over > 0) {
      u.w[0] = u.w[0] >> (8 * over) | u.w[1] << (64 - 8 * over);
      u.w[1] >>= 8 * over;
    }
  } else {                                        // a row of less than 16 bytes
#pragma unroll
    for (int i = 0; i < 16; ++i) u.b[i] = k + i < K ? p[k + i] : (int8_t)0;
  }
  return u.v;
}

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
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(vw, vx, acc, 0, 0, 0);
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

typedef int int16v __attribute__((ext_vector_type(16)));

// 16 bytes per lane from memory straight into LDS, at `lds` + 16 lane (lds the
// same for the wavefront). The compiler does not count these loads: they are
// waited for by wait_loads.
__device__ __forceinline__ void load_to_lds(const int8_t* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
}
// Waits until no more than LEFT of the wavefront's last loads are under way.
template <int LEFT>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory"); }

__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// Barrier of the workgroup that leaves the wavefront's own reads and loads under
// way (what has to have ended is waited for before it, or by its use).
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }

// First row and column of a workgroup's tile; false where it has none. Workgroups
// go round the 8 chiplets: each takes a run of tiles of its own, in groups of four
// tile rows, for its cache.
__device__ __forceinline__ bool tile_of(int tm, int tn, int TM, int TN, int64_t& m0, int64_t& n0) {
  const int per = (tm * tn + 7) / 8, id = (int)blockIdx.x / 8 + ((int)blockIdx.x % 8) * per;
  if ((int)blockIdx.x / 8 >= per || id >= tm * tn) return false;
  const int group = id / (4 * tn), rows = min(4, tm - 4 * group), in = id - group * 4 * tn;
  m0 = (int64_t)(4 * group + in % rows) * TM;
  n0 = (int64_t)(in / rows) * TN;
  return true;
}

// Scales and writes a wavefront's MB x NB blocks of 32 x 32 from row m1, column n1
// on; the blocks are transposed (w was the first operand), so a lane has four
// neighbouring columns of one row. They go through LDS (`region`, the wavefront's
// own) into whole rows of 16-byte stores; stored straight from the registers, two
// bytes a lane, a tile of 256 x 256 took 10 us for its 128 KB, as long as 500 of k.
template <typename O, int MB, int NB>
constexpr int region_bytes() { return 32 * (NB * 32 * (int)sizeof(O) + 16); }
template <typename O, int MB, int NB>
__device__ __forceinline__ void store_tile(const QProductArgs& a, const int16v (&acc)[MB][NB], int64_t m1, int64_t n1,
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

// Tiles of TM x TN, WR x WC wavefronts of 32 x 32 blocks of v_mfma_i32_32x32x32_i8
// each (lane l holds 16 bytes of row l % 32 of either operand from k = 16 (l / 32)
// on; register r of the result is D(row 8 (r / 4) + 4 (l / 32) + r % 4, column l %
// 32); w is the first operand), slices of 128 bytes of k through a ring of NS LDS
// stages: while one is multiplied the next NS - 1 are on their way. A row of a slice
// is eight 16-byte chunks, chunk c kept at place c ^ (row / 2 % 8), so that 16 lanes
// with 16 rows and one c read all 64 banks. Rows past the end repeat the last one
// and are not stored; a last slice that is not whole is brought up with zeros. WK >
// 1: so many groups of wavefronts, each with a ring of its own and every WK-th
// slice, for products with few tiles, whose time is the chain of slices (0.2 to 0.3
// us each); their sums are added in LDS. ALIGNED: rows start at multiples of 16
// bytes and go from memory to LDS without registers; else through registers, which
// hold the next two slices while one is multiplied.
template <typename O, int TM, int TN, int WR, int WC, int WK, int NS, bool ALIGNED>
__global__ __launch_bounds__(64 * WR * WC * WK) void qproduct_tile_kernel(QProductArgs a, int tm, int tn) {
  constexpr int NW = WR * WC, QA = TM / 8 / NW, QB = TN / 8 / NW;   // loads a wavefront, 8 rows each
  constexpr int MB = TM / WR / 32, NB = TN / WC / 32;
  constexpr int STAGE = (TM + TN) * 128;
  __shared__ __align__(16) int8_t lds[WK * NS * STAGE];
  int64_t m0, n0;
  if (!tile_of(tm, tn, TM, TN, m0, n0)) return;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = w / NW, wg = w % NW, wr = wg / WC, wc = wg % WC;
  // loads: row lr of eight, the byte of the slice by the row's place in sixteen
  static_assert(QA % 2 == 0 && QB % 2 == 0, "pairs of eight rows");
  const int lr = lane >> 3;
  const int lc[2] = {((lane & 7) ^ (lr >> 1)) * 16, ((lane & 7) ^ (4 + (lr >> 1))) * 16};
  const int8_t* pa[QA];
  const int8_t* pb[QB];
#pragma unroll
  for (int q = 0; q < QA; ++q) pa[q] = a.x + min(m0 + (wg * QA + q) * 8 + lr, a.M - 1) * a.ldx;
#pragma unroll
  for (int q = 0; q < QB; ++q) pb[q] = a.w + min(n0 + (wg * QB + q) * 8 + lr, a.N - 1) * a.ldw;
  int8_t* ring = lds + kg * (NS * STAGE);
  const uint32_t base = (uint32_t)(uintptr_t)ring;                  // LDS addresses have 32 bits
  const auto fetch = [&](int k, int st) {                           // ALIGNED: starts the loads of a whole slice
#pragma unroll
    for (int q = 0; q < QA; ++q) load_to_lds(pa[q] + k + lc[q & 1], base + st * STAGE + (wg * QA + q) * 1024);
#pragma unroll
    for (int q = 0; q < QB; ++q) load_to_lds(pb[q] + k + lc[q & 1], base + st * STAGE + TM * 128 + (wg * QB + q) * 1024);
  };
  const auto push = [&](const int4v (&va)[QA], const int4v (&vb)[QB], int st) {
#pragma unroll
    for (int q = 0; q < QA; ++q) *reinterpret_cast<int4v*>(ring + st * STAGE + (wg * QA + q) * 1024 + lane * 16) = va[q];
#pragma unroll
    for (int q = 0; q < QB; ++q)
      *reinterpret_cast<int4v*>(ring + st * STAGE + TM * 128 + (wg * QB + q) * 1024 + lane * 16) = vb[q];
  };
  int16v acc[MB][NB] = {};
  const int row = lane & 31, half = lane >> 5;
  const int8_t* la = ring + (wr * MB * 32 + row) * 128;
  const int8_t* lb = ring + TM * 128 + (wc * NB * 32 + row) * 128;
  const auto multiply = [&](int st) {
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      const int c = ((2 * ks + half) ^ (row >> 1 & 7)) * 16 + st * STAGE;
      int4v fa[MB], fb[NB];
#pragma unroll
      for (int i = 0; i < MB; ++i) fa[i] = *reinterpret_cast<const int4v*>(la + i * 32 * 128 + c);
#pragma unroll
      for (int j = 0; j < NB; ++j) fb[j] = *reinterpret_cast<const int4v*>(lb + j * 32 * 128 + c);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
  };
  const int whole = (int)a.K / 128, tail = (int)a.K % 128;
  const int rounds = (whole + WK - 1) / WK, mine = (whole - kg + WK - 1) / WK;       // slices kg, kg + WK, ..
  if constexpr (ALIGNED) {
    // slice s of a group goes to slot s % NS; it is read once the loads up to it
    // have landed and every wavefront is there, which frees the slot of s - 1 for
    // s + NS - 1
    constexpr int LEFT = (NS - 2) * (QA + QB);
    for (int s = 0; s < min(NS - 1, mine); ++s) fetch((s * WK + kg) * 128, s);
    int slot = 0;
    for (int s = 0; s < rounds; ++s) {
      if (s + NS - 1 <= mine) wait_loads<LEFT>();
      else wait_loads<0>();                                         // the last ones: all that is left
      __syncthreads();
      if (s + NS - 1 < mine) fetch(((s + NS - 1) * WK + kg) * 128, slot == 0 ? NS - 1 : slot - 1);
      if (s < mine) multiply(slot);
      slot = slot + 1 == NS ? 0 : slot + 1;
    }
  } else if (rounds > 0) {
    static_assert(ALIGNED || NS == 2, "two slices on their way, two stages");
    int4v ra[2][QA], rb[2][QB];
    const auto pull = [&](int s, int p) {                           // past the end: the last slice again, unused
      const int k = min(s * WK + kg, whole - 1) * 128;
#pragma unroll
      for (int q = 0; q < QA; ++q) __builtin_memcpy(&ra[p][q], pa[q] + k + lc[q & 1], 16);
#pragma unroll
      for (int q = 0; q < QB; ++q) __builtin_memcpy(&rb[p][q], pb[q] + k + lc[q & 1], 16);
    };
    pull(0, 0);
    pull(1, 1);
    int s = 0;
    for (; s + 2 < rounds; s += 2) {                                // (the stages alternate: one barrier each)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        push(ra[p], rb[p], p);
        __syncthreads();
        pull(s + p + 2, p);
        multiply(p);
      }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
      if (s + p < rounds) {
        push(ra[p], rb[p], p);
        __syncthreads();
        if (s + p < mine) multiply(p);
      }
  }
  if (tail > 0) {                                                   // the rest of k, zeros past its end
    __syncthreads();
    if (kg == WK - 1) {
      int4v va[QA], vb[QB];
#pragma unroll
      for (int q = 0; q < QA; ++q) va[q] = chunk16(pa[q], whole * 128 + lc[q & 1], a.K);
#pragma unroll
      for (int q = 0; q < QB; ++q) vb[q] = chunk16(pb[q], whole * 128 + lc[q & 1], a.K);
      push(va, vb, 0);
    }
    __syncthreads();
    if (kg == WK - 1) multiply(0);
  }
  __syncthreads();                                                  // the ring is free
  if constexpr (WK > 1) {                                           // the first group adds the others' sums
    int* sums = reinterpret_cast<int*>(lds);
    const auto at = [&](int g, int i, int j, int r) {
      return sums + (((g - 1) * NW + wg) * MB * NB + i * NB + j) * 1024 + r * 64 + lane;
    };
    if (kg > 0) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) *at(kg, i, j, r) = acc[i][j][r];
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int g = 1; g < WK; ++g)
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] += *at(g, i, j, r);
  }
  constexpr int REGION = region_bytes<O, MB, NB>(), SUMS = (WK - 1) * TM * TN * 4;   // regions lie behind the sums
  static_assert(SUMS + NW * REGION <= WK * NS * STAGE, "sums and regions fit the ring");
  store_tile<O, MB, NB>(a, acc, m0 + wr * MB * 32, n0 + wc * NB * 32, lane, lds + SUMS + wg * REGION);
}

// The larger forms, aligned rows: slices as in qproduct_tile_kernel in a ring of NS
// stages, and the operands of every 32 bytes of k are read from LDS while the 32
// before them are multiplied. The barrier of slice s stands before its last 32:
// their operands are in registers, so that the stage is free for slice s + NS, and
// slice s + 1 has landed, so that its first operands can be read behind the last
// products of s: no product waits for LDS or for the barrier. (Slices of 64 bytes
// through four stages had twice the requests to the second-level cache.)
template <typename O, int TM, int TN, int WR, int WC, int NS>
__global__ __launch_bounds__(64 * WR * WC) void qproduct_ahead_kernel(QProductArgs a, int tm, int tn) {
  constexpr int NW = WR * WC, MB = TM / WR / 32, NB = TN / WC / 32, QA = TM / 8 / NW, QB = TN / 8 / NW;
  constexpr int SL = 128, STAGE = (TM + TN) * SL;
  static_assert(QA % 2 == 0 && QB % 2 == 0, "pairs of eight rows");
  static_assert(NW * region_bytes<O, MB, NB>() <= NS * STAGE, "the regions fit the ring");
  __shared__ __align__(16) int8_t lds[NS * STAGE];
  int64_t m0, n0;
  if (!tile_of(tm, tn, TM, TN, m0, n0)) return;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = w / WC, wc = w % WC;
  const int lr = lane >> 3;                                           // loads: row of eight, byte of the slice
  const int lc[2] = {((lane & 7) ^ (lr >> 1)) * 16, ((lane & 7) ^ (4 + (lr >> 1))) * 16};
  const int8_t* pa[QA];
  const int8_t* pb[QB];
#pragma unroll
  for (int q = 0; q < QA; ++q) pa[q] = a.x + min(m0 + (w * QA + q) * 8 + lr, a.M - 1) * a.ldx + lc[q & 1];
#pragma unroll
  for (int q = 0; q < QB; ++q) pb[q] = a.w + min(n0 + (w * QB + q) * 8 + lr, a.N - 1) * a.ldw + lc[q & 1];
  const uint32_t base = (uint32_t)(uintptr_t)lds;                     // LDS addresses have 32 bits
  const auto fetch = [&](int s) {
    const uint32_t at = base + s % NS * STAGE;
#pragma unroll
    for (int q = 0; q < QA; ++q) load_to_lds(pa[q] + s * SL, at + (w * QA + q) * 1024);
#pragma unroll
    for (int q = 0; q < QB; ++q) load_to_lds(pb[q] + s * SL, at + TM * SL + (w * QB + q) * 1024);
  };
  int16v acc[MB][NB] = {};
  const int row = lane & 31, half = lane >> 5;
  const int8_t* la = lds + (wr * MB * 32 + row) * SL;
  const int8_t* lb = lds + TM * SL + (wc * NB * 32 + row) * SL;
  int4v fa[2][MB], fb[2][NB];
  const auto read = [&](int s, int h) {                               // bytes 32 h .. of slice s
    const int c = ((2 * h + half) ^ (row >> 1 & 7)) * 16 + s % NS * STAGE;
#pragma unroll
    for (int i = 0; i < MB; ++i) fa[h & 1][i] = *reinterpret_cast<const int4v*>(la + i * 32 * SL + c);
#pragma unroll
    for (int j = 0; j < NB; ++j) fb[h & 1][j] = *reinterpret_cast<const int4v*>(lb + j * 32 * SL + c);
    __builtin_amdgcn_sched_barrier(0);                                // (else the reads sink to their uses)
  };
  const auto multiply = [&](int h) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[h & 1][j], fa[h & 1][i], acc[i][j], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  const int whole = (int)a.K / SL, tail = (int)a.K % SL;
  if (whole > 0) {
    for (int s = 0; s < min(NS, whole); ++s) fetch(s);
    if (whole >= NS) wait_loads<(NS - 1) * (QA + QB)>();
    else wait_loads<0>();
    barrier();
    read(0, 0);
    for (int s = 0; s < whole; ++s) {
#pragma unroll
      for (int h = 0; h < 3; ++h) {
        read(s, h + 1);
        multiply(h);
      }
      if (s + NS <= whole) wait_loads<(NS - 2) * (QA + QB)>();        // s + 1 has landed, the later ones may not have
      else wait_loads<0>();
      wait_lds();                                                     // the last operands of s are here
      barrier();
      if (s + NS < whole) fetch(s + NS);
      if (s + 1 < whole) read(s + 1, 0);
      multiply(3);
    }
  }
  if (tail > 0) {                                                     // zeros past K
    __syncthreads();
#pragma unroll
    for (int q = 0; q < QA; ++q)
      *reinterpret_cast<int4v*>(lds + (w * QA + q) * 1024 + lane * 16) =
          chunk16(pa[q] - lc[q & 1], whole * SL + lc[q & 1], a.K);
#pragma unroll
    for (int q = 0; q < QB; ++q)
      *reinterpret_cast<int4v*>(lds + TM * SL + (w * QB + q) * 1024 + lane * 16) =
          chunk16(pb[q] - lc[q & 1], whole * SL + lc[q & 1], a.K);
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      read(0, h);
      multiply(h);
    }
  }
  __syncthreads();                                                    // the ring is free
  store_tile<O, MB, NB>(a, acc, m0 + wr * MB * 32, n0 + wc * NB * 32, lane, lds + w * region_bytes<O, MB, NB>());
}

// Every row at a multiple of 16 bytes (a single row's pitch means nothing).
bool aligned_rows(const QProductArgs& a) {
  const int64_t pitch = (a.M > 1 ? a.ldx : 0) | (a.N > 1 ? a.ldw : 0);
  return ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w) | (uintptr_t)pitch) & 15) == 0;
}

template <int TM, int TN, typename F>
int launch_tiles(hipStream_t s, const QProductArgs& a, F kernel, int threads) {
  const int tm = (int)ceil_div(a.M, TM), tn = (int)ceil_div(a.N, TN);
  hipLaunchKernelGGL(kernel, dim3((unsigned)round_up((int64_t)tm * tn, 8)), dim3(threads), 0, s, a, tm, tn);
  KMP_LAUNCH_CHECK();
  return 0;
}
template <typename O, int TM, int TN, int WR, int WC, int WK, int NS, bool ALIGNED>
int tiles_as(hipStream_t s, const QProductArgs& a) {
  return launch_tiles<TM, TN>(s, a, qproduct_tile_kernel<O, TM, TN, WR, WC, WK, NS, ALIGNED>, 64 * WR * WC * WK);
}
template <typename O, int TM, int TN, int WR, int WC, int NS>
int ahead_as(hipStream_t s, const QProductArgs& a) {
  return launch_tiles<TM, TN>(s, a, qproduct_ahead_kernel<O, TM, TN, WR, WC, NS>, 64 * WR * WC);
}

// Which form, by what keeps the chip's 256 compute units busy. us per launch at M x
// N x K, w from HBM: few tokens; tiles of 32 x 64 (four groups over k, ring of 3), 64
// x 64 (two groups, ring of 3, or of 2 and so two workgroups a compute unit); operands
// ahead in tiles of 128 and 256; the floor, the larger of the bytes at a copy's 4.82
// TB/s and the products at the 2040 TOP/s of the library's 8-bit product of order 8192:
//                      few  32x64  64,3  64,2   128   256  floor
//   1 x 4096 x 4096    6.0   7.5   9.7  12.0  20.9  48.7   3.5
//   16 x 8192 x 4096  11.6  10.4  11.4  16.6  30.0  51.2   7.0
//   16 x 32000 x 2048 21.2  18.2  18.5  15.6  20.3  30.4  13.8
//   64 x 1000 x 8192        11.8  15.8  21.6  39.6  91.8   1.8
//   64 x 4096 x 4096         8.1  10.1  12.9  22.2  49.2   3.6
//   128 x 4096 x 4096        8.7  10.7  12.8  23.4  50.2   3.8
//   256 x 4096 x 4096       14.6  11.7  13.2  23.5  52.2   4.2
//   64 x 12288 x 4096       20.8  16.5  19.8  32.3  52.6  10.8
//   64 x 32000 x 2048       27.5  21.3  18.0  21.2  31.4  14.5
//   512 x 4096 x 4096       27.0  19.6  16.6  24.0  52.0   8.4
//   2048 x 2048 x 2048      35.9  24.6  18.4  16.6  31.7   8.4
//   1024 x 8192 x 4096       132    89    74  45.6  60.5  33.7
//   3000 x 5000 x 1000       159    83    63  36.4  32.6  14.7
//   4096 x 4096 x 4096       224   169   135  87.0  71.0  67.4
//   4096 x 16384 x 4096      850   632   534   364   293   269
// Between 512 and 768 tiles of 64 those of 128 leave compute units idle: one group a
// tile of 64 and a ring of 2, up to five workgroups a compute unit (64,1; here and
// below in a recorded graph, 1 to 2 us more a launch):
//                       64,2  64,1   128  floor
//   600 x 4500 x 700    13.0   9.9  11.0   1.9
//   1500 x 1500 x 1500  17.3  12.7  14.5   3.3
//   1244 x 1824 x 10909 74.2  61.7  84.4  24.3
//   1000 x 3000 x 4096  34.1  28.7  32.5  12.0
//   768 x 4096 x 8192   51.1  50.6  59.5  25.3
//   1024 x 3584 x 4096  35.2  34.2  32.6  14.7
//   2048 x 2048 x 2048  18.3  18.8  16.0   8.4
// Up to 256 tiles of 128 have a compute unit each and room for a ring of 4 there,
// which hides more of the loads than a ring of 2 (128,4; in a recorded graph, both
// sides in turn):
//                       64,1   128  128,4
//   600 x 4500 x 700    10.7         11.4
//   1500 x 1500 x 1500  13.9         14.4
//   1244 x 1824 x 10909 63.6         48.4
//   4138 x 534 x 7988   44.9         39.0
//   1000 x 3000 x 4096  24.9         23.7
//   768 x 4096 x 8192   44.1         39.3
//   1024 x 3584 x 4096        26.7   23.9
//   2000 x 2000 x 8192        47.6   43.5
//   2048 x 2048 x 2048        17.1   16.1
// Few tokens with more channels than the first table's have 192 tiles of 256 and take
// them (in a recorded graph, w from HBM), though smaller ones are ahead (reading alone
// is a little faster than the copy that the floor's rate is of):
//                        few  32x64  64,3  64,2  64,1   128   256  floor
//   1 x 50257 x 2048    19.4  28.0  28.3  24.6  21.4  22.8  31.6  21.4
//   64 x 50257 x 2048         43.2  34.6  30.2  30.3  29.0  34.6  22.8
//   16 x 128256 x 4096   141   105   108   107   108   109   133   110
//   64 x 128256 x 4096         164   128   122   123   121   138   113
//   1 x 151936 x 4096    103   126   134   139   152   155   180   129
//   64 x 151936 x 4096         191   159   152   152   162   187   133
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
  if (!aligned_rows(a)) {
    if (tiles(32, 64) <= 256) return tiles_as<O, 32, 64, 1, 2, 4, 2, false>(s, a);
    if (tiles(64, 64) <= 512) return tiles_as<O, 64, 64, 2, 2, 1, 2, false>(s, a);
    return tiles_as<O, 128, 128, 2, 4, 1, 2, false>(s, a);
  }
  if (tiles(32, 64) <= 256) return tiles_as<O, 32, 64, 1, 2, 4, 3, true>(s, a);
  if (tiles(64, 64) <= 256) return tiles_as<O, 64, 64, 2, 2, 2, 3, true>(s, a);
  if (tiles(64, 64) <= 512) return tiles_as<O, 64, 64, 2, 2, 2, 2, true>(s, a);
  if (tiles(64, 64) <= 768 && (a.K < 2048 || tiles(128, 128) > 256)) return tiles_as<O, 64, 64, 2, 2, 1, 2, true>(s, a);
  if (tiles(128, 128) <= 256) return ahead_as<O, 128, 128, 2, 4, 4>(s, a);
  if (tiles(256, 256) < 192) return ahead_as<O, 128, 128, 2, 4, 2>(s, a);
  return ahead_as<O, 256, 256, 2, 4, 2>(s, a);
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
