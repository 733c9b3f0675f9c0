// Tiles of products of rows, out[m][n] = epilogue(sum_k x[m][k] w[n][k]), on the matrix
// cores (quantized.hip, linear.hip): operands of 1, 2 or 4 bytes an element, both with k
// along their rows, taken as bytes. What is done with a tile's sums is the epilogue's.
#pragma once

#include "kmp_operators.h"

namespace kmp {

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int16v __attribute__((ext_vector_type(16)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

struct TileArgs {
  const int8_t* x; int64_t ldx;         // M rows, ldx bytes apart
  const int8_t* w; int64_t ldw;         // N rows
  int64_t M, N, K;                      // K in bytes
};

// Products of blocks of 32 x 32 by 32 bytes of k. Lane l holds 16 bytes of row l % 32
// of either operand from byte 16 (l / 32) of k on; register r of the result is D(row 8
// (r / 4) + 4 (l / 32) + r % 4, column l % 32). Which k of 4-byte elements meet in which
// of their four products does not matter, as both operands are taken alike. Also by
// `multiply16`: blocks of 16 x 16 by 64 bytes, lane l holds row l % 16 from byte 16 (l
// / 16) on, and register r is D(row 4 (l / 16) + r, column l % 16).
template <typename E> struct Blocks;
template <> struct Blocks<int8_t> {
  typedef int sum_t;
  typedef int16v acc_t;
  typedef int4v acc16_t;
  static __device__ __forceinline__ acc_t multiply(const int4v& a, const int4v& b, const acc_t& c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ acc16_t multiply16(const int4v& a, const int4v& b, const acc16_t& c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
  }
};
template <> struct Blocks<bf16_t> {
  typedef float sum_t;
  typedef float16v acc_t;
  typedef float4v acc16_t;
  typedef bf16_t vec __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ acc_t multiply(const int4v& a, const int4v& b, const acc_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(vec, a), __builtin_bit_cast(vec, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ acc16_t multiply16(const int4v& a, const int4v& b, const acc16_t& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(vec, a), __builtin_bit_cast(vec, b), c, 0, 0, 0);
  }
};
template <> struct Blocks<f16_t> {
  typedef float sum_t;
  typedef float16v acc_t;
  typedef float4v acc16_t;
  typedef f16_t vec __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ acc_t multiply(const int4v& a, const int4v& b, const acc_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(vec, a), __builtin_bit_cast(vec, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ acc16_t multiply16(const int4v& a, const int4v& b, const acc16_t& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(vec, a), __builtin_bit_cast(vec, b), c, 0, 0, 0);
  }
};
template <> struct Blocks<float> {
  typedef float sum_t;
  typedef float16v acc_t;
  typedef float4v acc16_t;
  static __device__ __forceinline__ acc_t multiply(const int4v& a, const int4v& b, acc_t c) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__int_as_float(a[e]), __int_as_float(b[e]), c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ acc16_t multiply16(const int4v& a, const int4v& b, acc16_t c) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(a[e]), __int_as_float(b[e]), c, 0, 0, 0);
    return c;
  }
};

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

// What an epilogue has: Args, store<MB, NB>(args, acc, m1, n1, lane, region) for a
// wavefront's MB x NB blocks from row m1, column n1 on (rows and columns past the end
// are not stored), and region_bytes<MB, NB>() of LDS of the wavefront's own for it.

// Tiles of TM x TN, WR x WC wavefronts of 32 x 32 blocks each (w is the first operand,
// so the blocks are transposed), slices of 128 bytes of k through a ring of NS LDS
// stages: while one is multiplied the next NS - 1 are on their way. A row of a slice
// is eight 16-byte chunks, chunk c kept at place c ^ (row / 2 % 8), so that 16 lanes
// with 16 rows and one c read all 64 banks. Rows past the end repeat the last one
// and are not stored; a last slice that is not whole is brought up with zeros. WK >
// 1: so many groups of wavefronts, each with a ring of its own and every WK-th
// slice, for products with few tiles, whose time is the chain of slices (0.2 to 0.3
// us each); their sums are added in LDS. ALIGNED: rows start at multiples of 16
// bytes and go from memory to LDS without registers; else through registers, which
// hold the next two slices while one is multiplied.
template <typename E, typename Epi, int TM, int TN, int WR, int WC, int WK, int NS, bool ALIGNED>
__global__ __launch_bounds__(64 * WR * WC * WK) void tile_kernel(TileArgs a, typename Epi::Args out, int tm, int tn) {
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
  typename Blocks<E>::acc_t acc[MB][NB] = {};
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
        for (int j = 0; j < NB; ++j) acc[i][j] = Blocks<E>::multiply(fb[j], fa[i], acc[i][j]);
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
    typename Blocks<E>::sum_t* sums = reinterpret_cast<typename Blocks<E>::sum_t*>(lds);
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
  constexpr int REGION = Epi::template region_bytes<MB, NB>(), SUMS = (WK - 1) * TM * TN * 4;   // regions lie behind the sums
  static_assert(SUMS + NW * REGION <= WK * NS * STAGE, "sums and regions fit the ring");
  Epi::template store<MB, NB>(out, acc, m0 + wr * MB * 32, n0 + wc * NB * 32, lane, lds + SUMS + wg * REGION);
}

// Columns 32 b to 32 b + 31 of rows 16 h to 16 h + 15 of a turned slice of T columns, as
// an operand of Blocks::multiply (below).
typedef short short4v __attribute__((ext_vector_type(4)));
template <int T>
__device__ __forceinline__ int4v read_turned(const int8_t* slice, int b, int h, int lane) {
  const int l = lane & 15, group = lane >> 4;     // (16 lanes: 16 columns; groups 2 and 3: rows 8 on)
  const int at = (16 * h + 8 * (group >> 1) + (l >> 2)) * (T * 2) + ((b ^ (l >> 2)) * 4 + 2 * (group & 1) + (l >> 1 & 1)) * 16 + (l & 1) * 8;
  typedef __attribute__((address_space(3))) short4v* lds_t;
  union { short4v v[2]; int4v all; } u;
  u.v[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(uint32_t)(uintptr_t)(slice + at));
  u.v[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(uint32_t)(uintptr_t)(slice + at + 4 * (T * 2)));
  return u.all;
}
__device__ __forceinline__ int64_t round_up_to(int64_t a, int64_t b) { return (a + b - 1) / b * b; }

// The larger forms, aligned rows: slices as in tile_kernel in a ring of NS stages, and
// the operands of every 32 bytes of k are read from LDS while the 32 before them are
// multiplied: reads and loads are issued between the products, whose issue takes an
// eighth of the time that the matrix cores need for one (all of them ahead of a group of
// products left the cores idle: 8-bit 8192 x 8192 x 8192 523 / 479 us, 4096 x 16384 x 4096
// 279 / 262). The barrier of slice s stands within its last products: their operands are in
// registers, so that the stage is free for slice s + NS, and slice s + 1 has landed, so that
// its first operands can be read behind them. The last slices, behind which fewer than NS
// loads are under way, have waits of their own. (Slices of 64 bytes through four or five
// stages: 4 % slower.)
//
// XT, WT: that operand is given the other way round, K rows of M or of N elements (of two
// bytes, rows at multiples of 16 bytes), whose slice is 64 of these rows. Blocks of 4 rows
// by 16 columns come out of LDS turned by the hardware: of 16 lanes, lane l names the place
// of row l / 4, columns 4 (l % 4) on, and gets column l of the four rows. A row's 16-byte
// chunk c lies at place c ^ 4 (row % 4), so that the 32 bytes of each of four rows that 16
// lanes read, and those beside them that the next 16 read, lie on different banks.
template <typename E, typename Epi, int TM, int TN, int WR, int WC, int NS, bool XT = false, bool WT = false>
__global__ __launch_bounds__(64 * WR * WC) void ahead_kernel(TileArgs a, typename Epi::Args out, int tm, int tn) {
  constexpr int NW = WR * WC, MB = TM / WR / 32, NB = TN / WC / 32, QA = TM / 8 / NW, QB = TN / 8 / NW;
  constexpr int SL = 128, STAGE = (TM + TN) * SL;
  constexpr int READS = MB + NB, MULS = MB * NB, LOADS = QA + QB;
  static_assert(QA % 2 == 0 && QB % 2 == 0, "pairs of eight rows");
  static_assert(NW * Epi::template region_bytes<MB, NB>() <= NS * STAGE, "the regions fit the ring");
  __shared__ __align__(16) int8_t lds[NS * STAGE];
  int64_t m0, n0;
  if (!tile_of(tm, tn, TM, TN, m0, n0)) return;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = w / WC, wc = w % WC;
  const int lr = lane >> 3;                                           // loads: row of eight, byte of the slice
  const int lc[2] = {((lane & 7) ^ (lr >> 1)) * 16, ((lane & 7) ^ (4 + (lr >> 1))) * 16};
  static_assert(!(XT || WT) || (sizeof(E) == 2 && TM % 128 == 0 && TN % 128 == 0), "turned operands");
  const int8_t* pa[QA];
  const int8_t* pb[QB];
  // a turned operand's load q of width T from column c0 of C: its row of the slice, and the
  // address there (columns past the end: the last ones again)
  const auto turned_row = [&](int q, int Q, int T) { return (w * Q + q) * (512 / T) + lane / (T / 8); };
  const auto turned = [&](const int8_t* p, int64_t ld, int64_t c0, int64_t C, int q, int Q, int T) {
    const int r = turned_row(q, Q, T), c = ((lane & (T / 8 - 1)) ^ 4 * (r & 3)) * 8;
    return p + r * ld + min(c0 + c, round_up_to(C, 8) - 8) * 2;
  };
#pragma unroll
  for (int q = 0; q < QA; ++q)
    pa[q] = XT ? turned(a.x, a.ldx, m0, a.M, q, QA, TM) : a.x + min(m0 + (w * QA + q) * 8 + lr, a.M - 1) * a.ldx + lc[q & 1];
#pragma unroll
  for (int q = 0; q < QB; ++q)
    pb[q] = WT ? turned(a.w, a.ldw, n0, a.N, q, QB, TN) : a.w + min(n0 + (w * QB + q) * 8 + lr, a.N - 1) * a.ldw + lc[q & 1];
  const uint32_t base = (uint32_t)(uintptr_t)lds;                     // LDS addresses have 32 bits
  const int whole = (int)a.K / SL, tail = (int)a.K % SL;
  const auto fetch_one = [&](int s, int i) {                          // load i of LOADS of slice s
    const uint32_t at = base + s % NS * STAGE;
    if (i < QA) load_to_lds(pa[i < QA ? i : 0] + (XT ? s * 64 * a.ldx : s * SL), at + (w * QA + i) * 1024);
    else load_to_lds(pb[i < QA ? 0 : i - QA] + (WT ? s * 64 * a.ldw : s * SL), at + TM * SL + (w * QB + i - QA) * 1024);
  };
  typename Blocks<E>::acc_t acc[MB][NB] = {};
  const int row = lane & 31, half = lane >> 5;
  const int8_t* la = lds + (wr * MB * 32 + row) * SL;
  const int8_t* lb = lds + TM * SL + (wc * NB * 32 + row) * SL;
  int4v fa[2][MB], fb[2][NB];
  const auto read_one = [&](int s, int h, int i) {                    // operand i of READS: bytes 32 h .. of slice s
    const int c = ((2 * h + half) ^ (row >> 1 & 7)) * 16 + s % NS * STAGE;
    const int8_t* st = lds + s % NS * STAGE;
    if (i < NB) fb[h & 1][i < NB ? i : 0] = WT ? read_turned<TN>(st + TM * SL, wc * NB + i, h, lane) : *reinterpret_cast<const int4v*>(lb + i * 32 * SL + c);
    else fa[h & 1][i < NB ? 0 : i - NB] = XT ? read_turned<TM>(st, wr * MB + i - NB, h, lane) : *reinterpret_cast<const int4v*>(la + (i - NB) * 32 * SL + c);
  };
  const auto multiply_one = [&](int h, int i) {
    acc[i / NB][i % NB] = Blocks<E>::multiply(fb[h & 1][i % NB], fa[h & 1][i / NB], acc[i / NB][i % NB]);
  };
  // products [from, to) of step h, `ops` of op(0), op(1), .. dealt out between them
  const auto multiply = [&](int h, int from, int to, int ops, auto op) {
#pragma unroll
    for (int i = from; i < to; ++i) {
      multiply_one(h, i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int o = ops * (i - from) / (to - from); o < ops * (i - from + 1) / (to - from); ++o) op(o);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (whole > 0) {
#pragma unroll
    for (int s = 0; s < NS; ++s)
      if (s < whole) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) fetch_one(s, i);
      }
    if (whole >= NS) wait_loads<(NS - 1) * LOADS>();
    else wait_loads<0>();
    barrier();
#pragma unroll
    for (int i = 0; i < READS; ++i) read_one(0, 0, i);
    // slice s with `behind` slices behind it, NS or more as NS
    const auto slice = [&](int s, auto behind) {
      constexpr int BEHIND = behind.n;
#pragma unroll
      for (int h = 0; h < 3; ++h) multiply(h, 0, MULS, READS, [&](int i) { read_one(s, h + 1, i); });
      if constexpr (BEHIND == 0) {
        multiply(3, 0, MULS, 0, [](int) {});
      } else {
        multiply(3, 0, MULS / 2, 0, [](int) {});
        wait_loads<((BEHIND < NS ? BEHIND : NS - 1) - 1) * LOADS>();  // s + 1 has landed, the later ones may not have
        wait_lds();                                                   // the last operands of s are here
        barrier();
        multiply(3, MULS / 2, MULS, READS + (BEHIND == NS ? LOADS : 0), [&](int i) {
          if (i < READS) read_one(s + 1, 0, i);
          else fetch_one(s + NS, i - READS);
        });
      }
    };
    int s = 0;
    for (; s + NS < whole; ++s) slice(s, Count<NS>());
    static_assert(NS == 2 || NS == 4, "the last slices");
    if constexpr (NS == 4) {
      if (whole - s > 3) slice(s++, Count<3>());
      if (whole - s > 2) slice(s++, Count<2>());
    }
    if (whole - s > 1) slice(s++, Count<1>());
    slice(s, Count<0>());
  }
  if (tail > 0) {                                                     // zeros past K
    __syncthreads();
    const auto rest = [&](const int8_t* p, int64_t ld, int r) {       // of a turned operand: rows past K are zeros
      int4v v = {0, 0, 0, 0};
      if (2 * r < tail) __builtin_memcpy(&v, p + whole * 64 * ld, 16);
      return v;
    };
#pragma unroll
    for (int q = 0; q < QA; ++q)
      *reinterpret_cast<int4v*>(lds + (w * QA + q) * 1024 + lane * 16) =
          XT ? rest(pa[q], a.ldx, turned_row(q, QA, TM)) : chunk16(pa[q] - lc[q & 1], whole * SL + lc[q & 1], a.K);
#pragma unroll
    for (int q = 0; q < QB; ++q)
      *reinterpret_cast<int4v*>(lds + TM * SL + (w * QB + q) * 1024 + lane * 16) =
          WT ? rest(pb[q], a.ldw, turned_row(q, QB, TN)) : chunk16(pb[q] - lc[q & 1], whole * SL + lc[q & 1], a.K);
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 4; ++h) {
#pragma unroll
      for (int i = 0; i < READS; ++i) read_one(0, h, i);
#pragma unroll
      for (int i = 0; i < MULS; ++i) multiply_one(h, i);
    }
  }
  __syncthreads();                                                    // the ring is free
  Epi::template store<MB, NB>(out, acc, m0 + wr * MB * 32, n0 + wc * NB * 32, lane, lds + w * Epi::template region_bytes<MB, NB>());
}

// Every row at a multiple of 16 bytes (a single row's pitch means nothing).
inline bool aligned_rows(const TileArgs& a) {
  const int64_t pitch = (a.M > 1 ? a.ldx : 0) | (a.N > 1 ? a.ldw : 0);
  return ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w) | (uintptr_t)pitch) & 15) == 0;
}

template <int TM, int TN, typename F, typename Args>
int launch_tiles(hipStream_t s, const TileArgs& a, const Args& out, F kernel, int threads) {
  const int tm = (int)ceil_div(a.M, TM), tn = (int)ceil_div(a.N, TN);
  hipLaunchKernelGGL(kernel, dim3((unsigned)round_up((int64_t)tm * tn, 8)), dim3(threads), 0, s, a, out, tm, tn);
  KMP_LAUNCH_CHECK();
  return 0;
}
template <typename E, typename Epi, int TM, int TN, int WR, int WC, int WK, int NS, bool ALIGNED>
int tiles_as(hipStream_t s, const TileArgs& a, const typename Epi::Args& out) {
  return launch_tiles<TM, TN>(s, a, out, tile_kernel<E, Epi, TM, TN, WR, WC, WK, NS, ALIGNED>, 64 * WR * WC * WK);
}
template <typename E, typename Epi, int TM, int TN, int WR, int WC, int NS, bool XT = false, bool WT = false>
int ahead_as(hipStream_t s, const TileArgs& a, const typename Epi::Args& out) {
  return launch_tiles<TM, TN>(s, a, out, ahead_kernel<E, Epi, TM, TN, WR, WC, NS, XT, WT>, 64 * WR * WC);
}

}  // namespace kmp
