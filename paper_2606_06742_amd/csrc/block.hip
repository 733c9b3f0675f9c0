// The norms around a model's block, fused with the block's gate and the residual
// stream, forward and backward. With N(x) = (x - mu) r g + c (mu = 0 and r from the
// mean square for the norm by the root mean square):
//   n = N(b) or b,  h = rscale res + gate n,  y = N(h)
//   s = dh + r2 (w - mean(w) - xh2 mean(w xh2)),  w = dy g2,  xh2 = (h - mu2) r2
//   dres = rscale s,  t = gate s,  db = r1 (w1 - mean(w1) - xh1 mean(w1 xh1)) or t
// (w1 = t g1, xh1 = (b - mu1) r1; without the mean of w for the root mean square), and
// over the rows, with A = sum s xh1, B = sum s for a gate per column,
//   dgate = g1 A + c1 B,  dg1 = gate A,  dc1 = gate B,  dg2 = sum dy xh2,  dc2 = sum dy
// so that four sums a column serve five gradients (for a gate per row A and B are taken
// of t, and dgate = s n has no sum). Bound by memory: b and res are read, h and y
// written, and the backward pass reads dy, dh, h and b and writes db and dres, each
// once. y is formed from h in 32 bits; the backward pass reads h as it was rounded, as
// 32 bits of it would double that read.
#include "kmp_rows.h"

namespace kmp {
namespace {

typedef float float4v __attribute__((ext_vector_type(4)));

// N elements of a weight vector (ones or zeros where there is none) from j on.
template <typename W, int N>
__device__ __forceinline__ void load_weights(const void* p, int64_t j, float none, float (&v)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = none;
  if (p) load_n(static_cast<const W*>(p) + j, v);
}

// N elements as they come from memory, in the registers that their bytes take: half of
// what 32-bit ones would for 16-bit elements.
template <typename T, int N>
struct Kept {
  uint32_t u[N * sizeof(T) / 4];
  __device__ __forceinline__ void load(const void* p, int64_t j) {
    const char* q = static_cast<const char*>(p) + j * (int64_t)sizeof(T);
#pragma unroll
    for (int c = 0; c < N * (int)sizeof(T) / 16; ++c) __builtin_memcpy(u + 4 * c, q + 16 * c, 16);
  }
  __device__ __forceinline__ void fill(float v) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const T x = (T)v;
      if constexpr (sizeof(T) == 4) u[e] = __builtin_bit_cast(uint32_t, x);
      else u[e / 2] = (uint32_t)__builtin_bit_cast(uint16_t, x) * 0x10001u;
    }
  }
  __device__ __forceinline__ void load_or(const void* p, int64_t j, float none) {
    if (p) load(p, j);
    else fill(none);
  }
  // Keeps the compiler from converting what does not change once, ahead of a loop, into
  // twice the registers.
  __device__ __forceinline__ void pin() {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) asm volatile("" : "+v"(u[i]));
    }
  }
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, u[e]);
    else return (float)__builtin_bit_cast(T, (uint16_t)(u[e / 2] >> 16 * (e & 1)));
  }
};

// Which calls a kernel is for: any; or those whose rows fill their threads' vectors and
// which have every operand but a gate per row, or that, too (`ready_for`). In the latter
// no load or store stands behind a branch, so that how many of them are under way is
// known where one is waited for: behind branches every row waited for the stores of the
// one before (DESCRIBED BELOW).
enum { kAny, kFull, kFullGate };

// Rows that fit the registers of TPR threads, NV 16-byte vectors each (longer ones of
// TPR > 64 by as many wavefronts as the row has work for): b and res are read once. The
// weights stay in registers over the rows of a workgroup, and a row's registers take the
// next one's vectors as soon as they are free: b's behind the first norm, res and the
// gate behind h, so that the loads are under way during the sums without registers of
// their own.
template <typename T, typename W, int TPR, int NV, int FORM>
__global__ __launch_bounds__(threads_of(TPR)) void block_reg_kernel(BlockArgs a) {
  constexpr int VEC = vec_of<T>(), RPB = threads_of(TPR) / TPR;
  __shared__ float red[2][threads_of(TPR) / 64], fred[2][threads_of(TPR) / 64];
  int slot = 0, fslot = 0;
  if (threadIdx.x < threads_of(TPR) / 64) {       // (wavefronts that are not there add nothing)
    red[0][threadIdx.x] = red[1][threadIdx.x] = 0.0f;
    fred[0][threadIdx.x] = fred[1][threadIdx.x] = 0.0f;
  }
  __syncthreads();
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR, d = (int)a.d;
  const int stride = RPB > 1 ? TPR : (int)blockDim.x;
  constexpr bool FULL = FORM != kAny;
  const bool each = FULL ? FORM == kFullGate : a.ldg != 0;             // a gate per row
  const auto place = [&](int i) {
    Place<VEC> q((t + i * stride) * VEC, d);
    if (FULL) q.at = (t + i * stride) * VEC, q.skip = 0;
    return q;
  };
  Kept<W, VEC> g1[NV], c1[NV], g0[NV], g2[NV], c2[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = place(i).at;
    g1[i].load_or(a.gamma_after, at, 1.0f);
    c1[i].load_or(a.beta_after, at, 0.0f);
    g0[i].load_or(each ? nullptr : a.gate, at, 1.0f);
    g2[i].load_or(a.gamma, at, 1.0f);
    c2[i].load_or(a.beta, at, 0.0f);
  }
  Kept<T, VEC> b[NV], s[NV], g[NV];
  const auto fetch = [&](const void* p, int64_t ld, int64_t r, Kept<T, VEC> (&v)[NV]) {
    const T* q = static_cast<const T*>(p) + min(r, a.rows - 1) * ld;
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i].load(q, place(i).at);
  };
  // The row's elements less their mean (none for the root mean square), and the factor.
  const auto norm = [&](float (&v)[NV][VEC], float& mu, float& rs) {
    mu = 0.0f;
    if (!a.rms) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum += v[i][e];
      mu = row_total<float, TPR>(sum, red, slot) / (float)d;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i][e] -= mu;
        clear(place(i), v[i]);
      }
    }
    float q = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) q += v[i][e] * v[i][e];
    rs = inv_sqrt(row_total<float, TPR>(q, red, slot) / (float)d + a.eps);
  };
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t r0 = (int64_t)blockIdx.x * RPB;
  fetch(a.b, a.ldb, r0 + sub, b);
  if (FULL || a.res) fetch(a.res, a.ldr, r0 + sub, s);
  if (each) fetch(a.gate, a.ldg, r0 + sub, g);
  for (; r0 < a.rows; r0 += step) {               // (every thread takes part in every round: the barriers)
    const bool live = RPB == 1 || r0 + sub < a.rows;
    const int64_t r = live ? r0 + sub : a.rows - 1;
    float v[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      g1[i].pin(), c1[i].pin(), g0[i].pin(), g2[i].pin(), c2[i].pin();
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[i][e] = b[i][e];
      clear(place(i), v[i]);
    }
    fetch(a.b, a.ldb, r0 + sub + step, b);        // past the end: the last row again, unused
    __builtin_amdgcn_sched_barrier(0);
    float mu1 = 0.0f, r1 = 1.0f, mu2 = 0.0f, r2 = 1.0f;
    if (a.after) {
      norm(v, mu1, r1);
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i][e] = v[i][e] * r1 * g1[i][e] + c1[i][e];
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[i][e] *= each ? g[i][e] : g0[i][e];
    if (FULL || a.res) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i][e] = fmaf(a.rscale, s[i][e], v[i][e]);
      fetch(a.res, a.ldr, r0 + sub + step, s);
    }
    if (each) fetch(a.gate, a.ldg, r0 + sub + step, g);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if ((FULL || a.h) && live) store_at(static_cast<T*>(a.h) + r * a.ldh, place(i), v[i]);
      clear(place(i), v[i]);
    }
    if (FULL || a.y) {
      norm(v, mu2, r2);
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i][e] = v[i][e] * r2 * g2[i][e] + c2[i][e];
      if (!FULL && a.bytes) {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          clear(place(i), v[i]);
#pragma unroll
          for (int e = 0; e < VEC; ++e) most = larger(most, fabsf(v[i][e]));
        }
        const ByteScale bs(row_most<TPR>(most, fred, fslot));
        if (live) {
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            int8_t q[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) q[e] = bs(v[i][e]);
            store_at(static_cast<int8_t*>(a.y) + r * a.ldy, place(i), q);
          }
          if (t == 0) a.scale[r] = bs.scale;
        }
      } else if (live) {
#pragma unroll
        for (int i = 0; i < NV; ++i) store_at(static_cast<T*>(a.y) + r * a.ldy, place(i), v[i]);
      }
    }
    if (t == 0 && live && a.stats) {
      const float4v st = {mu1, r1, mu2, r2};
      __builtin_memcpy(a.stats + 4 * r, &st, 16);
    }
  }
}

// One workgroup per row, any length: every pass forms what it needs from b and res
// again, so that h may be written over res in the last one.
template <typename T, typename W>
__global__ __launch_bounds__(BIG) void block_row_kernel(BlockArgs a) {
  constexpr int VEC = vec_of<T>();
  __shared__ float red[BIG / 64];
  const float d = (float)a.d;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* b = static_cast<const T*>(a.b) + r * a.ldb;
    const T* res = static_cast<const T*>(a.res) + (a.res ? r * a.ldr : 0);
    float mu1 = 0.0f, r1 = 1.0f, mu2 = 0.0f, r2 = 1.0f;
    if (a.after) {
      if (!a.rms) {
        float s = 0.0f;
        over_row<VEC>(a.d, [&](int64_t j, auto c) {
          float v[c.n];
          load_n(b + j, v);
#pragma unroll
          for (int e = 0; e < c.n; ++e) s += v[e];
        });
        mu1 = block_total(s, red) / d;
      }
      float q = 0.0f;
      over_row<VEC>(a.d, [&](int64_t j, auto c) {
        float v[c.n];
        load_n(b + j, v);
#pragma unroll
        for (int e = 0; e < c.n; ++e) q += (v[e] - mu1) * (v[e] - mu1);
      });
      r1 = inv_sqrt(block_total(q, red) / d + a.eps);
    }
    const auto values = [&](int64_t j, auto& v) {            // h
      constexpr int N = sizeof(v) / sizeof(float);
      float g[N], c[N], s[N];
      load_n(b + j, v);
      if (a.after) {
        load_weights<W>(a.gamma_after, j, 1.0f, g);
        load_weights<W>(a.beta_after, j, 0.0f, c);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (v[e] - mu1) * r1 * g[e] + c[e];
      }
      if (a.ldg == 0) load_weights<W>(a.gate, j, 1.0f, g);
      else load_n(static_cast<const T*>(a.gate) + r * a.ldg + j, g);
#pragma unroll
      for (int e = 0; e < N; ++e) s[e] = 0.0f;
      if (a.res) load_n(res + j, s);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = fmaf(a.rscale, s[e], g[e] * v[e]);
    };
    if (a.y) {
      if (!a.rms) {
        float s = 0.0f;
        over_row<VEC>(a.d, [&](int64_t j, auto c) {
          float v[c.n];
          values(j, v);
#pragma unroll
          for (int e = 0; e < c.n; ++e) s += v[e];
        });
        mu2 = block_total(s, red) / d;
      }
      float q = 0.0f;
      over_row<VEC>(a.d, [&](int64_t j, auto c) {
        float v[c.n];
        values(j, v);
#pragma unroll
        for (int e = 0; e < c.n; ++e) q += (v[e] - mu2) * (v[e] - mu2);
      });
      r2 = inv_sqrt(block_total(q, red) / d + a.eps);
    }
    if (threadIdx.x == 0 && a.stats) {
      float* st = a.stats + 4 * r;
      st[0] = mu1, st[1] = r1, st[2] = mu2, st[3] = r2;
    }
    const auto norm = [&](int64_t j, auto& v) {              // y from h
      constexpr int N = sizeof(v) / sizeof(float);
      float g[N], c[N];
      load_weights<W>(a.gamma, j, 1.0f, g);
      load_weights<W>(a.beta, j, 0.0f, c);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = (v[e] - mu2) * r2 * g[e] + c[e];
    };
    float most = 0.0f;
    if (a.bytes) {
      over_row<VEC>(a.d, [&](int64_t j, auto c) {
        float v[c.n];
        values(j, v);
        norm(j, v);
#pragma unroll
        for (int e = 0; e < c.n; ++e) most = larger(most, fabsf(v[e]));
      });
      most = block_most(most, red);
    }
    const ByteScale bs(most);
    over_row<VEC>(a.d, [&](int64_t j, auto c) {
      float v[c.n];
      values(j, v);
      if (a.h) store_n(static_cast<T*>(a.h) + r * a.ldh + j, v);
      if (!a.y) return;
      norm(j, v);
      if (a.bytes) {
        int8_t q[c.n];
#pragma unroll
        for (int e = 0; e < c.n; ++e) q[e] = bs(v[e]);
        store_n(static_cast<int8_t*>(a.y) + r * a.ldy + j, q);
      } else {
        store_n(static_cast<T*>(a.y) + r * a.ldy + j, v);
      }
    });
    if (a.bytes && threadIdx.x == 0) a.scale[r] = bs.scale;
  }
}

// db, dres and a row's dgate, one workgroup per row, any length: a pass for the two
// means of h's norm, one for those of b's, one to write. The first two go to a.means
// for the sums over the rows.
template <typename T, typename W>
__global__ __launch_bounds__(BIG) void block_back_row_kernel(BlockBackArgs a) {
  constexpr int VEC = vec_of<T>();
  __shared__ float red[BIG / 64];
  const float d = (float)a.d;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* b = static_cast<const T*>(a.b) + r * a.ldb;
    const float mu1 = a.stats[4 * r], r1 = a.stats[4 * r + 1], mu2 = a.stats[4 * r + 2], r2 = a.stats[4 * r + 3];
    const auto second = [&](int64_t j, auto& xh, auto& w) {  // xh2 and w
      constexpr int N = sizeof(w) / sizeof(float);
      float g[N];
      load_n(static_cast<const T*>(a.h) + r * a.ldh + j, xh);
      load_n(static_cast<const T*>(a.dy) + r * a.lddy + j, w);
      load_weights<W>(a.gamma, j, 1.0f, g);
#pragma unroll
      for (int e = 0; e < N; ++e) xh[e] = (xh[e] - mu2) * r2, w[e] *= g[e];
    };
    float s1 = 0.0f, s2 = 0.0f;
    if (a.dy) {
      over_row<VEC>(a.d, [&](int64_t j, auto c) {
        float xh[c.n], w[c.n];
        second(j, xh, w);
#pragma unroll
        for (int e = 0; e < c.n; ++e) s1 += w[e], s2 += w[e] * xh[e];
      });
      s1 = a.rms ? 0.0f : block_total(s1, red) / d;
      s2 = block_total(s2, red) / d;
    }
    if (a.means && threadIdx.x == 0) {
      a.means[2 * r] = s1;
      a.means[2 * r + 1] = s2;
    }
    const auto stream = [&](int64_t j, auto& s) {            // s
      constexpr int N = sizeof(s) / sizeof(float);
#pragma unroll
      for (int e = 0; e < N; ++e) s[e] = 0.0f;
      if (a.dh) load_n(static_cast<const T*>(a.dh) + r * a.lddh + j, s);
      if (a.dy) {
        float xh[N], w[N];
        second(j, xh, w);
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] += r2 * (w[e] - s1 - xh[e] * s2);
      }
    };
    const auto first = [&](int64_t j, const auto& s, auto& xh, auto& t) {  // xh1 (or b) and t
      constexpr int N = sizeof(t) / sizeof(float);
      float g[N];
      load_n(b + j, xh);
      if (a.ldg == 0) load_weights<W>(a.gate, j, 1.0f, g);
      else load_n(static_cast<const T*>(a.gate) + r * a.ldg + j, g);
#pragma unroll
      for (int e = 0; e < N; ++e) xh[e] = a.after ? (xh[e] - mu1) * r1 : xh[e], t[e] = s[e] * g[e];
    };
    float m1 = 0.0f, m2 = 0.0f;
    if (a.after && a.db) {
      over_row<VEC>(a.d, [&](int64_t j, auto c) {
        float s[c.n], xh[c.n], t[c.n], g[c.n];
        stream(j, s);
        first(j, s, xh, t);
        load_weights<W>(a.gamma_after, j, 1.0f, g);
#pragma unroll
        for (int e = 0; e < c.n; ++e) m1 += t[e] * g[e], m2 += t[e] * g[e] * xh[e];
      });
      m1 = a.rms ? 0.0f : block_total(m1, red) / d;
      m2 = block_total(m2, red) / d;
    }
    over_row<VEC>(a.d, [&](int64_t j, auto c) {
      float s[c.n], xh[c.n], t[c.n], g[c.n], k[c.n];
      stream(j, s);
      first(j, s, xh, t);
      load_weights<W>(a.gamma_after, j, 1.0f, g);
      load_weights<W>(a.beta_after, j, 0.0f, k);
      if (a.dgate && a.ldg != 0) {
        float v[c.n];
#pragma unroll
        for (int e = 0; e < c.n; ++e) v[e] = s[e] * (a.after ? xh[e] * g[e] + k[e] : xh[e]);
        store_n(static_cast<T*>(a.dgate) + r * a.lddg + j, v);
      }
      if (a.db) {
#pragma unroll
        for (int e = 0; e < c.n; ++e) t[e] = a.after ? r1 * (t[e] * g[e] - m1 - xh[e] * m2) : t[e];
        store_n(static_cast<T*>(a.db) + r * a.lddb + j, t);
      }
      if (a.dres) {
#pragma unroll
        for (int e = 0; e < c.n; ++e) s[e] *= a.rscale;
        store_n(static_cast<T*>(a.dres) + r * a.lddres + j, s);
      }
    });
  }
}

// The gradients of rows in registers in one pass over dy, dh, h and b: workgroup p takes
// rows p, p + gridDim.x, .. (RPB at a time), keeps its threads' columns of the four sums
// in registers, adds its RPB row groups in LDS and writes partial[p]. A row's registers
// take the next one's vectors as soon as they are free: dy, h and dh behind s, whose
// loads are under way during the second half of the row, b and the gate behind db.
template <typename T, typename W, int TPR, int NV, int FORM>
__global__ __launch_bounds__(threads_of(TPR)) void block_back_reg_kernel(BlockBackArgs a) {
  constexpr int VEC = vec_of<T>(), RPB = threads_of(TPR) / TPR;
  __shared__ float red[2][2 * (threads_of(TPR) / 64)];
  __shared__ float joined[RPB > 1 ? TPR * NV * VEC : 1];
  int slot = 0;
  if (threadIdx.x < 2 * (threads_of(TPR) / 64)) red[0][threadIdx.x] = red[1][threadIdx.x] = 0.0f;
  __syncthreads();
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR, d = (int)a.d;
  const int stride = RPB > 1 ? TPR : (int)blockDim.x;
  constexpr bool FULL = FORM != kAny;
  const bool each = FULL ? FORM == kFullGate : a.ldg != 0;
  const auto place = [&](int i) {
    Place<VEC> q((t + i * stride) * VEC, d);
    if (FULL) q.at = (t + i * stride) * VEC, q.skip = 0;
    return q;
  };
  Kept<W, VEC> g1[NV], c1[NV], g0[NV], g2[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = place(i).at;
    g1[i].load_or(a.gamma_after, at, 1.0f);
    c1[i].load_or(each ? a.beta_after : nullptr, at, 0.0f);
    g0[i].load_or(each ? nullptr : a.gate, at, 1.0f);
    g2[i].load_or(a.gamma, at, 1.0f);
  }
  float sum[4][NV][VEC] = {};
  Kept<T, VEC> rb[NV], rh[NV], ry[NV], rs[NV], rg[NV];                 // of b, h, dy, dh, gate
#pragma unroll
  for (int i = 0; i < NV; ++i) rs[i].fill(0.0f);
  float st[4], nst[2];
  const auto fetch = [&](const void* p, int64_t ld, int64_t r, Kept<T, VEC> (&v)[NV]) {
    const T* q = static_cast<const T*>(p) + min(r, a.rows - 1) * ld;
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i].load(q, place(i).at);
  };
  const auto fetch_second = [&](int64_t r) {      // what h's norm takes
    __builtin_memcpy(nst, a.stats + 4 * min(r, a.rows - 1) + 2, 8);
    if (FULL || a.dy) {
      fetch(a.dy, a.lddy, r, ry);
      fetch(a.h, a.ldh, r, rh);
    }
    if (FULL || a.dh) fetch(a.dh, a.lddh, r, rs);
  };
  const auto fetch_first = [&](int64_t r) {       // what b's norm takes
    __builtin_memcpy(st, a.stats + 4 * min(r, a.rows - 1), 8);
    fetch(a.b, a.ldb, r, rb);
    if (each) fetch(a.gate, a.ldg, r, rg);
  };
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t r0 = (int64_t)blockIdx.x * RPB;
  fetch_second(r0 + sub);
  fetch_first(r0 + sub);
  for (; r0 < a.rows; r0 += step) {
    const int64_t r = r0 + sub;
    const bool live = RPB == 1 || r < a.rows;
    float w[NV][VEC], s[NV][VEC];
    st[2] = nst[0], st[3] = nst[1];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      g1[i].pin(), c1[i].pin(), g0[i].pin(), g2[i].pin();
#pragma unroll
      for (int e = 0; e < VEC; ++e) s[i][e] = live ? rs[i][e] : 0.0f;  // (a last round's missing rows add nothing)
      clear(place(i), s[i]);
    }
    if (FULL || a.dy) {
      float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[i][e] = live ? ry[i][e] : 0.0f;
        clear(place(i), w[i]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float xh = (rh[i][e] - st[2]) * st[3];
          sum[2][i][e] += w[i][e] * xh;
          sum[3][i][e] += w[i][e];
          w[i][e] *= g2[i][e];
          s1 += w[i][e];
          s2 += w[i][e] * xh;
        }
      }
      row_totals<float, TPR>(s1, s2, red, slot);
      s1 = a.rms ? 0.0f : s1 / (float)d;
      s2 /= (float)d;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float own = st[3] * (w[i][e] - s1 - (rh[i][e] - st[2]) * st[3] * s2);
          s[i][e] += live ? own : 0.0f;
        }
        clear(place(i), s[i]);
      }
    }
    fetch_second(r + step);                       // past the end: the last row again, unused
    __builtin_amdgcn_sched_barrier(0);
    if ((FULL || a.dres) && live) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[i][e] = a.rscale * s[i][e];
        store_at(static_cast<T*>(a.dres) + r * a.lddres, place(i), w[i]);
      }
    }
    const auto xh1 = [&](int i, int e) { return a.after ? (rb[i][e] - st[0]) * st[1] : rb[i][e]; };
    if ((FULL || a.dgate) && each && live) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[i][e] = s[i][e] * (a.after ? xh1(i, e) * g1[i][e] + c1[i][e] : rb[i][e]);
        store_at(static_cast<T*>(a.dgate) + r * a.lddg, place(i), w[i]);
      }
    }
    float m1 = 0.0f, m2 = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float t1 = s[i][e] * (each ? rg[i][e] : g0[i][e]), q = each ? t1 : s[i][e], xh = xh1(i, e);
        sum[0][i][e] += q * xh;
        sum[1][i][e] += q;
        w[i][e] = a.after ? t1 * g1[i][e] : t1;
        m1 += w[i][e];
        m2 += w[i][e] * xh;
      }
    if (FULL || a.db) {
      if (a.after) {
        row_totals<float, TPR>(m1, m2, red, slot);
        m1 = a.rms ? 0.0f : m1 / (float)d;
        m2 /= (float)d;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < VEC; ++e) w[i][e] = st[1] * (w[i][e] - m1 - xh1(i, e) * m2);
      }
      if (live) {
#pragma unroll
        for (int i = 0; i < NV; ++i) store_at(static_cast<T*>(a.db) + r * a.lddb, place(i), w[i]);
      }
    }
    fetch_first(r + step);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (!a.partial) return;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (RPB > 1) {
      for (int q = RPB - 1; q > 0; --q) {         // row group q adds to what those above it left
        if (sub == q) {
#pragma unroll
          for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              const int at = (i * VEC + e) * TPR + t;
              joined[at] = q == RPB - 1 ? sum[k][i][e] : joined[at] + sum[k][i][e];
            }
        }
        __syncthreads();
      }
      if (sub == 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < VEC; ++e) sum[k][i][e] += joined[(i * VEC + e) * TPR + t];
      }
      __syncthreads();
    }
    if (sub == 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) store_at(a.partial + ((int64_t)blockIdx.x * 4 + k) * a.d, place(i), sum[k][i]);
    }
  }
}

// The four sums of every column over the strip blockIdx.y of rows, a thread per column,
// at the means that block_back_row_kernel left: partial[strip][sum][column].
template <typename T, typename W>
__global__ __launch_bounds__(BT) void block_back_columns_kernel(BlockBackArgs a, int64_t strip) {
  const int64_t j = (int64_t)blockIdx.x * BT + threadIdx.x;
  if (j >= a.d) return;
  const int64_t from = (int64_t)blockIdx.y * strip, to = min(from + strip, a.rows);
  const float g2 = a.gamma ? (float)static_cast<const W*>(a.gamma)[j] : 1.0f;
  float sum[4] = {};
#pragma unroll 4
  for (int64_t r = from; r < to; ++r) {
    const float* st = a.stats + 4 * r;
    float s = a.dh ? (float)static_cast<const T*>(a.dh)[r * a.lddh + j] : 0.0f;
    if (a.dy) {
      const float dy = (float)static_cast<const T*>(a.dy)[r * a.lddy + j];
      const float xh = ((float)static_cast<const T*>(a.h)[r * a.ldh + j] - st[2]) * st[3];
      s += st[3] * (dy * g2 - a.means[2 * r] - xh * a.means[2 * r + 1]);
      sum[2] += dy * xh;
      sum[3] += dy;
    }
    float xh = (float)static_cast<const T*>(a.b)[r * a.ldb + j];
    if (a.after) xh = (xh - st[0]) * st[1];
    if (a.ldg != 0) s *= (float)static_cast<const T*>(a.gate)[r * a.ldg + j];
    sum[0] += s * xh;
    sum[1] += s;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) a.partial[((int64_t)blockIdx.y * 4 + i) * a.d + j] = sum[i];
}

// Adds the partial sums in a fixed order and forms the gradients: 64 columns a
// workgroup at a time, each of its 16 wavefronts every sixteenth part, then the
// sixteen. blockIdx.y: A and B, or the sums of dy xh2 and dy.
template <typename W>
__global__ __launch_bounds__(1024) void block_back_join_kernel(BlockBackArgs a, int64_t parts) {
  __shared__ float red[2][16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const bool vector = a.ldg == 0;
  if (blockIdx.y == 0 ? !((vector && a.dgate) || a.dgamma_after || a.dbeta_after) : !(a.dgamma || a.dbeta)) return;
  for (int64_t j0 = (int64_t)blockIdx.x * 64; j0 < a.d; j0 += (int64_t)gridDim.x * 64) {
    const int64_t j = j0 + lane;
    float u = 0.0f, v = 0.0f;
    if (j < a.d) {
#pragma unroll 4
      for (int64_t p = w; p < parts; p += 16) {
        u += a.partial[(p * 4 + 2 * blockIdx.y) * a.d + j];
        v += a.partial[(p * 4 + 2 * blockIdx.y + 1) * a.d + j];
      }
    }
    red[0][w][lane] = u;
    red[1][w][lane] = v;
    __syncthreads();
    if (w == 0 && j < a.d) {
#pragma unroll
      for (int i = 1; i < 16; ++i) u += red[0][i][lane], v += red[1][i][lane];
      const auto put = [&](void* p, float x) {
        if (p) static_cast<W*>(p)[j] = (W)x;
      };
      const auto weight = [&](const void* p, float none) { return p ? (float)static_cast<const W*>(p)[j] : none; };
      if (blockIdx.y == 1) {
        put(a.dgamma, u);
        put(a.dbeta, v);
      } else {
        const float g = vector ? weight(a.gate, 1.0f) : 1.0f;
        put(a.dgamma_after, g * u);
        put(a.dbeta_after, g * v);
        if (vector) put(a.dgate, a.after ? weight(a.gamma_after, 1.0f) * u + weight(a.beta_after, 0.0f) * v : u);
      }
    }
    __syncthreads();
  }
}

// 16-byte vectors of a row; rows shorter than a vector go with those too long for the
// registers.
int64_t vectors(int xtype, int64_t d) {
  const int vec = xtype == KMP_F32 ? 4 : 8;
  return d < vec ? INT32_MAX : ceil_div(d, vec);
}

// Threads for nv vectors, NV each: no more wavefronts than have any.
int threads_for(int tpr, int NV, int64_t nv) { return tpr <= 64 ? BT : (int)round_up(ceil_div(nv, NV), 64); }

// FORM for a call.
bool fills(int64_t nv, int NV, int64_t d, int vec) { return nv % (64 * NV) == 0 && nv * vec == d; }
int form_of(const BlockArgs& a, bool fills) {
  return !fills || !a.res || !a.h || !a.y || a.bytes ? kAny : a.ldg != 0 ? kFullGate : kFull;
}
int form_of(const BlockBackArgs& a, bool fills) {
  return !fills || !a.dy || !a.dh || !a.db || !a.dres || (a.ldg != 0 && !a.dgate) ? kAny : a.ldg != 0 ? kFullGate : kFull;
}

template <typename T, typename W>
int forward_as(hipStream_t s, const BlockArgs& a) {
  const int64_t nv = vectors(a.xtype, a.d);
  const auto reg = [&](auto tpr, auto each) -> int {
    constexpr int TPR = tpr.n, NV = each.n;
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(a.rows, threads_of(TPR) / TPR), 2048)), threads(threads_for(TPR, NV, nv));
    const int form = form_of(a, fills(nv, NV, a.d, vec_of<T>()));
    if constexpr (TPR > 64) {
      if (form == kFull) hipLaunchKernelGGL((block_reg_kernel<T, W, TPR, NV, kFull>), grid, threads, 0, s, a);
      else if (form == kFullGate) hipLaunchKernelGGL((block_reg_kernel<T, W, TPR, NV, kFullGate>), grid, threads, 0, s, a);
      else hipLaunchKernelGGL((block_reg_kernel<T, W, TPR, NV, kAny>), grid, threads, 0, s, a);
    } else {
      hipLaunchKernelGGL((block_reg_kernel<T, W, TPR, NV, kAny>), grid, threads, 0, s, a);
    }
    KMP_LAUNCH_CHECK();
    return 0;
  };
  if (nv <= 32) return reg(Count<32>(), Count<1>());
  if (nv <= 64) return reg(Count<64>(), Count<1>());
  if (nv <= 128) return reg(Count<64>(), Count<2>());
  if (nv <= 512) return reg(Count<512>(), Count<1>());
  if (nv <= 1024) return reg(Count<512>(), Count<2>());
  if (nv <= 2048) return reg(Count<1024>(), Count<2>());
  hipLaunchKernelGGL((block_row_kernel<T, W>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(BIG), 0, s, a);
  KMP_LAUNCH_CHECK();
  return 0;
}

template <typename T, typename W>
int backward_as(hipStream_t s, const BlockBackArgs& a) {
  const int64_t parts = block_partials(a.xtype, a.rows, a.d), nv = vectors(a.xtype, a.d);
  const bool sums = a.partial != nullptr;
  const auto reg = [&](auto tpr, auto each) {
    constexpr int TPR = tpr.n, NV = each.n;
    const dim3 grid((unsigned)parts), threads(threads_for(TPR, NV, nv));
    const int form = form_of(a, fills(nv, NV, a.d, vec_of<T>()));
    if constexpr (TPR > 64) {
      if (form == kFull) hipLaunchKernelGGL((block_back_reg_kernel<T, W, TPR, NV, kFull>), grid, threads, 0, s, a);
      else if (form == kFullGate) hipLaunchKernelGGL((block_back_reg_kernel<T, W, TPR, NV, kFullGate>), grid, threads, 0, s, a);
      else hipLaunchKernelGGL((block_back_reg_kernel<T, W, TPR, NV, kAny>), grid, threads, 0, s, a);
    } else {
      hipLaunchKernelGGL((block_back_reg_kernel<T, W, TPR, NV, kAny>), grid, threads, 0, s, a);
    }
  };
  if (a.rows > 0) {
    if (nv <= 32) reg(Count<32>(), Count<1>());
    else if (nv <= 64) reg(Count<64>(), Count<1>());
    else if (nv <= 128) reg(Count<64>(), Count<2>());
    else if (nv <= 512) reg(Count<512>(), Count<1>());
    else if (nv <= 1024) reg(Count<512>(), Count<2>());
    else {
      hipLaunchKernelGGL((block_back_row_kernel<T, W>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(BIG), 0, s, a);
      if (sums)
        hipLaunchKernelGGL((block_back_columns_kernel<T, W>), dim3((unsigned)ceil_div(a.d, BT), (unsigned)parts), dim3(BT), 0, s,
                           a, ceil_div(a.rows, parts));
    }
    KMP_LAUNCH_CHECK();
  }
  if (!sums) return 0;
  hipLaunchKernelGGL((block_back_join_kernel<W>), dim3((unsigned)std::min<int64_t>(ceil_div(a.d, 64), 1 << 20), 2), dim3(1024),
                     0, s, a, a.rows > 0 ? parts : 0);
  KMP_LAUNCH_CHECK();
  return 0;
}

}  // namespace

// Workgroups of the backward pass, each with its own column sums: two rounds of rows
// each up to 256 workgroups, at least four beyond, at most 512.
int64_t block_partials(int xtype, int64_t rows, int64_t d) {
  const int64_t nv = ceil_div(d, xtype == KMP_F32 ? 4 : 8);
  const int64_t groups = ceil_div(rows, nv <= 32 ? 8 : nv <= 128 ? 4 : 1);
  return std::max<int64_t>({1, std::min<int64_t>(ceil_div(groups, 2), 256), std::min<int64_t>(ceil_div(groups, 4), 512)});
}

int block_forward(hipStream_t s, const BlockArgs& a) {
  switch (a.xtype * 8 + a.wtype) {
    case KMP_F32 * 8 + KMP_F32: return forward_as<float, float>(s, a);
    case KMP_BF16 * 8 + KMP_BF16: return forward_as<bf16_t, bf16_t>(s, a);
    case KMP_BF16 * 8 + KMP_F32: return forward_as<bf16_t, float>(s, a);
    case KMP_F16 * 8 + KMP_F16: return forward_as<f16_t, f16_t>(s, a);
    default: return forward_as<f16_t, float>(s, a);
  }
}

int block_backward(hipStream_t s, const BlockBackArgs& a) {
  switch (a.xtype * 8 + a.wtype) {
    case KMP_F32 * 8 + KMP_F32: return backward_as<float, float>(s, a);
    case KMP_BF16 * 8 + KMP_BF16: return backward_as<bf16_t, bf16_t>(s, a);
    case KMP_BF16 * 8 + KMP_F32: return backward_as<bf16_t, float>(s, a);
    case KMP_F16 * 8 + KMP_F16: return backward_as<f16_t, f16_t>(s, a);
    default: return backward_as<f16_t, float>(s, a);
  }
}

}  // namespace kmp
