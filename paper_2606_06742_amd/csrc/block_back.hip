// The gradients of the norms around a model's block (formulas in kmp_block.h).
#include "kmp_block.h"

// No products and sums are joined but those written so: every kernel here gives the same
// bits, whichever outputs a call asks for.
#pragma clang fp contract(off)

namespace kmp {
namespace {

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
        for (int e = 0; e < c.n; ++e) s1 += w[e], s2 = fmaf(w[e], xh[e], s2);
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
        for (int e = 0; e < N; ++e) s[e] = fmaf(r2, fmaf(-xh[e], s2, w[e] - s1), s[e]);
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
        for (int e = 0; e < c.n; ++e) m1 += t[e] * g[e], m2 = fmaf(t[e] * g[e], xh[e], m2);
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
        for (int e = 0; e < c.n; ++e) v[e] = s[e] * (a.after ? fmaf(xh[e], g[e], k[e]) : xh[e]);
        store_n(static_cast<T*>(a.dgate) + r * a.lddg + j, v);
      }
      if (a.db) {
#pragma unroll
        for (int e = 0; e < c.n; ++e) t[e] = a.after ? r1 * fmaf(-xh[e], m2, t[e] * g[e] - m1) : t[e];
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
// loads are under way during the second half of the row, b and the gate behind db. By
// HBM: 16384 x 4096 bf16, six arrays, 184 to 205 us (3.9 to 4.4 TB/s), at two wavefronts a
// SIMD: its sums and rows fill the registers, and to force more of them in spilled and was
// slower.
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
  constexpr bool KNOWN = (FORM & kKnown) != 0, WHOLE = KNOWN && !(FORM & kRagged);
  const bool has_dh = KNOWN ? !(FORM & kOther) : a.dh != nullptr;
  const bool each = KNOWN ? (FORM & kGates) != 0 : a.ldg != 0;         // a gate per row
  const auto place = [&](int i) {
    Place<VEC> q((t + i * stride) * VEC, d);
    if (WHOLE) q.at = (t + i * stride) * VEC, q.skip = 0;
    return q;
  };
  const auto put = [&](auto* p, int i, const auto& v, bool live) {     // a row's vector i
    if (KNOWN) store_n(p + place(i).at, v);
    else if (live) store_at(p, place(i), v);
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
    if (KNOWN || a.dy) {
      fetch(a.dy, a.lddy, r, ry);
      fetch(a.h, a.ldh, r, rh);
    }
    if (has_dh) fetch(a.dh, a.lddh, r, rs);
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
    const int64_t at = live ? r : a.rows - 1;
    float w[NV][VEC], s[NV][VEC];
    st[2] = nst[0], st[3] = nst[1];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      g1[i].pin(), c1[i].pin(), g0[i].pin(), g2[i].pin();
#pragma unroll
      for (int e = 0; e < VEC; ++e) s[i][e] = has_dh ? rs[i][e] : 0.0f;
    }
    if (KNOWN || a.dy) {
      float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int skip = place(i).skip;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float xh = (rh[i][e] - st[2]) * st[3], dy = ry[i][e];
          sum[2][i][e] = live ? fmaf(dy, xh, sum[2][i][e]) : sum[2][i][e];      // (rows past the last one add nothing)
          sum[3][i][e] += live ? dy : 0.0f;
          w[i][e] = dy * g2[i][e];
          s1 += e < skip ? 0.0f : w[i][e];
          s2 = e < skip ? s2 : fmaf(w[i][e], xh, s2);
        }
      }
      row_totals<float, TPR>(s1, s2, red, slot);
      s1 = a.rms ? 0.0f : s1 / (float)d;
      s2 /= (float)d;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[i][e] = fmaf(st[3], fmaf(-((rh[i][e] - st[2]) * st[3]), s2, w[i][e] - s1), s[i][e]);
    }
    fetch_second(r + step);                       // past the end: the last row again, unused
    __builtin_amdgcn_sched_barrier(0);
    if (KNOWN || a.dres) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[i][e] = a.rscale * s[i][e];
        put(static_cast<T*>(a.dres) + at * a.lddres, i, values_of(w[i]).v, live);
      }
    }
    const auto xh1 = [&](int i, int e) { return a.after ? (rb[i][e] - st[0]) * st[1] : rb[i][e]; };
    if ((KNOWN || a.dgate) && each) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[i][e] = s[i][e] * (a.after ? fmaf(xh1(i, e), g1[i][e], c1[i][e]) : rb[i][e]);
        put(static_cast<T*>(a.dgate) + at * a.lddg, i, values_of(w[i]).v, live);
      }
    }
    float m1 = 0.0f, m2 = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int skip = place(i).skip;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float t1 = s[i][e] * (each ? rg[i][e] : g0[i][e]), q = each ? t1 : s[i][e], xh = xh1(i, e);
        sum[0][i][e] = live ? fmaf(q, xh, sum[0][i][e]) : sum[0][i][e];
        sum[1][i][e] += live ? q : 0.0f;
        w[i][e] = a.after ? t1 * g1[i][e] : t1;
        m1 += e < skip ? 0.0f : w[i][e];
        m2 = e < skip ? m2 : fmaf(w[i][e], xh, m2);
      }
    }
    if (KNOWN || a.db) {
      if (a.after) {
        row_totals<float, TPR>(m1, m2, red, slot);
        m1 = a.rms ? 0.0f : m1 / (float)d;
        m2 /= (float)d;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < VEC; ++e) w[i][e] = st[1] * fmaf(-xh1(i, e), m2, w[i][e] - m1);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) put(static_cast<T*>(a.db) + at * a.lddb, i, values_of(w[i]).v, live);
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

// The four sums of every column over the strip blockIdx.y of rows, a vector of columns
// a thread, at the means that block_back_row_kernel left: partial[strip][sum][column].
template <typename T, typename W>
__global__ __launch_bounds__(BT) void block_back_columns_kernel(BlockBackArgs a, int64_t strip) {
  constexpr int VEC = vec_of<T>();
  const int64_t j = ((int64_t)blockIdx.x * BT + threadIdx.x) * VEC;
  if (j >= a.d) return;
  const int64_t from = (int64_t)blockIdx.y * strip, to = min(from + strip, a.rows);
  const auto columns = [&](auto count, int64_t j) {
    constexpr int N = count.n;
    float g2[N], sum[4][N] = {};
    load_weights<W>(a.gamma, j, 1.0f, g2);
#pragma unroll 2
    for (int64_t r = from; r < to; ++r) {
      const float* st = a.stats + 4 * r;
      float s[N], xh[N];
#pragma unroll
      for (int e = 0; e < N; ++e) s[e] = 0.0f;
      if (a.dh) load_n(static_cast<const T*>(a.dh) + r * a.lddh + j, s);
      if (a.dy) {
        float dy[N];
        load_n(static_cast<const T*>(a.dy) + r * a.lddy + j, dy);
        load_n(static_cast<const T*>(a.h) + r * a.ldh + j, xh);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float x = (xh[e] - st[2]) * st[3];
          s[e] = fmaf(st[3], fmaf(-x, a.means[2 * r + 1], dy[e] * g2[e] - a.means[2 * r]), s[e]);
          sum[2][e] = fmaf(dy[e], x, sum[2][e]);
          sum[3][e] += dy[e];
        }
      }
      load_n(static_cast<const T*>(a.b) + r * a.ldb + j, xh);
      if (a.ldg != 0) {
        float g[N];
        load_n(static_cast<const T*>(a.gate) + r * a.ldg + j, g);
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] *= g[e];
      }
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float x = a.after ? (xh[e] - st[0]) * st[1] : xh[e];
        sum[0][e] = fmaf(s[e], x, sum[0][e]);
        sum[1][e] += s[e];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) store_n(a.partial + ((int64_t)blockIdx.y * 4 + i) * a.d + j, sum[i]);
  };
  if (j + VEC <= a.d) columns(Count<VEC>(), j);
  else
    for (int64_t c = j; c < a.d; ++c) columns(Count<1>(), c);
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

// FORM of a call. Whole rows have forms of their own in longer rows (8192 x 8192 in 16
// bits 203 / 221 us, 4096 x 5120 with a gate per row 135 / 162; no difference in the
// others, nor in the forward pass).
int form_of(const BlockBackArgs& a, bool whole) {
  if (!a.dy || !a.db || !a.dres || (a.ldg != 0 && !a.dgate)) return kAny;
  return kKnown | (a.ldg != 0 ? kGates : 0) | (whole ? 0 : kRagged) | (a.dh ? 0 : kOther);
}

template <typename T, typename W>
int backward_as(hipStream_t s, const BlockBackArgs& a) {
  const int64_t parts = block_partials(a.xtype, a.rows, a.d), nv = vectors(a.xtype, a.d);
  const bool sums = a.partial != nullptr;
  const auto reg = [&](auto tpr, auto each) {
    constexpr int TPR = tpr.n, NV = each.n;
    const dim3 grid((unsigned)parts), threads(threads_for(TPR, NV, nv));
    const bool whole = TPR > 64 && nv % (64 * NV) == 0 && nv * vec_of<T>() == a.d;
    with_form<(TPR > 64)>(form_of(a, whole), [&](auto form) {
      hipLaunchKernelGGL((block_back_reg_kernel<T, W, TPR, NV, form.n>), grid, threads, 0, s, a);
    });
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
        hipLaunchKernelGGL((block_back_columns_kernel<T, W>), dim3((unsigned)ceil_div(a.d, BT * vec_of<T>()), (unsigned)parts),
                           dim3(BT), 0, s, a, ceil_div(a.rows, parts));
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
