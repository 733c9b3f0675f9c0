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

// N elements of a weight vector (ones or zeros where there is none) from j on.
template <typename W, int N>
__device__ __forceinline__ void load_weights(const void* p, int64_t j, float none, float (&v)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = none;
  if (p) load_n(static_cast<const W*>(p) + j, v);
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
      for (int e = 0; e < N; ++e) v[e] = a.rscale * s[e] + g[e] * v[e];
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

template <typename T, typename W>
int forward_as(hipStream_t s, const BlockArgs& a) {
  hipLaunchKernelGGL((block_row_kernel<T, W>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(BIG), 0, s, a);
  KMP_LAUNCH_CHECK();
  return 0;
}

template <typename T, typename W>
int backward_as(hipStream_t s, const BlockBackArgs& a) {
  const int64_t parts = block_partials(a.xtype, a.rows, a.d);
  const bool sums = a.partial != nullptr;
  if (a.rows > 0) {
    hipLaunchKernelGGL((block_back_row_kernel<T, W>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(BIG), 0, s, a);
    if (sums)
      hipLaunchKernelGGL((block_back_columns_kernel<T, W>), dim3((unsigned)ceil_div(a.d, BT), (unsigned)parts), dim3(BT), 0, s,
                         a, ceil_div(a.rows, parts));
    KMP_LAUNCH_CHECK();
  }
  if (!sums) return 0;
  hipLaunchKernelGGL((block_back_join_kernel<W>), dim3((unsigned)std::min<int64_t>(ceil_div(a.d, 64), 1 << 20), 2), dim3(1024),
                     0, s, a, a.rows > 0 ? parts : 0);
  KMP_LAUNCH_CHECK();
  return 0;
}

}  // namespace

int64_t block_partials(int xtype, int64_t rows, int64_t d) {
  return std::max<int64_t>(1, std::min<int64_t>(ceil_div(rows, 8), 256));
}

bool block_long(int xtype, int64_t d) { return true; }

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
