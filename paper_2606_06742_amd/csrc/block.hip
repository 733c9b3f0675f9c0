// The norms around a model's block, forward (formulas in kmp_block.h).
#include "kmp_block.h"

// No products and sums are joined but those written so: every kernel here gives the same
// bits, whichever outputs a call asks for.
#pragma clang fp contract(off)

namespace kmp {
namespace {

// Rows that fit the registers of TPR threads, NV 16-byte vectors each (longer ones of
// TPR > 64 by as many wavefronts as the row has work for): b and res are read once. The
// weights stay in registers over the rows of a workgroup, and a row's registers take the
// next one's vectors as soon as they are free: b's behind the first norm, res and the
// gate behind h, so that the loads are under way during the sums without registers of
// their own. By HBM: 16384 x 4096 bf16, four arrays, 90 to 100 us (5.4 to 6.0 TB/s), 4096
// x 5120 f16 with a gate per row 53 (3.9); a single row of 4096 3.4, a chain of load, two
// sums, store.
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
  constexpr bool KNOWN = (FORM & kKnown) != 0;
  const bool BYTES = KNOWN ? (FORM & kOther) != 0 : a.bytes;
  const bool each = KNOWN ? (FORM & kGates) != 0 : a.ldg != 0;         // a gate per row
  const auto place = [&](int i) { return Place<VEC>((t + i * stride) * VEC, d); };
  const auto put = [&](auto* p, int i, const auto& v, bool live) {     // a row's vector i
    if (KNOWN) store_n(p + place(i).at, v);
    else if (live) store_at(p, place(i), v);
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
      for (int i = 0; i < NV; ++i) {
        const int skip = place(i).skip;
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum += e < skip ? 0.0f : v[i][e];
      }
      mu = row_total<float, TPR>(sum, red, slot) / (float)d;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i][e] -= mu;
    }
    float q = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int skip = place(i).skip;
#pragma unroll
      for (int e = 0; e < VEC; ++e) q = e < skip ? q : fmaf(v[i][e], v[i][e], q);
    }
    rs = inv_sqrt(row_total<float, TPR>(q, red, slot) / (float)d + a.eps);
  };
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t r0 = (int64_t)blockIdx.x * RPB;
  fetch(a.b, a.ldb, r0 + sub, b);
  if (KNOWN || a.res) fetch(a.res, a.ldr, r0 + sub, s);
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
    }
    fetch(a.b, a.ldb, r0 + sub + step, b);        // past the end: the last row again, unused
    __builtin_amdgcn_sched_barrier(0);
    float mu1 = 0.0f, r1 = 1.0f, mu2 = 0.0f, r2 = 1.0f;
    if (a.after) {
      norm(v, mu1, r1);
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i][e] = fmaf(v[i][e] * r1, g1[i][e], c1[i][e]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[i][e] *= each ? g[i][e] : g0[i][e];
    if (KNOWN || a.res) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i][e] = fmaf(a.rscale, s[i][e], v[i][e]);
      fetch(a.res, a.ldr, r0 + sub + step, s);
    }
    if (each) fetch(a.gate, a.ldg, r0 + sub + step, g);
    __builtin_amdgcn_sched_barrier(0);
    if (KNOWN || a.h) {
#pragma unroll
      for (int i = 0; i < NV; ++i) put(static_cast<T*>(a.h) + r * a.ldh, i, values_of(v[i]).v, live);
    }
    if (KNOWN || a.y) {
      norm(v, mu2, r2);
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i][e] = fmaf(v[i][e] * r2, g2[i][e], c2[i][e]);
      if (BYTES) {
        // (not of what another thread has, too: where h is written over res, that may have
        // been read after that thread's store)
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int skip = place(i).skip;
#pragma unroll
          for (int e = 0; e < VEC; ++e) most = e < skip ? most : larger(most, fabsf(v[i][e]));
        }
        const ByteScale bs(row_most<TPR>(most, fred, fslot));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          int8_t q[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) q[e] = bs(v[i][e]);
          put(static_cast<int8_t*>(a.y) + r * a.ldy, i, q, live);
        }
        if (t == 0 && live) a.scale[r] = bs.scale;
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) put(static_cast<T*>(a.y) + r * a.ldy, i, values_of(v[i]).v, live);
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
        for (int e = 0; e < c.n; ++e) q = fmaf(v[e] - mu1, v[e] - mu1, q);
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
        for (int e = 0; e < N; ++e) v[e] = fmaf((v[e] - mu1) * r1, g[e], c[e]);
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
        for (int e = 0; e < c.n; ++e) q = fmaf(v[e] - mu2, v[e] - mu2, q);
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
      for (int e = 0; e < N; ++e) v[e] = fmaf((v[e] - mu2) * r2, g[e], c[e]);
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

// FORM of a call.
int form_of(const BlockArgs& a) {
  if (!a.res || !a.h || !a.y || a.h == a.res) return kAny;
  return kKnown | kRagged | (a.ldg != 0 ? kGates : 0) | (a.bytes ? kOther : 0);
}

template <typename T, typename W>
int forward_as(hipStream_t s, const BlockArgs& a) {
  const int64_t nv = vectors(a.xtype, a.d);
  const auto reg = [&](auto tpr, auto each) -> int {
    constexpr int TPR = tpr.n, NV = each.n;
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(a.rows, threads_of(TPR) / TPR), 2048)), threads(threads_for(TPR, NV, nv));
    with_form<false>(form_of(a), [&](auto form) {
      hipLaunchKernelGGL((block_reg_kernel<T, W, TPR, NV, form.n>), grid, threads, 0, s, a);
    });
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

}  // namespace

int block_forward(hipStream_t s, const BlockArgs& a) {
  switch (a.xtype * 8 + a.wtype) {
    case KMP_F32 * 8 + KMP_F32: return forward_as<float, float>(s, a);
    case KMP_BF16 * 8 + KMP_BF16: return forward_as<bf16_t, bf16_t>(s, a);
    case KMP_BF16 * 8 + KMP_F32: return forward_as<bf16_t, float>(s, a);
    case KMP_F16 * 8 + KMP_F16: return forward_as<f16_t, f16_t>(s, a);
    default: return forward_as<f16_t, float>(s, a);
  }
}

}  // namespace kmp
