// Log probabilities of tokens under rows of logits x (T x V):
//   m = max_j x_j,  s = sum_j exp(x_j - m),  u = sum_j exp(x_j - m) (x_j - m)
//   log p_j = (x_j - m) - log s,  entropy H = -sum_j p_j log p_j = log s - u / s
// the top values in the order (value descending, index ascending), and the
// gradient of g logp + h H with respect to x:
//   dx_j = g (1[j = token] - p_j) - h p_j (log p_j + H).
// A logit of -inf has p = 0 and no term. A row of nothing but -inf has
// every log p = -inf, H = 0 and gradient 0. A row with NaN or +inf has
// NaN results (its alternatives are still in order: NaN, then +inf, first).
// A negative token stands for none: logp 0 and no g; a token from V on gives
// NaN in logp and in the row's gradient, and reads nothing.
#include "kmp_operators.h"

namespace kmp {
namespace {

constexpr int BT = 256;                // threads of a workgroup
constexpr int CAP = 512;               // candidates in LDS at a time
constexpr int kMaxSegs = 64;           // segments of a row at most
constexpr float kLog2e = 1.44269504088896340736f;

// Differences to the maximum are held at -256, where exp is 0 in 32 bits: a
// logit of -inf then adds 0 to s and to u. The maximum is NaN where any logit
// is, which marks the row (s and u then hold nothing of use).
__device__ __forceinline__ float most(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
__device__ __forceinline__ float held(float d) { return fmaxf(d, -256.0f); }

// m, s and u of a part of a row; of an empty part, or one of nothing but -inf,
// -inf, 0 and 0.
struct Part { float m, s, u; };
__device__ __forceinline__ Part join(const Part& a, const Part& b) {
  Part r;
  r.m = most(a.m, b.m);
  const float da = held(a.m - r.m), db = held(b.m - r.m), fa = exp_of(da), fb = exp_of(db);
  r.s = fa * a.s + fb * b.s;
  r.u = fa * (a.u + da * a.s) + fb * (b.u + db * b.s);
  return r;
}
// (A join rounds differently with its two parts exchanged, so the lanes' results
// differ in their last bits: lane 0's for all, whichever writes something with it.)
__device__ __forceinline__ float first_lane(float v) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}
__device__ __forceinline__ Part wave_join(Part p) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1)
    p = join(p, Part{__shfl_xor(p.m, off, kWave), __shfl_xor(p.s, off, kWave), __shfl_xor(p.u, off, kWave)});
  return Part{first_lane(p.m), first_lane(p.s), first_lane(p.u)};
}
__device__ __forceinline__ Part block_join(Part p, Part* red) {
  p = wave_join(p);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = p;
  __syncthreads();
  Part t = red[0];
#pragma unroll
  for (int i = 1; i < BT / 64; ++i) t = join(t, red[i]);
  return t;
}

// Adds U vectors of N logits to a part: their maximum first, so that one
// rescaling serves all. With TOP, `at` follows the first vector that holds the
// part's maximum (NaN, too): j + i * step for vector i.
template <bool TOP, int U, int N>
__device__ __forceinline__ void absorb(Part& p, const float (&w)[U][N], uint32_t& at, uint32_t j, uint32_t step) {
  float c = p.m, one[U];
  const float(&v)[U * N] = reinterpret_cast<const float(&)[U * N]>(w);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    one[i] = w[i][0];
#pragma unroll
    for (int e = 1; e < N; ++e) one[i] = most(one[i], w[i][e]);
  }
  if constexpr (TOP) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (one[i] > c || (one[i] != one[i] && c == c)) at = j + i * step;
      c = most(c, one[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < U; ++i) c = most(c, one[i]);
  }
  const float dm = held(p.m - c), f = exp_of(dm);
  p.u = f * (p.u + dm * p.s);
  p.s *= f;
  p.m = c;
#pragma unroll
  for (int i = 0; i < U * N; ++i) {
    const float d = held(v[i] - c), e = exp_of(d);
    p.s += e;
    p.u += e * d;
  }
}

// Order of the alternatives as one unsigned number: the value's bits mapped to
// increasing order (NaN highest, -0 as 0) above the complemented index. No
// value has key 0.
typedef unsigned long long key_t;
__device__ __forceinline__ uint32_t value_key(float v) {
  if (v != v) return 0xFFFFFFFFu;
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return k == 0xFFFFFFFFu ? __builtin_nanf("") : __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ key_t key_of(float v, uint32_t index) { return (key_t)value_key(v) << 32 | (uint32_t)~index; }

struct TopShared {
  key_t groups[64];
  key_t list[CAP], few[CAP];
  key_t bound;
  int count, flagged;
  uint8_t flag[BT];
};

// The k-th largest of the 64 groups' maxima, a group being four neighbouring
// threads, or 0 where fewer than k <= 64 groups have a key. Every lane counts the
// larger ones of one group's; all wavefronts do the same. Starts and ends with a
// barrier.
__device__ __forceinline__ key_t kth_of_groups(TopShared& sh, int k, key_t mine) {
  mine = max(mine, (key_t)__shfl_xor(mine, 1, kWave));
  mine = max(mine, (key_t)__shfl_xor(mine, 2, kWave));
  __syncthreads();
  if ((threadIdx.x & 3) == 0) sh.groups[threadIdx.x >> 2] = mine;
  if (threadIdx.x == 0) sh.bound = 0;
  __syncthreads();
  const key_t own = sh.groups[threadIdx.x & 63];
  int larger = 0;
#pragma unroll
  for (int j = 0; j < 64; ++j) larger += sh.groups[j] > own;
  if (threadIdx.x < 64 && own != 0 && larger == k - 1) sh.bound = own;
  __syncthreads();
  return sh.bound;
}

// Writes the k largest of the n <= CAP different keys in sh.list in order, through
// put(rank, key): every key's place is the number of larger ones. A long list is
// cut first, by the k-th of its groups' maxima.
template <typename Put>
__device__ __forceinline__ void place_top(TopShared& sh, int k, int n, Put put) {
  const int t = threadIdx.x;
  const key_t* list = sh.list;
  if (n > 96) {
    const key_t bound = kth_of_groups(sh, k, max(t < n ? sh.list[t] : (key_t)0, t + BT < n ? sh.list[t + BT] : (key_t)0));
    if (t == 0) sh.count = 0;
    __syncthreads();
    for (int i = t; i < n; i += BT)
      if (sh.list[i] >= bound) sh.few[atomicAdd(&sh.count, 1)] = sh.list[i];
    __syncthreads();
    n = sh.count;
    list = sh.few;
  }
  for (int i = t; i < n; i += BT) {
    const key_t key = list[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) rank += list[j] > key;
    if (rank < k) put(rank, key);
  }
}

// The k largest of the keys that the threads hold: thread t's are visited by
// visit(t, i) for i < per, each a call add(key); its largest lies in [lower,
// upper] (0: it has none; different threads' lowers differ). The largest keys of
// any k groups are k different ones, so the k-th largest lower bounds the k-th
// largest key from below, and only threads whose upper reaches it (24 on average
// for k = 20) need a second look: their visits are spread over the workgroup.
// More candidates than the list holds (the best ones all with one thread, say)
// raise the bound by those that were kept, in the same way, and the visits are
// repeated: as the keys all differ, the bound grows every time. Writes the keys
// in order through put(rank, key), 0 for ranks past the last key.
template <typename Visit, typename Put>
__device__ __forceinline__ void select_top(TopShared& sh, int k, key_t lower, key_t upper, int per, Visit visit, Put put) {
  const int t = threadIdx.x;
  key_t bound = kth_of_groups(sh, k, lower);
  if (t < k) put(t, (key_t)0);
  if (t == 0) sh.flagged = sh.count = 0;
  __syncthreads();
  if (lower != 0 && upper >= bound) sh.flag[atomicAdd(&sh.flagged, 1)] = (uint8_t)t;
  __syncthreads();
  const int flagged = sh.flagged, items = flagged * per;
  int n;
  for (;;) {
    for (int i = t; i < items; i += BT)
      visit((int)sh.flag[i % flagged], i / flagged, [&](key_t key) {
        if (key < bound) return;
        const int at = atomicAdd(&sh.count, 1);
        if (at < CAP) sh.list[at] = key;
      });
    __syncthreads();
    n = sh.count;
    if (n <= CAP) break;
    bound = kth_of_groups(sh, k, max(sh.list[t], sh.list[t + BT]));
    if (t == 0) sh.count = 0;
    __syncthreads();
  }
  place_top(sh, k, n, put);
}

__device__ __forceinline__ int64_t token_at(const void* tokens, bool wide, int64_t t) {
  return wide ? static_cast<const int64_t*>(tokens)[t] : static_cast<const int32_t*>(tokens)[t];
}

// A row's results from m, s, u: log p_j = (x_j - m) - log s, which keeps its
// digits at any size of m (masks of the type's lowest value).
struct Row { float m, logs; };
template <typename T>
__device__ __forceinline__ Row finish_row(const LogprobArgs& a, int64_t t, const Part& p) {
  // a NaN or +inf: NaN; nothing but -inf: -inf
  const bool nan = p.m != p.m || p.m == INFINITY, none = p.m == -INFINITY;
  const float x = nan ? __builtin_nanf("") : -INFINITY;
  const Row r{nan || none ? x : p.m, nan || none ? x : logf(p.s)};
  if (threadIdx.x == 0) {
    if (a.stats) {
      a.stats[2 * t] = r.m;
      a.stats[2 * t + 1] = r.logs;
    }
    if (a.entropy) a.entropy[t] = nan ? x : none ? 0.0f : fmaxf(r.logs - p.u / p.s, 0.0f);
    if (a.logp) {
      const int64_t id = token_at(a.tokens, a.wide, t);
      float v = 0.0f;
      if (id >= a.V) v = __builtin_nanf("");
      else if (id >= 0)
        v = none ? -INFINITY : ((float)static_cast<const T*>(a.logits)[t * a.ld + id] - r.m) - r.logs;
      a.logp[t] = v;
    }
  }
  return r;
}
__device__ __forceinline__ void put_top(const LogprobArgs& a, int64_t t, const Row& row, int rank, key_t key) {
  if (a.top_id) a.top_id[t * a.top + rank] = (int32_t)~(uint32_t)key;
  if (a.top_logp)
    a.top_logp[t * a.top + rank] =
        row.m == -INFINITY ? -INFINITY : (key_value((uint32_t)(key >> 32)) - row.m) - row.logs;
}

// Partial results of segment g of row t, in the workspace: the parts, then the
// keys of the segment's k best.
__device__ __forceinline__ Part* parts_of(const LogprobArgs& a) { return static_cast<Part*>(a.workspace); }
__device__ __forceinline__ key_t* keys_of(const LogprobArgs& a, int segs) {
  return reinterpret_cast<key_t*>(static_cast<char*>(a.workspace) + round_up(a.T * segs * (int64_t)sizeof(Part), 16));
}

// The lowest finite value, which masks are often made of.
template <typename T> __device__ constexpr float lowest();
template <> __device__ constexpr float lowest<float>() { return -0x1.fffffep127f; }
template <> __device__ constexpr float lowest<bf16_t>() { return -0x1.fep127f; }
template <> __device__ constexpr float lowest<f16_t>() { return -65504.0f; }

// One workgroup per segment of a row (gridDim.x of them, span elements each): one
// pass of 16-byte loads, U in flight, every thread with its own maximum and sums;
// with TOP a second look at the few threads that can hold the alternatives. With
// one segment the row is finished here.
template <typename T, bool TOP>
__global__ __launch_bounds__(BT, 8) void logprob_span_kernel(LogprobArgs a, int64_t span) {
  constexpr int VEC = vec_of<T>(), U = 16 / VEC;
  constexpr uint32_t STEP = BT * VEC;
  __shared__ Part red[BT / 64];
  __shared__ TopShared sh;
  const int segs = gridDim.x;
  for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y) {
    const int64_t unit = t * segs + blockIdx.x, e0 = blockIdx.x * span;
    const uint32_t len = (uint32_t)min(span, a.V - e0);
    const T* x = static_cast<const T*>(a.logits) + t * a.ld + e0;
    const auto load = [&](uint32_t j, float (&v)[VEC]) {   // -inf past the end
      if (j + VEC <= len) {
        load_n(x + j, v);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = j + e < len ? (float)x[j + e] : -INFINITY;
      }
    };
    Part p{-INFINITY, 0.0f, 0.0f};
    uint32_t j = threadIdx.x * VEC, at = j;       // (a first vector of nothing but -inf is at j)
    for (; j + (U - 1) * STEP + VEC <= len; j += U * STEP) {
      float v[U][VEC];
#pragma unroll
      for (int i = 0; i < U; ++i) load_n(x + j + i * STEP, v[i]);
      absorb<TOP>(p, v, at, j, STEP);
    }
    for (; j < len; j += STEP) {
      float v[1][VEC];
      load(j, v[0]);
      absorb<TOP>(p, v, at, j, STEP);
    }
    const float own = p.m;
    p = block_join(p, red);
    Row row{0.0f, 0.0f};
    if (segs == 1)
      row = finish_row<T>(a, t, p);
    else if (threadIdx.x == 0)
      parts_of(a)[unit] = p;
    if constexpr (TOP) {
      const auto put = [&](int rank, key_t key) {
        if (segs > 1) keys_of(a, segs)[unit * a.top + rank] = key;
        else if (key != 0) put_top(a, t, row, rank, key);
      };
      // a segment of masked tokens only (-inf, or the type's lowest value: s then
      // counts them): the first ones
      const uint32_t few = min((uint32_t)a.top, len);
      if (p.m == -INFINITY || (p.m == lowest<T>() && p.s == (float)len && len < 1u << 24)) {
        if (threadIdx.x < a.top)
          put(threadIdx.x, threadIdx.x < few ? key_of(p.m, (uint32_t)e0 + threadIdx.x) : (key_t)0);
        continue;
      }
      // this thread's best key lies between these two: its vector is known, not
      // the place in it
      const bool any = threadIdx.x * VEC < len;
      const key_t lower = any ? key_of(own, (uint32_t)e0 + at + (VEC - 1)) : 0, upper = any ? key_of(own, (uint32_t)e0 + at) : 0;
      select_top(
          sh, a.top, lower, upper, (int)((len + STEP - 1) / STEP),
          [&](int owner, int i, auto add) {
            const uint32_t at = i * STEP + owner * VEC;
            if (at >= len) return;
            float v[VEC];
            load(at, v);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
              if (at + e < len) add(key_of(v[e], (uint32_t)e0 + at + e));
          },
          put);
    }
  }
}

// Joins the segments of one row per workgroup.
template <typename T>
__global__ __launch_bounds__(BT) void logprob_join_kernel(LogprobArgs a, int segs) {
  __shared__ TopShared sh;
  const int lane = threadIdx.x & 63;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    // every wavefront joins all parts (at most 64 of them) for itself
    const Part none{-INFINITY, 0.0f, 0.0f};
    const Row row = finish_row<T>(a, t, wave_join(lane < segs ? parts_of(a)[t * segs + lane] : none));
    if (a.top > 0) {
      const key_t* keys = keys_of(a, segs) + t * segs * a.top;
      const int n = segs * a.top;
      const auto put = [&](int rank, key_t key) {
        if (key != 0) put_top(a, t, row, rank, key);
      };
      if (n <= CAP) {                             // (empty places: 0, the last ones)
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += BT) sh.list[i] = keys[i] != 0 ? keys[i] : (key_t)i;
        __syncthreads();
        place_top(sh, a.top, n, put);
        continue;
      }
      key_t mine = 0;
      for (int i = threadIdx.x; i < n; i += BT) mine = max(mine, keys[i]);
      select_top(
          sh, a.top, mine, mine, (n + BT - 1) / BT,
          [&](int owner, int i, auto add) {
            const int at = i * BT + owner;
            if (at < n && keys[at] != 0) add(keys[at]);
          },
          put);
    }
  }
}

// The gradient, one workgroup per 4 vectors of its threads: reads a logit,
// writes its gradient, an exponential between. The last rows come first: the
// forward call read them last, so that the last-level cache still has them.
template <typename T>
__global__ __launch_bounds__(BT) void logprob_back_kernel(LogprobBackArgs a) {
  constexpr int VEC = vec_of<T>(), U = 4, FULL = U * BT * VEC;
  const int64_t t = a.T - 1 - ((int64_t)blockIdx.z * gridDim.y + blockIdx.y);
  if (t < 0) return;
  const int64_t base = (int64_t)blockIdx.x * FULL;
  const int left = (int)min(a.V - base, (int64_t)FULL);
  const T* x = static_cast<const T*>(a.logits) + t * a.ld + base;
  T* dx = static_cast<T*>(a.dlogits) + t * a.ldd + base;
  float v[U][VEC];
  if (left == FULL) {
#pragma unroll
    for (int i = 0; i < U; ++i) load_n(x + (threadIdx.x + i * BT) * VEC, v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int j = (threadIdx.x + i * BT) * VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[i][e] = j + e < left ? (float)x[j + e] : 0.0f;
    }
  }
  const float m = a.stats[2 * t], logs = a.stats[2 * t + 1];
  const float h = a.dentropy ? a.dentropy[t] : 0.0f, H = a.dentropy ? a.entropy[t] : 0.0f;
  const int64_t id = a.dlogp ? token_at(a.tokens, a.wide, t) : -1;
  float g = id >= 0 ? a.dlogp[t] : 0.0f;
  if (id >= a.V || logs != logs) g = __builtin_nanf("");
  // the token's place in this chunk, if it is there
  const int at = m > -INFINITY && id >= base && id - base < left ? (int)(id - base) : -1;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int j = (threadIdx.x + i * BT) * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float lp = held((v[i][e] - m) - logs);         // -inf: p = 0, no term
      v[i][e] = -exp_of(lp) * (g + h * (lp + H));
    }
    if (at >= j && at < j + VEC) {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (j + e == at) v[i][e] += g;
    }
    if (left == FULL) {
      store_n(dx + j, v[i]);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (j + e < left) dx[j + e] = (T)v[i][e];
    }
  }
}

// Segments of a row: as many as make four workgroups a compute unit, of at least
// 4096 elements (8192: 2 x 32000 with 20 alternatives 12.1 -> 11.7 us, 1 x 128000
// 12.9 -> 13.5). One for rows of up to 64 KB, whose pass costs less than the join
// (16 x 20000 in 16 bits 11.1 / 7.9 us, with 20 alternatives 13.1 / 10.6), and in
// place of two or three for rows of up to 65536: 333 x 40009 in 32 bits 14.5 / 12.1,
// 512 x 50001 26.9 / 25.8, but 300 x 128000 in 16 bits 19.4 / 23.5, 500 x 128000
// 38.5 / 51.7.
struct Split { int segs; int64_t span; };
Split split(int64_t T, int64_t V, int size) {
  const int64_t segs = std::min<int64_t>({1024 / std::max<int64_t>(T, 1), ceil_div(V, 4096), kMaxSegs});
  if (segs <= 1 || V * size <= 65536 || (segs <= 3 && V <= 65536)) return {1, V};
  const int64_t span = round_up(ceil_div(V, segs), 1024);
  return {(int)ceil_div(V, span), span};
}

template <typename T>
int forward_as(hipStream_t s, const LogprobArgs& a) {
  const auto [segs, span] = split(a.T, a.V, (int)sizeof(T));
  const dim3 grid(segs, (unsigned)std::min<int64_t>(a.T, 65535));
  if (a.top > 0)
    hipLaunchKernelGGL((logprob_span_kernel<T, true>), grid, dim3(BT), 0, s, a, span);
  else
    hipLaunchKernelGGL((logprob_span_kernel<T, false>), grid, dim3(BT), 0, s, a, span);
  KMP_LAUNCH_CHECK();
  if (segs > 1) {
    hipLaunchKernelGGL(logprob_join_kernel<T>, dim3((unsigned)a.T), dim3(BT), 0, s, a, segs);
    KMP_LAUNCH_CHECK();
  }
  return 0;
}
template <typename T>
int backward_as(hipStream_t s, const LogprobBackArgs& a) {
  const int64_t rows = std::min<int64_t>(a.T, 65535);
  hipLaunchKernelGGL(logprob_back_kernel<T>,
                     dim3((unsigned)ceil_div(a.V, 4 * BT * vec_of<T>()), (unsigned)rows, (unsigned)ceil_div(a.T, rows)),
                     dim3(BT), 0, s, a);
  KMP_LAUNCH_CHECK();
  return 0;
}

}  // namespace

// A bound on what split() takes at T, V (of 32-bit logits, which are split the most)
// that never falls as T, V or top grows, so that the workspace of a program's largest
// call serves its smaller ones: T * segs is at most 1024 and T times the segments of a
// single row. 256 bytes where there is nothing to keep, so that 0 means an error.
size_t logprob_workspace(int64_t T, int64_t V, int top) {
  if (V * 4 <= 65536) return 256;
  const int64_t units = std::min<int64_t>(T * std::min<int64_t>(ceil_div(V, 4096), kMaxSegs), 1024);
  return std::max<size_t>(256, round_up(units * (int64_t)sizeof(Part), 16) + units * top * (int64_t)sizeof(key_t));
}

int token_logprobs(hipStream_t s, const LogprobArgs& a) {
  switch (a.type) {
    case KMP_F32: return forward_as<float>(s, a);
    case KMP_BF16: return forward_as<bf16_t>(s, a);
    default: return forward_as<f16_t>(s, a);
  }
}

int token_logprobs_backward(hipStream_t s, const LogprobBackArgs& a) {
  switch (a.type) {
    case KMP_F32: return backward_as<float>(s, a);
    case KMP_BF16: return backward_as<bf16_t>(s, a);
    default: return backward_as<f16_t>(s, a);
  }
}

}  // namespace kmp
