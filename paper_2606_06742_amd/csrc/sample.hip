// Tokens drawn from rows of logits x with given random numbers u:
//   w_j = exp((x_j - m) / temperature),  m = max_j x_j
// in the order (value descending, index ascending) the first k tokens are kept, of
// these the shortest run whose weight reaches p times theirs, of these the tokens with
// w >= min_p; the drawn one is the first kept one, by index, at which the running sum
// of the kept weights exceeds u times their total Z.
// All three rules keep a run of the order from its start, so that one 64-bit key (the
// value's bits above the complemented index) separates what they keep. A token hangs on
// comparisons of sums over the vocabulary, whose neighbours differ by one weight (1e-6
// of the sum and less): weights and sums are in 64 bits, where a wrong side is a matter
// of 1e-10, and every sum has a fixed order, or is one of whole numbers.
#include "kmp_keys.h"

namespace kmp {
namespace {

constexpr int NT = 1024, NW = NT / 64; // threads and wavefronts of a workgroup
constexpr int BINS = 256, COLS = 32;   // bins of a histogram, columns of each

struct Shared {
  union {
    struct {                           // two lanes share a column, on a bank of their own
      unsigned long long sum[BINS][COLS];
      uint32_t count[BINS][COLS];
    } h;
    key_t list[NT];
  };
  double red[NW];
  double bin_sum[BINS];
  uint32_t bin_count[BINS];
  key_t top[NW];
  int first[NW];
  int n;
};

// f(j, x_j) for the row's elements [from, to): wavefront w takes the w-th of sixteen
// neighbouring runs, in vectors of 16 bytes.
template <typename T>
__device__ __forceinline__ int64_t run_length(int64_t n) {
  constexpr int64_t STEP = 64 * vec_of<T>();
  return round_up(ceil_div(n, NW), STEP);
}
template <typename T, typename F>
__device__ __forceinline__ void visit(const T* x, int64_t from, int64_t to, F f) {
  constexpr int VEC = vec_of<T>();
  const int64_t run = run_length<T>(to - from), start = from + (threadIdx.x >> 6) * run, end = min(to, start + run);
  int64_t j = start + (threadIdx.x & 63) * VEC;
#pragma unroll 2
  for (; j + VEC <= end; j += 64 * VEC) {
    float v[VEC];
    load_n(x + j, v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) f(j + e, v[e]);
  }
  for (; j < end; ++j) f(j, (float)x[j]);         // (the run's last vector, of one lane)
}

// The block's largest key, its sum, its running sum; each starts with a barrier.
__device__ __forceinline__ key_t block_top(Shared& sh, key_t v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = max(v, (key_t)__shfl_xor(v, off, kWave));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.top[threadIdx.x >> 6] = v;
  __syncthreads();
  v = sh.top[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) v = max(v, sh.top[i]);
  return v;
}
__device__ __forceinline__ double wave_running(double v) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double up = __shfl_up(v, off, kWave);
    if ((int)(threadIdx.x & 63) >= off) v += up;
  }
  return v;
}
__device__ __forceinline__ double block_running(Shared& sh, double v, double& total) {
  v = wave_running(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) sh.red[threadIdx.x >> 6] = v;
  __syncthreads();
  double before = 0.0;
  total = 0.0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    if (i == (int)(threadIdx.x >> 6)) before = total;
    total += sh.red[i];
  }
  return before + v;
}
// The first thread with `is`, NT where there is none; the last one, -1.
__device__ __forceinline__ int block_first(Shared& sh, bool is) {
  const unsigned long long b = __ballot(is);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.first[threadIdx.x >> 6] = b ? (int)(threadIdx.x & ~63) + __ffsll(b) - 1 : NT;
  __syncthreads();
  int at = NT;
#pragma unroll
  for (int i = 0; i < NW; ++i) at = min(at, sh.first[i]);
  return at;
}
__device__ __forceinline__ int block_last(Shared& sh, bool is) {
  const unsigned long long b = __ballot(is);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.first[threadIdx.x >> 6] = b ? (int)(threadIdx.x & ~63) + 63 - __clzll(b) : -1;
  __syncthreads();
  int at = -1;
#pragma unroll
  for (int i = 0; i < NW; ++i) at = max(at, sh.first[i]);
  return at;
}

// The threads' keys in descending order (bitonic merges; within a wavefront by
// shuffles).
__device__ __forceinline__ key_t sorted(Shared& sh, key_t mine) {
  const int t = threadIdx.x;
  for (int k = 2; k <= NT; k <<= 1) {
    for (int s = k >> 1; s > 0; s >>= 1) {
      key_t other;
      if (s >= 64) {
        __syncthreads();
        sh.list[t] = mine;
        __syncthreads();
        other = sh.list[t ^ s];
      } else {
        other = __shfl_xor(mine, s, kWave);
      }
      mine = ((t & k) == 0) == ((t & s) == 0) ? max(mine, other) : min(mine, other);
    }
  }
  __syncthreads();
  return mine;
}

// One row's drawing.
template <typename T>
struct Row {
  Shared& sh;
  const T* x;
  int64_t V;
  float m;                             // its maximum
  double it;                           // 1 / temperature
  double min_p;                        // 0: none

  __device__ double weight(float v) const { return v == -INFINITY ? 0.0 : exp(((double)v - (double)m) * it); }

  // The keys for which is(key, x) holds, at most NT of them, one a thread, in
  // descending order (0: none).
  template <typename F>
  __device__ key_t gather(F is) {
    __syncthreads();
    sh.list[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    visit(x, 0, V, [&](int64_t j, float v) {
      const key_t key = key_of(v, (uint32_t)j);
      if (!is(key, v)) return;
      const int at = atomicAdd(&sh.n, 1);
      if (at < NT) sh.list[at] = key;
    });
    __syncthreads();
    return sorted(sh, sh.list[threadIdx.x]);
  }

  // Sums a histogram's columns: thread b < BINS has bin b's.
  __device__ void clear_bins() {
    __syncthreads();
    for (int i = threadIdx.x; i < BINS * COLS; i += NT) (&sh.h.sum[0][0])[i] = 0, (&sh.h.count[0][0])[i] = 0;
    __syncthreads();
  }
  __device__ void add(int bin, unsigned long long w) {
    const int c = threadIdx.x & (COLS - 1);
    atomicAdd(&sh.h.sum[bin][c], w);
    atomicAdd(&sh.h.count[bin][c], 1u);
  }
  __device__ void read_bins(unsigned long long& w, uint32_t& n) {
    __syncthreads();
    w = 0, n = 0;
    if (threadIdx.x < BINS)
      for (int c = 0; c < COLS; ++c) {            // (staggered over the banks)
        const int at = (c + threadIdx.x) & (COLS - 1);
        w += sh.h.sum[threadIdx.x][at];
        n += sh.h.count[threadIdx.x][at];
      }
    __syncthreads();
  }

  // The range of keys [lo, hi], with `above` counted or weighed before it, is narrowed
  // to where f(before, own) first holds for a bin of 1/256 of it, until it has at most
  // NT keys of those for which is(key, x) holds. WEIGHED: by weights w = scaled(x),
  // at most 1, in steps of 2^-q, else by their number.
  template <bool WEIGHED, typename Is, typename Scaled, typename Reach>
  __device__ void narrow(key_t& lo, key_t& hi, double& above, double unit, uint32_t n, Is is, Scaled scaled, int q, Reach reach) {
    while (n > NT && lo < hi) {
      const int bits = 64 - __clzll(hi - lo), shift = max(0, bits - 8);
      clear_bins();
      visit(x, 0, V, [&](int64_t j, float v) {
        const key_t key = key_of(v, (uint32_t)j);
        if (key < lo || key > hi || !is(key, v)) return;
        add((int)((hi - key) >> shift), WEIGHED ? (unsigned long long)rint(ldexp(scaled(v), q)) : 1ull);
      });
      unsigned long long w;
      uint32_t count;
      read_bins(w, count);
      const double own = WEIGHED ? ldexp((double)w, -q) * unit : (double)count;
      double total;
      const double running = block_running(sh, threadIdx.x < BINS ? own : 0.0, total);
      int b = block_first(sh, threadIdx.x < BINS && count > 0 && reach(above + running));
      if (b == NT) b = block_last(sh, threadIdx.x < BINS && count > 0);       // (rounding)
      if ((int)threadIdx.x == b) sh.bin_sum[0] = running - own, sh.bin_count[0] = count;
      __syncthreads();
      above += sh.bin_sum[0];
      n = sh.bin_count[0];
      const key_t top = hi - ((key_t)b << shift), width = ((key_t)1 << shift) - 1;
      lo = top - lo > width ? top - width : lo;
      hi = top;
      __syncthreads();
    }
  }

  // The key of the k-th token.
  __device__ key_t kth(int64_t k, key_t top) {
    key_t lo = 0, hi = top;
    double above = 0.0;
    const auto all = [](key_t, float) { return true; };
    narrow<false>(lo, hi, above, 1.0, (uint32_t)min(V, (int64_t)UINT32_MAX), all, [](float) { return 1.0; }, 0,
                  [&](double n) { return n >= (double)k; });
    const key_t mine = gather([&](key_t key, float) { return key >= lo && key <= hi; });
    __syncthreads();
    sh.list[threadIdx.x] = mine;
    __syncthreads();
    return sh.list[min((int64_t)NT - 1, k - 1 - (int64_t)above)];
  }

  // The last key of the shortest run of the keys from `cut` up whose weight reaches p
  // of theirs. A window of 256 bins spans 32 e-foldings of the weight from its top on,
  // each an eighth: a bin's weights are summed as whole numbers, scaled by its top. What
  // lies below (2^-46 and less of the top's weight each) is the next window's.
  __device__ key_t reach_p(double p, key_t cut) {
    const int q = 62 - (64 - __clzll((unsigned long long)V));
    const double fine = 8.0 * it;
    float top = m;
    double above = 0.0, goal = -1.0;
    for (;;) {
      clear_bins();
      double tail = 0.0;
      float below = -INFINITY;
      visit(x, 0, V, [&](int64_t j, float v) {
        if (v > top || v == -INFINITY || key_of(v, (uint32_t)j) < cut) return;
        const double at = ((double)top - (double)v) * fine;
        if (at < (double)BINS) {
          const int b = (int)at;
          add(b, (unsigned long long)rint(ldexp(exp(((double)v - (double)top) * it + 0.125 * b), q)));
        } else {
          below = fmaxf(below, v);
          if (goal < 0.0) tail += weight(v);
        }
      });
      unsigned long long w;
      uint32_t count;
      read_bins(w, count);
      const double scale = weight(top), unit = scale * exp(-0.125 * (threadIdx.x & (BINS - 1)));
      const double own = threadIdx.x < BINS ? ldexp((double)w, -q) * unit : 0.0;
      double total;
      const double running = block_running(sh, own, total);
      if (goal < 0.0) goal = p * (total + block_sum<NW>(tail, sh.red));
      const int b = block_first(sh, threadIdx.x < BINS && count > 0 && above + running >= goal);
      below = key_value((uint32_t)(block_top(sh, key_of(below, 0)) >> 32));
      if (b == NT && below > -INFINITY) {         // it lies below the window
        above += total;
        top = below;
        continue;
      }
      const int bin = b < NT ? b : block_last(sh, threadIdx.x < BINS && count > 0);
      if ((int)threadIdx.x == bin) {
        sh.bin_sum[0] = running - own;
        sh.bin_sum[1] = unit;
        sh.bin_count[0] = count;
      }
      __syncthreads();
      above += sh.bin_sum[0];
      const double of = sh.bin_sum[1];
      uint32_t n = sh.bin_count[0];
      __syncthreads();
      const auto is = [&](key_t key, float v) {
        if (v > top || v == -INFINITY || key < cut) return false;
        const double at = ((double)top - (double)v) * fine;
        return at < (double)BINS && (int)at == bin;
      };
      key_t lo = cut, hi = ~(key_t)0;
      // (its borders, outwards by more than their rounding; the test above is what decides)
      if (it > 0.0) {
        const double edge = bin / fine, next = (bin + 1) / fine;
        const float up = (float)((double)top - edge + (fabs((double)top) + edge) * 0x1p-48);
        const float down = (float)((double)top - next - (fabs((double)top) + next) * 0x1p-48);
        hi = (key_t)value_key(fminf(nextafterf(up, INFINITY), top)) << 32 | 0xFFFFFFFFu;
        lo = max(lo, (key_t)value_key(nextafterf(down, -INFINITY)) << 32);
      } else {
        hi = (key_t)value_key(top) << 32 | 0xFFFFFFFFu;
      }
      narrow<true>(lo, hi, above, of, n, is, [&](float v) { return exp(((double)v - (double)top) * it + 0.125 * bin); }, q,
                   [&](double s) { return s >= goal; });
      const key_t mine = gather([&](key_t key, float v) { return key >= lo && key <= hi && is(key, v); });
      const double sum = block_running(sh, mine != 0 ? weight(key_value((uint32_t)(mine >> 32))) : 0.0, total);
      int r = block_first(sh, mine != 0 && above + sum >= goal);
      if (r == NT) r = block_last(sh, mine != 0);
      __syncthreads();
      sh.list[threadIdx.x] = mine;
      __syncthreads();
      return sh.list[max(r, 0)];
    }
  }

  // The token drawn from the keys from `cut` up, and log(w / Z).
  __device__ int64_t draw(key_t cut, double u, double& logp) {
    const auto kept = [&](int64_t j, float v) -> double {
      if (key_of(v, (uint32_t)j) < cut) return 0.0;
      const double w = weight(v);
      return w >= min_p ? w : 0.0;
    };
    int64_t from = 0, to = V;
    double before = 0.0, goal = 0.0, Z = 0.0;
    for (bool whole = true;; whole = false) {     // the wavefront's run in which the sum passes
      double s = 0.0;
      visit(x, from, to, [&](int64_t j, float v) { s += kept(j, v); });
      s = wave_sum(s);
      __syncthreads();
      if ((threadIdx.x & 63) == 0) sh.red[threadIdx.x >> 6] = s;
      __syncthreads();
      if (whole) {
        for (int i = 0; i < NW; ++i) Z += sh.red[i];
        goal = u < 1.0 ? u * Z : INFINITY;
      }
      int at = -1;
      double sum = before, start = before;
      for (int i = 0; i < NW; ++i) {
        if (sh.red[i] > 0.0 && (at < 0 || start + sh.red[at] <= goal)) at = i, start = sum;
        sum += sh.red[i];
      }
      const int64_t run = run_length<T>(to - from);
      before = start;
      from += max(at, 0) * run;
      to = min(to, from + run);
      if (to - from <= 16 * NT) break;
    }
    const int64_t per = ceil_div(to - from, NT), j0 = from + threadIdx.x * per, j1 = min(to, j0 + per);
    double s = 0.0, total;
    for (int64_t j = j0; j < j1; ++j) s += kept(j, (float)x[j]);
    const double running = block_running(sh, s, total);
    int who = block_first(sh, s > 0.0 && before + running > goal);
    if (who == NT) who = block_last(sh, s > 0.0);
    __syncthreads();
    if ((int)threadIdx.x == who) {
      double sum = before + (running - s);
      int64_t token = -1;
      double own = 0.0;
      for (int64_t j = j0; j < j1; ++j) {
        const double w = kept(j, (float)x[j]);
        if (w <= 0.0) continue;
        token = j;
        own = w;
        sum += w;
        if (sum > goal) break;
      }
      sh.top[0] = (key_t)token;
      sh.red[0] = own;
    }
    __syncthreads();
    const int64_t token = (int64_t)sh.top[0];
    logp = log(sh.red[0] / Z);
    __syncthreads();
    return token;
  }
};

template <typename T>
__global__ __launch_bounds__(NT) void sample_kernel(SampleArgs a) {
  __shared__ Shared sh;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const T* x = static_cast<const T*>(a.logits) + t * a.ld;
    float best = -INFINITY;
    int64_t at = -1;
    visit(x, 0, a.V, [&](int64_t j, float v) {
      if (v > best || v != v) best = v, at = j;
    });
    // (-inf alone has a key, too: the first of a row of nothing else)
    const key_t top = block_top(sh, at < 0 ? 0 : key_of(best, (uint32_t)at));
    const float m = top == 0 ? -INFINITY : key_value((uint32_t)(top >> 32));
    const float temperature = a.temperature ? a.temperature[t] : 1.0f, p = a.top_p ? a.top_p[t] : 1.0f;
    const float min_p = a.min_p ? a.min_p[t] : 0.0f, u = a.u[t];
    const int64_t k = a.top_k && a.top_k[t] > 0 && a.top_k[t] < a.V ? a.top_k[t] : a.V;
    int64_t token = -1;
    double logp = __builtin_nan("");
    const bool nan = temperature != temperature || p != p || min_p != min_p || u != u || m != m || m == INFINITY;
    if (!nan && m == -INFINITY) {
      logp = -INFINITY;
    } else if (!nan && (temperature <= 0.0f || p <= 0.0f || k == 1)) {
      token = (int64_t)(uint32_t)~(uint32_t)top;
      logp = 0.0;
    } else if (!nan) {
      Row<T> row{sh, x, a.V, m, 1.0 / (double)temperature, min((double)max(min_p, 0.0f), 1.0)};
      key_t cut = 0;
      if (k < a.V) cut = row.kth(k, top);
      if (p < 1.0f) cut = row.reach_p((double)p, cut);
      token = row.draw(cut, max((double)u, 0.0), logp);
    }
    if (threadIdx.x == 0) {
      if (a.wide) static_cast<int64_t*>(a.tokens)[t] = token;
      else static_cast<int32_t*>(a.tokens)[t] = (int32_t)token;
      if (a.logp) a.logp[t] = (float)logp;
    }
    __syncthreads();
  }
}

template <typename T>
int sample_as(hipStream_t s, const SampleArgs& a) {
  hipLaunchKernelGGL(sample_kernel<T>, dim3((unsigned)std::min<int64_t>(a.T, 4096)), dim3(NT), 0, s, a);
  KMP_LAUNCH_CHECK();
  return 0;
}

}  // namespace

size_t sample_workspace(int64_t T, int64_t V) { return 256; }

int sample_tokens(hipStream_t s, const SampleArgs& a) {
  switch (a.type) {
    case KMP_F32: return sample_as<float>(s, a);
    case KMP_BF16: return sample_as<bf16_t>(s, a);
    default: return sample_as<f16_t>(s, a);
  }
}

}  // namespace kmp
