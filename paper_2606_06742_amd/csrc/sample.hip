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
// Two launches: segments of rows are read once for histograms of their weights, on one
// grid, so that a row's bins are sums of its segments'; then a workgroup per row finds the
// bins that hold its cuts, and lists and orders only their tokens. Bound by the 64-bit
// work on each logit (1024 x 128000 bf16: 179 us at 37 vector instructions a logit, where
// the reads take 53 at a copy's rate) and by reading the row again for the list (90 us);
// by sorting rows, 16.4 ms. One row: by two dependent launches (9 and 15 us).
#include "kmp_keys.h"

namespace kmp {
namespace {

constexpr int NT = 512, NW = NT / 64;  // threads and wavefronts of a workgroup
constexpr int BINS = 256, COLS = 32;   // bins of a histogram, columns of each

constexpr int GRID = 512;              // bins of a segment's histogram
constexpr int kMostSegs = 64;
constexpr int LISTED = 4096;           // tokens near the cuts that are listed at most

struct Common {
  double red[NW];
  key_t top[NW];
  int first[NW];
  int n;
};
struct Shared : Common {               // of passes over a row alone
  union {
    struct {                           // two lanes share a column, on a bank of their own
      unsigned long long sum[BINS][COLS];
      uint32_t count[BINS][COLS];
    } h;
    key_t list[NT];
  };
  double bin_sum[2];
  uint32_t bin_count;
};
struct PickShared : Common {           // with the histograms of its segments
  key_t listed[LISTED];
  union {
    double sums[LISTED];               // running sums of their weights
    key_t turned[LISTED];              // while they are put in order: by buckets
  };
  int filled[NT], most;                // keys of a bucket, its end
  double weight[GRID];                 // running sums of the bins, relative to the row's maximum
  double tokens[GRID];
  double before[kMostSegs];
  double base[kMostSegs];              // a segment's first bin's border; -INFINITY: it has no bins
  int offset[kMostSegs];               // its place on the row's grid; GRID: none of it is there
};

// f(j, x_j) for the row's elements [from, to): wavefront w takes the w-th of WAVES
// neighbouring runs, in vectors of 16 bytes, U of them in flight.
template <typename T, int WAVES = NW>
__device__ __forceinline__ int64_t run_length(int64_t n) {
  constexpr int64_t STEP = 64 * vec_of<T>();
  return round_up(ceil_div(n, WAVES), STEP);
}
template <int U, int WAVES = NW, typename T, typename F>
__device__ __forceinline__ void visit(const T* x, int64_t from, int64_t to, F f) {
  constexpr int VEC = vec_of<T>(), STEP = 64 * VEC;
  const int64_t run = run_length<T, WAVES>(to - from), start = from + (threadIdx.x >> 6) * run, end = min(to, start + run);
  int64_t j = start + (threadIdx.x & 63) * VEC;
  if constexpr (U > 1) {
    for (; j + (U - 1) * STEP + VEC <= end; j += U * STEP) {
      T v[U][VEC];
#pragma unroll
      for (int i = 0; i < U; ++i) __builtin_memcpy(v[i], x + j + i * STEP, 16);
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) f(j + i * STEP + e, (float)v[i][e]);
    }
  }
#pragma unroll 1
  for (; j + VEC <= end; j += STEP) {
    float v[VEC];
    load_n(x + j, v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) f(j + e, v[e]);
  }
  for (; j < end; ++j) f(j, (float)x[j]);         // (the run's last vector, of one lane)
}

// The block's largest key, its sum, its running sum; each starts with a barrier.
__device__ __forceinline__ key_t block_top(Common& sh, key_t v) {
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
__device__ __forceinline__ double block_running(Common& sh, double v, double& total) {
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
__device__ __forceinline__ int block_first(Common& sh, bool is) {
  const unsigned long long b = __ballot(is);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.first[threadIdx.x >> 6] = b ? (int)(threadIdx.x & ~63) + __ffsll(b) - 1 : NT;
  __syncthreads();
  int at = NT;
#pragma unroll
  for (int i = 0; i < NW; ++i) at = min(at, sh.first[i]);
  return at;
}
__device__ __forceinline__ int block_last(Common& sh, bool is) {
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

// One row.
template <typename T>
struct Row {
  Common& sh;
  const T* x;
  int64_t V;
  float m;                             // its maximum
  double it;                           // 1 / temperature
  double min_p;                        // 0: none

  __device__ double weight(float v) const { return v == -INFINITY ? 0.0 : exp(((double)v - (double)m) * it); }

  __device__ double kept(key_t cut, int64_t j, float v) const {
    if (key_of(v, (uint32_t)j) < cut) return 0.0;
    const double w = weight(v);
    return w >= min_p ? w : 0.0;
  }

  // The first of the elements [from, to) at which `before` and the running sum of the
  // weights from the key `cut` up exceed `goal`, or the last that has a weight.
  __device__ int64_t pass(key_t cut, int64_t from, int64_t to, double before, double goal, double& weight_of) {
    while (to - from > 4 * NT) {                  // the wavefront's run in which the sum passes
      double s = 0.0;
      visit<1>(x, from, to, [&](int64_t j, float v) { s += kept(cut, j, v); });
      s = wave_sum(s);
      __syncthreads();
      if ((threadIdx.x & 63) == 0) sh.red[threadIdx.x >> 6] = s;
      __syncthreads();
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
    }
    // four neighbouring elements a thread at most
    const int per = (int)ceil_div(to - from, NT);
    const int64_t j0 = from + threadIdx.x * per;
    const int n = (int)max((int64_t)0, min((int64_t)per, to - j0));
    double s = 0.0, total;
    for (int e = 0; e < n; ++e) s += kept(cut, j0 + e, (float)x[j0 + e]);
    const double running = block_running(sh, s, total);
    int who = block_first(sh, s > 0.0 && before + running > goal);
    if (who == NT) who = block_last(sh, s > 0.0);
    __syncthreads();
    if ((int)threadIdx.x == who) {
      double sum = before + (running - s), own = 0.0;
      int64_t token = -1;
      for (int e = 0; e < n; ++e) {
        const double w = kept(cut, j0 + e, (float)x[j0 + e]);
        if (w <= 0.0) continue;
        token = j0 + e;
        own = w;
        sum += w;
        if (sum > goal) break;
      }
      sh.top[0] = (key_t)token;
      sh.red[0] = own;
    }
    __syncthreads();
    const int64_t token = (int64_t)sh.top[0];
    weight_of = sh.red[0];
    __syncthreads();
    return token;
  }
};

// Its cuts and its draw by passes over the row alone.
template <typename T>
struct Passes : Row<T> {
  using Row<T>::x;
  using Row<T>::V;
  using Row<T>::m;
  using Row<T>::it;
  using Row<T>::weight;
  using Row<T>::kept;
  using Row<T>::pass;
  Shared& sh;
  __device__ Passes(Shared& shared, const Row<T>& row) : Row<T>(row), sh(shared) {}

  // The keys for which is(key, x) holds, at most NT of them, one a thread, in
  // descending order (0: none).
  template <typename F>
  __device__ key_t gather(F is) {
    __syncthreads();
    sh.list[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    visit<1>(x, 0, V, [&](int64_t j, float v) {
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
  __device__ void read_bins(double& w, uint32_t& n) {
    __syncthreads();
    unsigned long long low = 0, high = 0;         // (a column has up to 64 bits)
    n = 0;
    if (threadIdx.x < BINS)
      for (int c = 0; c < COLS; ++c) {            // (staggered over the banks)
        const int at = (c + threadIdx.x) & (COLS - 1);
        low += (uint32_t)sh.h.sum[threadIdx.x][at];
        high += sh.h.sum[threadIdx.x][at] >> 32;
        n += sh.h.count[threadIdx.x][at];
      }
    w = ldexp((double)high, 32) + (double)low;
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
      visit<1>(x, 0, V, [&](int64_t j, float v) {
        const key_t key = key_of(v, (uint32_t)j);
        if (key < lo || key > hi || !is(key, v)) return;
        add((int)((hi - key) >> shift), WEIGHED ? (unsigned long long)rint(ldexp(scaled(v), q)) : 1ull);
      });
      double w;
      uint32_t count;
      read_bins(w, count);
      const double own = WEIGHED ? ldexp(w, -q) * unit : (double)count;
      double total;
      const double running = block_running(sh, threadIdx.x < BINS ? own : 0.0, total);
      int b = block_first(sh, threadIdx.x < BINS && count > 0 && reach(above + running));
      if (b == NT) b = block_last(sh, threadIdx.x < BINS && count > 0);       // (rounding)
      if ((int)threadIdx.x == b) sh.bin_sum[0] = running - own, sh.bin_count = count;
      __syncthreads();
      above += sh.bin_sum[0];
      n = sh.bin_count;
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
    // (a column's elements, those of 16 threads, are V / 32 and 256 at most: 2^-47 up to 2^20
    // tokens, 2^-36 for the longest rows)
    const int q = min(52, __clzll((unsigned long long)(V / 32 + 256)) - 1);
    const double fine = 8.0 * it;
    float top = m;
    double above = 0.0, goal = -1.0;
    for (;;) {
      clear_bins();
      double tail = 0.0;
      float below = -INFINITY;
      visit<1>(x, 0, V, [&](int64_t j, float v) {
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
      double w;
      uint32_t count;
      read_bins(w, count);
      const double scale = weight(top), unit = scale * exp(-0.125 * (threadIdx.x & (BINS - 1)));
      const double own = threadIdx.x < BINS ? ldexp(w, -q) * unit : 0.0;
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
        sh.bin_count = count;
      }
      __syncthreads();
      above += sh.bin_sum[0];
      const double of = sh.bin_sum[1];
      uint32_t n = sh.bin_count;
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

  // The token drawn from the keys from `cut` up, and its weight over their total.
  __device__ int64_t draw(key_t cut, double u, double& share) {
    double Z = 0.0;
    visit<1>(x, 0, V, [&](int64_t j, float v) { Z += kept(cut, j, v); });
    Z = block_sum<NW>(Z, sh.red);
    double w;
    const int64_t token = pass(cut, 0, V, 0.0, u < 1.0 ? u * Z : INFINITY, w);
    share = w / Z;
    return token;
  }
};

// ---- Histograms of segments
// A segment's weights are counted on a grid that all segments of a row share without
// knowing its maximum: with y = 16 x / temperature, bin floor(y) and in it the weight
// exp(f / 16), f = y - floor(y); 512 bins down from the segment's largest logit's span 32
// e-foldings. A bin's count and the sum of its exp(f / 16) - 1 are one 64-bit whole
// number, added to by one LDS atomic: the sum in steps of 2^-q below, the count from bit
// 64 - c up, c bits being enough for a column's elements (each four lanes' own) of SEG
// neighbouring ones, after which the columns are summed: q is 43 or more, so that a weight
// is within 2^-44 of its size in rows of any length.
constexpr int COLUMNS = 16;
constexpr int CT = 512, CW = CT / 64;  // threads and wavefronts that count one
constexpr int SEG = 16384;             // elements of a segment of rows that are not longer than 64 such, and of a round of longer ones
constexpr double kFine = 16.0;

struct Segment {
  double weight[GRID];                 // sums of exp(f / 16), the first bin that of the maximum
  uint32_t count[GRID];
  double tail;                         // the weight below them, relative to the maximum
  key_t top;                           // its largest logit's key (the index of greedy rows only, else 0)
};

__host__ __device__ constexpr int64_t segment_length(int64_t V) {
  return V <= (int64_t)SEG * kMostSegs ? SEG : round_up(ceil_div(V, kMostSegs), SEG);
}
__host__ __device__ constexpr int64_t segments(int64_t V) { return ceil_div(V, segment_length(V)); }

// exp(r) - 1 for r = f / 16 in [0, 1 / 16]: Taylor's terms up to r^7, the next is below
// 2^-47.
__device__ __forceinline__ double grow(double r) {
  double p = 1.0 / 5040.0;
  p = fma(p, r, 1.0 / 720.0);
  p = fma(p, r, 1.0 / 120.0);
  p = fma(p, r, 1.0 / 24.0);
  p = fma(p, r, 1.0 / 6.0);
  p = fma(p, r, 0.5);
  p = fma(p, r, 1.0);
  return p * r;
}

// f / 16 = (v scale - bin) step. The product's rounding may have taken it up to a bin's
// border, from below: f is then below 0 by that much, and kept so. From 2^40 on f is 0:
// different logits are 2^-24 of them apart or more, so that only equal ones share a grid
// from 2^33 on, and from 2^53 on f is rounding alone.
__device__ __forceinline__ double step_of(double first) { return fabs(first) < 0x1p40 ? 1.0 / kFine : 0.0; }

// A row's choices.
struct Choice {
  float temperature, p, min_p, u;
  int64_t k;
  bool nan, greedy;                    // greedy: the first token of the order
  __device__ Choice(const SampleArgs& a, int64_t t) {
    temperature = a.temperature ? a.temperature[t] : 1.0f;
    p = a.top_p ? a.top_p[t] : 1.0f;
    min_p = a.min_p ? a.min_p[t] : 0.0f;
    u = a.u[t];
    k = a.top_k && a.top_k[t] > 0 && a.top_k[t] < a.V ? a.top_k[t] : a.V;
    nan = temperature != temperature || p != p || min_p != min_p || u != u;
    greedy = !nan && (temperature <= 0.0f || p <= 0.0f || k == 1);
  }
  template <typename T>
  __device__ Row<T> row(Common& sh, const T* x, int64_t V, float m) const {
    return Row<T>{sh, x, V, m, 1.0 / (double)temperature, min((double)max(min_p, 0.0f), 1.0)};
  }
};

static_assert(GRID == CT, "a bin a thread");

// One workgroup per segment of a row: a pass for the maximum, one for the histogram, one
// for what lies below it where there is any; all but the first find the segment in the
// cache. LONG: segments of more than SEG elements, in rounds of that many (as one kernel 1
// to 2 % slower where there is one round).
template <typename T, bool LONG>
__global__ __launch_bounds__(CT, 4) void sample_count_kernel(SampleArgs a) {
  __shared__ unsigned long long bins[GRID][COLUMNS];
  __shared__ float tops[CW];
  __shared__ double red[CW];
  __shared__ uint32_t counts[CW];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t length = segment_length(a.V), from = blockIdx.x * length, to = min(a.V, from + length);
  // a column's elements are whole vectors
  const int64_t most = vec_of<T>() * ceil_div(min((int64_t)SEG, a.V), (int64_t)COLUMNS * vec_of<T>());
  const int c = 64 - __clzll((unsigned long long)most) + 1, q = min(67 - 2 * c, 51);
  const unsigned long long half = (unsigned long long)1 << (63 - c);   // a sum of 0: a little below it takes none off the count
  for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y) {
    const T* x = static_cast<const T*>(a.logits) + t * a.ld;
    Segment* out = static_cast<Segment*>(a.workspace) + t * gridDim.x + blockIdx.x;
    for (int i = threadIdx.x; i < GRID * COLUMNS; i += CT) (&bins[0][0])[i] = half;
    float m = -INFINITY;
    visit<4, CW>(x, from, to, [&](int64_t, float v) { m = __builtin_elementwise_maximum(m, v); });   // NaN where one is
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) m = __builtin_elementwise_maximum(m, __shfl_xor(m, off, kWave));
    if (lane == 0) tops[w] = m;
    __syncthreads();
    m = tops[0];
#pragma unroll
    for (int i = 1; i < CW; ++i) m = __builtin_elementwise_maximum(m, tops[i]);
    const Choice choice(a, t);
    uint32_t at = UINT32_MAX;                     // a greedy row's token: the first with the maximum
    if (choice.greedy) {
#pragma unroll 1
      for (int64_t j = from + threadIdx.x; j < to && at == UINT32_MAX; j += CT)
        if ((float)x[j] == m) at = (uint32_t)j;
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) at = min(at, (uint32_t)__shfl_xor((int)at, off, kWave));
      if (lane == 0) counts[w] = at;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < CW; ++i) at = min(at, counts[i]);
      __syncthreads();
    }
    uint32_t tail_count = 0;
    // (rows that are greedy, not finite or have no choice need no more than the maximum)
    const bool some = m > -INFINITY && m < INFINITY && !choice.greedy;
    const double it = 1.0 / (double)choice.temperature, scale = kFine * it, first = floor((double)m * scale);
    const int g = threadIdx.x;                    // thread g sums bin g
    double above = 0.0;                           // of exp(f / 16) - 1
    uint32_t number = 0;
    const auto sum_bin = [&] {
      int64_t sum = 0;
      const unsigned long long low = ((unsigned long long)1 << (64 - c)) - 1;
#pragma unroll 4
      for (int k = 0; k < COLUMNS; ++k) {         // (staggered over the banks)
        const unsigned long long b = bins[g][(k + g) & (COLUMNS - 1)];
        sum += (int64_t)(b & low) - (int64_t)half;
        number += (uint32_t)(b >> (64 - c));
      }
      above += ldexp((double)sum, -q);
    };
    if (some) {
      // p + 1.5 2^(52 - q) holds p in steps of 2^-q in its last bits; the count's one is
      // added and the constant's bits taken off at once
      const double magic = ldexp(1.5, 52 - q), step = step_of(first);
      const unsigned long long one = ((unsigned long long)1 << (64 - c)) - (unsigned long long)__double_as_longlong(magic);
      unsigned long long* column = &bins[0][lane & (COLUMNS - 1)];
      for (int64_t round = from;;) {
        const int64_t next = LONG ? min(to, round + SEG) : to;
        visit<1, CW>(x, round, next, [&](int64_t, float v) {
          const double bin = floor((double)v * scale), place = first - bin;
          if (place < (double)GRID) {
            const double p = grow(fma((double)v, scale, -bin) * step);
            atomicAdd(column + (int)place * COLUMNS, (unsigned long long)__double_as_longlong(p + magic) + one);
          } else if (v > -INFINITY) {
            ++tail_count;
          }
        });
        if (!LONG || next == to) break;
        round = next;
        __syncthreads();
        sum_bin();
        __syncthreads();
        for (int i = threadIdx.x; i < GRID * COLUMNS; i += CT) (&bins[0][0])[i] = half;
        __syncthreads();
      }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) tail_count += __shfl_xor(tail_count, off, kWave);
    if (lane == 0) counts[w] = tail_count;
    __syncthreads();
    tail_count = 0;
#pragma unroll
    for (int i = 0; i < CW; ++i) tail_count += counts[i];
    double tail = 0.0;
    if (tail_count > 0) {
#pragma unroll 1
      for (int64_t j = from + threadIdx.x; j < to; j += CT) {
        const float v = (float)x[j];
        if (v > -INFINITY && !(first - floor((double)v * scale) < (double)GRID)) tail += exp(((double)v - (double)m) * it);
      }
      tail = block_sum<CW>(tail, red);
    }
    sum_bin();
    out->weight[g] = (double)number + above;
    out->count[g] = number;
    if (threadIdx.x == 0) {
      out->tail = tail;
      out->top = choice.greedy ? key_of(m, at) : key_of(m, 0);
    }
    __syncthreads();
  }
}

// ---- The draw, one workgroup per row
// The first n keys of sh.listed (all different; n <= LISTED) in descending order. Few: a
// key's place is the number of larger ones (50 keys: 0.8 us, by shuffles of one wavefront
// 3.2). Else by buckets, bucket_of(key) in [0, NT), of which none has a larger key than the
// one before it: a key's place is its bucket's plus the number of larger ones in that; where
// one has more than kCrowded keys, by bitonic merges (the rest up to the next power of two
// is cleared). 45 rows with 600 keys or so: 54.2 us by merges, 50 by buckets, 57 by counting
// up to 512.
constexpr int kCounted = 128, kCrowded = 256;
template <typename F>
__device__ __forceinline__ void sort_list(PickShared& sh, int n, F bucket_of) {
  const int t = threadIdx.x;
  if (n <= kCounted) {
    const key_t mine = t < n ? sh.listed[t] : 0;
    int rank = 0;
    if ((t & ~63) < n) {
#pragma unroll 8
      for (int j = 0; j < n; ++j) rank += sh.listed[j] > mine;
    }
    __syncthreads();
    if (t < n) sh.listed[rank] = mine;
    __syncthreads();
    return;
  }
  sh.filled[t] = 0;
  if (t == 0) sh.most = 0;
  __syncthreads();
  for (int i = t; i < n; i += NT) atomicAdd(&sh.filled[bucket_of(sh.listed[i])], 1);
  __syncthreads();
  const int own = sh.filled[t];
  double all;
  const int end = (int)block_running(sh, (double)own, all);   // (whole numbers: exact)
  if (own > kCrowded) sh.most = own;
  __syncthreads();
  if (sh.most == 0) {
    sh.filled[t] = end - own;
    __syncthreads();
    for (int i = t; i < n; i += NT) {
      const key_t key = sh.listed[i];
      sh.turned[atomicAdd(&sh.filled[bucket_of(key)], 1)] = key;
    }
    __syncthreads();
    for (int i = t; i < n; i += NT) {             // (filled: the bucket's end)
      const key_t key = sh.turned[i];
      const int b = bucket_of(key), from = b > 0 ? sh.filled[b - 1] : 0, to = sh.filled[b];
      int rank = from;
      for (int j = from; j < to; ++j) rank += sh.turned[j] > key;
      sh.listed[rank] = key;
    }
    __syncthreads();
    return;
  }
  int size = 2 * kCounted;
  while (size < n) size *= 2;
  for (int i = n + t; i < size; i += NT) sh.listed[i] = 0;
  __syncthreads();
  for (int k = 2; k <= size; k <<= 1)
    for (int s = k >> 1; s > 0; s >>= 1) {
      for (int i = t; i < size / 2; i += NT) {
        const int p = 2 * i - (i & (s - 1)), r = p + s;   // a pair s apart
        const key_t u = sh.listed[p], v = sh.listed[r];
        if (((p & k) == 0) == (u < v)) sh.listed[p] = v, sh.listed[r] = u;
      }
      __syncthreads();
    }
}
// sh.sums: running sums of weight(key) over the first n of sh.listed.
template <typename F>
__device__ __forceinline__ void sum_list(PickShared& sh, int n, F weight) {
  const int per = (n + NT - 1) / NT, j0 = threadIdx.x * per;
  if (n <= 64) {
    if (threadIdx.x < 64) {
      const double s = wave_running((int)threadIdx.x < n ? weight(sh.listed[threadIdx.x]) : 0.0);
      if ((int)threadIdx.x < n) sh.sums[threadIdx.x] = s;
    }
    __syncthreads();
    return;
  }
  double s = 0.0, total;
  for (int e = 0; e < per; ++e)
    if (j0 + e < n) s += weight(sh.listed[j0 + e]);
  double running = block_running(sh, s, total) - s;
  for (int e = 0; e < per; ++e)
    if (j0 + e < n) sh.sums[j0 + e] = running += weight(sh.listed[j0 + e]);
  __syncthreads();
}
// The first i < n for which is(i) holds, n where there is none (is() once true stays so
// but for rounding).
template <typename F>
__device__ __forceinline__ int first_of(PickShared& sh, int n, F is) {
  const int per = (n + NT - 1) / NT, j0 = threadIdx.x * per;
  int at = n;
  for (int e = per - 1; e >= 0; --e)
    if (j0 + e < n && is(j0 + e)) at = j0 + e;
  const int who = block_first(sh, at < n);
  if (who == NT) return n;
  __syncthreads();
  if ((int)threadIdx.x == who) sh.n = at;
  __syncthreads();
  return sh.n;
}

static_assert(GRID == NT, "a bin a thread");

// A row's token by its segments' histograms, or -1 where its cuts are not in them (below
// 32 e-foldings, or with more than LISTED tokens in their bins). The bins that hold the
// cuts are known from running sums over the bins; only their tokens are looked for in
// the row and put in order, and where all that is kept is few, these, too.
template <int WHOLE, typename T>
__device__ __forceinline__ int64_t pick(PickShared& sh, Row<T>& row, const Segment* seg, int segs, int64_t length, int64_t k, double p,
                        double u, double& share) {
  const double scale = kFine * row.it, y = (double)row.m * scale, first = floor(y), f0 = kFine * step_of(first) * fma((double)row.m, scale, -first);
  const int g = threadIdx.x;
  // a bin's weights relative to the row's maximum, from those relative to its border
  const auto border_weight = [&](double bin) { return exp(-(first - bin + f0) * (1.0 / kFine)); };
  if (g < segs) {
    const float m = key_value((uint32_t)(seg[g].top >> 32));
    const double base = m > -INFINITY ? floor((double)m * scale) : -INFINITY, d = first - base;
    sh.base[g] = base;
    sh.offset[g] = d < (double)GRID ? (int)d : GRID;
    sh.before[g] = m > -INFINITY ? seg[g].tail * row.weight(m) : 0.0;
  }
  __syncthreads();
  // running counts and weights over the row's bins; what lies below them
  double w = 0.0, n = 0.0, below = g < segs ? sh.before[g] : 0.0;
#pragma unroll 4
  for (int s = 0; s < segs; ++s) {
    const int off = sh.offset[s];
    // (thread g: the row's bin g, and the segment's bin g where that is below the grid)
    const double here = g >= off ? seg[s].weight[g - off] : 0.0, under = g + off >= GRID ? seg[s].weight[g] : 0.0;
    w += here;
    n += g >= off ? (double)seg[s].count[g - off] : 0.0;
    if (under > 0.0) below += under * border_weight(sh.base[s] - g);
  }
  w *= border_weight(first - g);
  below = block_sum<NW>(below, sh.red);
  double total, tokens;
  const double runw = block_running(sh, w, total), runn = block_running(sh, n, tokens);
  sh.weight[g] = runw, sh.tokens[g] = runn;
  __syncthreads();
  const auto weight_to = [&](int b) { return b >= 0 ? sh.weight[b] : 0.0; };   // of the bins up to b
  const auto count_to = [&](int b) { return b >= 0 ? (int64_t)sh.tokens[b] : 0; };
  // the bins in which the cuts lie: the k-th token's, those where the sum may reach p of
  // the first k tokens' (their weight is not known before they are in order), those
  // around min_p
  const bool by_p = p < 1.0, by_m = row.min_p > 0.0;
  // (where k is not below the number of tokens that have a weight, most others being ruled
  // out, it leaves none out: 300 x 50000 with 500 left and k = 1000 384 / 64 us)
  const bool by_k = k < row.V && (below > 0.0 || (double)k < tokens);
  int kb = GRID, lo = GRID, hi = GRID - 1;
  double least = total + below, most = least;
  if (by_k) {
    kb = first_of(sh, GRID, [&](int b) { return sh.tokens[b] >= (double)k; });
    if (kb == GRID) return -1;
    least = weight_to(kb - 1), most = weight_to(kb);
    lo = hi = kb;
  }
  if (by_p) {
    const int plo = first_of(sh, GRID, [&](int b) { return sh.weight[b] >= p * least * (1.0 - 1e-9); });
    const int phi = first_of(sh, GRID, [&](int b) { return sh.weight[b] >= p * most * (1.0 + 1e-9); });
    if (phi == GRID && !by_k) return -1;
    lo = min(lo, plo), hi = min(hi, phi);
  }
  if (by_m) {                                     // a token of bin b has -16 log w = b + f0 - f, 0 <= f < 1
    const double edge = -kFine * log(row.min_p) - f0;
    if (!(edge + 2.0 < (double)GRID)) return -1;
    lo = min(lo, (int)floor(max(edge - 1e-6, -1.0)) + 1);
    hi = min(hi, (int)ceil(edge + 1.0 + 1e-6));
  }
  key_t cut = 0;
  int listed = 0;
  double Z = total + below;
  if (by_k || by_p || by_m) {
    lo = min(lo, first_of(sh, GRID, [&](int b) { return sh.tokens[b] >= sh.tokens[hi]; }));   // (a bin that has tokens)
    const bool far = by_k && by_p && kb > hi;     // the k-th token's bin as well, for the weight of the first k
    // (all that may be kept where that is few, WHOLE at most: then no run of the row has to
    // be passed through for the draw. us with 512 / 2048: 1024 rows with 1280 tokens that
    // are not ruled out 517 / 394, one such row 52.9 / 55.9, so that few rows take 512)
    if (count_to(hi) + (far ? count_to(kb) - count_to(kb - 1) : 0) <= WHOLE) lo = 0;
    const int64_t near = count_to(hi) - count_to(lo - 1), more = far ? count_to(kb) - count_to(kb - 1) : 0;
    if (near + more > LISTED) return -1;
    // list them: logits below `low` are of later bins (a little lower than the border, for
    // its rounding; the bin decides)
    const int last = far ? kb : hi;
    const double border = (first - last) / scale;
    const float low = scale > 0.0 ? nextafterf((float)(border - fabs(border) * 0x1p-40), -INFINITY) : -INFINITY;
    __syncthreads();
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    const auto bin_of = [&](float v) {
      const double d = first - floor((double)v * scale);
      return d < (double)GRID ? (int)d : GRID;
    };
    visit<4>(row.x, 0, row.V, [&](int64_t j, float v) {
      bool is = v >= low && v > -INFINITY;
      if (!__any(is)) return;
      const int b = bin_of(v);
      is = is && ((b >= lo && b <= hi) || (far && b == kb));
      const unsigned long long which = __ballot(is);
      if (which == 0) return;
      int at = 0;                                 // (one atomic a wavefront)
      const int leader = __ffsll(which) - 1;
      if ((int)(threadIdx.x & 63) == leader) at = atomicAdd(&sh.n, __popcll(which));
      at = __shfl(at, leader, kWave) + __popcll(which & (((unsigned long long)1 << (threadIdx.x & 63)) - 1));
      if (is && at < LISTED) sh.listed[at] = key_of(v, (uint32_t)j);
    });
    __syncthreads();
    const int size = min(sh.n, LISTED);
    __syncthreads();
    const double edge = first - lo + 1.0, finer = (double)NT / (last - lo + 1);
    sort_list(sh, size, [&](key_t key) {
      const double d = edge - (double)key_value((uint32_t)(key >> 32)) * scale;
      return (int)min(max(d * finer, 0.0), (double)(NT - 1));
    });
    const auto weight = [&](key_t key) { return row.weight(key_value((uint32_t)(key >> 32))); };
    sum_list(sh, size, weight);
    const int run = (int)near;                    // the first of them, bins lo to hi
    const double before = weight_to(lo - 1);
    int end = run;                                // kept of them
    double of = total + below;
    if (by_k) {
      const int64_t rank = k - (far ? count_to(kb - 1) - run : count_to(lo - 1));   // the k-th token's place in the list
      if (rank >= 1 && rank <= size) {
        of = far ? weight_to(kb - 1) + (sh.sums[rank - 1] - sh.sums[run - 1]) : before + sh.sums[rank - 1];
        end = (int)min((int64_t)end, rank);
      } else if (by_p) {
        return -1;
      }
    }
    if (by_p) {
      const double reach = p * of;
      const int r = first_of(sh, run, [&](int i) { return before + sh.sums[i] >= reach; });
      end = min(end, r + 1);
    }
    if (by_m) end = min(end, first_of(sh, run, [&](int i) { return weight(sh.listed[i]) < row.min_p; }));
    if (end <= 0) return -1;
    cut = sh.listed[end - 1];
    Z = before + sh.sums[end - 1];
    listed = end;
    __syncthreads();
  }
  const double goal = u < 1.0 ? u * Z : INFINITY;
  if (listed > 0) {                               // by index: the complemented index above the value's bits
    for (int i = threadIdx.x; i < listed; i += NT) sh.listed[i] = sh.listed[i] << 32 | sh.listed[i] >> 32;
    __syncthreads();
    const double finer = (double)NT / (double)row.V;
    sort_list(sh, listed, [&](key_t key) { return min((int)((double)(uint32_t)~(uint32_t)(key >> 32) * finer), NT - 1); });
    sum_list(sh, listed, [&](key_t key) { return row.weight(key_value((uint32_t)key)); });
    if (lo == 0) {                                // all that is kept
      int i = first_of(sh, listed, [&](int i) { return sh.sums[i] > goal; });
      if (i == listed) i = listed - 1;
      // (the last that has a weight, and not one of none)
      while (i > 0 && row.weight(key_value((uint32_t)sh.listed[i])) <= 0.0) --i;
      share = row.weight(key_value((uint32_t)sh.listed[i])) / Z;
      return (int64_t)(uint32_t)~(uint32_t)(sh.listed[i] >> 32);
    }
  }
  // the segment in which the sum passes: its bins before `lo` (all of it without cuts)
  // and its listed tokens
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int s = wave; s < segs; s += NW) {
    const int off = sh.offset[s], bins = cut != 0 ? lo : GRID;
    const double base = sh.base[s], tail = sh.before[s];
    double sum = 0.0;
    if (base > -INFINITY) {
#pragma unroll 4
      for (int i = lane; i < GRID; i += 64) {
        const double own = cut == 0 || i + off < bins ? seg[s].weight[i] : 0.0;
        if (own > 0.0) sum += own * border_weight(base - i);
      }
      if (lane == 0 && cut == 0) sum += tail;
    }
    sum = wave_sum(sum);
    if (lane == 0) sh.before[s] = sum;
  }
  __syncthreads();
  if (listed > 0 && (int)threadIdx.x < segs) {    // thread s: the listed tokens of segment s
    const auto end_of = [&](int s) {              // how many lie before segment s + 1
      const uint32_t index = (uint32_t)((s + 1) * length);
      int a = 0, b = listed;
      while (a < b) {
        const int c = (a + b) / 2;
        if ((uint32_t)~(uint32_t)(sh.listed[c] >> 32) < index) a = c + 1;
        else b = c;
      }
      return a;
    };
    const int a = threadIdx.x == 0 ? 0 : end_of(threadIdx.x - 1), b = end_of(threadIdx.x);
    sh.before[threadIdx.x] += (b > 0 ? sh.sums[b - 1] : 0.0) - (a > 0 ? sh.sums[a - 1] : 0.0);
  }
  __syncthreads();
  int at = -1;
  double sum = 0.0, start = 0.0;
  for (int s = 0; s < segs; ++s) {
    const double own = sh.before[s];
    if (own > 0.0 && (at < 0 || start + sh.before[at] <= goal)) at = s, start = sum;
    sum += own;
  }
  __syncthreads();
  if (at < 0) return -1;
  double own;
  const double keep = row.min_p;
  row.min_p = 0.0;                                // (the cut has it)
  const int64_t token = row.pass(cut, at * length, min(row.V, (at + 1) * length), start, goal, own);
  row.min_p = keep;
  share = own / Z;
  return token;
}

constexpr int64_t kAside = -2;         // in a token's place: the row is left to sample_aside_kernel

__device__ __forceinline__ void put_token(const SampleArgs& a, int64_t t, int64_t token, double logp) {
  if (threadIdx.x != 0) return;
  if (a.wide) static_cast<int64_t*>(a.tokens)[t] = token;
  else static_cast<int32_t*>(a.tokens)[t] = (int32_t)token;
  if (a.logp) a.logp[t] = (float)logp;
}

// The rows whose cuts the histograms do not see: by passes over the row alone.
template <typename T>
__device__ __forceinline__ int64_t draw_aside(Shared& sh, const SampleArgs& a, const Choice& choice, const T* x, key_t top, double& logp) {
  Passes<T> row(sh, choice.row(sh, x, a.V, key_value((uint32_t)(top >> 32))));
  key_t cut = 0;
  if (choice.k < a.V) cut = row.kth(choice.k, top | UINT32_MAX);
  if (choice.p < 1.0f) cut = row.reach_p((double)choice.p, cut);
  double share;
  const int64_t token = row.draw(cut, max((double)choice.u, 0.0), share);
  logp = log(share);
  return token;
}

// ASIDE: those rows in the same launch, for no more rows than the chip has compute units
// (the registers and LDS of both allow one workgroup each there, of the draw alone two;
// a launch costs 4 us). Two need 128 registers, of which a few spill: us for one / two
// workgroups 1024 x 128000 bf16 286 / 268, 300 x 50000 f32 128 / 99, 2000 x 4000 f16 129 / 98.
template <typename T, bool ASIDE>
__global__ __launch_bounds__(NT, ASIDE ? 2 : 4) void sample_pick_kernel(SampleArgs a, int segs) {
  union All {
    PickShared pick;
    Shared aside;
    __device__ All() {}
  };
  __shared__ __align__(16) char memory[ASIDE ? sizeof(All) : sizeof(PickShared)];
  PickShared& sh = *reinterpret_cast<PickShared*>(memory);
  const int64_t length = segment_length(a.V);
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const T* x = static_cast<const T*>(a.logits) + t * a.ld;
    const Segment* seg = static_cast<const Segment*>(a.workspace) + t * segs;
    key_t top = 0;
    for (int s = threadIdx.x & 63; s < segs; s += 64) top = max(top, seg[s].top);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) top = max(top, (key_t)__shfl_xor(top, off, kWave));
    const float m = key_value((uint32_t)(top >> 32));
    const Choice choice(a, t);
    const bool nan = choice.nan || m != m || m == INFINITY;
    int64_t token = -1;
    double logp = __builtin_nan("");
    if (!nan && m == -INFINITY) {
      logp = -INFINITY;
    } else if (!nan && choice.greedy) {
      token = (int64_t)(uint32_t)~(uint32_t)top;
      logp = 0.0;
    } else if (!nan) {
      Row<T> row = choice.row(sh, x, a.V, m);
      double share = 0.0;
      token = pick<ASIDE ? NT : 2048>(sh, row, seg, segs, length, choice.k, (double)choice.p, max((double)choice.u, 0.0), share);
      logp = log(share);
      if (token < 0) {
        if constexpr (ASIDE) {
          __syncthreads();
          token = draw_aside(*reinterpret_cast<Shared*>(memory), a, choice, x, top, logp);
        } else {
          token = kAside;
        }
      }
    }
    put_token(a, t, token, logp);
    __syncthreads();
  }
}
template <typename T>
__global__ __launch_bounds__(NT) void sample_aside_kernel(SampleArgs a, int segs) {
  __shared__ Shared sh;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const int64_t mark = a.wide ? static_cast<const int64_t*>(a.tokens)[t] : static_cast<const int32_t*>(a.tokens)[t];
    if (mark != kAside) continue;
    const Segment* seg = static_cast<const Segment*>(a.workspace) + t * segs;
    key_t top = 0;
    for (int s = 0; s < segs; ++s) top = max(top, seg[s].top);
    double logp;
    const int64_t token = draw_aside(sh, a, Choice(a, t), static_cast<const T*>(a.logits) + t * a.ld, top, logp);
    put_token(a, t, token, logp);
    __syncthreads();
  }
}

template <typename T>
int sample_as(hipStream_t s, const SampleArgs& a) {
  const int segs = (int)segments(a.V);
  const dim3 grid((unsigned)segs, (unsigned)std::min<int64_t>(a.T, 65535));
  if (segment_length(a.V) == SEG) hipLaunchKernelGGL((sample_count_kernel<T, false>), grid, dim3(CT), 0, s, a);
  else hipLaunchKernelGGL((sample_count_kernel<T, true>), grid, dim3(CT), 0, s, a);
  const dim3 rows((unsigned)std::min<int64_t>(a.T, 65535));
  if (a.T <= 256) {
    hipLaunchKernelGGL((sample_pick_kernel<T, true>), rows, dim3(NT), 0, s, a, segs);
  } else {
    hipLaunchKernelGGL((sample_pick_kernel<T, false>), rows, dim3(NT), 0, s, a, segs);
    hipLaunchKernelGGL(sample_aside_kernel<T>, dim3(256), dim3(NT), 0, s, a, segs);
  }
  KMP_LAUNCH_CHECK();
  return 0;
}

}  // namespace

size_t sample_workspace(int64_t T, int64_t V) {
  // (a bound of the segments that does not fall: there are 64 up to 2^20 tokens, 33 from there on)
  return std::max<int64_t>(256, T * std::min<int64_t>(ceil_div(V, SEG), kMostSegs) * (int64_t)sizeof(Segment));
}

int sample_tokens(hipStream_t s, const SampleArgs& a) {
  switch (a.type) {
    case KMP_F32: return sample_as<float>(s, a);
    case KMP_BF16: return sample_as<bf16_t>(s, a);
    default: return sample_as<f16_t>(s, a);
  }
}

}  // namespace kmp
