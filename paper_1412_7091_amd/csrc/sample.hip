// The choice of a token from a row of outputs (lst_sample): temperature, top-k,
// top-p and min-p, and one random number u that picks from what is left.
//
// Order a row's entries by value, equal ones by index.  Each of the three filters
// keeps a beginning of that order (the k first; the fewest whose weights reach p of
// those that top-k left; the weights of at least min-p), so what all of them keep is
// again a beginning, described by its last entry: a value and an index.  With
// w_i = exp((x_i - max) / t) the token is the first i, by index, at which the sum of
// the kept weights up to i exceeds u times the sum of all of them.
//
// Weights are computed in float64 and added as integers, multiples of 2^-shift with
// the shift as large as their sum allows in 64 bits (51 at most): sums of integers do
// not depend on the order in which the atomics arrive, so the choice does not either.
// A sum is off by at most 2^-52 D of the row's total (2^-27 where D says what the sum is
// at most, kFixedUnit): by half a step for each of D weights, of which one is 1.
//
// Rows of up to 8192 entries take one block each.  Longer ones are read by many blocks,
// once for the largest key of every 64 entries.  From those a bound follows that few
// entries reach where top-k or min-p is on, and one block a row ends it.  Without either,
// the row's weights go into 4096 bins by value (a second read), and the bin that top-p's
// border falls into is listed while the weights before it are added up by stretches of
// 4096 entries (a third).  A row whose border lies among more than 8192 unequal entries
// of one bin, or that keeps more than 8192 by top-k, is left to one block that goes over it
// digit by digit (128 rows of 200 000 with top-k 20 000 take 774 us, with 3000 167).
//
// Measured: one row of 200 000 floats with top-k 27 us, six launches that wait for each
// other; 128 such rows with all kinds of settings 112 us (22 for the read of 102 MB), 64
// rows of 793 471 bfloat16 with top-p alone 182 us (27 for the read).  The second and
// third pass are bound by the weights' arithmetic (56 and 76 us), the rest by the latency
// of blocks that search.  One block a row alone took 438, 938 and 3500 us.
//
// A row's bins share out the distance from its largest entry to its smallest one.  Entries
// masked by a finite low value instead of -inf make them wide (64 t at most, without top-k),
// and then the border's bin may hold more than 8192 entries: of 64 rows of 793 471 floats, one
// entry in a hundred at -1e4, with top-p 0.9 all are left to one block each, 3.3 ms for 0.21.
#include <algorithm>

#include "dtypes.h"

namespace lst {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;
constexpr int kDigit = 11;     // bits of a pass: kBins = 2^kDigit
constexpr int kChunk = 64;     // entries whose largest key is kept
constexpr int kStretch = 4096; // entries of one block of the first launch
constexpr int kList = 4096;    // entries that one block lists, at most
constexpr int kFine = 4096;    // bins of a row's values
constexpr int kSegment = 16384; // entries of one block that sorts them into bins (128 rows of
                                // 200 000: 11 us, with 32768 17; 64 of 793 471: 57 with either,
                                // with 8192 89)
constexpr int kLong = 8192;    // entries of a row's list in memory, at most
// Rows up to this length take one launch.  128 rows with top-k 50 and top-p, top-p alone, and
// neither: 35, 27 and 15 us in one launch and 25, 43 and 24 in six at 4096 entries, 43, 38 and
// 19 against 25, 45 and 25 at 8000, 58, 58 and 29 against 26, 45 and 26 at 16 000.  With top-k
// six launches are the faster ones from 4096 entries on, without it not before 8192; which rows
// have it is known on the device alone, and the line is the latter one.
constexpr int kShort = 8192;
constexpr int kBatch = 1024;   // rows of one set of launches
// Rows up to this length have the step that D weights of 1 leave, which is 2^-27 of the total
// for all D weights together; longer ones each have their own.
constexpr int kFixedUnit = 1 << 18;
constexpr int kMostRows = 1 << 20;     // of short rows' one launch
constexpr int kMostEntries = 1 << 30;  // of a row: an index and a block's step stay below 2^31

// What the launches leave each other of a long row.
enum { ROW_OPEN = 0, ROW_DONE = 1, ROW_MASS = 2, ROW_COUNT = 3 };
struct RowPlan {
  int state;
  uint32_t top;     // the largest key
  float top_value, scale;  // bin = (top_value - x) scale
  int bin;          // the one that holds the last entry kept
  uint64_t left;    // ROW_MASS: what the bin's entries have to give
  double unit;      // 2^shift of the row's weights
  // on a line of its own, since blocks add to it while others read what is above
  int apart[22];
  unsigned listed;  // entries of the bin (ROW_COUNT: of all up to it)
  int behind[31];
};

struct SampleArgs {
  int m, D;
  int64_t ldx;
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* tokens;
  float* prob;
  double unit;  // 2^shift where D alone says what the weights' sum is at most
  // the workspace, for rows longer than kShort: the largest key of each chunk; of each stretch
  // the smallest and the largest key and the sum of its weights, relative to the largest, then
  // the weight of its entries in the bins before the last and the number of those in it; per
  // row its plan, bins, and a list
  int chunks, stretches, segments;
  uint32_t *chunk_max, *stretch_min, *stretch_max;
  double* stretch_sum;
  uint64_t* stretch_mass;
  int* stretch_count;
  uint32_t *stretch_least, *stretch_most;  // of the entries in the last bin
  RowPlan* plan;
  uint64_t* bins;
  uint32_t* list_keys;
  int* list_indexes;
};

// What one row asks for.
struct Wish {
  float t, p, q, u;
  int k;
  bool good;
};

__device__ inline Wish wish_of(const SampleArgs& a, int row) {
  Wish w;
  w.t = a.temperature ? a.temperature[row] : 1.f;
  w.k = a.top_k ? a.top_k[row] : 0;
  w.p = a.top_p ? a.top_p[row] : 1.f;
  w.q = a.min_p ? a.min_p[row] : 0.f;
  w.u = a.u[row];
  w.good = w.t >= 0.f && isfinite(w.t) && !isnan(w.p) && !isnan(w.q) && w.u >= 0.f && w.u < 1.f;
  // no weight is more than 1: the first of the largest entries is left, as with top-k 1, and
  // further on min-p keeps every entry that is as large as the largest
  if (w.q > 1.f) w.k = 1, w.q = 0.f;
  return w;
}

// Keys are ordered as the values are, both zeros alike; 0: not to be chosen (-inf, not a
// number).
__device__ inline uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t k = b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
  return x > -INFINITY ? k : 0;
}

__device__ inline float value_of(uint32_t k) {
  return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}

// Weights w = exp((x - top) / t) = 2^(y / 64) with y = (x - top) 64 / (t ln 2): a table of the
// 64 roots of two, and a polynomial of the rest, at most ln 2 / 128, to 4e-17.  The long rows'
// passes are bound by this arithmetic (each operation in 64 bits is 2 us of 64 rows of 793 471
// entries).
struct Weight {
  double power, rest;  // the weight 2^shift is their product
  __device__ double value() const { return power * rest; }
  // to the next integer, in one rounding: the lowest 52 bits of a sum with 2^52
  __device__ uint64_t bits() const { return __double_as_longlong(fma(power, rest, 0x1p52)); }
  __device__ uint64_t whole() const { return bits() & 0xFFFFFFFFFFFFFull; }
};

struct Weights {
  const double* roots;  // 2^(shift + i / 64), in LDS, less i 2^14 in the upper word
  double c, unit;       // unit = 2^shift, at most 2^51
  double floor;         // x - top at which w = 2^-200
  float top;

  // 2^(shift + i / 64): one sum of the upper word and i 2^14
  __device__ double power(int i) const {
    const double d = roots[i & 63];
    return __hiloint2double(__double2hiint(d) + (i << 14), __double2loint(d));
  }
  __device__ static double rest(double r) {
    double q = fma(r, 1.2417843701716923e-12, 5.732851688640402e-10);  // (ln 2 / 64)^k / k!
    q = fma(r, q, 2.1173137155464774e-07);
    q = fma(r, q, 5.864904955056169e-05);
    q = fma(r, q, 0.010830424696249145);
    return fma(r, q, 1.0);
  }
  // w 2^shift where w is at least 2^-200 and the top is finite; 2^-200 2^shift, less than any
  // sum of weights can tell, for all that is less, -inf and what is no number.  The integer of
  // y is in the lowest bits of its sum with 1.5 2^52 (rint, the conversion and ldexp are slower).
  __device__ Weight near(float x) const {
    const double dx = fmax((double)x - (double)top, floor), t = fma(dx, c, 0x1.8p52);
    return {power(__double2loint(t)), rest(fma(dx, c, 0x1.8p52 - t))};
  }
  __device__ Weight weight(float x) const { return x == top ? Weight{unit, 1.0} : near(x); }
  // the same however small it is
  __device__ double scaled(float x) const {
    const double y = ((double)x - (double)top) * c, n = rint(y);
    if (x == top || y > -64.0 * 199) return weight(x).value();
    const int i = (int)n;
    return y > -64.0 * 1200 ? __builtin_ldexp(power(i & 63) * rest(y - n), i >> 6) : 0.0;
  }
  __device__ uint64_t whole(uint32_t key) const { return weight(value_of(key)).whole(); }
  __device__ double of(uint32_t key) const { return scaled(value_of(key)) / unit; }
};

// roots: filled for the unit.
__device__ inline Weights weights_of(const double* roots, double unit, uint32_t top, float t) {
  const double c = 92.332482616893656 / (double)t;  // 64 / ln 2
  return {roots, c, unit, -64.0 * 200 / c, value_of(top)};
}

__device__ inline void fill_roots(double* roots, double unit) {
  const int i = threadIdx.x;
  if (i >= 64) return;
  const double d = exp2(i / 64.0) * unit;
  roots[i] = __hiloint2double(__double2hiint(d) - (i << 14), __double2loint(d));
}

// The bins go down from the largest value; the last one holds all that is far below.  An
// entry's bin is the whole part of this.
__device__ inline float bin_value(const RowPlan& p, float x) {
  return fminf((p.top_value - x) * p.scale, kFine - 0.5f);
}

struct Shared {
  double roots[64];
  uint64_t bin[kBins];
  uint64_t wave[kWaves];
  uint64_t above;
  int found;
  uint32_t key[kWaves];
  int idx[kWaves];
  // the entries among which a search ends, and what it ends with
  int few, few_at;
  uint32_t few_keys[64], few_key;
  int few_indexes[64];
  uint64_t few_values[64];
};

// The first bin at which the running sum reaches target (at most the total): sh.found, and
// the sum before it, sh.above.  Bin 0 should no bin reach it: what is found is always a bin,
// and the indexes made from it are those of entries.
__device__ void find_bin(Shared& sh, uint64_t target) {
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  if (tid == 0) sh.found = 0, sh.above = 0;
  __syncthreads();
  const uint64_t a = sh.bin[2 * tid], b = sh.bin[2 * tid + 1];
  uint64_t sum = a + b;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t up = __shfl_up(sum, o);
    if (l >= o) sum += up;
  }
  if (l == 63) sh.wave[w] = sum;
  __syncthreads();
  uint64_t before = 0;
  for (int i = 0; i < w; ++i) before += sh.wave[i];
  const uint64_t after = before + sum, start = after - a - b;
  if (start < target && target <= after) {
    const bool second = start + a < target;
    sh.found = 2 * tid + second;
    sh.above = second ? start + a : start;
  }
  __syncthreads();
}

__device__ uint64_t sum_bins(Shared& sh) {
  const int tid = threadIdx.x;
  __syncthreads();
  uint64_t sum = sh.bin[2 * tid] + sh.bin[2 * tid + 1];
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if ((tid & 63) == 0) sh.wave[tid >> 6] = sum;
  __syncthreads();
  uint64_t all = 0;
  for (int i = 0; i < kWaves; ++i) all += sh.wave[i];
  return all;
}

// The smallest `least` and the largest `most` of all threads.
__device__ void extremes(Shared& sh, uint32_t& least, uint32_t& most) {
  for (int o = 32; o; o >>= 1) {
    least = min(least, (uint32_t)__shfl_xor((int)least, o));
    most = max(most, (uint32_t)__shfl_xor((int)most, o));
  }
  __syncthreads();
  if (threadIdx.x % 64 == 0)
    sh.key[threadIdx.x / 64] = most, sh.idx[threadIdx.x / 64] = (int)least;
  __syncthreads();
  for (int i = 0; i < kWaves; ++i)
    most = max(most, sh.key[i]), least = min(least, (uint32_t)sh.idx[i]);
  __syncthreads();  // the row's own search writes them again
}

__device__ void clear_bins(Shared& sh) {
  __syncthreads();
  sh.bin[2 * threadIdx.x] = 0;
  sh.bin[2 * threadIdx.x + 1] = 0;
  __syncthreads();
}

// The last entry that is kept: entries of larger keys, and those of this key up to index last.
struct Border {
  uint32_t key;
  int last;
  __device__ bool holds(uint32_t k, int i) const { return k > key || (k == key && i <= last); }
};

// Where entries come from: a row in memory, or a list of some of its entries.
template <class T>
struct RowEntries {
  const T* x;
  int n;
  __device__ int from(int64_t first) const { return (int)first; }
  __device__ int to(int64_t end) const { return (int)end; }
  __device__ int index(int p) const { return p; }
  __device__ uint32_t key(int p) const { return key_of((float)x[p]); }
  __device__ uint64_t count(Shared& sh) const;  // of those that may be chosen
};

struct ListEntries {
  const uint32_t* keys;
  const int* indexes;
  int n;
  __device__ int from(int64_t) const { return 0; }
  __device__ int to(int64_t) const { return n; }
  __device__ int index(int p) const { return indexes[p]; }
  __device__ uint32_t key(int p) const { return keys[p]; }
  __device__ uint64_t count(Shared&) const { return n; }
};

// The largest keys of a row's chunks.
struct Maxima {
  const uint32_t* k;
  int n;
  __device__ int index(int p) const { return p; }
  __device__ uint32_t key(int p) const { return k[p]; }
};

// The end of a search: sh.few entries, at most 64, among which the sum of value(key) in the
// order of before(a key, its index, another key, its index) reaches target: sh.few_key and
// sh.few_at.  One wave compares every entry with every other.
template <class V, class B>
__device__ void settle(Shared& sh, uint64_t target, V value, B before) {
  const int l = threadIdx.x, n = sh.few;
  if (l < 64 && l < n) {
    const uint32_t key = sh.few_keys[l];
    const int index = sh.few_indexes[l];
    const uint64_t own = value(key);
    sh.few_values[l] = own;
    __builtin_amdgcn_wave_barrier();
    uint64_t sum = 0;
    for (int j = 0; j < n; ++j)
      if (before(sh.few_keys[j], sh.few_indexes[j], key, index)) sum += sh.few_values[j];
    if (sum < target && target <= sum + own) sh.few_key = key, sh.few_at = index;
  }
  __syncthreads();
}

// Collects the entries p in [from, to) that `wanted` for it; true when they are at most 64.
template <class S, class W>
__device__ bool collect(Shared& sh, const S& src, int from, int to, W wanted) {
  if (threadIdx.x == 0) sh.few = sh.few_at = 0, sh.few_key = 0;
  __syncthreads();
  for (int p = from + threadIdx.x; p < to; p += kThreads) {
    const uint32_t k = src.key(p);
    const int i = src.index(p);
    if (!wanted(k, i)) continue;
    const int at = atomicAdd(&sh.few, 1);
    if (at < 64) sh.few_keys[at] = k, sh.few_indexes[at] = i;
  }
  __syncthreads();
  return sh.few <= 64;
}

// The index at which the sum by index of value(key) over those entries that `in` holds reaches
// target, which it does.
template <class S, class V>
__device__ int index_at(Shared& sh, const S& src, int D, Border in, uint64_t target, V value) {
  // by stretches of indexes, and then within one
  int64_t first = 0, size = D;
  while (size > 1) {
    const int64_t end = first + size < D ? first + size : D;
    const uint32_t step = (uint32_t)((size + kBins - 1) / kBins);
    clear_bins(sh);
    for (int p = src.from(first) + threadIdx.x; p < src.to(end); p += kThreads) {
      const int i = src.index(p);
      const uint32_t k = src.key(p);
      if (i < first || i >= end || !k || !in.holds(k, i)) continue;
      const uint64_t v = value(k);
      if (v) atomicAdd((unsigned long long*)&sh.bin[(uint32_t)(i - first) / step],
                       (unsigned long long)v);
    }
    find_bin(sh, target);
    target -= sh.above;
    first += (int64_t)sh.found * step;
    size = step;
    if (size == 1) break;
    const int64_t last = first + size < D ? first + size : D;
    if (collect(sh, src, src.from(first), src.to(last), [&](uint32_t k, int i) {
          return i >= first && i < last && k && in.holds(k, i);
        })) {
      settle(sh, target, value, [](uint32_t, int i, uint32_t, int j) { return i < j; });
      return sh.few_at;
    }
  }
  return (int)first;
}

// One digit of the distance from the largest key at which the sum of value(key), from there
// down over those entries that `in` holds, reaches target: of target is left what the
// entries with this prefix have to give, of bits the ones behind it.
template <class S, class V>
__device__ void search_digit(Shared& sh, const S& src, uint32_t top, Border in, uint64_t& target,
                             V value, int& bits, uint32_t& prefix) {
  const int shift = max(bits - kDigit, 0);
  clear_bins(sh);
  for (int p = threadIdx.x; p < src.n; p += kThreads) {
    const uint32_t k = src.key(p);
    if (!k || !in.holds(k, src.index(p))) continue;
    const uint32_t d = top - k;
    if (bits < 32 && (d >> bits) != prefix) continue;
    atomicAdd((unsigned long long*)&sh.bin[(d >> shift) & ((1u << (bits - shift)) - 1)],
              (unsigned long long)value(k));
  }
  find_bin(sh, target);
  target -= sh.above;
  prefix = (prefix << (bits - shift)) | (uint32_t)sh.found;
  bits = shift;
}

// A key that at least `count` of the entries reach, and hardly more than that: at most
// `spare` of them are as near to it as the search tells.
template <class S>
__device__ uint32_t key_near(Shared& sh, const S& src, uint32_t top, uint32_t low,
                             uint64_t count, uint64_t spare) {
  int bits = 32 - __clz((int)(top - low) | 1);
  uint32_t prefix = 0;
  while (bits > 0) {
    search_digit(sh, src, top, Border{0, src.n}, count, [](uint32_t) { return (uint64_t)1; },
                 bits, prefix);
    if (sh.bin[sh.found] <= spare) break;
  }
  return top - min(top, (uint32_t)((((uint64_t)prefix + 1) << bits) - 1));
}

// The beginning of those that `in` holds whose values (value(key), an integer) reach target:
// of the entries with its last key the first ones by index.
template <class S, class V>
__device__ Border border_of(Shared& sh, const S& src, int D, uint32_t top, uint32_t low,
                            Border in, uint64_t target, V value) {
  int bits = 32 - __clz((int)(top - low) | 1);
  uint32_t prefix = 0;
  while (bits > 0) {
    search_digit(sh, src, top, in, target, value, bits, prefix);
    const int left = bits;
    if (collect(sh, src, 0, src.n, [&](uint32_t k, int i) {
          return k && (top - k) >> left == prefix && in.holds(k, i);
        })) {
      settle(sh, target, value, [](uint32_t k, int i, uint32_t l, int j) {
        return k > l || (k == l && i < j);
      });
      return {sh.few_key, sh.few_at};
    }
  }
  const uint32_t key = top - prefix;
  const uint64_t v = value(key), want = (target + v - 1) / v;
  return {key, index_at(sh, src, D, in, want, [&](uint32_t k) { return (uint64_t)(k == key); })};
}

template <class S, class V>
__device__ uint64_t sum_of(Shared& sh, const S& src, Border in, V value) {
  uint64_t sum = 0;
  for (int p = threadIdx.x; p < src.n; p += kThreads) {
    const uint32_t k = src.key(p);
    if (k && in.holds(k, src.index(p))) sum += value(k);
  }
  __syncthreads();
  sh.bin[2 * threadIdx.x] = sum;
  sh.bin[2 * threadIdx.x + 1] = 0;
  return sum_bins(sh);
}

template <class T>
__device__ uint64_t RowEntries<T>::count(Shared& sh) const {
  return sum_of(sh, *this, Border{0, n}, [](uint32_t) { return (uint64_t)1; });
}

// The three filters and the choice.  total: the sum of the row's weights where the entries are
// not all of them and top-k is off; 0: the sum of these is it.
template <class S>
__device__ void choose(Shared& sh, const SampleArgs& a, int row, const Wish& w, const Weights& of,
                       const S& src, uint32_t low, uint64_t total) {
  const int D = a.D;
  const uint32_t top = key_of(of.top);
  auto mass = [&](uint32_t k) { return of.whole(k); };
  Border b{0, D};
  if (w.k > 0 && w.k < D) {
    auto one = [](uint32_t) { return (uint64_t)1; };
    if (src.count(sh) > (uint64_t)w.k)
      b = border_of(sh, src, D, top, low, b, (uint64_t)w.k, one);
  }
  if (w.p < 1.f) {
    const uint64_t have = sum_of(sh, src, b, mass);
    const double want = ceil((double)w.p * (double)(total ? total : have));
    const uint64_t target = want > 1.0 ? (uint64_t)want : 1;
    if (target <= have) b = border_of(sh, src, D, top, low, b, target, mass);
  }
  const double q = w.q;
  auto kept = [&](uint32_t k) { return k == top || q <= 0.0 || of.of(k) >= q ? of.whole(k) : 0; };
  const uint64_t all = sum_of(sh, src, b, kept);
  int at;
  if (w.u == 0.f) {
    // the first entry with any weight, however small beside 2^-shift
    at = index_at(sh, src, D, b, 1, [&](uint32_t k) {
      const double v = of.of(k);
      return (uint64_t)(v > 0.0 && (k == top || v >= q));
    });
  } else {
    at = index_at(sh, src, D, b, (uint64_t)((double)w.u * (double)all) + 1, kept);
  }
  for (int p = src.from(at) + threadIdx.x; p < src.to(at + 1); p += kThreads)
    if (src.index(p) == at) {
      a.tokens[row] = at;
      if (a.prob) a.prob[row] = (float)(of.of(src.key(p)) / ((double)all / of.unit));
    }
}

__device__ inline void give(const SampleArgs& a, int row, int token, float prob) {
  a.tokens[row] = token;
  if (a.prob) a.prob[row] = prob;
}

// ------------------------------------------------------------- long rows
// Whether the sum of all of a row's weights is wanted before any entry is listed.
__device__ inline bool wants_sum(const Wish& w, int D) {
  const bool k = w.k > 0 && w.k < D;
  return w.good && w.t > 0.f && !k && (w.p < 1.f) == (w.q > 0.f);
}

// A thread's entries of a stretch, which 256 of them have: kWide neighbours at a time.  -inf
// behind the row's end.
constexpr int kWide = 8, kSteps = kStretch / (256 * kWide);
template <class T>
__device__ inline void load_stretch(const T* x, int64_t base, int D, float (&v)[kSteps][kWide]) {
  T r[kSteps][kWide];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int64_t i = base + s * 256 * kWide;
    if (i + kWide <= D) {
      load_vec(x + i, r[s]);
    } else {
#pragma unroll
      for (int j = 0; j < kWide; ++j) r[s][j] = i + j < D ? x[i + j] : (T)-INFINITY;
    }
  }
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
#pragma unroll
    for (int j = 0; j < kWide; ++j) v[s][j] = (float)r[s][j];
}

// The largest key of every chunk, and the smallest key and the sum of every stretch: one read
// of the row.  A block has one stretch, eight lanes a chunk at a time.
template <class T>
__global__ __launch_bounds__(256) void sample_stats_kernel(SampleArgs a, const T* logits) {
  __shared__ double roots[64];
  __shared__ float wave_max[4], wave_min[4];
  __shared__ double wave_sum[4];
  const int row = blockIdx.y, stretch = blockIdx.x, tid = threadIdx.x;
  const T* x = logits + row * a.ldx;
  const int64_t base = (int64_t)stretch * kStretch + kWide * tid;
  float v[kSteps][kWide];
  load_stretch(x, base, a.D, v);
  fill_roots(roots, a.unit);
  float high = -INFINITY, low = INFINITY;  // of those that may be chosen
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    float h = -INFINITY;
#pragma unroll
    for (int j = 0; j < kWide; ++j) {
      h = v[s][j] > h ? v[s][j] : h;
      low = v[s][j] < low && v[s][j] > -INFINITY ? v[s][j] : low;
    }
#pragma unroll
    for (int o = kChunk / kWide / 2; o; o >>= 1) h = fmaxf(h, __shfl_xor(h, o));
    const int64_t chunk = (base + s * 256 * kWide) / kChunk;
    if (tid % (kChunk / kWide) == 0 && chunk < a.chunks)
      a.chunk_max[(int64_t)row * a.chunks + chunk] = key_of(h);
    high = fmaxf(high, h);
  }
  for (int o = 32; o >= kChunk / kWide; o >>= 1) high = fmaxf(high, __shfl_xor(high, o));
  for (int o = 32; o; o >>= 1) low = fminf(low, __shfl_xor(low, o));
  if (tid % 64 == 0) wave_max[tid / 64] = high, wave_min[tid / 64] = low;
  __syncthreads();
  high = fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
  const uint32_t top = key_of(high);
  const int64_t at = (int64_t)row * a.stretches + stretch;
  if (tid == 0) {
    low = fminf(fminf(wave_min[0], wave_min[1]), fminf(wave_min[2], wave_min[3]));
    a.stretch_min[at] = top ? key_of(low) : 0;
    a.stretch_max[at] = top;
  }
  const Wish w = wish_of(a, row);
  if (!wants_sum(w, a.D)) return;
  const Weights of = weights_of(roots, a.unit, top, w.t);  // no weight is rounded here
  double sum = 0.0;
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
#pragma unroll
    for (int j = 0; j < kWide; ++j) {
      sum += of.weight(v[s][j]).value();
      if (j % 2) asm volatile("" : "+v"(sum));  // 16 weights at once: 82 registers, 34 us for 27
    }
  sum /= a.unit;
  if (top == 0) sum = 0.0;
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (tid % 64 == 0) wave_sum[tid / 64] = sum;
  __syncthreads();
  if (tid == 0) a.stretch_sum[at] = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
}

// choose() for at most kFewEntries entries and u > 0: every entry is compared with every other
// one, four threads an entry, instead of sorted.
constexpr int kFewEntries = kThreads / 4;
__device__ void choose_few(Shared& sh, const SampleArgs& a, int row, const Wish& w,
                           const Weights& of, const ListEntries& list, uint64_t total) {
  uint64_t *order = sh.bin, *weight = sh.bin + kFewEntries, *kept = sh.bin + 2 * kFewEntries;
  const int tid = threadIdx.x, i = tid / 4, part = tid % 4, n = list.n;
  __syncthreads();
  if (tid < n) {
    order[tid] = (uint64_t)~list.keys[tid] << 32 | (uint32_t)list.indexes[tid];
    weight[tid] = of.whole(list.keys[tid]);
  }
  if (tid == 0) sh.above = 0;
  __syncthreads();
  int rank = 0;
  uint64_t before = 0;
  if (i < n)
    for (int j = part; j < n; j += 4)
      if (order[j] < order[i]) ++rank, before += weight[j];
  for (int o = 1; o < 4; o <<= 1) rank += __shfl_xor(rank, o), before += __shfl_xor(before, o);
  const int most = w.k > 0 && w.k < n ? w.k : n;
  if (i < n && part == 0 && rank == most - 1) sh.above = before + weight[i];
  __syncthreads();
  const double want = w.p < 1.f ? ceil((double)w.p * (double)(total ? total : sh.above)) : 0.0;
  if (i < n && part == 0) {
    const bool in = rank == 0 || (rank < most && (w.p >= 1.f || (double)before < want) &&
                                  (w.q <= 0.f || of.of(list.keys[i]) >= (double)w.q));
    kept[i] = in ? weight[i] : 0;
  }
  __syncthreads();
  uint64_t upto = 0, all = 0;
  if (i < n)
    for (int j = part; j < n; j += 4) {
      all += kept[j];
      if (list.indexes[j] <= list.indexes[i]) upto += kept[j];
    }
  for (int o = 1; o < 4; o <<= 1) upto += __shfl_xor(upto, o), all += __shfl_xor(all, o);
  const uint64_t target = (uint64_t)((double)w.u * (double)all) + 1;
  if (i < n && part == 0 && upto >= target && upto - kept[i] < target)
    give(a, row, list.indexes[i], (float)(of.of(list.keys[i]) / ((double)all / of.unit)));
}

// 2^shift for a row of more than kFixedUnit entries: its weights' sum is at most 64 times that
// of the chunks' largest ones, and that times 2^shift stays below 2^62 (the float32 sum is near
// enough: 2^64 is where the integers end).  3 us of 64 rows of 793 471 entries.
__device__ double unit_of(Shared& sh, const SampleArgs& a, const uint32_t* cmax, uint32_t top,
                          float t) {
  // halves: the difference of two finite values may have no float
  const float high = 0.5f * value_of(top), c = 2.88539008f / t;
  float sum = 0.f;
  for (int i = threadIdx.x; i < a.chunks; i += kThreads) {
    const uint32_t k = cmax[i];
    sum += k == top ? 1.f : k ? __builtin_amdgcn_exp2f((0.5f * value_of(k) - high) * c) : 0.f;
  }
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (threadIdx.x % 64 == 0) sh.key[threadIdx.x / 64] = __float_as_uint(sum);
  __syncthreads();
  float all = 0.f;
  for (int i = 0; i < kWaves; ++i) all += __uint_as_float(sh.key[i]);
  __syncthreads();
  // kChunk all is less than 2^(the biased exponent of all - 126) kChunk
  const int log = (int)(__float_as_uint(all) >> 23) - 126 + 6;
  static_assert(kChunk == 1 << 6, "");
  return fmax(a.unit, __hiloint2double((1023 + min(51, 62 - log)) << 20, 0));
}

struct PlanShared {
  Shared sh;
  uint32_t keys[kList];
  int indexes[kList];
  int hits[kList];  // chunks that hold entries of the list
  int count, n_hits;
};

// One block a row: what the chunks' largest keys leave of it.  Takes the rows that ask for the
// largest entry, for all of them, or for few that a bound on the key tells apart.
template <class T>
__global__ __launch_bounds__(kThreads) void sample_plan_kernel(SampleArgs a, const T* logits) {
  __shared__ PlanShared ps;
  Shared& sh = ps.sh;
  const int row = blockIdx.x, tid = threadIdx.x, D = a.D, n = a.chunks;
  const T* x = logits + row * a.ldx;
  const uint32_t* cmax = a.chunk_max + (int64_t)row * n;
  const Wish w = wish_of(a, row);
  RowPlan& plan = a.plan[row];
  if (tid == 0) plan.state = ROW_OPEN, ps.count = ps.n_hits = 0;
  fill_roots(sh.roots, a.unit);
  uint32_t top = 0, low = 0xFFFFFFFFu;
  for (int i = tid; i < n; i += kThreads) {
    const uint32_t k = cmax[i];
    top = max(top, k);
    if (k) low = min(low, k);
  }
  extremes(sh, low, top);
  if (!w.good || top == 0) {
    if (tid == 0) give(a, row, -1, 0.f), plan.state = ROW_DONE;
    return;
  }
  const bool k_on = w.k > 0 && w.k < D;
  double unit = a.unit;
  if (D > kFixedUnit && w.t > 0.f) {
    unit = unit_of(sh, a, cmax, top, w.t);
    if (tid < 64) sh.roots[tid] *= unit / a.unit;
    __syncthreads();
  }
  if (tid == 0) plan.unit = unit;
  const Weights of = weights_of(sh.roots, unit, top, w.t);
  uint64_t total = 0;
  if (wants_sum(w, D) && w.u > 0.f && a.stretches <= kBins) {
    clear_bins(sh);
    for (int i = tid; i < a.stretches; i += kThreads) {
      const uint32_t k = a.stretch_max[(int64_t)row * a.stretches + i];
      const double sum = a.stretch_sum[(int64_t)row * a.stretches + i] * of.of(k);
      sh.bin[i] = k ? (uint64_t)(sum * unit + 0.5) : 0;
    }
    total = sum_bins(sh);
    if (w.q <= 0.f) {
      // nothing is left out: the stretch, and the entry in it
      find_bin(sh, (uint64_t)((double)w.u * (double)total) + 1);
      const int64_t first = (int64_t)sh.found * kStretch;
      uint64_t left = (uint64_t)((double)w.u * (double)total) + 1 - sh.above;
      const int64_t end = first + kStretch < D ? first + kStretch : D;
      for (int half = 0; half < kStretch / kBins; ++half) {
        clear_bins(sh);
        for (int j = tid; j < kBins; j += kThreads) {
          const int64_t i = first + half * kBins + j;
          if (i < end) sh.bin[j] = of.whole(key_of((float)x[i]));
        }
        const uint64_t have = sum_bins(sh);
        if (have >= left) {
          find_bin(sh, left);
          if (tid == 0) {
            const int i = (int)(first + half * kBins) + sh.found;
            give(a, row, i, (float)(of.of(key_of((float)x[i])) / ((double)total / unit)));
            plan.state = ROW_DONE;
          }
          return;
        }
        left -= have;
      }
      return;  // the entries' roundings fell short of the stretch's: the row's own block
    }
  }
  // no entry that is kept has a smaller key than this
  uint32_t least = top;
  if (w.t > 0.f) {
    least = 0;
    if (k_on && w.k <= n) {
      // the k-th largest of the chunks' largest keys, or a little less: k entries are at
      // least as large
      const Maxima maxima{cmax, n};
      auto one = [](uint32_t) { return (uint64_t)1; };
      if (sum_of(sh, maxima, Border{0, n}, one) >= (uint64_t)w.k)
        least = key_near(sh, maxima, top, low, (uint64_t)w.k, kList / 16);
    }
    // (not where top-p asks for the weight of all that top-k leaves)
    if (w.q > 0.f && (w.p >= 1.f || total)) {
      // w >= q: x >= top + t ln q, with room for the roundings
      const double x0 = (double)value_of(top) + (double)w.t * (log((double)w.q) - 1e-9);
      const double room = fabs((double)value_of(top)) * 1e-12;
      float f = (float)(x0 - room);
      if ((double)f > x0 - room) f = nextafterf(f, -INFINITY);
      if (top != key_of(INFINITY) && f > -INFINITY) least = max(least, min(key_of(f), top));
    }
    if (w.u == 0.f) return;  // the row's own block
  }
  if (least) {
    // the chunks that have such entries, and those entries
    for (int i = tid; i < n; i += kThreads)
      if (cmax[i] >= least) {
        const int h = atomicAdd(&ps.n_hits, 1);
        if (h < kList) ps.hits[h] = i;
      }
    __syncthreads();
    // a half-wave a chunk, four chunks under way: bound by what one block can fetch (chunks of
    // 128 took twice the time)
    const int hits = ps.n_hits <= kList ? ps.n_hits : 0;
    for (int h0 = tid / 32; h0 < hits; h0 += 4 * (kThreads / 32)) {
      T v[4][kChunk / 32];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int h = min(h0 + c * (kThreads / 32), hits - 1);
        const int64_t i = (int64_t)ps.hits[h] * kChunk + tid % 32;
#pragma unroll
        for (int j = 0; j < kChunk / 32; ++j) v[c][j] = x[min(i + 32 * j, (int64_t)D - 1)];
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int h = h0 + c * (kThreads / 32);
        if (h >= hits) break;
        const int64_t i = (int64_t)ps.hits[h] * kChunk + tid % 32;
#pragma unroll
        for (int j = 0; j < kChunk / 32; ++j) {
          const uint32_t k = key_of((float)v[c][j]);
          if (k < least || i + 32 * j >= D) continue;
          const int at = atomicAdd(&ps.count, 1);
          if (at < kList) ps.keys[at] = k, ps.indexes[at] = (int)(i + 32 * j);
        }
      }
    }
    __syncthreads();
    if (ps.n_hits <= kList && ps.count <= kList) {
      const ListEntries list{ps.keys, ps.indexes, ps.count};
      if (w.t == 0.f) {
        const int at = index_at(sh, list, D, Border{top - 1, -1}, 1,
                                [](uint32_t) { return (uint64_t)1; });
        if (tid == 0) give(a, row, at, 1.f);
      } else if (list.n <= kFewEntries) {
        choose_few(sh, a, row, w, of, list, total);
      } else {
        choose(sh, a, row, w, of, list, least, total);
      }
      if (tid == 0) plan.state = ROW_DONE;
      return;
    }
  }
  if (w.t == 0.f || a.stretches > kBins || !isfinite(value_of(top))) return;
  // more of them: all of the row's entries into bins by their value
  low = 0xFFFFFFFFu;
  for (int i = tid; i < a.stretches; i += kThreads) {
    const uint32_t k = a.stretch_min[(int64_t)row * a.stretches + i];
    if (k) low = min(low, k);
  }
  uint32_t unused = 0;
  extremes(sh, low, unused);
  uint64_t* bins = a.bins + (int64_t)row * kFine;
  for (int i = tid; i < kFine; i += kThreads) bins[i] = 0;
  if (tid == 0) {
    // weights below e^-64 of the largest do not move the border of a sum
    const float all = value_of(top) - value_of(low);
    const float range = k_on ? all : fminf(all, 64.f * w.t);
    plan.top = top;
    plan.top_value = value_of(top);
    plan.scale = range > 0.f && isfinite(range) ? fminf(kFine / range, 1e38f) : 0.f;
    plan.bin = kFine;  // without top-k and top-p: no border, and no bins are needed
    plan.listed = 0;
    plan.state = k_on ? ROW_COUNT : ROW_MASS;
  }
}

// The entries of a row into bins by their value: the number in each (ROW_COUNT), or their
// weight (ROW_MASS), added up as integers.
template <class T>
__global__ __launch_bounds__(kThreads) void sample_bins_kernel(SampleArgs a, const T* logits) {
  __shared__ uint64_t bins[kFine];
  __shared__ double roots[64];
  const int row = blockIdx.y, tid = threadIdx.x;
  RowPlan& plan = a.plan[row];
  const int state = plan.state;
  if (state != ROW_MASS && state != ROW_COUNT) return;
  const RowPlan p = plan;
  const Wish w = wish_of(a, row);
  if (state == ROW_MASS && w.p >= 1.f) return;
  const T* x = logits + row * a.ldx;
  fill_roots(roots, p.unit);
  for (int i = tid; i < kFine; i += kThreads) bins[i] = 0;
  __syncthreads();
  const Weights of = weights_of(roots, p.unit, p.top, w.t);
  const int64_t base = (int64_t)blockIdx.x * kSegment + 4 * tid;
  T next[4];
  auto fetch = [&](int64_t i) {
    if (i + 4 <= a.D) {
      load_vec(x + i, next);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) next[j] = i + j < a.D ? x[i + j] : (T)-INFINITY;
    }
  };
  fetch(base);
  for (int s = 0; s < kSegment; s += 4 * kThreads) {
    const int64_t i = base + s;
    if (i >= a.D) break;
    T v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = next[j];
    if (s + 4 * kThreads < kSegment) fetch(i + 4 * kThreads);
    // what is not to be chosen adds nothing, to whichever bin
    if (state == ROW_MASS) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        atomicAdd((unsigned long long*)&bins[(int)bin_value(p, (float)v[j])],
                  (unsigned long long)of.near((float)v[j]).whole());
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        atomicAdd((unsigned long long*)&bins[(int)bin_value(p, (float)v[j])],
                  (unsigned long long)((float)v[j] > -INFINITY));
    }
  }
  __syncthreads();
  unsigned long long* sums = (unsigned long long*)a.bins + (int64_t)row * kFine;
  for (int i = tid; i < kFine; i += kThreads)
    if (bins[i]) atomicAdd(&sums[i], (unsigned long long)bins[i]);
}

// The bin of the border, from a row's bins: four of them a thread.
__global__ __launch_bounds__(kThreads) void sample_border_kernel(SampleArgs a) {
  static_assert(kFine == 4 * kThreads, "");
  __shared__ uint64_t wave[kWaves];
  const int row = blockIdx.x, tid = threadIdx.x, l = tid % 64, w = tid / 64;
  RowPlan& plan = a.plan[row];
  const int state = plan.state;
  if (state != ROW_MASS && state != ROW_COUNT) return;
  const Wish wish = wish_of(a, row);
  if (state == ROW_MASS && wish.p >= 1.f) return;
  uint64_t v[4], upto = 0;
  load_vec(a.bins + (int64_t)row * kFine + 4 * tid, v);
#pragma unroll
  for (int j = 0; j < 4; ++j) upto += v[j];
  const uint64_t own = upto;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t up = __shfl_up(upto, o);
    if (l >= o) upto += up;
  }
  if (l == 63) wave[w] = upto;
  __syncthreads();
  uint64_t all = 0;
  for (int i = 0; i < kWaves; ++i) {
    if (i == w) upto += all;
    all += wave[i];
  }
  uint64_t target = min((uint64_t)max(wish.k, 1), all);  // fewer entries than top-k: all of them
  if (state == ROW_MASS) {
    const double want = ceil((double)wish.p * (double)all);
    target = want > 1.0 ? (uint64_t)want : 1;
  }
  uint64_t before = upto - own;
  if (before >= target || upto < target) return;
  int bin = 0;
  while (bin < 3 && before + v[bin] < target) before += v[bin++];
  plan.bin = 4 * tid + bin;
  plan.left = target - before;
}

// The entries of the border's bin into the row's list (ROW_COUNT: of the bins before it too),
// and for each stretch the weight of those in the bins before and the number of those in it.
template <class T>
__global__ __launch_bounds__(256) void sample_list_kernel(SampleArgs a, const T* logits) {
  __shared__ double roots[64];
  __shared__ uint64_t wave_mass[4];
  __shared__ int wave_count[4];
  __shared__ uint32_t wave_least[4], wave_most[4];
  __shared__ unsigned first;
  const int row = blockIdx.y, stretch = blockIdx.x, tid = threadIdx.x, l = tid % 64;
  RowPlan& plan = a.plan[row];
  const int state = plan.state;
  if (state != ROW_MASS && state != ROW_COUNT) return;
  const RowPlan p = plan;
  const Wish w = wish_of(a, row);
  const T* x = logits + row * a.ldx;
  const int64_t base = (int64_t)stretch * kStretch + kWide * tid;
  float v[kSteps][kWide];
  load_stretch(x, base, a.D, v);
  fill_roots(roots, p.unit);
  __syncthreads();
  const Weights of = weights_of(roots, p.unit, p.top, w.t);
  const double q = (double)w.q * p.unit;
  const float below = p.bin, from = state == ROW_COUNT ? -1.f : below, upto_bin = below + 1.f;
  uint64_t mass = 0;
  uint32_t listed = 0, least = 0xFFFFFFFFu, most = 0;  // listed: a bit an entry
  auto mark = [&](int i, float f, float b) {
    if (b >= from && b < upto_bin && f > -INFINITY) {
      listed |= 1u << i;
      least = min(least, key_of(f));
      most = max(most, key_of(f));
    }
  };
  auto weigh = [&](auto limited) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int j = 0; j < kWide; ++j) {
        // (-inf and what is no number has no weight, and counts for nothing)
        const float f = v[s][j], b = bin_value(p, f);
        Weight d = of.near(f);
        const bool kept = b < below && (!limited.value || d.value() >= q);
        // (without the upper word: less than any sum can tell)
        d.power = __hiloint2double(kept ? __double2hiint(d.power) : 0, __double2loint(d.power));
        mass += d.bits();
        // (here, not behind all of the marks: that takes 142 registers and 109 us for 77)
        if (j % 2) asm volatile("" : "+v"(mass));
        mark(kWide * s + j, f, b);
      }
    // what each sum with 2^52 holds beside the integer (all of it modulo 2^64)
    mass -= kSteps * kWide * Weight{0.0, 0.0}.bits();
  };
  if (state == ROW_MASS) {
    w.q > 0.f ? weigh(std::true_type{}) : weigh(std::false_type{});
  } else {
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int j = 0; j < kWide; ++j) mark(kWide * s + j, v[s][j], bin_value(p, v[s][j]));
  }
  const int own = __popc(listed);
  int upto = own;  // of the wave's lanes up to this one
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(upto, o);
    if (l >= o) upto += up;
  }
  for (int o = 32; o; o >>= 1) {
    mass += __shfl_xor(mass, o);
    least = min(least, (uint32_t)__shfl_xor((int)least, o));
    most = max(most, (uint32_t)__shfl_xor((int)most, o));
  }
  if (l == 63) {
    wave_mass[tid / 64] = mass, wave_count[tid / 64] = upto;
    wave_least[tid / 64] = least, wave_most[tid / 64] = most;
  }
  __syncthreads();
  const int n = wave_count[0] + wave_count[1] + wave_count[2] + wave_count[3];
  if (tid == 0) {
    if (n) first = atomicAdd(&plan.listed, (unsigned)n);
    const int64_t at = (int64_t)row * a.stretches + stretch;
    a.stretch_mass[at] = wave_mass[0] + wave_mass[1] + wave_mass[2] + wave_mass[3];
    a.stretch_count[at] = n;
    a.stretch_least[at] =
        min(min(wave_least[0], wave_least[1]), min(wave_least[2], wave_least[3]));
    a.stretch_most[at] = max(max(wave_most[0], wave_most[1]), max(wave_most[2], wave_most[3]));
  }
  if (n == 0) return;
  __syncthreads();
  if (first >= kLong) return;  // the list is full: its row goes by the numbers or by itself
  unsigned at = first + upto - own;
  for (int k = 0; k < tid / 64; ++k) at += wave_count[k];
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
#pragma unroll
    for (int j = 0; j < kWide; ++j)
      if (listed >> (kWide * s + j) & 1) {
        if (at < kLong) {
          a.list_keys[(int64_t)row * kLong + at] = key_of(v[s][j]);
          a.list_indexes[(int64_t)row * kLong + at] = (int)(base + s * 256 * kWide + j);
        }
        ++at;
      }
}

// The rest of a row whose entries are in bins; false: more of them at the border than the list
// holds, and not all alike.
template <class T>
__device__ bool finish_bins(Shared& sh, const SampleArgs& a, int row, const Wish& w,
                            const T* x) {
  const int tid = threadIdx.x, D = a.D;
  const RowPlan p = a.plan[row];
  const Weights of = weights_of(sh.roots, p.unit, p.top, w.t);
  const ListEntries list{a.list_keys + (int64_t)row * kLong, a.list_indexes + (int64_t)row * kLong,
                         (int)p.listed};
  if (p.state == ROW_COUNT) {
    if (p.listed > kLong) return false;
    choose(sh, a, row, w, of, list, 1, 0);
    return true;
  }
  const uint64_t* mass = a.stretch_mass + (int64_t)row * a.stretches;
  const int* count = a.stretch_count + (int64_t)row * a.stretches;
  const double q = w.q;
  auto kept = [&](uint32_t k) { return k == p.top || q <= 0.0 || of.of(k) >= q ? of.whole(k) : 0; };
  // the smallest and largest key of the last bin
  uint32_t least = 0xFFFFFFFFu, most = 0;
  for (int i = tid; i < a.stretches; i += kThreads) {
    least = min(least, a.stretch_least[(int64_t)row * a.stretches + i]);
    most = max(most, a.stretch_most[(int64_t)row * a.stretches + i]);
  }
  extremes(sh, least, most);
  Border b{0, D};
  if (w.p >= 1.f) {
    clear_bins(sh);
    for (int i = tid; i < a.stretches; i += kThreads) sh.bin[i] = mass[i];
  } else if (least == most) {
    // one key: the first ones by index, by the stretches' numbers
    const uint64_t v = of.whole(most), want = (p.left + v - 1) / v;
    clear_bins(sh);
    for (int i = tid; i < a.stretches; i += kThreads) sh.bin[i] = count[i];
    find_bin(sh, want);
    const int stretch = sh.found;
    const uint64_t rest = want - sh.above;
    const int64_t first = (int64_t)stretch * kStretch;
    const RowEntries<T> part{x + first, (int)(first + kStretch < D ? kStretch : D - first)};
    b = {most, (int)first + index_at(sh, part, part.n, Border{most - 1, -1}, rest,
                                       [&](uint32_t k) { return (uint64_t)(k == most); })};
    const uint64_t each = kept(most);
    clear_bins(sh);
    for (int i = tid; i < a.stretches; i += kThreads)
      sh.bin[i] = mass[i] + each * (i < stretch ? (uint64_t)count[i] : i == stretch ? rest : 0);
  } else {
    if (p.listed > kLong) return false;
    b = border_of(sh, list, D, most, least, Border{0, D}, p.left,
                  [&](uint32_t k) { return of.whole(k); });
    clear_bins(sh);
    for (int i = tid; i < a.stretches; i += kThreads) sh.bin[i] = mass[i];
    __syncthreads();
    for (int i = tid; i < list.n; i += kThreads)
      if (b.holds(list.keys[i], list.indexes[i]))
        atomicAdd((unsigned long long*)&sh.bin[list.indexes[i] / kStretch],
                  (unsigned long long)kept(list.keys[i]));
  }
  const uint64_t all = sum_bins(sh);
  find_bin(sh, (uint64_t)((double)w.u * (double)all) + 1);
  const uint64_t left = (uint64_t)((double)w.u * (double)all) + 1 - sh.above;
  const int64_t first = (int64_t)sh.found * kStretch;
  const RowEntries<T> part{x + first, (int)(first + kStretch < D ? kStretch : D - first)};
  const Border here{b.key, (int)(b.last - first < -1 ? -1 : b.last - first)};
  const int at = index_at(sh, part, part.n, here, left, kept);
  if (tid == 0)
    give(a, row, (int)first + at, (float)(of.of(part.key(at)) / ((double)all / p.unit)));
  return true;
}

// One block a row, over and over the row: short rows, and those that the other launches leave.
template <class T>
__global__ __launch_bounds__(kThreads) void sample_row_kernel(SampleArgs a, const T* logits) {
  __shared__ Shared sh;
  const int row = blockIdx.x, tid = threadIdx.x, D = a.D;
  if (a.plan && a.plan[row].state == ROW_DONE) return;
  const double unit = a.plan ? a.plan[row].unit : a.unit;
  fill_roots(sh.roots, unit);
  const RowEntries<T> src{logits + row * a.ldx, D};
  const Wish w = wish_of(a, row);
  if (a.plan && a.plan[row].state != ROW_OPEN) {
    __syncthreads();
    if (finish_bins(sh, a, row, w, logits + row * a.ldx)) return;
  }
  // the largest key, its first index, and the smallest key
  uint32_t top = 0, low = 0xFFFFFFFFu;
  int at = D;
  for (int i = tid; i < D; i += kThreads) {
    const uint32_t k = src.key(i);
    if (k > top) top = k, at = i;
    if (k) low = min(low, k);
  }
  for (int o = 32; o; o >>= 1) {
    const uint32_t k = __shfl_xor(top, o);
    const int i = __shfl_xor(at, o);
    if (k > top || (k == top && i < at)) top = k, at = i;
    low = min(low, (uint32_t)__shfl_xor(low, o));
  }
  if ((tid & 63) == 0) sh.key[tid >> 6] = top, sh.idx[tid >> 6] = at, sh.wave[tid >> 6] = low;
  __syncthreads();
  for (int i = 0; i < kWaves; ++i) {
    const uint32_t k = sh.key[i];
    if (k > top || (k == top && sh.idx[i] < at)) top = k, at = sh.idx[i];
    low = min(low, (uint32_t)sh.wave[i]);
  }
  if (!w.good || top == 0 || w.t == 0.f) {
    const bool none = !w.good || top == 0;
    if (tid == 0) give(a, row, none ? -1 : at, none ? 0.f : 1.f);
    return;
  }
  choose(sh, a, row, w, weights_of(sh.roots, unit, top, w.t), src, low, 0);
}

struct Layout {
  SampleArgs args;
  int64_t bytes;
};

// The workspace of rows longer than kShort.
Layout layout(int m, int D, char* p) {
  Layout r{};
  SampleArgs& a = r.args;
  a.chunks = (int)(((int64_t)D + kChunk - 1) / kChunk);
  a.stretches = (int)(((int64_t)D + kStretch - 1) / kStretch);
  a.segments = (int)(((int64_t)D + kSegment - 1) / kSegment);
  int64_t at = 0;
  auto take = [&](auto*& q, int64_t n) {
    q = (std::remove_reference_t<decltype(q)>)(p + at);
    at += (n * (int64_t)sizeof(*q) + 127) / 128 * 128;
  };
  take(a.stretch_sum, (int64_t)m * a.stretches);
  take(a.stretch_min, (int64_t)m * a.stretches);
  take(a.stretch_max, (int64_t)m * a.stretches);
  take(a.chunk_max, (int64_t)m * a.chunks);
  take(a.stretch_mass, (int64_t)m * a.stretches);
  take(a.stretch_count, (int64_t)m * a.stretches);
  take(a.stretch_least, (int64_t)m * a.stretches);
  take(a.stretch_most, (int64_t)m * a.stretches);
  take(a.plan, m);
  take(a.bins, (int64_t)m * kFine);
  take(a.list_keys, (int64_t)m * kLong);
  take(a.list_indexes, (int64_t)m * kLong);
  r.bytes = at;
  return r;
}

}  // namespace
}  // namespace lst

using namespace lst;

extern "C" {

int64_t lst_sample_workspace(int32_t m, int32_t D) {
  if (m < 0 || D < 1 || D > kMostEntries) return -1;
  return D <= kShort ? 0 : layout(std::min(m, kBatch), D, nullptr).bytes;
}

int lst_sample(int32_t dtype, int32_t m, int32_t D, const void* logits, int64_t ldx,
               const float* temperature, const int32_t* top_k, const float* top_p,
               const float* min_p, const float* u, int32_t* tokens, float* prob, void* workspace,
               void* hip_stream) {
  if (!known_dtype(dtype) || m < 0 || D < 1 || D > kMostEntries) return LST_EINVAL;
  if (m == 0) return LST_OK;
  if (!logits || !u || !tokens || ldx < D) return LST_EINVAL;
  if (D > kShort && (!workspace || ((uintptr_t)workspace & 15))) return LST_EINVAL;
  int log = 0;
  while (((int64_t)1 << log) < D) ++log;
  hipStream_t s = (hipStream_t)hip_stream;
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    // long rows a batch at a time: the workspace is that of a batch
    const int batch = D > kShort ? kBatch : kMostRows;
    for (int64_t r = 0; r < m; r += batch) {
      const int n = (int)std::min<int64_t>(batch, m - r);
      SampleArgs a{};
      if (D > kShort) a = layout(n, D, (char*)workspace).args;
      a.m = n, a.D = D, a.ldx = ldx, a.u = u + r, a.tokens = tokens + r;
      if (temperature) a.temperature = temperature + r;
      if (top_k) a.top_k = top_k + r;
      if (top_p) a.top_p = top_p + r;
      if (min_p) a.min_p = min_p + r;
      if (prob) a.prob = prob + r;
      a.unit = (double)((int64_t)1 << std::min(51, 62 - log));
      const T* x = (const T*)logits + r * ldx;
      if (D > kShort) {
        hipLaunchKernelGGL(sample_stats_kernel<T>, dim3(a.stretches, n), dim3(256), 0, s, a, x);
        hipLaunchKernelGGL(sample_plan_kernel<T>, dim3(n), dim3(kThreads), 0, s, a, x);
        hipLaunchKernelGGL(sample_bins_kernel<T>, dim3(a.segments, n), dim3(kThreads), 0, s, a,
                           x);
        hipLaunchKernelGGL(sample_border_kernel, dim3(n), dim3(kThreads), 0, s, a);
        hipLaunchKernelGGL(sample_list_kernel<T>, dim3(a.stretches, n), dim3(256), 0, s, a, x);
      }
      hipLaunchKernelGGL(sample_row_kernel<T>, dim3(n), dim3(kThreads), 0, s, a, x);
    }
    return launched();
  });
}

}  // extern "C"
