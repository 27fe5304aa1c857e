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
// the shift as large as D sums of at most 1 allow: sums of integers do not depend on
// the order in which the atomics arrive, so the choice does not either.
#include "dtypes.h"

namespace lst {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;
constexpr int kDigit = 11;  // bits of a pass: kBins = 2^kDigit

struct SampleArgs {
  int m, D;
  int64_t ldx;
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* tokens;
  float* prob;
  double unit;  // 2^shift
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

__device__ inline double weight(uint32_t key, uint32_t top, double t) {
  if (key == top) return 1.0;  // also where the largest is infinite
  if (key == 0) return 0.0;
  return exp(((double)value_of(key) - (double)value_of(top)) / t);
}

struct Shared {
  uint64_t bin[kBins];
  uint64_t wave[kWaves];
  uint64_t above;
  int found;
  uint32_t key[kWaves];
  int idx[kWaves];
};

// The first bin at which the running sum reaches target (at most the total): sh.found, and
// the sum before it, sh.above.
__device__ void find_bin(Shared& sh, uint64_t target) {
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
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

// The beginning of those that `in` holds whose values (value(key), an integer) reach target.
template <class T, class V>
__device__ Border border_of(Shared& sh, const T* x, int D, uint32_t top, uint32_t low, Border in,
                            uint64_t target, V value) {
  // by the distance of the keys from the largest one, from its leading digit down
  int bits = 32 - __clz((int)(top - low) | 1);
  uint32_t prefix = 0;
  uint64_t above = 0;
  while (bits > 0) {
    const int shift = max(bits - kDigit, 0);
    clear_bins(sh);
    for (int i = threadIdx.x; i < D; i += kThreads) {
      const uint32_t k = key_of((float)x[i]);
      if (!k || !in.holds(k, i)) continue;
      const uint32_t d = top - k;
      if (bits < 32 && (d >> bits) != prefix) continue;
      atomicAdd((unsigned long long*)&sh.bin[(d >> shift) & ((1u << (bits - shift)) - 1)],
                (unsigned long long)value(k));
    }
    find_bin(sh, target - above);
    above += sh.above;
    prefix = (prefix << (bits - shift)) | (uint32_t)sh.found;
    bits = shift;
  }
  Border out{top - prefix, D};
  // of the equal ones the first ones by index
  const uint64_t v = value(out.key);
  const uint64_t want = (target - above + v - 1) / v;
  const int size = (int)(((int64_t)D + kBins - 1) / kBins);
  clear_bins(sh);
  for (int i = threadIdx.x; i < D; i += kThreads)
    if (key_of((float)x[i]) == out.key && in.holds(out.key, i))
      atomicAdd((unsigned long long*)&sh.bin[i / size], 1ull);
  find_bin(sh, want);
  const int64_t first = (int64_t)sh.found * size;
  const int end = (int)min((int64_t)D, first + size);
  uint64_t left = want - sh.above;
  for (int64_t at = first; at < end; at += kBins) {  // rarely more than once
    clear_bins(sh);
    for (int j = threadIdx.x; j < kBins; j += kThreads) {
      const int64_t i = at + j;
      if (i < end) sh.bin[j] = key_of((float)x[i]) == out.key && in.holds(out.key, (int)i);
    }
    const uint64_t have = sum_bins(sh);
    if (have >= left) {
      find_bin(sh, left);
      out.last = (int)(at + sh.found);
      break;
    }
    left -= have;
  }
  return out;
}

// One block a row, over and over the row.
template <class T>
__global__ __launch_bounds__(kThreads) void sample_row_kernel(SampleArgs a, const T* logits) {
  __shared__ Shared sh;
  const int row = blockIdx.x, tid = threadIdx.x, D = a.D;
  const T* x = logits + row * a.ldx;
  const Wish w = wish_of(a, row);
  // the largest key, its first index, and the smallest key
  uint32_t top = 0, low = 0xFFFFFFFFu;
  int at = D;
  for (int i = tid; i < D; i += kThreads) {
    const uint32_t k = key_of((float)x[i]);
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
    if (tid == 0) {
      const bool none = !w.good || top == 0;
      a.tokens[row] = none ? -1 : at;
      if (a.prob) a.prob[row] = none ? 0.f : 1.f;
    }
    return;
  }
  const double t = w.t;
  auto whole = [&](double v) { return (uint64_t)(v * a.unit + 0.5); };
  auto mass = [&](uint32_t k) { return whole(weight(k, top, t)); };
  // u = 0 takes the first entry with any weight, however small beside 2^-shift
  const bool any = w.u == 0.f;
  auto part = [&](double v) { return any ? (uint64_t)(v > 0.0) : (uint64_t)(v * a.unit + 0.5); };
  // sums of the weights from q on that b holds, by stretches of indexes
  auto sums = [&](Border b, double q, int size, auto part) {
    clear_bins(sh);
    for (int i = tid; i < D; i += kThreads) {
      const uint32_t k = key_of((float)x[i]);
      if (!k || !b.holds(k, i)) continue;
      const double v = weight(k, top, t);
      if (k != top && v < q) continue;
      const uint64_t n = part(v);
      if (n) atomicAdd((unsigned long long*)&sh.bin[i / size], (unsigned long long)n);
    }
    return sum_bins(sh);
  };
  const int size = (int)(((int64_t)D + kBins - 1) / kBins);
  Border b{0, D};
  if (w.k > 0 && w.k < D) {
    clear_bins(sh);  // as many as there are, when they are fewer than k
    int n = 0;
    for (int i = tid; i < D; i += kThreads) n += key_of((float)x[i]) != 0;
    sh.bin[tid] = n;
    if (sum_bins(sh) > (uint64_t)w.k)
      b = border_of(sh, x, D, top, low, b, (uint64_t)w.k, [](uint32_t) { return (uint64_t)1; });
  }
  if (w.p < 1.f) {
    const uint64_t all = sums(b, 0.0, size, whole);
    const double want = ceil((double)w.p * (double)all);
    b = border_of(sh, x, D, top, low, b, want > 1.0 ? (uint64_t)want : 1, mass);
  }
  const uint64_t all = sums(b, (double)w.q, size, whole);
  if (any) sums(b, (double)w.q, size, part);
  const uint64_t want = (uint64_t)floor((double)w.u * (double)all) + 1;
  find_bin(sh, want);
  const int64_t first = (int64_t)sh.found * size;
  const int end = (int)min((int64_t)D, first + size);
  uint64_t left = want - sh.above;
  for (int64_t i0 = first; i0 < end; i0 += kBins) {
    clear_bins(sh);
    for (int j = tid; j < kBins; j += kThreads) {
      const int64_t i = i0 + j;
      if (i >= end) break;
      const uint32_t k = key_of((float)x[i]);
      if (!k || !b.holds(k, (int)i)) continue;
      const double v = weight(k, top, t);
      if (k == top || v >= (double)w.q) sh.bin[j] = part(v);
    }
    const uint64_t have = sum_bins(sh);
    if (have >= left) {
      find_bin(sh, left);
      if (tid == 0) {
        const int i = (int)(i0 + sh.found);
        a.tokens[row] = i;
        if (a.prob)
          a.prob[row] = (float)(weight(key_of((float)x[i]), top, t) / ((double)all / a.unit));
      }
      break;
    }
    left -= have;
  }
}

}  // namespace
}  // namespace lst

using namespace lst;

extern "C" {

int64_t lst_sample_workspace(int32_t m, int32_t D) { return m < 0 || D < 1 ? -1 : 0; }

int lst_sample(int32_t dtype, int32_t m, int32_t D, const void* logits, int64_t ldx,
               const float* temperature, const int32_t* top_k, const float* top_p,
               const float* min_p, const float* u, int32_t* tokens, float* prob, void* workspace,
               void* hip_stream) {
  if (!known_dtype(dtype) || m < 0 || D < 1) return LST_EINVAL;
  if (m == 0) return LST_OK;
  if (!logits || !u || !tokens || ldx < D) return LST_EINVAL;
  SampleArgs a{};
  a.m = m, a.D = D, a.ldx = ldx;
  a.temperature = temperature, a.top_k = top_k, a.top_p = top_p, a.min_p = min_p, a.u = u;
  a.tokens = tokens, a.prob = prob;
  int log = 0;
  while (((int64_t)1 << log) < D) ++log;
  a.unit = (double)((int64_t)1 << (62 - log));
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(sample_row_kernel<T>, dim3(m), dim3(kThreads), 0, (hipStream_t)hip_stream,
                       a, (const T*)logits);
    return launched();
  });
}

}  // extern "C"
