// Log probabilities of given tokens, the entropy and the likeliest tokens of rows of outputs
// (lst_logprobs), and the gradient of the first two (lst_logprobs_backward).
//
//   z_j = (x_j - max) / T,  S = sum e^z,  p_j = e^z_j / S
//   logp_k = z_{t_k} - log S,   H = log S - sum e^z z / S
//   dL/dx_j = (sum_k g_k [j = t_k] - p_j (sum_k g_k + h (log p_j + H))) / T
//
// A row is read once forwards: each thread keeps the largest value so far, and S and sum e^z z
// relative to it, for its own entries.  Entries that are -inf or no number have no probability;
// where some are infinite, those share all of it.
//
// The likeliest tokens come from the largest value of each segment of 128 entries, which the same
// pass leaves: ordered by value and then by index, the first n entries lie in the first n
// segments of the same order, since each segment before an entry's own has an entry before it.
//
// A row of more than kShort entries takes two launches forwards: blocks of it that leave their
// sums, and one block that joins them and searches the n segments.  Shorter rows take one (16 384
// entries 4.6 us, 16 385 5.6; the 32 likeliest of them 10 and 11).
//
// Measured: 128 x 200 000 float32 20.5 us forwards, 5.0 TB/s, 4 more to join, 35 backwards, 5.8
// TB/s (the logits partly from the cache); 64 x 793 471 bfloat16 28 us, 3.6 TB/s, and 8 to join
// with the five likeliest, 54 backwards, 3.7 TB/s.  In 16 bits forwards the vector units work two
// thirds of the time that the compute units are busy (counted: 15 instructions, 66 clocks, a wave
// and entry, 51 000 of 76 000 clocks; five of the 15 are the exponent, its power and the two
// sums).  The rest is waiting: a block reads its four passes at once and sums with nothing under
// way, and 6208 blocks, where 2048 are resident, are three rounds and a little.
#include <algorithm>

#include "dtypes.h"

namespace lst {
namespace {

constexpr int kThreads = 256;
constexpr int kSegment = 128;              // entries whose largest value is kept: 16 lanes
constexpr int kPass = 8 * kThreads;        // entries of a block's pass
constexpr int kShort = 16384;
constexpr int kMostTop = 64;
constexpr int kMostTokens = 1024;
constexpr int64_t kMostEntries = 1 << 30;
constexpr int64_t kMostBlocks = 0xFFFFFF;  // of a launch: 2^32 threads
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Sums {  // relative to m: s = sum e^z, t = sum e^z z / ln 2
  float m, s, t;
};

// x - m, halved: entries may be further apart than the largest float.  (Halving is exact down to
// the smallest floats, and 2 c and t take it back: no other bit than without it.)
__device__ inline float half_of(float x, float m) { return fmaf(x, 0.5f, -0.5f * m); }

// An exponent of two that is never infinite: below 2^-1000 all is zero.  What is no number, and
// so a masked entry that is none, counts as the smallest.
__device__ inline float exponent(float x, float m, float c) {
  return fmaxf(half_of(x, m) * (2.f * c), -1e4f);
}

// c: log2(e) / T.  Eight entries more.
__device__ inline void add_entries(Sums& a, const float (&x)[8], float largest, float c) {
  const float m = fmaxf(a.m, largest);
  if (m > a.m) {
    const float d = exponent(fmaxf(a.m, kLowest), fmaxf(m, kLowest), c), f = exp2f(d);
    a.t = f * (a.t + d * a.s);
    a.s *= f;
    a.m = m;
  }
  if (m == INFINITY) {
#pragma unroll
    for (int i = 0; i < 8; ++i) a.s += x[i] == INFINITY ? 1.f : 0.f;
    return;
  }
  const float from = fmaxf(m, kLowest);  // so that -inf is below it
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float d = exponent(x[i], from, c), e = __builtin_amdgcn_exp2f(d);
    a.s += e;
    a.t = fmaf(e, d, a.t);
  }
}

// What a's sums are relative to m >= a.m.
__device__ inline void move_to(Sums& a, float m, float c) {
  const float d = a.m == m ? 0.f : exponent(fmaxf(a.m, kLowest), fmaxf(m, kLowest), c);
  const float f = exp2f(d);
  a.t = f * (a.t + d * a.s);
  a.s *= f;
  a.m = m;
}

// What the lane holds whose number differs in bit O: without LDS, whose shuffles take several
// times as long.
template <int O>
__device__ inline unsigned exchange(unsigned v) {
  if constexpr (O == 1) return __builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true);
  if constexpr (O == 2) return __builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true);
  if constexpr (O == 4) {  // the eight mirrored, then the four
    const int m = __builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true);
    return __builtin_amdgcn_update_dpp(0, m, 0x1B, 0xF, 0xF, true);
  }
  if constexpr (O == 8) return __builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, true);
  if constexpr (O == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  }
  const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return threadIdx.x & 32 ? r[0] : r[1];
}
template <int O>
__device__ inline float exchange(float v) {
  return __uint_as_float(exchange<O>(__float_as_uint(v)));
}

__device__ inline float wave_max(float v) {
  v = fmaxf(v, exchange<1>(v));
  v = fmaxf(v, exchange<2>(v));
  v = fmaxf(v, exchange<4>(v));
  v = fmaxf(v, exchange<8>(v));
  v = fmaxf(v, exchange<16>(v));
  return fmaxf(v, exchange<32>(v));
}
__device__ inline float wave_sum(float v) {
  v += exchange<1>(v);
  v += exchange<2>(v);
  v += exchange<4>(v);
  v += exchange<8>(v);
  v += exchange<16>(v);
  return v + exchange<32>(v);
}

// The block's sums, in every thread.
template <int THREADS>
__device__ inline Sums block_sums(Sums a, float c) {
  constexpr int kWaves = THREADS / 64;
  __shared__ Sums lds[kWaves];
  const int wave = threadIdx.x / 64;
  move_to(a, wave_max(a.m), c);
  a.s = wave_sum(a.s);
  a.t = wave_sum(a.t);
  if (threadIdx.x % 64 == 0) lds[wave] = a;
  __syncthreads();
  float m = lds[0].m;
#pragma unroll
  for (int i = 1; i < kWaves; ++i) m = fmaxf(m, lds[i].m);
  Sums all{m, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    Sums b = lds[i];
    move_to(b, m, c);
    all.s += b.s;
    all.t += b.t;
  }
  return all;
}

// Largest value of 16 neighbouring lanes, in each of them.
__device__ inline float row_max(float v) {
  v = fmaxf(v, exchange<1>(v));
  v = fmaxf(v, exchange<2>(v));
  v = fmaxf(v, exchange<4>(v));
  return fmaxf(v, exchange<8>(v));
}

struct Args {
  int64_t ldx;
  int D, K, top, chunks, segments, row0;
  const float* temperature;
  const int32_t* tokens;
  float *logp, *entropy, *saved;
  int32_t* ids;
  float* best;
  int32_t* status;
  float4* partial;  // a batch's rows x chunks
  float* largest;   // a batch's rows x segments
};

// T, or 0 for one that is not above zero and finite.  One below the normal floats counts as the
// smallest of these, so that twice its rate is a float.
__device__ inline float temperature_of(const float* temperature, int row) {
  const float t = temperature ? temperature[row] : 1.f;
  return t > 0.f && t < INFINITY ? fmaxf(t, 0x1p-126f) : 0.f;
}
__device__ inline float rate_of(float t) { return t > 0.f ? kLog2e / t : 1.f; }

// Entries col .. col + 7 of a row, -inf behind the last.
template <class T>
__device__ inline void load_entries(const T* x, int64_t col, int D, float (&v)[8]) {
  T raw[8];
  if (col + 8 <= D) {
    load_vec(x + col, raw);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)raw[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i] = x[min(col + i, (int64_t)D - 1)];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + i < D ? (float)raw[i] : -INFINITY;
  }
}

// Eight entries' weights, relative to 2^from, a whole number: the exponent is one rounding of
// x c - from, without the difference x - m, whose rounding c would scale.
__device__ inline void add_near(float& s, float& t, const float (&x)[8], float from, float c) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float d = fmaxf(fmaf(x[i], c, -from), -1e4f), e = __builtin_amdgcn_exp2f(d);
    s += e;
    t = fmaf(e, d, t);
  }
}

// N passes of a block over a row from entry `first`.
template <class T, int THREADS, int N>
__device__ inline void read_entries(Sums& sums, const T* x, int64_t first, int D, float c,
                                    float* largest) {
  float v[N][8], of[N], m = -INFINITY;
#pragma unroll
  for (int j = 0; j < N; ++j)
    load_entries(x, first + (int64_t)(j * THREADS + threadIdx.x) * 8, D, v[j]);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    of[j] = v[j][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) of[j] = fmaxf(of[j], v[j][i]);
    of[j] = fmaxf(of[j], -INFINITY);  // where all are no numbers
    m = fmaxf(m, of[j]);
    if (largest) {
      const float best = row_max(of[j]);
      const int64_t at = first + (int64_t)(j * THREADS + threadIdx.x) * 8;
      if (threadIdx.x % 16 == 0 && at < D) largest[at / kSegment] = best;
    }
  }
  Sums a{-INFINITY, 0.f, 0.f};
  const float top = m * c;
  if (fabsf(top) < 4194304.f) {
    const float from = rintf(top), d = fmaf(m, c, -from);
#pragma unroll
    for (int j = 0; j < N; ++j) add_near(a.s, a.t, v[j], from, c);
    const float f = __builtin_amdgcn_exp2f(-d);  // relative to m
    a.t = f * (a.t - d * a.s);
    a.s *= f;
    a.m = m;
  } else {  // large entries or small temperatures, infinite ones, or none
#pragma unroll
    for (int j = 0; j < N; ++j) add_entries(a, v[j], of[j], c);
  }
  m = fmaxf(sums.m, m);
  move_to(sums, m, c);
  move_to(a, m, c);
  sums.s += a.s;
  sums.t += a.t;
}

template <class T, int N>
__global__ __launch_bounds__(kThreads) void stats_kernel(Args a, const T* logits) {
  const int i = blockIdx.x / a.chunks, chunk = blockIdx.x - i * a.chunks, row = a.row0 + i;
  const float c = rate_of(temperature_of(a.temperature, row));
  Sums sums{-INFINITY, 0.f, 0.f};
  read_entries<T, kThreads, N>(sums, logits + row * a.ldx, (int64_t)chunk * kPass * N, a.D, c,
                               a.top ? a.largest + (int64_t)i * a.segments : nullptr);
  sums = block_sums<kThreads>(sums, c);
  if (threadIdx.x == 0) a.partial[blockIdx.x] = float4{sums.m, sums.s, sums.t, 0.f};
}

// ------------------------------------------------------------------ the likeliest tokens
// Order of an entry: by value, equal ones by index; 0 for one that has no probability.
__device__ inline uint64_t key_of(float x, uint32_t index) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(x + 0.f);  // one zero
  return (uint64_t)(b ^ (b >> 31 ? ~0u : 0x80000000u)) << 32 | ~index;
}
__device__ inline float value_of(uint64_t key) {
  const uint32_t b = (uint32_t)(key >> 32);
  return __uint_as_float(b >> 31 ? b ^ 0x80000000u : ~b);
}

template <int O>
__device__ inline uint64_t exchange(uint64_t k) {
  return (uint64_t)exchange<O>((unsigned)(k >> 32)) << 32 | exchange<O>((unsigned)k);
}

// One step of a bitonic sort: of two lanes the one that `first` names takes the larger key.
template <int O>
__device__ inline void order(uint64_t& k, bool first) {
  const uint64_t other = exchange<O>(k);
  k = first == (k > other) ? k : other;
}

// Keys that rise and then fall (or fall and rise): largest first, a lane each.
template <int WIDTH>
__device__ inline void merge(uint64_t& k, int lane, bool down) {
  if constexpr (WIDTH > 1) {
    order<WIDTH / 2>(k, ((lane & WIDTH / 2) == 0) == down);
    merge<WIDTH / 2>(k, lane, down);
  }
}
// The keys of a wave, smallest first.
__device__ inline uint64_t sort_up(uint64_t k, int lane) {
  merge<2>(k, lane, (lane & 2) == 0);
  merge<4>(k, lane, (lane & 4) == 0);
  merge<8>(k, lane, (lane & 8) == 0);
  merge<16>(k, lane, (lane & 16) == 0);
  merge<32>(k, lane, (lane & 32) == 0);
  merge<64>(k, lane, false);
  return k;
}
// The 64 largest of two sets, one largest first, the other smallest first.
__device__ inline uint64_t join(uint64_t a, uint64_t up, int lane) {
  uint64_t k = max(a, up);
  merge<64>(k, lane, true);
  return k;
}

__device__ inline uint64_t key_at(uint64_t k, int lane) {  // the same lane for the whole wave
  return (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 |
         (unsigned)__builtin_amdgcn_readlane((int)k, lane);
}

// Takes a key a lane (0: none) into the sorted list of a wave, of which the first n count.
__device__ inline void take(uint64_t& list, uint64_t k, int n, int lane) {
  uint64_t in = __ballot(k > key_at(list, n - 1));
  if (!in) return;
  if (__popcll(in) > 4) {
    list = join(list, sort_up(k, lane), lane);
    return;
  }
  for (; in; in &= in - 1) {
    const uint64_t one = key_at(k, __builtin_ctzll(in));
    const int at = __popcll(__ballot(list > one));
    const uint64_t before = (uint64_t)__shfl_up((unsigned long long)list, 1);
    list = lane < at ? list : lane == at ? one : before;
  }
}

// The n-th largest of the lanes' values: of many more values, n are no smaller.
__device__ inline float border_of(float v, int n, int lane) {
  const uint64_t up = sort_up(key_of(v, 0), lane);
  const uint64_t k = key_at(up, 64 - n);
  return k ? value_of(k) : -INFINITY;
}

// Takes N values a lane, whose indices `index` gives, into a wave's list: those that are no
// smaller than `least`, nor than the n-th of the lanes' largest.  They wait in the wave's `own`
// part of LDS: a loop over registers would have its body N times.
template <int N, class F>
__device__ inline void take_all(uint64_t& list, const float (&v)[N], float least, int n, int lane,
                                float (*own)[64], F index) {
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    own[i][lane] = v[i];
    m = fmaxf(m, v[i]);
  }
  least = fmaxf(least, border_of(m, n, lane));
#pragma unroll 1
  for (int i = 0; i < N; ++i) {
    const float x = own[i][lane];
    if (__ballot(x >= least)) take(list, x >= least ? key_of(x, index(i)) : 0, n, lane);
  }
}

// The waves' lists joined: in the first wave's registers, and in lds[0 .. 63] of every thread.
template <int WAVES>
__device__ inline uint64_t join_waves(uint64_t list, uint64_t (&lds)[WAVES][64]) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  __syncthreads();  // what was there has been read
  lds[wave][lane] = list;
  __syncthreads();
#pragma unroll
  for (int w = WAVES / 2; w; w >>= 1) {
    if (wave < w) {
      list = join(list, lds[wave + w][63 - lane], lane);
      lds[wave][lane] = list;
    }
    __syncthreads();
  }
  return list;
}

// The n likeliest of a row, largest first: put(rank, key).  A bound that n entries reach comes
// from the lanes' largest segments: the n-th of any wave, or the (n / waves)-th of every wave.
// Segments that reach it, then their entries that do, are gathered without an order, and each
// entry's rank is counted.  False, and nothing is put, where too many reach it (rows of few
// values) or the row has more segments than the lanes take.
template <class T, int THREADS, class F>
__device__ inline bool few_candidates(int segments, int D, int n, const T* x,
                                      const float* largest, F put) {
  constexpr int kWaves = THREADS / 64, kEach = 16, kSegments = 128, kKeys = 1024;
  __shared__ float bounds[2][2][kWaves];
  __shared__ int counts[2];
  __shared__ uint32_t found[kSegments];
  __shared__ __attribute__((aligned(16))) uint64_t keys[kKeys];
  if (segments > kEach * THREADS) return false;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  if (threadIdx.x < 2) counts[threadIdx.x] = 0;
  float v[kEach];
  // few segments go to all waves (many: neighbouring lanes read neighbours, 8 us for 11)
  const int own = segments < THREADS ? lane * kWaves + wave : threadIdx.x;
  auto bound_of = [&](int turn) {
    float m = v[0];
#pragma unroll
    for (int i = 1; i < kEach; ++i) m = fmaxf(m, v[i]);
    const uint64_t up = sort_up(key_of(m, 0), lane);
    const float value = up ? value_of(up) : -INFINITY;
    if (lane == 64 - n) bounds[turn][0][wave] = value;
    if (lane == 64 - (n + kWaves - 1) / kWaves) bounds[turn][1][wave] = value;
    __syncthreads();
    float any = bounds[turn][0][0], every = bounds[turn][1][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
      any = fmaxf(any, bounds[turn][0][w]);
      every = fminf(every, bounds[turn][1][w]);
    }
    return fmaxf(any, every);
  };
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int s = i * THREADS + own;
    v[i] = s < segments ? largest[s] : -INFINITY;
  }
  float bound = fmaxf(bound_of(0), kLowest);  // -inf is none
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (v[i] >= bound) {
      const int at = atomicAdd(&counts[0], 1);
      if (at < kSegments) found[at] = i * THREADS + own;
    }
  __syncthreads();
  const int segs = counts[0];
  if (segs > kSegments) return false;
  for (int s0 = wave; s0 - wave < segs; s0 += kEach / 2 * kWaves) {
    uint32_t first[kEach / 2];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int s = s0 + i / 2 * kWaves;
      if (i % 2 == 0) first[i / 2] = s < segs ? found[s] * kSegment + lane : 0xFFFFFFFFu;
      const uint32_t at = first[i / 2] + i % 2 * 64;
      v[i] = s < segs && at < (uint32_t)D ? (float)x[at] : -INFINITY;
    }
    // too few segments to tell a bound, or a low one: one from their entries
    if ((bound == kLowest || segments < 8 * n) && segs <= kEach / 2 * kWaves)
      bound = fmaxf(bound, bound_of(1));
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (v[i] >= bound) {
        const int at = atomicAdd(&counts[1], 1);
        if (at < kKeys) keys[at] = key_of(v[i], first[i / 2] + i % 2 * 64);
      }
  }
  __syncthreads();
  const int all = counts[1];
  if (all > kKeys) return false;
  for (int k = threadIdx.x; k < all; k += THREADS) {
    const uint64_t key = keys[k];
    int rank = 0;
    for (int j = 0; j < all; ++j) rank += keys[j] > key;
    if (rank < n) put(rank, key);
  }
  if ((int)threadIdx.x >= all && threadIdx.x < n) put(threadIdx.x, 0);
  return true;
}

// The same for any row: the waves' sorted lists of segments, and then of entries, joined.
template <class T, int THREADS, class F>
__device__ inline void many_candidates(int segments, int D, int n, const T* x,
                                       const float* largest, F put) {
  constexpr int kWaves = THREADS / 64;
  constexpr int kEach = 2 * kMostTop / kWaves;  // values of a lane at a time
  __shared__ uint64_t lists[kWaves][64];
  __shared__ float values[kWaves][kEach][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  uint64_t list = 0;
  for (int s0 = 0; s0 < segments; s0 += kEach * THREADS) {
    float v[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int64_t s = s0 + (int64_t)i * THREADS + threadIdx.x;
      v[i] = s < segments ? largest[s] : -INFINITY;
    }
    take_all(list, v, -INFINITY, n, lane, values[wave],
             [&](int i) { return s0 + i * THREADS + threadIdx.x; });
  }
  join_waves<kWaves>(list, lists);
  const float least = lists[0][n - 1] ? value_of(lists[0][n - 1]) : -INFINITY;
  auto segment = [&](int i) {  // where part i of the wave's segments begins; -1 for none
    const int at = i / 2 * kWaves + wave;
    const uint64_t k = at < n ? lists[0][at] : 0;
    return k ? (int64_t)(uint32_t)~k * kSegment + i % 2 * 64 : -1;
  };
  static_assert(kSegment == 128, "two parts of 64");
  float v[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int64_t first = segment(i);
    v[i] = first >= 0 && first + lane < D ? (float)x[first + lane] : -INFINITY;
  }
  list = 0;
  take_all(list, v, least, n, lane, values[wave],
           [&](int i) { return (uint32_t)segment(i) + lane; });
  list = join_waves<kWaves>(list, lists);
  if (threadIdx.x < n) put(threadIdx.x, list);
}

// ------------------------------------------------------------------------------- a row
// What is left for one block when a row's sums and segments are known.
// The first token of a thread, read before the row's sums are known.
struct Token {
  int token;
  float value;
};
template <class T>
__device__ inline Token token_of(const Args& a, int row, const T* x, int k) {
  Token t{-1, 0.f};
  if (k < a.K) {
    t.token = a.tokens[(int64_t)row * a.K + k];
    if (t.token >= 0 && t.token < a.D) t.value = (float)x[t.token];
  }
  return t;
}

template <class T, int THREADS>
__device__ inline void finish_row(const Args& a, int row, const T* x, Sums sums, float t,
                                  const float* largest, Token first) {
  const bool some = sums.m > -INFINITY && t > 0.f;
  const float log_s = some ? logf(sums.s) : 0.f;
  const float entropy = some ? log_s - kLn2 * sums.t / sums.s : 0.f;
  auto log_of = [&](float v) {
    if (!some || !(v > -INFINITY)) return -INFINITY;
    if (sums.m == INFINITY) return v == INFINITY ? -log_s : -INFINITY;
    return 2.f * (half_of(v, sums.m) / t) - log_s;
  };
  float* saved = a.saved ? a.saved + (int64_t)row * (a.K + 4) : nullptr;
  if (threadIdx.x == 0) {
    if (a.entropy) a.entropy[row] = entropy;
    if (saved) {
      saved[0] = sums.m;
      saved[1] = sums.s;
      saved[2] = entropy;
      saved[3] = some ? 1.f : 0.f;
    }
  }
  for (int k = threadIdx.x; k < a.K; k += THREADS) {
    const int64_t at = (int64_t)row * a.K + k;
    const Token one = k < THREADS ? first : token_of(a, row, x, k);
    const int token = one.token;
    float v = __builtin_nanf(""), l = 0.f;
    if (token >= 0 && token < a.D) {
      v = one.value;
      l = log_of(v);
      if (l == -INFINITY) v = __builtin_nanf("");  // no gradient
    } else if (token != -1 && a.status) {
      atomicCAS(a.status, 0, LST_EINDEX);
    }
    a.logp[at] = l;
    if (saved) saved[4 + k] = v;
  }
  if (!a.top) return;
  const int n = a.top;
  auto put = [&](int rank, uint64_t key) {
    const int64_t at = (int64_t)row * n + rank;
    // beside an infinite entry the others have no probability
    const bool one = key && (sums.m < INFINITY || value_of(key) == INFINITY);
    a.ids[at] = one ? (int32_t)~(uint32_t)key : -1;
    a.best[at] = one ? log_of(value_of(key)) : -INFINITY;
  };
  if (!some) {
    if (threadIdx.x < n) put(threadIdx.x, 0);
  } else if (!few_candidates<T, THREADS>(a.segments, a.D, n, x, largest, put)) {
    many_candidates<T, THREADS>(a.segments, a.D, n, x, largest, put);
  }
}

template <class T>
__global__ __launch_bounds__(512) void join_kernel(Args a, const T* logits) {
  const int row = a.row0 + blockIdx.x;
  const float t = temperature_of(a.temperature, row), c = rate_of(t);
  const Token first = token_of(a, row, logits + row * a.ldx, threadIdx.x);
  Sums sums{-INFINITY, 0.f, 0.f};
  for (int i = threadIdx.x; i < a.chunks; i += 512) {
    const float4 p = a.partial[(int64_t)blockIdx.x * a.chunks + i];
    Sums b{p.x, p.y, p.z};
    const float m = fmaxf(sums.m, b.m);
    move_to(sums, m, c);
    move_to(b, m, c);
    sums.s += b.s;
    sums.t += b.t;
  }
  sums = block_sums<512>(sums, c);
  finish_row<T, 512>(a, row, logits + row * a.ldx, sums, t,
                     a.top ? a.largest + (int64_t)blockIdx.x * a.segments : nullptr, first);
}

template <class T>
__global__ __launch_bounds__(512) void short_kernel(Args a, const T* logits) {
  __shared__ float largest[kShort / kSegment];
  const int row = a.row0 + blockIdx.x;
  const float t = temperature_of(a.temperature, row), c = rate_of(t);
  const T* x = logits + row * a.ldx;
  const Token first = token_of(a, row, x, threadIdx.x);
  Sums sums{-INFINITY, 0.f, 0.f};
  for (int at = 0; at < a.D; at += 8 * 512)
    read_entries<T, 512, 1>(sums, x, at, a.D, c, a.top ? largest : nullptr);
  sums = block_sums<512>(sums, c);  // and its barrier is behind the last of `largest`
  finish_row<T, 512>(a, row, x, sums, t, largest, first);
}

// -------------------------------------------------------------------------- the gradient
struct BackArgs {
  int64_t ldx, ldg;
  int D, K, chunks, row0;
  const float* temperature;
  const int32_t* tokens;
  const float *saved, *grad_logp, *grad_entropy;
};

// Bound by memory: an entry is read and written once.  Tokens' own terms are added by a second
// store of theirs, behind a barrier, from the values that the forward pass saved: the entries of
// x may be gone, since the gradient may take their place.
template <class T, int N>
__global__ __launch_bounds__(kThreads) void backward_kernel(BackArgs a, const T* logits, T* grad) {
  const int i = blockIdx.x / a.chunks, chunk = blockIdx.x - i * a.chunks, row = a.row0 + i;
  const T* x = logits + row * a.ldx;
  T* out = grad + row * a.ldg;
  const float* saved = a.saved + (int64_t)row * (a.K + 4);
  const int32_t* tokens = a.tokens + (int64_t)row * a.K;
  const float* gk = a.grad_logp + (int64_t)row * a.K;
  const int64_t first = (int64_t)chunk * kPass * N;
  float v[N][8];
#pragma unroll
  for (int j = 0; j < N; ++j)
    load_entries(x, first + (int64_t)(j * kThreads + threadIdx.x) * 8, a.D, v[j]);
  const float t = saved[3] != 0.f ? temperature_of(a.temperature, row) : 0.f;
  const float m = saved[0], c = rate_of(t);
  const float scale = t > 0.f ? 1.f / saved[1] : 0.f, log_s = t > 0.f ? logf(saved[1]) : 0.f;
  const float back = t > 0.f ? 1.f / t : 0.f;
  const float h = a.grad_entropy ? a.grad_entropy[row] : 0.f;
  float sum = 0.f;
  for (int k = threadIdx.x % 64; k < a.K; k += 64)
    if (saved[4 + k] == saved[4 + k]) sum += gk[k];
  sum = wave_sum(sum);
  const float plus = saved[2] - log_s, from = fmaxf(m, kLowest);
  // without the tokens' own terms
  auto slope = [&](float x) {
    float d = exponent(x, from, c);
    if (m == INFINITY) d = x == INFINITY ? 0.f : -1e4f;
    const float p = __builtin_amdgcn_exp2f(d) * scale;
    return -p * fmaf(h, fmaf(d, kLn2, plus), sum);
  };
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int64_t col = first + (int64_t)(j * kThreads + threadIdx.x) * 8;
    T o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (T)(slope(v[j][e]) * back);
    if (col + 8 <= a.D) {
      store_vec(out + col, o);
    } else {
      for (int e = 0; e < 8; ++e)
        if (col + e < a.D) out[col + e] = o[e];
    }
  }
  if (!a.K) return;
  __syncthreads();
  for (int k = threadIdx.x; k < a.K; k += kThreads) {
    const int token = tokens[k];
    const float own = saved[4 + k];
    if (token < first || token >= first + (int64_t)kPass * N || own != own) continue;
    bool named = false;
    for (int j = 0; j < k; ++j) named |= tokens[j] == token;
    if (named) continue;  // the first of equal ones adds all of them, in order
    float g = 0.f;
    for (int j = k; j < a.K; ++j)
      if (tokens[j] == token) g += gk[j];
    out[token] = (T)((slope(own) + g) * back);
  }
}

int passes_of(int64_t rows, int32_t D) { return rows * D >= (int64_t)2048 * 4 * kPass ? 4 : 1; }
int chunks_of(int passes, int32_t D) { return (int)(((int64_t)D + passes * kPass - 1) / (passes * kPass)); }
int segments_of(int32_t D) { return (int)(((int64_t)D + kSegment - 1) / kSegment); }
// rows that one pair of launches takes, and whose workspace there is
int batch_of(int32_t m, int32_t D) {
  return (int)std::min<int64_t>(m, std::max<int64_t>(1, std::min(kMostBlocks / chunks_of(1, D),
                                                                kMostEntries / D)));
}

bool good_sizes(int32_t m, int32_t D, int32_t K, int32_t top) {
  return m >= 0 && D >= 1 && D <= kMostEntries && K >= 0 && K <= kMostTokens && top >= 0 &&
         top <= kMostTop;
}

}  // namespace
}  // namespace lst

using namespace lst;

extern "C" {

int64_t lst_logprobs_workspace(int32_t m, int32_t D, int32_t top) {
  if (!good_sizes(m, D, 0, top)) return -1;
  if (D <= kShort || m == 0) return 0;
  const int64_t rows = batch_of(m, D);
  return rows * (chunks_of(1, D) * (int64_t)sizeof(float4) +
                 (top ? segments_of(D) * (int64_t)sizeof(float) : 0));
}

int64_t lst_logprobs_saved(int32_t m, int32_t K) {
  if (m < 0 || K < 0 || K > kMostTokens) return -1;
  return (int64_t)m * (K + 4);
}

int lst_logprobs(int32_t dtype, int32_t m, int32_t D, int32_t K, int32_t top, const void* logits,
                 int64_t ldx, const float* temperature, const int32_t* tokens, float* logp,
                 float* entropy, int32_t* top_ids, float* top_logp, float* saved, void* workspace,
                 int32_t* status, void* hip_stream) {
  if (!known_dtype(dtype) || !good_sizes(m, D, K, top)) return LST_EINVAL;
  if (m == 0) return LST_OK;
  if (!logits || ldx < D || (K && (!tokens || !logp)) || (top && (!top_ids || !top_logp)))
    return LST_EINVAL;
  if (D > kShort && (!workspace || ((uintptr_t)workspace & 15))) return LST_EINVAL;
  hipStream_t s = (hipStream_t)hip_stream;
  Args a{ldx, D, K, top, 0, segments_of(D), 0, temperature, tokens, logp, entropy, saved,
         top_ids, top_logp, status, nullptr, nullptr};
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    const T* x = (const T*)logits;
    const int64_t batch = D <= kShort ? kMostBlocks / 2 : batch_of(m, D);
    for (int64_t r = 0; r < m; r += batch) {
      const int n = (int)std::min<int64_t>(batch, m - r);
      a.row0 = (int)r;
      if (D <= kShort) {
        hipLaunchKernelGGL(short_kernel<T>, dim3(n), dim3(512), 0, s, a, x);
        continue;
      }
      const int passes = passes_of(n, D);
      a.chunks = chunks_of(passes, D);
      a.partial = (float4*)workspace;
      a.largest = (float*)(a.partial + (int64_t)n * a.chunks);
      if (passes == 1)
        hipLaunchKernelGGL((stats_kernel<T, 1>), dim3(n * a.chunks), dim3(kThreads), 0, s, a, x);
      else
        hipLaunchKernelGGL((stats_kernel<T, 4>), dim3(n * a.chunks), dim3(kThreads), 0, s, a, x);
      hipLaunchKernelGGL(join_kernel<T>, dim3(n), dim3(512), 0, s, a, x);
    }
    return launched();
  });
}

int lst_logprobs_backward(int32_t dtype, int32_t m, int32_t D, int32_t K, const void* logits,
                          int64_t ldx, const float* temperature, const int32_t* tokens,
                          const float* saved, const float* grad_logp, const float* grad_entropy,
                          void* grad_logits, int64_t ldg, void* hip_stream) {
  if (!known_dtype(dtype) || !good_sizes(m, D, K, 0)) return LST_EINVAL;
  if (m == 0) return LST_OK;
  if (!logits || ldx < D || !saved || !grad_logits || ldg < D || (K && (!tokens || !grad_logp)))
    return LST_EINVAL;
  if (logits == grad_logits && ldx != ldg) return LST_EINVAL;
  BackArgs a{ldx, ldg, D, K, 0, 0, temperature, tokens, saved, grad_logp, grad_entropy};
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    const int64_t batch = batch_of(m, D);
    for (int64_t r = 0; r < m; r += batch) {
      const int n = (int)std::min<int64_t>(batch, m - r), passes = passes_of(n, D);
      a.row0 = (int)r;
      a.chunks = chunks_of(passes, D);
      auto run = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(n * a.chunks), dim3(kThreads), 0,
                           (hipStream_t)hip_stream, a, (const T*)logits, (T*)grad_logits);
      };
      passes == 1 ? run(backward_kernel<T, 1>) : run(backward_kernel<T, 4>);
    }
    return launched();
  });
}

}  // extern "C"
