// A gated linear recurrence over packed sequences (lst_recur_forward, _backward
// and _step):
//
//   f_t = sigmoid(g_t),   h_t = f_t h_{t-1} + (1 - f_t) x_t,   y_t = h_t
//
// for each channel by itself.  With L_t = dL/dh_t (all of it, the later rows'
// included) the gradients are
//
//   L_t = dL/dy_t + f_{t+1} L_{t+1}    (+ the gradient of the last state at the end)
//   dL/dx_t = (1 - f_t) L_t,   dL/dg_t = (h_{t-1} - x_t) f_t (1 - f_t) L_t,
//   dL/dh_{-1} = f_0 L_0.
//
// f and 1 - f are both formed from exp(-|g|): neither loses its digits where the
// gate saturates.  States, gates and sums are float32.
//
// Both passes read each row once.  The packed rows are cut into chunks of 128,
// whatever sequences they hold, and a block has one chunk of 64 or 128 channels:
// waves of 16 rows (8 of two channels a lane in the backward pass), held in registers.
// A row's map h -> f h + (1 - f) x, and so every stretch of rows, is a pair (A, B) with
// h -> A h + B.  The block publishes the pair of its chunk, gathers those of the chunks
// before it, back to the one in which the sequence of its first row begins, and only then
// runs over its rows: the one-pass scan with look-back of Merrill and Garland ("Single-pass
// parallel prefix scan with decoupled look-back", 2016), on pairs and by whole sequences.
//
//  - Blocks take their chunks by a ticket, so the chunks that a block waits for have
//    blocks that run already, and a block publishes before it waits: no wait is
//    without end.
//  - A pair is one 64-bit word, written and read by one atomic access, and no fence is
//    needed; the workspace starts out as words that no pair has.
//  - Every sixteenth block publishes the pair of its sixteen chunks too, so a block
//    reads at most 31 pairs and one for each sixteen chunks farther back (one sequence of
//    1 048 576 rows of 64 floats takes 285 us forward, of 4 194 304 1860; as sequences of
//    1024 rows 193 and 694).  Which pairs it reads and how it joins them depends on the
//    chunk alone: the result does not depend on which block was faster.
//  - The first row of a sequence forgets what comes in.  Its pair has A = -0, which no
//    product of gates has (they are not negative): h -> B then, also where h is no
//    number.  (A product of small gates may be 0, and 0 times an infinite state no number,
//    where row after row it would stay infinite: it is not finite either way.)
//
// The backward pass runs the same way from the last chunk to the first on
// (f L)_t = f_t (dL/dy_t + (f L)_{t+1}), and computes the states within a chunk again
// from the state before it, which the forward pass saves.
//
// Measured at 65 536 rows of 512 floats (two sequences): 111 us forward (403 MB) and
// 155 us backward (671 MB), together 4.0 TB/s, where a copy of 1 GiB reaches 5.1; without
// the waits the forward pass takes 94 us.  What counts is bytes in flight: with 133
// registers (one block a compute unit) instead of 105 the backward pass took 248 us, and
// with gates computed again in each phase instead of held 179.  8191 rows of 500 bfloat16
// in 311 sequences are 256 blocks, one a compute unit: 17 and 22 us, a block's own latency.
#include <algorithm>

#include "dtypes.h"

namespace lst {
namespace {

constexpr int kChunk = LST_RECUR_CHUNK;

struct RecurArgs {
  int rows, n_seq, d;
  int64_t ldx, ldg, ldy, lddx, lddg;
  const int32_t* offsets;
  const float *h0, *grad_last, *saved_in;
  float *h_last, *saved, *grad_h0;
  int32_t* status;
};

// exp(-|g|), whose relative error is that of f or 1 - f, whichever is smaller: to float32's
// digits for all types, since the states are float32.  A product m log2(e) that is rounded would
// cost |m| 2^-24.  The first 24 bits less a 16-bit type's own (8, 11) of log2(e) make one that is
// exact, 2^(m hi), and the rest is exp(q) with q = m (1 - hi ln 2): at least -5e-4 and -5e-3
// where the result is a normal number, so that one term and two are enough.
template <class T>
__device__ inline float exp_of(float m) {
  constexpr bool bf16 = std::is_same_v<T, __bf16>;
  const float kHi = bf16 ? 47274.f / 32768 : 5909.f / 4096;
  const float kRest = bf16 ? 4.8884953e-06f : 4.719484e-05f;
  const float q = fmaxf(m * kRest, -0.01f);  // finite for m = -inf
  const float e = __builtin_amdgcn_exp2f(m * kHi);
  return fmaf(e, bf16 ? q : q * fmaf(q, 0.5f, 1.f), e);
}

// 2^t (1 + r ln 2) with m log2(e) = t + r, r the product's rounding
template <>
__device__ inline float exp_of<float>(float m) {
  const float kLog2e = 1.44269504f, kLog2eLow = 1.925963033e-8f, kLn2 = 0.693147181f;
  const float t = m * kLog2e, r = fmaf(m, kLog2eLow, fmaf(m, kLog2e, -t));
  const float e = __builtin_amdgcn_exp2f(t);
  return m < -150.f ? 0.f : fmaf(e, r * kLn2, e);  // -inf: t + r is not a number
}

template <class T>
__device__ inline void gate(float g, float& f, float& i) {
  const float e = exp_of<T>(-fabsf(g));
  const float big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
  f = g < 0.f ? small : big;
  i = g < 0.f ? big : small;
}

__device__ inline void raise(int32_t* status) {
  if (status) atomicCAS(status, 0, LST_EINDEX);
}

// The wave's number, known to be the same for all of its lanes: row addresses stay in scalar
// registers.
__device__ inline int wave_of() { return __builtin_amdgcn_readfirstlane(threadIdx.x / 64); }

// -------------------------------------------------------------- pairs (A, B)
struct Pair {
  float a, b;
};

__device__ inline bool forgets(float a) { return __float_as_uint(a) == 0x80000000u; }
__device__ inline float through(Pair p, float h) { return forgets(p.a) ? p.b : fmaf(p.a, h, p.b); }
// first p, then q
__device__ inline Pair join(Pair p, Pair q) {
  return {forgets(q.a) ? q.a : q.a * p.a, through(q, p.b)};
}

constexpr unsigned long long kNone = ~0ull;  // A: a number that pack() does not leave

__device__ inline unsigned long long pack(Pair p) {
  const float a = p.a == p.a ? p.a : __uint_as_float(0x7FC00000u);
  return (unsigned long long)__float_as_uint(a) << 32 | __float_as_uint(p.b);
}

__device__ inline Pair unpack(unsigned long long v) {
  return {__uint_as_float((uint32_t)(v >> 32)), __uint_as_float((uint32_t)v)};
}

// ------------------------------------------------------------- the workspace
constexpr int kGroupChunks = 16;             // chunks whose pair is published together
constexpr int kHead = 64;                    // bytes before the words: the ticket
constexpr int kPolls = 1 << 22;              // several seconds: never reached
constexpr int kMost = 1 << 30;               // rows, sequences: with a block's step below 2^31
constexpr int kMostSlots = 1 << 16;          // of a step: each is compared with those before it

struct Shape {
  int chunks, tiles, width;  // width: channels of all tiles
  int groups;
  bool joined() const { return chunks > 1; }
  int64_t words() const { return joined() ? (int64_t)(chunks + groups) * width : 0; }
};

Shape shape_of(int rows, int d, int vec) {
  Shape s;
  s.chunks = rows ? (int)(((int64_t)rows + kChunk - 1) / kChunk) : 1;
  s.tiles = (d + 64 * vec - 1) / (64 * vec);
  s.width = s.tiles * 64 * vec;
  s.groups = s.chunks / kGroupChunks;
  return s;
}

__global__ __launch_bounds__(256) void recur_clear_kernel(unsigned long long* words, int64_t n,
                                                          unsigned* ticket) {
  int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i == 0) *ticket = 0;
  for (; i < n; i += (int64_t)gridDim.x * 256) words[i] = kNone;
}

struct Workspace {
  unsigned* ticket;
  unsigned long long *chunk, *group;  // pairs, width words each
};

// ------------------------------------------------- what a block knows of its rows
// VEC: channels a lane, ROWS: rows a wave.
template <int VEC, int ROWS>
struct Block {
  static constexpr int kWaves = kChunk / ROWS, kThreads = 64 * kWaves;
  float2 own[kWaves][64 * VEC];   // the waves' pairs
  float2 far[kWaves][64 * VEC];   // of the chunks before: groups (first half), chunks
  int start[kChunk], end[kChunk];  // 1 + the sequence whose first (last) row it is, or 0
  int ticket;
  int s0;     // first sequence that ends behind the first row
  int reach;  // first row (forward) or last row (backward) of the sequence that goes on
};

// A thread's pair of offsets where there are no more sequences than threads, asked for before
// the rows are: what is asked for later arrives later.
struct Early {
  int b, e;
  __device__ Early(const RecurArgs& a, int threads) : b(0x7FFFFFFF), e(0) {
    if (a.offsets && a.n_seq <= threads && (int)threadIdx.x < a.n_seq) {
      b = a.offsets[threadIdx.x];
      e = a.offsets[threadIdx.x + 1];
    }
  }
};

// The sequences' borders among rows [r0, r1) of the chunk, and how far the sequence
// that enters the chunk (forward: at its first row, else at its last) reaches.
template <bool FORWARD, int VEC, int ROWS>
__device__ void find_borders(Block<VEC, ROWS>& sh, const RecurArgs& a, Early early, int r0,
                             int r1) {
  constexpr int kThreads = Block<VEC, ROWS>::kThreads;
  const int tid = threadIdx.x, n = a.n_seq;
  if (tid < kChunk) sh.start[tid] = sh.end[tid] = 0;
  const int enter = FORWARD ? r0 : r1 - 1;
  if (tid == 0) sh.reach = enter;
  auto mark = [&](int s, int b, int e) {
    if (b < 0 || b >= e || e > a.rows) return;
    if (b >= r0 && b < r1) sh.start[b - r0] = s + 1;
    if (e > r0 && e <= r1) sh.end[e - 1 - r0] = s + 1;
    if (b <= enter && enter < e) sh.reach = FORWARD ? b : e - 1;
  };
  if (!a.offsets) {
    const int len = a.rows / n;
    __syncthreads();
    if (len && tid < kChunk && r0 + tid < r1) {
      const int s = (r0 + tid) / len;
      if (tid == 0 || (r0 + tid) % len == 0) mark(s, s * len, s * len + len);
    }
    __syncthreads();
    return;
  }
  if (n <= kThreads) {
    __syncthreads();
    mark(tid, early.b, early.e);
    __syncthreads();
    return;
  }
  // the first sequence that ends behind r0, by kThreads probes at a time
  int lo = 0, hi = n;
  while (hi - lo > kThreads) {
    const int64_t step = ((int64_t)hi - lo + kThreads - 1) / kThreads;
    if (tid == 0) sh.s0 = kThreads;
    __syncthreads();
    if (a.offsets[min(lo + (tid + 1) * step, (int64_t)hi)] > r0) atomicMin(&sh.s0, tid);
    __syncthreads();
    const int t = sh.s0;
    __syncthreads();
    const int64_t from = t == kThreads ? hi : lo + t * step;
    hi = (int)min(from + step - 1, (int64_t)hi);
    lo = (int)min(from, (int64_t)hi);
  }
  __syncthreads();
  for (int base = lo; base < n; base += kThreads) {
    const int s = base + tid;
    const int b = s < n ? a.offsets[s] : 0x7FFFFFFF;
    if (s < n) mark(s, b, a.offsets[s + 1]);
    if (__syncthreads_or(s >= n || b >= r1)) break;
  }
  __syncthreads();
}

// The sequences without rows among this chunk's share of all of them: to <- from (zeros); and
// the status, once for every pair of offsets that is none.
template <int VEC, int ROWS>
__device__ void empty_sequences(const RecurArgs& a, int chunk, int chunks, int c, bool on,
                                const float* from, float* to, bool check) {
  const int64_t n = a.n_seq;
  const int s0 = (int)(n * chunk / chunks), s1 = (int)(n * (chunk + 1) / chunks);
  for (int s = s0 + wave_of(); s < s1; s += kChunk / ROWS) {
    int b = 0, e = 0;
    if (a.offsets) {
      b = a.offsets[s];
      e = a.offsets[s + 1];
    } else {
      e = a.rows / a.n_seq;
    }
    if (check && (b < 0 || b > e || e > a.rows)) raise(a.status);
    if (b == e && to && on)
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        to[(int64_t)s * a.d + c + v] = from ? from[(int64_t)s * a.d + c + v] : 0.f;
  }
}

// The pairs [from, to) of `words` joined, first to last; lane l's VEC channels are at `at`.
template <int VEC>
__device__ void gather(const unsigned long long* words, int64_t width, int64_t at, int from,
                       int to, Pair (&out)[VEC], int32_t* status) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) out[v] = {1.f, 0.f};
  constexpr int kAhead = 4;  // words under way together
  for (int i0 = from; i0 < to; i0 += kAhead) {
    unsigned long long w[kAhead][VEC];
    for (int poll = 0;; ++poll) {
      bool have = true;
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = min(i0 + j, to - 1);
#pragma unroll
        for (int v = 0; v < VEC; ++v)
          w[j][v] = __hip_atomic_load(words + i * width + at + v, __ATOMIC_RELAXED,
                                      __HIP_MEMORY_SCOPE_AGENT);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
#pragma unroll
        for (int v = 0; v < VEC; ++v) have &= w[j][v] != kNone;
      if (__all(have)) break;
      if (poll == kPolls) {
        if (status) atomicCAS(status, 0, LST_EHIP);
        break;
      }
      __builtin_amdgcn_s_sleep(1);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (i0 + j < to)
#pragma unroll
        for (int v = 0; v < VEC; ++v) out[v] = join(out[v], unpack(w[j][v]));
  }
}

// What comes into the chunk.  j counts chunks in the direction of the scan, j0 is the
// one in which the sequence that comes in begins; the waves' pairs are in sh.own,
// ORDER(w) the w-th of them in that direction.  Publishes the chunk's pair, and the
// group's where it is complete.
template <int VEC, int ROWS, class Order>
__device__ void come_in(Block<VEC, ROWS>& sh, const Shape& z, Workspace ws, int j, int j0,
                        int64_t at, Order order, float (&carry)[VEC], int32_t* status) {
  constexpr int kWaves = Block<VEC, ROWS>::kWaves;
  const int w = wave_of(), l = threadIdx.x % 64;
#pragma unroll
  for (int v = 0; v < VEC; ++v) carry[v] = 0.f;
  if (z.chunks == 1) return;
  if (w == 0)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      Pair all{1.f, 0.f};
#pragma unroll 2
      for (int k = 0; k < kWaves; ++k) {
        const float2 p = sh.own[order(k)][l * VEC + v];
        all = join(all, {p.x, p.y});
      }
      __hip_atomic_store(ws.chunk + (int64_t)j * z.width + at + v, pack(all), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
    }
  const int group = j / kGroupChunks, g0 = group * kGroupChunks;
  if (w == 0 && j % kGroupChunks == kGroupChunks - 1 && j + 1 + kGroupChunks < z.chunks) {
    // before this block waits for other groups
    Pair all[VEC];
    gather<VEC>(ws.chunk, z.width, at, g0, j + 1, all, status);
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      __hip_atomic_store(ws.group + (int64_t)group * z.width + at + v, pack(all[v]),
                         __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (j0 >= j) return;
  // Half of the waves take the chunks of this group and the one before, half the groups
  // before those: a group's pair comes later than its chunks', and by then it is there.
  constexpr int kHalf = kWaves / 2;
  const int n0 = max(g0 - kGroupChunks, 0);  // the first chunk taken by itself
  const bool near = w >= kHalf;
  const int first = near ? max(n0, j0) : j0 / kGroupChunks;
  const int last = near ? j : n0 / kGroupChunks;
  const int per = (max(last - first, 0) + kHalf - 1) / kHalf;
  const int from = first + (w % kHalf) * per, to = min(last, from + per);
  Pair p[VEC];
  const unsigned long long *chunk = ws.chunk, *far = ws.group;
  gather<VEC>(near ? chunk : far, z.width, at, from, to, p, status);
#pragma unroll
  for (int v = 0; v < VEC; ++v) sh.far[w][l * VEC + v] = make_float2(p[v].a, p[v].b);
  __syncthreads();
#pragma unroll
  for (int v = 0; v < VEC; ++v)
#pragma unroll 2
    for (int k = 0; k < kWaves; ++k) {
      const float2 q = sh.far[k][l * VEC + v];
      carry[v] = through({q.x, q.y}, carry[v]);
    }
}

// A lane's VEC elements of a row in one register: two of 16 bits, or one.
template <class T, int VEC>
__device__ inline uint32_t load_word(const T* p) {
  if constexpr (sizeof(T) == 4) return __float_as_uint(*p);
  if constexpr (VEC == 1) return *reinterpret_cast<const uint16_t*>(p);
  typedef uint32_t word __attribute__((aligned(2)));
  return *reinterpret_cast<const word*>(p);
}

template <class T>
__device__ inline float part(uint32_t w, int v) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(w);
  if constexpr (std::is_same_v<T, __bf16>)
    return __uint_as_float(v ? w & 0xFFFF0000u : w << 16);
  else
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(v ? w >> 16 : w));
}

template <class T, int VEC, int ROWS>
__device__ inline void load_rows(const T* p, int64_t ld, int r, int rows, int c,
                                 uint32_t (&w)[ROWS]) {
#pragma unroll
  for (int t = 0; t < ROWS; ++t)
    w[t] = load_word<T, VEC>(p + (int64_t)min(r + t, rows - 1) * ld + (uint32_t)c);
}

// The borders among a wave's rows.
template <int ROWS>
struct Borders {
  uint32_t start, end;  // a bit a row
  int seq;              // lane t: 1 + the sequence that starts in row t, lane ROWS + t: that ends
  int first, last;      // rows [first, last) belong to sequences,
  bool whole;           // all of the wave's among them

  __device__ bool holds(int row) const { return whole || (row >= first && row < last); }
  __device__ int starts(int t) const { return __builtin_amdgcn_readlane(seq, t) - 1; }
  __device__ int ends(int t) const { return __builtin_amdgcn_readlane(seq, ROWS + t) - 1; }
};

template <int VEC, int ROWS>
__device__ inline Borders<ROWS> borders_of(const Block<VEC, ROWS>& sh, const RecurArgs& a, int w,
                                           int r, int r1) {
  const int l = threadIdx.x % 64;
  Borders<ROWS> b;
  b.seq = l < ROWS ? sh.start[w * ROWS + l] : l < 2 * ROWS ? sh.end[w * ROWS + l - ROWS] : 0;
  const uint64_t any = __ballot(b.seq != 0);
  b.start = (uint32_t)any & ((1u << ROWS) - 1);
  b.end = (uint32_t)(any >> ROWS);
  b.first = a.offsets ? a.offsets[0] : 0;
  b.last = min(a.offsets ? a.offsets[a.n_seq] : a.rows, r1);
  b.whole = r >= b.first && r + ROWS <= b.last;
  return b;
}

// n_seq x d floats (null: zeros), one row of them for each bit of `mask`: the states that the
// wave's sequences start from (END: the gradients that they end with).  The first and the
// last one are loaded ahead: a wave has rarely more, and those between belong to sequences
// that begin and end among the wave's own rows (so that one buffer for the states at both
// ends is read before it is written).
template <int VEC, int ROWS, bool END>
struct States {
  const float* p;
  int64_t d;
  uint32_t mask;
  float first[VEC], last[VEC];

  __device__ void load(const Borders<ROWS>& b, int t, float (&out)[VEC]) const {
    const float* q = p + (int64_t)(END ? b.ends(t) : b.starts(t)) * d;
#pragma unroll
    for (int v = 0; v < VEC; ++v) out[v] = p ? q[v] : 0.f;
  }
  __device__ States(const float* p_, int64_t d_, const Borders<ROWS>& b, int c, bool on)
      : p(on && p_ ? p_ + c : nullptr), d(d_), mask(END ? b.end : b.start) {
    if (!mask) return;
    load(b, __builtin_ctz(mask), first);
    if (mask & (mask - 1)) load(b, 31 - __builtin_clz(mask), last);
  }
  // h becomes, in a row of the mask, what stands for it
  __device__ void replace(const Borders<ROWS>& b, int t, float (&h)[VEC]) const {
    const uint32_t bit = 1u << t;
    if (!(mask & bit)) return;
    if (!(mask & (bit - 1))) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) h[v] = first[v];
    } else if (mask < 2 * bit) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) h[v] = last[v];
    } else {
      load(b, t, h);
    }
  }
};

// 16 rows a wave, their gates in registers from the first use to the last.
template <class T, int VEC, int ROWS>
__global__ __launch_bounds__(64 * kChunk / ROWS) void recur_forward_kernel(
    RecurArgs a, Shape z, Workspace ws, const T* x, const T* g, T* y) {
  __shared__ Block<VEC, ROWS> sh;
  const int w = wave_of(), l = threadIdx.x % 64;
  if (threadIdx.x == 0) sh.ticket = z.chunks > 1 ? (int)atomicAdd(ws.ticket, 1u) : blockIdx.x;
  __syncthreads();
  const int ticket = __builtin_amdgcn_readfirstlane(sh.ticket);
  const int j = ticket / z.tiles, tile = ticket % z.tiles;
  const int r0 = j * kChunk, r1 = min(a.rows, r0 + kChunk), r = r0 + w * ROWS;
  const int c = (tile * 64 + l) * VEC;
  const bool on = c < a.d;
  if (a.rows == 0) {
    empty_sequences<VEC, ROWS>(a, j, z.chunks, c, on, a.h0, a.h_last, tile == 0);
    return;
  }
  const Early early(a, blockDim.x);
  uint32_t rx[ROWS], rg[ROWS];
  load_rows<T, VEC, ROWS>(x, a.ldx, r, a.rows, on ? c : 0, rx);
  load_rows<T, VEC, ROWS>(g, a.ldg, r, a.rows, on ? c : 0, rg);
  find_borders<true>(sh, a, early, r0, r1);
  const Borders<ROWS> b = borders_of(sh, a, w, r, r1);
  const States<VEC, ROWS, false> first(a.h0, a.d, b, c, on);
  float f[ROWS][VEC], in[ROWS][VEC];
#pragma unroll
  for (int t = 0; t < ROWS; ++t)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float i;
      gate<T>(part<T>(rg[t], v), f[t][v], i);
      in[t][v] = i * part<T>(rx[t], v);
      asm volatile("" : "+v"(f[t][v]), "+v"(in[t][v]));  // these two, not what made them
    }
  float h[VEC], prod[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) h[v] = 0.f, prod[v] = 1.f;
#pragma unroll
  for (int t = 0; t < ROWS; ++t) {
    first.replace(b, t, h);
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      h[v] = fmaf(f[t][v], h[v], in[t][v]);
      prod[v] *= f[t][v];
    }
  }
#pragma unroll
  for (int v = 0; v < VEC; ++v)
    sh.own[w][l * VEC + v] = make_float2(b.start ? -0.f : prod[v], h[v]);
  __syncthreads();
  come_in(sh, z, ws, j, sh.reach / kChunk, c, [](int k) { return k; }, h, a.status);
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    if (w == 0 && a.saved && on) a.saved[(int64_t)j * a.d + c + v] = h[v];
#pragma unroll 2
    for (int k = 0; k < w; ++k) {
      const float2 p = sh.own[k][l * VEC + v];
      h[v] = through({p.x, p.y}, h[v]);
    }
  }
#pragma unroll
  for (int t = 0; t < ROWS; ++t) {
    first.replace(b, t, h);
    T out[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      h[v] = fmaf(f[t][v], h[v], in[t][v]);
      out[v] = (T)h[v];
    }
    if (on && b.holds(r + t)) store_vec(y + (int64_t)(r + t) * a.ldy + (uint32_t)c, out);
    if ((b.end >> t & 1) && a.h_last && on)
#pragma unroll
      for (int v = 0; v < VEC; ++v) a.h_last[(int64_t)b.ends(t) * a.d + c + v] = h[v];
  }
  empty_sequences<VEC, ROWS>(a, j, z.chunks, c, on, a.h0, a.h_last, tile == 0);
}

template <class T, int VEC, int ROWS>
__global__ __launch_bounds__(64 * kChunk / ROWS) void recur_backward_kernel(
    RecurArgs a, Shape z, Workspace ws, const T* x, const T* g, const T* dy, T* dx, T* dg) {
  __shared__ Block<VEC, ROWS> sh;
  constexpr int kWaves = Block<VEC, ROWS>::kWaves;
  const int w = wave_of(), l = threadIdx.x % 64;
  if (threadIdx.x == 0) sh.ticket = z.chunks > 1 ? (int)atomicAdd(ws.ticket, 1u) : blockIdx.x;
  __syncthreads();
  const int ticket = __builtin_amdgcn_readfirstlane(sh.ticket);
  // from the last chunk to the first
  const int j = ticket / z.tiles, tile = ticket % z.tiles, chunk = z.chunks - 1 - j;
  const int r0 = chunk * kChunk, r1 = min(a.rows, r0 + kChunk), r = r0 + w * ROWS;
  const int c = (tile * 64 + l) * VEC;
  const bool on = c < a.d;
  if (a.rows == 0) {
    empty_sequences<VEC, ROWS>(a, chunk, z.chunks, c, on, a.grad_last, a.grad_h0, tile == 0);
    return;
  }
  const Early early(a, blockDim.x);
  uint32_t rx[ROWS], rg[ROWS], ry[ROWS];
  load_rows<T, VEC, ROWS>(x, a.ldx, r, a.rows, on ? c : 0, rx);
  load_rows<T, VEC, ROWS>(g, a.ldg, r, a.rows, on ? c : 0, rg);
  load_rows<T, VEC, ROWS>(dy, a.ldy, r, a.rows, on ? c : 0, ry);
  float before[VEC];  // the state before the chunk
#pragma unroll
  for (int v = 0; v < VEC; ++v) before[v] = on ? a.saved_in[(int64_t)chunk * a.d + c + v] : 0.f;
  find_borders<false>(sh, a, early, r0, r1);
  const Borders<ROWS> b = borders_of(sh, a, w, r, r1);
  const States<VEC, ROWS, false> first(a.h0, a.d, b, c, on);
  const States<VEC, ROWS, true> last(a.grad_last, a.d, b, c, on);
  float f[ROWS][VEC], i[ROWS][VEC];
#pragma unroll
  for (int t = 0; t < ROWS; ++t)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      gate<T>(part<T>(rg[t], v), f[t][v], i[t][v]);
      asm volatile("" : "+v"(f[t][v]), "+v"(i[t][v]));
    }
  // the states before the waves' rows
  float h[VEC], prod[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) h[v] = 0.f, prod[v] = 1.f;
#pragma unroll
  for (int t = 0; t < ROWS; ++t) {
    first.replace(b, t, h);
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      h[v] = fmaf(f[t][v], h[v], i[t][v] * part<T>(rx[t], v));
      prod[v] *= f[t][v];
    }
  }
#pragma unroll
  for (int v = 0; v < VEC; ++v)
    sh.own[w][l * VEC + v] = make_float2(b.start ? -0.f : prod[v], h[v]);
  __syncthreads();
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    h[v] = before[v];
#pragma unroll 2
    for (int k = 0; k < w; ++k) {
      const float2 p = sh.own[k][l * VEC + v];
      h[v] = through({p.x, p.y}, h[v]);
    }
  }
  __syncthreads();
  // what the gates' gradients are of L
  float of[ROWS][VEC];
#pragma unroll
  for (int t = 0; t < ROWS; ++t) {
    first.replace(b, t, h);
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const float in = part<T>(rx[t], v);
      of[t][v] = (h[v] - in) * (f[t][v] * i[t][v]);
      asm volatile("" : "+v"(of[t][v]));  // the product, not its three factors
      h[v] = fmaf(f[t][v], h[v], i[t][v] * in);
    }
  }
  // the waves' pairs from the end
  float m[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) m[v] = 0.f;
#pragma unroll
  for (int t = ROWS - 1; t >= 0; --t) {
    last.replace(b, t, m);
#pragma unroll
    for (int v = 0; v < VEC; ++v) m[v] = f[t][v] * (part<T>(ry[t], v) + m[v]);
  }
#pragma unroll
  for (int v = 0; v < VEC; ++v)
    sh.own[w][l * VEC + v] = make_float2(b.end ? -0.f : prod[v], m[v]);
  __syncthreads();
  come_in(sh, z, ws, j, z.chunks - 1 - sh.reach / kChunk, c,
          [](int k) { return kWaves - 1 - k; }, m, a.status);
#pragma unroll
  for (int v = 0; v < VEC; ++v)
#pragma unroll 2
    for (int k = kWaves - 1; k > w; --k) {
      const float2 p = sh.own[k][l * VEC + v];
      m[v] = through({p.x, p.y}, m[v]);
    }
#pragma unroll
  for (int t = ROWS - 1; t >= 0; --t) {
    last.replace(b, t, m);
    T ox[VEC], og[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const float L = part<T>(ry[t], v) + m[v];
      ox[v] = (T)(i[t][v] * L);
      og[v] = (T)(of[t][v] * L);
      m[v] = f[t][v] * L;
    }
    if (on && b.holds(r + t)) {
      store_vec(dx + (int64_t)(r + t) * a.lddx + (uint32_t)c, ox);
      store_vec(dg + (int64_t)(r + t) * a.lddg + (uint32_t)c, og);
    }
    if ((b.start >> t & 1) && a.grad_h0 && on)
#pragma unroll
      for (int v = 0; v < VEC; ++v) a.grad_h0[(int64_t)b.starts(t) * a.d + c + v] = m[v];
  }
  empty_sequences<VEC, ROWS>(a, chunk, z.chunks, c, on, a.grad_last, a.grad_h0, tile == 0);
}

template <class T>
__global__ __launch_bounds__(256) void recur_step_kernel(int n_slots, int d, const T* x,
                                                         int64_t ldx, const T* g, int64_t ldg,
                                                         const int32_t* slots, float* h, T* y,
                                                         int64_t ldy, int32_t* status) {
  const int64_t row = blockIdx.x;
  const int slot = slots ? slots[row] : (int)row;
  // a slot that an earlier row names already: that row has it
  bool twice = false;
  if (slots)
    for (int j = threadIdx.x; j < row; j += 256) twice |= slots[j] == slot;
  if (__syncthreads_or(twice && slot >= 0) || slot < -1 || slot >= n_slots) {
    if (threadIdx.x == 0) raise(status);
    return;
  }
  if (slot < 0) return;
  for (int c = threadIdx.x; c < d; c += 256) {
    float f, i;
    gate<T>((float)g[row * ldg + c], f, i);
    float* p = h + (int64_t)slot * d + c;
    const float v = f * *p + i * (float)x[row * ldx + c];
    *p = v;
    y[row * ldy + c] = (T)v;
  }
}

int check_recur(int dtype, int rows, int n_seq, int d, const void* x, int64_t ldx, const void* g,
                int64_t ldg, const int32_t* offsets) {
  if (!known_dtype(dtype) || rows < 0 || n_seq < 0 || d < 1 || d > 4096) return LST_EINVAL;
  if (rows > kMost || n_seq > kMost) return LST_EINVAL;
  if (n_seq == 0 && rows != 0 && !offsets) return LST_EINVAL;
  if (!offsets && n_seq && rows % n_seq) return LST_EINVAL;
  if (rows && (!x || !g || ldx < d || ldg < d)) return LST_EINVAL;
  return LST_OK;
}

// A launch has fewer than 2^32 threads, and blocks take their chunks by a ticket that goes on
// from one launch to the next: a pass of more threads comes in several launches.
template <class F>
void in_launches(int64_t blocks, int threads, F launch) {
  const int64_t most = 0xFFFFFFFFu / threads;
  for (; blocks > 0; blocks -= most) launch(dim3((unsigned)std::min(blocks, most)), dim3(threads));
}

// Calls run with the element type, the channels a lane, the shape and the workspace, cleared.
template <class F>
int with_shape(int dtype, int rows, int d, void* workspace, hipStream_t stream, F run) {
  return with_dtype(dtype, [&](auto t) {
    auto go = [&](auto vec) {
      const Shape z = shape_of(rows, d, decltype(vec)::value);
      if ((int64_t)z.chunks * z.tiles > 0x7FFFFFFF) return (int)LST_EINVAL;
      Workspace ws{};
      if (z.joined()) {
        if (!workspace || ((uintptr_t)workspace & 15)) return (int)LST_EINVAL;
        ws.ticket = (unsigned*)workspace;
        ws.chunk = (unsigned long long*)((char*)workspace + kHead);
        ws.group = ws.chunk + (int64_t)z.chunks * z.width;
        const int64_t blocks = std::min<int64_t>((z.words() + 255) / 256, 1 << 22);
        hipLaunchKernelGGL(recur_clear_kernel, dim3((unsigned)blocks), dim3(256), 0, stream,
                           ws.chunk, z.words(), ws.ticket);
      }
      run(t, vec, z, ws);
      return launched();
    };
    // two channels a lane where they make up the 4 bytes that a lane loads
    if constexpr (sizeof(t) == 2)
      if (d % 2 == 0) return go(std::integral_constant<int, 2>{});
    return go(std::integral_constant<int, 1>{});
  });
}

}  // namespace
}  // namespace lst

using namespace lst;

extern "C" {

int64_t lst_recur_saved(int32_t rows, int32_t d) {
  return rows < 0 || rows > kMost || d < 1 || d > 4096 ? -1 : ((int64_t)rows + kChunk - 1) / kChunk * d;
}

int64_t lst_recur_workspace(int32_t rows, int32_t d) {
  if (rows < 0 || rows > kMost || d < 1 || d > 4096) return -1;
  const Shape s = shape_of(rows, d, 2);  // as wide as with one channel a lane, or wider
  return s.joined() ? kHead + s.words() * (int64_t)sizeof(unsigned long long) : 0;
}

int lst_recur_forward(int32_t dtype, int32_t rows, int32_t n_seq, int32_t d, const void* x,
                      int64_t ldx, const void* g, int64_t ldg, const int32_t* offsets,
                      const float* h0, void* y, int64_t ldy, float* h_last, float* saved,
                      void* workspace, int32_t* status, void* hip_stream) {
  int rc = check_recur(dtype, rows, n_seq, d, x, ldx, g, ldg, offsets);
  if (rc != LST_OK) return rc;
  if (rows && (!y || ldy < d)) return LST_EINVAL;
  if (n_seq == 0) return LST_OK;
  RecurArgs a{};
  a.rows = rows, a.n_seq = n_seq, a.d = d;
  a.ldx = ldx, a.ldg = ldg, a.ldy = ldy;
  a.offsets = offsets, a.h0 = h0, a.h_last = h_last, a.saved = saved, a.status = status;
  return with_shape(dtype, rows, d, workspace, (hipStream_t)hip_stream,
                    [&](auto t, auto vec, const Shape& z, const Workspace& ws) {
    using T = decltype(t);
    constexpr int VEC = decltype(vec)::value, ROWS = 16;
    in_launches((int64_t)z.chunks * z.tiles, 64 * kChunk / ROWS, [&](dim3 grid, dim3 block) {
      hipLaunchKernelGGL((recur_forward_kernel<T, VEC, ROWS>), grid, block, 0,
                         (hipStream_t)hip_stream, a, z, ws, (const T*)x, (const T*)g, (T*)y);
    });
  });
}

int lst_recur_backward(int32_t dtype, int32_t rows, int32_t n_seq, int32_t d, const void* x,
                       int64_t ldx, const void* g, int64_t ldg, const int32_t* offsets,
                       const float* h0, const void* grad_y, int64_t ldgy, const float* grad_last,
                       const float* saved, void* grad_x, int64_t ldgx, void* grad_g,
                       int64_t ldgg, float* grad_h0, void* workspace, int32_t* status,
                       void* hip_stream) {
  int rc = check_recur(dtype, rows, n_seq, d, x, ldx, g, ldg, offsets);
  if (rc != LST_OK) return rc;
  if (rows && (!grad_y || !saved || !grad_x || !grad_g || ldgy < d || ldgx < d || ldgg < d))
    return LST_EINVAL;
  if (n_seq == 0) return LST_OK;
  RecurArgs a{};
  a.rows = rows, a.n_seq = n_seq, a.d = d;
  a.ldx = ldx, a.ldg = ldg, a.ldy = ldgy, a.lddx = ldgx, a.lddg = ldgg;
  a.offsets = offsets, a.h0 = h0, a.grad_last = grad_last, a.saved_in = saved;
  a.grad_h0 = grad_h0, a.status = status;
  return with_shape(dtype, rows, d, workspace, (hipStream_t)hip_stream,
                    [&](auto t, auto vec, const Shape& z, const Workspace& ws) {
    using T = decltype(t);
    // 8 rows a wave with two channels a lane: 16 would take all registers
    constexpr int VEC = decltype(vec)::value, ROWS = 16 / VEC;
    in_launches((int64_t)z.chunks * z.tiles, 64 * kChunk / ROWS, [&](dim3 grid, dim3 block) {
      hipLaunchKernelGGL((recur_backward_kernel<T, VEC, ROWS>), grid, block, 0,
                         (hipStream_t)hip_stream, a, z, ws, (const T*)x, (const T*)g,
                         (const T*)grad_y, (T*)grad_x, (T*)grad_g);
    });
  });
}

int lst_recur_step(int32_t dtype, int32_t rows, int32_t n_slots, int32_t d, const void* x,
                   int64_t ldx, const void* g, int64_t ldg, const int32_t* slots, float* h,
                   void* y, int64_t ldy, int32_t* status, void* hip_stream) {
  if (!known_dtype(dtype) || rows < 0 || n_slots < 0 || d < 1 || d > 4096) return LST_EINVAL;
  if (slots ? rows > kMostSlots : rows > n_slots || rows > 0xFFFFFF) return LST_EINVAL;
  if (rows == 0) return LST_OK;
  if (!x || !g || !h || !y || ldx < d || ldg < d || ldy < d) return LST_EINVAL;
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(recur_step_kernel<T>, dim3(rows), dim3(256), 0, (hipStream_t)hip_stream,
                       n_slots, d, (const T*)x, ldx, (const T*)g, ldg, slots, h, (T*)y, ldy,
                       status);
    return launched();
  });
}

}  // extern "C"
