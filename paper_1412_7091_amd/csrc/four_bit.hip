// Weights in 4 bits (lst_quantize_four) and a layer's outputs from them (lst_scores_four).
//
// A row is cut into blocks of 32 columns.  A block holds e2m1 codes q (0, 1/2, 1, 3/2, 2, 3, 4, 6
// and a sign), two a byte with the lower column in the lower half, and one exponent e with 6 2^e
// the smallest such bound on the block's values.  The rows of H are quantised in the same way in
// each call:
//
//   O[i][r] = sum_b 2^(e_ib + e_rb) sum_{k in b} qh_ik qw_rk
//
// The scaled matrix instruction takes both sides as they are held: lane (n, q) of 16 x 4 gives
// the 32 columns of one block, 16 bytes, and its exponent.  Its sums of 4-bit products are those
// of float32 (measured: a product of 1/4 beside one of 36 2^40 or beside an accumulator of that
// size is rounded as float32 rounds it, where sums of 8-bit products lose what is 2^-14 of the
// largest), and it has four times the rate of the bfloat16 instruction.
#include <algorithm>

#include "eight_bit.h"
#include "gemm_tile.h"

namespace lst {
namespace {

constexpr int kSmall = 32;         // columns that share a scale
constexpr int kStep = 128;         // columns of one matrix instruction
constexpr int kPiece = 64 * 16;    // bytes of its operand: 16 rows
constexpr int kGroup = 4;          // steps whose scales share a word, and a stage of LDS

typedef int int32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Biased exponent of the scale for the bits of a block's largest magnitude: 6 = 1.5 2^2, so
// 1.f 2^E needs 2^(E - 2) when 1.f <= 1.5, else 2^(E - 1).
__device__ inline int small_scale_of(uint32_t big) {
  const int e = (int)(big >> 23) - ((big & 0x7FFFFF) <= 0x400000 ? 2 : 1);
  return max(e, 0);
}

// Codes of eight columns, a block being in four neighbouring lanes, and the block's biased
// exponent.  The type has no code that is no number: a block with a value that is not finite
// gets the exponent 255, which makes all of it no number, and codes of zero for such values.
__device__ inline uint32_t small_codes(float (&v)[8], int& e) {
  uint32_t bad, big = largest_finite(v, bad);
  int worst = bad != 0;
#pragma unroll
  for (int o = 2; o; o >>= 1) {
    big = max(big, (uint32_t)__shfl_xor((int)big, o));
    worst |= __shfl_xor(worst, o);
  }
  e = small_scale_of(big);
  const float s = __uint_as_float((uint32_t)(254 - e) << 23);  // exact: e is at most 253
  uint32_t q = 0;
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0] * s, v[1] * s, 1.f, 0);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2] * s, v[3] * s, 1.f, 1);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4] * s, v[5] * s, 1.f, 2);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6] * s, v[7] * s, 1.f, 3);
  if (worst) e = 255;
  return q;
}

template <class T>
__device__ inline uint32_t row_codes(const T* row, int col, int cols, int& e) {
  T raw[8];
  load_part(row, col, cols, raw);
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)raw[i];
  return small_codes(v, e);
}

// Four lanes a block, eight columns a lane.  Bound by memory: 793 471 x 300 floats (1.09 GB with
// the codes) take 202 us, 5.4 TB/s.
template <class T>
__global__ __launch_bounds__(256) void quantize_kernel(const T* x, int64_t ldx, int64_t rows,
                                                       int cols, int blocks, uint32_t* codes,
                                                       uint8_t* scales) {
  const unsigned at = blockIdx.x * 64 + threadIdx.x / 4;  // the block
  if (at >= (unsigned)(rows * blocks)) return;
  const unsigned row = at / (unsigned)blocks;
  const int l = threadIdx.x % 4, col = (int)(at - row * (unsigned)blocks) * kSmall + 8 * l;
  int e;
  const uint32_t q = row_codes(x + (int64_t)row * ldx, col, cols, e);
  codes[(int64_t)at * 4 + l] = q;
  if (l == 0) scales[at] = (uint8_t)e;
}

// Rows of H into operands: piece (tile of 16 rows, step), and behind the pieces the exponents of
// four steps a word, for each lane of a tile.  Rows behind the last one of the last tile and
// blocks behind a row's last are zeros.
template <class T>
__global__ __launch_bounds__(256) void operands_kernel(const T* x, int64_t ldx, int m, int cols,
                                                       int blocks, int steps, int tiles,
                                                       uint32_t* out, uint8_t* scales) {
  const int at = blockIdx.x * 64 + threadIdx.x / 4;
  if (at >= tiles * 16 * steps * 4) return;
  const int n = at / (steps * 4), b = at - n * (steps * 4), l = threadIdx.x % 4;
  const int step = b / 4, lane = b % 4 * 16 + n % 16, tile = n / 16;
  uint32_t q = 0;
  int e = 127;
  if (n < m && b < blocks) q = row_codes(x + (int64_t)n * ldx, b * kSmall + 8 * l, cols, e);
  out[((int64_t)tile * steps + step) * (kPiece / 4) + lane * 4 + l] = q;
  if (l == 0)
    scales[(((int64_t)tile * ((steps + kGroup - 1) / kGroup) + step / kGroup) * 64 + lane) * kGroup +
           step % kGroup] = (uint8_t)e;
}

__device__ inline int32x8 operand(uintx4 q) {
  return int32x8{(int)q[0], (int)q[1], (int)q[2], (int)q[3], 0, 0, 0, 0};
}

template <int BYTE, int BYTE_A = 0>  // of sb and of sa
__device__ inline f32x4 multiply(uintx4 a, int sa, uintx4 b, int sb, f32x4 c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(a), operand(b), c, 4, 4, BYTE_A,
                                                          sa, BYTE, sb);
}

template <class T>
using Sixteen = T __attribute__((ext_vector_type(16 / sizeof(T))));  // bytes

// What a lane gives to one step of a tile of W.  Blocks behind a row's last one are read as the
// last one: the other side is zero there.
struct Weights {
  uintx4 q;
  int e;
  template <bool ONCE>
  __device__ void load(const uint8_t* w, const uint8_t* scale, int block, int blocks) {
    const int b = min(block, blocks - 1);
    const uintx4* p = reinterpret_cast<const uintx4*>(w + b * 16);
    q = ONCE ? __builtin_nontemporal_load(p) : *p;
    e = scale[b];
  }
};

template <class T, int N>
__device__ inline void store_rows(T* O, int64_t ldo, int m, int64_t D, int n, int64_t r,
                                  const float (&acc)[N]) {
  if (n >= m || r >= D) return;
  T* o = O + n * ldo + r;
  T v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (T)acc[i];
  if (r + N <= D) {
    store_vec(o, v);
  } else {
    for (int i = 0; i < N; ++i)
      if (r + i < D) o[i] = v[i];
  }
}

template <class T>
__device__ inline void store_bytes(T* O, int64_t ldo, int m, int64_t D, int n, int64_t r,
                                   uintx4 bytes) {
  constexpr int N = 16 / (int)sizeof(T);
  const auto u = __builtin_bit_cast(Sixteen<T>, bytes);
  if (n >= m || r >= D) return;
  T* o = O + n * ldo + r;
  T v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = u[i];
  if (r + N <= D) {
    store_vec(o, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (r + i < D) o[i] = v[i];
  }
}

// At most 16 rows of H: one launch.  Every block quantises them by itself, into LDS, and its
// waves go through tiles of 16 rows of W, four steps at a time, the next four's codes under way.
// Bound by memory: one row by 200 000 x 500 (55 MB) takes 12.1 us, 4.6 TB/s (13.9 without the next
// codes under way).  WIDE: a row has a multiple of 16
// blocks, so that its exponents are loaded by words.
template <class TH, class T, bool WIDE>
__global__ __launch_bounds__(512) void few_kernel(const TH* H, int64_t ldh, int d,
                                                  const uint8_t* W, const uint8_t* sw, int m,
                                                  int64_t D, int blocks, int steps, T* O,
                                                  int64_t ldo) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  const int l = threadIdx.x % 64, i16 = l % 16, q4 = l / 16;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t ld = (int64_t)blocks * 16, tiles = (D + 15) / 16;
  struct Four {
    uintx4 q[kGroup];
    unsigned e[kGroup];
  };
  auto load = [&](int64_t tile, int s0) {
    Four c;
    const int64_t row = min(tile * 16 + i16, D - 1);
    const uint8_t *p = W + row * ld, *ps = sw + row * blocks;
#pragma unroll
    for (int j = 0; j < kGroup; ++j) {
      // blocks behind a row's last one are read as the last: the other side is zero there
      const int b = min((s0 + j) * 4 + q4, blocks - 1);
      c.q[j] = *reinterpret_cast<const uintx4*>(p + b * 16);
      if constexpr (!WIDE) c.e[j] = ps[b];
    }
    if constexpr (WIDE) {  // the exponents of four steps, all of the row's, in one load
      typedef unsigned words __attribute__((ext_vector_type(4), aligned(1)));
      const words u = *reinterpret_cast<const words*>(ps + 4 * s0);
#pragma unroll
      for (int j = 0; j < kGroup; ++j) c.e[j] = u[j];
    }
    return c;
  };
  // of the lane's own blocks: taken where they are used, or the load would be waited for at once
  const int shift = WIDE ? 8 * q4 : 0;
  int64_t tile = (int64_t)blockIdx.x * 8 + w;
  Four next = load(tile, 0);
  int* exponents = (int*)(lds + steps * (kPiece / 4));
  for (int at = threadIdx.x / 4; at < 16 * 4 * steps; at += 512 / 4) {
    const int n = at / (4 * steps), b = at - n * (4 * steps), c = threadIdx.x % 4;
    uint32_t q = 0;
    int e = 127;
    if (n < m && b < blocks) q = row_codes(H + n * ldh, b * kSmall + 8 * c, d, e);
    const int lane = b / 4 * 64 + b % 4 * 16 + n;
    lds[lane * 4 + c] = q;
    if (c == 0) exponents[lane] = e;
  }
  __syncthreads();
  const uintx4* operands = reinterpret_cast<const uintx4*>(lds);
  f32x4 acc = {};
  for (int s0 = 0; tile < tiles;) {
    const Four c = next;
    const int64_t at = tile;
    const int s = s0;
    s0 += kGroup;
    const bool done = s0 >= steps;
    if (done) s0 = 0, tile += (int64_t)gridDim.x * 8;
    next = load(tile, s0);  // behind the last tile, where W's last row is read, too
#pragma unroll
    for (int j = 0; j < kGroup; ++j)
      if (s + j < steps)
        acc = multiply<0>(c.q[j], c.e[j] >> shift, operands[(s + j) * 64 + l],
                          exponents[(s + j) * 64 + l], acc);
    if (done) {
      const float v[4] = {acc[0], acc[1], acc[2], acc[3]};
      store_rows(O, ldo, m, D, i16, at * 16 + 4 * q4, v);
      acc = f32x4{};
    }
  }
}

// Rows of more than 1024 columns, which do not fit a wave's registers.
//
// 16 MT rows of W a wave, four waves a block one after another, 16 NT rows of H a block.  Four
// steps of H's operands go to LDS by DMA while the four before are multiplied; the codes of a
// wave's own rows go to registers, two steps ahead.
template <class T, int MT, int NT, bool ONCE>
__global__ __launch_bounds__(256, 2) void scores_kernel(const uint8_t* W, const uint8_t* sw,
                                                        const uint8_t* H, const int* sh, int m,
                                                        int64_t D, int blocks, int steps,
                                                        int row_blocks, T* O, int64_t ldo) {
  __shared__ __attribute__((aligned(16))) uint8_t hb[2][kGroup * NT * kPiece];
  const int l = threadIdx.x % 64, i16 = l % 16, q4 = l / 16;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  // the blocks of the same rows of W follow each other on one XCD, and share its L2
  const int tiles = (m + 15) / 16, cols = (tiles + NT - 1) / NT;
  const int xcd = blockIdx.x % 8, i = blockIdx.x / 8;
  const int row_block = i / cols * 8 + xcd, t0 = i % cols * NT;
  if (row_block >= row_blocks) return;
  const int64_t r0 = ((int64_t)row_block * 4 + w) * 16 * MT, ld = (int64_t)blocks * 16;
  // 16-bit outputs: rows of W are dealt to pairs of tiles in fours, so that a lane holds eight
  // neighbouring outputs and four lanes 64 bytes of a row of O
  constexpr bool kPairs = sizeof(T) == 2 && MT % 2 == 0;
  const uint8_t *p[MT], *ps[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int at = kPairs ? t / 2 * 32 + i16 / 4 * 8 + t % 2 * 4 + i16 % 4 : 16 * t + i16;
    const int64_t row = min(r0 + at, D - 1);
    p[t] = W + row * ld;
    ps[t] = sw + row * blocks;
  }
  auto fetch = [&](int g) {  // NT pieces for each step of the group, a quarter of them a wave
#pragma unroll
    for (int k = 0; k < NT; ++k) {
      const int piece = w * NT + k, step = g * kGroup + piece / NT, t = t0 + piece % NT;
      dma16((const float*)(H + ((int64_t)min(t, tiles - 1) * steps + min(step, steps - 1)) * kPiece +
                           l * 16),
            lds_u32(&hb[g % 2][piece * kPiece]));
    }
  };
  f32x4 acc[MT][NT] = {};
  Weights c[kGroup][MT];
  int e[NT];
  auto load = [&](int slot, int step) {
#pragma unroll
    for (int t = 0; t < MT; ++t)
      c[slot][t].template load<ONCE>(p[t], ps[t], min(step, steps - 1) * 4 + q4, blocks);
  };
  fetch(0);
  load(0, 0);
  load(1, 1);
  const int groups = (steps + kGroup - 1) / kGroup;
  for (int g = 0; g < groups; ++g) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
      e[n] = sh[((int64_t)min(t0 + n, tiles - 1) * groups + g) * 64 + l];
    wait_vm_le(0);
    lds_barrier();  // group g has landed; every wave is done with the one before
    if (g + 1 < groups) fetch(g + 1);
    const uintx4* h = reinterpret_cast<const uintx4*>(hb[g % 2]);
    auto run = [&](auto byte) {
      constexpr int s = byte;
      if (g * kGroup + s >= steps) return;
      load((s + 2) % kGroup, g * kGroup + s + 2);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uintx4 b = h[(s * NT + n) * 64 + l];
#pragma unroll
        for (int t = 0; t < MT; ++t)
          acc[t][n] = multiply<s>(c[s][t].q, c[s][t].e, b, e[n], acc[t][n]);
      }
    };
    run(std::integral_constant<int, 0>{});
    run(std::integral_constant<int, 1>{});
    run(std::integral_constant<int, 2>{});
    run(std::integral_constant<int, 3>{});
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int t = 0; t < MT; t += kPairs ? 2 : 1) {
      const int row = (t0 + n) * 16 + i16;
      if constexpr (kPairs) {
        const f32x4 a = acc[t][n], b = acc[t + 1][n];
        const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        store_rows(O, ldo, m, D, row, r0 + 16 * t + 8 * q4, v);
      } else {
        const f32x4 a = acc[t][n];
        const float v[4] = {a[0], a[1], a[2], a[3]};
        store_rows(O, ldo, m, D, row, r0 + 16 * t + 4 * q4, v);
      }
    }
}

// Trades places: register b of the lanes with bit BIT clear for register a of those with it set,
// a neighbour's in the four.
template <int BIT>
__device__ inline void trade(uintx4& a, uintx4& b, bool set) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int give = (int)(set ? a[i] : b[i]);
    const unsigned got = (unsigned)__builtin_amdgcn_update_dpp(0, give, BIT ? 0x4E : 0xB1, 0xF,
                                                               0xF, true);
    a[i] = set ? got : a[i];
    b[i] = set ? b[i] : got;
  }
}

constexpr int kHeldSteps = 8;    // of a wave's rows of W in registers: 1024 columns, two sets
constexpr int kHeldBlocks = 256; // of that launch, one a compute unit
constexpr int kHeldBytes = 144 * 1024;  // of LDS for H

// All of H's rows that LDS holds, and waves that go through W by themselves: a wave has 16 MT rows
// of W in registers, KS steps of them, the next ones' loads under way, multiplies them with one
// tile of H's rows after another and stores what comes out.  Where H takes several parts, blocks
// of one XCD take them for the same rows of W, which come from its L2 to all but the first.
//
// The barriers in the loop stand for no data: they keep the waves, which have neighbouring tiles
// of W, near each other, so that what two of them store of the same line of memory meets in L2
// (512 rows of H in bfloat16 by 793 471 x 300: 321 us, with one for each tile of W 356, without
// 415; by 500 000 x 1024 265, 260 and 251: no more than one a tile there).
//
// A wave reads all of a tile's operands before it multiplies them: with a branch for each step,
// which the number of steps as an argument asks for, each read was waited for by itself, and 512
// rows by 500 000 x 1024 took 251 us.
//
// Measured: 128 rows by 200 000 x 500, float32 outputs, 36 us (157 MB, 4.4 TB/s); 512 rows by
// 500 000 x 1024 in bfloat16 214 us (784 MB, 3.7 TB/s; 2.5 PFLOP/s).  W through LDS by DMA with H
// in registers, which halves what LDS gives, took 243 us where this took 251, and twice as long
// for rows of O at odd addresses; two tiles of H at a time, and the next tile's operands under
// way, nothing to gain (231, 235, where this took 226: the registers).  WIDE as for few rows: with
// the choice made by each load, all loads under way were waited for, 226 us where this takes 214.
template <class T, int MT, int KS, bool WIDE>
__global__ __launch_bounds__(512, 1) void held_kernel(const uint8_t* W, const uint8_t* sw,
                                                      const uint8_t* H, const int* sh, int m,
                                                      int64_t D, int blocks, int part, int parts,
                                                      int near, T* O, int64_t ldo) {
  constexpr int kTogether = KS > 4 ? 0xFFFF : 3;  // tiles of H between two barriers, less one
  constexpr int G = (KS + kGroup - 1) / kGroup;  // words of exponents
  __shared__ __attribute__((aligned(16))) uint8_t held[kHeldBytes];
  const int l = threadIdx.x % 64, i16 = l % 16, q4 = l / 16;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int xcd = blockIdx.x % 8, i = blockIdx.x / 8;
  const int t0 = i % parts * part, tiles = min(part, (m + 15) / 16 - t0);
  int* exponents = (int*)(held + (int64_t)part * KS * kPiece);
  for (int p = w; p < tiles * KS; p += 8)
    dma16((const float*)(H + ((int64_t)t0 * KS + p) * kPiece + l * 16),
          lds_u32(held + p * kPiece));
  for (int p = threadIdx.x; p < tiles * G * 64; p += 512)
    exponents[p] = sh[(int64_t)t0 * G * 64 + p];
  const int64_t ld = (int64_t)blocks * 16, all = (D + 16 * MT - 1) / (16 * MT);
  const int64_t each = (int64_t)(gridDim.x / 8 / parts) * 64;  // waves beside each other
  uintx4 q[2][MT][KS];
  unsigned raw[2][MT][G * kGroup];  // exponents as they were read
  const unsigned pick = 0x0400u + 0x0101u * q4;  // byte q4 of one word, and of another
  auto load = [&](auto slot, int64_t tile) {
    constexpr int S = slot;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      // the four sums of a lane are neighbours, tile after tile
      const int at = i16 / 4 * 4 * MT + 4 * t + i16 % 4;
      const int64_t row = min(tile * 16 * MT + at, D - 1);
      const uint8_t *p = W + row * ld, *ps = sw + row * blocks;
#pragma unroll
      for (int s = 0; s < KS; ++s)  // blocks behind a row's last one are read as the last: the
                                    // other side is zero there
        q[S][t][s] = *reinterpret_cast<const uintx4*>(p + min(4 * s + q4, blocks - 1) * 16);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        if constexpr (WIDE) {  // all of the row's, in one load
          typedef unsigned words __attribute__((ext_vector_type(4), aligned(1)));
          const words u = *reinterpret_cast<const words*>(ps + 16 * g);
#pragma unroll
          for (int s = 0; s < kGroup; ++s) raw[S][t][kGroup * g + s] = u[s];
        } else {
#pragma unroll
          for (int s = 0; s < kGroup; ++s)
            raw[S][t][kGroup * g + s] = ps[min(16 * g + 4 * s + q4, blocks - 1)];
        }
      }
    }
  };
  auto run = [&](auto slot, int64_t tile) {
    constexpr int S = slot;
    // four steps of the lane's own blocks a word: put together here, or the loads would be waited
    // for where they are issued
    int e[MT][G];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const unsigned* u = raw[S][t] + kGroup * g;
        const unsigned how = WIDE ? pick : 0x0400u;
        e[t][g] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], how),
                                        __builtin_amdgcn_perm(u[1], u[0], how), 0x05040100);
      }
    for (int n = 0; n < tiles; ++n) {
      if ((n & kTogether) == 0) __builtin_amdgcn_s_barrier();
      if (tile >= all) continue;
      f32x4 acc[MT] = {};
      const uintx4* h = reinterpret_cast<const uintx4*>(held) + (int64_t)n * KS * 64 + l;
      uintx4 b[KS];
      int eh[G];
#pragma unroll
      for (int s = 0; s < KS; ++s) b[s] = h[s * 64];
#pragma unroll
      for (int g = 0; g < G; ++g) eh[g] = exponents[(n * G + g) * 64 + l];
      auto step = [&](auto at) {
        constexpr int s = at;
        if constexpr (s < KS)
#pragma unroll
          for (int t = 0; t < MT; ++t)
            acc[t] = multiply<s % kGroup, s % kGroup>(q[S][t][s], e[t][s / kGroup], b[s],
                                                      eh[s / kGroup], acc[t]);
      };
      step(std::integral_constant<int, 0>{});
      step(std::integral_constant<int, 1>{});
      step(std::integral_constant<int, 2>{});
      step(std::integral_constant<int, 3>{});
      step(std::integral_constant<int, 4>{});
      step(std::integral_constant<int, 5>{});
      step(std::integral_constant<int, 6>{});
      step(std::integral_constant<int, 7>{});
      // 16 bytes of a row of O a register set; neighbouring lanes trade them for those of the
      // same row, so that a store has 256 bytes of a row (128 of 16 bits or with two tiles)
      constexpr int kSets = MT * (int)sizeof(T) / 4, kEach = 16 / (int)sizeof(T);
      uintx4 v[kSets];
#pragma unroll
      for (int t = 0; t < kSets; ++t) {
        if constexpr (sizeof(T) == 4) {
          v[t] = __builtin_bit_cast(uintx4, acc[t]);
        } else {
          T __attribute__((ext_vector_type(8))) u;
#pragma unroll
          for (int i = 0; i < 8; ++i) u[i] = (T)acc[2 * t + i / 4][i % 4];
          v[t] = __builtin_bit_cast(uintx4, u);
        }
      }
      if constexpr (kSets >= 2)
#pragma unroll
        for (int t = 0; t < kSets; t += 2) trade<0>(v[t], v[t + 1], l & 1);
      if constexpr (kSets == 4) {
        trade<1>(v[0], v[2], l & 2);
        trade<1>(v[1], v[3], l & 2);
      }
      const int64_t r = tile * 16 * MT + 4 * MT * q4 + kEach * (l % kSets);
#pragma unroll
      for (int j = 0; j < kSets; ++j)
        store_bytes(O, ldo, m, D, (t0 + n) * 16 + i16 / kSets * kSets + j, r, v[j]);
    }
  };
  // neighbouring tiles in one block: what its waves store of a row of O is one piece
  int64_t tile = (w / near * (each / 8) + (int64_t)(i / parts) * 8 + xcd) * near + w % near;
  std::integral_constant<int, 0> even;
  std::integral_constant<int, 1> odd;
  load(even, tile);
  wait_vm_le(0);
  __syncthreads();
  const int64_t first = ((int64_t)(i / parts) * 8 + xcd) * near;  // of the block's waves
  for (int64_t u = first; u < all; u += 2 * each, tile += 2 * each) {
    // also behind the last tile, where all lanes read W's last row: a load that a branch may leave
    // out cannot be told from those before it, and would be waited for with them
    load(odd, tile + each);
    run(even, tile);
    load(even, tile + 2 * each);
    run(odd, tile + each);
  }
}

constexpr int kFew = 16;         // rows of H that one launch takes: a pass of 16 by 200 000 x 500
                                 // codes 17.1 us, with operands first 19.5; one row 13.3 and 17.6;
                                 // 16 by 200 000 x 1024 27.8 and 31.1, by 5000 x 500 10.7 and 13.5
constexpr int kFewBlocks = 512;  // blocks of that launch, two a compute unit
constexpr int64_t kMostBlocks = (1 << 30) - 64;  // of a matrix: 2^32 threads

int64_t blocks_of(int32_t cols) { return ((int64_t)cols + kSmall - 1) / kSmall; }
int64_t steps_of(int32_t cols) { return ((int64_t)cols + kStep - 1) / kStep; }
int64_t pieces_bytes(int32_t m, int32_t d) {
  return ((int64_t)m + 15) / 16 * steps_of(d) * kPiece;
}

}  // namespace
}  // namespace lst

using namespace lst;

extern "C" {

int lst_quantize_four(int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t ldx,
                      uint8_t* codes, uint8_t* scales, void* hip_stream) {
  if (!known_dtype(dtype) || rows < 0 || cols < 1 || cols > 4096) return LST_EINVAL;
  if (rows == 0) return LST_OK;
  if (!x || !codes || !scales || ldx < cols || ((uintptr_t)codes & 15)) return LST_EINVAL;
  if (rows > kMostBlocks / blocks_of(cols)) return LST_EINVAL;
  const int64_t n = (rows * blocks_of(cols) + 63) / 64;
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(quantize_kernel<T>, dim3((unsigned)n), dim3(256), 0,
                       (hipStream_t)hip_stream, (const T*)x, ldx, rows, cols,
                       (int)blocks_of(cols), (uint32_t*)codes, scales);
    return launched();
  });
}

int64_t lst_scores_four_workspace(int32_t m, int32_t d) {
  if (m < 0 || d < 1 || d > 4096) return -1;
  const int64_t groups = (steps_of(d) + kGroup - 1) / kGroup;
  return pieces_bytes(m, d) + ((int64_t)m + 15) / 16 * groups * 64 * kGroup;
}

int lst_scores_four(int32_t dtype, int32_t out_dtype, int32_t m, int64_t D, int32_t d,
                    const void* H, int64_t ldh, const uint8_t* codes, const uint8_t* scales,
                    void* O, int64_t ldo, void* workspace, void* hip_stream) {
  if (!known_dtype(dtype) || !known_dtype(out_dtype) || m < 0 || D < 1 || d < 1 || d > 4096)
    return LST_EINVAL;
  if (m == 0) return LST_OK;
  if (!H || !codes || !scales || !O || !workspace || ldh < d || ldo < D) return LST_EINVAL;
  if (((uintptr_t)codes & 15) || ((uintptr_t)workspace & 15)) return LST_EINVAL;
  if (m > 1 << 20 || D > (int64_t)1 << 36) return LST_EINVAL;
  hipStream_t s = (hipStream_t)hip_stream;
  const int blocks = (int)blocks_of(d), steps = (int)steps_of(d), tiles = (m + 15) / 16;
  if (m <= kFew)
    return with_dtype(dtype, [&](auto th) {
      return with_dtype(out_dtype, [&](auto t) {
        using TH = decltype(th);
        using T = decltype(t);
        const int64_t groups = (D + 127) / 128;
        const size_t lds = (size_t)steps * (kPiece + 64 * sizeof(int));
        auto run = [&](auto kernel) {
          hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(groups, kFewBlocks)),
                             dim3(512), lds, s, (const TH*)H, ldh, d, codes, scales, m, D, blocks,
                             steps, (T*)O, ldo);
          return launched();
        };
        return blocks % 16 == 0 ? run(few_kernel<TH, T, true>) : run(few_kernel<TH, T, false>);
      });
    });
  // 256 rows of W and up to 8 tiles of H a block; no more than there are: 17 rows of H by 200 000
  // x 2048 codes take 92 us with 2 tiles and 97 with 8, 64 take 105 with 4 and 107 with 8
  const int nt = tiles <= 2 ? 2 : tiles <= 4 ? 4 : 8;
  const int64_t row_blocks = (D + 255) / 256;
  const int64_t grid = (row_blocks + 7) / 8 * 8 * ((tiles + nt - 1) / nt);
  if (grid > 0xFFFFFF) return LST_EINVAL;  // a launch has 2^32 threads at most
  uint8_t *pieces = (uint8_t*)workspace, *exponents = pieces + pieces_bytes(m, d);
  const int rc = with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(operands_kernel<T>, dim3(tiles * steps), dim3(256), 0, s, (const T*)H, ldh,
                       m, d, blocks, steps, tiles, (uint32_t*)pieces, exponents);
    return launched();
  });
  if (rc != LST_OK) return rc;
  if (steps <= kHeldSteps)
    return with_dtype(out_dtype, [&](auto t) {
      using T = decltype(t);
      const int groups = (steps + kGroup - 1) / kGroup;
      const int bytes = steps * kPiece + groups * 64 * (int)sizeof(int);  // of a tile of H
      const int most = kHeldBytes / bytes, parts = (tiles + most - 1) / most;
      const int part = (tiles + parts - 1) / parts;
      auto run = [&](auto kernel, int rows) {
        // blocks of a part on an XCD: as many as leave the fewest of its 32 compute units idle
        int strips = 1;
        double best = 0;
        for (int k = 1; k <= std::max(4, kHeldBlocks / 8 / parts); ++k) {
          const int64_t n = (int64_t)k * parts, rounds = (n + 31) / 32;
          const double share = n / (32.0 * rounds);
          if (share > best) best = share, strips = k;
        }
        // few rows of W go to as many compute units as there are
        const int near = (D + 16 * rows - 1) / (16 * rows) < strips * 64 ? 2 : 8;
        hipLaunchKernelGGL(kernel, dim3(strips * parts * 8), dim3(512), 0, s, codes, scales,
                           pieces, (const int*)exponents, m, D, blocks, part, parts, near, (T*)O,
                           ldo);
        return launched();
      };
      const bool wide = blocks % 16 == 0;  // whole words of exponents
      switch (steps) {
        case 1: return run(held_kernel<T, 4, 1, false>, 4);
        case 2: return run(held_kernel<T, 4, 2, false>, 4);
        case 3: return run(held_kernel<T, 4, 3, false>, 4);
        case 4: return wide ? run(held_kernel<T, 4, 4, true>, 4)
                            : run(held_kernel<T, 4, 4, false>, 4);
        case 5: return run(held_kernel<T, 2, 5, false>, 2);
        case 6: return run(held_kernel<T, 2, 6, false>, 2);
        case 7: return run(held_kernel<T, 2, 7, false>, 2);
        default: return wide ? run(held_kernel<T, 2, 8, true>, 2)
                             : run(held_kernel<T, 2, 8, false>, 2);
      }
    });
  return with_dtype(out_dtype, [&](auto t) {
    using T = decltype(t);
    auto run = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), 0, s, codes, scales, pieces,
                         (const int*)exponents, m, D, blocks, steps, (int)row_blocks, (T*)O, ldo);
      return launched();
    };
    if (nt == 2) return run(scores_kernel<T, 4, 2, true>);
    if (nt == 4) return run(scores_kernel<T, 4, 4, true>);
    return tiles <= 8 ? run(scores_kernel<T, 4, 8, true>) : run(scores_kernel<T, 4, 8, false>);
  });
}

}  // extern "C"
