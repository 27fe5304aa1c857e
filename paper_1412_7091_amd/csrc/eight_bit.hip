// Weights in 8 bits (lst_quantize) and a layer's outputs from them (lst_scores).
//
// A row is cut into blocks of 128 columns.  A block holds e4m3 codes q and one
// exponent e with 448 2^e the smallest such bound on the block's values, so that
// x ~ q 2^e.  A power of two costs at most one of the type's 18 binades and none
// of its digits, and x 2^-e is exact.
//
//   O[i][r] = sum_b 2^(e_ib + e_rb) sum_{k in b} qh_ik qw_rk
//
// The products are made by the bfloat16 matrix instruction: q 2^e is a bfloat16
// without rounding (four digits, any exponent), one instruction turns two codes
// into two of them with the scale applied, and so no scale is left for the sums.
// The 8-bit matrix instructions have twice the rate, but they lose what is 2^-14
// of the largest product that is summed with it (measured: a product of 2^2 beside
// one of 2^16), which is an error of 1.2e-5 in the sums of 128 ordinary products.
//
// The rows of H are quantised in the same way, by the operator's definition (this instruction
// would take eight binary digits at the same rate, where e4m3 has four), and left in bfloat16, in the order in
// which the matrix instruction takes them: a fragment, 16 rows by 32 columns, is 64
// lanes of 16 bytes.
#include <algorithm>

#include "dtypes.h"
#include "eight_bit.h"
#include "gemm_tile.h"

namespace lst {
namespace {

constexpr int kFragment = 64 * 8;          // bfloat16 of a fragment: 16 rows, 32 columns
constexpr int kTile = 4 * kFragment;       // of 16 rows of one block

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ inline float scale_value(int e) {
  return __uint_as_float(e ? (uint32_t)e << 23 : 0x400000u);  // 2^(e - 127)
}

__device__ inline bf16x8 widen(uintx2 q, float scale) {
  bf16x8 f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[i], scale, false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[i], scale, true);
    f[4 * i] = lo[0], f[4 * i + 1] = lo[1], f[4 * i + 2] = hi[0], f[4 * i + 3] = hi[1];
  }
  return f;
}

// Eight columns from `col` of a row, a block being in 16 neighbouring lanes: their codes and
// the block's biased exponent.
template <class T>
__device__ inline void block_codes(const T* row, int col, int cols, uint32_t (&q)[2], int& e) {
  T raw[8];
  load_part(row, col, cols, raw);
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)raw[i];
  values_codes(v, q, e);
}

// Rows of H as the kernels take them: values that they quantise, or codes as lst_quantize and
// lst_norm_forward leave them.
template <class T>
struct Values {
  const T* x;
  int64_t ld;
  int cols;
  __device__ void block(int64_t n, int b, int c, uint32_t (&q)[2], int& e) const {
    block_codes(x + n * ld, b * kBlock + 8 * c, cols, q, e);
  }
};
struct Coded {
  const uint8_t *codes, *scales;
  int blocks;
  __device__ void block(int64_t n, int b, int c, uint32_t (&q)[2], int& e) const {
    const int64_t at = n * blocks + b;
    const uintx2 v = reinterpret_cast<const uintx2*>(codes)[at * 16 + c];
    q[0] = v[0], q[1] = v[1];
    e = scales[at];
  }
};

// 16 lanes a block, eight columns a lane.  Bound by memory: 793 471 x 300 floats (1.26 GB
// with the codes) take 222 us, 5.7 TB/s; 32 lanes a block, four columns a lane with an access
// for each, took 305 us.
template <class T>
__global__ __launch_bounds__(256) void quantize_kernel(const T* x, int64_t ldx, int64_t rows,
                                                       int cols, int blocks, uint8_t* codes,
                                                       uint8_t* scales) {
  const unsigned at = blockIdx.x * 16 + threadIdx.x / 16;  // the block
  if (at >= (unsigned)(rows * blocks)) return;
  const unsigned row = at / (unsigned)blocks;
  const int l = threadIdx.x % 16, col = (int)(at - row * (unsigned)blocks) * kBlock + 8 * l;
  uint32_t q[2];
  int e;
  block_codes(x + (int64_t)row * ldx, col, cols, q, e);
  reinterpret_cast<uintx2*>(codes)[(int64_t)at * 16 + l] = uintx2{q[0], q[1]};
  if (l == 0) scales[at] = (uint8_t)e;
}

// Where the eight columns of lane l of a block belong among the fragments of 16 rows.  Lane q
// of four takes columns 16 q .. 16 q + 15 of each half of a block: which columns one
// instruction adds up is free as long as both sides agree, and a wave then reads 64
// contiguous bytes of each row of codes at a time.
__device__ inline int fragment_at(int n16, int l) {
  const int s = l % 2 + 2 * (l / 8), q = l / 2 % 4;
  return s * kFragment + (q * 16 + n16) * 8;
}

// Rows of H into fragments, tiles of 16 rows of one block: tile (b, n / 16) of the workspace.
// Rows behind the last one of the last tile are zeros.
template <class R>
__global__ __launch_bounds__(256) void fragments_kernel(R rows, int m, int blocks, int tiles,
                                                        __bf16* out) {
  const int at = blockIdx.x * 16 + threadIdx.x / 16;
  if (at >= tiles * 16 * blocks) return;
  const int n = at / blocks, b = at - n * blocks, l = threadIdx.x % 16;
  uint32_t q[2] = {0, 0};
  int e = 0;
  if (n < m) rows.block(n, b, l, q, e);
  __bf16* p = out + ((int64_t)b * tiles + n / 16) * kTile + fragment_at(n % 16, l);
  *reinterpret_cast<bf16x8*>(p) = widen(uintx2{q[0], q[1]}, scale_value(e));
}

// A lane's codes of one block of a row of W, and their scale.
struct Codes {
  uintx4 lo, hi;
  int e;
  // ONCE: no other block reads them
  template <bool ONCE>
  __device__ void load(const uint8_t* w, const uint8_t* scale) {
    const uintx4 *p = reinterpret_cast<const uintx4*>(w),
                 *q = reinterpret_cast<const uintx4*>(w + 64);
    lo = ONCE ? __builtin_nontemporal_load(p) : *p;
    hi = ONCE ? __builtin_nontemporal_load(q) : *q;
    e = *scale;
  }
  __device__ bf16x8 fragment(int s) const {
    const uintx4 c = s < 2 ? lo : hi;
    return widen(uintx2{c[s % 2 * 2], c[s % 2 * 2 + 1]}, scale_value(e));
  }
};

// The sums of 16 rows of W (from r) and 16 rows of H (from n): four rows of W a lane.
template <class T>
__device__ inline void store_tile(T* O, int64_t ldo, int m, int64_t D, int n, int64_t r,
                                  f32x4 acc) {
  if (n >= m || r >= D) return;
  T* o = O + n * ldo + r;
  T v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (T)acc[i];
  if (r + 4 <= D) {
    store_vec(o, v);
  } else {
    for (int i = 0; i < 4; ++i)
      if (r + i < D) o[i] = v[i];
  }
}

// At most 16 rows of H: one launch.  Every block quantises them by itself, into LDS, and its
// waves go through tiles of 16 rows of W, four blocks' codes under way at a time.  Bound by
// memory: one row by 200 000 x 512 codes (104 MB) takes 21 us, 5.0 TB/s; with the
// quantisation in a launch of its own 27.
template <class R, class T>
__global__ __launch_bounds__(512) void scores_few_kernel(R rows, const uint8_t* W,
                                                         const uint8_t* sw, int m, int64_t D,
                                                         int blocks, T* O, int64_t ldo) {
  extern __shared__ __attribute__((aligned(16))) __bf16 few_lds[];
  const int l = threadIdx.x % 64, i16 = l % 16, q4 = l / 16;
  for (int at = threadIdx.x / 16; at < 16 * blocks; at += 512 / 16) {
    const int n = at / blocks, b = at - n * blocks, c = threadIdx.x % 16;
    uint32_t q[2] = {0, 0};
    int e = 0;
    if (n < m) rows.block(n, b, c, q, e);
    *reinterpret_cast<bf16x8*>(few_lds + b * kTile + fragment_at(n, c)) =
        widen(uintx2{q[0], q[1]}, scale_value(e));
  }
  __syncthreads();
  const int64_t ld = (int64_t)blocks * kBlock, tiles = (D + 15) / 16;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  for (int64_t tile = (int64_t)blockIdx.x * 8 + w; tile < tiles; tile += (int64_t)gridDim.x * 8) {
    const int64_t row = min(tile * 16 + i16, D - 1);
    const uint8_t *p = W + row * ld + 16 * q4, *ps = sw + row * blocks;
    f32x4 acc = {};
    for (int b0 = 0; b0 < blocks; b0 += 4) {
      Codes c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int b = min(b0 + j, blocks - 1);
        c[j].load<false>(p + b * kBlock, ps + b);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (b0 + j < blocks)
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const bf16x8 h = *reinterpret_cast<const bf16x8*>(few_lds + (b0 + j) * kTile +
                                                              s * kFragment + l * 8);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c[j].fragment(s), h, acc, 0, 0, 0);
          }
    }
    store_tile(O, ldo, m, D, i16, tile * 16 + 4 * q4, acc);
  }
}

// 16 MT rows of W a wave, four waves a block one after another, 16 NT rows of H a block.  A
// block of H's columns goes to LDS by DMA while the one before is multiplied; the codes of a
// wave's own rows go to registers.
//
// 128 rows of H by 200 000 x 512 codes take 59 us (205 MB at 3.5 TB/s; 63 with loads that
// stay in the caches, which no other block reads; the same with all of H held in LDS and
// waves that go through W by themselves: 56), 512 rows by 500 000 x 1024 take 555 us
// (0.95 PFLOP/s, where a large bfloat16 product of the library reaches 1.2 and this one 0.87;
// 666 with loads past the caches, where four blocks read the same codes).
template <class T, int MT, int NT, bool ONCE>
__global__ __launch_bounds__(256, 2) void scores_kernel(const uint8_t* W, const uint8_t* sw,
                                                     const __bf16* H, int m, int64_t D,
                                                     int blocks, int row_blocks, T* O,
                                                     int64_t ldo) {
  __shared__ __attribute__((aligned(16))) __bf16 hb[2][NT * kTile];
  const int l = threadIdx.x % 64, i16 = l % 16, q4 = l / 16;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  // the blocks of the same rows of W follow each other on one XCD, and share its L2
  const int tiles = (m + 15) / 16, cols = (tiles + NT - 1) / NT;
  const int xcd = blockIdx.x % 8, i = blockIdx.x / 8;
  const int row_block = i / cols * 8 + xcd, t0 = i % cols * NT;
  if (row_block >= row_blocks) return;
  const int64_t r0 = ((int64_t)row_block * 4 + w) * 16 * MT, ld = (int64_t)blocks * kBlock;
  const uint8_t *p[MT], *ps[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t row = min(r0 + 16 * t + i16, D - 1);
    p[t] = W + row * ld + 16 * q4;
    ps[t] = sw + row * blocks;
  }
  auto fetch = [&](int b) {  // NT tiles of 4 KB, a quarter of them a wave
#pragma unroll
    for (int k = 0; k < NT; ++k) {
      const int piece = w * NT + k, t = min(t0 + piece / 4, tiles - 1);
      dma16((const float*)(H + ((int64_t)b * tiles + t) * kTile + piece % 4 * kFragment + l * 8),
            lds_u32(&hb[b % 2][piece * kFragment]));
    }
  };
  f32x4 acc[MT][NT] = {};
  Codes next[MT];
  fetch(0);
#pragma unroll
  for (int t = 0; t < MT; ++t) next[t].template load<ONCE>(p[t], ps[t]);
  for (int b = 0; b < blocks; ++b) {
    wait_vm_le(0);
    lds_barrier();  // block b has landed; every wave is done with block b - 1
    Codes c[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) c[t] = next[t];
    if (b + 1 < blocks) {
      fetch(b + 1);
#pragma unroll
      for (int t = 0; t < MT; ++t) next[t].template load<ONCE>(p[t] + (b + 1) * kBlock, ps[t] + b + 1);
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      bf16x8 a[MT];
#pragma unroll
      for (int t = 0; t < MT; ++t) a[t] = c[t].fragment(s);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const bf16x8 h = *reinterpret_cast<const bf16x8*>(
            &hb[b % 2][n * kTile + s * kFragment + l * 8]);
#pragma unroll
        for (int t = 0; t < MT; ++t)
          acc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], h, acc[t][n], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int t = 0; t < MT; ++t)
      store_tile(O, ldo, m, D, (t0 + n) * 16 + i16, r0 + 16 * t + 4 * q4, acc[t][n]);
}

constexpr int kFew = 16;          // rows of H that one launch takes: 23 us (16 by 200 000 x
                                  // 512 codes), by fragments and tiles 33
constexpr int kFewColumns = 2048;  // that fit 64 KB of LDS in bfloat16
constexpr int kFewBlocks = 512;   // blocks of that launch, two a compute unit
constexpr int64_t kMostBlocks = (1 << 28) - 16;  // of a matrix: 2^32 threads

int64_t blocks_of(int32_t cols) { return ((int64_t)cols + kBlock - 1) / kBlock; }

template <class R>
int scores(const R& rows, int32_t out_dtype, int32_t m, int64_t D, int32_t d,
           const uint8_t* codes, const uint8_t* scales, void* O, int64_t ldo, void* workspace,
           hipStream_t s) {
  if (!known_dtype(out_dtype) || m < 0 || D < 1 || d < 1 || d > 4096) return LST_EINVAL;
  if (m == 0) return LST_OK;
  if (!codes || !scales || !O || !workspace || ldo < D) return LST_EINVAL;
  if (((uintptr_t)codes & 15) || ((uintptr_t)workspace & 15)) return LST_EINVAL;
  if (m > 1 << 20 || D > (int64_t)1 << 36) return LST_EINVAL;
  const int blocks = (int)blocks_of(d), tiles = (m + 15) / 16;
  if (m <= kFew && blocks <= kFewColumns / kBlock)
    return with_dtype(out_dtype, [&](auto t) {
      using T = decltype(t);
      const int64_t groups = (D + 127) / 128;
      const size_t lds = (size_t)blocks * kTile * sizeof(__bf16);
      hipLaunchKernelGGL((scores_few_kernel<R, T>),
                         dim3((unsigned)std::min<int64_t>(groups, kFewBlocks)), dim3(512), lds, s,
                         rows, codes, scales, m, D, blocks, (T*)O, ldo);
      return launched();
    });
  // 256 rows of W and up to 8 tiles of H a block; no more than there are: 32 rows of H by
  // 200 000 x 512 codes take 37 us with 2 tiles and 47 with 8, 64 take 44 with 4 and 52 with 8
  const int nt = tiles <= 2 ? 2 : tiles <= 4 ? 4 : 8;
  const int64_t row_blocks = (D + 255) / 256;
  const int64_t grid = (row_blocks + 7) / 8 * 8 * ((tiles + nt - 1) / nt);
  if (grid > 0xFFFFFF) return LST_EINVAL;  // a launch has 2^32 threads at most
  __bf16* fragments = (__bf16*)workspace;
  hipLaunchKernelGGL(fragments_kernel<R>, dim3(tiles * blocks), dim3(256), 0, s, rows, m, blocks,
                     tiles, fragments);
  const int rc = launched();
  if (rc != LST_OK) return rc;
  return with_dtype(out_dtype, [&](auto t) {
    using T = decltype(t);
    auto run = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), 0, s, codes, scales, fragments,
                         m, D, blocks, (int)row_blocks, (T*)O, ldo);
      return launched();
    };
    if (nt == 2) return run(scores_kernel<T, 4, 2, true>);
    if (nt == 4) return run(scores_kernel<T, 4, 4, true>);
    return tiles <= 8 ? run(scores_kernel<T, 4, 8, true>) : run(scores_kernel<T, 4, 8, false>);
  });
}

}  // namespace
}  // namespace lst

using namespace lst;

extern "C" {

int lst_quantize(int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t ldx,
                 uint8_t* codes, uint8_t* scales, void* hip_stream) {
  if (!known_dtype(dtype) || rows < 0 || cols < 1 || cols > 4096) return LST_EINVAL;
  if (rows == 0) return LST_OK;
  if (!x || !codes || !scales || ldx < cols || ((uintptr_t)codes & 15)) return LST_EINVAL;
  if (rows > kMostBlocks / blocks_of(cols)) return LST_EINVAL;
  const int64_t n = (rows * blocks_of(cols) + 15) / 16;
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(quantize_kernel<T>, dim3((unsigned)n), dim3(256), 0,
                       (hipStream_t)hip_stream, (const T*)x, ldx, rows, cols,
                       (int)blocks_of(cols), codes, scales);
    return launched();
  });
}

int64_t lst_scores_workspace(int32_t m, int32_t d) {
  if (m < 0 || d < 1 || d > 4096) return -1;
  return ((int64_t)m + 15) / 16 * blocks_of(d) * kTile * (int64_t)sizeof(__bf16);
}

int lst_scores(int32_t dtype, int32_t out_dtype, int32_t m, int64_t D, int32_t d, const void* H,
               int64_t ldh, const uint8_t* codes, const uint8_t* scales, void* O, int64_t ldo,
               void* workspace, void* hip_stream) {
  if (!known_dtype(dtype)) return LST_EINVAL;
  if (m > 0 && (!H || ldh < d)) return LST_EINVAL;
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    return scores(Values<T>{(const T*)H, ldh, d}, out_dtype, m, D, d, codes, scales, O, ldo,
                  workspace, (hipStream_t)hip_stream);
  });
}

int lst_scores_coded(int32_t out_dtype, int32_t m, int64_t D, int32_t d, const uint8_t* h_codes,
                     const uint8_t* h_scales, const uint8_t* codes, const uint8_t* scales, void* O,
                     int64_t ldo, void* workspace, void* hip_stream) {
  if (m > 0 && (!h_codes || !h_scales || ((uintptr_t)h_codes & 15))) return LST_EINVAL;
  return scores(Coded{h_codes, h_scales, (int)blocks_of(d)}, out_dtype, m, D, d, codes, scales, O,
                ldo, workspace, (hipStream_t)hip_stream);
}

}  // extern "C"
