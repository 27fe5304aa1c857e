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
// The rows of H are quantised in the same way by a launch of their own, and left in
// bfloat16: they are few, and every wave reads them.
#include "dtypes.h"

namespace lst {
namespace {

constexpr int kBlock = 128;

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

// Biased exponent of the scale for the bits of a block's largest finite magnitude:
// 448 = 1.75 2^8, so 1.f 2^E needs 2^(E - 8) when 1.f <= 1.75, else 2^(E - 7).
__device__ inline int scale_of(uint32_t big) {
  const int e = (int)(big >> 23) - ((big & 0x7FFFFF) <= 0x600000 ? 8 : 7);
  return max(e, 0);
}

// Codes of values times 2^(127 - e), which is exact: e is at most 254 - 7.
template <int N>
__device__ inline void codes_of(const float (&v)[N], int e, uint32_t (&q)[N / 4]) {
  const float s = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * s, v[4 * i + 1] * s, 0, false);
    q[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * s, v[4 * i + 3] * s, lo, true);
  }
}

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

// 16 lanes a block, eight columns a lane.  Bound by memory: 793 471 x 300 floats (1.26 GB
// with the codes) take 213 us, 5.9 TB/s; 32 lanes a block, four columns a lane with an access
// for each, took 305 us.  WIDE: the values in bfloat16 instead of codes.
template <class T, class I, bool WIDE>
__global__ __launch_bounds__(256) void quantize_kernel(const T* x, int64_t ldx, int64_t rows,
                                                       int cols, int blocks, void* codes,
                                                       uint8_t* scales) {
  const I at = (I)blockIdx.x * 16 + threadIdx.x / 16;  // the block
  if (at >= (I)(rows * blocks)) return;
  const I row = at / (I)blocks;
  const int l = threadIdx.x % 16, col = (int)(at - row * (I)blocks) * kBlock + 8 * l;
  const T* p = x + (int64_t)row * ldx + col;
  T raw[8];
  if (col + 8 <= cols) {
    load_vec(p, raw);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i] = col + i < cols ? p[i] : (T)0.f;
  }
  float v[8];
  uint32_t big = 0;  // largest magnitude, by its bits
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = (float)raw[i];
    big = max(big, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  }
  uint64_t bad = 0;  // lanes' bytes that are no number in e4m3
  if (big >= 0x7F800000u) {
    big = 0;
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = __float_as_uint(v[i]) & 0x7FFFFFFFu;
      if (b >= 0x7F800000u) {
        bad |= (uint64_t)0x7F << (8 * i);
        v[i] = 0.f;
      } else {
        big = max(big, b);
      }
    }
  }
#pragma unroll
  for (int o = 8; o; o >>= 1) big = max(big, (uint32_t)__shfl_xor((int)big, o));
  const int e = scale_of(big);
  uint32_t q[2];
  codes_of(v, e, q);
  q[0] |= (uint32_t)bad;
  q[1] |= (uint32_t)(bad >> 32);
  if constexpr (WIDE) {
    reinterpret_cast<bf16x8*>(codes)[(int64_t)at * 16 + l] =
        widen(uintx2{q[0], q[1]}, scale_value(e));
  } else {
    reinterpret_cast<uintx2*>(codes)[(int64_t)at * 16 + l] = uintx2{q[0], q[1]};
    if (l == 0) scales[at] = (uint8_t)e;
  }
}

// 16 rows of W and 16 NT rows of H a wave; four waves a block on neighbouring rows.
template <class T, int NT>
__global__ __launch_bounds__(256) void scores_kernel(const uint8_t* W, const uint8_t* sw,
                                                     const __bf16* H, int m, int64_t D,
                                                     int blocks, T* O, int64_t ldo) {
  const int l = threadIdx.x % 64, i16 = l % 16, q = l / 16;
  const int64_t r0 = ((int64_t)blockIdx.x * 4 + threadIdx.x / 64) * 16;
  const int n0 = blockIdx.y * 16 * NT;
  if (r0 >= D) return;
  const int64_t row = min(r0 + i16, D - 1);
  const int64_t ld = (int64_t)blocks * kBlock;
  floatx4 acc[NT] = {};
  for (int b = 0; b < blocks; ++b) {
    // the order of k within a block is free as long as both sides have the same
    const uint8_t* w = W + row * ld + b * kBlock + 16 * q;
    const uintx4 lo = *reinterpret_cast<const uintx4*>(w);
    const uintx4 hi = *reinterpret_cast<const uintx4*>(w + 64);
    const float e = scale_value(sw[row * blocks + b]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uintx4 c = k < 2 ? lo : hi;
      const bf16x8 a = widen(uintx2{c[k % 2 * 2], c[k % 2 * 2 + 1]}, e);
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int n = min(n0 + 16 * j + i16, m - 1);
        const bf16x8 h = *reinterpret_cast<const bf16x8*>(H + n * ld + b * kBlock + 16 * q +
                                                          8 * (k % 2) + 64 * (k / 2));
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, h, acc[j], 0, 0, 0);
      }
    }
  }
  for (int j = 0; j < NT; ++j) {
    const int n = n0 + 16 * j + i16;
    if (n >= m) break;
    T* o = O + n * ldo + r0 + 4 * q;
    const int have = (int)min((int64_t)4, D - r0 - 4 * q);
    for (int i = 0; i < have; ++i) o[i] = (T)acc[j][i];
  }
}

int64_t blocks_of(int32_t cols) { return ((int64_t)cols + kBlock - 1) / kBlock; }

template <bool WIDE>
int quantize(int dtype, int64_t rows, int32_t cols, const void* x, int64_t ldx, void* codes,
             uint8_t* scales, hipStream_t s) {
  const int64_t blocks = rows * blocks_of(cols), n = (blocks + 15) / 16;
  if (n > 0x7FFFFFFF) return LST_EINVAL;
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    auto run = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(256), 0, s, (const T*)x, ldx, rows, cols,
                         (int)blocks_of(cols), codes, scales);
    };
    blocks <= 0x7FFFFFFF ? run(quantize_kernel<T, uint32_t, WIDE>)
                         : run(quantize_kernel<T, int64_t, WIDE>);
    return launched();
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
  return quantize<false>(dtype, rows, cols, x, ldx, codes, scales, (hipStream_t)hip_stream);
}

int64_t lst_scores_workspace(int32_t m, int32_t d) {
  if (m < 0 || d < 1 || d > 4096) return -1;
  return m * blocks_of(d) * kBlock * (int64_t)sizeof(__bf16);
}

int lst_scores(int32_t dtype, int32_t out_dtype, int32_t m, int64_t D, int32_t d, const void* H,
               int64_t ldh, const uint8_t* codes, const uint8_t* scales, void* O, int64_t ldo,
               void* workspace, void* hip_stream) {
  if (!known_dtype(dtype) || !known_dtype(out_dtype) || m < 0 || D < 1 || d < 1 || d > 4096)
    return LST_EINVAL;
  if (m == 0) return LST_OK;
  if (!H || !codes || !scales || !O || !workspace || ldh < d || ldo < D) return LST_EINVAL;
  if (((uintptr_t)codes & 15) || ((uintptr_t)workspace & 15)) return LST_EINVAL;
  const int64_t groups = (D + 63) / 64;
  if (groups > 0x7FFFFFFF) return LST_EINVAL;
  hipStream_t s = (hipStream_t)hip_stream;
  const int blocks = (int)blocks_of(d);
  int rc = quantize<true>(dtype, m, d, H, ldh, workspace, nullptr, s);
  if (rc != LST_OK) return rc;
  return with_dtype(out_dtype, [&](auto t) {
    using T = decltype(t);
    auto run = [&](auto kernel, int nt) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)groups, (m + 16 * nt - 1) / (16 * nt)), dim3(256),
                         0, s, codes, scales, (const __bf16*)workspace, m, D, blocks, (T*)O, ldo);
    };
    m <= 16 ? run(scores_kernel<T, 1>, 1) : run(scores_kernel<T, 4>, 4);
    return launched();
  });
}

}  // extern "C"
