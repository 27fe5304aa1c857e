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

// Biased exponent of the scale for a block's largest finite magnitude:
// 448 = 1.75 2^8, so 1.f 2^E needs 2^(E - 8) when 1.f <= 1.75, else 2^(E - 7).
__device__ inline int scale_of(float big) {
  const uint32_t b = __float_as_uint(big);
  const int e = (int)(b >> 23) - ((b & 0x7FFFFF) <= 0x600000 ? 8 : 7);
  return max(e, 0);
}

__device__ inline uint32_t code4(const float (&v)[4], int e) {
  float w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = ldexpf(v[i], 127 - e);
  int q = __builtin_amdgcn_cvt_pk_fp8_f32(w[0], w[1], 0, false);
  q = __builtin_amdgcn_cvt_pk_fp8_f32(w[2], w[3], q, true);
#pragma unroll
  for (int i = 0; i < 4; ++i)  // what is not finite is no number in e4m3
    if (!isfinite(v[i])) q |= 0x7F << (8 * i);
  return (uint32_t)q;
}

__device__ inline float scale_value(int e) {
  return __uint_as_float(e ? (uint32_t)e << 23 : 0x400000u);  // 2^(e - 127)
}

// Half a wave a block, four columns a lane.  WIDE: the values in bfloat16 instead of codes.
template <class T, bool WIDE>
__global__ __launch_bounds__(256) void quantize_kernel(const T* x, int64_t ldx, int64_t rows,
                                                       int cols, int blocks, void* codes,
                                                       uint8_t* scales) {
  const int64_t at = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;  // the block
  if (at >= rows * blocks) return;
  const int64_t row = at / blocks;
  const int l = threadIdx.x % 32, col = (int)(at - row * blocks) * kBlock + 4 * l;
  float v[4], big = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = col + i < cols ? (float)x[row * ldx + col + i] : 0.f;
    if (isfinite(v[i])) big = fmaxf(big, fabsf(v[i]));
  }
  for (int o = 16; o; o >>= 1) big = fmaxf(big, __shfl_xor(big, o));
  const int e = scale_of(big);
  const uint32_t q = code4(v, e);
  if constexpr (WIDE) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale_value(e), false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale_value(e), true);
    reinterpret_cast<bf16x4*>(codes)[at * 32 + l] = bf16x4{lo[0], lo[1], hi[0], hi[1]};
  } else {
    reinterpret_cast<uint32_t*>(codes)[at * 32 + l] = q;
    if (l == 0) scales[at] = (uint8_t)e;
  }
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
  const int64_t n = (rows * blocks_of(cols) + 7) / 8;
  if (n > 0x7FFFFFFF) return LST_EINVAL;
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL((quantize_kernel<T, WIDE>), dim3((unsigned)n), dim3(256), 0, s,
                       (const T*)x, ldx, rows, cols, (int)blocks_of(cols), codes, scales);
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
