// Root-mean-square norm of rows (lst_norm_forward, lst_norm_backward), with the residual's
// addition before it and, for rows on their way to outputs from 8 bits, codes behind it.
//
//   s = x + r,  q = 1 / sqrt(mean(s^2) + eps),  y = q s w
//   a = dy w,   dx = q (a - q s mean(a q s)) + ds,   dw = sum over the rows of dy q s
//
// A row is held in registers by 16, 32, 64 or 256 neighbouring lanes, eight columns a lane and
// group, so that each matrix is read once and written once.  The squares are summed in float64: no row
// overflows it, and the factor is the same whichever lanes hold the row.
#include <algorithm>

#include "dtypes.h"
#include "eight_bit.h"

namespace lst {
namespace {

constexpr int kCols = 4096;
constexpr int kPartials = 512;  // blocks of the backward pass, and rows of its partial sums

// Sum over the lanes that share a row; 256 of them are the whole block, whose waves leave their
// sums in `lds` (eight of them, two sets in turn, so that one barrier a sum is enough).
template <int LANES, class S>
__device__ inline S sum_lanes(S v, S* lds, int& turn) {
  constexpr int kWave = LANES < 64 ? LANES : 64;
#pragma unroll
  for (int o = kWave / 2; o; o >>= 1) v += __shfl_xor(v, o);
  if constexpr (LANES > 64) {
    S* at = lds + 4 * turn;
    turn ^= 1;
    if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = v;
    __syncthreads();
    v = at[0] + at[1] + at[2] + at[3];
  }
  return v;
}

template <class T>
__device__ inline void store_part(T* row, int col, int cols, const T (&v)[8]) {
  if (col + 8 <= cols) {
    store_vec(row + col, v);
  } else {
    for (int i = 0; i < 8; ++i)
      if (col + i < cols) row[col + i] = v[i];
  }
}

struct ForwardArgs {
  int64_t rows, ldx, ldr, lds, ldy;
  int cols, blocks;
  double eps;
  const float* weight;
  float* rstd;
  uint8_t *codes, *scales;
};

// LANES lanes a row, GROUPS groups of eight columns a lane.
template <class T, int LANES, int GROUPS, bool CODED>
__global__ __launch_bounds__(256) void forward_kernel(ForwardArgs a, const T* x, const T* r, T* s,
                                                      T* y) {
  constexpr int kRows = 256 / LANES;  // of a block
  __shared__ double sums[8];
  int turn = 0;
  const int l = threadIdx.x % LANES;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; row < a.rows;
       row += (int64_t)gridDim.x * kRows) {
    T raw[GROUPS][8], res[GROUPS][8];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) load_part(x + row * a.ldx, (g * LANES + l) * 8, a.cols, raw[g]);
    if (r) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) load_part(r + row * a.ldr, (g * LANES + l) * 8, a.cols, res[g]);
#pragma unroll
      for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        // the norm is of the sum as it is stored, which is what the backward pass reads
        for (int i = 0; i < 8; ++i) raw[g][i] = (T)((float)raw[g][i] + (float)res[g][i]);
    }
    double sum = 0;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double v = (float)raw[g][i];
        sum = fma(v, v, sum);
      }
    sum = sum_lanes<LANES>(sum, sums, turn);
    const double q = 1.0 / sqrt(sum / a.cols + a.eps);
    if (l == 0 && a.rstd) a.rstd[row] = (float)q;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int col = (g * LANES + l) * 8;
      float w[8];
      load_part(a.weight, col, a.cols, w);
      if (s) store_part(s + row * a.lds, col, a.cols, raw[g]);
      if constexpr (CODED) {
        // in float64: a value that float32's roundings move over a border of the codes would
        // be off by a sixteenth
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)  // zeros behind the last column, also where q is no number
          v[i] = col + i < a.cols ? (float)((double)(float)raw[g][i] * q * (double)w[i]) : 0.f;
        uint32_t code[2];
        int e;
        values_codes(v, code, e);
        const int block = col / kBlock;
        if (block < a.blocks) {
          const int64_t at = row * a.blocks + block;
          reinterpret_cast<uintx2*>(a.codes)[at * 16 + l % 16] = uintx2{code[0], code[1]};
          if (l % 16 == 0) a.scales[at] = (uint8_t)e;
        }
      }
      if (y) {
        T out[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = (T)((float)raw[g][i] * (float)q * w[i]);
        store_part(y + row * a.ldy, col, a.cols, out);
      }
    }
  }
}

struct BackwardArgs {
  int64_t rows, lds, ldgy, ldgs, ldgx;
  int cols;
  const float *weight, *rstd;
  float* partial;  // gridDim.x rows of cols
};

// Eight waves a block; one row of the widest.
constexpr int threads_of(int lanes) { return lanes > 64 ? lanes : 512; }

// A wave goes through rows by itself and keeps its sums for dw in registers; the waves' sums are
// added in order in LDS, the blocks' by sum_kernel: no order depends on timing.
template <class T, int LANES, int GROUPS>
__global__ __launch_bounds__(threads_of(LANES)) void backward_kernel(BackwardArgs a, const T* s, const T* gy,
                                                       const T* gs, T* gx) {
  constexpr int kThreads = threads_of(LANES), kRows = kThreads / LANES;
  __shared__ float lds[LANES * GROUPS * 8], sums[8];
  int turn = 0;
  const int l = threadIdx.x % LANES;
  float dw[GROUPS][8] = {};
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; row < a.rows;
       row += (int64_t)gridDim.x * kRows) {
    T rs[GROUPS][8], ry[GROUPS][8], rd[GROUPS][8];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int col = (g * LANES + l) * 8;
      load_part(s + row * a.lds, col, a.cols, rs[g]);
      load_part(gy + row * a.ldgy, col, a.cols, ry[g]);
      if (gs) load_part(gs + row * a.ldgs, col, a.cols, rd[g]);
    }
    const float q = a.rstd[row];
    float inner = 0.f;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      float w[8];
      load_part(a.weight, (g * LANES + l) * 8, a.cols, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) inner = fmaf((float)ry[g][i] * w[i], (float)rs[g][i] * q, inner);
    }
    inner = sum_lanes<LANES>(inner, sums, turn) / a.cols;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int col = (g * LANES + l) * 8;
      float w[8];
      load_part(a.weight, col, a.cols, w);
      T out[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float hat = (float)rs[g][i] * q, dy = (float)ry[g][i];
        float v = q * (dy * w[i] - hat * inner);
        if (gs) v += (float)rd[g][i];
        out[i] = (T)v;
        dw[g][i] = fmaf(dy, hat, dw[g][i]);
      }
      store_part(gx + row * a.ldgx, col, a.cols, out);
    }
  }
#pragma unroll
  for (int g = 0; g < GROUPS; ++g)
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int o = LANES; o < 64; o <<= 1) dw[g][i] += __shfl_xor(dw[g][i], o);
  const int wave = threadIdx.x / 64;
  for (int k = 0; k < kThreads / 64; ++k) {
    if (wave == k && (LANES > 64 || threadIdx.x % 64 < LANES)) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float* p = lds + (g * LANES + l) * 8 + i;
          *p = k && LANES <= 64 ? *p + dw[g][i] : dw[g][i];
        }
    }
    __syncthreads();
  }
  for (int c = threadIdx.x; c < a.cols; c += kThreads)
    a.partial[(int64_t)blockIdx.x * a.cols + c] = lds[c];
}

// Column sums of the blocks' partial sums: 64 columns a block, 16 parts of the rows.
__global__ __launch_bounds__(1024) void sum_kernel(const float* partial, int n, int cols,
                                                   float* out) {
  __shared__ float lds[16][64];
  const int c = blockIdx.x * 64 + threadIdx.x % 64, part = threadIdx.x / 64;
  float v = 0.f;
  if (c < cols)
    for (int i = part; i < n; i += 16) v += partial[(int64_t)i * cols + c];
  lds[part][threadIdx.x % 64] = v;
  __syncthreads();
  if (part == 0 && c < cols) {
    for (int i = 1; i < 16; ++i) v += lds[i][threadIdx.x];
    out[c] = v;
  }
}

// Calls f with the lanes that share a row, and the groups of eight columns of each.
template <class F>
int with_shape(int cols, F f) {
  using std::integral_constant;
  integral_constant<int, 1> one;
  integral_constant<int, 2> two;
  if (cols <= 128) return f(integral_constant<int, 16>{}, one);
  if (cols <= 256) return f(integral_constant<int, 32>{}, one);
  if (cols <= 512) return f(integral_constant<int, 64>{}, one);
  if (cols <= 1024) return f(integral_constant<int, 64>{}, two);
  if (cols <= 2048) return f(integral_constant<int, 256>{}, one);
  return f(integral_constant<int, 256>{}, two);
}

int lanes_of(int cols) { return cols <= 128 ? 16 : cols <= 256 ? 32 : cols <= 1024 ? 64 : 256; }

int partials_of(int64_t rows, int cols) {
  const int lanes = lanes_of(cols), per = threads_of(lanes) / lanes;
  return (int)std::min<int64_t>((rows + per - 1) / per, kPartials);
}

constexpr int64_t kMostRows = (int64_t)1 << 40;

}  // namespace
}  // namespace lst

using namespace lst;

extern "C" {

int lst_norm_forward(int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t ldx,
                     const void* residual, int64_t ldr, const float* weight, double eps, void* sum,
                     int64_t lds, void* y, int64_t ldy, uint8_t* codes, uint8_t* scales,
                     float* rstd, void* hip_stream) {
  if (!known_dtype(dtype) || rows < 0 || rows > kMostRows || cols < 1 || cols > kCols)
    return LST_EINVAL;
  if (!(eps >= 0x1p-100 && eps <= 0x1p100)) return LST_EINVAL;
  if (rows == 0) return LST_OK;
  if (!x || !weight || ldx < cols || (residual && ldr < cols) || (sum && lds < cols))
    return LST_EINVAL;
  if ((!y && !codes) || (y && (ldy < cols || y == sum)) || !codes != !scales) return LST_EINVAL;
  if ((uintptr_t)codes & 15) return LST_EINVAL;
  ForwardArgs a{rows, ldx, ldr, lds, ldy, cols, (cols + kBlock - 1) / kBlock, eps, weight,
                rstd, codes, scales};
  const int per = 256 / lanes_of(cols);
  const unsigned grid = (unsigned)std::min<int64_t>((rows + per - 1) / per, 1 << 20);
  return with_dtype(dtype, [&](auto t) {
    return with_shape(cols, [&](auto lanes, auto groups) {
      using T = decltype(t);
      auto run = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, (hipStream_t)hip_stream, a,
                           (const T*)x, (const T*)residual, (T*)sum, (T*)y);
        return launched();
      };
      return codes ? run(forward_kernel<T, lanes, groups, true>)
                   : run(forward_kernel<T, lanes, groups, false>);
    });
  });
}

int64_t lst_norm_workspace(int64_t rows, int32_t cols) {
  if (rows < 0 || rows > kMostRows || cols < 1 || cols > kCols) return -1;
  return (int64_t)partials_of(rows, cols) * cols * (int64_t)sizeof(float);
}

int lst_norm_backward(int32_t dtype, int64_t rows, int32_t cols, const void* sum, int64_t lds,
                      const float* weight, const float* rstd, const void* grad_y, int64_t ldgy,
                      const void* grad_sum, int64_t ldgs, void* grad_x, int64_t ldgx,
                      float* grad_weight, void* workspace, void* hip_stream) {
  if (!known_dtype(dtype) || rows < 0 || rows > kMostRows || cols < 1 || cols > kCols)
    return LST_EINVAL;
  if (!weight || !grad_weight) return LST_EINVAL;
  if (rows > 0 && (!sum || !rstd || !grad_y || !grad_x || !workspace || lds < cols ||
                   ldgy < cols || ldgx < cols || (grad_sum && ldgs < cols)))
    return LST_EINVAL;
  if ((uintptr_t)workspace & 15) return LST_EINVAL;
  hipStream_t stream = (hipStream_t)hip_stream;
  const int n = partials_of(rows, cols);
  float* partial = n == 1 ? grad_weight : (float*)workspace;
  if (n > 0) {
    BackwardArgs a{rows, lds, ldgy, ldgs, ldgx, cols, weight, rstd, partial};
    const int rc = with_dtype(dtype, [&](auto t) {
      return with_shape(cols, [&](auto lanes, auto groups) {
        using T = decltype(t);
        hipLaunchKernelGGL((backward_kernel<T, lanes, groups>), dim3(n), dim3(threads_of(lanes)), 0, stream, a,
                           (const T*)sum, (const T*)grad_y, (const T*)grad_sum, (T*)grad_x);
        return launched();
      });
    });
    if (rc != LST_OK || n == 1) return rc;
  }
  hipLaunchKernelGGL(sum_kernel, dim3((cols + 63) / 64), dim3(1024), 0, stream, partial, n, cols,
                     grad_weight);
  return launched();
}

}  // extern "C"
