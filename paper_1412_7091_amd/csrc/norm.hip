// Root-mean-square norm of rows (lst_norm_forward, lst_norm_backward), with the residual's
// addition before it and, for rows on their way to outputs from 8 bits, codes behind it.
//
//   s = x + r,  q = 1 / sqrt(mean(s^2) + eps),  y = q s w
//   a = dy w,   dx = q (a - q s mean(a q s)) + ds,   dw = sum over the rows of dy q s
//
// A row is held in registers by 16, 32, 64 or 256 neighbouring lanes, eight columns a lane and
// group, so that each matrix is read once and written once.  The squares are summed in float64: no row
// overflows it, and the factor is the same whichever lanes hold the row.
//
// Bound by memory: 65 536 x 1024 bfloat16 with a residual (537 MB each way) take 89 us forwards
// and 104 backwards, 6.0 and 5.2 TB/s (backwards without the next row's loads under way 188);
// 65 536 x 500 (262 MB) 44 and 52; 8191 x 500 float32 (66 MB) 15 us each way.
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

// Eight columns of a row as they are in memory (16 bits: four registers).
template <class T>
using Eight = T __attribute__((ext_vector_type(8)));

template <class T, int N>
using At = T __attribute__((ext_vector_type(N), aligned(sizeof(T))));

// How a row's columns fall on eights: all of them do (kWhole); the last lane takes the row's last
// eight, of which it shares the first `skip` with the lane before (kShared: they count once in the
// sums, and both write the same); or the row has fewer than eight (kTiny).  A lane that reads one
// to seven columns by themselves waits for them before it can read on: 65 536 rows of 500 in
// bfloat16 took 56 and 75 us so, and now take 44 and 52.
enum { kWhole, kShared, kTiny };

struct Columns {
  int at, skip;  // skip = 8: none
};
template <int MODE>
__device__ inline Columns columns_of(int col, int cols) {
  if (MODE == kShared && col < cols && col + 8 > cols) return {cols - 8, col - (cols - 8)};
  return {col, col < cols ? 0 : 8};
}

template <int MODE, class T>
__device__ inline Eight<T> load_eight(const T* row, Columns c, int cols) {
  Eight<T> v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (T)0.f;
  if (c.skip == 8) return v;
  if constexpr (MODE == kTiny) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < cols) v[i] = row[i];
  } else {
    v = *reinterpret_cast<const At<T, 8>*>(row + c.at);
  }
  return v;
}

template <int MODE, class T>
__device__ inline void store_eight(T* row, Columns c, int cols, Eight<T> v) {
  if (c.skip == 8) return;
  if constexpr (MODE == kTiny) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < cols) row[i] = v[i];
  } else {
    *reinterpret_cast<At<T, 8>*>(row + c.at) = v;
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
template <class T, int LANES, int GROUPS, int MODE, bool CODED>
__global__ __launch_bounds__(256) void forward_kernel(ForwardArgs a, const T* x, const T* r, T* s,
                                                      T* y) {
  constexpr int kRows = 256 / LANES;  // of a block
  __shared__ double sums[8];
  int turn = 0;
  const int l = threadIdx.x % LANES;
  Columns c[GROUPS];
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) c[g] = columns_of<MODE>((g * LANES + l) * 8, a.cols);
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; row < a.rows;
       row += (int64_t)gridDim.x * kRows) {
    Eight<T> v[GROUPS], res[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) v[g] = load_eight<MODE>(x + row * a.ldx, c[g], a.cols);
    if (r) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) res[g] = load_eight<MODE>(r + row * a.ldr, c[g], a.cols);
#pragma unroll
      for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        // the norm is of the sum as it is stored, which is what the backward pass reads
        for (int i = 0; i < 8; ++i) v[g][i] = (T)((float)v[g][i] + (float)res[g][i]);
    }
    double sum = 0;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double f = MODE == kShared && i < c[g].skip ? 0.f : (float)v[g][i];
        sum = fma(f, f, sum);
      }
    sum = sum_lanes<LANES>(sum, sums, turn);
    const double q = 1.0 / sqrt(sum / a.cols + a.eps);
    if (l == 0 && a.rstd) a.rstd[row] = (float)q;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const Eight<float> w = load_eight<MODE>(a.weight, c[g], a.cols);
      if (s) store_eight<MODE>(s + row * a.lds, c[g], a.cols, v[g]);
      if constexpr (CODED) {
        // in float64: a value that float32's roundings move over a border of the codes would
        // be off by a sixteenth
        const int col = (g * LANES + l) * 8, move = MODE == kShared ? c[g].skip : 0;
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)((double)(float)v[g][i] * q * (double)w[i]);
        if constexpr (MODE == kShared) {  // the lane's own columns to the front
#pragma unroll
          for (int o = 4; o; o >>= 1)
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (move & o) f[i] = i + o < 8 ? f[i + o] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)  // zeros behind the last column, also where q is no number
          f[i] = col + i < a.cols ? f[i] : 0.f;
        uint32_t code[2];
        int e;
        values_codes(f, code, e);
        const int block = col / kBlock;
        if (block < a.blocks) {
          const int64_t at = row * a.blocks + block;
          reinterpret_cast<uintx2*>(a.codes)[at * 16 + l % 16] = uintx2{code[0], code[1]};
          if (l % 16 == 0) a.scales[at] = (uint8_t)e;
        }
      }
      if (y) {
        Eight<T> out;
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = (T)((float)v[g][i] * (float)q * w[i]);
        store_eight<MODE>(y + row * a.ldy, c[g], a.cols, out);
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

// A wave goes through rows by itself, the next one's loads under way, and keeps its sums for dw
// in registers; the waves' sums are added in order in LDS, the blocks' by sum_kernel: no order
// depends on timing.
template <class T, int LANES, int GROUPS, int MODE>
__global__ __launch_bounds__(threads_of(LANES)) void backward_kernel(BackwardArgs a, const T* s,
                                                                     const T* gy, const T* gs,
                                                                     T* gx) {
  constexpr int kThreads = threads_of(LANES), kRows = kThreads / LANES;
  __shared__ float lds[LANES * GROUPS * 8], sums[8];
  int turn = 0;
  const int l = threadIdx.x % LANES;
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
  Columns c[GROUPS];
  Eight<float> w[GROUPS], dw[GROUPS] = {};
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) {
    c[g] = columns_of<MODE>((g * LANES + l) * 8, a.cols);
    w[g] = load_eight<MODE>(a.weight, c[g], a.cols);
  }
  struct Row {
    Eight<T> s[GROUPS], y[GROUPS], d[GROUPS];
    float q;
  };
  auto load = [&](int64_t row) {
    Row r;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      r.s[g] = load_eight<MODE>(s + row * a.lds, c[g], a.cols);
      r.y[g] = load_eight<MODE>(gy + row * a.ldgy, c[g], a.cols);
      if (gs) r.d[g] = load_eight<MODE>(gs + row * a.ldgs, c[g], a.cols);
    }
    r.q = a.rstd[row];
    return r;
  };
  Row next;
  if (row < a.rows) next = load(row);
  for (; row < a.rows; row += step) {
    const Row r = next;
    if (row + step < a.rows) next = load(row + step);
    float inner = 0.f;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float hat = (float)r.s[g][i] * r.q;
        // columns that the lane before has count there
        const float dy = MODE == kShared && i < c[g].skip ? 0.f : (float)r.y[g][i];
        inner = fmaf(dy * w[g][i], hat, inner);
        dw[g][i] = fmaf(dy, hat, dw[g][i]);
      }
    inner = sum_lanes<LANES>(inner, sums, turn) / a.cols;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      Eight<T> out;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float hat = (float)r.s[g][i] * r.q;
        float v = r.q * ((float)r.y[g][i] * w[g][i] - hat * inner);
        if (gs) v += (float)r.d[g][i];
        out[i] = (T)v;
      }
      store_eight<MODE>(gx + row * a.ldgx, c[g], a.cols, out);
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
          if (c[g].skip == 8 || (MODE == kShared && i < c[g].skip)) continue;
          float* p = lds + c[g].at + i;
          *p = k && LANES <= 64 ? *p + dw[g][i] : dw[g][i];
        }
    }
    __syncthreads();
  }
  for (int c = threadIdx.x; c < a.cols; c += kThreads)
    a.partial[(int64_t)blockIdx.x * a.cols + c] = lds[c];
}

// Column sums of the blocks' partial sums: 16 columns a block, 64 parts of the rows, whose loads
// do not wait for each other.
__global__ __launch_bounds__(1024) void sum_kernel(const float* partial, int n, int cols,
                                                   float* out) {
  __shared__ float lds[64][16];
  const int l = threadIdx.x % 16, c = blockIdx.x * 16 + l, part = threadIdx.x / 16;
  float v[kPartials / 64];
#pragma unroll
  for (int i = 0; i < kPartials / 64; ++i) {
    const int row = part + 64 * i;
    v[i] = c < cols && row < n ? partial[(int64_t)row * cols + c] : 0.f;
  }
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < kPartials / 64; ++i) sum += v[i];
  lds[part][l] = sum;
  __syncthreads();
  if (part < 4) {
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += lds[part * 16 + i][l];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (part == 0 && c < cols) out[c] = sum;
  }
}

// Calls f with the lanes that share a row, the groups of eight columns of each, and how the
// columns fall on them.
template <class F>
int with_shape(int cols, F f) {
  using std::integral_constant;
  integral_constant<int, 1> one;
  integral_constant<int, 2> two;
  integral_constant<int, 16> few;
  if (cols < 8) return f(few, one, integral_constant<int, kTiny>{});
  auto whole = [&](auto mode) {
    if (cols <= 128) return f(few, one, mode);
    if (cols <= 256) return f(integral_constant<int, 32>{}, one, mode);
    if (cols <= 512) return f(integral_constant<int, 64>{}, one, mode);
    if (cols <= 1024) return f(integral_constant<int, 64>{}, two, mode);
    if (cols <= 2048) return f(integral_constant<int, 256>{}, one, mode);
    return f(integral_constant<int, 256>{}, two, mode);
  };
  return cols % 8 ? whole(integral_constant<int, kShared>{})
                  : whole(integral_constant<int, kWhole>{});
}

int lanes_of(int cols) { return cols <= 128 ? 16 : cols <= 256 ? 32 : cols <= 1024 ? 64 : 256; }

int partials_of(int64_t rows, int cols) {
  const int lanes = lanes_of(cols), per = threads_of(lanes) / lanes;
  return (int)std::min<int64_t>((rows + per - 1) / per, kPartials);
}

constexpr int64_t kMostRows = (int64_t)1 << 40;

// Whether a matrix may be written while another is read: it is another one, or the same rows.
bool may_be(const void* out, int64_t ldo, const void* in, int64_t ld, int64_t rows) {
  return out != in || ldo == ld || rows <= 1;
}

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
  for (int i = 0; i < 2; ++i) {
    const void *out = i ? y : sum, *in[2] = {x, residual};
    const int64_t ldo = i ? ldy : lds, ld[2] = {ldx, ldr};
    for (int j = 0; j < 2; ++j)
      if (out && !may_be(out, ldo, in[j], ld[j], rows)) return LST_EINVAL;
  }
  ForwardArgs a{rows, ldx, ldr, lds, ldy, cols, (cols + kBlock - 1) / kBlock, eps, weight,
                rstd, codes, scales};
  const int per = 256 / lanes_of(cols);
  const unsigned grid = (unsigned)std::min<int64_t>((rows + per - 1) / per, 1 << 20);
  return with_dtype(dtype, [&](auto t) {
    return with_shape(cols, [&](auto lanes, auto groups, auto mode) {
      using T = decltype(t);
      auto run = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, (hipStream_t)hip_stream, a,
                           (const T*)x, (const T*)residual, (T*)sum, (T*)y);
        return launched();
      };
      return codes ? run(forward_kernel<T, lanes, groups, mode, true>)
                   : run(forward_kernel<T, lanes, groups, mode, false>);
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
  if (rows > 0 && (!may_be(grad_x, ldgx, sum, lds, rows) ||
                   !may_be(grad_x, ldgx, grad_y, ldgy, rows) ||
                   !may_be(grad_x, ldgx, grad_sum, ldgs, rows)))
    return LST_EINVAL;
  hipStream_t stream = (hipStream_t)hip_stream;
  const int n = partials_of(rows, cols);
  float* partial = n == 1 ? grad_weight : (float*)workspace;
  if (n > 0) {
    BackwardArgs a{rows, lds, ldgy, ldgs, ldgx, cols, weight, rstd, partial};
    const int rc = with_dtype(dtype, [&](auto t) {
      return with_shape(cols, [&](auto lanes, auto groups, auto mode) {
        using T = decltype(t);
        auto run = [&](auto kernel) {
          hipLaunchKernelGGL(kernel, dim3(n), dim3(threads_of(lanes)), 0, stream, a,
                             (const T*)sum, (const T*)grad_y, (const T*)grad_sum, (T*)grad_x);
          return launched();
        };
        return run(backward_kernel<T, lanes, groups, mode>);
      });
    });
    if (rc != LST_OK || n == 1) return rc;
  }
  hipLaunchKernelGGL(sum_kernel, dim3((cols + 15) / 16), dim3(1024), 0, stream, partial, n, cols,
                     grad_weight);
  return launched();
}

}  // extern "C"
