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

// exp(-|g|) = 2^t (1 + r ln 2) with -|g| log2(e) = t + r, r the product's rounding: the rounded
// product alone would cost |g| 2^-24 of the result.
__device__ inline void gate(float g, float& f, float& i) {
  const float kLog2e = 1.44269504f, kLog2eLow = 1.925963033e-8f, kLn2 = 0.693147181f;
  const float m = -fabsf(g), t = m * kLog2e;
  const float r = fmaf(m, kLog2eLow, fmaf(m, kLog2e, -t));
  float e = __builtin_amdgcn_exp2f(t);
  e = fmaf(e, r * kLn2, e);
  // -inf: t + r is not a number
  e = m < -150.f ? 0.f : e;
  const float big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
  f = g < 0.f ? small : big;
  i = g < 0.f ? big : small;
}

__device__ inline void raise(int32_t* status) {
  if (status) atomicCAS(status, 0, LST_EINDEX);
}

// Rows [b, e) of sequence s; false (and the status) when they are not rows of the call.
__device__ inline bool rows_of(const RecurArgs& a, int s, int& b, int& e) {
  if (a.offsets) {
    b = a.offsets[s];
    e = a.offsets[s + 1];
  } else {
    const int n = a.rows / a.n_seq;
    b = s * n;
    e = b + n;
  }
  if (b >= 0 && b <= e && e <= a.rows) return true;
  raise(a.status);
  return false;
}

template <class T>
__global__ __launch_bounds__(64) void recur_forward_kernel(RecurArgs a, const T* x, const T* g,
                                                           T* y) {
  const int c = blockIdx.y * 64 + threadIdx.x, s = blockIdx.x;
  int b, e;
  if (c >= a.d || !rows_of(a, s, b, e)) return;
  float h = a.h0 ? a.h0[(int64_t)s * a.d + c] : 0.f;
  for (int64_t t = b; t < e; ++t) {
    if (a.saved && t % kChunk == 0) a.saved[t / kChunk * a.d + c] = h;
    float f, i;
    gate((float)g[t * a.ldg + c], f, i);
    h = f * h + i * (float)x[t * a.ldx + c];
    y[t * a.ldy + c] = (T)h;
  }
  if (a.h_last) a.h_last[(int64_t)s * a.d + c] = h;
}

template <class T>
__global__ __launch_bounds__(64) void recur_backward_kernel(RecurArgs a, const T* x, const T* g,
                                                            const T* dy, T* dx, T* dg) {
  __shared__ float before[kChunk][64];  // the state that each row of a chunk starts from
  const int l = threadIdx.x, c = blockIdx.y * 64 + l, s = blockIdx.x;
  int b, e;
  if (c >= a.d || !rows_of(a, s, b, e)) return;
  float m = a.grad_last ? a.grad_last[(int64_t)s * a.d + c] : 0.f;
  for (int hi = e; hi > b;) {
    const int lo = max(b, (hi - 1) / kChunk * kChunk);
    float h = lo > b || lo % kChunk == 0
                  ? a.saved_in[(int64_t)(lo / kChunk) * a.d + c]
                  : (a.h0 ? a.h0[(int64_t)s * a.d + c] : 0.f);
    for (int64_t t = lo; t < hi; ++t) {
      before[t - lo][l] = h;
      float f, i;
      gate((float)g[t * a.ldg + c], f, i);
      h = f * h + i * (float)x[t * a.ldx + c];
    }
    for (int64_t t = hi - 1; t >= lo; --t) {
      float f, i;
      gate((float)g[t * a.ldg + c], f, i);
      const float L = (float)dy[t * a.ldy + c] + m;
      dx[t * a.lddx + c] = (T)(i * L);
      dg[t * a.lddg + c] = (T)((before[t - lo][l] - (float)x[t * a.ldx + c]) * (f * i) * L);
      m = f * L;
    }
    hi = lo;
  }
  if (a.grad_h0) a.grad_h0[(int64_t)s * a.d + c] = m;
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
  for (int c = blockIdx.y * 256 + threadIdx.x; c < d; c += gridDim.y * 256) {
    float f, i;
    gate((float)g[row * ldg + c], f, i);
    float* p = h + (int64_t)slot * d + c;
    const float v = f * *p + i * (float)x[row * ldx + c];
    *p = v;
    y[row * ldy + c] = (T)v;
  }
}

int check_recur(int dtype, int rows, int n_seq, int d, const void* x, int64_t ldx, const void* g,
                int64_t ldg, const int32_t* offsets) {
  if (!known_dtype(dtype) || rows < 0 || n_seq < 0 || d < 1 || d > 4096) return LST_EINVAL;
  if (n_seq == 0 && rows != 0 && !offsets) return LST_EINVAL;
  if (!offsets && n_seq && rows % n_seq) return LST_EINVAL;
  if (rows && (!x || !g || ldx < d || ldg < d)) return LST_EINVAL;
  return LST_OK;
}

}  // namespace
}  // namespace lst

using namespace lst;

extern "C" {

int64_t lst_recur_saved(int32_t rows, int32_t d) {
  return rows < 0 || d < 1 ? -1 : ((int64_t)rows + kChunk - 1) / kChunk * d;
}

int64_t lst_recur_workspace(int32_t rows, int32_t d) { return rows < 0 || d < 1 ? -1 : 0; }

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
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(recur_forward_kernel<T>, dim3(n_seq, (d + 63) / 64), dim3(64), 0,
                       (hipStream_t)hip_stream, a, (const T*)x, (const T*)g, (T*)y);
    return launched();
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
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(recur_backward_kernel<T>, dim3(n_seq, (d + 63) / 64), dim3(64), 0,
                       (hipStream_t)hip_stream, a, (const T*)x, (const T*)g, (const T*)grad_y,
                       (T*)grad_x, (T*)grad_g);
    return launched();
  });
}

int lst_recur_step(int32_t dtype, int32_t rows, int32_t n_slots, int32_t d, const void* x,
                   int64_t ldx, const void* g, int64_t ldg, const int32_t* slots, float* h,
                   void* y, int64_t ldy, int32_t* status, void* hip_stream) {
  if (!known_dtype(dtype) || rows < 0 || n_slots < 0 || d < 1 || d > 4096) return LST_EINVAL;
  if (!slots && rows > n_slots) return LST_EINVAL;
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
