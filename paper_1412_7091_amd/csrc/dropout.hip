// Dropout from a counter-based generator (lst_dropout): the mask of an element
// is a function of (seed, offset, row, column) and is drawn again wherever it is
// needed, so that no mask is stored between the forward and the backward pass.
//
// The generator is Philox4x32 with ten rounds (Salmon, Moraes, Dror and Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", 2011): a block of four words
// from a counter of four words and a key of two.  Eight neighbouring columns
// share a block, 16 bits each: with 32 bits an element the twenty 32 x 32 bit
// products of a block would cost more time than the element's memory accesses.
//
// Bound by memory: 65 536 x 1024 bfloat16, forward with a residual and backward
// (671 MB) take 130 us, 5.15 TB/s, where a copy of 1 GiB reaches 5.1.  One group a
// thread with an access for each element took 369 us.
#include "dtypes.h"

namespace lst {
namespace {

constexpr int kGroup = 8;     // columns that share a block of random words
constexpr int kThreads = 256;
constexpr int kItems = 4;     // groups a thread

struct Words {
  uint32_t w[4];
};

__device__ inline Words philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0,
                               uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)b;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}

struct DropoutArgs {
  int64_t rows;
  int cols, groups;  // groups: blocks of random words a row
  int64_t ldx, ldr, ldy;
  uint32_t drop;  // an element is kept when its 16 bits are at least this
  float factor;
  uint64_t seed, offset;
  const uint64_t* counter;
};

// kItems groups of eight columns a thread, each thread's kThreads groups apart: the
// loads of all of them are under way before the first block of words is drawn.
// I: the integer that counts the call's groups (division by 32 bits is far shorter).
template <class T, class I, bool RES, bool WHOLE>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutArgs a, const T* x,
                                                           const T* res, T* y) {
  const I total = (I)(a.rows * a.groups);
  const uint64_t off = a.offset + (a.counter ? *a.counter : 0);
  const I first = (I)blockIdx.x * (kThreads * kItems) + threadIdx.x;
  T v[kItems][kGroup], r[kItems][kGroup];
  I row[kItems];
  int group[kItems];
#pragma unroll
  for (int j = 0; j < kItems; ++j) {
    const I at = first + j * kThreads;
    row[j] = at / (I)a.groups;
    group[j] = (int)(at - row[j] * (I)a.groups);
    if (at >= total) continue;
    const int col = group[j] * kGroup;
    const T *px = x + (int64_t)row[j] * a.ldx, *pr = res + (int64_t)row[j] * a.ldr;
    const int cols = WHOLE ? col + kGroup : a.cols;
    load_part(px, col, cols, v[j]);
    if (RES) load_part(pr, col, cols, r[j]);
  }
#pragma unroll
  for (int j = 0; j < kItems; ++j) {
    const I at = first + j * kThreads;
    if (at >= total) break;
    const Words w = philox((uint32_t)group[j], (uint32_t)row[j], (uint32_t)off,
                           (uint32_t)(off >> 32), (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
    T out[kGroup];
#pragma unroll
    for (int i = 0; i < kGroup; ++i) {
      const uint32_t bits = i & 1 ? w.w[i >> 1] >> 16 : w.w[i >> 1] & 0xFFFFu;
      // a dropped element is zero whatever it holds, also when it is not finite
      float f = bits >= a.drop ? (float)v[j][i] * a.factor : 0.f;
      if (RES) f += (float)r[j][i];
      out[i] = (T)f;
    }
    const int col = group[j] * kGroup;
    T* py = y + (int64_t)row[j] * a.ldy + col;
    if (WHOLE || col + kGroup <= a.cols) {
      store_vec(py, out);
    } else {
      for (int i = 0; i < kGroup; ++i)
        if (col + i < a.cols) py[i] = out[i];
    }
  }
}

}  // namespace
}  // namespace lst

using namespace lst;

extern "C" int lst_dropout(int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t ldx,
                           const void* residual, int64_t ldr, void* y, int64_t ldy, double p,
                           uint64_t seed, uint64_t offset, const uint64_t* counter,
                           void* hip_stream) {
  if (!known_dtype(dtype) || rows < 0 || rows > (int64_t)1 << 32 || cols < 1 || cols > 1 << 30)
    return LST_EINVAL;
  if (!(p >= 0.0) || !(p <= 1.0)) return LST_EINVAL;
  if (rows == 0) return LST_OK;
  if (!x || !y || ldx < cols || ldy < cols || (residual && ldr < cols)) return LST_EINVAL;
  DropoutArgs a;
  a.rows = rows;
  a.cols = cols;
  a.groups = (int)(((int64_t)cols + kGroup - 1) / kGroup);
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldy = ldy;
  a.drop = (uint32_t)(p * 65536.0 + 0.5);
  a.factor = a.drop < 65536 ? (float)(65536.0 / (65536.0 - a.drop)) : 0.f;
  a.seed = seed;
  a.offset = offset;
  a.counter = counter;
  const int64_t total = rows * a.groups, per = kThreads * kItems;
  if ((total + per - 1) / per > 0xFFFFFF) return LST_EINVAL;  // a launch has 2^32 threads at most
  const unsigned blocks = (unsigned)((total + per - 1) / per);
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    auto run = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, (hipStream_t)hip_stream, a,
                         (const T*)x, (const T*)residual, (T*)y);
    };
    auto sized = [&](auto index) {
      using I = decltype(index);
      if (cols % kGroup == 0)
        residual ? run(dropout_kernel<T, I, true, true>) : run(dropout_kernel<T, I, false, true>);
      else
        residual ? run(dropout_kernel<T, I, true, false>)
                 : run(dropout_kernel<T, I, false, false>);
    };
    total <= 0x7FFFFFFF - per ? sized(uint32_t{}) : sized(int64_t{});
    return launched();
  });
}
