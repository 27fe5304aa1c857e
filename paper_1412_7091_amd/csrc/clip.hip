// The norm over all gradients of a step, and the gradients scaled to a largest one (lst_clip).
//
//   n = sqrt(sum over all matrices of g^2),  g <- g min(1, max_norm / n)
//
// One pass for the squares, one that scales.  The squares are summed in float64: no value that a
// type has overflows them, and millions of small ones are not lost beside a large one.  The
// matrices' addresses and shapes travel as arguments of the launches, kTable of them at a time,
// so nothing of the caller's host memory is read after the call.  Blocks take tiles of 8192
// elements in turn, through the matrices in the order of the list; each leaves its sum, and the
// blocks of the second pass add these up by themselves, in the same order every time.
//
// Bound by memory: 24 matrices of 260 000 000 floats (3.12 GB: read, read and written) take 626
// us, 5.0 TB/s.  With neighbouring tiles for each block 717 (their streams meet in the same
// channels), with groups of four elements or sixteen 658 and 703, with stores past the caches
// 633.  40 matrices of 400 000 values take 5 and 7 us a launch.
#include <algorithm>
#include <new>
#include <vector>

#include "dtypes.h"

namespace lst {
namespace {

constexpr int kThreads = 256;
constexpr int kItems = 4;                        // groups of eight elements a thread and tile
constexpr int64_t kGroups = kThreads * kItems;   // groups of a tile
constexpr int kTable = 60;                       // matrices of a launch: 4 KB of arguments
constexpr int kBlocks = 2048;                    // of a launch: eight a compute unit
constexpr int kMost = 65536;

struct Entry {
  const void* data;
  void* out;
  int64_t rows, cols, ld, ldo, groups;  // groups: of a row
  int32_t dtype;
  uint32_t first;  // its first tile among those of the launch
};

struct Table {
  Entry e[kTable];
  int n;
  uint32_t tiles;
};

__device__ inline double block_sum(double v, double* lds) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) v += lds[i];
  return v;
}

// Where a group of a matrix is.
struct Place {
  int64_t row, col;
  __device__ Place(const Entry& e, int64_t group) {
    if (e.rows == 1) {
      row = 0;
      col = group * 8;
    } else if (e.rows * e.groups <= 0x7FFFFFFF) {
      const uint32_t r = (uint32_t)group / (uint32_t)e.groups;
      row = r;
      col = (int64_t)((uint32_t)group - r * (uint32_t)e.groups) * 8;
    } else {
      row = group / e.groups;
      col = (group - row * e.groups) * 8;
    }
  }
};

// A group's elements, zeros behind the row's last.
template <class T>
__device__ inline void load_group(const Entry& e, int64_t group, T (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (T)0.f;
  if (group >= e.rows * e.groups) return;
  const Place at(e, group);
  const T* p = (const T*)e.data + at.row * e.ld;
  if (at.col + 8 <= e.cols) {
    load_vec(p + at.col, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[min(at.col + i, e.cols - 1)];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = at.col + i < e.cols ? v[i] : (T)0.f;
  }
}

template <class T>
__device__ inline double tile_squares(const Entry& e, uint32_t tile) {
  const int64_t group = tile * kGroups + threadIdx.x;
  T v[kItems][8];
#pragma unroll
  for (int j = 0; j < kItems; ++j) load_group(e, group + j * kThreads, v[j]);
  double sum = 0;
#pragma unroll
  for (int j = 0; j < kItems; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double x = (float)v[j][i];
      sum = fma(x, x, sum);
    }
  return sum;
}

template <class T>
__device__ inline void scale_tile(const Entry& e, uint32_t tile, float factor, int power) {
  const int64_t group = tile * kGroups + threadIdx.x;
  T v[kItems][8];
#pragma unroll
  for (int j = 0; j < kItems; ++j) load_group(e, group + j * kThreads, v[j]);
#pragma unroll
  for (int j = 0; j < kItems; ++j) {
    const int64_t g = group + j * kThreads;
    if (g >= e.rows * e.groups) return;
    const Place at(e, g);
    T* p = (T*)e.out + at.row * e.ldo + at.col;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float f = (float)v[j][i] * factor;
      // float16's values and a factor that needs a power give zeros without it, too
      v[j][i] = (T)(std::is_same_v<T, _Float16> ? f : __builtin_ldexpf(f, power));
    }
    if (at.col + 8 <= e.cols) {
      store_vec(p, v[j]);
    } else {
      for (int i = 0; i < 8; ++i)
        if (at.col + i < e.cols) p[i] = v[j][i];
    }
  }
}

// The matrix that holds a tile: every lane looks at one of the table's (a search by one thread is
// a chain of loads: 40 gradients took 15 us a launch).
__device__ inline int entry_of(const Table& t, uint32_t tile) {
  const int lane = threadIdx.x % 64;
  const uint32_t first = t.e[min(lane, kTable - 1)].first;
  return __popcll(__ballot(lane < t.n && first <= tile)) - 1;
}

__global__ __launch_bounds__(kThreads) void squares_kernel(Table t, double* partial) {
  __shared__ double lds[kThreads / 64];
  double sum = 0;
  for (uint32_t tile = blockIdx.x; tile < t.tiles; tile += gridDim.x) {
    const Entry& e = t.e[entry_of(t, tile)];
    const uint32_t at = tile - e.first;
    sum += e.dtype == LST_F32    ? tile_squares<float>(e, at)
           : e.dtype == LST_BF16 ? tile_squares<__bf16>(e, at)
                                 : tile_squares<_Float16>(e, at);
  }
  sum = block_sum(sum, lds);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__device__ inline double total_of(const double* partial, int n, double* lds) {
  double v = 0;
  for (int i = threadIdx.x; i < n; i += kThreads) v += partial[i];
  return block_sum(v, lds);
}

// Many launches' sums into one.
__global__ __launch_bounds__(kThreads) void join_kernel(const double* partial, int n,
                                                        double* total) {
  __shared__ double lds[kThreads / 64];
  const double v = total_of(partial, n, lds);
  if (threadIdx.x == 0) *total = v;
}

// Tiles from the last to the first: what the pass before read last is the likeliest to be in the
// caches still.
__global__ __launch_bounds__(kThreads) void scale_kernel(Table t, const double* partial, int n,
                                                         double max_norm, float* norm,
                                                         int32_t* status, int first) {
  __shared__ double lds[kThreads / 64];
  const double all = sqrt(total_of(partial, n, lds));
  const bool finite = all < (double)INFINITY;
  const double ratio = finite && all > max_norm ? max_norm / all : 1.0;
  // a ratio that is no normal float goes as a fraction and a power of two
  int power = 0;
  const float factor = (float)(ratio < 0x1p-126 ? __builtin_frexp(ratio, &power) : ratio);
  if (first && blockIdx.x == 0 && threadIdx.x == 0) {
    *norm = (float)all;
    if (!finite && status) atomicCAS(status, 0, LST_ENONFINITE);
  }
  for (uint32_t i = blockIdx.x; i < t.tiles; i += gridDim.x) {
    const uint32_t tile = t.tiles - 1 - i;
    const Entry& e = t.e[entry_of(t, tile)];
    if (factor == 1.f && power == 0 && e.out == e.data) continue;
    const uint32_t at = tile - e.first;
    if (e.dtype == LST_F32)
      scale_tile<float>(e, at, factor, power);
    else if (e.dtype == LST_BF16)
      scale_tile<__bf16>(e, at, factor, power);
    else
      scale_tile<_Float16>(e, at, (float)ratio, 0);
  }
}

int64_t size_of(int dtype) { return dtype == LST_F32 ? 4 : 2; }

// Memory that a matrix takes: `width` bytes of each `stride`, or once for a single row.
struct Region {
  uintptr_t from, to;
  int64_t stride, width;
  bool single, written;
};

// Elements of a region as rows and columns of a matrix whose row stride is the region's, or any
// for a single row.
struct Box {
  int64_t row0, row1, col0, col1;
  bool written;
};

void add_boxes(const Region& r, uintptr_t base, int64_t stride, std::vector<Box>& boxes) {
  const int64_t from = (int64_t)(r.from - base), row = from / stride, col = from % stride;
  const int64_t rows = r.single ? 1 : (int64_t)(r.to - r.from - r.width) / stride + 1;
  const int64_t head = std::min(r.width, stride - col), rest = r.width - head;
  const int64_t full = rest / stride, tail = rest % stride;  // full: of a single row alone
  boxes.push_back({row, row + rows, col, col + head, r.written});
  if (full) boxes.push_back({row + 1, row + 1 + full, 0, stride, r.written});
  if (tail) boxes.push_back({row + 1 + full, row + 1 + full + rows, 0, tail, r.written});
}

// How many of the numbers that are in it are below another one.
struct Count {
  std::vector<int32_t> n;
  explicit Count(size_t size) : n(size + 1) {}
  void add(size_t at, int32_t v) {
    for (++at; at < n.size(); at += at & -at) n[at] += v;
  }
  int32_t below(size_t at) const {
    int32_t sum = 0;
    for (; at; at -= at & -at) sum += n[at];
    return sum;
  }
};

// Whether two boxes meet, one of which is written: the columns are gone through, and of the boxes
// that have a column the rows are counted, so that n boxes take n log n steps (65 536 matrices of
// neighbouring columns 15 ms on the host; compared by pairs 7.7 s).
bool meet(const std::vector<Box>& boxes) {
  struct Event {
    int64_t col;
    int begins;  // ends come first
    size_t box;
  };
  std::vector<int64_t> rows;
  std::vector<Event> events;
  for (size_t i = 0; i < boxes.size(); ++i) {
    rows.push_back(boxes[i].row0);
    rows.push_back(boxes[i].row1);
    events.push_back({boxes[i].col0, 1, i});
    events.push_back({boxes[i].col1, 0, i});
  }
  std::sort(rows.begin(), rows.end());
  rows.erase(std::unique(rows.begin(), rows.end()), rows.end());
  std::sort(events.begin(), events.end(), [](const Event& a, const Event& b) {
    return a.col != b.col ? a.col < b.col : a.begins < b.begins;
  });
  auto at = [&](int64_t row) {
    return (size_t)(std::lower_bound(rows.begin(), rows.end(), row) - rows.begin());
  };
  // where rows of the open boxes begin and end, of those that are only read and of the written
  Count first[2] = {Count(rows.size()), Count(rows.size())}, last[2] = {first[0], first[0]};
  for (const Event& e : events) {
    const Box& b = boxes[e.box];
    const size_t lo = at(b.row0), hi = at(b.row1);
    if (e.begins)
      for (int w = !b.written; w < 2; ++w)
        if (first[w].below(hi) > last[w].below(lo + 1)) return true;
    first[b.written].add(lo, e.begins ? 1 : -1);
    last[b.written].add(hi, e.begins ? 1 : -1);
  }
  return false;
}

// The furthest end of the regions so far, and that of those with another stride.
struct Reach {
  uintptr_t to[2] = {0, 0};
  int64_t stride[2] = {0, 0};
  void add(const Region& r) {
    if (r.stride == stride[0]) {
      to[0] = std::max(to[0], r.to);
    } else if (r.to > to[0]) {
      to[1] = to[0], stride[1] = stride[0];
      to[0] = r.to, stride[0] = r.stride;
    } else if (r.to > to[1]) {
      to[1] = r.to, stride[1] = r.stride;
    }
  }
  bool other(const Region& r) const { return to[stride[0] == r.stride] > r.from; }
};

// Whether regions that reach into each other, in order, share no element that is written.
bool apart(const Region* r, size_t n) {
  // several rows of different strides are not followed through each other
  Reach all, written;
  std::vector<int64_t> strides;
  for (size_t i = 0; i < n; ++i) {
    if (r[i].single) continue;
    if ((r[i].written ? all : written).other(r[i])) return false;
    all.add(r[i]);
    if (r[i].written) written.add(r[i]);
    strides.push_back(r[i].stride);
  }
  std::sort(strides.begin(), strides.end());
  strides.erase(std::unique(strides.begin(), strides.end()), strides.end());
  if (strides.empty()) strides.push_back((int64_t)1 << 62);
  std::vector<Box> boxes;
  for (const int64_t stride : strides) {
    boxes.clear();
    for (size_t i = 0; i < n; ++i)
      if (r[i].single || r[i].stride == stride) add_boxes(r[i], r[0].from, stride, boxes);
    if (meet(boxes)) return false;
  }
  return true;
}

bool good(const lst_gradient& g) {
  if (!known_dtype(g.dtype) || g.rows < 0 || g.cols < 0) return false;
  if (g.rows == 0 || g.cols == 0) return true;
  if (!g.data || g.rows > (int64_t)1 << 40 || g.cols > (int64_t)1 << 40) return false;
  if (g.rows > ((int64_t)1 << 40) / g.cols || g.ld < g.cols) return false;
  if (g.rows > 1 && g.ld > ((int64_t)1 << 50) / g.rows) return false;
  const bool apart = g.out && g.out != g.data;
  if (apart && (g.ldo < g.cols || (g.rows > 1 && g.ldo > ((int64_t)1 << 50) / g.rows)))
    return false;
  return apart || !g.out || g.rows <= 1 || g.ldo == g.ld;
}

// Whether every matrix that is written is memory of its own.
bool apart(int n, const lst_gradient* grads) {
  std::vector<Region> all;
  all.reserve(2 * (size_t)n);
  for (int i = 0; i < n; ++i) {
    const lst_gradient& g = grads[i];
    if (g.rows == 0 || g.cols == 0) continue;
    const int64_t e = size_of(g.dtype), width = g.cols * e;
    auto add = [&](const void* p, int64_t ld, bool written) {
      const uintptr_t from = (uintptr_t)p;
      const int64_t stride = g.rows == 1 ? width : ld * e;
      all.push_back({from, from + (uintptr_t)((g.rows - 1) * stride + width), stride, width,
                     g.rows == 1, written});
    };
    const bool own = !g.out || g.out == g.data;
    add(g.data, g.ld, own);
    if (!own) add(g.out, g.ldo, true);
  }
  std::sort(all.begin(), all.end(),
            [](const Region& a, const Region& b) { return a.from < b.from; });
  for (size_t i = 0, end; i < all.size(); i = end) {  // groups that reach into each other
    uintptr_t to = all[i].to;
    for (end = i + 1; end < all.size() && all[end].from < to; ++end) to = std::max(to, all[end].to);
    if (end - i > 1 && !apart(&all[i], end - i)) return false;
  }
  return true;
}

// Fills a table with matrices from `at` on, and moves it behind the last one taken.
Table fill(int n, const lst_gradient* grads, int& at) {
  Table t{};
  for (; at < n && t.n < kTable; ++at) {
    const lst_gradient& g = grads[at];
    if (g.rows == 0 || g.cols == 0) continue;
    const bool own = !g.out || g.out == g.data;
    Entry& e = t.e[t.n++];
    e.data = g.data;
    e.out = own ? const_cast<void*>(g.data) : g.out;
    e.rows = g.rows;
    e.cols = g.cols;
    e.ld = g.ld;
    e.ldo = own ? g.ld : g.ldo;
    e.dtype = g.dtype;
    if (e.rows > 1 && e.ld == e.cols && e.ldo == e.cols) {
      e.cols *= e.rows;
      e.rows = 1;
    }
    e.groups = (e.cols + 7) / 8;
    e.first = t.tiles;
    t.tiles += (uint32_t)((e.rows * e.groups + kGroups - 1) / kGroups);
  }
  return t;
}

unsigned blocks_of(const Table& t) { return std::min<unsigned>(std::max(1u, t.tiles), kBlocks); }

int tables_of(int n) { return std::max(1, (n + kTable - 1) / kTable); }

}  // namespace
}  // namespace lst

using namespace lst;

extern "C" {

int64_t lst_clip_workspace(int32_t n) {
  if (n < 0 || n > kMost) return -1;
  return ((int64_t)tables_of(n) * kBlocks + 1) * (int64_t)sizeof(double);
}

int lst_clip(int32_t n, const lst_gradient* grads, double max_norm, float* norm, void* workspace,
             int32_t* status, void* hip_stream) {
  if (n < 0 || n > kMost || (n && !grads) || !(max_norm >= 0.0) || !norm || !workspace ||
      ((uintptr_t)workspace & 15))
    return LST_EINVAL;
  int64_t most = 0;  // elements of the call: a launch's tiles are counted in 32 bits
  for (int i = 0; i < n; ++i) {
    if (!good(grads[i])) return LST_EINVAL;
    most += grads[i].rows * grads[i].cols;
    if (most > (int64_t)1 << 40) return LST_EINVAL;
  }
  try {
    if (!apart(n, grads)) return LST_EINVAL;
  } catch (const std::bad_alloc&) {
    return LST_ENOMEM;
  }
  hipStream_t s = (hipStream_t)hip_stream;
  double *total = (double*)workspace, *partial = total + 1;
  int count = 0, launches = 0;
  for (int at = 0; launches == 0 || at < n; ++launches) {
    const Table t = fill(n, grads, at);
    hipLaunchKernelGGL(squares_kernel, dim3(blocks_of(t)), dim3(kThreads), 0, s, t,
                       partial + count);
    count += (int)blocks_of(t);
  }
  if (launches > 1) {
    hipLaunchKernelGGL(join_kernel, dim3(1), dim3(kThreads), 0, s, partial, count, total);
    partial = total;
    count = 1;
  }
  int rc = launched();
  for (int at = 0, k = 0; rc == LST_OK && (k == 0 || at < n); ++k) {
    const Table t = fill(n, grads, at);
    hipLaunchKernelGGL(scale_kernel, dim3(blocks_of(t)), dim3(kThreads), 0, s, t, partial, count,
                       max_norm, norm, status, k == 0);
    rc = launched();
  }
  return rc;
}

}  // extern "C"
