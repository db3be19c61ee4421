// Rows of dense state arrays replaced in place by those of their parents: x[i] <- x_old[parents[i]], several arrays in a launch.
//
// A workgroup takes a slice of the bytes of all rows: it loads what the rows that change are to hold into registers, waits until all its waves
// have theirs, and writes.  Slices have no bytes in common, so nothing else has to be ordered, whatever the parents are (cycles, rows taken
// many times), and rows that stay cost nothing.  The fewer rows change, the wider the slice (24 of 32: 1 KB of each row).
//
// Bound by memory: low-rank keys of 32 rows of which 24 change, 1.9 GB read and written, take 350 to 386 us (4.9 to 5.4 TB/s; a copy reaches
// 4.8), with the next slice on its way while one is written; 607 us where a workgroup waits for its writes before it reads on.  67 MB in 17
// arrays: 17.6 us.
#include "common.hpp"
#include "kernels.hpp"

namespace skv {
namespace {

constexpr int kThreads = 256;
constexpr int kHeld = 8;                                  // pieces of a thread
constexpr int kSlots = kThreads * kHeld;                  // >= kMaxReorderRows: a slice is one unit wide at least
static_assert(kSlots >= kMaxReorderRows, "a slice holds a unit of every row");

// Columns first .. first + 2^shift - 1 (in units) of a piece of all rows that change.
struct Slice {
  uint8_t* base;
  int64_t row, first, units;
};
template <class T>
struct Held {
  T x[kHeld];
};
template <class T>
__device__ __forceinline__ Held<T> load_slice(const Slice& s, const uint32_t* pairs, int n, int shift) {
  Held<T> h;
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int item = k * kThreads + threadIdx.x, i = item >> shift;
    const int64_t u = s.first + (item & ((1 << shift) - 1));
    if (i < n && u < s.units) h.x[k] = *reinterpret_cast<const T*>(s.base + (int64_t)(pairs[i] & 0xffffu) * s.row + u * (int64_t)sizeof(T));
  }
  return h;
}
template <class T>
__device__ __forceinline__ void store_slice(const Slice& s, const Held<T>& h, const uint32_t* pairs, int n, int shift) {
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int item = k * kThreads + threadIdx.x, i = item >> shift;
    const int64_t u = s.first + (item & ((1 << shift) - 1));
    if (i < n && u < s.units) *reinterpret_cast<T*>(s.base + (int64_t)(pairs[i] >> 16) * s.row + u * (int64_t)sizeof(T)) = h.x[k];
  }
}
// what is loaded is there before any wave writes
template <class T>
__device__ __forceinline__ void loaded(const Held<T>& h) {
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    if constexpr (sizeof(T) == 16) asm volatile("" ::"v"(h.x[k].x), "v"(h.x[k].y), "v"(h.x[k].z), "v"(h.x[k].w));
    else asm volatile("" ::"v"((uint32_t)h.x[k]));
  }
  __syncthreads();
}

__global__ __launch_bounds__(kThreads) void reorder_rows_kernel(ReorderArgs g) {
  __shared__ uint32_t pairs[kMaxReorderRows];             // (row << 16) | parent of the rows that change
  __shared__ int64_t until[kMaxReorderArrays];            // slices of the arrays up to this one
  __shared__ int n_shared, wave_sum[kThreads / kWave];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  if (tid == 0) n_shared = 0;
  __syncthreads();
  for (int i0 = 0; i0 < g.n_rows; i0 += kThreads) {
    const int i = i0 + tid;
    const int p = i < g.n_rows ? g.parents[i] : -1;
    const bool changes = p >= 0 && p < g.n_rows && p != i;
    const uint64_t m = __ballot(changes);
    if (lane == 0) wave_sum[wave] = __popcll(m);
    __syncthreads();
    int at = n_shared + __popcll(m & ((1ull << lane) - 1));
    for (int v = 0; v < wave; ++v) at += wave_sum[v];
    if (changes) pairs[at] = ((uint32_t)i << 16) | (uint32_t)p;
    __syncthreads();
    if (tid == kThreads - 1) n_shared = at + (changes ? 1 : 0);
    __syncthreads();
  }
  const int n = n_shared;
  if (n == 0) return;
  const int shift = 31 - __clz(kSlots / n);               // 2^shift units wide: n << shift <= kSlots
  if (tid == 0) {
    int64_t sum = 0;
    for (int k = 0; k < g.n_arrays; ++k) {
      sum += (int64_t)g.a[k].n_outer * ((g.a[k].units + (1 << shift) - 1) >> shift);
      until[k] = sum;
    }
  }
  __syncthreads();
  const int64_t total = until[g.n_arrays - 1], wide = g.n_wide ? until[g.n_wide - 1] : 0, step = gridDim.x;
  int k = 0;
  auto slice = [&](int64_t t) {
    while (t >= until[k]) ++k;
    const ReorderArray& a = g.a[k];
    const int64_t per = (a.units + (1 << shift) - 1) >> shift, in = t - (k ? until[k - 1] : 0);
    const int64_t outer = a.n_outer == 1 ? 0 : in / per;
    return Slice{a.p + outer * a.outer, a.row, (in - outer * per) << shift, a.units};
  };
  int64_t t = blockIdx.x;
  if (t < wide) {                                         // the next slice is on its way while this one is written
    Slice s = slice(t);
    Held<uint4> h = load_slice<uint4>(s, pairs, n, shift);
    for (;;) {
      t += step;
      Slice next = s;
      Held<uint4> h2 = h;
      if (t < wide) {
        next = slice(t);
        h2 = load_slice<uint4>(next, pairs, n, shift);
      }
      loaded(h);
      store_slice(s, h, pairs, n, shift);
      if (t >= wide) break;
      s = next;
      h = h2;
    }
  }
  for (; t < total; t += step) {
    const Slice s = slice(t);
    if (g.a[k].unit == 4) {
      const Held<uint32_t> h = load_slice<uint32_t>(s, pairs, n, shift);
      loaded(h);
      store_slice(s, h, pairs, n, shift);
    } else {
      const Held<uint8_t> h = load_slice<uint8_t>(s, pairs, n, shift);
      loaded(h);
      store_slice(s, h, pairs, n, shift);
    }
  }
}

}  // namespace

hipError_t launch_reorder_rows(const ReorderArgs& a, hipStream_t st) {
  // slices if all rows change; a workgroup takes several where there are more than fill the chip
  int64_t slices = 0;
  int shift = 0;
  while ((a.n_rows << (shift + 1)) <= kSlots) ++shift;
  for (int k = 0; k < a.n_arrays; ++k) slices += (int64_t)a.a[k].n_outer * ((a.a[k].units + (1 << shift) - 1) >> shift);
  if (slices == 0) return hipSuccess;
  reorder_rows_kernel<<<dim3((unsigned)(slices < 2048 ? slices : 2048)), kThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace skv
