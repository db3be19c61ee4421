// Pages of a cache that several sequences share: forked, freed, grown, compacted and copied.  The state is the page table, the
// sequences' lengths and a count of holders per page; a page is free where its count is 0, and pages are given out lowest first, so
// what a call does follows from its arguments alone.
#include "common.hpp"
#include "kernels.hpp"

namespace skv {
namespace {

// ---- sequences become beginnings of others -----------------------------------------------------------------------------
// Like rows of dense state: a workgroup takes some columns of the table for all rows, loads, waits, writes.  Counts change where an entry
// does: what rows of a group share (their prompt) is the same before and after, and costs a comparison.
constexpr int kForkThreads = 256, kForkHeld = 16;
constexpr int kForkSlots = kForkThreads * kForkHeld;
static_assert(kForkSlots >= kMaxPoolRows, "a slice holds an entry of every row");

__device__ __forceinline__ int held_pages(int len, int shift) { return (int)(((int64_t)len + (1 << shift) - 1) >> shift); }
__device__ __forceinline__ int clamp_len(const PoolArg& p, int len) {
  const int64_t most = (int64_t)p.per_seq << p.shift;
  return len < 0 ? 0 : (int64_t)len > most ? (int)most : len;
}
// tokens that row i keeps of its parent
__device__ __forceinline__ int kept_len(const PoolArg& p, const int32_t* parents, const int32_t* keep, int i) {
  const int from = parents ? parents[i] : i;
  if (from < 0 || from >= p.batch) return 0;
  const int len = clamp_len(p, p.lens[from]);
  return keep ? min(len, max(keep[i], 0)) : len;
}

struct ForkRow {
  uint16_t row, from;
  int had, keeps;                                         // pages before and after
};

__global__ __launch_bounds__(kForkThreads) void pages_fork_kernel(PoolArg p, const int32_t* parents, const int32_t* keep) {
  __shared__ ForkRow rows[kMaxPoolRows];
  __shared__ int n_shared, width;
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  if (tid == 0) { n_shared = 0; width = 0; }
  __syncthreads();
  for (int i0 = 0; i0 < p.batch; i0 += kForkThreads) {    // (in any order: rows do not depend on each other's place here)
    const int i = i0 + tid;
    ForkRow r{(uint16_t)i, 0, 0, 0};
    bool changes = false;
    if (i < p.batch) {
      const int from = parents ? parents[i] : i;
      r.from = (uint16_t)from;                            // (of a row that keeps nothing it is not looked at)
      const int len = clamp_len(p, p.lens[i]), kept = kept_len(p, parents, keep, i);
      r.had = held_pages(len, p.shift);
      r.keeps = held_pages(kept, p.shift);
      changes = (from != i || r.had != r.keeps) && (r.had || r.keeps);
    }
    const uint64_t m = __ballot(changes);
    int at = 0;
    if (lane == 0 && m) at = atomicAdd(&n_shared, __popcll(m));
    at = __shfl(at, 0, kWave) + __popcll(m & ((1ull << lane) - 1));
    if (changes) {
      rows[at] = r;
      atomicMax(&width, max(r.had, r.keeps));
    }
  }
  __syncthreads();
  const int n = n_shared;
  if (n == 0) return;
  const int shift = 31 - __clz(kForkSlots / n), cols = 1 << shift;
  for (int first = blockIdx.x << shift; first < width; first += gridDim.x << shift) {
    int mine[kForkHeld], next[kForkHeld];
#pragma unroll
    for (int k = 0; k < kForkHeld; ++k) {
      const int item = k * kForkThreads + tid, i = item >> shift, j = first + (item & (cols - 1));
      mine[k] = next[k] = -1;
      if (i < n) {
        const ForkRow r = rows[i];
        if (j < r.had) mine[k] = p.table[(int64_t)r.row * p.stride + j];
        if (j < r.keeps) next[k] = p.table[(int64_t)r.from * p.stride + j];
      }
    }
    __builtin_amdgcn_s_waitcnt(0);                        // what is loaded is there before any wave writes
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kForkHeld; ++k) {
      const int item = k * kForkThreads + tid, i = item >> shift, j = first + (item & (cols - 1));
      if (i < n && mine[k] != next[k]) {
        p.table[(int64_t)rows[i].row * p.stride + j] = next[k];
        if (mine[k] >= 0 && mine[k] < p.n_pages) atomicSub(&p.refs[mine[k]], 1);
        if (next[k] >= 0 && next[k] < p.n_pages) atomicAdd(&p.refs[next[k]], 1);
      }
    }
  }
}

// ---- pages for new tokens -----------------------------------------------------------------------------------------------
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / kWave;

// exclusive prefix sum over the workgroup's threads, and the total
template <class T>
__device__ __forceinline__ T block_scan(T x, T* sums, T* total) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  T incl = x;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const T y = __shfl_up(incl, d, kWave);
    if (lane >= d) incl += y;
  }
  __syncthreads();                                        // (sums may still be read from the last time)
  if (lane == kWave - 1) sums[wave] = incl;
  __syncthreads();
  T before = 0, all = 0;
  for (int v = 0; v < kPlanWaves; ++v) {
    if (v < wave) before += sums[v];
    all += sums[v];
  }
  *total = all;
  return before + incl - x;
}

constexpr int kRowsPerThread = kMaxPoolRows / kPlanThreads;

// One workgroup.  A thread has rows tid * rpt ...: consecutive ones, so that prefix sums over threads are in order of rows.
__global__ __launch_bounds__(kPlanThreads) void pages_grow_kernel(PoolArg p, const int32_t* parents, const int32_t* keep, const int32_t* n_new,
                                                                  int n_new_all, MovesArg m, int32_t* free_list) {
  __shared__ int tail[kMaxPoolRows], first_col[kMaxPoolRows], begin32[kMaxPoolRows];
  __shared__ int64_t sums64[kPlanWaves];
  __shared__ int sums[kPlanWaves];
  __shared__ int stop;                                    // first row that is not granted
  const int tid = threadIdx.x, rpt = (p.batch + kPlanThreads - 1) / kPlanThreads;
  const int64_t room = (int64_t)p.per_seq << p.shift;
  const int page_mask = (1 << p.shift) - 1;
  int kept[kRowsPerThread], grow[kRowsPerThread], want[kRowsPerThread];
  bool copies[kRowsPerThread], shared[kRowsPerThread];
  if (tid == 0) stop = p.batch;
  for (int k = 0; k < rpt; ++k) {
    const int i = tid * rpt + k;
    kept[k] = grow[k] = want[k] = 0;
    copies[k] = shared[k] = false;
    if (i >= p.batch) continue;
    kept[k] = kept_len(p, parents, keep, i);
    const int g = max(n_new ? n_new[i] : n_new_all, 0);
    grow[k] = (int64_t)kept[k] + g <= room ? g : 0;
    int page = -1;
    if (grow[k] > 0 && (kept[k] & page_mask)) {
      page = p.table[(int64_t)i * p.stride + (kept[k] >> p.shift)];
      if (page >= p.n_pages || page < 0) page = -1;
    }
    tail[i] = page;
  }
  __syncthreads();
  int64_t mine = 0;
  for (int k = 0; k < rpt; ++k) {
    const int i = tid * rpt + k;
    if (i >= p.batch || grow[k] == 0) continue;
    if (tail[i] >= 0) {
      int earlier = 0;
      for (int j = 0; j < i; ++j) earlier += tail[j] == tail[i];
      const int holders = p.refs[tail[i]];
      copies[k] = earlier < holders - 1;
      shared[k] = holders > 1;
    }
    first_col[i] = copies[k] ? kept[k] >> p.shift : held_pages(kept[k], p.shift);
    want[k] = held_pages(kept[k] + grow[k], p.shift) - first_col[i];
    mine += want[k];
  }
  int64_t asked;
  int64_t begin = block_scan<int64_t>(mine, sums64, &asked);
  // the lowest free pages, as many as are asked for
  const int need = (int)(asked < p.n_pages ? asked : p.n_pages);
  int found = 0;
  for (int p0 = 0; p0 < p.n_pages && found < need; p0 += kPlanThreads * 4) {
    const int at = p0 + tid * 4;
    int page[4], n = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (at + e < p.n_pages && p.refs[at + e] == 0) page[n++] = at + e;
    int total;
    const int before = found + block_scan<int>(n, sums, &total);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n && before + e < need) free_list[before + e] = page[e];
    found += total;
  }
  found = min(found, need);
  // rows up to the first that the free pages do not suffice for
  int64_t b = begin;
  for (int k = 0; k < rpt; ++k) {
    const int i = tid * rpt + k;
    if (i < p.batch && want[k] > 0 && b + want[k] > found) atomicMin(&stop, i);
    b += want[k];
  }
  __syncthreads();
  int granted = 0, n_copies = 0;
  b = begin;
  for (int k = 0; k < rpt; ++k) {
    const int i = tid * rpt + k;
    if (i < p.batch) {
      if (i >= stop && (want[k] > 0 || shared[k])) grow[k] = 0;
      if (grow[k] == 0) copies[k] = false;
      begin32[i] = i < stop ? (int)b : 0x7fffffff;
      if (i < stop) granted = (int)(b + want[k]);
      n_copies += copies[k];
      p.lens[i] = kept[k] + grow[k];
    }
    b += want[k];
  }
  int all_copies;
  int at = block_scan<int>(n_copies, sums, &all_copies);
  if (tid == 0) *m.count = all_copies;
  for (int k = 0; k < rpt; ++k) {
    const int i = tid * rpt + k;
    if (i < p.batch && copies[k]) {
      m.src[at] = tail[i];
      m.dst[at] = free_list[begin32[i]];
      m.rows[at] = kept[k] & page_mask;
      atomicSub(&p.refs[tail[i]], 1);
      ++at;
    }
  }
  // the pages themselves: the q-th belongs to the last row that begins at or before q
  __shared__ int n_granted;
  if (tid == 0) n_granted = 0;
  __syncthreads();
  atomicMax(&n_granted, granted);
  __syncthreads();
  for (int q = tid; q < n_granted; q += kPlanThreads) {
    int lo = 0, hi = p.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (begin32[mid] <= q) lo = mid; else hi = mid - 1;
    }
    const int page = free_list[q];
    p.table[(int64_t)lo * p.stride + first_col[lo] + (q - begin32[lo])] = page;
    p.refs[page] = 1;
  }
}

// ---- compaction -----------------------------------------------------------------------------------------------------------
// One workgroup: used pages are counted, then the free places below that border are listed from below and the used ones above it from
// above; there are equally many.  info: [0] least page that moves.
__global__ __launch_bounds__(kPlanThreads) void pages_compact_kernel(PoolArg p, int max_moves, MovesArg m, int32_t* n_used, int32_t* new_id, int32_t* info) {
  __shared__ int sums[kPlanWaves];
  __shared__ int top;
  const int tid = threadIdx.x;
  if (tid == 0) top = 0;
  int border = 0, total, n = 0;
  for (int i = tid; i < p.n_pages; i += kPlanThreads) n += p.refs[i] != 0;
  block_scan<int>(n, sums, &border);
  const int most = min(max_moves, m.capacity);
  int holes = 0;
  for (int p0 = 0; p0 < border; p0 += kPlanThreads) {
    const int i = p0 + tid;
    const bool hole = i < border && p.refs[i] == 0;
    const int at = holes + block_scan<int>(hole, sums, &total);
    if (hole && at < most) m.dst[at] = i;
    holes += total;
  }
  const int moved = min(holes, most);
  int seen = 0;
  for (int p0 = border; p0 < p.n_pages; p0 += kPlanThreads) {
    const int i = p0 + tid;
    const bool used = i < p.n_pages && p.refs[i] != 0;
    const int at = holes - 1 - (seen + block_scan<int>(used, sums, &total));
    if (used && at < moved) m.src[at] = i;
    if (used && at == moved) top = i + 1;                // the highest page that stays above the border
    seen += total;
  }
  __threadfence_block();
  __syncthreads();
  for (int i = tid; i < moved; i += kPlanThreads) {
    const int from = m.src[i], to = m.dst[i];
    if (m.rows) m.rows[i] = 1 << p.shift;
    new_id[from] = to;
    p.refs[to] = p.refs[from];
    p.refs[from] = 0;
  }
  if (tid == 0) {
    *m.count = moved;
    info[0] = moved ? m.src[moved - 1] : p.n_pages;
    if (n_used) *n_used = moved < holes ? top : border;
  }
}

__global__ __launch_bounds__(256) void pages_rename_kernel(PoolArg p, const int32_t* new_id, const int32_t* info) {
  const int least = info[0];
  if (least >= p.n_pages) return;
  for (int i = blockIdx.y; i < p.batch; i += gridDim.y) {
    const int n = held_pages(clamp_len(p, p.lens[i]), p.shift);
    int32_t* row = p.table + (int64_t)i * p.stride;
    for (int j = blockIdx.x * 256 + threadIdx.x; j < n; j += gridDim.x * 256) {
      const int page = row[j];
      if (page >= least && page < p.n_pages) row[j] = new_id[page];
    }
  }
}

// ---- copies -----------------------------------------------------------------------------------------------------------------
// A workgroup per (move, layer, keys or values), several where there are more.
__global__ __launch_bounds__(256) void pages_copy_kernel(PagesCopyArgs a) {
  const int count = a.m.count ? min(*a.m.count, a.m.capacity) : a.m.capacity;
  const int vec = a.row_bytes / 16;
  const int64_t tasks = (int64_t)count * a.n_layers * 2 * a.hkv;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & (kWave - 1);
  for (int64_t t = (int64_t)blockIdx.x * 4 + wave; t < tasks; t += (int64_t)gridDim.x * 4) {
    const int head = (int)(t % a.hkv);
    const int64_t u = t / a.hkv;
    const int layer = (int)(u / 2 % a.n_layers), move = (int)(u / 2 / a.n_layers);
    const bool v = u & 1;
    const int src = a.m.src[move], dst = a.m.dst[move];
    if (src < 0 || src >= a.from_pages || dst < 0 || dst >= a.to_pages) continue;
    const int rows = a.m.rows ? min(max(a.m.rows[move], 0), a.page_size) : a.page_size;
    const int64_t* fs = v ? a.fv : a.fk;
    const int64_t* ts = v ? a.tv : a.tk;
    const uint8_t* f = (v ? a.from_v : a.from_k)[layer] + src * fs[0] + head * fs[1];
    uint8_t* o = (v ? a.to_v : a.to_k)[layer] + dst * ts[0] + head * ts[1];
    for (int i = lane; i < rows * vec; i += kWave) {
      const int r = i / vec, c = i % vec;
      *reinterpret_cast<uint4*>(o + r * ts[2] + c * 16) = *reinterpret_cast<const uint4*>(f + r * fs[2] + c * 16);
    }
  }
}

}  // namespace

hipError_t launch_pages_update(const PoolArg& p, const int32_t* parents, const int32_t* keep, const int32_t* n_new, int n_new_all, const MovesArg& m,
                               int32_t* free_list, hipStream_t st) {
  if (parents || keep) {
    int shift = 0;
    while ((p.batch << (shift + 1)) <= kForkSlots) ++shift;
    const int blocks = (int)(((int64_t)p.per_seq + (1 << shift) - 1) >> shift);
    pages_fork_kernel<<<dim3(blocks < 256 ? blocks : 256), kForkThreads, 0, st>>>(p, parents, keep);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  pages_grow_kernel<<<dim3(1), kPlanThreads, 0, st>>>(p, parents, keep, n_new, n_new_all, m, free_list);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PoolArg& p, int max_moves, const MovesArg& m, int32_t* n_used, int32_t* new_id, int32_t* info, hipStream_t st) {
  pages_compact_kernel<<<dim3(1), kPlanThreads, 0, st>>>(p, max_moves, m, n_used, new_id, info);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int across = (p.per_seq + 255) / 256;
  pages_rename_kernel<<<dim3(across < 64 ? across : 64, p.batch < 1024 ? p.batch : 1024), 256, 0, st>>>(p, new_id, info);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PagesCopyArgs& a, hipStream_t st) {
  const int64_t blocks = ((int64_t)a.m.capacity * a.n_layers * 2 * a.hkv + 3) / 4;
  if (blocks == 0) return hipSuccess;
  pages_copy_kernel<<<dim3((unsigned)(blocks < 4096 ? blocks : 4096)), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace skv
