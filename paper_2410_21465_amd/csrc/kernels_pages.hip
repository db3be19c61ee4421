// Pages of a cache that several sequences share: forked, freed, grown, compacted and copied.  The state is the page table, the sequences'
// lengths and a count of holders per page; a page is free where its count is 0, and pages are given out lowest first, so what a call does
// follows from its arguments alone.
//
// Planning is one workgroup's chain of dependent reads (lengths; table; counts) and prefix sums: 10.0 us for 16 x 4 beams over 1300 pages, 11.4
// for 256 rows over 30000; more workgroups would need more launches, of 2 us each.  Copies are bound by memory: 1 GB of pages in 410 us (5.1
// TB/s read and written).
#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"

namespace skv {
namespace {

__device__ __forceinline__ int held_pages(int len, int shift) { return (int)(((int64_t)len + (1 << shift) - 1) >> shift); }
__device__ __forceinline__ int clamp_len(const PoolArg& p, int len) {
  const int64_t most = (int64_t)p.per_seq << p.shift;
  return len < 0 ? 0 : (int64_t)len > most ? (int)most : len;
}
// the row that row i continues (-1: none), and the tokens it keeps of it
__device__ __forceinline__ int parent_of(const PoolArg& p, const int32_t* parents, int i) {
  const int from = parents ? parents[i] : i;
  return from >= 0 && from < p.batch ? from : -1;
}
__device__ __forceinline__ int kept_len(int parent_len, const int32_t* keep, int i) { return keep ? min(parent_len, max(keep[i], 0)) : parent_len; }

// ---- sequences become beginnings of others -----------------------------------------------------------------------------
// Like rows of dense state: some columns of the table for all rows that change are loaded, then written.  Counts change where an entry does:
// what rows of a group share (their prompt) is the same before and after, and costs a comparison.
struct ForkRow {
  uint16_t row, from;
  int had, keeps;                                         // pages before and after
};
template <int THREADS, int HELD>
__device__ __forceinline__ void fork_columns(const PoolArg& p, const ForkRow* rows, int n, int shift, int first) {
  const int tid = threadIdx.x, cols = 1 << shift;
  int mine[HELD], next[HELD];
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    const int item = k * THREADS + tid, i = item >> shift, j = first + (item & (cols - 1));
    mine[k] = next[k] = -1;
    if (i < n) {
      const ForkRow r = rows[i];
      if (j < r.had) mine[k] = p.table[(int64_t)r.row * p.stride + j];
      if (j < r.keeps) next[k] = p.table[(int64_t)r.from * p.stride + j];
    }
  }
  __builtin_amdgcn_s_waitcnt(0);                          // what is loaded is there before any wave writes
  __syncthreads();
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    const int item = k * THREADS + tid, i = item >> shift, j = first + (item & (cols - 1));
    if (i < n && mine[k] != next[k]) {
      p.table[(int64_t)rows[i].row * p.stride + j] = next[k];
      if (mine[k] >= 0 && mine[k] < p.n_pages) atomicSub(&p.refs[mine[k]], 1);
      if (next[k] >= 0 && next[k] < p.n_pages) atomicAdd(&p.refs[next[k]], 1);
    }
  }
}
// puts a row into the list if anything of it changes
__device__ __forceinline__ void list_fork(const ForkRow& r, bool changes, ForkRow* rows, int* n_shared, int* width) {
  const int lane = threadIdx.x & (kWave - 1);
  const uint64_t m = __ballot(changes);
  int at = 0;
  if (lane == 0 && m) at = atomicAdd(n_shared, __popcll(m));
  at = __shfl(at, 0, kWave) + __popcll(m & ((1ull << lane) - 1));
  if (changes) {
    rows[at] = r;
    atomicMax(width, max(r.had, r.keeps));
  }
}

constexpr int kForkThreads = 256, kForkHeld = 16;
constexpr int kForkSlots = kForkThreads * kForkHeld;
static_assert(kForkSlots >= kMaxPoolRows, "a slice holds an entry of every row");

__global__ __launch_bounds__(kForkThreads) void pages_fork_kernel(PoolArg p, const int32_t* parents, const int32_t* keep) {
  __shared__ ForkRow rows[kMaxPoolRows];
  __shared__ int n_shared, width;
  const int tid = threadIdx.x;
  if (tid == 0) { n_shared = 0; width = 0; }
  __syncthreads();
  for (int i0 = 0; i0 < p.batch; i0 += kForkThreads) {
    const int i = i0 + tid;
    ForkRow r{(uint16_t)i, 0, 0, 0};
    bool changes = false;
    if (i < p.batch) {
      const int from = parent_of(p, parents, i);
      r.from = (uint16_t)from;                            // (of a row that keeps nothing it is not looked at)
      r.had = held_pages(clamp_len(p, p.lens[i]), p.shift);
      r.keeps = from < 0 ? 0 : held_pages(kept_len(clamp_len(p, p.lens[from]), keep, i), p.shift);
      changes = (from != i || r.had != r.keeps) && (r.had || r.keeps);
    }
    list_fork(r, changes, rows, &n_shared, &width);
  }
  __syncthreads();
  const int n = n_shared;
  if (n == 0) return;
  const int shift = 31 - __clz(kForkSlots / n);
  for (int first = blockIdx.x << shift; first < width; first += gridDim.x << shift) fork_columns<kForkThreads, kForkHeld>(p, rows, n, shift, first);
}

// ---- pages for new tokens -----------------------------------------------------------------------------------------------
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / kWave;

// exclusive prefix sums over the workgroup's threads, and the totals; the first sum stays at its largest value instead of wrapping around
__device__ __forceinline__ uint32_t op_add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
struct Scan3 {
  uint32_t x, y, z;
};
#define SKV_SCAN(x, OP)                                                                               \
  x = OP(x, dpp_u32<0x111>(0u, x)); x = OP(x, dpp_u32<0x112>(0u, x)); x = OP(x, dpp_u32<0x114>(0u, x)); \
  x = OP(x, dpp_u32<0x118>(0u, x)); x = OP(x, dpp_u32<0x142, 0xa>(0u, x)); x = OP(x, dpp_u32<0x143, 0xc>(0u, x));
__device__ __forceinline__ uint32_t lane_before(uint32_t x) { return dpp_u32<0x138>(0u, x); }   // wave_shr:1
__device__ __forceinline__ Scan3 block_scan(Scan3 v, Scan3* sums, Scan3* total) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  SKV_SCAN(v.x, op_add_sat) SKV_SCAN(v.y, op_add) SKV_SCAN(v.z, op_add)
  __syncthreads();                                        // (sums may still be read from the last time)
  if (lane == kWave - 1) sums[wave] = v;
  __syncthreads();
  Scan3 w = lane < kPlanWaves ? sums[lane] : Scan3{0u, 0u, 0u};
  SKV_SCAN(w.x, op_add_sat) SKV_SCAN(w.y, op_add) SKV_SCAN(w.z, op_add)
  auto at = [](uint32_t x, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)x, l); };
  *total = Scan3{at(w.x, kPlanWaves - 1), at(w.y, kPlanWaves - 1), at(w.z, kPlanWaves - 1)};
  Scan3 r{lane_before(v.x), lane_before(v.y), lane_before(v.z)};
  const int uw = __builtin_amdgcn_readfirstlane(wave);
  if (uw > 0) {
    r.x = op_add_sat(r.x, at(w.x, uw - 1));
    r.y += at(w.y, uw - 1);
    r.z += at(w.z, uw - 1);
  }
  return r;
}
#undef SKV_SCAN

constexpr int kRefsPerThread = 16;                        // looked at together
constexpr int kRefsAtOnce = kPlanThreads * kRefsPerThread;
// which of a thread's pages, of those from p0 on, are free
__device__ __forceinline__ uint32_t free_pages(const PoolArg& p, int p0) {
  uint32_t mask = 0;
  const int at = p0 + (int)threadIdx.x * kRefsPerThread;
  if (at + kRefsPerThread <= p.n_pages && p.refs_aligned) {
    int4 r[kRefsPerThread / 4];
#pragma unroll
    for (int e = 0; e < kRefsPerThread / 4; ++e) r[e] = *reinterpret_cast<const int4*>(p.refs + at + 4 * e);
#pragma unroll
    for (int e = 0; e < kRefsPerThread / 4; ++e)
      mask |= (uint32_t)(r[e].x == 0) << 4 * e | (uint32_t)(r[e].y == 0) << (4 * e + 1) | (uint32_t)(r[e].z == 0) << (4 * e + 2) |
              (uint32_t)(r[e].w == 0) << (4 * e + 3);
  } else if (at < p.n_pages) {
    for (int e = 0; e < kRefsPerThread && at + e < p.n_pages; ++e) mask |= (uint32_t)(p.refs[at + e] == 0) << e;
  }
  return mask;
}
constexpr int kListRoom = 2048;                           // free pages in LDS; more of them in the workspace
constexpr int kForkInPlan = 1024;                         // rows that the plan forks by itself
constexpr int kPlanHeld = 8;
// Pages that a row which stays gives up one by one, by its thread; rows that give up more go with the forks, which costs a look at every column of theirs.
// 256 rows of 252, captured, as events around a replay see it, 8 / 16 / 32 / 64 pages of each: 26.3 / 31.6 / 49.8 / 86.8 us one by one, 32.3 / 32.3 / 33.0 /
// 33.8 with the forks.  All 65,536 pages of one row: 18.8 ms one by one, 33 us with the forks.
constexpr int kFewCut = 16;
// Entries of the page table that the plan's workgroup deals with by itself.  An update that forks half of its rows, captured: 64 rows of 70 entries 9.7 us,
// and 13.9 with a launch for the forks; 256 of 252 13.0 and 15.1; 1000 of 64 14.5 and 22.1 (one launch is the faster up to the border, and may be beyond
// it; all entries of 8 x 8192 taken from their rows: 32 us, of 2 x 65,536 with the other launch 18).  Compaction: 64 of 70 6.9 us, 8.0 with a
// launch that rewrites the table; 256 of 64 13.7 and 9.9.
constexpr int64_t kForkEntries = 65536, kRenameEntries = 8192;

// One workgroup.  A thread has rows tid * rpt ...: consecutive ones, so that prefix sums over threads are in order of rows.  kFork: the rows
// are forked here first (at most kForkInPlan); else that has been done by the launch before.
template <bool kFork>
__global__ __launch_bounds__(kPlanThreads) void pages_grow_kernel(PoolArg p, const int32_t* parents, const int32_t* keep, const int32_t* n_new,
                                                                  int n_new_all, MovesArg m, int32_t* free_list) {
  constexpr int kRows = kFork ? kForkInPlan : kMaxPoolRows, kRowsPerThread = kRows / kPlanThreads;
  __shared__ int32_t lens[kRows];                         // lengths before, then where a row's pages begin in the list
  __shared__ int first_col[kRows], list_lds[kListRoom];
  // last pages that rows share and will write, hashed: the rows that will, and the last of them
  constexpr int kSlots = 2 * kRows;
  __shared__ int shared_page[kSlots], writers[kSlots], last_writer[kSlots];
  __shared__ ForkRow forks[kFork ? kForkInPlan : 1];
  __shared__ Scan3 sums[kPlanWaves];
  __shared__ int stop, n_granted, n_copied, n_forks, width;   // stop: first row that is not granted
  int32_t* begin = lens;
  const int tid = threadIdx.x, rpt = (p.batch + kPlanThreads - 1) / kPlanThreads;
  const int64_t room = (int64_t)p.per_seq << p.shift;
  const int page_mask = (1 << p.shift) - 1;
  if (tid == 0) { stop = p.batch; n_forks = width = 0; }
  for (int i = tid; i < kSlots; i += kPlanThreads) { shared_page[i] = -1; writers[i] = 0; last_writer[i] = -1; }
  // (all that does not depend on anything is asked for at once)
  int from[kRowsPerThread], most[kRowsPerThread], grow[kRowsPerThread], kept[kRowsPerThread], page[kRowsPerThread];
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) {
    const int i = tid * rpt + k;
    from[k] = -1;
    most[k] = grow[k] = kept[k] = 0;
    page[k] = -1;
    if (k < rpt && i < p.batch) {
      from[k] = parent_of(p, parents, i);
      most[k] = keep ? max(keep[i], 0) : 0x7fffffff;
      grow[k] = max(n_new ? n_new[i] : n_new_all, 0);
      lens[i] = clamp_len(p, p.lens[i]);
    }
  }
  __syncthreads();
  int cut_from = 0, cut_to = 0;                           // the few pages that a row which is its own parent gives up
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) {
    const int i = tid * rpt + k;
    ForkRow f{(uint16_t)i, 0, 0, 0};
    bool changes = false;
    if (k < rpt && i < p.batch) {
      if (from[k] >= 0) kept[k] = min(lens[from[k]], most[k]);
      if ((int64_t)kept[k] + grow[k] > room) grow[k] = 0;
      // (of the parent's row, which holds the same pages and is not written yet, or of its own)
      if (grow[k] > 0 && (kept[k] & page_mask)) page[k] = p.table[(int64_t)(kFork ? from[k] : i) * p.stride + (kept[k] >> p.shift)];
      if constexpr (kFork) {
        f.from = (uint16_t)from[k];
        f.had = held_pages(lens[i], p.shift);
        f.keeps = held_pages(kept[k], p.shift);
        changes = from[k] == i ? f.had - f.keeps > kFewCut : (f.had || f.keeps);
        if (from[k] == i && !changes) { cut_from = f.keeps; cut_to = f.had; }
      }
    }
    if constexpr (kFork) list_fork(f, changes, forks, &n_forks, &width);   // (a row a thread)
  }
  __syncthreads();
  if constexpr (kFork) {
    const int n = n_forks;
    if (n) {
      const int shift = 31 - __clz(kPlanThreads * kPlanHeld / n);
      for (int first = 0; first < width; first += 1 << shift) fork_columns<kPlanThreads, kPlanHeld>(p, forks, n, shift, first);
      __syncthreads();                                    // (rows may have been read beyond what they keep themselves)
    }
    for (int j = cut_from; j < cut_to; ++j) {
      int32_t* entry = p.table + (int64_t)tid * p.stride + j;
      const int gone = *entry;
      *entry = -1;
      if (gone >= 0 && gone < p.n_pages) atomicSub(&p.refs[gone], 1);
    }
    __builtin_amdgcn_s_waitcnt(0);                        // the counts are changed before they are read
    __syncthreads();
  }
  // counts of the first pages, and of the rows' last ones
  int holders[kRowsPerThread], slot[kRowsPerThread];
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) {
    const int i = tid * rpt + k;
    if (page[k] < 0 || page[k] >= p.n_pages) page[k] = -1;
    holders[k] = page[k] >= 0 ? p.refs[page[k]] : 0;
    slot[k] = 0;
    if (holders[k] > 1) {                                 // (there are more slots than rows)
      int h = (int)((uint32_t)page[k] * 2654435769u >> 16) & (kSlots - 1);
      for (;;) {
        const int held = atomicCAS(&shared_page[h], -1, page[k]);
        if (held == -1 || held == page[k]) break;
        h = (h + 1) & (kSlots - 1);
      }
      atomicAdd(&writers[h], 1);
      atomicMax(&last_writer[h], i);
      slot[k] = h;
    }
  }
  uint32_t free_mask = free_pages(p, 0);
  __syncthreads();
  uint32_t want[kRowsPerThread];
  bool copies[kRowsPerThread];
  Scan3 mine{0u, 0u, (uint32_t)__popc(free_mask)};
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) {
    const int i = tid * rpt + k;
    want[k] = 0;
    copies[k] = false;
    if (grow[k] == 0) continue;
    // rows before this one take copies; if nobody else holds the page, the last of its writers keeps it
    if (holders[k] > 1) copies[k] = holders[k] > writers[slot[k]] || i != last_writer[slot[k]];
    const int first = copies[k] ? kept[k] >> p.shift : held_pages(kept[k], p.shift);
    first_col[i] = first;
    want[k] = (uint32_t)(held_pages(kept[k] + grow[k], p.shift) - first);
    mine.x = op_add_sat(mine.x, want[k]);
    mine.y += copies[k];
  }
  Scan3 all;
  const Scan3 before = block_scan(mine, sums, &all);
  const uint32_t asked = all.x, all_copies = all.y;
  // the lowest free pages, as many as are asked for
  const int need = (int)(asked < (uint32_t)p.n_pages ? asked : (uint32_t)p.n_pages);
  int* list = need <= kListRoom ? list_lds : free_list;
  int found = 0, at = (int)before.z, p0 = 0;
  for (;;) {
    const int base = p0 + tid * kRefsPerThread;
    while (free_mask && at < need) {
      const int e = __ffs(free_mask) - 1;
      free_mask &= free_mask - 1;
      list[at++] = base + e;
    }
    found += (int)all.z;
    p0 += kRefsAtOnce;
    if (found >= need || p0 >= p.n_pages) break;
    free_mask = free_pages(p, p0);
    at = found + (int)block_scan(Scan3{0u, 0u, (uint32_t)__popc(free_mask)}, sums, &all).z;
  }
  found = min(found, need);
  // rows up to the first that the free pages do not suffice for
  uint32_t b = before.x;
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) {
    const int i = tid * rpt + k;
    const uint32_t end = op_add_sat(b, want[k]);
    if (want[k] > 0 && end > (uint32_t)found) atomicMin(&stop, i);
    b = end;
  }
  __syncthreads();
  const int last = stop;
  int move = (int)before.y;
  if (tid == 0 && last == p.batch) { n_granted = (int)asked; n_copied = (int)all_copies; }
  b = before.x;
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) {
    const int i = tid * rpt + k;
    if (k < rpt && i < p.batch) {
      if (i == last) { n_granted = (int)b; n_copied = move; }
      if (i >= last && (want[k] > 0 || holders[k] > 1)) grow[k] = 0;
      begin[i] = i < last ? (int)b : 0x7fffffff;
      p.lens[i] = kept[k] + grow[k];
      if (i < last && copies[k]) {
        m.src[move] = page[k];
        m.dst[move] = list[b];
        m.rows[move] = kept[k] & page_mask;
        atomicSub(&p.refs[page[k]], 1);
        ++move;
      }
    }
    b = op_add_sat(b, want[k]);
  }
  __syncthreads();
  if (tid == 0) *m.count = n_copied;
  // the pages themselves: the q-th belongs to the last row that begins at or before q
  for (int q = tid; q < n_granted; q += kPlanThreads) {
    int lo = 0, hi = p.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (begin[mid] <= q) lo = mid; else hi = mid - 1;
    }
    const int fresh = list[q];
    p.table[(int64_t)lo * p.stride + first_col[lo] + (q - begin[lo])] = fresh;
    p.refs[fresh] = 1;
  }
}

// ---- compaction -----------------------------------------------------------------------------------------------------------
// One workgroup: used pages are counted, then the free places below that border are listed from below and the used ones above it from
// above; there are equally many.  info: [0] least page that moves.  kRename: the page table is rewritten here too.
__device__ __forceinline__ void rename_row(const PoolArg& p, int32_t* row, int j, const int32_t* new_id, int least) {
  const int page = row[j];
  if (page >= least && page < p.n_pages) row[j] = new_id[page];
}
template <bool kRename>
__global__ __launch_bounds__(kPlanThreads) void pages_compact_kernel(PoolArg p, int max_moves, MovesArg m, int32_t* n_used, int32_t* new_id, int32_t* info) {
  __shared__ Scan3 sums[kPlanWaves];
  __shared__ int top;
  const int tid = threadIdx.x;
  if (tid == 0) top = 0;
  auto pages_of = [&](int p0) { return min(max(p.n_pages - p0 - tid * kRefsPerThread, 0), kRefsPerThread); };   // a thread's
  Scan3 all;
  uint32_t free_mask = free_pages(p, 0);
  uint32_t used = (uint32_t)(pages_of(0) - __popc(free_mask));
  for (int p0 = kRefsAtOnce; p0 < p.n_pages; p0 += kRefsAtOnce) used += (uint32_t)(pages_of(p0) - __popc(free_pages(p, p0)));
  block_scan(Scan3{0u, used, 0u}, sums, &all);
  const int border = (int)all.y, most = min(max_moves, m.capacity);
  // (the number of moves is known before the last of them: holes below the border are as many as used pages above it)
  int holes = 0;
  for (int p0 = 0; p0 < border; p0 += kRefsAtOnce) {
    if (p0 > 0) free_mask = free_pages(p, p0);
    const int base = p0 + tid * kRefsPerThread, below = min(max(border - base, 0), kRefsPerThread);
    uint32_t mask = free_mask & ((1u << below) - 1u);
    int at = holes + (int)block_scan(Scan3{0u, (uint32_t)__popc(mask), 0u}, sums, &all).y;
    while (mask && at < most) {
      const int e = __ffs(mask) - 1;
      mask &= mask - 1;
      m.dst[at++] = base + e;
    }
    holes += (int)all.y;
  }
  const int moved = min(holes, most);
  int seen = 0;
  for (int p0 = border / kRefsAtOnce * kRefsAtOnce; p0 < p.n_pages; p0 += kRefsAtOnce) {
    if (p.n_pages > kRefsAtOnce) free_mask = free_pages(p, p0);
    const int base = p0 + tid * kRefsPerThread, n = pages_of(p0), below = min(max(border - base, 0), n);
    uint32_t mask = ~free_mask & ((1u << n) - 1u) & ~((1u << below) - 1u);
    int at = holes - 1 - (seen + (int)block_scan(Scan3{0u, (uint32_t)__popc(mask), 0u}, sums, &all).y);
    while (mask) {
      const int e = __ffs(mask) - 1;
      mask &= mask - 1;
      if (at < moved) m.src[at] = base + e;
      if (at == moved) top = base + e + 1;               // the highest page that stays above the border
      --at;
    }
    seen += (int)all.y;
  }
  __syncthreads();
  constexpr int kAtOnce = 4;                              // moves of a thread on their way together
  for (int i0 = tid; i0 < moved; i0 += kPlanThreads * kAtOnce) {
    int from[kAtOnce], to[kAtOnce], held[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = min(i0 + k * kPlanThreads, moved - 1);
      from[k] = m.src[i];
      to[k] = m.dst[i];
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) held[k] = p.refs[from[k]];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = i0 + k * kPlanThreads;
      if (i >= moved) break;
      if (m.rows) m.rows[i] = 1 << p.shift;
      new_id[from[k]] = to[k];
      p.refs[to[k]] = held[k];
      p.refs[from[k]] = 0;
    }
  }
  const int least = moved ? m.src[moved - 1] : p.n_pages;
  if (tid == 0) {
    *m.count = moved;
    info[0] = least;
    if (n_used) *n_used = moved < holes ? top : border;
  }
  if constexpr (kRename) {
    __syncthreads();
    if (moved == 0) return;
    for (int i = tid >> 6; i < p.batch; i += kPlanWaves) {   // a wave a row
      const int n = held_pages(clamp_len(p, p.lens[i]), p.shift);
      for (int j = tid & (kWave - 1); j < n; j += kWave) rename_row(p, p.table + (int64_t)i * p.stride, j, new_id, least);
    }
  }
}

__global__ __launch_bounds__(256) void pages_rename_kernel(PoolArg p, const int32_t* new_id, const int32_t* info) {
  const int least = info[0];
  if (least >= p.n_pages) return;
  for (int i = blockIdx.y; i < p.batch; i += gridDim.y) {
    const int n = held_pages(clamp_len(p, p.lens[i]), p.shift);
    for (int j = blockIdx.x * 256 + threadIdx.x; j < n; j += gridDim.x * 256) rename_row(p, p.table + (int64_t)i * p.stride, j, new_id, least);
  }
}

// ---- copies -----------------------------------------------------------------------------------------------------------------
// A wave per head of a layer's keys or values, for every gridDim.y-th move; four times 16 bytes of a lane on their way.
__global__ __launch_bounds__(256) void pages_copy_kernel(PagesCopyArgs a) {
  const int count = a.m.count ? min(*a.m.count, a.m.capacity) : a.m.capacity;
  const int vec = a.row_bytes / 16, lane = threadIdx.x & (kWave - 1);
  const uint32_t side = blockIdx.x * 4 + (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const uint32_t head = side % (uint32_t)a.hkv, layer = side / (uint32_t)a.hkv >> 1;
  const bool v = side / (uint32_t)a.hkv & 1;
  if (layer >= (uint32_t)a.n_layers) return;
  const int64_t f_page = v ? a.fv[0] : a.fk[0], f_tok = v ? a.fv[2] : a.fk[2], o_page = v ? a.tv[0] : a.tk[0], o_tok = v ? a.tv[2] : a.tk[2];
  const uint8_t* from_head = (v ? a.from_v[layer] : a.from_k[layer]) + head * (v ? a.fv[1] : a.fk[1]);
  uint8_t* to_head = (v ? a.to_v[layer] : a.to_k[layer]) + head * (v ? a.tv[1] : a.tk[1]);
  for (int move = blockIdx.y; move < count; move += gridDim.y) {
    const int src = a.m.src[move], dst = a.m.dst[move], some = a.m.rows ? a.m.rows[move] : a.page_size;
    if (src < 0 || src >= a.from_pages || dst < 0 || dst >= a.to_pages) continue;
    const int rows = min(max(some, 0), a.page_size);
    const uint8_t* f = from_head + src * f_page;
    uint8_t* o = to_head + dst * o_page;
    // rows of a head that lie one behind the other are one row
    const bool flat = f_tok == a.row_bytes && o_tok == a.row_bytes;
    const int each = flat ? kWave : kWave / vec;         // pieces, or rows, that a wave's lanes move at a time
    const int mine = flat ? lane : lane / vec, n = flat ? rows * vec : lane < each * vec ? rows : 0;
    const int64_t f_step = flat ? 16 : f_tok, o_step = flat ? 16 : o_tok, in_row = flat ? 0 : lane % vec * 16;
    auto from = [&](int i) { return *reinterpret_cast<const uint4*>(f + min(i, n - 1) * f_step + in_row); };
    auto to = [&](int i, const uint4& x) { if (i < n) *reinterpret_cast<uint4*>(o + i * o_step + in_row) = x; };
    for (int i = mine; i < n; i += each * 4) {
      const uint4 x0 = from(i), x1 = from(i + each), x2 = from(i + 2 * each), x3 = from(i + 3 * each);
      to(i, x0);
      to(i + each, x1);
      to(i + 2 * each, x2);
      to(i + 3 * each, x3);
    }
  }
}

}  // namespace

hipError_t launch_pages_update(const PoolArg& p, const int32_t* parents, const int32_t* keep, const int32_t* n_new, int n_new_all, const MovesArg& m,
                               int32_t* free_list, hipStream_t st) {
  const bool forks = parents || keep;
  if (forks && p.batch <= kForkInPlan && (int64_t)p.batch * p.per_seq <= kForkEntries) {
    pages_grow_kernel<true><<<dim3(1), kPlanThreads, 0, st>>>(p, parents, keep, n_new, n_new_all, m, free_list);
    return hipGetLastError();
  }
  if (forks) {
    int shift = 0;
    while ((p.batch << (shift + 1)) <= kForkSlots) ++shift;
    const int blocks = (int)(((int64_t)p.per_seq + (1 << shift) - 1) >> shift);
    pages_fork_kernel<<<dim3(blocks < 256 ? blocks : 256), kForkThreads, 0, st>>>(p, parents, keep);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  pages_grow_kernel<false><<<dim3(1), kPlanThreads, 0, st>>>(p, parents, keep, n_new, n_new_all, m, free_list);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PoolArg& p, int max_moves, const MovesArg& m, int32_t* n_used, int32_t* new_id, int32_t* info, hipStream_t st) {
  if ((int64_t)p.batch * p.per_seq <= kRenameEntries) {
    pages_compact_kernel<true><<<dim3(1), kPlanThreads, 0, st>>>(p, max_moves, m, n_used, new_id, info);
    return hipGetLastError();
  }
  pages_compact_kernel<false><<<dim3(1), kPlanThreads, 0, st>>>(p, max_moves, m, n_used, new_id, info);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int across = (p.per_seq + 255) / 256;
  pages_rename_kernel<<<dim3(across < 64 ? across : 64, p.batch < 1024 ? p.batch : 1024), 256, 0, st>>>(p, new_id, info);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PagesCopyArgs& a, hipStream_t st) {
  const int64_t across = ((int64_t)a.n_layers * 2 * a.hkv + 3) / 4;
  const int64_t down = std::min<int64_t>(a.m.capacity, std::max<int64_t>(4096 / across, 1));
  if (down == 0) return hipSuccess;
  pages_copy_kernel<<<dim3((unsigned)across, (unsigned)down), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace skv
