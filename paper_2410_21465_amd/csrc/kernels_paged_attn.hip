// Attention over a paged cache: the rule that picks a kernel, the launches, and the join of items that several workgroups
// shared (see paged_attn_kernels.hpp).  FP8 caches: kernels_paged_attn_fp8.hip.
#include "paged_attn_kernels.hpp"

namespace skv {

// Joins the parts of the items that are left unfinished, in ascending order: workgroup w of the first kernel began one
// (kPartTail, slot 2 w + 1), the workgroups behind it went on with it (kPartHead, slots 2 w') up to the one that finished it
// (kPartLast).  Groups of 32 threads, each with the columns of a row.
struct Joined {   // a row's state as parts are added
  float m = -INFINITY, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ void add(const float2 ml, const float4 v) {
    if (ml.x == -INFINITY && ml.y == 0.f) return;
    const float top = fmaxf(m, ml.x);
    const float fo = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top), fn = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
    m = top;
    l = l * fo + ml.y * fn;
    x[0] = x[0] * fo + v.x * fn; x[1] = x[1] * fo + v.y * fn; x[2] = x[2] * fo + v.z * fn; x[3] = x[3] * fo + v.w * fn;
  }
  __device__ __forceinline__ void finish(const PagedAttnArgs& a, int64_t qrow, int h, int c) const {
    const float f = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
    *reinterpret_cast<uint2*>(a.out.p + qrow * a.out.tok + h * a.out.head + c * 2) =
        make_uint2(pack_bf16(x[0] * f, x[1] * f), pack_bf16(x[2] * f, x[3] * f));
    if (a.lse && c == 0) a.lse[qrow * a.hq + h] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
  }
};

// All is latency: one load and a vote find the parts, eight of them are requested at a time.
// The rows of an item are shared by the workgroups whose like worked at it.  Where it has few parts each group joins a
// row of its own, half of the groups for the item that began here and half for the one that goes on or ends here; where it has
// more, the groups share the parts of a row.  5 us for 31 parts of 4 rows, 11 us for some ten parts each of 60 ragged items of up to 32
// rows, 5 us behind a prompt of 8K tokens; 3 us of that go into finding the parts.  256 threads for up to 32 rows (with 512 the first
// two took 6 and 13, with 128 the 256 parts of a token over 1M keys 22 instead of 15), 512 for 128 rows (1024: 34 us against 28 for 32 tokens
// over 16.7K keys on 14/2 heads, the whole call).
constexpr int kMaxWg = 512;
template <int NT>
__global__ __launch_bounds__(NT) void paged_attn_join_kernel(PagedAttnArgs a, int block_rows) {
  static_assert(kMaxWg % NT == 0);
  constexpr int kGroups = NT / 32, kHalf = kGroups / 2, kAhead = 8, kWords = kMaxWg / kWave;
  __shared__ float acc_s[kGroups][128];
  __shared__ float2 ml_s[kGroups];
  __shared__ uint64_t tails[kWords], heads[kWords], lasts[kWords];
  const int me = blockIdx.x, tid = threadIdx.x, grp = tid >> 5, c = (tid & 31) * 4, col = min(c, a.d - 4);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave), n = a.n_wg;
  const int4 mine = a.desc[me];
#pragma unroll
  for (int i0 = 0; i0 < kMaxWg; i0 += NT) {
    const int i = i0 + tid, flags = i < n ? a.desc[i].x : 0;
    const uint64_t t = __ballot(flags & kPartTail), h = __ballot(flags & kPartHead), l = __ballot(flags & kPartLast);
    if (tid % kWave == 0) { tails[i / kWave] = t; heads[i / kWave] = h; lasts[i / kWave] = l; }
  }
  __syncthreads();
  auto end_of = [&](int w) {   // the first behind w that finished an item
    uint64_t m = w % 64 == 63 ? 0 : lasts[w / 64] >> (w % 64 + 1) << (w % 64 + 1);
    int i = w / 64;
    while (m == 0 && ++i < kWords) m = lasts[i];
    return m ? i * 64 + __ffsll((unsigned long long)m) - 1 : a.n_wg - 1;
  };
  auto begin_of = [&](int w) {   // the last before w that began one, -1: none
    uint64_t m = tails[w / 64] & ((1ull << (w % 64)) - 1);
    int i = w / 64;
    while (m == 0 && --i >= 0) m = tails[i];
    return m ? i * 64 + 63 - __clzll((long long)m) : -1;
  };
  struct Item { int w, parts; int4 desc; };
  auto item_of = [&](int e) {   // 0: what began here, 1: what lies around this workgroup's part; parts = 0: none
    const int w = e ? begin_of(me) : (mine.x & kPartTail ? me : -1);
    const int end = w < 0 ? -1 : end_of(w);
    if (end < me) return Item{0, 0, mine};
    return Item{w, end - w + 1, e ? a.desc[w] : mine};
  };
  // parts first, first + step, ... of R rows that lie row_step apart, kAhead / R parts at a time
  auto gather = [&](auto rows, const Item& it, int row, int row_step, int first, int step, Joined (&j)[decltype(rows)::value]) {
    constexpr int R = decltype(rows)::value, kParts = kAhead / R;
    for (int i0 = first; i0 < it.parts; i0 += step * kParts) {
      float2 ml[kAhead];
      float4 v[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {   // (places in the workspace, whatever they hold)
        const int i = min(i0 + k % kParts * step, it.parts - 1);
        const int64_t slot = (2 * (int64_t)(it.w + i) + (i == 0 ? 1 : 0)) * block_rows + min(row + k / kParts * row_step, it.desc.w - 1);
        ml[k] = a.part_ml[slot];
        v[k] = *reinterpret_cast<const float4*>(a.part_acc + slot * a.d + col);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = i0 + k % kParts * step;   // (workgroups inside that had less than a tile to do have no part)
        if (i < it.parts && (i == 0 || (heads[(it.w + i) / 64] >> ((it.w + i) % 64) & 1))) j[k / kParts].add(ml[k], v[k]);
      }
    }
  };
  auto finish = [&](const Item& it, const Joined& j, int row) {
    const int tl = row / a.G;
    if (c < a.d) j.finish(a, (int64_t)it.desc.y + tl, it.desc.z * a.G + row - tl * a.G, c);
  };
  const Item own = item_of(0), around = item_of(1);
  // One way takes a trip to memory per eight parts, the other one per row of a workgroup, of which it has rows / parts: the border
  // lies where parts^2 is some multiple of the rows.  Whole calls, at 3 / 12 / 48 times: 32 tokens over 8K and 30K keys on 32/4 heads 44.5 / 38.0 /
  // 38.0 and 69.6 / 63.2 / 63.3 us, over 16K on 32/8 heads 38.1 / 38.1 / 43.5, ten tokens over 3K on 32/2 heads 23.5 / 23.5 / 26.4.
  auto few = [&](const Item& it) { return it.parts * it.parts <= 12 * it.desc.w; };
  auto join_few = [&](const Item& it, bool is_own) {
    if (it.parts == 0 || !few(it)) return;
    const bool alone = it.desc.w <= kHalf;   // (joined where it began, whose descriptor is at hand)
    if (alone && !is_own) return;
    const int first = alone ? grp % kHalf : me - it.w + grp % kHalf * it.parts, step = alone ? kHalf : kHalf * it.parts;
    auto go = [&](auto rows) {
      constexpr int R = decltype(rows)::value;
      for (int row = first; row < it.desc.w; row += R * step) {
        Joined j[R];
        gather(rows, it, row, step, 0, 1, j);
#pragma unroll
        for (int r = 0; r < R; ++r)
          if (row + r * step < it.desc.w) finish(it, j[r], row + r * step);
      }
    };
    if (it.parts <= 2) go(std::integral_constant<int, 4>{});
    else if (it.parts <= 4) go(std::integral_constant<int, 2>{});
    else go(std::integral_constant<int, 1>{});
  };
  if (wave < NT / kWave / 2) join_few(own, true);
  else join_few(around, false);
  auto join_many = [&](const Item& it) {
    if (few(it)) return;
    for (int row = me - it.w; row < it.desc.w; row += it.parts) {
      Joined js[1];
      gather(std::integral_constant<int, 1>{}, it, row, 0, grp, kGroups, js);
      const Joined& j = js[0];
      __syncthreads();   // (the row before)
      if (c < a.d) *reinterpret_cast<float4*>(&acc_s[grp][c]) = make_float4(j.x[0], j.x[1], j.x[2], j.x[3]);
      if (c == 0) ml_s[grp] = make_float2(j.m, j.l);
      __syncthreads();
      if (grp == 0) {
        Joined all;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) all.add(ml_s[i], *reinterpret_cast<const float4*>(&acc_s[i][col]));
        finish(it, all, row);
      }
    }
  };
  join_many(own);
  join_many(around);
}

// (up to 32 rows the kernel that reads keys fastest and weighs in two terms, else the one with the most products per byte read)
int paged_attn_block_rows(int G, long rows) { return G <= 16 && rows <= 16 ? 16 : G <= 32 && rows <= 32 ? 32 : kTileRows; }
int paged_attn_workgroups() { return kMaxWg; }   // two per compute unit; a multiple of eight

hipError_t launch_paged_attention(PagedAttnArgs a, int block_rows, hipStream_t st) {
  hipError_t e = a.kv_bytes == 1 ? launch_paged_attn_fp8(a, block_rows, st) : launch_paged_attn_eb<2>(a, block_rows, st);
  if (e != hipSuccess) return e;
  if (block_rows == kTileRows) hipLaunchKernelGGL(paged_attn_join_kernel<512>, dim3(a.n_wg), dim3(512), 0, st, a, block_rows);
  else hipLaunchKernelGGL(paged_attn_join_kernel<256>, dim3(a.n_wg), dim3(256), 0, st, a, block_rows);
  return hipGetLastError();
}

}  // namespace skv
