// Attention over a paged cache: the rule that picks a kernel, the launches, and the join of items that several workgroups
// shared (see paged_attn_kernels.hpp).  FP8 caches: kernels_paged_attn_fp8.hip.
#include "paged_attn_kernels.hpp"

namespace skv {

// Joins the parts of the items that are left unfinished, in ascending order: workgroup w of the first kernel began one
// (kPartTail, slot 2 w + 1), the workgroups behind it went on with it (kPartHead, slots 2 w') up to the one that finished it
// (kPartLast).  Groups of 32 threads, each with the columns of a row.  GROUPED (16 or 32 rows and up to hundreds of parts of a long
// cache): eight groups share the parts of one row; otherwise 32 groups have a row each and go through the block's rows.
template <bool GROUPED>
__global__ __launch_bounds__(GROUPED ? 256 : 1024) void paged_attn_join_kernel(PagedAttnArgs a, int block_rows) {
  const int w = blockIdx.x, tid = threadIdx.x, grp = tid >> 5, c = (tid & 31) * 4;
  const int4 desc = a.desc[w];
  if (!(desc.x & kPartTail)) return;
  const SeqRun run = get_run(a.runs, a.pt, desc.y);
  float m, l, x[4];
  int row, tl, g, tok;
  bool ok;
  auto start = [&](int r) {
    row = r;
    tl = row / a.G;
    g = row - tl * a.G;
    tok = desc.w * a.tb + tl;
    ok = tl < a.tb && tok < run.n && c < a.d;
    m = -INFINITY;
    l = x[0] = x[1] = x[2] = x[3] = 0.f;
  };
  auto add = [&](const float2 ml, const float4 v) {
    if (ml.x == -INFINITY && ml.y == 0.f) return;
    const float top = fmaxf(m, ml.x);
    const float fo = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top), fn = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
    m = top;
    l = l * fo + ml.y * fn;
    x[0] = x[0] * fo + v.x * fn; x[1] = x[1] * fo + v.y * fn; x[2] = x[2] * fo + v.z * fn; x[3] = x[3] * fo + v.w * fn;
  };
  auto part = [&](int64_t slot) {
    add(a.part_ml[slot * block_rows + row], *reinterpret_cast<const float4*>(a.part_acc + (slot * block_rows + row) * a.d + c));
  };
  auto finish = [&]() {
    const float f = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
    const int64_t qrow = run.start + tok;
    const int h = desc.z * a.G + g;
    *reinterpret_cast<uint2*>(a.out.p + qrow * a.out.tok + h * a.out.head + c * 2) =
        make_uint2(pack_bf16(x[0] * f, x[1] * f), pack_bf16(x[2] * f, x[3] * f));
    if (a.lse && c == 0) a.lse[qrow * a.hq + h] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
  };
  if constexpr (!GROUPED) {
    for (int r = grp; r < a.tb * a.G; r += 32) {
      start(r);
      if (!ok) continue;
      part(2 * (int64_t)w + 1);
      for (int i = w + 1; i < a.n_wg; ++i) {
        const int f = a.desc[i].x;
        if (f & kPartHead) part(2 * (int64_t)i);
        if (f & kPartLast) break;
      }
      finish();
    }
  } else {
    __shared__ float acc_s[8][128];
    __shared__ float2 ml_s[8];
    __shared__ int end_s;
    if (tid == 0) end_s = a.n_wg;
    __syncthreads();
    // the first that finished an item is the one that finished this
    for (int i = w + 1 + tid; i <= min((desc.x >> 3) + 1, a.n_wg - 1); i += 256)
      if (a.desc[i].x & kPartLast) atomicMin(&end_s, i);
    __syncthreads();
    const int end = min(end_s, a.n_wg - 1);
    start((int)blockIdx.y);
    if (tl >= a.tb || tok >= run.n) return;
    if (ok) {
#pragma unroll 4
      for (int i = w + grp; i <= end; i += 8)
        if (i == w) part(2 * (int64_t)w + 1);
        else if (a.desc[i].x & kPartHead) part(2 * (int64_t)i);
    }
    if (c < a.d) *reinterpret_cast<float4*>(&acc_s[grp][c]) = make_float4(x[0], x[1], x[2], x[3]);
    if (c == 0) ml_s[grp] = make_float2(m, l);
    __syncthreads();
    if (grp > 0 || c >= a.d) return;
    m = -INFINITY;
    l = x[0] = x[1] = x[2] = x[3] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) add(ml_s[i], *reinterpret_cast<const float4*>(&acc_s[i][c]));
    finish();
  }
}

int paged_attn_block_rows(int G, long rows) { return G <= 16 && rows <= 16 ? 16 : G <= 32 && rows <= 32 ? 32 : kTileRows; }
int paged_attn_workgroups(int block_rows) { return 512; }   // two per compute unit

hipError_t launch_paged_attention(PagedAttnArgs a, int block_rows, hipStream_t st) {
  hipError_t e = a.kv_bytes == 1 ? launch_paged_attn_fp8(a, block_rows, st) : launch_paged_attn_eb<2>(a, block_rows, st);
  if (e != hipSuccess) return e;
  if (block_rows == kTileRows) hipLaunchKernelGGL(paged_attn_join_kernel<false>, dim3(a.n_wg), dim3(1024), 0, st, a, block_rows);
  else hipLaunchKernelGGL(paged_attn_join_kernel<true>, dim3(a.n_wg, a.tb * a.G), dim3(256), 0, st, a, block_rows);
  return hipGetLastError();
}

}  // namespace skv
