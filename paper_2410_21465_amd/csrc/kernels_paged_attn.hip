// Attention over a paged cache: the rule that picks a kernel, the launches, and the join of items that several workgroups
// shared (see paged_attn_kernels.hpp).  FP8 caches: kernels_paged_attn_fp8.hip.
#include "paged_attn_kernels.hpp"

namespace skv {

// Joins the parts of the items that are left unfinished, in ascending order: workgroup w of the first kernel began one
// (kPartTail, slot 2 w + 1), the workgroups behind it went on with it (kPartHead, slots 2 w') up to the one that finished it
// (kPartLast).  256 threads: eight groups of 32, each with the columns of a row.  GROUPED: the groups share the parts of one row
// (long caches, hundreds of parts); otherwise each has a row of its own.
template <bool GROUPED>
__global__ __launch_bounds__(256) void paged_attn_join_kernel(PagedAttnArgs a, int block_rows) {
  const int w = blockIdx.x, tid = threadIdx.x, grp = tid >> 5, c = (tid & 31) * 4;
  const int4 desc = a.desc[w];
  if (!(desc.x & kPartTail)) return;
  __shared__ int end_s;
  __shared__ float acc_s[8][128];
  __shared__ float2 ml_s[8];
  if (tid == 0) end_s = a.n_wg - 1;
  __syncthreads();
  for (int i = w + 1 + tid; i < a.n_wg; i += 256)
    if (a.desc[i].x & kPartLast) atomicMin(&end_s, i);
  __syncthreads();
  const int end = end_s, row = GROUPED ? (int)blockIdx.y : (int)blockIdx.y * 8 + grp;
  const SeqRun run = get_run(a.runs, a.pt, desc.y);
  const int tl = row / a.G, g = row - tl * a.G, tok = desc.w * a.tb + tl;
  const bool ok = row < block_rows && tl < a.tb && tok < run.n && c < a.d;
  if (GROUPED && !(tl < a.tb && tok < run.n)) return;
  float m = -INFINITY, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](int64_t slot) {
    const float2 ml = a.part_ml[slot * block_rows + row];
    const float4 v = *reinterpret_cast<const float4*>(a.part_acc + (slot * block_rows + row) * a.d + c);
    if (ml.x == -INFINITY && ml.y == 0.f) return;
    const float top = fmaxf(m, ml.x);
    const float fo = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top), fn = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
    m = top;
    l = l * fo + ml.y * fn;
    x[0] = x[0] * fo + v.x * fn; x[1] = x[1] * fo + v.y * fn; x[2] = x[2] * fo + v.z * fn; x[3] = x[3] * fo + v.w * fn;
  };
  if (ok) {
    const int step = GROUPED ? 8 : 1;
#pragma unroll 4
    for (int i = w + (GROUPED ? grp : 0); i <= end; i += step)
      if (i == w) add(2 * (int64_t)w + 1);
      else if (a.desc[i].x & kPartHead) add(2 * (int64_t)i);
  }
  if (GROUPED) {
    if (c < a.d) *reinterpret_cast<float4*>(&acc_s[grp][c]) = make_float4(x[0], x[1], x[2], x[3]);
    if (c == 0) ml_s[grp] = make_float2(m, l);
    __syncthreads();
    if (grp > 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, ml_s[i].x);
    m = top;
    l = 0.f;
    x[0] = x[1] = x[2] = x[3] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 ml = ml_s[i];
      if (ml.x == -INFINITY && ml.y == 0.f) continue;
      const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
      l += ml.y * f;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += (c < a.d ? acc_s[i][c + e] : 0.f) * f;
    }
  }
  if (!ok) return;
  const float f = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
  const int64_t qrow = run.start + tok;
  const int h = desc.z * a.G + g;
  *reinterpret_cast<uint2*>(a.out.p + qrow * a.out.tok + h * a.out.head + c * 2) =
      make_uint2(pack_bf16(x[0] * f, x[1] * f), pack_bf16(x[2] * f, x[3] * f));
  if (a.lse && c == 0) a.lse[qrow * a.hq + h] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

int paged_attn_block_rows(int G, long rows) { return G <= 16 && rows <= 16 ? 16 : G <= 32 && rows <= 32 ? 32 : kTileRows; }
int paged_attn_workgroups(int block_rows) { return 512; }   // two per compute unit

hipError_t launch_paged_attention(PagedAttnArgs a, int block_rows, hipStream_t st) {
  hipError_t e = a.kv_bytes == 1 ? launch_paged_attn_fp8(a, block_rows, st) : launch_paged_attn_eb<2>(a, block_rows, st);
  if (e != hipSuccess) return e;
  if (block_rows == kTileRows)
    hipLaunchKernelGGL(paged_attn_join_kernel<false>, dim3(a.n_wg, kTileRows / 8), dim3(256), 0, st, a, block_rows);
  else
    hipLaunchKernelGGL(paged_attn_join_kernel<true>, dim3(a.n_wg, a.tb * a.G), dim3(256), 0, st, a, block_rows);
  return hipGetLastError();
}

}  // namespace skv
