// Attention over a paged cache stored as FP8 E5M2: the kernels of paged_attn_kernels.hpp on one-byte elements (a file of its
// own so that the two compile side by side).
#include "paged_attn_kernels.hpp"

namespace skv {

hipError_t launch_paged_attn_fp8(const PagedAttnArgs& a, int block_rows, hipStream_t st) { return launch_paged_attn_eb<1>(a, block_rows, st); }

}  // namespace skv
