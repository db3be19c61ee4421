// Rotary positions: heads turned to their tokens' positions, in memory of any strides (shadowkv_rotate) and on the way into a
// paged cache (shadowkv_paged_append).  For a pair (x_i, x_j) with frequency w and a = pos w:
//   y_i = m (x_i cos a - x_j sin a),  y_j = m (x_j cos a + x_i sin a).
// Both read what they are given once and write it once: HBM bounds them, and latency where there are few tokens.  The keys of four
// prompts of 32K tokens (8 heads of 128): 100 us, 5.4 TB/s, a copy's rate; 20K tokens of three sequences in FP8 85 us, 4.3 TB/s; six
// chunks into an FP8 cache 50 us, 4.7 TB/s (41 in the kernel); 16 tokens 5 us, 64 tokens appended 6 us.
//
// A thread owns one slot of a token -- P pairs, so 2 P elements: P from each half of the rotated part, or 2 P side by side --
// and takes it through up to kHeadsPerBlock heads: an angle costs an fp64 product, its reduction and two hardware functions, about as
// much as rotating three heads with it.  P = 8 makes 16-byte accesses in bf16; rotated parts that are no multiple of 16 take P = 4.
#include "kernels.hpp"

namespace skv {

constexpr int kRopeNT = 256;
constexpr int kHeadsPerBlock = 4;

template <int P>
struct Turn {
  float c[P], s[P];
};

// P elements as stored
template <int P, int EB>
struct Piece {
  uint32_t w[RawWords<P, EB>::n];
};
template <int P, int EB>
__device__ __forceinline__ void pack_f32(const float (&x)[P], Piece<P, EB>& o) {
#pragma unroll
  for (int i = 0; i < RawWords<P, EB>::n; ++i) {
    if constexpr (EB == 2) o.w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    else o.w[i] = pack_e5m2(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  }
}

// Cosines and sines of slot `slot` at position pos: the angle in fp64 revolutions, reduced to [-1/2, 1/2], then the hardware
// functions of 2 pi x.
template <int P>
__device__ __forceinline__ void make_turn(const RopeArgs& r, int slot, int64_t pos, Turn<P>& t) {
#pragma unroll
  for (int e = 0; e < P; ++e) {
    const int i = slot * P + e;
    const double f = r.inv_freq ? (double)r.inv_freq[i] * 0.15915494309189533577 : r.rev[i];
    const double rev = (double)pos * f;
    const float x = (float)(rev - rint(rev));
    t.c[e] = __builtin_amdgcn_cosf(x) * r.mag;
    t.s[e] = __builtin_amdgcn_sinf(x) * (r.mag * r.sign);
  }
}

// Elements at which the two pieces of a slot begin.
template <int P>
__device__ __forceinline__ void slot_at(const RopeArgs& r, int slot, bool turned, int& a, int& b) {
  const bool apart = turned && !r.interleaved;
  a = apart ? slot * P : slot * 2 * P;
  b = apart ? a + r.rot / 2 : a + P;
}

// The two pieces of a slot, as one access of 16 bytes where they lie side by side and are of 8 (rotate's FP8 heads, turned by pairs
// side by side or not turned: 104 us -> 85 us for 20K tokens of three sequences, 32 heads of 96).
typedef uint32_t U32x4 __attribute__((ext_vector_type(4), aligned(8)));
template <int P, int EB>
__device__ __forceinline__ void load_pieces(const uint8_t* p, int a, int b, Piece<P, EB>& x, Piece<P, EB>& y) {
  if constexpr (P * EB == 8) {
    if (b == a + P) {
      const U32x4 v = *reinterpret_cast<const U32x4*>(p + a * EB);
      x.w[0] = v[0]; x.w[1] = v[1]; y.w[0] = v[2]; y.w[1] = v[3];
      return;
    }
  }
  load_raw<P, EB>(p + a * EB, x.w);
  load_raw<P, EB>(p + b * EB, y.w);
}
template <int P, int EB>
__device__ __forceinline__ void store_pieces(uint8_t* p, int a, int b, const Piece<P, EB>& x, const Piece<P, EB>& y) {
  if constexpr (P * EB == 8) {
    if (b == a + P) {
      const U32x4 v = {x.w[0], x.w[1], y.w[0], y.w[1]};
      *reinterpret_cast<U32x4*>(p + a * EB) = v;
      return;
    }
  }
  store_raw<P, EB>(p + a * EB, x.w);
  store_raw<P, EB>(p + b * EB, y.w);
}

// One slot of n <= kHeadsPerBlock heads, src and dst at the first head.
template <int P, int EBI, int EBO>
__device__ __forceinline__ void turn_heads(const uint8_t* src, int64_t src_head, uint8_t* dst, int64_t dst_head, int n, int a, int b,
                                           bool turned, bool interleaved, const Turn<P>& t) {
  Piece<P, EBI> x[kHeadsPerBlock], y[kHeadsPerBlock];
#pragma unroll
  for (int h = 0; h < kHeadsPerBlock; ++h)
    if (h < n) load_pieces<P, EBI>(src + h * src_head, a, b, x[h], y[h]);
#pragma unroll
  for (int h = 0; h < kHeadsPerBlock; ++h) {
    if (h >= n) break;
    Piece<P, EBO> ox, oy;
    if (EBI == EBO && !turned) {
#pragma unroll
      for (int i = 0; i < RawWords<P, EBO>::n; ++i) { ox.w[i] = x[h].w[i]; oy.w[i] = y[h].w[i]; }
    } else {
      float u[P], v[P], p[P], q[P];
      unpack_kv<P, EBI>(x[h].w, u);
      unpack_kv<P, EBI>(y[h].w, v);
      if (!turned) {
#pragma unroll
        for (int e = 0; e < P; ++e) { p[e] = u[e]; q[e] = v[e]; }
      } else if (!interleaved) {
#pragma unroll
        for (int e = 0; e < P; ++e) {
          p[e] = u[e] * t.c[e] - v[e] * t.s[e];
          q[e] = v[e] * t.c[e] + u[e] * t.s[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < P / 2; ++e) {
          p[2 * e] = u[2 * e] * t.c[e] - u[2 * e + 1] * t.s[e];
          p[2 * e + 1] = u[2 * e + 1] * t.c[e] + u[2 * e] * t.s[e];
          q[2 * e] = v[2 * e] * t.c[P / 2 + e] - v[2 * e + 1] * t.s[P / 2 + e];
          q[2 * e + 1] = v[2 * e + 1] * t.c[P / 2 + e] + v[2 * e] * t.s[P / 2 + e];
        }
      }
      pack_f32<P, EBO>(p, ox);
      pack_f32<P, EBO>(q, oy);
    }
    store_pieces<P, EBO>(dst + h * dst_head, a, b, ox, oy);
  }
}

template <int P, int EBI, int EBO>
__global__ __launch_bounds__(kRopeNT) void rotate_kernel(RopeArgs rope, HeadsArg x, HeadsArg out, const int32_t* __restrict__ positions,
                                                         const int32_t* __restrict__ pos_offset, int n_tokens, int64_t total, int n_heads,
                                                         int slots, int tokens_per_wg) {
  const int tid = threadIdx.x, tl = tid / slots, slot = tid - tl * slots;
  const int64_t flat = (int64_t)blockIdx.x * tokens_per_wg + tl;
  if (tl >= tokens_per_wg || flat >= total) return;   // (total < 2^31)
  const int seq = (int)flat / n_tokens, tok = (int)flat - seq * n_tokens;
  const bool turned = slot < rope.rot / (2 * P);
  Turn<P> t{};
  if (turned) make_turn<P>(rope, slot, positions ? (int64_t)positions[flat] : (int64_t)(pos_offset ? pos_offset[seq] : 0) + tok, t);
  int a, b;
  slot_at<P>(rope, slot, turned, a, b);
  const int h0 = blockIdx.y * kHeadsPerBlock;
  turn_heads<P, EBI, EBO>(x.p + seq * x.seq + tok * x.tok + h0 * x.head, x.head, out.p + seq * out.seq + tok * out.tok + h0 * out.head,
                          out.head, min(kHeadsPerBlock, n_heads - h0), a, b, turned, rope.interleaved != 0, t);
}

template <int P, int EBI, int EBO>
static hipError_t launch_rotate_t(const RopeArgs& rope, const HeadsArg& x, const HeadsArg& out, const int32_t* positions,
                                  const int32_t* pos_offset, int64_t total, int n_tokens, int n_heads, hipStream_t st) {
  const int slots = rope.d / (2 * P), tokens = kRopeNT / slots;
  hipLaunchKernelGGL((rotate_kernel<P, EBI, EBO>), dim3((unsigned)((total + tokens - 1) / tokens), (n_heads + kHeadsPerBlock - 1) / kHeadsPerBlock),
                     dim3(kRopeNT), 0, st, rope, x, out, positions, pos_offset, n_tokens, total, n_heads, slots, tokens);
  return hipGetLastError();
}

hipError_t launch_rotate(const RopeArgs& rope, const HeadsArg& x, const HeadsArg& out, const int32_t* positions,
                         const int32_t* pos_offset, int n_seqs, int n_tokens, int n_heads, hipStream_t st) {
  const int64_t total = (int64_t)n_seqs * n_tokens;
  auto go = [&](auto p) {
    constexpr int P = decltype(p)::value;
    if (x.eb == 2) return out.eb == 2 ? launch_rotate_t<P, 2, 2>(rope, x, out, positions, pos_offset, total, n_tokens, n_heads, st)
                                      : launch_rotate_t<P, 2, 1>(rope, x, out, positions, pos_offset, total, n_tokens, n_heads, st);
    return out.eb == 2 ? launch_rotate_t<P, 1, 2>(rope, x, out, positions, pos_offset, total, n_tokens, n_heads, st)
                       : launch_rotate_t<P, 1, 1>(rope, x, out, positions, pos_offset, total, n_tokens, n_heads, st);
  };
  return rope.rot % 16 == 0 ? go(std::integral_constant<int, 8>{}) : go(std::integral_constant<int, 4>{});
}

// ---- append -----------------------------------------------------------------------------------------------------------
// blockIdx.y: first the blocks of key heads, as many of value heads, then those of query heads.  The sequence of a token is
// found by bisection of seq_starts, from LDS where they fit (64 sequences: six dependent reads there instead of from memory).
constexpr int kStartsInLds = 1024;

template <int P, int EBI, int EBO>
__global__ __launch_bounds__(kRopeNT) void append_paged_kernel(RopeArgs rope, int turn_keys, PagesArg kp, PagesArg vp, PageTableArg pt,
                                                               HeadsArg k, HeadsArg v, HeadsArg q, HeadsArg q_out, int hkv, int hq,
                                                               RunsArg runs, const int32_t* __restrict__ pos_offset, int slots,
                                                               int tokens_per_wg) {
  __shared__ int starts[kStartsInLds + 1];
  const bool in_lds = runs.seq_starts && runs.batch <= kStartsInLds;
  if (in_lds) {
    for (int i = threadIdx.x; i <= runs.batch; i += kRopeNT) starts[i] = runs.seq_starts[i];
    __syncthreads();
  }
  const int tid = threadIdx.x, tl = tid / slots, slot = tid - tl * slots;
  const int64_t tok64 = (int64_t)blockIdx.x * tokens_per_wg + tl;
  if (tl >= tokens_per_wg || tok64 >= runs.n_tokens) return;
  const int tok = (int)tok64;
  int seq, end;   // the sequence, and the row behind its last
  if (!runs.seq_starts) {
    const int each = runs.n_tokens / runs.batch;
    seq = tok / each;
    end = (seq + 1) * each;
  } else {
    const int32_t* __restrict__ g = runs.seq_starts;
    int lo = 0, hi = runs.batch + 1;   // number of entries <= tok, in [lo, hi]
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if ((in_lds ? starts[mid] : g[mid]) <= tok) lo = mid + 1; else hi = mid;
    }
    seq = lo - 1;
    if (seq < 0 || seq >= runs.batch) return;   // outside every run
    end = min(in_lds ? starts[seq + 1] : g[seq + 1], runs.n_tokens);   // (held to the rows there are, as attention holds it)
  }
  const int64_t place = (int64_t)runs.kv_lens[seq] - ((int64_t)end - tok);
  const int blocks = (hkv + kHeadsPerBlock - 1) / kHeadsPerBlock, y = blockIdx.y;
  const bool is_v = y >= blocks && y < 2 * blocks, is_q = y >= 2 * blocks;
  const bool turned = !is_v && turn_keys && slot < rope.rot / (2 * P);
  Turn<P> t{};
  if (turned) make_turn<P>(rope, slot, place + (pos_offset ? pos_offset[seq] : 0), t);
  int a, b;
  slot_at<P>(rope, slot, turned, a, b);
  if (is_q) {
    const int h0 = (y - 2 * blocks) * kHeadsPerBlock;
    turn_heads<P, 2, 2>(q.p + tok * q.tok + h0 * q.head, q.head, q_out.p + tok * q_out.tok + h0 * q_out.head, q_out.head,
                        min(kHeadsPerBlock, hq - h0), a, b, turned, rope.interleaved != 0, t);
    return;
  }
  if (place < 0 || (place >> pt.shift) >= pt.per_seq) return;
  const int page = pt.table[seq * pt.stride + (place >> pt.shift)];
  if ((unsigned)page >= (unsigned)pt.n_pages) return;
  const int h0 = (is_v ? y - blocks : y) * kHeadsPerBlock, n = min(kHeadsPerBlock, hkv - h0);
  const int row = (int)(place & ((1 << pt.shift) - 1));
  const HeadsArg& from = is_v ? v : k;
  const PagesArg& to = is_v ? vp : kp;
  turn_heads<P, EBI, EBO>(from.p + tok * from.tok + h0 * from.head, from.head, to.p + page * to.page + h0 * to.head + row * to.tok, to.head,
                          n, a, b, turned, rope.interleaved != 0, t);
}

template <int P, int EBI, int EBO>
static hipError_t launch_append_t(const RopeArgs& rope, int turn_keys, const PagesArg& kp, const PagesArg& vp, const PageTableArg& pt,
                                  const HeadsArg& k, const HeadsArg& v, const HeadsArg& q, const HeadsArg& q_out, int hkv, int hq,
                                  const RunsArg& runs, const int32_t* pos_offset, hipStream_t st) {
  const int slots = rope.d / (2 * P), tokens = kRopeNT / slots;
  const int y = 2 * ((hkv + kHeadsPerBlock - 1) / kHeadsPerBlock) + (hq + kHeadsPerBlock - 1) / kHeadsPerBlock;
  hipLaunchKernelGGL((append_paged_kernel<P, EBI, EBO>), dim3((unsigned)(((int64_t)runs.n_tokens + tokens - 1) / tokens), y), dim3(kRopeNT), 0, st,
                     rope, turn_keys, kp, vp, pt, k, v, q, q_out, hkv, hq, runs, pos_offset, slots, tokens);
  return hipGetLastError();
}

hipError_t launch_paged_append(const RopeArgs* rope, const PagesArg& kp, const PagesArg& vp, const PageTableArg& pt, int kv_bytes,
                               const HeadsArg& k, const HeadsArg& v, const HeadsArg& q, const HeadsArg& q_out, int d, int hkv,
                               int hq, const RunsArg& runs, const int32_t* pos_offset, hipStream_t st) {
  RopeArgs r{};
  if (rope) r = *rope;
  r.d = d;
  const int turn = rope ? 1 : 0;
  auto go = [&](auto p) {
    constexpr int P = decltype(p)::value;
    if (k.eb == 1) return launch_append_t<P, 1, 1>(r, turn, kp, vp, pt, k, v, q, q_out, hkv, hq, runs, pos_offset, st);
    return kv_bytes == 2 ? launch_append_t<P, 2, 2>(r, turn, kp, vp, pt, k, v, q, q_out, hkv, hq, runs, pos_offset, st)
                         : launch_append_t<P, 2, 1>(r, turn, kp, vp, pt, k, v, q, q_out, hkv, hq, runs, pos_offset, st);
  };
  return r.rot % 16 == 0 ? go(std::integral_constant<int, 8>{}) : go(std::integral_constant<int, 4>{});
}

}  // namespace skv
