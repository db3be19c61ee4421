// Attention of new tokens over a paged cache (shadowkv_paged_attention):
//   out = sum over the places l a row sees of softmax_l(scale <q, k_l>) v_l.
// A row is one (token, query head); the G = h_q / h_kv rows of a token that share a KV head lie side by side in a block of rows, so
// that K and V are read once for all of them.  One pass over the keys with a reference m of the logits and a running sum l in fp32
// (log2 units): a tile's logits S, P = 2^(S - m), l' = l + sum P, O' = O + P V, out = O / l, lse = m + log l.  Where a logit passes m, m
// moves 2^8 beyond the largest one (l and O by the same factor), so that it seldom moves and no weight ever passes one: P V overflows
// only where the softmax with its maximum taken out would too.  (With m at the maximum, and weights of up to 2^8 let through before it
// moves, which is the same arithmetic 2^8 higher up, finite values from 2^120 on came out infinite.)  The largest weight lies in
// [2^-8, 1]; weights and sums are fp32, whose exponents have room for that at the lower end: bf16's smallest values come out exact.
// A row's m follows its own logits alone, so that no bit of its result depends on the rows beside it and on keys that only they see.
//
// Both kernels form S^T = K Q^T, so that a lane of the matrix instruction's result holds one row's logits: the maximum
// and the sum stay in the lane but for one exchange, the factors of a row are scalars of its lane, and P^T is already laid out as
// the right operand of O^T = V^T P^T.  V^T is read from LDS with the transposing loads (ds_read_b64_tr_b16: lane i of 16 gets
// column i of four rows of 16; checked on the chip).  The order of the keys inside a product is the one in which S^T leaves them.
//
// The work is shared out to at most n_wg workgroups without the host knowing any length.  An item is (sequence, KV head, row block), in
// that order; its work is counted in keys, kItemKeys for itself and what its last row sees at most.  Workgroup w
// takes the keys [w X / n, (w + 1) X / n) of the whole, X its sum, cut at tiles; an item that it leaves unfinished goes to the
// workspace as (m, l, O), and a second kernel joins the parts in ascending order.  A long cache with few rows is split so, and many
// short sequences are packed.
#pragma once
#include "kernels.hpp"

namespace skv {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kItemKeys = 128;   // what starting and ending an item costs, in keys
constexpr int kPartTail = 1, kPartHead = 2, kPartLast = 4;   // flags of a workgroup's unfinished items

// ---- sharing out ----------------------------------------------------------------------------------------------------
struct SeqRun {
  int start, n, len;   // first row, new tokens, tokens in the cache
  int first;           // place of the first new token (below 0 or beyond len where the cache does not hold it)
};
__device__ __forceinline__ SeqRun get_run(const RunsArg& r, const PageTableArg& pt, int i) {
  SeqRun s;
  if (r.seq_starts) {   // (held to [0, T]: whatever the array says, rows stay inside q and out)
    const int lo = min(max(r.seq_starts[i], 0), r.n_tokens), hi = min(max(r.seq_starts[i + 1], 0), r.n_tokens);
    s.start = lo;
    s.n = max(0, hi - lo);
  } else {
    s.n = r.n_tokens / r.batch;
    s.start = i * s.n;
  }
  const int len = max(r.kv_lens[i], 0);
  s.len = (int)min((int64_t)len, (int64_t)pt.per_seq << pt.shift);
  s.first = len - s.n;
  return s;
}
// Work of one head of a sequence, in keys.  Block m's is base + slope (m + 1); the blocks are taken from both ends in turn (last,
// first, last but one, ...), so that any even number of neighbours is the same work.
struct SeqCost {
  int64_t base, slope;
  int blocks;
  __device__ __forceinline__ int block(int p) const { return p % 2 ? p / 2 : blocks - 1 - p / 2; }   // the p-th one taken
  __device__ __forceinline__ int64_t cost(int p) const { return base + slope * (block(p) + 1); }
  __device__ __forceinline__ int64_t pair() const { return 2 * base + slope * (blocks + 1); }
  __device__ __forceinline__ int64_t before(int p) const { return p / 2 * pair() + (p % 2 ? cost(p - 1) : 0); }
  __device__ __forceinline__ int64_t head() const { return before(blocks); }
};
__device__ __forceinline__ SeqCost get_cost(const SeqRun& s, int tb, int causal) {
  SeqCost c;
  c.blocks = (s.n + tb - 1) / tb;
  c.base = kItemKeys + (causal ? min(max(s.first, 0), s.len) : s.len);
  c.slope = causal ? tb : 0;
  return c;
}

__device__ __forceinline__ int64_t uniform64(int64_t x) {   // a value that all lanes hold, in scalar registers
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

struct Share {
  int64_t x0, x1;     // this workgroup's part of the work
  int w;              // its number
  bool idle;          // there is no part for it
  int seq, head, p;   // the item in which x0 lies (the p-th block taken of a head),
  int64_t xs;         // and where that begins
};

// a / b for 0 <= a < 2^52, b > 0, through fp64: the quotient is off by one at most before it is put right (the compiler's 64-bit
// division is some hundred instructions)
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  int64_t q = (int64_t)((double)a * (1.0 / (double)b));
  const int64_t r = a - q * b;
  if (r < 0) --q;
  if (r >= b) ++q;
  return q;
}
// inclusive sum over the wave's lanes, as wave_incl_scan_u32
__device__ __forceinline__ int64_t dpp_add_i64(int64_t x, int lo, int hi) { return x + (int64_t)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo); }
__device__ __forceinline__ int64_t wave_scan_i64(int64_t x) {
#define SKV_STEP(CTRL, MASK)                                                                        \
  x = dpp_add_i64(x, __builtin_amdgcn_update_dpp(0, (int)x, CTRL, MASK, 0xf, false),                \
                  __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, MASK, 0xf, false));
  SKV_STEP(0x111, 0xf) SKV_STEP(0x112, 0xf) SKV_STEP(0x114, 0xf) SKV_STEP(0x118, 0xf) SKV_STEP(0x142, 0xa) SKV_STEP(0x143, 0xc)
#undef SKV_STEP
  return x;
}
__device__ __forceinline__ int64_t last_lane_i64(int64_t x) {
  return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), kWave - 1) << 32) |
                   (uint32_t)__builtin_amdgcn_readlane((int)x, kWave - 1));
}

// Every wave for itself, 64 sequences at a time; found: 8 int64 of LDS of its own.
__device__ __forceinline__ Share get_share(const PagedAttnArgs& a, int64_t* found) {
  const int lane = threadIdx.x & (kWave - 1), b = a.runs.batch;
  auto cost_of = [&](int i, SeqCost& c) {
    c = get_cost(get_run(a.runs, a.pt, min(i, b - 1)), a.tb, a.causal);
    return i < b ? c.head() * a.hkv : 0;
  };
  SeqCost c;
  int64_t incl = wave_scan_i64(cost_of(lane, c)), total = last_lane_i64(incl);   // of the first 64
  for (int i0 = kWave; i0 < b; i0 += kWave) {
    SeqCost d;
    total += last_lane_i64(wave_scan_i64(cost_of(i0 + lane, d)));
  }
  Share sh;
  const int64_t n64 = quotient(total + a.min_share - 1, a.min_share);
  const int n = (int)(n64 < a.n_wg ? n64 : a.n_wg);
  // neighbouring shares to one XCD (workgroups go round the eight of them), whose L2 then holds a head's K and V for all
  // (n_wg is a multiple of eight, and every number below it is some workgroup's)
  const int per = (n + 7) / 8, x = (int)blockIdx.x % 8, y = (int)blockIdx.x / 8, w = y < per ? x * per + y : 8 * y + x;
  sh.w = w;
  sh.idle = w >= n;
  if (sh.idle) return sh;
  const int64_t each = quotient(total, n);
  const int more = (int)(total - each * n);   // (below n, and n below 2^11)
  const int64_t cut0 = each * w + more * w / n, cut1 = each * (w + 1) + more * (w + 1) / n;
  // A cut within `near` keys of an item's end is made there: a split item costs its parts' way through memory (a prompt of 8K tokens,
  // together with the order of the blocks: 686 -> 620 us).
  const int64_t near = min(max((int64_t)kItemKeys, each / 32), each / 8);
  int64_t before = 0;   // work of the sequences before these 64
  if (lane == 0) found[4] = w + 1 == n ? total : -1;
  for (int i0 = 0; i0 < b; i0 += kWave) {
    if (i0 > 0) {
      before += last_lane_i64(incl);
      incl = wave_scan_i64(cost_of(i0 + lane, c));
    }
    const int64_t mine = i0 + lane < b ? c.head() * a.hkv : 0, from = before + incl - mine;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int64_t cut = e ? cut1 : cut0;
      if (mine > 0 && cut >= from && cut < from + mine) {
        const int64_t head = c.head();
        int64_t h = quotient(cut - from, head);
        const int64_t rest = (cut - from) - h * head;
        int p = 2 * (int)quotient(rest, c.pair());
        if (rest - c.before(p) >= c.cost(p)) ++p;
        const int64_t left = rest - c.before(p), right = c.cost(p) - left;
        int64_t at = cut;
        if (left <= near && left <= right) at = cut - left;
        else if (right <= near) at = cut + right;
        if (e) {
          found[4] = at;
        } else {
          int s = i0 + lane;
          if (at == cut + right && ++p == c.blocks) {   // the item behind
            p = 0;
            if (++h == a.hkv) {
              h = 0;
              do ++s; while (s < b && get_run(a.runs, a.pt, s).n == 0);
            }
          }
          found[0] = s;
          found[1] = h;
          found[2] = p;
          found[3] = at;
          found[5] = at == cut ? at - left : at;
        }
      }
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (written by one lane, read by all)
  __builtin_amdgcn_wave_barrier();
  sh.seq = __builtin_amdgcn_readfirstlane((int)found[0]);
  sh.head = __builtin_amdgcn_readfirstlane((int)found[1]);
  sh.p = __builtin_amdgcn_readfirstlane((int)found[2]);
  sh.x0 = uniform64(found[3]);
  sh.x1 = uniform64(found[4]);
  sh.xs = uniform64(found[5]);
  sh.idle = sh.x0 >= sh.x1;
  return sh;
}

// The workgroup's items one after the other: work(run, seq, head, blk, first tile, last tile + 1, part slot or -1).  What is only wanted
// between items waits in LDS (a copy per wave): in scalar registers it made the loops over keys spill theirs.  Ten to 63 scalar registers
// are still put into lanes of vector registers, outside those loops but for two to five reads a tile in the branch for masked ones.
template <int TILE, class F>
__device__ __forceinline__ void for_items(const PagedAttnArgs& a, F&& work) {
  struct State {
    int64_t x0, x1, xs;
    int w, seq, head, p, done;
    int4 desc;
  };
  __shared__ int64_t found[4][8];   // (256 threads)
  __shared__ State state[4];
  State& st = state[threadIdx.x / kWave];
  {
    const Share sh = get_share(a, found[threadIdx.x / kWave]);
    if (sh.idle) {   // every entry of desc is written by every call
      if (threadIdx.x == 0) a.desc[sh.w] = make_int4(0, 0, 0, 0);
      return;
    }
    st.x0 = sh.x0; st.x1 = sh.x1; st.xs = sh.xs;
    st.w = sh.w; st.seq = sh.seq; st.head = sh.head; st.p = sh.p; st.done = 0;
    st.desc = make_int4(0, 0, 0, 0);
  }
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  while (true) {
    asm volatile("" ::: "memory");
    if (uniform(st.done)) break;
    const int seq = uniform(st.seq), head = uniform(st.head), p = uniform(st.p), w = uniform(st.w);
    const int64_t xs = uniform64(st.xs), x0 = uniform64(st.x0), x1 = uniform64(st.x1);
    const SeqRun run = get_run(a.runs, a.pt, seq);
    const SeqCost c = get_cost(run, a.tb, a.causal);
    const int64_t cost = c.cost(p);
    const int blk = c.block(p);
    const int seen = a.causal ? min(max(run.first + min(run.n, (blk + 1) * a.tb), 0), run.len) : run.len;
    const int tiles = (seen + TILE - 1) / TILE;
    auto tile_at = [&](int64_t x) {
      return x >= cost ? tiles : x <= kItemKeys ? 0 : (int)min((int64_t)tiles, (x - kItemKeys) / TILE);
    };
    const int t0 = tile_at(x0 - xs), t1 = tile_at(x1 - xs);
    const bool some = t0 < t1 || (tiles == 0 && xs >= x0);
    int slot = -1;
    if (some) {
      if (t0 > 0) {
        slot = 2 * w;
        st.desc.x |= kPartHead | (t1 == tiles ? kPartLast : 0);
      } else if (t1 < tiles) {
        slot = 2 * w + 1;
        st.desc = make_int4(uniform(st.desc.x) | kPartTail, run.start + blk * a.tb, head, min(a.tb, run.n - blk * a.tb) * a.G);
      }
    }
    st.xs = xs + cost;
    if (xs + cost >= x1) {
      st.done = 1;
      if (threadIdx.x == 0) a.desc[w] = st.desc;
    } else if (p + 1 < c.blocks) {
      st.p = p + 1;
    } else {
      st.p = 0;
      if (head + 1 < a.hkv) {
        st.head = head + 1;
      } else {
        st.head = 0;
        int s = seq;
        do ++s; while (get_run(a.runs, a.pt, s).n == 0);   // (xs < x1: there is one)
        st.seq = s;
      }
    }
    asm volatile("" ::: "memory");
    if (some) work(run, seq, head, blk, t0, t1, slot);
  }
}

// ---- elements -------------------------------------------------------------------------------------------------------
// upper halves of two 32-bit words
__device__ __forceinline__ uint32_t upper_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }
// four E5M2 bytes as four bf16 (exact)
__device__ __forceinline__ uint2 e5m2x4_to_bf16(uint32_t w) {
  const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true);
  return make_uint2(upper_halves(__float_as_uint(lo[0]), __float_as_uint(lo[1])),
                    upper_halves(__float_as_uint(hi[0]), __float_as_uint(hi[1])));
}
// whether one of two bf16 is infinite or NaN
__device__ __forceinline__ bool not_finite(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
// the same of four E5M2 bytes
__device__ __forceinline__ bool not_finite_e5m2(uint32_t w) { return ((w & 0x7c7c7c7cu) + 0x04040404u) & 0x80808080u; }
// the same two with infinities and NaN as zero
__device__ __forceinline__ uint32_t only_finite(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
}
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
// transposing load: four rows of 16 columns from the 16 lanes' addresses; lane i gets column i
__device__ __forceinline__ uint2 read_tr(const uint8_t* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
}
__device__ __forceinline__ float max_halves(float x) {   // over lanes l and l ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_quarters(float x) {  // over the four lanes l % 16
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_quarters(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return sum_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kHeadroom = 8.f;   // how far beyond the largest logit the reference of a row moves, in powers of two

// Where a key's rows lie: offsets of its K and V rows (head excluded) in 16-byte units (the host sees to it that they fit).  Keys
// without a row get the cache's first one (in bounds; what is read there is masked out) and ok = false.
struct KeyRow {
  uint32_t k, v;
  bool ok;
};
// (always a load, of the last token's entry for keys behind it: whether the key has a row is asked when the entry is used)
__device__ __forceinline__ int page_entry(const PagedAttnArgs& a, const int32_t* table, int key, int len) {
  return table[min(key, max(len - 1, 0)) >> a.pt.shift];
}
__device__ __forceinline__ KeyRow key_row(const PagedAttnArgs& a, int page, int key, int len) {
  KeyRow r;
  r.ok = key < len && (unsigned)page < (unsigned)a.pt.n_pages;
  const uint32_t pg = r.ok ? page : 0, row = r.ok ? (key & ((1 << a.pt.shift) - 1)) : 0;
  r.k = pg * (uint32_t)(a.kp.page >> 4) + row * (uint32_t)(a.kp.tok >> 4);
  r.v = pg * (uint32_t)(a.vp.page >> 4) + row * (uint32_t)(a.vp.tok >> 4);
  return r;
}
__device__ __forceinline__ uint64_t row_offset(uint32_t units, int src) {   // bytes, of lane src's key
  return (uint64_t)(uint32_t)__shfl((int)units, src, kWave) << 4;
}

// ---- 128 rows: the four waves of a workgroup take 32 rows each -----------------------------------------------------------
// Tiles of 64 keys, K and V through registers into two LDS buffers: while one tile is multiplied the next is on its way, one barrier a
// tile.  FP8 is widened to bf16 between registers and LDS.  Per tile a wave issues D / 4 v_mfma_f32_32x32x16_bf16.
// Row pitches: K's 16-byte reads of 16 rows and V's transposing reads of four rows of 64 bytes fall on all 64 banks.
//
// Bound by the matrix pipe and the softmax's vector instructions, each busy for 44 % of a prompt's cycles: with two waves per SIMD
// (256 registers a wave) they overlap only in part.  32/8 heads of 128: a prompt of 8K tokens 605 us = 0.91 PFLOP/s, 2K tokens after
// 28K 1.04 ms = 0.94 PFLOP/s, on other cards up to 693 us and 1.19 ms (a bf16 product of 8192^3 reaches 1.3; zeros in place of random
// data run a third faster there and a quarter here: both are held by power).  Slower: the next tile's first half multiplied behind the
// weights (710 against 687 us),
// 64 rows a wave and one wave per SIMD (0.5 to 0.7 of the rate), the maximum settled per 32 keys (643 against 621 us).
// The weights are rounded to bf16 for P V, since a second term as for few rows would make half as many products again of what bounds the
// kernel; the sum l takes them unrounded.  Each is off by 2^-8 of itself at most, either way, so the errors of a row's many keys
// cancel for the most part: against 64 bits the outputs of a prompt and of chunks are off by 0.0022 of their size (root mean square), where
// their own rounding to bf16 alone makes 0.0017.
constexpr int kTileKeys = 64, kTileRows = 128, kTileNT = 256;
template <int D>
struct TilePitch {
  static constexpr int k = 2 * D + 16;
  static constexpr int v = D == 128 ? 320 : 192;
  static constexpr int bytes = kTileKeys * (k + v);
};

template <int D, int EB>
__global__ __launch_bounds__(kTileNT, 2) void paged_attn_tiles_kernel(PagedAttnArgs a) {
  constexpr int kPieces = D * EB / 16;                                   // 16-byte pieces of a row
  constexpr int kLoads = (kTileKeys * kPieces + kTileNT - 1) / kTileNT;  // per thread, for K and for V
  constexpr bool kEven = kTileKeys * kPieces % kTileNT == 0;
  constexpr int PK = TilePitch<D>::k, PV = TilePitch<D>::v, QS = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * TilePitch<D>::bytes];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, col = lane & 31, half = lane >> 5;
  // this thread's pieces of a tile: piece pc of rows pr + j kRowStep (a row's pieces lie on neighbouring threads)
  const int pr = tid / kPieces, pc = tid - pr * kPieces;

  for_items<kTileKeys>(a, [&](const SeqRun& run, int seq, int head, int blk, int t0, int t1, int slot) {
    const int G = a.G, row = wave * 32 + col, tl = row / G, g = row - tl * G, tok = blk * a.tb + tl;
    const bool row_ok = tl < a.tb && tok < run.n;
    const int limit = row_ok ? (a.causal ? run.first + tok : run.len - 1) : -1;   // last key the row sees
    // tiles before `clear` are seen whole by every row of the block
    const int first = a.causal ? run.first + blk * a.tb : run.len - 1, clear = max(first + 1, 0) / kTileKeys;
    const int64_t qrow = run.start + tok;
    bf16x8 qf[QS];
    {
      // (rows that are none take row 0 of q: what they make is not written)
      const uint8_t* qp = a.q.p + (row_ok ? qrow * a.q.tok + (head * G + g) * a.q.head : 0) + half * 16;
#pragma unroll
      for (int s = 0; s < QS; ++s) {
        qf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(qp + s * 32));
      }
    }
    // (waited for here: left to the loop's first products, every turn of it would wait as long)
#pragma unroll
    for (int i = 0; i < QS; ++i) asm volatile("" : "+v"(qf[i]));
    f32x16 o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    float m = -INFINITY, l = 0.f;

    const int32_t* table = a.pt.table + seq * a.pt.stride;
    const uint8_t* kbase = a.kp.p + head * a.kp.head;
    const uint8_t* vbase = a.vp.p + head * a.vp.head;
    KeyRow kv{0, 0, false};   // of key `lane` of the tile on its way
    uint64_t have = 0;        // keys of it that have a row
    uint4 stage[kLoads];
    // (a piece's row is found again from its number: j * 256 / kPieces rows on where that is whole)
    auto piece = [&](int j, int& r, int& c) {
      if constexpr (kTileNT % kPieces == 0) { r = pr + j * (kTileNT / kPieces); c = pc; }
      else { const int p = tid + j * kTileNT; r = p / kPieces; c = p - r * kPieces; }
    };
    uint32_t at_k[kLoads], at_v[kLoads];   // where the rows of this thread's pieces lie, from the lanes that looked them up
    auto locate = [&]() {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        int r, c;
        piece(j, r, c);
        at_k[j] = (uint32_t)__shfl((int)kv.k, r, kWave);
        at_v[j] = (uint32_t)__shfl((int)kv.v, r, kWave);
      }
    };
    auto request = [&](const uint8_t* base, const uint32_t (&at)[kLoads]) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        if (kEven || tid + j * kTileNT < kTileKeys * kPieces) {
          int r, c;
          piece(j, r, c);
          stage[j] = *reinterpret_cast<const uint4*>(base + ((uint64_t)at[j] << 4) + c * 16);
        }
    };
    // registers -> LDS, rows of a pitch
    auto store = [&](uint8_t* dst, int pitch) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        if (kEven || tid + j * kTileNT < kTileKeys * kPieces) {
          int r, c;
          piece(j, r, c);
          uint8_t* d = dst + r * pitch + c * (32 / EB);
          if constexpr (EB == 2) {
            *reinterpret_cast<uint4*>(d) = stage[j];
          } else {
            const uint2 w0 = e5m2x4_to_bf16(stage[j].x), w1 = e5m2x4_to_bf16(stage[j].y), w2 = e5m2x4_to_bf16(stage[j].z), w3 = e5m2x4_to_bf16(stage[j].w);
            *reinterpret_cast<uint4*>(d) = make_uint4(w0.x, w0.y, w1.x, w1.y);
            *reinterpret_cast<uint4*>(d + 16) = make_uint4(w2.x, w2.y, w3.x, w3.y);
          }
        }
    };
    // Values of keys without a row become zero, since a weight of zero does not make NaN harmless; whether any is infinite or NaN.
    auto clean = [&]() {
      uint32_t odd = 0;
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        if (kEven || tid + j * kTileNT < kTileKeys * kPieces) {
          int r, c;
          piece(j, r, c);
          if (!((have >> r) & 1)) stage[j] = make_uint4(0, 0, 0, 0);
          const uint32_t w[4] = {stage[j].x, stage[j].y, stage[j].z, stage[j].w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            odd |= EB == 2 ? not_finite(w[e]) : not_finite_e5m2(w[e]);
        }
      return odd != 0;
    };
    auto masked = [&](int t) { return t >= clear || have != ~0ull; };

    bool mask = false, odd = false;   // of the tile in use: not all seen by all; of its values some are infinite or NaN
    uint64_t have_now = 0;
    int page_next = 0;
    if (t0 < t1) {   // (so run.len > 0)
      int page = page_entry(a, table, t0 * kTileKeys + lane, run.len);
      kv = key_row(a, page, t0 * kTileKeys + lane, run.len);
      page_next = page_entry(a, table, (t0 + 1) * kTileKeys + lane, run.len);
      have_now = have = __ballot(kv.ok);
      locate();
      request(kbase, at_k);
      __syncthreads();   // (the buffers may still be read for the item before)
      store(lds, PK);
      request(vbase, at_v);
      mask = masked(t0);
      bool bad = false;
      if (mask) bad = clean();
      store(lds + kTileKeys * PK, PV);
      if (mask) odd = __syncthreads_or(bad); else __syncthreads();
    }
#pragma unroll 1
    for (int t = t0; t < t1; ++t) {
      uint8_t* buf = lds + ((t - t0) & 1) * TilePitch<D>::bytes;
      uint8_t* next = lds + (((t - t0) & 1) ^ 1) * TilePitch<D>::bytes;
      // The next tile, or behind the last one (t + 1 == t1) whatever follows, which nothing uses: no branch, so that the loads stay
      // in flight (where a branch joined them, the compiler's copies waited for them at once).
      kv = key_row(a, page_next, (t + 1) * kTileKeys + lane, run.len);
      page_next = page_entry(a, table, (t + 2) * kTileKeys + lane, run.len);
      have = __ballot(kv.ok);
      locate();
      request(kbase, at_k);
      f32x16 s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int j = 0; j < 16; ++j) s[kb][j] = 0.f;
      {
        // operands of two products per key block are read while the two before are multiplied
        const uint8_t* kp = buf + col * PK + half * 16;
        uint4 kf[2][4];
        auto read = [&](int i, uint4 (&f)[4]) {
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = *reinterpret_cast<const uint4*>(kp + (e & 1) * 32 * PK + (i + (e >> 1)) * 32);
        };
        read(0, kf[0]);
        __builtin_amdgcn_s_setprio(1);   // over the other workgroup's wave, which forms weights meanwhile (a prompt of 8K: 620 -> 607 us)
#pragma unroll
        for (int i = 0; i < QS; i += 2) {
          if (i + 2 < QS) read(i + 2, kf[(i / 2 + 1) % 2]);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[e & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[i / 2 % 2][e]), qf[i + (e >> 1)], s[e & 1], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      __builtin_amdgcn_s_setprio(0);
      // (FP8's conversions go behind the first weights: 341 us against 347 in four ragged chunks of up to 1.3K tokens; bf16, which has
      // nothing to convert, the other way round: 1052 us against 1064 in 2K tokens after 28K)
      if constexpr (EB == 2) {
        store(next, PK);
        request(vbase, at_v);
      }
      if (mask) {
        const int rel = limit - t * kTileKeys - 4 * half;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (kb * 32 + 8 * (j >> 2) + (j & 3) > rel) s[kb][j] = -INFINITY;
        if (have_now != ~0ull) {
          const uint64_t h = have_now >> (4 * half);
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (!((h >> (kb * 32 + 8 * (j >> 2) + (j & 3))) & 1)) s[kb][j] = -INFINITY;
        }
      }
      float top = s[0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int j = 0; j < 16; ++j) top = fmaxf(top, s[kb][j]);
      const uint8_t* vp = buf + kTileKeys * PK + (4 * half + ((lane & 15) >> 2)) * PV + (16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
      uint4 vf[2][DB];
      auto read_values = [&](int u, uint4 (&f)[DB]) {   // 16 keys
#pragma unroll
        for (int i = 0; i < DB; ++i) {
          const uint2 x = read_tr(vp + u * 16 * PV + i * 64), y = read_tr(vp + (u * 16 + 8) * PV + i * 64);
          f[i] = make_uint4(x.x, x.y, y.x, y.y);
        }
      };
      read_values(0, vf[0]);   // arrives while the weights are formed
      top = max_halves(top) * a.scale_log2;
      if (__any(top > m)) {
        const float next_m = top > m ? top + kHeadroom : m, f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - next_m);
        m = next_m;
        l *= f;
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) o[i][j] *= f;
      }
      const float mm = m == -INFINITY ? 0.f : m;
      uint32_t pw[2][8];
      float sum = 0.f;
      auto weigh = [&](int kb, int c) {   // two keys
        const float p0 = __builtin_amdgcn_exp2f(s[kb][2 * c] * a.scale_log2 - mm), p1 = __builtin_amdgcn_exp2f(s[kb][2 * c + 1] * a.scale_log2 - mm);
        sum += p0 + p1;
        pw[kb][c] = pack_bf16(p0, p1);
      };
#pragma unroll
      for (int c = 0; c < 8; ++c) weigh(0, c);
      if constexpr (EB == 1) {
        store(next, PK);
        request(vbase, at_v);
      }
      uint8_t* vt = buf + kTileKeys * PK;
      if (odd) {
        // infinities and NaN go to the rows that see their keys, and are zero for the product
        for (int k = 0; k < kTileKeys; ++k) {
          if (t * kTileKeys + k > limit || !((have_now >> k) & 1)) continue;
#pragma unroll
          for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
              const uint2 w = *reinterpret_cast<const uint2*>(vt + k * PV + half * 8 + i * 64 + j * 4);
              const float e[4] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
#pragma unroll
              for (int n = 0; n < 4; ++n)
                if ((__float_as_uint(e[n]) & 0x7f800000u) == 0x7f800000u) o[i][j + n] += e[n];
            }
        }
        __syncthreads();
        for (int p = tid; p < kTileKeys * D / 4; p += kTileNT) {
          uint2* w = reinterpret_cast<uint2*>(vt + p / (D / 4) * PV + p % (D / 4) * 8);
          *w = make_uint2(only_finite(w->x), only_finite(w->y));
        }
        __syncthreads();
      }
      {
        __builtin_amdgcn_s_setprio(1);
        if (odd) read_values(0, vf[0]);   // (they were read before they were cleaned)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (u < 3) read_values(u + 1, vf[(u + 1) % 2]);
          __builtin_amdgcn_sched_barrier(0);
          const uint32_t* p = pw[u / 2] + 4 * (u % 2);
          const bf16x8 pf = __builtin_bit_cast(bf16x8, make_uint4(p[0], p[1], p[2], p[3]));
#pragma unroll
          for (int i = 0; i < DB; ++i) {
            o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[u % 2][i]), pf, o[i], 0, 0, 0);
            // the weights of the second 32 keys beside the products of the first
            if (u < 2) {
#pragma unroll
              for (int c = 8 * (u * DB + i) / (2 * DB); c < 8 * (u * DB + i + 1) / (2 * DB); ++c) {
                weigh(1, c);
                asm volatile("" : "+v"(pw[1][c]), "+v"(sum));   // (keeps them here)
              }
              __builtin_amdgcn_sched_barrier(0);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        l += sum;
      }
      __builtin_amdgcn_s_setprio(0);
      mask = t + 1 < t1 && masked(t + 1);
      bool bad = false;
      if (mask) bad = clean();
      store(next + kTileKeys * PK, PV);
      have_now = have;
      if (mask) odd = __syncthreads_or(bad); else { odd = false; __syncthreads(); }
    }

    l = sum_halves(l);
    if (slot < 0) {
      if (!row_ok) return;
      // (no weight at all: zero, whatever infinite values made of o)
      if (l == 0.f) {
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
      }
      const float f = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
      uint8_t* dst = a.out.p + qrow * a.out.tok + (head * G + g) * a.out.head + half * 8;
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int j = 0; j < 16; j += 4)
          *reinterpret_cast<uint2*>(dst + i * 64 + j * 4) = make_uint2(pack_bf16(o[i][j] * f, o[i][j + 1] * f), pack_bf16(o[i][j + 2] * f, o[i][j + 3] * f));
      if (a.lse && half == 0) a.lse[qrow * a.hq + head * G + g] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    } else {
      float* dst = a.part_acc + ((int64_t)slot * kTileRows + row) * D + half * 4;
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int j = 0; j < 16; j += 4)
          *reinterpret_cast<float4*>(dst + i * 32 + j * 2) = make_float4(o[i][j], o[i][j + 1], o[i][j + 2], o[i][j + 3]);
      if (half == 0) a.part_ml[(int64_t)slot * kTileRows + row] = make_float2(m, l);
    }
  });
}

// ---- 16 or 32 rows: the four waves of a workgroup take the keys in turn, 32 at a time ------------------------------------------
// Bound by reading K and V.  K goes from memory straight into operand registers: of v_mfma_f32_16x16x32_bf16's left operand a lane
// holds eight elements of one key, which four lanes of a row request as 64 neighbouring bytes; the order of the elements inside
// the product is free as long as Q's is the same.  V goes through a piece of LDS of the wave's own, so nothing waits for
// another wave before the end.  The next 32 keys are requested as soon as the registers are free.  The softmax weights enter as two bf16 terms:
// the matrix pipe has the time (32 keys of two waves take a SIMD's 0.3 us, and their bytes 6 us at 5.2 TB/s).
// 16 sequences of 32K keys, a token each, 32/8 heads of 128: 237 us + 6 for the join, 5.5 TB/s (a large copy: 5.0 to 5.4, read and
// written); one of 1M keys, 32/2 heads: 191 us + 13; one of 4K keys: 14 us + 5, a chain of latencies (the share 3, page table and Q 2, keys 3,
// the merge 2 us).  For 17 to 32 rows the kernel for 128 would take 49 us against 37 (24 chats' drafts, FP8, 14/2 heads of 64), 180
// against 119 (16 sequences of 16K FP8 keys, 8 tokens each, 32/8 heads of 128), 398 against 351 (bf16, heads of 96, 20 rows), but 219
// against 221 and 34 against 38 with bf16 heads of 128, whose registers do not hold two blocks of rows: the price of the second term there.
constexpr int kRowsKeys = 32, kRowsNT = 256;
template <int D>
struct RowsPitch {
  static constexpr int v = 2 * D + 32;   // 32 bytes of eight rows on all 64 banks
};

template <int D, int EB, int NB>
__global__ __launch_bounds__(kRowsNT, 2) void paged_attn_rows_kernel(PagedAttnArgs a) {
  constexpr int BR = 16 * NB, NW = kRowsNT / kWave, DB = D / 16;
  constexpr int kSteps = D / 32;                          // products of 32 elements
  constexpr int kPieces = D * EB / 16, kLoads = kRowsKeys * kPieces / kWave;   // V: 16-byte pieces of a row; per lane
  constexpr int PV = RowsPitch<D>::v;
  constexpr int kVBytes = NW * kRowsKeys * PV, kMergeBytes = NW * BR * (D * 4 + 8);
  __shared__ __attribute__((aligned(16))) uint8_t lds[kVBytes > kMergeBytes ? kVBytes : kMergeBytes];
  // Q of two row blocks of long heads waits in LDS, in operand order: in registers, heads of 128 spilled 54 of theirs (259 us
  // against 234, 16 sequences of 16K keys, 8 tokens each, 32 heads on 8), while heads of 64 have room for it (41.4 us against 42.4).
  // bf16 heads of 128 still spill 26, to scratch and back outside the loop over keys.
  constexpr bool kQInLds = NB == 2 && D > 64;
  __shared__ uint4 q_lds[kQInLds ? NB * kSteps : 1][kWave];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, col = lane & 15, quarter = lane >> 4;

  for_items<kRowsKeys * NW>(a, [&](const SeqRun& run, int seq, int head, int blk, int t0, int t1, int slot) {
    const int G = a.G;
    // Element order of step s: bf16, 32 s + 8 quarter + 0..7; FP8, whose 16-byte pieces hold 16 elements, steps 2 p and 2 p + 1
    // take the halves of piece 64 p + 16 quarter (a last odd step 8-byte pieces).
    auto elem = [&](int s) {
      if (EB == 2 || (s == kSteps - 1 && kSteps % 2)) return 32 * s + 8 * quarter;
      return 64 * (s / 2) + 16 * quarter + 8 * (s % 2);
    };
    const int32_t* table = a.pt.table + seq * a.pt.stride;
    const int seen = a.causal ? min(max(run.first + min(run.n, (blk + 1) * a.tb), 0), run.len) : run.len;
    const int s0 = t0 * NW + wave, last = min(t1 * NW, (seen + kRowsKeys - 1) / kRowsKeys);   // in tiles of 32 keys
    auto lookup = [&](int t) { return page_entry(a, table, t * kRowsKeys + (lane & 31), run.len); };
    const int page0 = lookup(s0);
    int page = lookup(s0 + NW);   // of the tile after next
    bf16x8 qf[kQInLds ? 1 : NB][kSteps];
    int limit[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int row = 16 * n + col, tl = row / G, g = row - tl * G, tok = blk * a.tb + tl;
      const bool ok = tl < a.tb && tok < run.n;
      limit[n] = ok ? (a.causal ? run.first + tok : run.len - 1) : -1;
      // (rows that are none take row 0 of q: what they make is not written)
      const uint8_t* qp = a.q.p + (ok ? (run.start + tok) * a.q.tok + (head * G + g) * a.q.head : 0);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        if constexpr (kQInLds) {
          if ((n * kSteps + s) % NW == wave) q_lds[n * kSteps + s][lane] = *reinterpret_cast<const uint4*>(qp + elem(s) * 2);
        } else {
          qf[n][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(qp + elem(s) * 2));
        }
      }
    }
    if constexpr (kQInLds) __syncthreads();
    const int first = a.causal ? run.first + blk * a.tb : run.len - 1, clear = max(first + 1, 0) / kRowsKeys;
    f32x4 o[NB][DB];
    float m[NB], l[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      m[n] = -INFINITY;
      l[n] = 0.f;
#pragma unroll
      for (int i = 0; i < DB; ++i) o[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const uint8_t* kbase = a.kp.p + head * a.kp.head;
    const uint8_t* vbase = a.vp.p + head * a.vp.head;
    uint8_t* mine = lds + wave * kRowsKeys * PV;

    constexpr int kW = (D * EB / 4 + 15) / 16;   // 16-byte pieces of K per lane and 16 keys (the last may be half used)
    uint4 kr[2][kW], vr[kLoads];
    KeyRow kv;             // of key (lane % 32) of the tile whose rows are requested next
    uint32_t have = 0;
    auto request_k = [&]() {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint8_t* p = kbase + row_offset(kv.k, kb * 16 + col);
#pragma unroll
        for (int s = 0; s < kW; ++s) {
          if constexpr (EB == 1 && D % 64 != 0) {
            if (s == kW - 1) {
              const uint2 w = *reinterpret_cast<const uint2*>(p + s * 64 + 8 * quarter);
              kr[kb][s] = make_uint4(w.x, w.y, 0, 0);
              continue;
            }
          }
          kr[kb][s] = *reinterpret_cast<const uint4*>(p + s * 64 + 16 * quarter);
        }
      }
    };
    auto request_v = [&]() {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int p = lane + j * kWave, r = p / kPieces, c = p - r * kPieces;
        vr[j] = *reinterpret_cast<const uint4*>(vbase + row_offset(kv.v, r) + c * 16);
      }
    };
    if (s0 < last) {
      kv = key_row(a, page0, s0 * kRowsKeys + (lane & 31), run.len);
      have = (uint32_t)__ballot(kv.ok);
      request_k();
      request_v();
    }
    for (int t = s0; t < last; t += NW) {
      const uint32_t h = have;
      f32x4 s[NB][2];
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) s[n][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
      int at = lane;
      if constexpr (kQInLds) asm volatile("" : "+v"(at));   // (read in every turn)
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        bf16x8 qs[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          if constexpr (kQInLds) qs[n] = __builtin_bit_cast(bf16x8, q_lds[n * kSteps + i][at]);
          else qs[n] = qf[n][i];
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          bf16x8 kf;
          if constexpr (EB == 2) {
            kf = __builtin_bit_cast(bf16x8, kr[kb][i]);
          } else {
            const uint4 w = kr[kb][i / 2];
            const uint2 x = e5m2x4_to_bf16(i % 2 ? w.z : w.x), y = e5m2x4_to_bf16(i % 2 ? w.w : w.y);
            kf = __builtin_bit_cast(bf16x8, make_uint4(x.x, x.y, y.x, y.y));
          }
#pragma unroll
          for (int n = 0; n < NB; ++n) s[n][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qs[n], s[n][kb], 0, 0, 0);
        }
      }
      // (behind the wave's last keys whatever follows, which nothing uses)
      kv = key_row(a, page, (t + NW) * kRowsKeys + (lane & 31), run.len);
      have = (uint32_t)__ballot(kv.ok);
      request_k();
      const bool mask = t >= clear || h != ~0u;
      bool odd = false;   // infinities or NaN among the values of a tile that not all rows see whole
      if (mask) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          if (!((h >> ((lane + j * kWave) / kPieces)) & 1)) vr[j] = make_uint4(0, 0, 0, 0);
          if constexpr (EB == 2) odd |= not_finite(vr[j].x) || not_finite(vr[j].y) || not_finite(vr[j].z) || not_finite(vr[j].w);
          else odd |= not_finite_e5m2(vr[j].x) || not_finite_e5m2(vr[j].y) || not_finite_e5m2(vr[j].z) || not_finite_e5m2(vr[j].w);
        }
        odd = __any(odd);
      }
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int p = lane + j * kWave, r = p / kPieces, c = p - r * kPieces;
        const uint4 v = vr[j];
        if constexpr (EB == 2) {
          *reinterpret_cast<uint4*>(mine + r * PV + c * 16) = v;
        } else {
          const uint2 v0 = e5m2x4_to_bf16(v.x), v1 = e5m2x4_to_bf16(v.y), v2 = e5m2x4_to_bf16(v.z), v3 = e5m2x4_to_bf16(v.w);
          *reinterpret_cast<uint4*>(mine + r * PV + c * 32) = make_uint4(v0.x, v0.y, v1.x, v1.y);
          *reinterpret_cast<uint4*>(mine + r * PV + c * 32 + 16) = make_uint4(v2.x, v2.y, v3.x, v3.y);
        }
      }
      request_v();
      page = lookup(t + 2 * NW);
      uint32_t ph[NB][4], pl[NB][4];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = s[n][j >> 2][j & 3] * a.scale_log2;
          const int k = 16 * (j >> 2) + 4 * quarter + (j & 3);
          if (mask && (t * kRowsKeys + k > limit[n] || !((h >> k) & 1))) x[j] = -INFINITY;
        }
        float top = x[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
        top = max_quarters(top);
        if (__any(top > m[n])) {
          const float next = top > m[n] ? top + kHeadroom : m[n], f = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[n] - next);
          m[n] = next;
          l[n] *= f;
#pragma unroll
          for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[n][i][j] *= f;
        }
        const float mm = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const float p0 = __builtin_amdgcn_exp2f(x[j] - mm), p1 = __builtin_amdgcn_exp2f(x[j + 1] - mm);
          l[n] += p0 + p1;
          // the upper halves, and what they leave out (exact), rounded.  Taken from the number below, so that no weight but zero leaves
          // nothing out: zero times an infinite value would be NaN.
          const uint32_t u0 = __builtin_elementwise_sub_sat(__float_as_uint(p0), 1u), u1 = __builtin_elementwise_sub_sat(__float_as_uint(p1), 1u);
          ph[n][j >> 1] = upper_halves(u0, u1);
          pl[n][j >> 1] = pack_bf16(p0 - __uint_as_float(u0 & 0xffff0000u), p1 - __uint_as_float(u1 & 0xffff0000u));
        }
      }
      // V in the wave's LDS: written above by other lanes
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (odd) {   // they go to the rows that see their keys, and are zero for the product (a weight of zero does not make them harmless)
        for (int k = 0; k < kRowsKeys; ++k) {
          if (!((h >> k) & 1)) continue;
#pragma unroll
          for (int i = 0; i < DB; ++i) {
            const uint2 w = *reinterpret_cast<const uint2*>(mine + k * PV + i * 32 + quarter * 8);
            const float e[4] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int n = 0; n < NB; ++n)
                if (t * kRowsKeys + k <= limit[n] && (__float_as_uint(e[j]) & 0x7f800000u) == 0x7f800000u) o[n][i][j] += e[j];
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        for (int j = lane; j < kRowsKeys * D / 4; j += kWave) {
          uint2* w = reinterpret_cast<uint2*>(mine + j / (D / 4) * PV + j % (D / 4) * 8);
          *w = make_uint2(only_finite(w->x), only_finite(w->y));
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
      const uint8_t* vp = mine + (4 * quarter + (col >> 2)) * PV + (col & 3) * 8;
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        const uint2 x = read_tr(vp + i * 32), y = read_tr(vp + 16 * PV + i * 32);
        const bf16x8 vf = __builtin_bit_cast(bf16x8, make_uint4(x.x, x.y, y.x, y.y));
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, make_uint4(ph[n][0], ph[n][1], ph[n][2], ph[n][3])),
                                                            o[n][i], 0, 0, 0);
          o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, make_uint4(pl[n][0], pl[n][1], pl[n][2], pl[n][3])),
                                                            o[n][i], 0, 0, 0);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }

    // the four waves' states
    __syncthreads();   // (V's pieces of LDS are free)
    float* macc = reinterpret_cast<float*>(lds);
    float2* mml = reinterpret_cast<float2*>(lds + NW * BR * D * 4);
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      l[n] = sum_quarters(l[n]);
#pragma unroll
      for (int i = 0; i < DB; ++i)
        *reinterpret_cast<float4*>(macc + (wave * BR + 16 * n + col) * D + 16 * i + 4 * quarter) = make_float4(o[n][i][0], o[n][i][1], o[n][i][2], o[n][i][3]);
      if (quarter == 0) mml[wave * BR + 16 * n + col] = make_float2(m[n], l[n]);
    }
    __syncthreads();
    for (int p = tid; p < BR * D / 4; p += kRowsNT) {
      const int row = p / (D / 4), c = (p - row * (D / 4)) * 4;
      const int tl = row / G, g = row - tl * G, tok = blk * a.tb + tl;
      if (tl >= a.tb || tok >= run.n) continue;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < NW; ++w) top = fmaxf(top, mml[w * BR + row].x);
      float sum = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float2 ml = mml[w * BR + row];
        if (ml.x == -INFINITY && ml.y == 0.f) continue;   // (no weight at all)
        const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
        const float4 v = *reinterpret_cast<const float4*>(macc + (w * BR + row) * D + c);
        sum += ml.y * f;
        x[0] += v.x * f; x[1] += v.y * f; x[2] += v.z * f; x[3] += v.w * f;
      }
      if (slot < 0) {
        const float f = sum > 0.f ? 1.f / sum : (sum == sum ? 0.f : sum);
        const int64_t qrow = run.start + tok;
        *reinterpret_cast<uint2*>(a.out.p + qrow * a.out.tok + (head * G + g) * a.out.head + c * 2) =
            make_uint2(pack_bf16(x[0] * f, x[1] * f), pack_bf16(x[2] * f, x[3] * f));
        if (a.lse && c == 0) a.lse[qrow * a.hq + head * G + g] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
      } else {
        *reinterpret_cast<float4*>(a.part_acc + ((int64_t)slot * BR + row) * D + c) = make_float4(x[0], x[1], x[2], x[3]);
        if (c == 0) a.part_ml[(int64_t)slot * BR + row] = make_float2(top, sum);
      }
    }
    __syncthreads();
  });
}

template <int D, int EB>
inline hipError_t launch_paged_attn_d(const PagedAttnArgs& a, int block_rows, hipStream_t st) {
  if (block_rows == 16) hipLaunchKernelGGL((paged_attn_rows_kernel<D, EB, 1>), dim3(a.n_wg), dim3(kRowsNT), 0, st, a);
  else if (block_rows == 32) hipLaunchKernelGGL((paged_attn_rows_kernel<D, EB, 2>), dim3(a.n_wg), dim3(kRowsNT), 0, st, a);
  else hipLaunchKernelGGL((paged_attn_tiles_kernel<D, EB>), dim3(a.n_wg), dim3(kTileNT), 0, st, a);
  return hipGetLastError();
}
template <int EB>
inline hipError_t launch_paged_attn_eb(const PagedAttnArgs& a, int block_rows, hipStream_t st) {
  return a.d == 64 ? launch_paged_attn_d<64, EB>(a, block_rows, st)
         : a.d == 96 ? launch_paged_attn_d<96, EB>(a, block_rows, st) : launch_paged_attn_d<128, EB>(a, block_rows, st);
}
hipError_t launch_paged_attn_fp8(const PagedAttnArgs& a, int block_rows, hipStream_t st);   // kernels_paged_attn_fp8.hip

}  // namespace skv
