// The n best continuations of every group of beams, by summed log-probability:
//   score = s + c x_v - log sum_w exp(c x_w),   rank = score / length^a.
// Two launches.  The first reads the logits once: a wave takes a part of a row, sums its exponentials (fp64) and keeps the largest logit of
// every block of 256 tokens, nothing else.  The second has a workgroup per group and a wave per row: the
// n best tokens of a row lie in the n blocks with the largest maxima (whatever lies in another block has n better ones, one in each of
// those), so it finds these, reads them again, and keeps their n best; then the first wave ranks what all rows offer.
//
// Ranks of different rows meet in the choice, so the sums are fp64: exp as 2^t = 2^round(t) 2^f, f in [-1/2, 1/2], with 2^f the Chebyshev
// interpolation of degree 8 (off by 1.1e-12 at most), 2^round(t) added to the exponent's bits.  Lanes take the same tokens in the same
// order in every row, whatever its address is, so rows of equal logits get equal sums.
#include <algorithm>

#include "../../include/shadowkv.h"
#include "common.hpp"
#include "kernels.hpp"

namespace skv {
namespace {

constexpr int kElems = 16;                      // consecutive logits of a lane
constexpr int kTogether = 4;                    // of which so many exponentials are formed in step
constexpr int kChunk = kWave * kElems;
constexpr int kBlock = 16 * kElems;             // tokens of a block: a row of 16 lanes
constexpr double kLog2e = 1.4426950408889634074;

// 2^f for f in [-1/2, 1/2], times 2^n
constexpr double kExp2[9] = {1.3255179556479267e-06, 1.5310080611926545e-05, 0.00015403456082633648, 0.0013333450563173552, 0.009618129159053034,
                             0.055504109412108156, 0.24022650695814518, 0.6931471805459332, 1.0000000000000004};
__device__ __forceinline__ double exp2_frac(double f, int n) {
  double p = fma(kExp2[0], f, kExp2[1]);
#pragma unroll
  for (int k = 2; k < 9; ++k) p = fma(p, f, kExp2[k]);
  return __hiloint2double(__double2hiint(p) + (n << 20), __double2loint(p));
}
constexpr double kRound = 6755399441055744.0;   // 1.5 2^52: the low bits of t + kRound are round(t)
// 2^t, t held to at least -1000
__device__ __forceinline__ double exp2_f64(double t) {
  t = fmax(t, -1000.0);
  const double a = t + kRound;
  return exp2_frac(t - (a - kRound), __double2loint(a));
}
// sum + 2^(x_0 c) + ... of N logits, |x c| < 1000 (the products are never rounded), in step with each other
template <int N>
__device__ __forceinline__ double add_exp2_of_products(double sum, const float* x, double c) {
  double f[N], p[N];
  int n[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const double a = fma((double)x[i], c, kRound);
    n[i] = __double2loint(a);
    f[i] = fma((double)x[i], c, -(a - kRound));
  }
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = fma(kExp2[0], f[i], kExp2[1]);
#pragma unroll
  for (int k = 2; k < 9; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = fma(p[i], f[i], kExp2[k]);
#pragma unroll
  for (int i = 0; i < N; ++i) sum += __hiloint2double(__double2hiint(p[i]) + (n[i] << 20), __double2loint(p[i]));
  return sum;
}

__device__ __forceinline__ uint32_t f32_key(float x) {   // larger value <=> larger key, never 0 but for NaN
  x += 0.f;                                              // (-0 is +0)
  const uint32_t u = __float_as_uint(x);
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
constexpr uint32_t kLowestKey = 0x007fffffu;             // of minus infinity
__device__ __forceinline__ float key_f32(uint32_t k) { return __uint_as_float((k >> 31) ? (k & 0x7fffffffu) : ~k); }
__device__ __forceinline__ float wave_max_f32(float v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor(v, m, kWave));
  return v;
}

template <int DT>
struct Logit;
template <>
struct Logit<SHADOWKV_LOGITS_BF16> {
  static constexpr int bytes = 2;
  static __device__ __forceinline__ float one(const uint8_t* p) { return bf16_to_f32(*reinterpret_cast<const uint16_t*>(p)); }
  template <int N>
  static __device__ __forceinline__ void unpack(const uint32_t* w, float* x) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
  }
};
template <>
struct Logit<SHADOWKV_LOGITS_FP16> {
  static constexpr int bytes = 2;
  static __device__ __forceinline__ float one(const uint8_t* p) { return (float)*reinterpret_cast<const _Float16*>(p); }
  template <int N>
  static __device__ __forceinline__ void unpack(const uint32_t* w, float* x) {
    typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const half2_t h = __builtin_bit_cast(half2_t, w[i]);
      x[2 * i] = (float)h[0]; x[2 * i + 1] = (float)h[1];
    }
  }
};
template <>
struct Logit<SHADOWKV_LOGITS_FP32> {
  static constexpr int bytes = 4;
  static __device__ __forceinline__ float one(const uint8_t* p) { return *reinterpret_cast<const float*>(p); }
  template <int N>
  static __device__ __forceinline__ void unpack(const uint32_t* w, float* x) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __uint_as_float(w[i]);
  }
};

// whether a row takes part at all
__device__ __forceinline__ bool row_lives(float score) { return fabsf(score) < INFINITY; }

// Logits x with -800 < x c < 900 (c in units of log 2) are summed as they are, 2^(x c); a chunk with others (masks, infinities, logits far apart)
// is summed relative to a logit that it or an earlier one holds, in a sum of its own.
struct BeamScale {
  double c;
  float low, high;                              // x between them
  float absent;                                 // adds 2^-900: what stands behind the last token
};
__device__ __forceinline__ BeamScale beam_scale(double scale) {
  BeamScale s;
  s.c = scale * kLog2e;
  const bool fits = s.c > 0x1p-60 && s.c < 0x1p60;   // (else the borders leave fp32's range)
  s.low = fits ? (float)(-800.0 / s.c) : INFINITY;
  s.high = fits ? (float)(900.0 / s.c) : -INFINITY;
  s.absent = fits ? (float)(-900.0 / s.c) : -INFINITY;
  return s;
}

template <int DT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(6, 6))) void beam_parts_kernel(BeamArgs a) {
  constexpr int EB = Logit<DT>::bytes, WORDS = kElems * EB / 4;
  const int lane = threadIdx.x & (kWave - 1);
  const uint32_t w = blockIdx.x * 4 + (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (w >= (uint32_t)(a.groups * a.beams) * (uint32_t)a.n_parts) return;
  const int row = (int)(w / (uint32_t)a.n_parts), part = (int)(w % (uint32_t)a.n_parts);
  if (!row_lives(a.scores[row]) || (a.finished && a.finished[row])) return;   // (the second launch asks the same)
  const uint8_t* p = a.logits + (row / a.beams) * a.group_stride + (row % a.beams) * a.beam_stride;
  const int t0 = part * a.part_len, t1 = min(a.vocab, t0 + a.part_len);
  uint32_t* peak = a.peaks + (int64_t)row * a.n_blocks + t0 / kBlock;
  const BeamScale sc = beam_scale(a.scale);
  const float reach = (float)fmin(500.0 / sc.c, 1e38);
  uint32_t raw[WORDS];
  // rows of an odd vocabulary begin at any element; a lane that the end cuts off reads the last kElems tokens
  auto load = [&](int base) {
    const int at = min(base + lane * kElems, t1 - kElems);
    if (a.vocab >= kElems) {
      __builtin_memcpy(raw, p + (int64_t)at * EB, kElems * EB);
    } else {
      uint16_t* half = reinterpret_cast<uint16_t*>(raw);
      for (int e = 0; e < kElems; ++e) {        // token e - (kElems - vocab), as if there were more before it
        const int64_t t = max(e - (kElems - a.vocab), 0);
        if constexpr (EB == 4) raw[e] = *reinterpret_cast<const uint32_t*>(p + t * EB);
        else half[e] = *reinterpret_cast<const uint16_t*>(p + t * EB);
      }
    }
  };
  struct Sums {
    double plain, far;
    float ref;
    bool bad;
  };
  auto chunk = [&](auto whole, int base, Sums u) -> Sums {   // (by value: references end up in memory)
    constexpr bool kWhole = decltype(whole)::value;
    float x[kElems];
    Logit<DT>::template unpack<kElems>(raw, x);
    if (base + kChunk < t1) load(base + kChunk);
    const int gone = min(base + (lane + 1) * kElems - t1, kElems);   // of a cut lane's logits the first so many are not its own
    if constexpr (!kWhole) {
#pragma unroll
      for (int e = 0; e < kElems; ++e) x[e] = gone == kElems ? 0.f : e < gone ? x[kElems - 1] : x[e];
    }
    float most = x[0], least = x[0];
#pragma unroll
    for (int e = 1; e < kElems; ++e) {
      most = __builtin_elementwise_maximum(most, x[e]);              // (NaN if one is)
      least = __builtin_elementwise_minimum(least, x[e]);
    }
    u.bad |= !(most < INFINITY);
    const bool plainly = __ballot(!(least > sc.low && most < sc.high)) == 0;
    if constexpr (!kWhole) {
      if (gone == kElems) most = -INFINITY;
#pragma unroll
      for (int e = 0; e < kElems; ++e) x[e] = e < gone ? (plainly ? sc.absent : -INFINITY) : x[e];
    }
    if (__builtin_expect(plainly, 1)) {
#pragma unroll
      for (int e = 0; e < kElems; e += kTogether) u.plain = add_exp2_of_products<kTogether>(u.plain, x + e, sc.c);
    } else {
      // the reference moves up only where 2^t might leave fp64's range
      if (__ballot(most > u.ref + reach)) {
        const float to = wave_max_f32(most);
        u.far *= exp2_f64(((double)u.ref - (double)to) * sc.c);
        u.ref = to;
      }
      if (u.ref > -INFINITY) {
#pragma unroll
        for (int e = 0; e < kElems; ++e) u.far += exp2_f64(((double)x[e] - (double)u.ref) * sc.c);
      }
    }
    uint32_t m = f32_key(most);                 // lane 15 of 16 ends with the largest of them
    m = op_max(m, dpp_u32<0x111>(0u, m));
    m = op_max(m, dpp_u32<0x112>(0u, m));
    m = op_max(m, dpp_u32<0x114>(0u, m));
    m = op_max(m, dpp_u32<0x118>(0u, m));
    const int block = (base - t0) / kBlock + lane / 16;
    if (lane % 16 == 15 && (kWhole || block * kBlock < t1 - t0)) peak[block] = m;
    return u;
  };
  load(t0);
  Sums u{0.0, 0.0, -INFINITY, false};
  int base = t0;
  for (; base + kChunk <= t1; base += kChunk) u = chunk(std::true_type(), base, u);
  if (base < t1) u = chunk(std::false_type(), base, u);
  u.far = wave_sum_f64_dpp(u.far);
  u.plain = wave_sum_f64_dpp(u.plain);
  const bool bad = __ballot(u.bad) != 0;
  if (lane == 0) a.parts[w] = BeamPart{u.plain, u.far, u.ref, bad};
}

// ---- the n largest of many keys, by one wave ------------------------------------------------------------------------------
// What reaches a bound that n keys reach, and few others do, is put into LDS in order of items and sorted by counting, for each, what is
// larger (the earlier of equals first).
constexpr int kSortRoom = 256;
struct SortRoom {
  uint64_t key[kSortRoom];
  uint32_t item[kSortRoom];
};
// between writes and reads of LDS by different lanes of a wave
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// the n-th largest of the lanes' keys (1 if that is 0, no key)
__device__ __forceinline__ uint64_t lane_bound(uint64_t mine, int n, SortRoom& room, int lane) {
  room.key[lane] = mine;
  wave_sync();
  int larger = 0;
#pragma unroll 4
  for (int j = 0; j < kWave; ++j) { const uint64_t k = room.key[j]; larger += k > mine || (k == mine && j < lane); }
  const uint64_t bound = room.key[__ffsll((unsigned long long)__ballot(larger == n - 1)) - 1];
  wave_sync();
  return bound ? bound : 1;
}
// c: keys that have been taken, counted beyond the room as well
__device__ __forceinline__ void take(uint64_t k, uint32_t item, bool takes, SortRoom& room, int& c, int lane) {
  const uint64_t taken = __ballot(takes);
  const int at = c + __popcll(taken & ((1ull << lane) - 1));
  if (takes && at < kSortRoom) { room.key[at] = k; room.item[at] = item; }
  c += __popcll(taken);
}
// the n best of the c <= kSortRoom in the room, in order; returns how many there are
__device__ __forceinline__ int sort_room(SortRoom& room, int c, int n, uint64_t* keys, uint32_t* items, int lane) {
  wave_sync();
  for (int i = lane; i < c; i += kWave) {
    const uint64_t k = room.key[i];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < c; ++j) { const uint64_t o = room.key[j]; rank += o > k || (o == k && j < i); }
    if (rank < n) { keys[rank] = k; items[rank] = room.item[i]; }
  }
  wave_sync();
  return min(c, n);
}
// Where more than the room reach a bound (many equal keys, say): the largest bound that n keys reach, bit by bit, and of the
// keys that equal it the first.  key(i): of item i < n_items, 0: none.
template <int BITS, class Key>
__device__ __forceinline__ int take_exactly(Key key, int n_items, int n, uint64_t bound, SortRoom& room, int lane) {
  auto count = [&](uint64_t from) {
    int c = 0;
    for (int i0 = 0; i0 < n_items; i0 += kWave) c += __popcll(__ballot(i0 + lane < n_items && key(i0 + lane) >= from));
    return c;
  };
  for (int b = BITS - 1; b >= 0; --b) {
    const uint64_t up = (bound >> b | 1ull) << b;         // (bits above b are right; where bit b is set already this is not more)
    const int reach = up > bound ? count(up) : 0;
    if (reach >= n) bound = up;
    if (reach == n) break;
  }
  const int spare = n - count(bound + 1);
  int c = 0, equal = 0;
  wave_sync();
  for (int i0 = 0; i0 < n_items; i0 += kWave) {
    const uint64_t k = i0 + lane < n_items ? key(i0 + lane) : 0, same = __ballot(k == bound);
    take(k, (uint32_t)(i0 + lane), k > bound || (k == bound && equal + __popcll(same & ((1ull << lane) - 1)) < spare), room, c, lane);
    equal += __popcll(same);
  }
  return c;
}
// the n largest of key(i), i < n_items, equals in order of items
template <int BITS, class Key>
__device__ __forceinline__ int top_items(Key key, int n_items, int n, SortRoom& room, uint64_t* keys, uint32_t* items, int lane) {
  uint64_t mine = 0;
#pragma unroll 4
  for (int i = lane; i < n_items; i += kWave) { const uint64_t k = key(i); mine = k > mine ? k : mine; }
  const uint64_t bound = lane_bound(mine, n, room, lane);
  int c = 0;
#pragma unroll 4
  for (int i0 = 0; i0 < n_items; i0 += kWave) {
    const uint64_t k = i0 + lane < n_items ? key(i0 + lane) : 0;
    take(k, (uint32_t)(i0 + lane), k >= bound, room, c, lane);
  }
  if (__builtin_expect(c > kSortRoom, 0)) c = take_exactly<BITS>(key, n_items, n, bound, room, lane);
  return sort_room(room, c, n, keys, items, lane);
}

// What a row offers: candidate i is (logit, token); score = base + c (logit - ref).
struct RowOffer {
  double base;
  float ref;
  int count;
};
struct JoinWave {
  SortRoom room;
  uint64_t keys[64];
  uint32_t items[64];
};

template <int DT>
__global__ __launch_bounds__(1024) void beam_join_kernel(BeamArgs a) {
  constexpr int EB = Logit<DT>::bytes, kEach = 8, kLanes = kBlock / kEach, kAtOnce = kWave / kLanes;   // blocks are read two at a time
  extern __shared__ __align__(16) uint8_t lds[];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, waves = blockDim.x >> 6, group = blockIdx.x;
  JoinWave& mine = reinterpret_cast<JoinWave*>(lds)[wave];
  uint64_t* rank = reinterpret_cast<uint64_t*>(lds + waves * sizeof(JoinWave));    // [beams, n] keys of the ranks, 0: none
  uint2* cand = reinterpret_cast<uint2*>(rank + a.beams * a.n);                    // [beams, n]
  RowOffer* offer = reinterpret_cast<RowOffer*>(cand + a.beams * a.n);             // [beams]
  const double c_log2 = a.scale * kLog2e;
  for (int b = wave; b < a.beams; b += waves) {
    const int row = group * a.beams + b;
    const float s = a.scores[row];
    const bool done = a.finished && a.finished[row];
    double weight = 1.0;
    if (a.penalty != 0.0) weight = pow(fmax((double)a.lengths[row] + (done ? 0.0 : 1.0), 1.0), a.penalty);
    RowOffer o{(double)s, 0.f, 0};
    if (row_lives(s) && done) {
      o.count = 1;
      if (lane == 0) cand[b * a.n] = make_uint2(0u, (uint32_t)a.end_token);
    } else if (row_lives(s)) {
      const BeamPart* parts = a.parts + (int64_t)row * a.n_parts;
      bool bad = false, plain = false;
      float ref = -INFINITY;
      for (int i = lane; i < a.n_parts; i += kWave) {
        const BeamPart q = parts[i];
        bad |= q.bad != 0;
        plain |= q.plain > 0.0;
        ref = fmaxf(ref, q.ref);
      }
      ref = wave_max_f32(ref);
      if (__ballot(plain)) ref = fmaxf(ref, 0.f);       // (plain sums are relative to a logit of 0)
      if (!__ballot(bad) && ref > -INFINITY) {
        const uint32_t* peak = a.peaks + (int64_t)row * a.n_blocks;
        const int n_best = top_items<32>([&](int i) -> uint64_t { const uint32_t k = peak[i]; return k > kLowestKey ? k : 0u; }, a.n_blocks, a.n,
                                         mine.room, mine.keys, mine.items, lane);
        double sum = 0.0;
        for (int i = lane; i < a.n_parts; i += kWave) {
          const BeamPart q = parts[i];
          sum += q.plain * exp2_f64(-(double)ref * c_log2);
          if (q.ref > -INFINITY) sum += q.sum * exp2_f64(((double)q.ref - (double)ref) * c_log2);
        }
        sum = wave_sum_f64_dpp(sum);
        o.base = (double)s - log(sum);
        o.ref = ref;
        // tokens of those blocks that are not less than the n-th block's largest (of fewer blocks: than the n-th lane's)
        const uint8_t* p = a.logits + group * a.group_stride + b * a.beam_stride;
        auto key_of = [&](float x, int t) { return x > -INFINITY ? ((uint64_t)f32_key(x) << 32) | (uint32_t)~t : 0ull; };
        auto each_token = [&](auto f) {
          for (int i0 = 0; i0 < n_best; i0 += kAtOnce) {
            const int i = i0 + lane / kLanes;
            const int at = i < n_best ? (int)mine.items[i] * kBlock + lane % kLanes * kEach : a.vocab;
            float x[kEach];
            if (at + kEach <= a.vocab) {
              uint32_t raw[kEach * EB / 4];
              __builtin_memcpy(raw, p + (int64_t)at * EB, kEach * EB);
              Logit<DT>::template unpack<kEach>(raw, x);
            } else {
#pragma unroll
              for (int e = 0; e < kEach; ++e) x[e] = at + e < a.vocab ? Logit<DT>::one(p + (int64_t)(at + e) * EB) : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < kEach; ++e) f(key_of(x[e], at + e));
          }
        };
        uint64_t bound;
        if (n_best == a.n) {
          bound = mine.keys[n_best - 1] << 32;
        } else {
          uint64_t best = 0;
          each_token([&](uint64_t k) { best = k > best ? k : best; });
          bound = lane_bound(best, a.n, mine.room, lane);
        }
        int c = 0;
        each_token([&](uint64_t k) { if (__ballot(k >= bound)) take(k, 0, k >= bound, mine.room, c, lane); });
        if (__builtin_expect(c > kSortRoom, 0))
          c = take_exactly<64>([&](int i) -> uint64_t {
            const int t = (int)mine.items[i / kBlock] * kBlock + i % kBlock;
            return t < a.vocab ? key_of(Logit<DT>::one(p + (int64_t)t * EB), t) : 0;
          }, n_best * kBlock, a.n, bound, mine.room, lane);
        o.count = sort_room(mine.room, c, a.n, mine.keys, mine.items, lane);
        if (lane < o.count) cand[b * a.n + lane] = make_uint2(__float_as_uint(key_f32((uint32_t)(mine.keys[lane] >> 32))), ~(uint32_t)mine.keys[lane]);
      }
    }
    wave_sync();
    if (lane == 0) offer[b] = o;
    if (lane < a.n) rank[b * a.n + lane] = lane < o.count ? f64_key((o.base + a.scale * ((double)__uint_as_float(cand[b * a.n + lane].x) - (double)o.ref)) / weight) : 0;
  }
  __syncthreads();
  if (wave) return;
  // of all rows' candidates, in order of rows and places
  const int count = top_items<64>([&](int i) { return rank[i]; }, a.beams * a.n, a.n, mine.room, mine.keys, mine.items, lane);
  // (all that this group's rows held has been read before anything is written: the outputs may be the inputs)
  float out_s = -INFINITY;
  int parent = -1, token = -1, length = 0;
  bool ended = false;
  if (lane < count) {
    const int i = (int)mine.items[lane], b = i / a.n, row = group * a.beams + b;
    const bool was = a.finished && a.finished[row];
    out_s = (float)(offer[b].base + a.scale * ((double)__uint_as_float(cand[i].x) - (double)offer[b].ref));
    parent = row;
    token = (int)cand[i].y;
    ended = was || (a.end_token >= 0 && token == a.end_token);
    if (a.out_lengths) length = a.lengths[row] + (was ? 0 : 1);
  }
  __builtin_amdgcn_s_waitcnt(0);
  if (lane < a.n) {
    const int at = group * a.n + lane;
    a.out_scores[at] = out_s;
    a.out_parents[at] = parent;
    a.out_tokens[at] = token;
    if (a.out_finished) a.out_finished[at] = ended;
    if (a.out_lengths) a.out_lengths[at] = length;
  }
}

template <int DT>
hipError_t launch(const BeamArgs& a, hipStream_t st) {
  const int64_t waves = (int64_t)a.groups * a.beams * a.n_parts;
  beam_parts_kernel<DT><<<dim3((unsigned)((waves + 3) / 4)), 256, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int join = a.beams < 16 ? a.beams : 16;
  const size_t lds = join * sizeof(JoinWave) + (size_t)a.beams * (sizeof(RowOffer) + a.n * (sizeof(uint2) + sizeof(uint64_t)));
  if (lds > 65536) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(&beam_join_kernel<DT>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  beam_join_kernel<DT><<<dim3((unsigned)a.groups), join * kWave, lds, st>>>(a);
  return hipGetLastError();
}

}  // namespace

// Tokens of a part: as many chunks as leave 8192 waves, a third more than the chip holds.  (32 x 16 rows of 256K bf16, 8 / 16 / 32 chunks: 93.3 / 93.4 /
// 99.8 us.)
int beam_part_len(int64_t rows, int vocab) {
  const int64_t per = (rows * (((int64_t)vocab + kChunk - 1) / kChunk) + 8191) / 8192;
  return (int)std::min<int64_t>(std::max<int64_t>(per, 1), 1024) * kChunk;
}
int beam_blocks(int vocab) { return (int)(((int64_t)vocab + kBlock - 1) / kBlock); }

hipError_t launch_beam_select(const BeamArgs& a, hipStream_t st) {
  switch (a.dtype) {
    case SHADOWKV_LOGITS_BF16: return launch<SHADOWKV_LOGITS_BF16>(a, st);
    case SHADOWKV_LOGITS_FP16: return launch<SHADOWKV_LOGITS_FP16>(a, st);
    default: return launch<SHADOWKV_LOGITS_FP32>(a, st);
  }
}

}  // namespace skv
