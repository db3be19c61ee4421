// The n best continuations of every group of beams, by summed log-probability:
//   score = s + c x_v - log sum_w exp(c x_w),   rank = score / length^a.
// Three launches.  The first reads the logits once: a wave takes a part of a row, sums its exponentials (fp64) and keeps the largest logit of
// every block of 256 tokens, nothing else.  The second has a workgroup per row.  The n best tokens of a row lie in the n blocks with the
// largest maxima (whatever lies in another block has n better ones, one in each of those), so it finds these, reads them again, and keeps
// their n best.  The third, a workgroup per group, ranks what all rows offer; small calls do both in one launch.  (Done by the group's last
// workgroup of the second launch instead, behind a counter, the choice costs more than its launch: every workgroup has to write its L2 back
// first.  32 x 16 rows: 82 us for both.)
//
// Ranks of different rows meet in the choice, so the sums are fp64: exp as 2^t = 2^round(t) 2^f, f in [-1/2, 1/2], with 2^f the Chebyshev
// interpolation of degree 8 (off by 1.1e-12 at most), 2^round(t) added to the exponent's bits.  fp64 costs the vector pipes what fp32 costs.
// Lanes take the same tokens in the same order in every row, whatever its address is, so rows of equal logits get equal sums.
//
// 32 x 16 rows of 256K bf16, 32 places: 87 + 15 + 7.6 us.  The first launch issues 19.5 vector instructions a logit, 14 of them the
// exponential, 12 of all in fp64: four cycles each, they fill 84 % of the cycles (at 2.19 GHz; what the others wait for is not known).  16 x 4 rows
// of 128K, 8 places: 9.8 + 8.3 + 3.9, latencies for the most part.
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
template <int DT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(5, 5))) void beam_parts_kernel(BeamArgs a) {
  constexpr int EB = Logit<DT>::bytes, WORDS = kElems * EB / 4;
  const int lane = threadIdx.x & (kWave - 1);
  const uint32_t w = blockIdx.x * 4 + (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (w >= (uint32_t)(a.groups * a.beams) * (uint32_t)a.n_parts) return;
  const int row = (int)(w / (uint32_t)a.n_parts), part = (int)(w % (uint32_t)a.n_parts);
  const uint8_t* p = a.logits + (row / a.beams) * a.group_stride + (row % a.beams) * a.beam_stride;
  const int t0 = part * a.part_len, t1 = min(a.vocab, t0 + a.part_len);
  uint32_t* peak = a.peaks + (int64_t)row * a.n_blocks + t0 / kBlock;
  const BeamRange sc = a.range;
  uint32_t raw[WORDS];
  // rows of an odd vocabulary begin at any element; a lane that the end cuts off reads the last kElems tokens
  auto load = [&](int base) {
    const int at = min(base + lane * kElems, t1 - kElems);
    if (a.vocab >= kElems) {
      __builtin_memcpy(raw, p + (int64_t)at * EB, kElems * EB);
    } else {
      for (int e = 0; e < kElems; ++e) {        // token e - (kElems - vocab), as if there were more before it
        const uint8_t* q = p + (int64_t)max(e - (kElems - a.vocab), 0) * EB;   // (volatile: not to be merged with the reads above)
        if constexpr (EB == 4) {
          raw[e] = *reinterpret_cast<const volatile uint32_t*>(q);
        } else {
          const uint32_t h = *reinterpret_cast<const volatile uint16_t*>(q);
          raw[e / 2] = e & 1 ? (raw[e / 2] & 0xffffu) | (h << 16) : h;
        }
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
      if (__ballot(most > u.ref + sc.reach)) {
        const float to = wave_max_f32(most);
        u.far *= exp2(((double)u.ref - (double)to) * sc.c);   // (not held to 2^-1000: the sum may be up to 2^990)
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
  // (asked after the first chunk, so that its logits do not wait for the answer; the second launch asks the same)
  const float score = a.scores[row];
  const uint8_t done = a.finished ? a.finished[row] : 0;
  Sums u{0.0, 0.0, -INFINITY, false};
  int base = t0;
  for (; base + kChunk <= t1; base += kChunk) {
    u = chunk(std::true_type(), base, u);
    if (!row_lives(score) || done) return;
  }
  if (base < t1) u = chunk(std::false_type(), base, u);
  u.far = wave_sum_f64_dpp(u.far);
  u.plain = wave_sum_f64_dpp(u.plain);
  const bool bad = __ballot(u.bad) != 0;
  if (lane == 0) a.parts[w] = BeamPart{u.plain, u.far, u.ref, bad};
}

// ---- the n largest of many keys, by a team: a workgroup (T = 256) or a wave (T = 64) ----------------------------------------------
// What reaches a bound that n keys reach, and few others do, is put into LDS and sorted by counting, for each, what is larger.  Keys are 64 bits
// wide, 0 is none; they come with a number, and of equal keys the lower number goes first (kTies; other keys are never equal).
constexpr int kJoinThreads = 256;
template <int T>
struct __align__(16) JoinRoom {
  static constexpr int kRoom = T == kWave ? 128 : 256;
  uint64_t key[kRoom];
  uint32_t item[kRoom];
  uint32_t upper[T == kWave ? 4 : T];                     // (a wave reads its lanes)
  uint64_t best[64];                                      // what comes out, in order
  uint32_t best_item[64];
  uint32_t bound;
  int count, other;
};
template <int T>
__device__ __forceinline__ void team_sync() {
  if constexpr (T == kWave) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  } else {
    __syncthreads();
  }
}
template <int T>
__device__ __forceinline__ void take(uint64_t k, uint32_t item, bool takes, JoinRoom<T>& room, int lane) {
  const uint64_t taken = __ballot(takes);
  if (taken == 0) return;
  int at = 0;
  if (lane == 0) at = atomicAdd(&room.count, __popcll(taken));
  at = __builtin_amdgcn_readfirstlane(at) + __popcll(taken & ((1ull << lane) - 1));
  if (takes && at < JoinRoom<T>::kRoom) { room.key[at] = k; room.item[at] = item; }
}
// what is in the room, in order; all threads, after a barrier
template <bool kTies, int T>
__device__ __forceinline__ int sort_room(JoinRoom<T>& room, int n, int tid) {
  const int c = room.count;
  if (c + tid < ((c + 7) & ~7)) { room.key[c + tid] = 0; room.item[c + tid] = ~0u; }
  team_sync<T>();
  for (int i = tid; i < c; i += T) {
    const uint64_t k = room.key[i];
    const uint32_t item = room.item[i];
    int rank = 0;
    for (int j = 0; j < c; j += 8) {
      uint32_t items[8];
      if constexpr (kTies) {                              // (asked for with the keys, not where one is equal: each is to itself)
        *reinterpret_cast<uint4*>(items) = *reinterpret_cast<const uint4*>(&room.item[j]);
        *reinterpret_cast<uint4*>(items + 4) = *reinterpret_cast<const uint4*>(&room.item[j + 4]);
      }
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(&room.key[j + e]);
        rank += (int)(o.x > k) + (int)(o.y > k);
        if constexpr (kTies) rank += ((int)(o.x == k) & (int)(items[e] < item)) + ((int)(o.y == k) & (int)(items[e + 1] < item));
      }
    }
    if (rank < n) { room.best[rank] = k; room.best_item[rank] = item; }
  }
  team_sync<T>();
  return min(c, n);
}
// A key that n keys reach, from the upper halves (at least 1: a key of 0 is none): the n-th largest of the threads' own largest, or up to kFewPlaces
// places, which 64 values are enough for, of the largest of four threads.
constexpr int kFewPlaces = 16;
template <int T>
__device__ __forceinline__ uint64_t find_bound(uint64_t largest, int n, JoinRoom<T>& room, int tid) {
  const int lane = tid & (kWave - 1);
  uint32_t mine = (uint32_t)(largest >> 32), bound;
  int larger = 0;
  if (tid == 0) { room.count = 0; room.bound = ~0u; }
  if constexpr (T > kWave) room.upper[tid] = mine;
  team_sync<T>();
  if (T == kWave || n <= kFewPlaces) {                    // (every wave finds it by itself)
    if constexpr (T > kWave) {
      mine = room.upper[lane];
#pragma unroll
      for (int v = 1; v < T / kWave; ++v) mine = op_max(mine, room.upper[v * kWave + lane]);
    }
#pragma unroll 8
    for (int j = 0; j < kWave; ++j) larger += (uint32_t)__builtin_amdgcn_readlane((int)mine, j) > mine;
    bound = wave_min_u32(larger < n ? mine : ~0u);
  } else {
#pragma unroll 4
    for (int j = 0; j < T; j += 4) {
      const uint4 o = *reinterpret_cast<const uint4*>(&room.upper[j]);
      larger += o.x > mine;
      larger += o.y > mine;
      larger += o.z > mine;
      larger += o.w > mine;
    }
    const uint32_t least = wave_min_u32(larger < n ? mine : ~0u);
    if (lane == 0) atomicMin(&room.bound, least);
    team_sync<T>();
    bound = room.bound;
  }
  return bound ? (uint64_t)bound << 32 : 1;
}
// Where more reach the bound than there is room for (many equal ones, say): the largest bound that n keys reach, bit by bit, and of the keys that
// equal it the lowest numbers.  key(i, item): of entry i < n_entries, and its number.
template <bool kTies, int T, class Key>
__device__ __forceinline__ void take_exactly(Key key, int n_entries, int n, uint64_t bound, JoinRoom<T>& room, int tid) {
  const int lane = tid & (kWave - 1);
  // how many are above `from`, or equal it and have a number below `below`
  auto count = [&](uint64_t from, uint32_t below) {
    team_sync<T>();
    if (tid == 0) room.other = 0;
    team_sync<T>();
    int c = 0;
    for (int i = tid; i < n_entries; i += T) {
      uint32_t item = 0;
      const uint64_t k = key(i, item);
      c += k > from || (k == from && item < below);
    }
    if (c) atomicAdd(&room.other, c);
    team_sync<T>();
    return room.other;
  };
  for (int b = 63; b >= 0; --b) {
    const uint64_t up = (bound >> b | 1ull) << b;         // (bits above b are right; where bit b is set already this is not more)
    const int reach = up > bound ? count(up - 1, 0) : 0;
    if (reach >= n) bound = up;
    if (reach == n) break;
  }
  uint32_t below = ~0u;
  if constexpr (kTies) {                                  // the most numbers that do not make n yet, and one more
    below = 0;
    for (int b = 31; b >= 0; --b)
      if (count(bound, below | 1u << b) < n) below |= 1u << b;
    ++below;
  }
  if (tid == 0) room.count = 0;
  team_sync<T>();
  for (int i0 = 0; i0 < n_entries; i0 += T) {
    uint32_t item = 0;
    const uint64_t k = i0 + tid < n_entries ? key(i0 + tid, item) : 0;
    take(k, item, k > bound || (k == bound && item < below), room, lane);
  }
  team_sync<T>();
}
template <bool kTies, int T, class Key>
__device__ __forceinline__ int top_items(Key key, int n_entries, int n, JoinRoom<T>& room, int tid) {
  const int lane = tid & (kWave - 1);
  uint64_t mine = 0;
  uint32_t item = 0;
#pragma unroll 4
  for (int i = tid; i < n_entries; i += T) { const uint64_t k = key(i, item); mine = k > mine ? k : mine; }
  const uint64_t bound = find_bound(mine, n, room, tid);
#pragma unroll 4
  for (int i0 = 0; i0 < n_entries; i0 += T) {
    const uint64_t k = i0 + tid < n_entries ? key(i0 + tid, item) : 0;
    take(k, item, k >= bound, room, lane);
  }
  team_sync<T>();
  if (__builtin_expect(room.count > JoinRoom<T>::kRoom, 0)) take_exactly<kTies>(key, n_entries, n, bound, room, tid);
  return sort_room<kTies>(room, n, tid);
}

struct RowSum {
  double log_sum;
  float ref;
};
// log of a row's sum of exponentials relative to `ref`, by a wave; ref = -inf: the row offers nothing.  Plain sums lie in 2^-800 .. 2^930, far ones
// are 1 .. 2^990 of a reference that may be anywhere (a logit counts up to 2^960 before it moves its wave's).  So a power is taken in two halves
// where it brings a far sum down by more than fp64's range, and vanishes only where what it stands for does: next to a plain sum of 2^-800 too.
__device__ __forceinline__ RowSum row_sum(const BeamArgs& a, int row, int lane) {
  const BeamPart* parts = a.parts + (int64_t)row * a.n_parts;
  const double c = a.range.c;
  bool bad = false, plain = false;
  float ref = -INFINITY;
  for (int i = lane; i < a.n_parts; i += kWave) {
    const BeamPart q = parts[i];
    bad |= q.bad != 0;
    plain |= q.plain > 0.0;
    ref = fmaxf(ref, q.ref);
  }
  ref = wave_max_f32(ref);
  if (__ballot(plain)) ref = fmaxf(ref, 0.f);             // (plain sums are relative to a logit of 0)
  if (__ballot(bad) || ref == -INFINITY) return RowSum{0.0, -INFINITY};
  double sum = 0.0;
  for (int i = lane; i < a.n_parts; i += kWave) {
    const BeamPart q = parts[i];
    if (q.plain > 0.0) sum += q.plain * exp2(-(double)ref * c);   // (then ref >= 0; otherwise the power may be anything)
    if (q.ref > -INFINITY) {
      const double half = exp2(0.5 * ((double)q.ref - (double)ref) * c);
      sum += q.sum * half * half;
    }
  }
  return RowSum{log(wave_sum_f64_dpp(sum)), ref};
}

// what a row offers, in order, n places, by a workgroup
template <int DT>
__device__ __forceinline__ void row_offers(const BeamArgs& a, int row, JoinRoom<kJoinThreads>& room, RowSum& shared_sum, BeamOffer* offer, int tid) {
  constexpr int EB = Logit<DT>::bytes, kEach = 8, kLanes = kBlock / kEach, kAtOnce = kJoinThreads / kLanes;
  const int lane = tid & (kWave - 1), wave = tid >> 6, group = row / a.beams;
  const float s = a.scores[row];
  const bool lives = row_lives(s), done = a.finished && a.finished[row];
  double weight = 1.0;
  if (a.penalty != 0.0) weight = pow(fmax((double)a.lengths[row] + (done ? 0.0 : 1.0), 1.0), a.penalty);
  int count = 0;
  if (lives && done) {
    count = 1;
    if (tid == 0) offer[0] = BeamOffer{f64_key((double)s / weight), s, a.end_token};
  } else if (lives) {
    if (wave == kJoinThreads / kWave - 1) {               // (the other waves go ahead)
      const RowSum sum = row_sum(a, row, lane);
      if (lane == 0) shared_sum = sum;
    }
    const uint8_t* p = a.logits + (int64_t)group * a.group_stride + (int64_t)(row % a.beams) * a.beam_stride;
    // (logit, ~number): among equal logits the lower token or block goes first
    auto key_of = [](uint32_t upper, int number) -> uint64_t { return upper > kLowestKey ? ((uint64_t)upper << 32) | (uint32_t)~number : 0; };
    auto token_key = [&](int t, uint32_t&) { return key_of(f32_key(Logit<DT>::one(p + (int64_t)t * EB)), t); };
    if (a.n_blocks <= a.n) {                              // all blocks are among the n best
      count = top_items<false>(token_key, a.vocab, a.n, room, tid);
    } else {
      const uint32_t* peak = a.peaks + (int64_t)row * a.n_blocks;
      const int n_best = top_items<false>([&](int i, uint32_t&) { return key_of(peak[i], i); }, a.n_blocks, a.n, room, tid);
      auto block = [&](int i) { return (int)~(uint32_t)room.best[i]; };
      auto each_token = [&](auto f) {
        for (int i0 = 0; i0 < n_best; i0 += kAtOnce) {
          const int i = i0 + tid / kLanes;
          const int at = i < n_best ? block(i) * kBlock + tid % kLanes * kEach : a.vocab;
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
          for (int e = 0; e < kEach; ++e) f(key_of(f32_key(x[e]), at + e));
        }
      };
      // tokens that are not less than the n-th block's largest (where fewer blocks hold any: than the n-th of the threads' largest)
      uint64_t bound = n_best == a.n ? room.best[n_best - 1] >> 32 << 32 : 0;
      if (bound == 0) {
        uint64_t mine = 0;
        each_token([&](uint64_t k) { mine = k > mine ? k : mine; });
        bound = find_bound(mine, a.n, room, tid);
      }
      if (tid == 0) room.count = 0;
      __syncthreads();
      each_token([&](uint64_t k) { take(k, 0, k >= bound, room, lane); });
      __syncthreads();
      if (__builtin_expect(room.count > JoinRoom<kJoinThreads>::kRoom, 0))
        take_exactly<false>([&](int i, uint32_t& item) -> uint64_t {
          const int t = block(i / kBlock) * kBlock + i % kBlock;
          return t < a.vocab ? token_key(t, item) : 0;
        }, n_best * kBlock, a.n, bound, room, tid);
      count = sort_room<false>(room, a.n, tid);
    }
    const RowSum sum = shared_sum;
    if (sum.ref == -INFINITY) count = 0;
    if (tid < count) {
      const double score = (double)s - sum.log_sum + a.scale * ((double)key_f32((uint32_t)(room.best[tid] >> 32)) - (double)sum.ref);
      offer[tid] = BeamOffer{f64_key(score / weight), (float)score, (int32_t)~(uint32_t)room.best[tid]};
    }
  }
  if (tid >= count && tid < a.n) offer[tid] = BeamOffer{0, -INFINITY, -1};
}

// place `tid` of a group's choice: offer `item`, if there is one.  (By one wave, so that all that the group's rows held has been read before anything is
// written: the outputs may be the inputs.)
__device__ __forceinline__ void give_out(const BeamArgs& a, int group, const BeamOffer* all, bool there, int item, int tid) {
  float out_s = -INFINITY;
  int parent = -1, token = -1, length = 0;
  bool ended = false;
  if (there) {
    const BeamOffer o = all[item];
    parent = group * a.beams + item / a.n;
    const bool was = a.finished && a.finished[parent];
    out_s = o.score;
    token = o.token;
    ended = was || (a.end_token >= 0 && token == a.end_token);
    if (a.out_lengths) length = a.lengths[parent] + (was ? 0 : 1);
  }
  __builtin_amdgcn_s_waitcnt(0);
  if (tid < a.n) {
    const int at = group * a.n + tid;
    a.out_scores[at] = out_s;
    a.out_parents[at] = parent;
    a.out_tokens[at] = token;
    if (a.out_finished) a.out_finished[at] = ended;
    if (a.out_lengths) a.out_lengths[at] = length;
  }
}

// of what the rows of a group offer, the best
__device__ __forceinline__ void choose(const BeamArgs& a, int group, const BeamOffer* all, JoinRoom<kJoinThreads>& room, int tid) {
  const int found = top_items<true>([&](int i, uint32_t& item) -> uint64_t {
    item = (uint32_t)i;                                   // in order of rows, then of places
    return all[i].rank;
  }, a.beams * a.n, a.n, room, tid);
  give_out(a, group, all, tid < found, tid < found ? (int)room.best_item[tid] : 0, tid);
}

template <int DT>
__global__ __launch_bounds__(kJoinThreads) void beam_join_kernel(BeamArgs a) {
  __shared__ JoinRoom<kJoinThreads> room;
  __shared__ RowSum sum;
  row_offers<DT>(a, blockIdx.x, room, sum, a.offers + (int64_t)blockIdx.x * a.n, threadIdx.x);
}
__global__ __launch_bounds__(kJoinThreads) void beam_choose_kernel(BeamArgs a) {
  __shared__ JoinRoom<kJoinThreads> room;
  choose(a, blockIdx.x, a.offers + (int64_t)blockIdx.x * a.beams * a.n, room, threadIdx.x);
}
// ---- small calls: both in one launch, two waves for each of a group's rows -----------------------------------------------------
// One wave of a row finds its best tokens, the other its sum.  Few places out of few keys are taken one by one, without LDS: the largest of the
// wave, n times, 0.6 us a place; a third launch costs 2.5 us on the host and 2 on the GPU.  Captured and replayed, rows of 32000: 10.8 us at 1 x 4 with 4
// places and 13.2 in three launches, 11.6 and 15.5 at 64 x 2 with 2, but 14.7 and 13.1 at 1 x 4 with 8; a row at a time of 1000, 7.8 and 12.1.  (Beams and
// blocks end where a wave holds an offer a lane, and two keys a lane: nothing has been measured beyond.)
constexpr int kFewBeams = 4, kFewInOne = 4, kFewBlocks = 128;
struct Taken {
  uint64_t key;                                           // lane i: the i-th largest, 0 if there are fewer
  int lane;                                               // whose it was
};
// equal keys go in order of lanes
template <int K>
__device__ __forceinline__ Taken take_in_turn(uint64_t (&k)[K], int n, int lane) {
  Taken t{0, 0};
  for (int i = 0; i < n; ++i) {
    uint64_t mine = k[0];
#pragma unroll
    for (int e = 1; e < K; ++e) mine = k[e] > mine ? k[e] : mine;
    const uint32_t upper = wave_max_u32((uint32_t)(mine >> 32));
    const uint32_t lower = wave_max_u32((uint32_t)(mine >> 32) == upper ? (uint32_t)mine : 0u);
    const uint64_t top = (uint64_t)upper << 32 | lower;
    if (top == 0) break;
    const int from = __ffsll((unsigned long long)__ballot(mine == top)) - 1;
    bool here = lane == from;
#pragma unroll
    for (int e = 0; e < K; ++e)
      if (here && k[e] == top) { k[e] = 0; here = false; }
    if (lane == i) t = Taken{top, from};
  }
  return t;
}

template <int DT>
__global__ __launch_bounds__(2 * kFewBeams * kWave) void beam_finish_kernel(BeamArgs a) {
  constexpr int EB = Logit<DT>::bytes, kEach = 8, kLanes = kBlock / kEach, kAtOnce = kWave / kLanes, kBatch = kFewInOne / kAtOnce;
  __shared__ JoinRoom<kWave> rooms[kFewBeams];
  __shared__ BeamOffer offers[kFewBeams * kFewInOne];
  __shared__ RowSum sums[kFewBeams];
  const int w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & (kWave - 1), group = blockIdx.x;
  const int b = w < a.beams ? w : w - a.beams, row = group * a.beams + b;
  const float s = a.scores[row];
  const bool lives = row_lives(s), done = a.finished && a.finished[row];
  JoinRoom<kWave>& room = rooms[b];
  uint64_t best = 0;                                      // lane i: (logit, ~token) of the row's i-th best
  int count = 0;
  if (w >= a.beams) {
    const RowSum sum = lives && !done ? row_sum(a, row, lane) : RowSum{0.0, -INFINITY};
    if (lane == 0) sums[b] = sum;
  } else if (lives && !done) {
    const uint8_t* p = a.logits + (int64_t)group * a.group_stride + (int64_t)b * a.beam_stride;
    const uint32_t* peak = a.peaks + (int64_t)row * a.n_blocks;
    auto key_of = [](uint32_t upper, int number) -> uint64_t { return upper > kLowestKey ? ((uint64_t)upper << 32) | (uint32_t)~number : 0; };
    uint64_t k[kFewBlocks / kWave];
#pragma unroll
    for (int e = 0; e < kFewBlocks / kWave; ++e) {
      const int i = e * kWave + lane;
      k[e] = i < a.n_blocks ? key_of(peak[i], i) : 0;
    }
    const Taken blocks = take_in_turn(k, a.n, lane);
    const int n_best = __popcll(__ballot(blocks.key != 0));
    if (a.vocab >= kEach) {
      uint32_t raw[kBatch][kEach * EB / 4];
      int at[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int i = j * kAtOnce + lane / kLanes;
        const int block = (int)~(uint32_t)__shfl((int)(uint32_t)blocks.key, i, kWave);
        at[j] = i < n_best ? block * kBlock + lane % kLanes * kEach : a.vocab;
        __builtin_memcpy(raw[j], p + (int64_t)min(at[j], a.vocab - kEach) * EB, kEach * EB);
      }
      // (a lane at the row's end reads its last tokens, and leaves out what is another's)
      auto each_token = [&](auto f) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          float x[kEach];
          Logit<DT>::template unpack<kEach>(raw[j], x);
          const int first = min(at[j], a.vocab - kEach);
#pragma unroll
          for (int e = 0; e < kEach; ++e) f(first + e >= at[j] ? key_of(f32_key(x[e]), first + e) : 0);
        }
      };
      // tokens that are not less than the n-th block's largest (where fewer blocks hold any: than the n-th of the lanes' largest)
      uint64_t bound = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(blocks.key >> 32), a.n - 1) << 32;
      if (n_best < a.n) {
        uint64_t mine = 0;
        each_token([&](uint64_t key) { mine = key > mine ? key : mine; });
        bound = find_bound(mine, a.n, room, lane);
      }
      if (lane == 0) room.count = 0;
      team_sync<kWave>();
      each_token([&](uint64_t key) { take(key, 0, key >= bound, room, lane); });
      team_sync<kWave>();
      if (__builtin_expect(room.count > JoinRoom<kWave>::kRoom, 0))
        take_exactly<false>([&](int i, uint32_t&) -> uint64_t {
          const int t = (int)~(uint32_t)__shfl((int)(uint32_t)blocks.key, i / kBlock, kWave) * kBlock + i % kBlock;
          return t < a.vocab ? key_of(f32_key(Logit<DT>::one(p + (int64_t)t * EB)), t) : 0;
        }, n_best * kBlock, a.n, bound, room, lane);
      count = min(room.count, JoinRoom<kWave>::kRoom);
      uint64_t held[JoinRoom<kWave>::kRoom / kWave];
#pragma unroll
      for (int e = 0; e < JoinRoom<kWave>::kRoom / kWave; ++e) held[e] = e * kWave + lane < count ? room.key[e * kWave + lane] : 0;
      best = take_in_turn(held, a.n, lane).key;
    } else {
      count = top_items<false>([&](int t, uint32_t&) { return key_of(f32_key(Logit<DT>::one(p + (int64_t)t * EB)), t); }, a.vocab, a.n, room, lane);
      best = lane < count ? room.best[lane] : 0;
    }
  }
  __syncthreads();
  if (w < a.beams && lane < a.n) {
    BeamOffer o{0, -INFINITY, -1};
    double weight = 1.0;
    if (a.penalty != 0.0) weight = pow(fmax((double)a.lengths[row] + (done ? 0.0 : 1.0), 1.0), a.penalty);
    if (lives && done) {
      if (lane == 0) o = BeamOffer{f64_key((double)s / weight), s, a.end_token};
    } else if (best != 0 && sums[b].ref > -INFINITY) {
      const double score = (double)s - sums[b].log_sum + a.scale * ((double)key_f32((uint32_t)(best >> 32)) - (double)sums[b].ref);
      o = BeamOffer{f64_key(score / weight), (float)score, (int32_t)~(uint32_t)best};
    }
    offers[b * a.n + lane] = o;
  }
  __syncthreads();
  if (w) return;
  static_assert(kFewBeams * kFewInOne <= kWave, "an offer a lane");
  uint64_t k[1] = {lane < a.beams * a.n ? offers[lane].rank : 0};
  const Taken t = take_in_turn(k, a.n, lane);
  give_out(a, group, offers, t.key != 0, t.lane, lane);
}

template <int DT>
hipError_t launch(const BeamArgs& a, hipStream_t st) {
  const int rows = a.groups * a.beams;
  beam_parts_kernel<DT><<<dim3((unsigned)(((int64_t)rows * a.n_parts + 3) / 4)), 256, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.beams <= kFewBeams && a.n <= kFewInOne && a.n_blocks <= kFewBlocks) {
    beam_finish_kernel<DT><<<dim3((unsigned)a.groups), 2 * a.beams * kWave, 0, st>>>(a);
    return hipGetLastError();
  }
  beam_join_kernel<DT><<<dim3((unsigned)rows), kJoinThreads, 0, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  beam_choose_kernel<<<dim3((unsigned)a.groups), kJoinThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

// Tokens of a part: as many chunks as leave 8192 waves, 60 % more than the 5120 that the chip holds of this kernel (5 a SIMD).  (32 x 16 rows of 256K
// bf16, 8 / 16 / 32 chunks: 93.3 / 93.4 / 99.8 us; taken at this size alone, by an earlier form of the kernel.)
int beam_part_len(int64_t rows, int vocab) {
  const int64_t per = (rows * (((int64_t)vocab + kChunk - 1) / kChunk) + 8191) / 8192;
  return (int)std::min<int64_t>(std::max<int64_t>(per, 1), 1024) * kChunk;
}
BeamRange beam_range(double scale) {
  BeamRange r;
  r.c = scale * kLog2e;
  const bool fits = r.c > 0x1p-60 && r.c < 0x1p60;   // (else the borders leave fp32's range)
  r.low = fits ? (float)(-800.0 / r.c) : INFINITY;
  r.high = fits ? (float)(900.0 / r.c) : -INFINITY;
  r.absent = fits ? (float)(-900.0 / r.c) : -INFINITY;
  // (rounding of fp32 can double a step that is not taken: 2^960 for each of 2^30 tokens stays in fp64's range)
  r.reach = (float)std::min(480.0 / r.c, 1e38);
  return r;
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
