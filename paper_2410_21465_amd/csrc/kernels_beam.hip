// The n best continuations of every group of beams, by summed log-probability:
//   score = s + c x_v - log sum_w exp(c x_w),   rank = score / length^a.
// Two launches.  The first reads the logits once: a wave takes a part of a row, sums its exponentials (fp64, relative to a logit of the
// part) and keeps the largest logit of every block of 128 tokens, nothing else.  The second has a workgroup per group and a wave per row: the
// n best tokens of a row lie in the n blocks with the largest maxima (whatever lies in another block has n better ones, one in each of
// those), so it finds these, reads them again, and keeps their n best; then the first wave ranks what all rows offer.
//
// Ranks of different rows meet in the choice, so the sums are fp64: exp as 2^t = 2^round(t) 2^f, f in [-1/2, 1/2], with 2^f the Chebyshev
// interpolation of degree 8 (off by 1.1e-12 at most), 2^round(t) added to the exponent's bits.  Lanes take the same tokens in the same
// order in every row, whatever its address is, so rows of equal logits get equal sums.
#include "../../include/shadowkv.h"
#include "common.hpp"
#include "kernels.hpp"

namespace skv {
namespace {

constexpr int kElems = 8;                       // consecutive logits of a lane
constexpr int kChunk = kWave * kElems;
constexpr int kBlock = 16 * kElems;             // tokens of a block: a row of 16 lanes
constexpr double kLog2e = 1.4426950408889634074;

// 2^t for t in [-1000, 1000]
__device__ __forceinline__ double exp2_f64(double t) {
  const double big = 6755399441055744.0;        // 1.5 2^52: the low bits of t + big are round(t)
  const double a = t + big, f = t - (a - big);
  double p = 1.3255179556479267e-06;
  p = fma(p, f, 1.5310080611926545e-05);
  p = fma(p, f, 0.00015403456082633648);
  p = fma(p, f, 0.0013333450563173552);
  p = fma(p, f, 0.009618129159053034);
  p = fma(p, f, 0.055504109412108156);
  p = fma(p, f, 0.24022650695814518);
  p = fma(p, f, 0.6931471805459332);
  p = fma(p, f, 1.0000000000000004);
  return __hiloint2double(__double2hiint(p) + (__double2loint(a) << 20), __double2loint(p));
}

__device__ __forceinline__ uint32_t f32_key(float x) {   // larger value <=> larger key, never 0 but for NaN
  x += 0.f;                                              // (-0 is +0)
  const uint32_t u = __float_as_uint(x);
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
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
  static __device__ __forceinline__ void unpack(const uint32_t* w, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
  }
};
template <>
struct Logit<SHADOWKV_LOGITS_FP16> {
  static constexpr int bytes = 2;
  static __device__ __forceinline__ float one(const uint8_t* p) { return (float)*reinterpret_cast<const _Float16*>(p); }
  static __device__ __forceinline__ void unpack(const uint32_t* w, float* x) {
    typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const half2_t h = __builtin_bit_cast(half2_t, w[i]);
      x[2 * i] = (float)h[0]; x[2 * i + 1] = (float)h[1];
    }
  }
};
template <>
struct Logit<SHADOWKV_LOGITS_FP32> {
  static constexpr int bytes = 4;
  static __device__ __forceinline__ float one(const uint8_t* p) { return *reinterpret_cast<const float*>(p); }
  static __device__ __forceinline__ void unpack(const uint32_t* w, float* x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
  }
};

// whether a row takes part at all
__device__ __forceinline__ bool row_lives(float score) { return fabsf(score) < INFINITY; }

template <int DT>
__global__ __launch_bounds__(256) void beam_parts_kernel(BeamArgs a) {
  constexpr int EB = Logit<DT>::bytes, WORDS = kElems * EB / 4;
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (w >= (int64_t)a.groups * a.beams * a.n_parts) return;
  const int row = (int)(w / a.n_parts), part = (int)(w % a.n_parts);
  if (!row_lives(a.scores[row]) || (a.finished && a.finished[row])) return;   // (the second launch asks the same)
  const uint8_t* p = a.logits + (row / a.beams) * a.group_stride + (row % a.beams) * a.beam_stride;
  const int t0 = part * a.part_len, t1 = min(a.vocab, t0 + a.part_len);
  float* peak = a.peaks + (int64_t)row * a.n_blocks + t0 / kBlock;
  const double cl = a.scale * kLog2e;
  const float reach = (float)fmin(500.0 / cl, 1e38);
  float ref = -INFINITY;
  double sum = 0.0;
  bool bad = false;
  uint32_t raw[WORDS];
  auto load = [&](int base) {                   // (rows of an odd vocabulary begin at any element; behind the last one: minus infinity)
    const int at = base + lane * kElems;
    if (at + kElems <= t1) {
      __builtin_memcpy(raw, p + (int64_t)at * EB, kElems * EB);
    } else {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) raw[i] = DT == SHADOWKV_LOGITS_BF16 ? 0xff80ff80u : DT == SHADOWKV_LOGITS_FP16 ? 0xfc00fc00u : 0xff800000u;
      for (int e = 0; e < kElems; ++e) {
        if (at + e >= t1) break;
        if constexpr (EB == 4) {
#pragma unroll
          for (int i = 0; i < WORDS; ++i)
            if (i == e) raw[i] = *reinterpret_cast<const uint32_t*>(p + (int64_t)(at + e) * EB);
        } else {
          const uint32_t h = *reinterpret_cast<const uint16_t*>(p + (int64_t)(at + e) * EB);
#pragma unroll
          for (int i = 0; i < WORDS; ++i)
            if (i == e / 2) raw[i] = e & 1 ? (raw[i] & 0xffffu) | (h << 16) : (raw[i] & 0xffff0000u) | h;
        }
      }
    }
  };
  load(t0);
  for (int base = t0; base < t1; base += kChunk) {
    float x[kElems];
    Logit<DT>::unpack(raw, x);
    if (base + kChunk < t1) load(base + kChunk);
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < kElems; ++e) mx = __builtin_elementwise_maximum(mx, x[e]);   // (NaN if one is)
    bad |= !(mx < INFINITY);
    // the reference moves up only where 2^t might leave fp64's range
    if (__ballot(mx > ref + reach)) {
      const float to = wave_max_f32(mx);
      sum *= exp2_f64(fmax(((double)ref - (double)to) * cl, -1000.0));
      ref = to;
    }
    if (ref > -INFINITY) {
#pragma unroll
      for (int e = 0; e < kElems; ++e) sum += exp2_f64(fmax(((double)x[e] - (double)ref) * cl, -1000.0));
    }
    float m = mx;                               // lane 15 of 16 ends with the largest of them
    m = fmaxf(m, __uint_as_float(dpp_u32<0x111>(__float_as_uint(m), __float_as_uint(m))));
    m = fmaxf(m, __uint_as_float(dpp_u32<0x112>(__float_as_uint(m), __float_as_uint(m))));
    m = fmaxf(m, __uint_as_float(dpp_u32<0x114>(__float_as_uint(m), __float_as_uint(m))));
    m = fmaxf(m, __uint_as_float(dpp_u32<0x118>(__float_as_uint(m), __float_as_uint(m))));
    const int block = (base - t0) / kBlock + lane / 16;
    if (lane % 16 == 15 && block * kBlock < t1 - t0) peak[block] = m;
  }
  sum = wave_sum_f64_dpp(sum);
  const bool any_bad = __ballot(bad) != 0;
  if (lane == 0) a.parts[w] = BeamPart{sum, ref, any_bad};
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
#pragma unroll 16
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
#pragma unroll 8
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
template <class K, class Key>
__device__ __forceinline__ int top_items(Key key, int n_items, int n, SortRoom& room, uint64_t* keys, uint32_t* items, int lane) {
  constexpr int kHeld = 16;                               // keys of a lane at a time
  K held[kHeld], mine = 0;
  const int step = kHeld * kWave;
  auto load = [&](int i0) {
#pragma unroll
    for (int e = 0; e < kHeld; ++e) { const int i = i0 + e * kWave + lane; held[e] = i < n_items ? key(i) : 0; }
  };
  for (int i0 = 0; i0 < n_items; i0 += step) {
    load(i0);
#pragma unroll
    for (int e = 0; e < kHeld; ++e) mine = held[e] > mine ? held[e] : mine;
  }
  const uint64_t bound = lane_bound(mine, n, room, lane);
  int c = 0;
  for (int i0 = 0; i0 < n_items; i0 += step) {
    if (n_items > step) load(i0);
#pragma unroll
    for (int e = 0; e < kHeld; ++e)
      if (i0 + e * kWave < n_items) take(held[e], (uint32_t)(i0 + e * kWave + lane), held[e] >= bound, room, c, lane);
  }
  if (c > kSortRoom) c = take_exactly<sizeof(K) * 8>(key, n_items, n, bound, room, lane);
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
  constexpr int EB = Logit<DT>::bytes, WORDS = kElems * EB / 4, kAtOnce = kWave / 16;   // blocks that a wave reads at a time
  extern __shared__ __align__(16) uint8_t lds[];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, waves = blockDim.x >> 6, group = blockIdx.x;
  JoinWave& mine = reinterpret_cast<JoinWave*>(lds)[wave];
  uint64_t* rank = reinterpret_cast<uint64_t*>(lds + waves * sizeof(JoinWave));    // [beams, n] keys of the ranks, 0: none
  uint2* cand = reinterpret_cast<uint2*>(rank + a.beams * a.n);                    // [beams, n]
  RowOffer* offer = reinterpret_cast<RowOffer*>(cand + a.beams * a.n);             // [beams]
  const double cl = a.scale * kLog2e;
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
      bool bad = false;
      float ref = -INFINITY;
      for (int i = lane; i < a.n_parts; i += kWave) { bad |= parts[i].bad != 0; ref = fmaxf(ref, parts[i].ref); }
      ref = wave_max_f32(ref);
      if (!__ballot(bad) && ref > -INFINITY) {
        const float* peak = a.peaks + (int64_t)row * a.n_blocks;
        const int n_best = top_items<uint32_t>([&](int i) { const float x = peak[i]; return x > -INFINITY ? f32_key(x) : 0u; }, a.n_blocks, a.n,
                                         mine.room, mine.keys, mine.items, lane);
        double sum = 0.0;
        for (int i = lane; i < a.n_parts; i += kWave)
          if (parts[i].ref > -INFINITY) sum += parts[i].sum * exp2_f64(fmax(((double)parts[i].ref - (double)ref) * cl, -1000.0));
        sum = wave_sum_f64_dpp(sum);
        o.base = (double)s - log(sum);
        o.ref = ref;
        // tokens of those blocks that are not less than the n-th block's largest (of fewer blocks: than the n-th lane's)
        const uint8_t* p = a.logits + group * a.group_stride + b * a.beam_stride;
        auto key_of = [&](float x, int t) { return x > -INFINITY ? ((uint64_t)f32_key(x) << 32) | (uint32_t)~t : 0ull; };
        auto each_token = [&](auto f) {
          for (int i0 = 0; i0 < n_best; i0 += kAtOnce) {
            const int i = i0 + lane / 16;
            const int at = i < n_best ? (int)mine.items[i] * kBlock + lane % 16 * kElems : a.vocab;
            float x[kElems];
            if (at + kElems <= a.vocab) {
              uint32_t raw[WORDS];
              __builtin_memcpy(raw, p + (int64_t)at * EB, kElems * EB);
              Logit<DT>::unpack(raw, x);
            } else {
#pragma unroll
              for (int e = 0; e < kElems; ++e) x[e] = at + e < a.vocab ? Logit<DT>::one(p + (int64_t)(at + e) * EB) : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < kElems; ++e) f(key_of(x[e], at + e));
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
        if (c > kSortRoom)
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
  const int count = top_items<uint64_t>([&](int i) { return rank[i]; }, a.beams * a.n, a.n, mine.room, mine.keys, mine.items, lane);
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

int beam_part_len(int64_t rows, int vocab) {
  const int64_t all = rows * (((int64_t)vocab + kChunk - 1) / kChunk);   // chunks
  const int64_t per = (all + 8191) / 8192;
  return (int)(per < 1 ? 1 : per > 1024 ? 1024 : per) * kChunk;
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
