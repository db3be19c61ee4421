// The n best continuations of every group of beams, by summed log-probability:
//   score = s + c x_v - log sum_w exp(c x_w),   rank = score / length^a.
// Two launches.  The first reads the logits once: a wave takes a part of a row and keeps the part's sum of exponentials (fp64, relative to a
// logit of the part) and its n best logits in order.  The second, a workgroup per group, joins the parts of every row, forms the ranks of
// what the rows offer, and keeps the n best of those.
//
// Ranks of different rows meet in the choice, so the sums are fp64: exp as 2^t = 2^round(t) 2^f, f in [-1/2, 1/2], with 2^f the Chebyshev
// interpolation of degree 8 (off by 1.1e-12 at most), 2^round(t) added to the exponent's bits.  Lanes take the same tokens in the same
// order in every row, whatever its address is, so rows of equal logits get equal sums.
#include "../../include/shadowkv.h"
#include "common.hpp"
#include "kernels.hpp"

namespace skv {
namespace {

constexpr int kElems = 8;                       // logits of a lane at a time
constexpr int kChunk = kWave * kElems;
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
__device__ __forceinline__ uint64_t readlane_u64(uint64_t v, int lane) {
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
__device__ __forceinline__ uint64_t from_lane_below(uint64_t v, int lane) {
  const int src = lane > 0 ? lane - 1 : 0;
  return ((uint64_t)(uint32_t)__shfl((int)(v >> 32), src, kWave) << 32) | (uint32_t)__shfl((int)(uint32_t)v, src, kWave);
}
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
  static __device__ __forceinline__ void unpack(const uint4& w, float* x) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(u[i]); x[2 * i + 1] = bf16_hi(u[i]); }
  }
};
template <>
struct Logit<SHADOWKV_LOGITS_FP16> {
  static constexpr int bytes = 2;
  static __device__ __forceinline__ float one(const uint8_t* p) { return (float)*reinterpret_cast<const _Float16*>(p); }
  static __device__ __forceinline__ void unpack(const uint4& w, float* x) {
    typedef _Float16 half8 __attribute__((ext_vector_type(8)));
    const half8 h = __builtin_bit_cast(half8, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)h[i];
  }
};
template <>
struct Logit<SHADOWKV_LOGITS_FP32> {
  static constexpr int bytes = 4;
  static __device__ __forceinline__ float one(const uint8_t* p) { return *reinterpret_cast<const float*>(p); }
  static __device__ __forceinline__ void unpack(const uint4& w, float* x) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
  }
};

// whether a row takes part at all
__device__ __forceinline__ bool row_lives(float score) { return fabsf(score) < INFINITY; }

// c (the same in all lanes) into the wave's list of 64, lane i the i-th largest
__device__ __forceinline__ void insert(uint64_t& list, uint64_t c, int lane) {
  const int pos = __popcll(__ballot(list > c));
  const uint64_t below = from_lane_below(list, lane);
  list = lane < pos ? list : lane == pos ? c : below;
}

template <int DT>
__global__ __launch_bounds__(256) void beam_parts_kernel(BeamArgs a) {
  constexpr int EB = Logit<DT>::bytes, VEC = 16 / EB;
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (w >= (int64_t)a.groups * a.beams * a.n_parts) return;
  const int row = (int)(w / a.n_parts), part = (int)(w % a.n_parts);
  if (!row_lives(a.scores[row]) || (a.finished && a.finished[row])) return;   // (the second launch asks the same)
  const uint8_t* p = a.logits + (row / a.beams) * a.group_stride + (row % a.beams) * a.beam_stride;
  const int t0 = part * a.part_len, t1 = min(a.vocab, t0 + a.part_len);
  const double cl = a.scale * kLog2e;
  float ref = -INFINITY, least = -INFINITY;     // least: what the list's n-th logit is
  double sum = 0.0;
  bool bad = false;
  uint64_t list = 0;                            // (key of the logit, ~token); 0: nothing
  for (int base = t0; base < t1; base += kChunk) {
    float x[kElems];
#pragma unroll
    for (int i = 0; i < kElems / VEC; ++i) {
      const int at = base + (i * kWave + lane) * VEC;
      if (at + VEC <= t1) {
        uint4 v;
        __builtin_memcpy(&v, p + (int64_t)at * EB, 16);      // (rows of an odd vocabulary begin at any element)
        Logit<DT>::unpack(v, x + i * VEC);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[i * VEC + e] = at + e < t1 ? Logit<DT>::one(p + (int64_t)(at + e) * EB) : -INFINITY;
      }
    }
    float mx = x[0];
#pragma unroll
    for (int e = 0; e < kElems; ++e) {
      bad |= __builtin_isnan(x[e]) || x[e] == INFINITY;
      mx = fmaxf(mx, x[e]);
    }
    // the reference moves up only where 2^t might leave fp64's range
    if (__ballot(((double)mx - (double)ref) * cl > 500.0)) {
      const float to = wave_max_f32(mx);
      sum *= exp2_f64(fmax(((double)ref - (double)to) * cl, -1000.0));
      ref = to;
    }
    if (ref > -INFINITY) {
#pragma unroll
      for (int e = 0; e < kElems; ++e) sum += exp2_f64(fmax(((double)x[e] - (double)ref) * cl, -1000.0));
    }
    if (__ballot(mx > least)) {                 // (a later token of an equal logit is not better)
#pragma unroll
      for (int e = 0; e < kElems; ++e) {
        const uint32_t token = (uint32_t)(base + ((e / VEC) * kWave + lane) * VEC + e % VEC);
        const uint64_t mine = ((uint64_t)f32_key(x[e]) << 32) | (uint32_t)~token;
        uint64_t some = __ballot(x[e] >= least && x[e] > -INFINITY);
        while (some) {
          const int from = __ffsll((unsigned long long)some) - 1;
          some &= some - 1;
          const uint64_t c = readlane_u64(mine, from);
          if (c > readlane_u64(list, a.n - 1)) insert(list, c, lane);
        }
        const uint64_t last = readlane_u64(list, a.n - 1);
        least = last ? key_f32((uint32_t)(last >> 32)) : -INFINITY;
      }
    }
  }
  sum = wave_sum_f64_dpp(sum);
  const bool any_bad = __ballot(bad) != 0;
  if (lane == 0) a.parts[w] = BeamPart{sum, ref, any_bad};
  if (lane < a.n) a.best[w * a.n + lane] = make_uint2(__float_as_uint(key_f32((uint32_t)(list >> 32))), list ? ~(uint32_t)list : ~0u);
}

// What a row offers, in LDS: candidate i is (logit, token); score = base + c (logit - ref).
struct RowOffer {
  double base, weight;                          // weight: length^penalty
  float ref;
  int count;
};

__global__ __launch_bounds__(256) void beam_join_kernel(BeamArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  RowOffer* offer = reinterpret_cast<RowOffer*>(lds);                        // [beams]
  uint2* cand = reinterpret_cast<uint2*>(offer + a.beams);                   // [beams, n]
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, group = blockIdx.x;
  const double cl = a.scale * kLog2e;
  for (int b = wave; b < a.beams; b += 4) {
    const int row = group * a.beams + b;
    const float s = a.scores[row];
    const bool done = a.finished && a.finished[row];
    RowOffer o{(double)s, 1.0, 0.f, 0};
    if (a.penalty != 0.0) o.weight = pow(fmax((double)a.lengths[row] + (done ? 0.0 : 1.0), 1.0), a.penalty);
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
        double sum = 0.0;
        for (int i = lane; i < a.n_parts; i += kWave)
          if (parts[i].ref > -INFINITY) sum += parts[i].sum * exp2_f64(fmax(((double)parts[i].ref - (double)ref) * cl, -1000.0));
        sum = wave_sum_f64_dpp(sum);
        o.base = (double)s - log(sum);
        o.ref = ref;
        // the n best of the parts' lists, best places first
        const uint2* best = a.best + (int64_t)row * a.n_parts * a.n;
        uint64_t list = 0;
        for (int place = 0; place < a.n; ++place)
          for (int i0 = 0; i0 < a.n_parts; i0 += kWave) {
            uint64_t mine = 0;
            if (i0 + lane < a.n_parts) {
              const uint2 c = best[(int64_t)(i0 + lane) * a.n + place];
              if (c.y != ~0u) mine = ((uint64_t)f32_key(__uint_as_float(c.x)) << 32) | (uint32_t)~c.y;
            }
            uint64_t some = __ballot(mine > readlane_u64(list, a.n - 1));
            while (some) {
              const int from = __ffsll((unsigned long long)some) - 1;
              some &= some - 1;
              const uint64_t c = readlane_u64(mine, from);
              if (c > readlane_u64(list, a.n - 1)) insert(list, c, lane);
            }
          }
        o.count = __popcll(__ballot(lane < a.n && list != 0));
        if (lane < a.n) cand[b * a.n + lane] = make_uint2(__float_as_uint(key_f32((uint32_t)(list >> 32))), ~(uint32_t)list);
      }
    }
    if (lane == 0) offer[b] = o;
  }
  __syncthreads();
  if (wave) return;
  // ranks of all rows' candidates, best places first; lane i holds the i-th best: key of the rank, and (row, place) upside down
  uint64_t key = 0;
  uint32_t who = 0;
  for (int place = 0; place < a.n; ++place)
    for (int b0 = 0; b0 < a.beams; b0 += kWave) {
      uint64_t k = 0;
      uint32_t o = 0;
      if (b0 + lane < a.beams) {
        const int b = b0 + lane;
        if (place < offer[b].count) {
          const double score = offer[b].base + a.scale * ((double)__uint_as_float(cand[b * a.n + place].x) - (double)offer[b].ref);
          k = f64_key(score / offer[b].weight);
          o = ~(uint32_t)(b * 64 + place);
        }
      }
      uint64_t last = readlane_u64(key, a.n - 1);
      uint32_t last_who = (uint32_t)__builtin_amdgcn_readlane((int)who, a.n - 1);
      uint64_t some = __ballot(k > last || (k == last && o > last_who));
      while (some) {
        const int from = __ffsll((unsigned long long)some) - 1;
        some &= some - 1;
        const uint64_t ck = readlane_u64(k, from);
        const uint32_t co = (uint32_t)__builtin_amdgcn_readlane((int)o, from);
        const int pos = __popcll(__ballot(key > ck || (key == ck && who > co)));
        const uint64_t key_below = from_lane_below(key, lane);
        const uint32_t who_below = (uint32_t)__shfl((int)who, lane > 0 ? lane - 1 : 0, kWave);
        key = lane < pos ? key : lane == pos ? ck : key_below;
        who = lane < pos ? who : lane == pos ? co : who_below;
      }
    }
  // (all that this group's rows held has been read before anything is written: the outputs may be the inputs)
  float out_s = -INFINITY;
  int parent = -1, token = -1, length = 0;
  bool ended = false;
  if (lane < a.n && key) {
    const int b = (int)(~who >> 6), place = (int)(~who & 63u), row = group * a.beams + b;
    const uint2 c = cand[b * a.n + place];
    const bool was = a.finished && a.finished[row];
    out_s = (float)(offer[b].base + a.scale * ((double)__uint_as_float(c.x) - (double)offer[b].ref));
    parent = row;
    token = (int)c.y;
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

}  // namespace

int beam_part_len(int64_t rows, int vocab) {
  (void)rows; (void)vocab;
  return 2048;
}

hipError_t launch_beam_select(const BeamArgs& a, hipStream_t st) {
  const int64_t waves = (int64_t)a.groups * a.beams * a.n_parts;
  const dim3 grid((unsigned)((waves + 3) / 4));
  switch (a.dtype) {
    case SHADOWKV_LOGITS_BF16: beam_parts_kernel<SHADOWKV_LOGITS_BF16><<<grid, 256, 0, st>>>(a); break;
    case SHADOWKV_LOGITS_FP16: beam_parts_kernel<SHADOWKV_LOGITS_FP16><<<grid, 256, 0, st>>>(a); break;
    default: beam_parts_kernel<SHADOWKV_LOGITS_FP32><<<grid, 256, 0, st>>>(a); break;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const size_t lds = (size_t)a.beams * (sizeof(RowOffer) + a.n * sizeof(uint2));
  beam_join_kernel<<<dim3((unsigned)a.groups), 256, lds, st>>>(a);
  return hipGetLastError();
}

}  // namespace skv
