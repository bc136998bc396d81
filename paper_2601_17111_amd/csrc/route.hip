// Routing of tokens to experts (llep_route) and its gradient
// (llep_route_backward).
//
// A row of E logits belongs to 4, 16 or 64 lanes of a wavefront, in registers: read
// once, and neither scores nor keys go to memory. Up to 8 experts of a row are
// found with sorted lists: every lane sorts its experts' keys eight (or four) at a
// time and merges them into its best so far, then the lanes of a row merge theirs.
// What the lists do not take (more than 8 experts, more groups than lanes) and what
// they cannot decide goes to rounds, a maximum over the row for each expert
// (pick_exact).
#include <math.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "rows.h"

namespace llep {

constexpr int kRouteThreads = 256;

// ---------------------------------------------------------------------------
// reductions over the lanes of a row, the result in each of them: exchanges between
// halves of twice the size each time, so that a sum has the same order, and the same
// bits, in every lane (with rotations it had not, and equal keys came out different)
// ---------------------------------------------------------------------------

template <int kCtrl, typename V>
__device__ __forceinline__ V rotated(V v) {
  if constexpr (sizeof(V) == 8) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(V, (uint64_t(dpp<kCtrl, 0xf>(uint32_t(u >> 32))) << 32) |
                                     dpp<kCtrl, 0xf>(uint32_t(u)));
  } else {
    return __builtin_bit_cast(V, dpp<kCtrl, 0xf>(__builtin_bit_cast(uint32_t, v)));
  }
}
template <bool k32, typename V>
__device__ __forceinline__ void exchange(V v, V &a, V &b) {
  auto swap = [](uint32_t w, uint32_t &x, uint32_t &y) {
    if constexpr (k32) {
      const auto r = __builtin_amdgcn_permlane32_swap(w, w, false, false);
      x = r[0], y = r[1];
    } else {
      const auto r = __builtin_amdgcn_permlane16_swap(w, w, false, false);
      x = r[0], y = r[1];
    }
  };
  if constexpr (sizeof(V) == 8) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    uint32_t al, ah, bl, bh;
    swap(uint32_t(u), al, bl);
    swap(uint32_t(u >> 32), ah, bh);
    a = __builtin_bit_cast(V, (uint64_t(ah) << 32) | al);
    b = __builtin_bit_cast(V, (uint64_t(bh) << 32) | bl);
  } else {
    uint32_t x, y;
    swap(__builtin_bit_cast(uint32_t, v), x, y);
    a = __builtin_bit_cast(V, x);
    b = __builtin_bit_cast(V, y);
  }
}
template <int kLanes, typename V, class Op>
__device__ __forceinline__ V over_row(V v, Op op) {
  v = op(v, rotated<0xb1>(v));  // quad_perm 1 0 3 2, 2 3 0 1
  v = op(v, rotated<0x4e>(v));
  if constexpr (kLanes >= 16) {
    v = op(v, rotated<0x141>(v));  // row_half_mirror: a lane of the other four; row_mirror
    v = op(v, rotated<0x140>(v));
  }
  if constexpr (kLanes == 64) {
    V a, b;
    exchange<false>(v, a, b);
    v = op(a, b);
    exchange<true>(v, a, b);
    v = op(a, b);
  }
  return v;
}
// (of doubles, none of them NaN, one instruction each)
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t smaller(uint32_t a, uint32_t b) { return a > b ? b : a; }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ double smaller(double a, double b) { return fmin(a, b); }
template <int kLanes, typename V>
__device__ __forceinline__ V row_max(V v) {
  return over_row<kLanes>(v, [](V a, V b) { return larger(a, b); });
}
template <int kLanes, typename V>
__device__ __forceinline__ V row_sum(V v) {
  return over_row<kLanes>(v, [](V a, V b) { return a + b; });
}

__device__ __forceinline__ float route_load(const uint16_t *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float route_load(const float *p) { return *p; }

// kPer logits from expert e0 on, those from E on -infinity; rows of any length and
// alignment (16-byte vectors where all of them are in the row)
template <int kPer, typename L>
__device__ __forceinline__ void route_load_row(const L *row, int e0, int E, float (&l)[kPer]) {
  constexpr int kVec = kPer < 8 ? kPer : 8;
  typedef L vec __attribute__((ext_vector_type(kVec), aligned(sizeof(L))));
#pragma unroll
  for (int c = 0; c < kPer; c += kVec) {
    if (e0 + c + kVec <= E) {
      const vec v = *reinterpret_cast<const vec *>(row + e0 + c);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const L x = v[j];
        l[c + j] = route_load(&x);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        l[c + j] = e0 + c + j < E ? route_load(row + e0 + c + j) : -__builtin_huge_valf();
    }
  }
}

// ---------------------------------------------------------------------------
// keys
//
// What is only ordered (kByLogit) is ordered by the logits themselves, with the
// expert's index below them, so that one maximum finds the largest and of equal ones
// the first: bfloat16 logits in 32 bits, float32 logits in float64, whose last bits
// they leave free. Where scores are added up (with the bias, or two of a group) the
// key is that sum in float64: scores a rounding apart are not told apart in 32 bits,
// and the choice would depend on the instruction that computed them.
// ---------------------------------------------------------------------------

// the float's bits in its order, above 0 for all but NaN with the sign set
__device__ __forceinline__ uint32_t ordered(float f) {
  f += 0.0f;  // -0 is equal to 0
  const uint32_t u = __float_as_uint(f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

// A float64 with an index in its last 9 bits, the larger the lower the index: a
// maximum of such numbers is one instruction (of 64-bit integers, three). An infinity
// becomes the largest finite number.
struct IndexedDouble {
  using V = double;
  static constexpr V kNone = -__builtin_huge_val();
  static constexpr uint64_t kIndex = 511;
  static __device__ __forceinline__ V make(double key, int e) {
    const int64_t u = __builtin_bit_cast(int64_t, fmin(key + 0.0, 0x1.fffffffffffffp1023));
    const uint64_t low = uint64_t(u < 0 ? e : int(kIndex) - e);
    return __builtin_bit_cast(V, (uint64_t(u) & ~kIndex) | low);
  }
  static __device__ __forceinline__ int index(V v) {
    const int64_t u = __builtin_bit_cast(int64_t, v);
    const int low = int(u & int64_t(kIndex));
    return u < 0 ? low : int(kIndex) - low;
  }
  static __device__ __forceinline__ double value(V v) {
    return __builtin_bit_cast(V, __builtin_bit_cast(uint64_t, v) & ~kIndex);
  }
};
static_assert(LLEP_MAX_EXPERTS <= IndexedDouble::kIndex + 1, "the index");

template <typename L, bool kByLogit>
struct RouteKey;
template <>
struct RouteKey<uint16_t, true> {
  using V = uint32_t;
  static constexpr V kNone = 0;
  static __device__ __forceinline__ V make(float l, int e) {
    return (ordered(l) & 0xffff0000u) | uint32_t(0xffff - e);
  }
  static __device__ __forceinline__ int index(V v) { return 0xffff - int(v & 0xffffu); }
  static __device__ __forceinline__ float logit(V v) {
    return __uint_as_float(__float_as_uint(unordered(v & 0xffff0000u)) & 0xffff0000u);
  }
};
template <>
struct RouteKey<float, true> : IndexedDouble {
  static __device__ __forceinline__ float logit(V v) {
    return v >= 0x1p1000 ? __builtin_huge_valf() : float(value(v));
  }
};
template <typename L>
struct RouteKey<L, false> {
  using V = double;
  static constexpr V kNone = -__builtin_huge_val();
};

// 1 / (1 + e^-l)
__device__ __forceinline__ float route_sigmoid(float l) { return 1.0f / (1.0f + expf(-l)); }

// of a wavefront's rows, those of a workgroup being kRows
template <int kRows, int kLanes>
__device__ __forceinline__ int64_t first_row() {
  return int64_t(blockIdx.x) * kRows +
         __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * (kWave / kLanes);
}

// The LDS of a wavefront is its own, so that its accesses, which are in order,
// need no barrier: this keeps the compiler from moving them.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <int kPer, int kLanes, typename V>
struct ExactLds {
  V keys[64 / kLanes][kPer * kLanes];
  V scores[64 / kLanes][64];
};

// A lane's keys: registers, or (kCold: a branch that few rows take, whose code and
// registers are kept small) LDS.
template <int kPer, int kLanes, typename V, bool kCold>
struct ExactKeys {
  V v[kPer];
  __device__ __forceinline__ explicit ExactKeys(V *) {}
  __device__ __forceinline__ V &operator[](int j) { return v[j]; }
};
template <int kPer, int kLanes, typename V>
struct ExactKeys<kPer, kLanes, V, true> {
  V *p;
  __device__ __forceinline__ explicit ExactKeys(V *row) : p(row + threadIdx.x % kLanes) {}
  __device__ __forceinline__ V &operator[](int j) { return p[j * kLanes]; }
};

// The K best of a row, one after another: lane k of the row returns the k-th
// expert, or -1. logit(j) is that of the expert j kLanes + t in lane t; `most` and
// `total` (kByLogit: not used) are the row's largest logit and, of softmax, the sum
// of e^(l - most).
template <typename L, int kPer, int kLanes, bool kByLogit, bool kCold, class Logit, typename Lds>
__device__ __forceinline__ int pick_exact(const RouteArgs &a, Logit logit, float most, Lds &lds) {
  using Key = RouteKey<L, kByLogit>;
  using V = typename Key::V;
  constexpr int kSlots = 64 / kLanes;  // groups per lane
  constexpr int kUnroll = kCold ? 1 : kPer;
  const int lane = lane_id(), t = lane % kLanes, mine = lane / kLanes;
  const float kInf = __builtin_huge_valf();
  ExactKeys<kPer, kLanes, V, kCold> v(lds.keys[mine]);
  wave_fence();
  if constexpr (kByLogit) {
#pragma unroll kUnroll
    for (int j = 0; j < kPer; ++j)
      v[j] = logit(j) > -kInf ? Key::make(logit(j), j * kLanes + t) : Key::kNone;
  } else {
    double wide = 0.0;
#pragma unroll kUnroll
    for (int j = 0; j < kPer; ++j) {
      const double x = logit(j);
      const double e = exp(a.score == LLEP_SCORE_SOFTMAX ? x - double(most) : -x);
      const double s = a.score == LLEP_SCORE_SOFTMAX ? e : 1.0 / (1.0 + e);
      v[j] = s;
      wide += s;
    }
    wide = a.score == LLEP_SCORE_SOFTMAX ? row_sum<kLanes>(wide) : 1.0;
#pragma unroll kUnroll
    for (int j = 0; j < kPer; ++j) {
      const int e = j * kLanes + t;
      const double k = v[j] / wide + (a.bias && e < a.E ? double(a.bias[e]) : 0.0);
      // (a key that is NaN is not above -infinity either)
      v[j] = logit(j) > -kInf && k > Key::kNone ? k : Key::kNone;
    }
  }
  if (a.groups > 1) {
    const int size = a.E / a.groups;
    const float per = 1.0f / float(size);
    if constexpr (!kCold) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) lds.keys[mine][j * kLanes + t] = v[j];
    }
    wave_fence();
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const int g = s * kLanes + t;
      if (g >= a.groups) break;
      V one = Key::kNone, two = Key::kNone;
      int i = t % size;  // from lane to lane other banks
      for (int n = 0; n < size; ++n) {
        const V k = lds.keys[mine][g * size + i];
        two = k > one ? one : k > two ? k : two;
        one = k > one ? k : one;
        i = i + 1 == size ? 0 : i + 1;
      }
      if constexpr (!kByLogit)
        if (a.group_score == LLEP_GROUP_TOP2 && two > Key::kNone) one += two;
      lds.scores[mine][g] = one;
    }
    wave_fence();
    uint64_t keep = 0;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const int g = s * kLanes + t;
      bool in = g < a.groups;
      if (in) {
        const V own = lds.scores[mine][g];
        int before = 0;
        for (int h = 0; h < a.groups; ++h) {
          const V k = lds.scores[mine][h];
          before += k > own || (k == own && h < g);
        }
        in = before < a.top_groups;
      }
      const uint64_t all = __ballot(in);
      if constexpr (kLanes == 64)
        keep = all;
      else
        keep |= ((all >> (lane & 48)) & 0xffffu) << (16 * s);
    }
#pragma unroll kUnroll
    for (int j = 0; j < kPer; ++j) {
      // e / size (the quotient's distance from a whole number is at least
      // 1 / (2 size), far above its rounding)
      const int g = int((float(j * kLanes + t) + 0.5f) * per);
      if (g < 64 && !((keep >> g) & 1)) v[j] = Key::kNone;
    }
  }
  int id = -1;
  for (int k = 0; k < a.K; ++k) {
    V best = v[0];
#pragma unroll kUnroll
    for (int j = 1; j < kPer; ++j) {
      const V x = v[j];
      best = x > best ? x : best;
    }
    best = row_max<kLanes>(best);
    int e;
    if constexpr (kByLogit) {
      e = Key::index(best);
    } else {
      uint32_t first = 0xffff;
#pragma unroll kUnroll
      for (int j = kPer - 1; j >= 0; --j)
        if (v[j] == best) first = uint32_t(j * kLanes + t);
      e = int(over_row<kLanes>(first, [](uint32_t x, uint32_t y) { return min(x, y); }));
    }
    if (t == k) id = best > Key::kNone ? e : -1;
#pragma unroll kUnroll
    for (int j = 0; j < kPer; ++j)
      if (j * kLanes + t == e) v[j] = Key::kNone;
  }
  return id;
}

// Gates (before `scale`) of kSlots experts that a lane holds, ids -1: none. `at`:
// their logits; most and total: of the softmax over all experts.
template <int kLanes, int kSlots>
__device__ __forceinline__ void route_gates(const RouteArgs &a, const int (&id)[kSlots],
                                            const float (&at)[kSlots], float most, float total,
                                            float (&gate)[kSlots]) {
  const float kInf = __builtin_huge_valf();
  if (!a.renormalize) {
#pragma unroll
    for (int s = 0; s < kSlots; ++s)
      gate[s] = id[s] < 0                       ? 0.0f
                : a.score == LLEP_SCORE_SOFTMAX ? expf(at[s] - most) / total
                                                : route_sigmoid(at[s]);
    return;
  }
  // over the chosen, relative to the largest of them: the sum is at least 1 however
  // small the scores are (log sigmoid(l) = min(l, 0) - log(1 + e^-|l|))
  float z[kSlots], top = -kInf, sum = 0.0f;
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    z[s] = id[s] < 0                       ? -kInf
           : a.score == LLEP_SCORE_SOFTMAX ? at[s]
                                           : fminf(at[s], 0.0f) - log1pf(expf(-fabsf(at[s])));
    top = fmaxf(top, z[s]);
  }
  top = over_row<kLanes>(top, [](float x, float y) { return fmaxf(x, y); });
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    gate[s] = id[s] < 0 ? 0.0f : expf(z[s] - top);
    sum += gate[s];
  }
  sum = row_sum<kLanes>(sum);
#pragma unroll
  for (int s = 0; s < kSlots; ++s)
    if (id[s] >= 0) gate[s] /= sum;
}

template <typename L, int kPer, int kLanes, bool kByLogit>
__global__ __launch_bounds__(kRouteThreads) void route_rounds_kernel(RouteArgs a) {
  constexpr int kRows = kRouteThreads / kLanes;
  __shared__ ExactLds<kPer, kLanes, typename RouteKey<L, kByLogit>::V> lds[kRouteThreads / kWave];
  const int t = threadIdx.x % kLanes;
  const float kInf = __builtin_huge_valf();
  const int64_t step = int64_t(gridDim.x) * kRows;
  // every lane of a wavefront takes part in the reductions, also past the end
  for (int64_t row0 = first_row<kRows, kLanes>(); row0 < a.T; row0 += step) {
    const int64_t row = row0 + lane_id() / kLanes;
    const L *logits = static_cast<const L *>(a.logits) + (row < a.T ? row : a.T - 1) * a.E;
    float l[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int e = j * kLanes + t;
      l[j] = e < a.E ? route_load(logits + e) : -kInf;
    }
    // of the softmax over all experts
    float most = -kInf, total = 0.0f;
    if (a.score == LLEP_SCORE_SOFTMAX) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) most = fmaxf(most, l[j]);
      most = over_row<kLanes>(most, [](float x, float y) { return fmaxf(x, y); });
      if (most == -kInf) most = 0.0f;  // nothing to choose from: sums of zeros, not NaN
      if (!a.renormalize) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) total += expf(l[j] - most);
        total = row_sum<kLanes>(total);
      }
    }
    const int id[1] = {pick_exact<L, kPer, kLanes, kByLogit, false>(
        a, [&](int j) { return l[j]; }, most, lds[threadIdx.x / kWave])};
    const float at[1] = {id[0] >= 0 ? route_load(logits + id[0]) : -kInf};
    float gate[1];
    route_gates<kLanes>(a, id, at, most, total, gate);
    if (row < a.T && t < a.K) {
      a.ids[row * a.K + t] = id[0];
      a.gates[row * a.K + t] = gate[0] * a.scale;
    }
  }
}

// ---------------------------------------------------------------------------
// lists: lane t of a row's kLanes holds kPer experts next to each other, of one group
// (with groups, each has 2^wide_log2 lanes, the last of which may hold fewer)
// ---------------------------------------------------------------------------

struct LaneExperts {
  int first, end;  // (first >= end: none)
};
template <int kPer>
__device__ __forceinline__ LaneExperts lane_experts(const RouteArgs &a, int t) {
  if (a.groups == 1) return {t * kPer, a.E};
  const int g = t >> a.wide_log2, in = t & ((1 << a.wide_log2) - 1);
  return {g * a.group_size + in * kPer, g < a.groups ? (g + 1) * a.group_size : 0};
}

template <typename V>
__device__ __forceinline__ void order2(V &a, V &b) {
  const V x = larger(a, b), y = smaller(a, b);
  a = x, b = y;
}
// descending, by compare-exchange networks
template <typename V>
__device__ __forceinline__ void sort_list(V (&v)[4]) {
  order2(v[0], v[1]), order2(v[2], v[3]), order2(v[0], v[2]), order2(v[1], v[3]), order2(v[1], v[2]);
}
template <typename V>
__device__ __forceinline__ void sort_list(V (&v)[8]) {
  order2(v[0], v[1]), order2(v[2], v[3]), order2(v[4], v[5]), order2(v[6], v[7]);
  order2(v[0], v[2]), order2(v[1], v[3]), order2(v[4], v[6]), order2(v[5], v[7]);
  order2(v[1], v[2]), order2(v[5], v[6]), order2(v[0], v[4]), order2(v[1], v[5]);
  order2(v[2], v[6]), order2(v[3], v[7]), order2(v[2], v[4]), order2(v[3], v[5]);
  order2(v[1], v[2]), order2(v[3], v[4]), order2(v[5], v[6]);
}
// a: the kTop largest of two descending lists, descending
template <int kTop, typename V>
__device__ __forceinline__ void merge_lists(V (&a)[kTop], const V (&b)[kTop]) {
#pragma unroll
  for (int i = 0; i < kTop; ++i) a[i] = larger(a[i], b[kTop - 1 - i]);
#pragma unroll
  for (int d = kTop / 2; d > 0; d /= 2)
#pragma unroll
    for (int i = 0; i < kTop; ++i)
      if (!(i & d)) order2(a[i], a[i + d]);
}
// the value of the lane whose number differs in one bit (1, 2, 4, 8)
template <int kBit, typename V>
__device__ __forceinline__ V partner(V v) {
  // quad_perm 1 0 3 2, 2 3 0 1; row_half_mirror and row_mirror turn 4 and 8 around as
  // well as the bits below, which are equal by then
  constexpr int kCtrl = kBit == 1 ? 0xb1 : kBit == 2 ? 0x4e : kBit == 4 ? 0x141 : 0x140;
  return rotated<kCtrl>(v);
}

// the lists of a lane's kPer keys, then of all lanes
template <int kPer, int kTop, typename V>
__device__ __forceinline__ void lane_list(const V (&key)[kPer], V none, V (&top)[kTop]) {
#pragma unroll
  for (int c = 0; c < kPer; c += kTop) {
    V v[kTop];
#pragma unroll
    for (int j = 0; j < kTop; ++j) v[j] = c + j < kPer ? key[c + j < kPer ? c + j : 0] : none;
    sort_list(v);
    if (c == 0) {
#pragma unroll
      for (int j = 0; j < kTop; ++j) top[j] = v[j];
    } else {
      merge_lists(top, v);
    }
  }
}
template <int kLanes, int kTop, typename V>
__device__ __forceinline__ void row_list(V (&top)[kTop]) {
  auto with = [&](auto bit) {
    V v[kTop];
#pragma unroll
    for (int j = 0; j < kTop; ++j) v[j] = partner<decltype(bit)::value>(top[j]);
    merge_lists(top, v);
  };
  with(std::integral_constant<int, 1>{});
  with(std::integral_constant<int, 2>{});
  if constexpr (kLanes >= 16) {
    with(std::integral_constant<int, 4>{});
    with(std::integral_constant<int, 8>{});
  }
  auto across = [&](auto k32) {  // the rows of 16, the halves
    V v[kTop];
#pragma unroll
    for (int j = 0; j < kTop; ++j) {
      const V w = top[j];
      exchange<decltype(k32)::value>(w, top[j], v[j]);
    }
    merge_lists(top, v);
  };
  if constexpr (kLanes == 64) {
    across(std::false_type{});
    across(std::true_type{});
  }
}
// a lane's kSlots of the chosen, by their places t kSlots ..
template <int kTop, int kSlots, typename V>
__device__ __forceinline__ V list_slot(const V (&top)[kTop], int t, int s, int K, V none) {
  V v = none;
#pragma unroll
  for (int k = 0; k < kTop; ++k)
    if (k == t * kSlots + s && k < K) v = top[k];
  return v;
}

// Keys that are the logits.
template <typename L, int kPer, int kLanes, int kTop>
__global__ __launch_bounds__(kRouteThreads) void route_lists_kernel(RouteArgs a) {
  using Key = RouteKey<L, true>;
  using V = typename Key::V;
  constexpr int kRows = kRouteThreads / kLanes;
  constexpr int kSlots = kTop > kLanes ? kTop / kLanes : 1;  // of the chosen, per lane
  const int t = threadIdx.x % kLanes;
  const float kInf = __builtin_huge_valf();
  const int64_t step = int64_t(gridDim.x) * kRows;
  // every lane of a wavefront takes part in the reductions, also past the end
  for (int64_t row0 = first_row<kRows, kLanes>(); row0 < a.T; row0 += step) {
    const int64_t row = row0 + lane_id() / kLanes;
    const L *logits = static_cast<const L *>(a.logits) + (row < a.T ? row : a.T - 1) * a.E;
    float l[kPer];
    const LaneExperts mine = lane_experts<kPer>(a, t);
    route_load_row<kPer>(logits, mine.first, mine.end, l);
    V key[kPer], top[kTop];
#pragma unroll
    for (int j = 0; j < kPer; ++j) key[j] = l[j] > -kInf ? Key::make(l[j], mine.first + j) : Key::kNone;
    lane_list(key, Key::kNone, top);
    if (kLanes == 16 && a.groups > 1) {
      // the best of each group, then the groups before it
      const int wide = 1 << a.wide_log2;
      V own = top[0];
      auto fold = [&](V x) { own = larger(own, x); };
      if (wide > 1) fold(partner<1>(own));
      if (wide > 2) fold(partner<2>(own));
      if (wide > 4) fold(partner<4>(own));
      int before = 0;
      V other = own;
      for (int r = 1; r < 16; ++r) {
        other = rotated<0x121>(other);  // row_ror:1
        before += other > own;
      }
      if (before >= a.top_groups * wide) {
#pragma unroll
        for (int j = 0; j < kTop; ++j) top[j] = Key::kNone;
      }
    }
    row_list<kLanes>(top);
    int id[kSlots];
    float at[kSlots], gate[kSlots];
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const V v = list_slot<kTop, kSlots>(top, t, s, a.K, Key::kNone);
      id[s] = v != Key::kNone ? Key::index(v) : -1;
      at[s] = Key::logit(v);
    }
    float most = 0.0f, total = 0.0f;
    if (a.score == LLEP_SCORE_SOFTMAX && !a.renormalize) {
      // (nothing to choose from: sums of zeros, not NaN)
      float best = -kInf;
#pragma unroll
      for (int j = 0; j < kPer; ++j) best = fmaxf(best, l[j]);
      best = over_row<kLanes>(best, [](float x, float y) { return fmaxf(x, y); });
      most = best == -kInf ? 0.0f : best;
#pragma unroll
      for (int j = 0; j < kPer; ++j) total += expf(l[j] - most);
      total = row_sum<kLanes>(total);
    }
    route_gates<kLanes>(a, id, at, most, total, gate);
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const int k = t * kSlots + s;
      if (row < a.T && k < a.K) {
        a.ids[row * a.K + k] = id[s];
        a.gates[row * a.K + k] = gate[s] * a.scale;
      }
    }
  }
}

// Keys that are sums of scores, float64, cut to 43 bits of fraction with the index
// below them (IndexedDouble). Keys nearer to each other than kDoubt, of 1 (a score is at
// most 1, and a bias rounds the sum in units of itself) or of the larger, may be in
// another order than uncut ones, or computed in another order of the softmax's sum. The
// sum of a group's two best is off by up to 2^-42 of the larger of them, cut again by as
// much, however small the sum is (a bias of +64 and one of -64): groups are told apart
// beyond 2 kDoubt of the largest key that went into either. Where keys are nearer among
// the chosen, between the last of them and any other, or between two groups, all rows of
// the wavefront go to pick_exact, unless equal logits and biases say that keys are equal.
// With random logits hardly any do (with keys in float32 ten of 8192 rows of 256 experts
// did, and the launch, of 24 us, was as long as theirs).
constexpr double kDoubt = 0x1p-40;

// 1 / d for 1 <= d, in float64 up to a rounding or two (of an infinity: not 0, but
// nothing next to what it is added to or compared with)
__device__ __forceinline__ double reciprocal(double d) {
  d = fmin(d, 1e300);
  double r = __builtin_amdgcn_rcp(d);
  r = fma(fma(-d, r, 1.0), r, r);
  return fma(fma(-d, r, 1.0), r, r);
}

template <typename L, int kPer, int kLanes, int kTop>
__global__ __launch_bounds__(kRouteThreads) void route_sums_kernel(RouteArgs a) {
  constexpr int kRows = kRouteThreads / kLanes;
  using Key = IndexedDouble;
  constexpr double kNone = Key::kNone;
  __shared__ ExactLds<kPer, kLanes, double> lds[kRouteThreads / kWave];
  int t = threadIdx.x % kLanes;
  const float kInf = __builtin_huge_valf();
  const int64_t step = int64_t(gridDim.x) * kRows;
  const bool softmax = a.score == LLEP_SCORE_SOFTMAX;
  // (without a bias: sigmoids below 1e-300, which reciprocal() does not tell apart)
  const double unit = a.bias ? 1.0 : 0x1p-900;
  auto near = [&](double x, double y) {  // neither of them none
    const double u = Key::value(x), v = Key::value(y);
    return fabs(u - v) <= kDoubt * fmax(unit, fmax(fabs(u), fabs(v)));
  };
  // of keys below x (as they are cut) those from here on
  auto lowest_near = [&](double x) { return Key::value(x) - kDoubt * fmax(unit, fabs(x)); };
  // Whether one of the lane's keys below `last` is near it without being equal. Its row is
  // read again, whole: few rows come here, but those of a router whose logits are all equal,
  // as before its training, do (8192 x 256 of them 17 us; with a load for each near key 25).
  auto another_near = [&](const double (&key)[kPer], double last, const L *logits) {
    const LaneExperts mine = lane_experts<kPer>(a, t);
    const double low = lowest_near(last);
    const int e = last != kNone ? Key::index(last) : 0;
    const float l = route_load(logits + e), b = a.bias ? a.bias[e] : 0.0f;
    float ls[kPer], bs[kPer];
    route_load_row<kPer>(logits, mine.first, mine.end, ls);
    bool found = false;
    if (a.bias) {
      route_load_row<kPer>(a.bias, mine.first, mine.end, bs);
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        found |= key[j] < last && key[j] >= low && (ls[j] != l || bs[j] != b);
    } else {
#pragma unroll
      for (int j = 0; j < kPer; ++j) found |= key[j] < last && key[j] >= low && ls[j] != l;
    }
    return found;
  };
  // every lane of a wavefront takes part in the reductions, also past the end
  for (int64_t row0 = first_row<kRows, kLanes>(); row0 < a.T; row0 += step) {
    // (hidden from the compiler, which would keep what t compares to in registers
    // from row to row)
    asm volatile("" : "+v"(t));
    const int64_t row = row0 + lane_id() / kLanes;
    const L *logits = static_cast<const L *>(a.logits) + (row < a.T ? row : a.T - 1) * a.E;
    float l[kPer], b[kPer];
    const LaneExperts mine = lane_experts<kPer>(a, t);
    route_load_row<kPer>(logits, mine.first, mine.end, l);
#pragma unroll
    for (int j = 0; j < kPer; ++j) b[j] = 0.0f;
    if (a.bias) route_load_row<kPer>(a.bias, mine.first, mine.end, b);
    float most = 0.0f, total = 0.0f;
    double s[kPer], scale = 1.0;
    if (softmax) {
      most = -kInf;
#pragma unroll
      for (int j = 0; j < kPer; ++j) most = fmaxf(most, l[j]);
      most = over_row<kLanes>(most, [](float x, float y) { return fmaxf(x, y); });
      if (most == -kInf) most = 0.0f;  // nothing to choose from: sums of zeros, not NaN
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      s[j] = exp(softmax ? double(l[j]) - double(most) : -double(l[j]));
    if (softmax) {
      double sum = 0.0;
#pragma unroll
      for (int j = 0; j < kPer; ++j) sum += s[j];
      sum = row_sum<kLanes>(sum);
      total = float(sum);
      scale = 1.0 / sum;
    } else {
#pragma unroll
      for (int j = 0; j < kPer; ++j) s[j] = reciprocal(1.0 + s[j]);
    }
    double key[kPer], top[kTop];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const double k = fma(s[j], scale, double(b[j]));
      key[j] = l[j] > -kInf && k > -__builtin_huge_val() ? Key::make(k, mine.first + j) : kNone;
    }
    lane_list(key, kNone, top);
    bool doubt = false;
    if (a.groups > 1) {
      // the two best of each group, then the groups before it
      const int wide = 1 << a.wide_log2, own_group = t >> a.wide_log2;
      double one = top[0], two = top[1];
      auto fold = [&](double x, double y) {
        two = larger(larger(two, y), smaller(one, x));
        one = larger(one, x);
      };
      if (wide > 1) fold(partner<1>(one), partner<1>(two));
      if (wide > 2) fold(partner<2>(one), partner<2>(two));
      if (wide > 4) fold(partner<4>(one), partner<4>(two));
      if (kLanes == 64 && wide > 8) fold(partner<8>(one), partner<8>(two));
      const bool both = a.group_score == LLEP_GROUP_TOP2 && two != kNone;
      double sum = Key::value(one), size = one != kNone ? fabs(sum) : 0.0;
      if (both) sum += Key::value(two), size = fmax(size, fabs(Key::value(two)));
      const double own = one != kNone ? Key::make(sum, own_group) : kNone;
      const double limit = 2.0 * kDoubt * fmax(unit, row_max<kLanes>(size));
      int before = 0;
      for (int g = 0; g < a.groups; ++g) {
        const double other = __shfl(own, g * wide, kLanes);
        before += other > own;
        // (whether the two are on both sides of the border is left to pick_exact)
        if (g != own_group && other != kNone && own != kNone)
          doubt |= fabs(Key::value(other) - Key::value(own)) <= limit;
      }
      // Pair by pair. Of 8192 rows of bfloat16 logits without a bias hundreds have two
      // groups whose two best are equal: their order is known (8192 x 160 30 -> 15 us), if
      // no other key of theirs is as near.
      if (__any(doubt)) {
        const int e = one != kNone ? Key::index(one) : 0, f = both ? Key::index(two) : 0;
        const float le = route_load(logits + e), lf = both ? route_load(logits + f) : -kInf;
        const float be = a.bias ? a.bias[e] : 0.0f, bf = a.bias && both ? a.bias[f] : 0.0f;
        const uint64_t others = __ballot(another_near(key, both ? two : one, logits));
        const int sure = ((others >> (lane_id() & -wide)) & ((1u << wide) - 1)) == 0;
        doubt = false;
        for (int g = 0; g < a.groups; ++g) {
          const double other = __shfl(own, g * wide, kLanes);
          const double most_key = fmax(unit, fmax(size, __shfl(size, g * wide, kLanes)));
          const bool equal =
              __shfl(le, g * wide, kLanes) == le && __shfl(lf, g * wide, kLanes) == lf &&
              __shfl(be, g * wide, kLanes) == be && __shfl(bf, g * wide, kLanes) == bf &&
              (__shfl(sure, g * wide, kLanes) & sure);
          if (g != own_group && other != kNone && own != kNone)
            doubt |= fabs(Key::value(other) - Key::value(own)) <= 2.0 * kDoubt * most_key && !equal;
        }
      }
      if (before >= a.top_groups) {
#pragma unroll
        for (int j = 0; j < kTop; ++j) top[j] = kNone;
#pragma unroll
        for (int j = 0; j < kPer; ++j) key[j] = kNone;
      }
    }
    row_list<kLanes>(top);
    // the lane's one of the chosen, and the next of them
    const double v = list_slot<kTop, 1>(top, t, 0, a.K, kNone);
    const double w = list_slot<kTop, 1>(top, t + 1, 0, a.K, kNone);
    if (w != kNone && near(v, w)) {
      const int e = Key::index(v), f = Key::index(w);
      doubt |= Key::value(v) != Key::value(w) || route_load(logits + e) != route_load(logits + f) ||
               (a.bias && a.bias[e] != a.bias[f]);
    }
    // the last of them, and what is as near (which may be equal to it, or hidden behind
    // one that is)
    double last = top[0];
#pragma unroll
    for (int k = 1; k < kTop; ++k)
      if (k < a.K) last = top[k];
    const double low = lowest_near(last);
    bool border = false;
#pragma unroll
    for (int j = 0; j < kPer; ++j) border |= key[j] < last && key[j] >= low;
    if (__any(border)) doubt |= another_near(key, last, logits);
    int id[1] = {v != kNone ? Key::index(v) : -1};
    if (__any(doubt)) {
      id[0] = pick_exact<L, kPer, kLanes, false, true>(
          a,
          [&](int j) {
            const int e = j * kLanes + t;
            return e < a.E ? route_load(logits + e) : -kInf;
          },
          most, lds[threadIdx.x / kWave]);
    }
    const float at[1] = {id[0] >= 0 ? route_load(logits + id[0]) : -kInf};
    float gate[1];
    route_gates<kLanes>(a, id, at, most, total, gate);
    if (row < a.T && t < a.K) {
      a.ids[row * a.K + t] = id[0];
      a.gates[row * a.K + t] = gate[0] * a.scale;
    }
  }
}

// ---------------------------------------------------------------------------
// backward: with p = gate / scale and c_k the gate's own slope,
//   renormalised   dl[e] += gate_k c_k (dg_k - sum_j p_j dg_j),   e = ids[k]
//   else           dl[e] += gate_k c_k dg_k, and of softmax
//                  dl[e] -= softmax(l)[e] sum_j gate_j dg_j for every e
// (c_k: 1 of softmax, 1 - sigmoid(l) of sigmoid). Rows are written whole. An
// expert that a row names twice gets both, in the order of k.
// ---------------------------------------------------------------------------

__device__ __forceinline__ uint16_t route_value(uint16_t, float v) { return f32_to_bf16(v); }
__device__ __forceinline__ float route_value(float, float v) { return v; }
// Lane t's j-th expert: 16 bytes of a row are a lane's, the next 16 the next lane's, so
// that the lanes of a row load and store whole pieces of it (with a lane's experts next
// to each other 32768 x 256 in float32 took 17 us for 12).
template <typename L, int kPer, int kLanes>
struct RowPieces {
  static constexpr int kVec = kPer < int(16 / sizeof(L)) ? kPer : int(16 / sizeof(L));
  typedef L vec __attribute__((ext_vector_type(kVec), aligned(sizeof(L))));
  static __device__ __forceinline__ int expert(int t, int j) {
    return (j / kVec * kLanes + t) * kVec + j % kVec;
  }
  static __device__ __forceinline__ void load(const L *row, int t, int E, float (&x)[kPer]) {
#pragma unroll
    for (int c = 0; c < kPer; c += kVec) {
      const int e = expert(t, c);
      if (e + kVec <= E) {
        const vec v = *reinterpret_cast<const vec *>(row + e);
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
          const L y = v[j];
          x[c + j] = route_load(&y);
        }
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
          x[c + j] = e + j < E ? route_load(row + e + j) : -__builtin_huge_valf();
      }
    }
  }
  static __device__ __forceinline__ void store(L *row, int t, int E, const float (&x)[kPer]) {
#pragma unroll
    for (int c = 0; c < kPer; c += kVec) {
      const int e = expert(t, c);
      if (e + kVec <= E) {
        vec v;
#pragma unroll
        for (int j = 0; j < kVec; ++j) v[j] = route_value(L{}, x[c + j]);
        *reinterpret_cast<vec *>(row + e) = v;
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
          if (e + j < E) row[e + j] = route_value(L{}, x[c + j]);
      }
    }
  }
};

template <typename L, int kPer, int kLanes>
__global__ __launch_bounds__(kRouteThreads) void route_backward_kernel(RouteArgs a) {
  using Row = RowPieces<L, kPer, kLanes>;
  constexpr int kRows = kRouteThreads / kLanes;
  const int t = threadIdx.x % kLanes;
  const float kInf = __builtin_huge_valf();
  const int64_t step = int64_t(gridDim.x) * kRows;
  const bool full = a.score == LLEP_SCORE_SOFTMAX && !a.renormalize;
  for (int64_t row0 = first_row<kRows, kLanes>(); row0 < a.T; row0 += step) {
    const int64_t at = row0 + lane_id() / kLanes;
    const int64_t row = at < a.T ? at : a.T - 1;
    const L *logits = static_cast<const L *>(a.logits) + row * a.E;
    int id = -1;
    float gate = 0.0f, dg = 0.0f;
    if (t < a.K) {
      id = a.ids[row * a.K + t];
      gate = a.gates[row * a.K + t];
      dg = a.d_gates[row * a.K + t];
      if (uint32_t(id) >= uint32_t(a.E)) id = -1, gate = dg = 0.0f;
    }
    float out[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) out[j] = 0.0f;
    float each = gate * dg;
    const float sum = a.renormalize || full ? row_sum<kLanes>(each) : 0.0f;
    if (a.renormalize) each = id >= 0 ? gate * (dg - sum / a.scale) : 0.0f;
    if (a.score == LLEP_SCORE_SIGMOID && id >= 0) each *= route_sigmoid(-route_load(logits + id));
    if (full) {
      float most = -kInf, total = 0.0f;
      Row::load(logits, t, a.E, out);
#pragma unroll
      for (int j = 0; j < kPer; ++j) most = fmaxf(most, out[j]);
      most = over_row<kLanes>(most, [](float x, float y) { return fmaxf(x, y); });
      if (most == -kInf) most = 0.0f;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        out[j] = expf(out[j] - most);
        total += out[j];
      }
      total = row_sum<kLanes>(total);
      const float c = total > 0.0f || total != total ? sum / total : 0.0f;
#pragma unroll
      for (int j = 0; j < kPer; ++j) out[j] *= -c;
    }
    for (int k = 0; k < a.K; ++k) {
      const int e = __shfl(id, k, kLanes);
      const float d = __shfl(each, k, kLanes);
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (Row::expert(t, j) == e) out[j] += d;
    }
    if (at < a.T) Row::store(static_cast<L *>(a.d_logits) + row * a.E, t, a.E, out);
  }
}

// ---------------------------------------------------------------------------
// launch
// ---------------------------------------------------------------------------

template <int kLanes>
dim3 route_grid(const RouteArgs &a) {
  constexpr int kRows = kRouteThreads / kLanes;
  return dim3(uint32_t(std::min<int64_t>((a.T + kRows - 1) / kRows, 256 * 8)));
}

template <typename L, int kPer, int kLanes>
hipError_t run_rounds(const RouteArgs &a, bool backward, bool sum, hipStream_t stream) {
  const dim3 grid = route_grid<kLanes>(a), threads(kRouteThreads);
  if (backward)
    hipLaunchKernelGGL((route_backward_kernel<L, kPer, kLanes>), grid, threads, 0, stream, a);
  else if (sum)
    hipLaunchKernelGGL((route_rounds_kernel<L, kPer, kLanes, false>), grid, threads, 0, stream, a);
  else
    hipLaunchKernelGGL((route_rounds_kernel<L, kPer, kLanes, true>), grid, threads, 0, stream, a);
  return hipGetLastError();
}

template <typename L, int kPer, int kLanes, int kTop, bool kSum>
hipError_t run_lists(const RouteArgs &a, hipStream_t stream) {
  const dim3 grid = route_grid<kLanes>(a), threads(kRouteThreads);
  if constexpr (kSum)
    hipLaunchKernelGGL((route_sums_kernel<L, kPer, kLanes, kTop>), grid, threads, 0, stream, a);
  else
    hipLaunchKernelGGL((route_lists_kernel<L, kPer, kLanes, kTop>), grid, threads, 0, stream, a);
  return hipGetLastError();
}
// lanes of 8, 16 or 32 experts, or (64 lanes) 2, 4 or 8
template <typename L, int kLanes, int kTop, bool kSum>
hipError_t lists_per(const RouteArgs &a, int per, hipStream_t stream) {
  if constexpr (kLanes == 64) {
    if (per == 2) return run_lists<L, 2, 64, kTop, kSum>(a, stream);
    if (per == 4) return run_lists<L, 4, 64, kTop, kSum>(a, stream);
    return run_lists<L, 8, 64, kTop, kSum>(a, stream);
  } else {
    if (per == 8) return run_lists<L, 8, kLanes, kTop, kSum>(a, stream);
    if (per == 16) return run_lists<L, 16, kLanes, kTop, kSum>(a, stream);
    return run_lists<L, 32, kLanes, kTop, kSum>(a, stream);
  }
}

template <typename L, int kLanes, bool kSum>
hipError_t lists_top(const RouteArgs &a, int per, hipStream_t stream) {
  return a.K <= 4 ? lists_per<L, kLanes, 4, kSum>(a, per, stream)
                  : lists_per<L, kLanes, 8, kSum>(a, per, stream);
}
// Experts of a lane (and a group's lanes, into `a`), 0: the groups do not fit.
static int list_shape(RouteArgs &a, int lanes) {
  const int least = lanes == 64 ? 2 : 8, most = lanes == 64 ? 16 : 8;  // lanes of a group
  int held = lanes;
  if (a.groups > 1) {
    if (a.groups > lanes) return 0;
    while (a.wide_log2 < 6 && (2 << a.wide_log2) * a.groups <= lanes && (2 << a.wide_log2) <= most &&
           (least << a.wide_log2) < a.group_size)
      ++a.wide_log2;
    held = 1 << a.wide_log2;
  }
  int per = least;
  while (per < 4 * least && per * held < a.group_size) per *= 2;
  return per * held >= a.group_size ? per : 0;
}

template <typename L>
hipError_t route_t(const RouteArgs &a, bool backward, hipStream_t stream) {
  static_assert(LLEP_MAX_EXPERTS == 512 && LLEP_MAX_ROUTE_TOPK == 64, "a row fits a wavefront");
  const bool sum = a.bias || (a.groups > 1 && a.group_score == LLEP_GROUP_TOP2);
  // Lanes for a row: more for few rows. Sums, 64 / 16 lanes: 1024 x 256 with groups
  // 6.7 / 8.2 us, 2048 8.3 / 8.4, 4096 12.4 / 8.6, 1024 x 512 5.9 / 9.0, 4096 12.6 / 9.5.
  // Logits, 16 / 4 lanes: 8192 x 128 bf16 4.1 / 4.6, 16384 5.7 / 4.8, 32768 8.6 / 6.1, but
  // 4096 x 32 3.4 / 3.0. (More than 8 experts of 128, 64 / 16: 2048 rows 4.8 / 5.1, 4096
  // 6.5 / 5.3; the gradient of 8 of 128: 4096 3.4 / 3.6, 8192 4.2 / 3.7.)
  if (!backward && a.K <= 8) {
    const bool few = sum && a.T <= 1024;
    const int lanes = few                                                         ? 64
                      : sum || (a.T < 12288 && a.E > 32) || a.E > 128 || a.groups > 1 ? 16
                                                                                      : 4;
    // (64 lanes hold 8 experts each at most, which few large groups do not fit)
    for (int n : {lanes, few ? 16 : lanes}) {
      RouteArgs b = a;
      const int per = list_shape(b, n);
      if (per == 0) continue;
      if (n == 64)
        return lists_top<L, 64, true>(b, per, stream);
      if (n == 4) return lists_top<L, 4, false>(b, per, stream);
      return sum ? lists_top<L, 16, true>(b, per, stream) : lists_top<L, 16, false>(b, per, stream);
    }
  }
  if (a.T <= (backward ? 4096 : 2048) || a.K > 16) {
    if (a.E <= 64) return run_rounds<L, 1, 64>(a, backward, sum, stream);
    if (a.E <= 128) return run_rounds<L, 2, 64>(a, backward, sum, stream);
    if (a.E <= 256) return run_rounds<L, 4, 64>(a, backward, sum, stream);
    return run_rounds<L, 8, 64>(a, backward, sum, stream);
  }
  if (a.E <= 32) return run_rounds<L, 2, 16>(a, backward, sum, stream);
  if (a.E <= 64) return run_rounds<L, 4, 16>(a, backward, sum, stream);
  if (a.E <= 128) return run_rounds<L, 8, 16>(a, backward, sum, stream);
  if (a.E <= 256) return run_rounds<L, 16, 16>(a, backward, sum, stream);
  return run_rounds<L, 32, 16>(a, backward, sum, stream);
}

hipError_t launch_route(const RouteArgs &a, bool backward, hipStream_t stream) {
  if (a.T == 0) return hipSuccess;
  RouteArgs b = a;
  b.group_size = a.E / a.groups;
  b.wide_log2 = 0;
  return a.dtype == LLEP_BF16 ? route_t<uint16_t>(b, backward, stream)
                              : route_t<float>(b, backward, stream);
}

}  // namespace llep
