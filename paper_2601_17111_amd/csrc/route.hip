// Routing of tokens to experts (llep_route) and its gradient
// (llep_route_backward).
//
// A row of E logits belongs to kLanes lanes of a wavefront (16: four rows per
// wavefront; 64), lane t holding the experts j kLanes + t, j < kPer, in
// registers: read once, and neither the scores nor the keys go to memory. The K
// best are taken one after another, each by a maximum over the row's lanes.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "rows.h"

namespace llep {

constexpr int kRouteThreads = 256;

// ---------------------------------------------------------------------------
// reductions over the lanes of a row, the result in each of them: rotations
// within 16 lanes, then exchanges between the rows of 16
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
  v = op(v, rotated<0x121>(v));  // row_ror:1, :2, :4, :8
  v = op(v, rotated<0x122>(v));
  v = op(v, rotated<0x124>(v));
  v = op(v, rotated<0x128>(v));
  if constexpr (kLanes == 64) {
    V a, b;
    exchange<false>(v, a, b);
    v = op(a, b);
    exchange<true>(v, a, b);
    v = op(a, b);
  }
  return v;
}
template <int kLanes, typename V>
__device__ __forceinline__ V row_max(V v) {
  return over_row<kLanes>(v, [](V a, V b) { return a > b ? a : b; });
}
template <int kLanes, typename V>
__device__ __forceinline__ V row_sum(V v) {
  return over_row<kLanes>(v, [](V a, V b) { return a + b; });
}

__device__ __forceinline__ float route_load(const uint16_t *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float route_load(const float *p) { return *p; }

// ---------------------------------------------------------------------------
// keys
//
// What is only ordered (kByLogit) is ordered by the logits themselves, packed
// with the expert's index below them, so that one maximum finds the largest and
// of equal ones the first: bfloat16 logits in 32 bits, float32 logits in 64.
// Where scores are added up (with the bias, or two of a group) the key is that
// sum in float64: scores a rounding apart are not told apart in 32 bits, and
// the choice would depend on the instruction that computed them. 0 (and, of
// float64, -infinity): not to be taken.
// ---------------------------------------------------------------------------

// the float's bits in its order, above 0 for all but NaN with the sign set
__device__ __forceinline__ uint32_t ordered(float f) {
  f += 0.0f;  // -0 is equal to 0
  const uint32_t u = __float_as_uint(f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

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
};
template <>
struct RouteKey<float, true> {
  using V = uint64_t;
  static constexpr V kNone = 0;
  static __device__ __forceinline__ V make(float l, int e) {
    return (uint64_t(ordered(l)) << 32) | uint32_t(0xffff - e);
  }
  static __device__ __forceinline__ int index(V v) { return 0xffff - int(uint32_t(v)); }
};
template <typename L>
struct RouteKey<L, false> {
  using V = double;
  static constexpr V kNone = -__builtin_huge_val();
};

// 1 / (1 + e^-l)
__device__ __forceinline__ float route_sigmoid(float l) { return 1.0f / (1.0f + expf(-l)); }

template <typename L, int kPer, int kLanes, bool kByLogit>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(RouteArgs a) {
  using Key = RouteKey<L, kByLogit>;
  using V = typename Key::V;
  constexpr int kRows = kRouteThreads / kLanes;
  constexpr int kSlots = 64 / kLanes;  // groups per lane
  __shared__ V keys[kRows][kPer * kLanes];
  __shared__ V scores[kRows][64];
  const int t = threadIdx.x % kLanes, mine = threadIdx.x / kLanes;
  const int lane = lane_id();
  const float kInf = __builtin_huge_valf();
  const int size = a.E / a.groups;
  const float per = 1.0f / float(size);
  const int64_t step = int64_t(gridDim.x) * kRows;
  // every lane of a wavefront takes part in the reductions, also past the end
  const int64_t rounds = (a.T + step - 1) / step;
  for (int64_t it = 0; it < rounds; ++it) {
    const int64_t row = it * step + int64_t(blockIdx.x) * kRows + mine;
    const L *logits = static_cast<const L *>(a.logits) + (row < a.T ? row : a.T - 1) * a.E;
    float l[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int e = j * kLanes + t;
      l[j] = e < a.E ? route_load(logits + e) : -kInf;
    }
    // maximum and sum of the softmax over all experts
    float most = -kInf, total = 0.0f;
    const bool full = a.score == LLEP_SCORE_SOFTMAX && (!kByLogit || !a.renormalize);
    if (full) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) most = fmaxf(most, l[j]);
      most = over_row<kLanes>(most, [](float x, float y) { return fmaxf(x, y); });
      if (most == -kInf) most = 0.0f;  // nothing to choose from: sums of zeros, not NaN
    }
    V v[kPer];
    if constexpr (kByLogit) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const int e = j * kLanes + t;
        v[j] = l[j] > -kInf ? Key::make(l[j], e) : Key::kNone;
      }
      if (full) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) total += expf(l[j] - most);
        total = row_sum<kLanes>(total);
      }
    } else {
      double wide = 0.0;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const double x = l[j];
        v[j] = a.score == LLEP_SCORE_SOFTMAX ? exp(x - double(most)) : 1.0 / (1.0 + exp(-x));
        wide += v[j];
      }
      if (a.score == LLEP_SCORE_SOFTMAX) {
        wide = row_sum<kLanes>(wide);
        total = float(wide);
      }
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const int e = j * kLanes + t;
        if (a.score == LLEP_SCORE_SOFTMAX) v[j] /= wide;
        if (a.bias) v[j] += double(e < a.E ? a.bias[e] : 0.0f);
        // (a key that is NaN is not above -infinity either)
        if (!(l[j] > -kInf) || !(v[j] > Key::kNone)) v[j] = Key::kNone;
      }
    }
    if (a.groups > 1) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kPer; ++j) keys[mine][j * kLanes + t] = v[j];
      __syncthreads();
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int g = s * kLanes + t;
        if (g >= a.groups) break;
        V one = Key::kNone, two = Key::kNone;
        int i = t % size;  // from lane to lane other banks
        for (int n = 0; n < size; ++n) {
          const V k = keys[mine][g * size + i];
          two = k > one ? one : k > two ? k : two;
          one = k > one ? k : one;
          i = i + 1 == size ? 0 : i + 1;
        }
        if constexpr (!kByLogit)
          if (a.group_score == LLEP_GROUP_TOP2 && two > Key::kNone) one += two;
        scores[mine][g] = one;
      }
      __syncthreads();
      uint64_t keep = 0;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int g = s * kLanes + t;
        bool in = g < a.groups;
        if (in) {
          const V own = scores[mine][g];
          int before = 0;
          for (int h = 0; h < a.groups; ++h) {
            const V k = scores[mine][h];
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
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        // e / size (the quotient's distance from a whole number is at least
        // 1 / (2 size), far above its rounding)
        const int g = int((float(j * kLanes + t) + 0.5f) * per);
        if (g < 64 && !((keep >> g) & 1)) v[j] = Key::kNone;
      }
    }
    // the K best: lane k of the row keeps the k-th
    int id = -1;
    for (int k = 0; k < a.K; ++k) {
      V best = v[0];
#pragma unroll
      for (int j = 1; j < kPer; ++j) best = v[j] > best ? v[j] : best;
      best = row_max<kLanes>(best);
      int e;
      if constexpr (kByLogit) {
        e = Key::index(best);
      } else {
        uint32_t first = 0xffff;
#pragma unroll
        for (int j = kPer - 1; j >= 0; --j)
          if (v[j] == best) first = uint32_t(j * kLanes + t);
        e = int(over_row<kLanes>(first, [](uint32_t x, uint32_t y) { return min(x, y); }));
      }
      const bool found = best > Key::kNone;
      if (t == k) id = found ? e : -1;
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (j * kLanes + t == e) v[j] = Key::kNone;
    }
    // gates of the lanes that hold an expert
    const float at = id >= 0 ? route_load(logits + id) : -kInf;
    float gate = 0.0f;
    if (a.score == LLEP_SCORE_SOFTMAX && !a.renormalize) {
      if (id >= 0) gate = expf(at - most) / total;
    } else if (!a.renormalize) {
      if (id >= 0) gate = route_sigmoid(at);
    } else {
      // over the chosen, relative to the largest of them: the sum is at least 1
      // however small the scores are (log sigmoid(l) = min(l, 0) - log(1 + e^-|l|))
      const float z = a.score == LLEP_SCORE_SOFTMAX ? at
                      : id >= 0 ? fminf(at, 0.0f) - log1pf(expf(-fabsf(at)))
                                : -kInf;
      const float top = over_row<kLanes>(z, [](float x, float y) { return fmaxf(x, y); });
      const float p = id >= 0 ? expf(z - top) : 0.0f;
      const float sum = row_sum<kLanes>(p);
      if (id >= 0) gate = p / sum;
    }
    if (row < a.T && t < a.K) {
      a.ids[row * a.K + t] = id;
      a.gates[row * a.K + t] = gate * a.scale;
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

__device__ __forceinline__ void route_store(uint16_t *p, float v) { *p = f32_to_bf16(v); }
__device__ __forceinline__ void route_store(float *p, float v) { *p = v; }

template <typename L, int kPer, int kLanes>
__global__ __launch_bounds__(kRouteThreads) void route_backward_kernel(RouteArgs a) {
  constexpr int kRows = kRouteThreads / kLanes;
  const int t = threadIdx.x % kLanes, mine = threadIdx.x / kLanes;
  const float kInf = __builtin_huge_valf();
  const int64_t step = int64_t(gridDim.x) * kRows;
  const int64_t rounds = (a.T + step - 1) / step;
  const bool full = a.score == LLEP_SCORE_SOFTMAX && !a.renormalize;
  for (int64_t it = 0; it < rounds; ++it) {
    const int64_t at = it * step + int64_t(blockIdx.x) * kRows + mine;
    const int64_t row = at < a.T ? at : a.T - 1;
    const L *logits = static_cast<const L *>(a.logits) + row * a.E;
    int id = -1;
    float gate = 0.0f, dg = 0.0f;
    if (t < a.K) {
      id = a.ids[row * a.K + t];
      if (uint32_t(id) >= uint32_t(a.E)) id = -1;
      if (id >= 0) {
        gate = a.gates[row * a.K + t];
        dg = a.d_gates[row * a.K + t];
      }
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
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const int e = j * kLanes + t;
        out[j] = e < a.E ? route_load(logits + e) : -kInf;
        most = fmaxf(most, out[j]);
      }
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
        if (j * kLanes + t == e) out[j] += d;
    }
    L *d_logits = static_cast<L *>(a.d_logits) + row * a.E;
    if (at < a.T)
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const int e = j * kLanes + t;
        if (e < a.E) route_store(d_logits + e, out[j]);
      }
  }
}

// ---------------------------------------------------------------------------
// launch
// ---------------------------------------------------------------------------

template <typename L, int kPer, int kLanes>
hipError_t run_route(const RouteArgs &a, bool backward, hipStream_t stream) {
  constexpr int kRows = kRouteThreads / kLanes;
  const int64_t wgs = (a.T + kRows - 1) / kRows;
  const dim3 grid(uint32_t(std::min<int64_t>(wgs, 256 * 8)));
  if (backward)
    hipLaunchKernelGGL((route_backward_kernel<L, kPer, kLanes>), grid, dim3(kRouteThreads), 0,
                       stream, a);
  else if (a.bias || (a.groups > 1 && a.group_score == LLEP_GROUP_TOP2))
    hipLaunchKernelGGL((route_kernel<L, kPer, kLanes, false>), grid, dim3(kRouteThreads), 0,
                       stream, a);
  else
    hipLaunchKernelGGL((route_kernel<L, kPer, kLanes, true>), grid, dim3(kRouteThreads), 0, stream,
                       a);
  return hipGetLastError();
}

template <typename L>
hipError_t route_t(const RouteArgs &a, bool backward, hipStream_t stream) {
  static_assert(LLEP_MAX_EXPERTS == 512 && LLEP_MAX_ROUTE_TOPK == 64, "a row fits a wavefront");
  if (a.T <= 4096 || a.K > 16) {
    if (a.E <= 64) return run_route<L, 1, 64>(a, backward, stream);
    if (a.E <= 128) return run_route<L, 2, 64>(a, backward, stream);
    if (a.E <= 256) return run_route<L, 4, 64>(a, backward, stream);
    return run_route<L, 8, 64>(a, backward, stream);
  }
  if (a.E <= 32) return run_route<L, 2, 16>(a, backward, stream);
  if (a.E <= 64) return run_route<L, 4, 16>(a, backward, stream);
  if (a.E <= 128) return run_route<L, 8, 16>(a, backward, stream);
  if (a.E <= 256) return run_route<L, 16, 16>(a, backward, stream);
  return run_route<L, 32, 16>(a, backward, stream);
}

hipError_t launch_route(const RouteArgs &a, bool backward, hipStream_t stream) {
  if (a.T == 0) return hipSuccess;
  return a.dtype == LLEP_BF16 ? route_t<uint16_t>(a, backward, stream)
                              : route_t<float>(a, backward, stream);
}

}  // namespace llep
