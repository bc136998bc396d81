// Rows held in registers: what the kernels that work row by row share (block
// norms, 8-bit rows). A row of D elements belongs to n threads, a workgroup of
// just as many wavefronts as cover it, or one wavefront of four; thread t
// holds the kPer vectors of kVec elements at (j n + t) kVec, j < kPer.
// Everything a row needs is read once; sums over it are of 32 bits or more.
#pragma once

#include <type_traits>

#include "common.h"

namespace llep {

// Threads for a row: a wavefront per 64 kPer vectors. Rows of one wavefront
// share workgroups of four (no barriers between them).
constexpr int kRowWaves = 4;
inline int row_threads(int32_t D, int vec, int per) {
  return (D + kWave * vec * per - 1) / (kWave * vec * per) * kWave;
}

// One vector of kVec elements as floats (8: 16-byte accesses, rows that start
// on 16-byte boundaries and are whole vectors; 1: any row).
template <typename T, int kVec>
__device__ __forceinline__ void load_vec(const T *p, float (&v)[kVec]) {
  if constexpr (kVec == 1) {
    if constexpr (sizeof(T) == 2)
      v[0] = bf16_to_f32(*p);
    else
      v[0] = *p;
  } else if constexpr (sizeof(T) == 2) {
    static_assert(kVec == 8, "16-byte vectors");
    const i32x4 q = *reinterpret_cast<const i32x4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(uint32_t(q[i]) << 16);
      v[2 * i + 1] = __uint_as_float(uint32_t(q[i]) & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int h = 0; h < kVec / 4; ++h) {
      const f32x4 q = *reinterpret_cast<const f32x4 *>(p + 4 * h);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * h + i] = q[i];
    }
  }
}

// 16 bytes that are aligned to their elements alone.
typedef int32_t i32x4_by2 __attribute__((ext_vector_type(4), aligned(2)));
typedef int32_t i32x4_by4 __attribute__((ext_vector_type(4), aligned(4)));

// The same vector as it lies in memory, for rows that are read ahead of their
// use, and as floats.
template <typename T, int kVec>
struct RawVec {
  static constexpr int kElems = kVec;
  static constexpr int kWords = kVec == 1 ? 1 : int(sizeof(T)) * kVec / 16;
  using Word = std::conditional_t<kVec == 1, T, i32x4>;
  Word w[kWords];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = Word{};
  }
  __device__ __forceinline__ void load(const T *p) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const Word *>(p)[i];
  }
  // of a row that starts anywhere (the compiler knows the vectors aligned to
  // their elements alone): the first `left` elements, the others 0
  __device__ __forceinline__ void load_any(const T *p, int left) {
    static_assert(kVec == 8, "whole vectors, or a row's end");
    using any = std::conditional_t<sizeof(T) == 2, i32x4_by2, i32x4_by4>;
    if (left >= kVec) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const any *>(p)[i];
      return;
    }
    zero();
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (i < left) {
        if constexpr (sizeof(T) == 2)
          w[0][i / 2] |= int32_t(uint32_t(p[i]) << (16 * (i & 1)));
        else
          w[i / 4][i % 4] = __float_as_int(p[i]);
      }
  }
  __device__ __forceinline__ float operator[](int i) const {  // i: known when compiled
    if constexpr (kVec == 1) {
      if constexpr (sizeof(T) == 2)
        return bf16_to_f32(w[0]);
      else
        return w[0];
    } else if constexpr (sizeof(T) == 2) {
      const uint32_t u = uint32_t(w[0][i / 2]);
      return __uint_as_float(i & 1 ? u & 0xffff0000u : u << 16);
    } else {
      return __int_as_float(w[i / 4][i % 4]);
    }
  }
};

template <typename T, int kVec>
__device__ __forceinline__ void store_vec(T *p, const float (&v)[kVec]) {
  if constexpr (kVec == 1) {
    if constexpr (sizeof(T) == 2)
      *p = f32_to_bf16(v[0]);
    else
      *p = v[0];
  } else if constexpr (sizeof(T) == 2) {
    i32x4 q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = int32_t(pack_bf16x2(v[2 * i], v[2 * i + 1]));
    *reinterpret_cast<i32x4 *>(p) = q;
  } else {
#pragma unroll
    for (int h = 0; h < kVec / 4; ++h) {
      const f32x4 q = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
      *reinterpret_cast<f32x4 *>(p + 4 * h) = q;
    }
  }
}

// The same for a row that starts anywhere: the first `left` elements.
template <typename T, int kVec>
__device__ __forceinline__ void store_any(T *p, const float (&v)[kVec], int left) {
  using any = std::conditional_t<sizeof(T) == 2, i32x4_by2, i32x4_by4>;
  if (left >= kVec) {
    if constexpr (sizeof(T) == 2) {
      i32x4 q;
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = int32_t(pack_bf16x2(v[2 * i], v[2 * i + 1]));
      *reinterpret_cast<any *>(p) = q;
    } else {
#pragma unroll
      for (int h = 0; h < kVec / 4; ++h)
        reinterpret_cast<any *>(p)[h] =
            i32x4{__float_as_int(v[4 * h]), __float_as_int(v[4 * h + 1]),
                  __float_as_int(v[4 * h + 2]), __float_as_int(v[4 * h + 3])};
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    if (i < left) {
      const float x[1] = {v[i]};
      store_vec<T, 1>(p + i, x);
    }
}

// v of the lane that the DPP control names, or 0 where there is none
template <int kCtrl, int kRowMask>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), kCtrl, kRowMask, 0xf, false));
}
template <int kCtrl, int kRowMask>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(dpp<kCtrl, kRowMask>(__float_as_uint(v)));
}
template <int kCtrl, int kRowMask>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t(dpp<kCtrl, kRowMask>(uint32_t(u >> 32))) << 32) |
                                        dpp<kCtrl, kRowMask>(uint32_t(u)));
}
__device__ __forceinline__ uint32_t read_lane(uint32_t v, int lane) {
  return uint32_t(__builtin_amdgcn_readlane(int(v), lane));
}
__device__ __forceinline__ float read_lane(float v, int lane) {
  return __uint_as_float(read_lane(__float_as_uint(v), lane));
}
__device__ __forceinline__ double read_lane(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t(read_lane(uint32_t(u >> 32), lane)) << 32) |
                                        read_lane(uint32_t(u), lane));
}

// Sum (or, of unsigned integers, maximum) over the wavefront's first 16 lanes
// (kAll false) or all 64, in every lane and always in the same order: shifts
// within the rows of 16 lanes, then from row to row. 0 is neutral for both.
template <bool kAll, int N, typename V, class Op>
__device__ __forceinline__ void wave_reduce(V (&v)[N], Op op) {
#define LLEP_DPP_STEP(ctrl, rows) \
  _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = op(v[i], dpp<ctrl, rows>(v[i]));
  LLEP_DPP_STEP(0x111, 0xf)  // row_shr:1, :2, :4, :8
  LLEP_DPP_STEP(0x112, 0xf)
  LLEP_DPP_STEP(0x114, 0xf)
  LLEP_DPP_STEP(0x118, 0xf)
  if constexpr (kAll) {
    LLEP_DPP_STEP(0x142, 0xa)  // row_bcast:15, :31
    LLEP_DPP_STEP(0x143, 0xc)
  }
#undef LLEP_DPP_STEP
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = read_lane(v[i], kAll ? 63 : 15);
}

// Sums and maxima over the wavefronts of a workgroup (at most 16) or, with
// kOne, over one wavefront; the same in every thread and on every run. The LDS
// halves alternate from one reduction to the next: a half is written again
// only after the barrier of the reduction between.
template <bool kOne>
struct RowReduce {
  static constexpr int kMost = 4;  // values per reduction
  static constexpr int kLds = kOne ? 1 : 2 * 16 * kMost;  // of 8 bytes
  double *lds;
  int half = 0;
  __device__ __forceinline__ explicit RowReduce(double *lds_) : lds(lds_) {}

  template <int N, typename V, class Op>
  __device__ __forceinline__ void reduce(V (&v)[N], Op op) {
    static_assert(N <= kMost, "room in LDS");
    wave_reduce<true>(v, op);
    if constexpr (!kOne) {
      V *s = reinterpret_cast<V *>(lds + half * 16 * kMost);
      half ^= 1;
      const int lane = lane_id(), waves = blockDim.x / kWave;
      if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i * 16 + threadIdx.x / kWave] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = lane < waves ? s[i * 16 + (lane & 15)] : V(0);
      wave_reduce<false>(v, op);
    }
  }
  template <int N, typename V>
  __device__ __forceinline__ void sum(V (&v)[N]) {
    reduce(v, [](V a, V b) { return a + b; });
  }
  // the largest by the bits of non-negative floats: NaN above infinity
  __device__ __forceinline__ float max_bits(uint32_t bits) {
    uint32_t x[1] = {bits};
    reduce(x, [](uint32_t a, uint32_t b) { return max(a, b); });
    return __uint_as_float(x[0]);
  }
};

// ---------------------------------------------------------------------------
// 8-bit rows: q = rint(v * (127 * (1 / max|v|))), scale = max|v| * (1 / 127),
// each step rounded to 32 bits; q * scale stands for v. A row whose largest magnitude is below
// 2^-120 (the reciprocal would leave the range) counts as zero: scale and q
// are 0. A row with an infinity or a NaN gets the scale NaN and q = 0, so that
// everything computed from it is NaN.
// ---------------------------------------------------------------------------

struct RowScale {
  float scale, inv;
};

__device__ __forceinline__ RowScale row_scale(float most) {
  if (__float_as_uint(most) >= 0x7f800000u) return {__uint_as_float(0x7fc00000u), 0.0f};
  if (most < 0x1p-120f) return {0.0f, 0.0f};
  return {most * (1.0f / 127.0f), 127.0f * (1.0f / most)};
}

// Four at a time. v inv + 1.5 * 2^23 has rint(v inv) in its low byte (the sum
// is rounded to a whole number, ties to even; the product is rounded before it,
// so the two are not contracted). At most 127: inv is rounded once.
__device__ __forceinline__ uint32_t quantize4(const float *v, float inv) {
#pragma clang fp contract(off)
  uint32_t q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float p = v[i] * inv;
    q[i] = __float_as_uint(p + 12582912.0f);
  }
  // bytes 0 of each: v_perm_b32 picks from (second operand: 0-3, first: 4-7)
  const uint32_t lo = __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400u);
  const uint32_t hi = __builtin_amdgcn_perm(q[3], q[2], 0x04000c0cu);
  return lo | hi;
}

// The vectors of thread t of n of an 8-bit row of `bytes` bytes (a multiple of
// 64): elements from D on are zero.
template <int kVec, int kPer>
__device__ __forceinline__ void store_int8_row(int8_t *row, int32_t D, int32_t bytes, int t, int n,
                                               const float (&v)[kPer][kVec], RowScale s) {
  static_assert(kVec == 8, "whole vectors");
  const bool zero = s.inv == 0.0f;  // whatever the values are
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int c = (j * n + t) * kVec;
    if (c < D)  // (8-bit rows are whole vectors; values from D on are 0)
      *reinterpret_cast<uint2 *>(row + c) =
          make_uint2(zero ? 0u : quantize4(v[j], s.inv), zero ? 0u : quantize4(v[j] + 4, s.inv));
  }
  for (int c = (D + 7) / 8 * 8 + t; c < bytes; c += n) row[c] = 0;
}

}  // namespace llep
