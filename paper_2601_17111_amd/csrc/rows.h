// Rows held in registers: what the kernels that work row by row share (block
// norms, 8-bit rows). A row of D elements belongs to kThreads threads (a
// wavefront, or a whole workgroup); thread t holds the kPer vectors of kVec
// elements at (j * kThreads + t) * kVec, j < kPer, as floats. Everything a
// row needs is read once; sums over it are of 32 bits or more.
#pragma once

#include "common.h"

namespace llep {

constexpr int kRowWg = 256;  // threads of a workgroup that works on one row per wavefront

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

// Sums and maxima over the threads of a row, the same in every thread and on
// every run. The LDS halves alternate from one reduction to the next: a half
// is written again only after the barrier of the reduction between.
template <int kThreads, typename V = float>
struct RowReduce {
  static constexpr int kWaves = kThreads / kWave;
  static constexpr int kMost = 4;  // values per reduction
  static constexpr int kLds = kWaves > 1 ? 2 * kWaves * kMost : 1;
  V *lds;
  int half = 0;
  __device__ __forceinline__ explicit RowReduce(V *lds_) : lds(lds_) {}

  template <int N, class Op>
  __device__ __forceinline__ void reduce(V (&v)[N], Op op) {
    static_assert(N <= kMost, "room in LDS");
#pragma unroll
    for (int o = kWave / 2; o >= 1; o >>= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = op(v[i], __shfl_xor(v[i], o));
    if constexpr (kWaves > 1) {
      V *s = lds + half * kWaves * kMost;
      half ^= 1;
      if (lane_id() == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) s[threadIdx.x / kWave * kMost + i] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = s[i];
      for (int w = 1; w < kWaves; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = op(v[i], s[w * kMost + i]);
    }
  }
  template <int N>
  __device__ __forceinline__ void sum(V (&v)[N]) {
    reduce(v, [](V a, V b) { return a + b; });
  }
  // the largest by the bits of non-negative floats: NaN above infinity
  __device__ __forceinline__ float max_bits(float v) {
    float x[1] = {v};
    reduce(x, [](float a, float b) {
      return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
    });
    return x[0];
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

__device__ __forceinline__ int32_t quantize(float v, RowScale s) {
  // inv == 0 (zero rows, rows that are not finite): 0 whatever v is
  const float q = fminf(fmaxf(rintf(v * s.inv), -127.0f), 127.0f);
  return s.inv != 0.0f ? int32_t(q) : 0;
}

// Vector j of thread t of an 8-bit row of `bytes` bytes (a multiple of 64):
// elements from D on are zero.
template <int kThreads, int kVec, int kPer>
__device__ __forceinline__ void store_int8_row(int8_t *row, int32_t D, int32_t bytes, int t,
                                               const float (&v)[kPer][kVec], RowScale s) {
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int c = (j * kThreads + t) * kVec;
    if constexpr (kVec == 8) {
      if (c < D) {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i / 4] |= (uint32_t(quantize(v[j][i], s)) & 255u) << (8 * (i % 4));
        *reinterpret_cast<uint2 *>(row + c) = make_uint2(w[0], w[1]);
      }
    } else {
      if (c < D) row[c] = int8_t(quantize(v[j][0], s));
    }
  }
  for (int c = D + t; c < bytes; c += kThreads) row[c] = 0;
}

}  // namespace llep
