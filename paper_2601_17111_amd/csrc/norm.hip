// The norms around a block with its gate and residual scale, forward and
// backward (llep_block_norm, llep_block_norm_backward).
//
// Forward, per row (rms(v) = 1 / sqrt(mean(v^2) + eps)):
//   n = b rms(b) w_post,  r = x + alpha g n,  h = r rms(r) w_pre
// Backward, from r, b, d r and d h, with i_r = rms(r), i_b = rms(b):
//   e = d h w_pre,   d x = D = d r + i_r e - i_r^3 r mean(e r)
//   m = alpha g D,   f = m w_post,   d b = i_b f - i_b^3 b mean(f b)
//   d w_pre = sum_t d h r i_r,  d w_post = sum_t m b i_b,
//   d g = alpha D n summed over the axes that the gate is broadcast along.
// Bound by HBM: 4 (forward) and 6 (backward) values per element for about 12
// and 25 operations, so a row is read once into registers (rows.h) and every
// sum over it is taken there. All in float32, each output rounded once; h is
// computed from the r that was not rounded yet. Forward of 16384 x 2880 bf16
// with a gate per channel 78 us (4.8 TB/s), of 8192 x 2880 float32 75 us (5.0
// TB/s), one row 2.6 us; with 8-bit rows in place of h 75 us (16384 x 2880);
// backward of 8192 x 7168 bf16 148 us (4.8 TB/s), of 1777 x 2048 float32 with a
// full gate 29 us.
#include <algorithm>

#include "kernels.h"
#include "rows.h"

namespace llep {

constexpr int kVec = 8;  // elements of a thread's vectors

// kOdd: rows that are not whole 16-byte vectors, or not on 16-byte boundaries
// (8192 x 2879 bf16 86 us; element by element 127).
template <bool kOdd, typename T>
__device__ __forceinline__ void fetch(RawVec<T, kVec> &v, const T *p, uint32_t left) {
  if constexpr (kOdd)
    v.load_any(p, int(left));
  else
    v.load(p);
}
template <bool kOdd, typename T>
__device__ __forceinline__ void put(T *p, const float (&v)[kVec], uint32_t left) {
  if constexpr (kOdd)
    store_any<T, kVec>(p, v, int(left));
  else
    store_vec<T, kVec>(p, v);
}

// The weights of a thread's columns (norm weights, and the gate where it
// varies by channel alone), read once per workgroup.
template <typename T, int kPer, bool kOdd>
struct ColumnWeights {
  RawVec<T, kVec> post[kPer], pre[kPer], gate[kPer];
  __device__ __forceinline__ ColumnWeights(const NormArgs &a, uint32_t t, uint32_t n) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * n + t) * kVec;
      post[j].zero();
      pre[j].zero();
      gate[j].zero();
      if (c >= uint32_t(a.D)) continue;
      const uint32_t left = a.D - c;
      if (a.w_post) fetch<kOdd>(post[j], static_cast<const T *>(a.w_post) + c, left);
      if (a.w_pre) fetch<kOdd>(pre[j], static_cast<const T *>(a.w_pre) + c, left);
      if (a.gate_shape == LLEP_GATE_CHANNEL)
        fetch<kOdd>(gate[j], static_cast<const T *>(a.gate) + c, left);
    }
  }
};

// The gate's values of one row (requested with the row).
template <typename T, int kPer, bool kOdd>
struct RowGate {
  RawVec<T, kVec> full[kPer];
  float token;
  __device__ __forceinline__ void load(const NormArgs &a, int64_t row, uint32_t t, uint32_t n) {
    const T *p = static_cast<const T *>(a.gate);
    token = 1.0f;
    if (a.gate_shape == LLEP_GATE_TOKEN) {
      float v[1];
      llep::load_vec<T, 1>(p + row, v);
      token = v[0];
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * n + t) * kVec;
      full[j].zero();
      if (a.gate_shape == LLEP_GATE_FULL && c < uint32_t(a.D))
        fetch<kOdd>(full[j], p + row * a.D + c, a.D - c);
    }
  }
  __device__ __forceinline__ float at(const NormArgs &a, const ColumnWeights<T, kPer, kOdd> &w, int j,
                                      int i) const {
    return a.gate_shape == LLEP_GATE_CHANNEL ? w.gate[j][i]
           : a.gate_shape == LLEP_GATE_FULL  ? full[j][i]
                                             : token;
  }
};

template <typename T, int kPer, bool kOne, bool kOdd>
__global__ __launch_bounds__(kOne ? kRowWaves * kWave : 1024) void block_norm_kernel(NormArgs a) {
  __shared__ double lds[RowReduce<kOne>::kLds];
  RowReduce<kOne> red(lds);
  using Raw = RawVec<T, kVec>;
  const uint32_t n = kOne ? kWave : blockDim.x, t = kOne ? threadIdx.x % kWave : threadIdx.x;
  const uint32_t D = a.D;
  const float per_d = 1.0f / float(D);
  const T *w_post = static_cast<const T *>(a.w_post), *w_pre = static_cast<const T *>(a.w_pre);
  const int64_t step = int64_t(gridDim.x) * (kOne ? kRowWaves : 1);
  int64_t row = kOne ? int64_t(blockIdx.x) * kRowWaves +
                           __builtin_amdgcn_readfirstlane(threadIdx.x / kWave)
                     : blockIdx.x;
  Raw x[kPer], b[kPer];
  RowGate<T, kPer, kOdd> gate;
  auto request = [&]() {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * n + t) * kVec;
      x[j].zero();
      b[j].zero();
      if (c >= D) continue;
      fetch<kOdd>(x[j], static_cast<const T *>(a.x) + row * D + c, D - c);
      if (a.b) fetch<kOdd>(b[j], static_cast<const T *>(a.b) + row * D + c, D - c);
    }
    gate.load(a, row, t, n);
  };
  if (row < a.T) request();
  const ColumnWeights<T, kPer, kOdd> w(a, t, n);
  while (row < a.T) {
    float r[kPer][kVec];
    if (a.b) {
      float s = a.alpha;
      if (w_post) {
        float q[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < kPer; ++j)
#pragma unroll
          for (int i = 0; i < kVec; ++i) q[0] = fmaf(b[j][i], b[j][i], q[0]);
        red.sum(q);
        s *= rsqrtf(q[0] * per_d + a.eps);
      }
#pragma unroll
      for (int j = 0; j < kPer; ++j)
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          const float g = gate.at(a, w, j, i);
          r[j][i] = fmaf(b[j][i] * s, w_post ? g * w.post[j][i] : g, x[j][i]);
        }
    } else {
#pragma unroll
      for (int j = 0; j < kPer; ++j)
#pragma unroll
        for (int i = 0; i < kVec; ++i) r[j][i] = x[j][i];
    }
    const int64_t base = row * D;
    row += step;
    if (row < a.T) request();  // the next row, while this one is worked on
    if (a.r) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const uint32_t c = (j * n + t) * kVec;
        if (c < D) put<kOdd>(static_cast<T *>(a.r) + base + c, r[j], D - c);
      }
    }
    if (w_pre) {
      float q[1] = {0.0f};
#pragma unroll
      for (int j = 0; j < kPer; ++j)
#pragma unroll
        for (int i = 0; i < kVec; ++i) q[0] = fmaf(r[j][i], r[j][i], q[0]);
      red.sum(q);
      const float s = rsqrtf(q[0] * per_d + a.eps);
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const uint32_t c = (j * n + t) * kVec;
#pragma unroll
        for (int i = 0; i < kVec; ++i) r[j][i] *= s * w.pre[j][i];
        if (a.h && c < D) put<kOdd>(static_cast<T *>(a.h) + base + c, r[j], D - c);
      }
      if (a.h_q) {
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j)
#pragma unroll
          for (int i = 0; i < kVec; ++i) most = max(most, __float_as_uint(fabsf(r[j][i])));
        const RowScale s8 = row_scale(red.max_bits(most));
        const int64_t at = (row - step);
        store_int8_row<kVec, kPer>(a.h_q + at * a.q_bytes, D, a.q_bytes, t, n, r, s8);
        if (t == 0) a.h_scale[at] = s8.scale;
      }
    }
  }
}

// Backward. A workgroup takes rows g, g + G, ... (the next one is requested
// while the present one is worked on) and keeps the column sums of the weight
// gradients in registers; they go to the workspace as one row of [2][D] per
// workgroup, which norm_columns_kernel adds up in a fixed order. The two sums:
// sum_t d h r i_r, and s = sum_t [g] D b i_b, with the gate inside only where
// it varies along t. With a gate per channel (or none) d w_post = alpha g s
// and d g = alpha w_post s: one sum serves both.
template <typename T, int kPer, int kMaxThreads>
__global__ __launch_bounds__(kMaxThreads) void block_norm_bwd_kernel(NormBwdArgs a) {
  using Raw = RawVec<T, kVec>;
  __shared__ double lds[RowReduce<false>::kLds];
  RowReduce<false> red(lds);
  const uint32_t n = blockDim.x, t = threadIdx.x;
  const uint32_t D = a.n.D;
  const float per_d = 1.0f / float(D);
  const bool varies = a.n.gate_shape == LLEP_GATE_TOKEN || a.n.gate_shape == LLEP_GATE_FULL;
  const bool has_post = a.n.w_post != nullptr, has_pre = a.n.w_pre != nullptr;
  float sum_pre[kPer][kVec], sum_post[kPer][kVec];
#pragma unroll
  for (int j = 0; j < kPer; ++j)
#pragma unroll
    for (int i = 0; i < kVec; ++i) sum_pre[j][i] = sum_post[j][i] = 0.0f;
  Raw next_r[kPer], next_b[kPer], next_dr[kPer], next_dh[kPer];
  RowGate<T, kPer, false> next_gate;
  auto request = [&](int64_t row) {
    const int64_t base = row * D;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * n + t) * kVec;
      next_r[j].zero();
      next_b[j].zero();
      next_dr[j].zero();
      next_dh[j].zero();
      if (c >= D) continue;
      next_dr[j].load(static_cast<const T *>(a.d_r) + base + c);
      if (has_pre) {
        next_r[j].load(static_cast<const T *>(a.r) + base + c);
        next_dh[j].load(static_cast<const T *>(a.d_h) + base + c);
      }
      if (a.n.b) next_b[j].load(static_cast<const T *>(a.n.b) + base + c);
    }
    next_gate.load(a.n, row, t, n);
  };
  constexpr bool kAhead = kPer == 1;  // else there are no registers for it
  if (kAhead && blockIdx.x < a.n.T) request(blockIdx.x);
  const ColumnWeights<T, kPer, false> w(a.n, t, n);
  for (int64_t row = blockIdx.x; row < a.n.T; row += gridDim.x) {
    if (!kAhead) request(row);
    const int64_t base = row * D;
    Raw r[kPer], b[kPer], dh[kPer];
    float dr[kPer][kVec];
    const RowGate<T, kPer, false> gate = next_gate;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      r[j] = next_r[j];
      b[j] = next_b[j];
      dh[j] = next_dh[j];
#pragma unroll
      for (int i = 0; i < kVec; ++i) dr[j][i] = next_dr[j][i];
    }
    if (kAhead && row + gridDim.x < a.n.T) request(row + gridDim.x);
    // sums over the row: r^2, e r, b^2
    float q[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < kPer; ++j)
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        q[0] = fmaf(r[j][i], r[j][i], q[0]);
        q[1] = fmaf(dh[j][i] * w.pre[j][i], r[j][i], q[1]);
        q[2] = fmaf(b[j][i], b[j][i], q[2]);
      }
    if (has_pre || has_post) red.sum(q);
    const float i_b = has_post ? rsqrtf(q[2] * per_d + a.n.eps) : 1.0f;
    if (has_pre) {
      // one factor at a time: i_r^3 leaves the range of 32 bits for rows of 1e13
      // (and 1e-13) and more
      const float i_r = rsqrtf(q[0] * per_d + a.n.eps);
      const float k = i_r * (q[1] * per_d);
#pragma unroll
      for (int j = 0; j < kPer; ++j)
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          const float ri = r[j][i] * i_r;
          sum_pre[j][i] = fmaf(dh[j][i], ri, sum_pre[j][i]);
          dr[j][i] = fmaf(i_r, fmaf(dh[j][i], w.pre[j][i], -k * ri), dr[j][i]);
        }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * n + t) * kVec;
      if (c < D) store_vec<T, kVec>(static_cast<T *>(a.dx) + base + c, dr[j]);
    }
    if (!a.n.b) continue;
    // f . b / alpha, and D . n (d g of a gate per token)
    float p[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * n + t) * kVec;
      float dg[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float bi = b[j][i] * i_b;
        const float wi = has_post ? w.post[j][i] : 1.0f;
        const float g = gate.at(a.n, w, j, i);
        sum_post[j][i] = fmaf(varies ? dr[j][i] * g : dr[j][i], bi, sum_post[j][i]);
        dg[i] = a.n.alpha * dr[j][i] * (bi * wi);
        p[1] += dg[i];
        dr[j][i] *= g * wi;  // f / alpha from here on
        p[0] = fmaf(dr[j][i], b[j][i], p[0]);
      }
      if (a.n.gate_shape == LLEP_GATE_FULL && c < D)
        store_vec<float, kVec>(a.d_gate + base + c, dg);
    }
    float k = 0.0f;
    if (has_post || a.n.gate_shape == LLEP_GATE_TOKEN) {
      red.sum(p);
      if (has_post) k = i_b * (p[0] * per_d);
      if (a.n.gate_shape == LLEP_GATE_TOKEN && t == 0) a.d_gate[row] = p[1];
    }
    // (without w_post b does not enter db, whatever is in it)
    const float s = a.n.alpha * i_b;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * n + t) * kVec;
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        dr[j][i] = s * (has_post ? fmaf(-k, b[j][i] * i_b, dr[j][i]) : dr[j][i]);
      if (c < D) store_vec<T, kVec>(static_cast<T *>(a.db) + base + c, dr[j]);
    }
  }
  float *part = a.parts + int64_t(blockIdx.x) * 2 * D;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const uint32_t c = (j * n + t) * kVec;
    if (c >= D) continue;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      if (a.dw_pre) part[c + i] = sum_pre[j][i];
      if (a.column_sums) part[D + c + i] = sum_post[j][i];
    }
  }
}

// Backward of odd rows: element by element, several times over the row, which
// the cache holds; what has to stay in 32 bits between two sweeps is kept in
// LDS, every element by its thread, and the column sums in the workspace. In a
// row of one element a norm's gradient is the small rest of large terms (f eps /
// (b^2 + eps)), so the row sums and what they enter have 64 bits; rows of eight
// elements and more do without them (whole rows run in 32 bits), so that the
// sweeps and the 64 bits of longer odd rows are not needed, only not replaced:
// 8192 x 2879 255 us where its bytes take 54. (The 64 bits in registers, with
// 16-byte loads, take as long: 260 and 264 us, 300 x 501 15 and 11.5.)
template <typename T>
__device__ __forceinline__ float load1(const void *p, int64_t i) {
  float v[1];
  load_vec<T, 1>(static_cast<const T *>(p) + i, v);
  return v[0];
}
template <typename T>
__device__ __forceinline__ void store1(void *p, int64_t i, float v) {
  const float x[1] = {v};
  store_vec<T, 1>(static_cast<T *>(p) + i, x);
}
template <typename T>
__device__ __forceinline__ float gate1(const NormArgs &a, int64_t row, int c) {
  switch (a.gate_shape) {
    case LLEP_GATE_CHANNEL: return load1<T>(a.gate, c);
    case LLEP_GATE_TOKEN: return load1<T>(a.gate, row);
    case LLEP_GATE_FULL: return load1<T>(a.gate, row * a.D + c);
    default: return 1.0f;
  }
}

template <typename T>
__global__ __launch_bounds__(1024) void block_norm_bwd_odd_kernel(NormBwdArgs a) {
  __shared__ double lds[RowReduce<false>::kLds];
  __shared__ float kept[LLEP_MAX_NORM_DIM];
  RowReduce<false> red(lds);
  const NormArgs &f = a.n;
  const int n = blockDim.x, t = threadIdx.x, D = f.D;
  const bool varies = f.gate_shape == LLEP_GATE_TOKEN || f.gate_shape == LLEP_GATE_FULL;
  float *part = a.parts + int64_t(blockIdx.x) * 2 * D;
  for (int64_t row = blockIdx.x; row < f.T; row += gridDim.x) {
    const int64_t base = row * D;
    const bool fresh = row == blockIdx.x;
    double q[3] = {0.0, 0.0, 0.0};
    for (int c = t; c < D; c += n) {
      if (f.w_pre) {
        const double r = load1<T>(a.r, base + c);
        q[0] += r * r;
        q[1] += double(load1<T>(a.d_h, base + c)) * double(load1<T>(f.w_pre, c)) * r;
      }
      const double b = f.b ? load1<T>(f.b, base + c) : 0.0;
      q[2] += b * b;
    }
    red.sum(q);
    const double i_b = f.w_post ? 1.0 / sqrt(q[2] / D + double(f.eps)) : 1.0;
    const double i_r = 1.0 / sqrt(q[0] / D + double(f.eps));
    double k = i_r * i_r * i_r * (q[1] / D);
    double p[2] = {0.0, 0.0};  // f . b / alpha, and D . n
    for (int c = t; c < D; c += n) {
      float dr = load1<T>(a.d_r, base + c);
      if (f.w_pre) {
        const float r = load1<T>(a.r, base + c), dh = load1<T>(a.d_h, base + c);
        part[c] = (fresh ? 0.0f : part[c]) + dh * (r * float(i_r));
        dr = float(double(dr) + (i_r * (double(dh) * double(load1<T>(f.w_pre, c))) - k * double(r)));
      }
      store1<T>(a.dx, base + c, dr);
      if (!f.b) continue;
      const float b = load1<T>(f.b, base + c), bi = b * float(i_b);
      const float g = gate1<T>(f, row, c), w = f.w_post ? load1<T>(f.w_post, c) : 1.0f;
      if (a.column_sums)
        part[D + c] = (fresh ? 0.0f : part[D + c]) + (varies ? dr * g : dr) * bi;
      const float dg = f.alpha * dr * (bi * w);
      if (f.gate_shape == LLEP_GATE_FULL) a.d_gate[base + c] = dg;
      dr *= g * w;
      kept[c] = dr;
      p[0] += double(dr) * double(b);
      p[1] += double(dg);
    }
    if (!f.b) continue;
    red.sum(p);
    if (f.gate_shape == LLEP_GATE_TOKEN && t == 0) a.d_gate[row] = float(p[1]);
    k = f.w_post ? i_b * i_b * (p[0] / D) : 0.0;
    for (int c = t; c < D; c += n) {
      double d = kept[c];
      if (f.w_post) d -= k * double(load1<T>(f.b, base + c));
      store1<T>(a.db, base + c, float(double(f.alpha) * i_b * d));
    }
  }
}

// The workgroups' column sums added up: a thread per column and 1/16 of the
// rows, joined through LDS.
constexpr int kColumnWaves = 16;

template <typename T>
__global__ __launch_bounds__(kColumnWaves * kWave) void norm_columns_kernel(NormBwdArgs a,
                                                                            int n_parts) {
  __shared__ float lds[kColumnWaves][kWave];
  const int D = a.n.D;
  const int which = blockIdx.y;  // 0: d w_pre, 1: the sum of d w_post and d g
  if (which == 0 ? a.dw_pre == nullptr : !a.column_sums) return;
  const int c = blockIdx.x * kWave + threadIdx.x % kWave, w = threadIdx.x / kWave;
  float s = 0.0f;
  if (c < D) {
#pragma unroll 8
    for (int p = w; p < n_parts; p += kColumnWaves) s += a.parts[(int64_t(p) * 2 + which) * D + c];
  }
  lds[w][threadIdx.x % kWave] = s;
  __syncthreads();
  if (w != 0 || c >= D) return;
  for (int i = 1; i < kColumnWaves; ++i) s += lds[i][threadIdx.x];
  if (which == 0) {
    a.dw_pre[c] = s;
    return;
  }
  float g[1] = {1.0f}, wp[1] = {1.0f};
  if (a.n.gate_shape == LLEP_GATE_CHANNEL) load_vec<T, 1>(static_cast<const T *>(a.n.gate) + c, g);
  if (a.n.w_post) load_vec<T, 1>(static_cast<const T *>(a.n.w_post) + c, wp);
  s *= a.n.alpha;
  if (a.dw_post) a.dw_post[c] = s * g[0];
  if (a.n.gate_shape == LLEP_GATE_CHANNEL) a.d_gate[c] = s * wp[0];
}

// ---------------------------------------------------------------------------
// launch
// ---------------------------------------------------------------------------

bool rows_aligned(int32_t D, std::initializer_list<const void *> ps) {
  uintptr_t u = 0;
  for (const void *p : ps) u |= reinterpret_cast<uintptr_t>(p);
  return D % 8 == 0 && (u & 15) == 0;
}

// Wavefronts of a compute unit that the grids are sized for. Workgroups stay
// and take several rows, the next row requested ahead. (8 / 16 / 24 / 32: forward of
// 16384 x 2880 bf16 106 / 79 / 84 / 79 us, backward 131 / 119 / 146 / 147.)
constexpr int kNormWaves = 16;

// at most `most` workgroups for n rows, with as many rows each
static int64_t even_grid(int64_t n, int64_t most) {
  if (n <= most) return n;
  const int64_t rows = (n + most - 1) / most;
  return (n + rows - 1) / rows;
}

template <typename T, bool kOne, bool kOdd>
hipError_t run_norm(const NormArgs &a, hipStream_t stream) {
  const int threads = kOne ? kRowWaves * kWave : row_threads(a.D, kVec, 1);
  const int64_t wgs = kOne ? (a.T + kRowWaves - 1) / kRowWaves : a.T;
  const int64_t grid = even_grid(wgs, int64_t(256) * std::max(1, kNormWaves * kWave / threads));
  hipLaunchKernelGGL((block_norm_kernel<T, 1, kOne, kOdd>), dim3(uint32_t(grid)), dim3(threads), 0,
                     stream, a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_norm_t(const NormArgs &a, hipStream_t stream) {
  static_assert(LLEP_MAX_NORM_DIM == 1024 * kVec, "a row fits a workgroup");
  const bool one = a.D <= kWave * kVec;
  if (rows_aligned(a.D, {a.x, a.b, a.gate_shape == LLEP_GATE_TOKEN ? nullptr : a.gate, a.w_post,
                         a.w_pre, a.r, a.h}))
    return one ? run_norm<T, true, false>(a, stream) : run_norm<T, false, false>(a, stream);
  return one ? run_norm<T, true, true>(a, stream) : run_norm<T, false, true>(a, stream);
}

hipError_t launch_block_norm(const NormArgs &a, hipStream_t stream) {
  if (a.T == 0) return hipSuccess;
  return a.dtype == LLEP_BF16 ? launch_norm_t<uint16_t>(a, stream) : launch_norm_t<float>(a, stream);
}

// Workgroups of the backward, all with as many rows (but the last): one row up
// to 256 workgroups, then four, so that the rows of column sums stay a small
// part of what is moved, then what the chip has room for.
static int norm_bwd_grid(int64_t T, int32_t D) {
  const int waves = row_threads(D, kVec, 1) / kWave;
  const int64_t most =
      int64_t(256) * std::max(1, std::min(kNormWaves / waves, kNormBwdGrid / 256));
  return int(even_grid(T, std::max<int64_t>(256, std::min(most, (T + 3) / 4))));
}

size_t norm_bwd_workspace_bytes(int64_t T, int32_t D) {
  return size_t(norm_bwd_grid(T, D)) * 2 * size_t(D) * 4;
}

template <typename T>
hipError_t launch_norm_bwd_t(const NormBwdArgs &a, hipStream_t stream) {
  const int32_t D = a.n.D;
  const int grid = norm_bwd_grid(a.n.T, D);
  if (grid > 0) {
    const bool whole =
        rows_aligned(D, {a.r, a.n.b, a.n.gate_shape == LLEP_GATE_TOKEN ? nullptr : a.n.gate,
                         a.n.w_post, a.n.w_pre, a.d_r, a.d_h, a.dx, a.db,
                         a.n.gate_shape == LLEP_GATE_FULL ? a.d_gate : nullptr});
    // 128 registers a thread, as 16 wavefronts have, hold a bf16 row's vectors
    // and the next row's; long float32 rows take half the threads
    if (!whole)
      hipLaunchKernelGGL(block_norm_bwd_odd_kernel<T>, dim3(grid), dim3(std::min(1024, (D + kWave - 1) / kWave * kWave)), 0, stream,
                         a);
    else if (D <= 512 * kVec)
      hipLaunchKernelGGL((block_norm_bwd_kernel<T, 1, 512>), dim3(grid),
                         dim3(row_threads(D, kVec, 1)), 0, stream, a);
    else if constexpr (sizeof(T) == 2)
      hipLaunchKernelGGL((block_norm_bwd_kernel<T, 1, 1024>), dim3(grid),
                         dim3(row_threads(D, kVec, 1)), 0, stream, a);
    else
      hipLaunchKernelGGL((block_norm_bwd_kernel<T, 2, 512>), dim3(grid),
                         dim3(row_threads(D, kVec, 2)), 0, stream, a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  if (a.dw_pre || a.column_sums)  // with no rows: zeros
    hipLaunchKernelGGL((norm_columns_kernel<T>), dim3((D + kWave - 1) / kWave, 2),
                       dim3(kColumnWaves * kWave), 0, stream, a, grid);
  return hipGetLastError();
}

hipError_t launch_block_norm_backward(const NormBwdArgs &a, hipStream_t stream) {
  return a.n.dtype == LLEP_BF16 ? launch_norm_bwd_t<uint16_t>(a, stream)
                                : launch_norm_bwd_t<float>(a, stream);
}

}  // namespace llep
