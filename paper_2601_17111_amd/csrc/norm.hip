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
// computed from the r that was not rounded yet.
#include <algorithm>

#include "kernels.h"
#include "rows.h"

namespace llep {

constexpr int64_t kNormGrid = 65536;  // workgroups at most; they then take several rows

__device__ __forceinline__ float inv_sqrt(float v) { return rsqrtf(v); }
__device__ __forceinline__ double inv_sqrt(double v) { return 1.0 / sqrt(v); }

template <typename T, int kVec>
__device__ __forceinline__ void gate_vec(const NormArgs &a, int64_t row, uint32_t c,
                                         float (&g)[kVec]) {
  const T *p = static_cast<const T *>(a.gate);
  if (a.gate_shape == LLEP_GATE_CHANNEL) {
    load_vec<T, kVec>(p + c, g);
  } else if (a.gate_shape == LLEP_GATE_FULL) {
    load_vec<T, kVec>(p + row * a.D + c, g);
  } else {
    float v[1] = {1.0f};
    if (a.gate_shape == LLEP_GATE_TOKEN) load_vec<T, 1>(p + row, v);
#pragma unroll
    for (int i = 0; i < kVec; ++i) g[i] = v[0];
  }
}

template <typename T, int kThreads, int kVec, int kPer>
__global__ __launch_bounds__(kThreads < kRowWg ? kRowWg : kThreads) void block_norm_kernel(
    NormArgs a) {
  constexpr int kRows = kThreads < kRowWg ? kRowWg / kThreads : 1;
  __shared__ float lds[RowReduce<kThreads>::kLds];
  RowReduce<kThreads> red(lds);
  const int t = threadIdx.x % kThreads;
  const uint32_t D = a.D;
  const float per_d = 1.0f / float(D);
  const T *w_post = static_cast<const T *>(a.w_post), *w_pre = static_cast<const T *>(a.w_pre);
  const int first = kRows == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
  for (int64_t row = int64_t(blockIdx.x) * kRows + first; row < a.T;
       row += int64_t(gridDim.x) * kRows) {
    const T *x = static_cast<const T *>(a.x) + row * a.D;
    float r[kPer][kVec];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * kThreads + t) * kVec;
#pragma unroll
      for (int i = 0; i < kVec; ++i) r[j][i] = 0.0f;
      if (c < D) load_vec<T, kVec>(x + c, r[j]);
    }
    if (a.b) {
      const T *b = static_cast<const T *>(a.b) + row * a.D;
      float v[kPer][kVec];
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const uint32_t c = (j * kThreads + t) * kVec;
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[j][i] = 0.0f;
        if (c < D) load_vec<T, kVec>(b + c, v[j]);
      }
      float s = a.alpha;
      if (w_post) {
        float q[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < kPer; ++j)
#pragma unroll
          for (int i = 0; i < kVec; ++i) q[0] = fmaf(v[j][i], v[j][i], q[0]);
        red.sum(q);
        s *= rsqrtf(q[0] * per_d + a.eps);
      }
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const uint32_t c = (j * kThreads + t) * kVec;
        if (c >= D) continue;
        float g[kVec], w[kVec];
        gate_vec<T, kVec>(a, row, c, g);
        if (w_post) load_vec<T, kVec>(w_post + c, w);
#pragma unroll
        for (int i = 0; i < kVec; ++i)
          r[j][i] = fmaf(v[j][i] * s, w_post ? g[i] * w[i] : g[i], r[j][i]);
      }
    }
    if (a.r) {
      T *o = static_cast<T *>(a.r) + row * a.D;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const uint32_t c = (j * kThreads + t) * kVec;
        if (c < D) store_vec<T, kVec>(o + c, r[j]);
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
        const uint32_t c = (j * kThreads + t) * kVec;
        if (c >= D) continue;
        float w[kVec];
        load_vec<T, kVec>(w_pre + c, w);
#pragma unroll
        for (int i = 0; i < kVec; ++i) r[j][i] *= s * w[i];
        if (a.h) store_vec<T, kVec>(static_cast<T *>(a.h) + row * a.D + c, r[j]);
      }
      if (a.h_q) {
        float most = 0.0f;
#pragma unroll
        for (int j = 0; j < kPer; ++j)
#pragma unroll
          for (int i = 0; i < kVec; ++i)
            most = __uint_as_float(max(__float_as_uint(most), __float_as_uint(fabsf(r[j][i]))));
        const RowScale s = row_scale(red.max_bits(most));
        store_int8_row<kThreads, kVec, kPer>(a.h_q + row * a.q_bytes, a.D, a.q_bytes, t, r, s);
        if (t == 0) a.h_scale[row] = s.scale;
      }
    }
  }
}

// Backward. A workgroup (or wavefront) takes rows g, g + G, ... and keeps the
// column sums of the weight gradients in registers; they go to the workspace
// as one row of [2][D] per workgroup, which norm_columns_kernel adds up in a
// fixed order. The two sums: sum_t d h r i_r, and s = sum_t [g] D b i_b, with
// the gate inside only where it varies along t. With a gate per channel (or
// none) d w_post = alpha g s and d g = alpha w_post s: one sum serves both.
template <typename T, int kThreads, int kVec, int kPer>
__global__ __launch_bounds__(kThreads) void block_norm_bwd_kernel(NormBwdArgs a) {
  // In short rows a norm's gradient is the small rest of large terms (with one
  // element, f eps / (b^2 + eps)), so the path that takes odd rows, which is
  // not the fast one, has its row sums and what they enter in 64 bits.
  using A = std::conditional_t<kVec == 1, double, float>;
  __shared__ A lds[RowReduce<kThreads, A>::kLds];
  RowReduce<kThreads, A> red(lds);
  const int t = threadIdx.x;
  const A per_d = A(1) / A(a.n.D);
  const uint32_t D = a.n.D;
  const bool varies = a.n.gate_shape == LLEP_GATE_TOKEN || a.n.gate_shape == LLEP_GATE_FULL;
  const T *w_post = static_cast<const T *>(a.n.w_post), *w_pre = static_cast<const T *>(a.n.w_pre);
  float sum_pre[kPer][kVec], sum_post[kPer][kVec];
#pragma unroll
  for (int j = 0; j < kPer; ++j)
#pragma unroll
    for (int i = 0; i < kVec; ++i) sum_pre[j][i] = sum_post[j][i] = 0.0f;
  for (int64_t row = blockIdx.x; row < a.n.T; row += gridDim.x) {
    const int64_t base = row * D;
    float r[kPer][kVec], b[kPer][kVec], dr[kPer][kVec], dh[kPer][kVec];
    // sums over the row: r^2, e r, b^2
    A q[3] = {A(0), A(0), A(0)};
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * kThreads + t) * kVec;
#pragma unroll
      for (int i = 0; i < kVec; ++i) r[j][i] = b[j][i] = dr[j][i] = dh[j][i] = 0.0f;
      if (c >= D) continue;
      load_vec<T, kVec>(static_cast<const T *>(a.d_r) + base + c, dr[j]);
      if (w_pre) {
        load_vec<T, kVec>(static_cast<const T *>(a.r) + base + c, r[j]);
        load_vec<T, kVec>(static_cast<const T *>(a.d_h) + base + c, dh[j]);
      }
      if (a.n.b) load_vec<T, kVec>(static_cast<const T *>(a.n.b) + base + c, b[j]);
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * kThreads + t) * kVec;
      if (c >= D) continue;
      float w[kVec];
      if (w_pre) load_vec<T, kVec>(w_pre + c, w);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        if (w_pre) {
          q[0] += A(r[j][i]) * A(r[j][i]);
          q[1] += A(dh[j][i]) * A(w[i]) * A(r[j][i]);
        }
        q[2] += A(b[j][i]) * A(b[j][i]);
      }
    }
    if (w_pre || w_post) red.sum(q);
    const A i_b = w_post ? inv_sqrt(q[2] * per_d + A(a.n.eps)) : A(1);
    if (w_pre) {
      const A i_r = inv_sqrt(q[0] * per_d + A(a.n.eps));
      const A k = i_r * i_r * i_r * (q[1] * per_d);
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const uint32_t c = (j * kThreads + t) * kVec;
        if (c >= D) continue;
        float w[kVec];
        load_vec<T, kVec>(w_pre + c, w);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          sum_pre[j][i] = fmaf(dh[j][i], r[j][i] * float(i_r), sum_pre[j][i]);
          dr[j][i] = float(A(dr[j][i]) + (i_r * (A(dh[j][i]) * A(w[i])) - k * A(r[j][i])));
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * kThreads + t) * kVec;
      if (c < D) store_vec<T, kVec>(static_cast<T *>(a.dx) + base + c, dr[j]);
    }
    if (!a.n.b) continue;
    // f . b / alpha, and D . n (d g of a gate per token)
    A p[2] = {A(0), A(0)};
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * kThreads + t) * kVec;
      if (c >= D) continue;
      float g[kVec], w[kVec];
      gate_vec<T, kVec>(a.n, row, c, g);
      if (w_post) load_vec<T, kVec>(w_post + c, w);
      float dg[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float bi = b[j][i] * float(i_b);
        const float wi = w_post ? w[i] : 1.0f;
        sum_post[j][i] = fmaf(varies ? dr[j][i] * g[i] : dr[j][i], bi, sum_post[j][i]);
        dg[i] = a.n.alpha * dr[j][i] * (bi * wi);
        p[1] += A(dg[i]);
        dr[j][i] *= g[i] * wi;  // f / alpha from here on
        p[0] += A(dr[j][i]) * A(b[j][i]);
      }
      if (a.n.gate_shape == LLEP_GATE_FULL) store_vec<float, kVec>(a.d_gate + base + c, dg);
    }
    A k = A(0);
    if (w_post || a.n.gate_shape == LLEP_GATE_TOKEN) {
      red.sum(p);
      if (w_post) k = i_b * i_b * (p[0] * per_d);
      if (a.n.gate_shape == LLEP_GATE_TOKEN && t == 0) a.d_gate[row] = float(p[1]);
    }
    const A s = A(a.n.alpha) * i_b;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * kThreads + t) * kVec;
      if (c >= D) continue;
#pragma unroll
      for (int i = 0; i < kVec; ++i) dr[j][i] = float(s * (A(dr[j][i]) - k * A(b[j][i])));
      store_vec<T, kVec>(static_cast<T *>(a.db) + base + c, dr[j]);
    }
  }
  float *part = a.parts + int64_t(blockIdx.x) * 2 * D;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const uint32_t c = (j * kThreads + t) * kVec;
    if (c >= D) continue;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      if (a.dw_pre) part[c + i] = sum_pre[j][i];
      if (a.column_sums) part[D + c + i] = sum_post[j][i];
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
  const int c = blockIdx.x * kWave + threadIdx.x % kWave, w = threadIdx.x / kWave;
  float s = 0.0f;
  if (c < D)
    for (int p = w; p < n_parts; p += kColumnWaves) s += a.parts[(int64_t(p) * 2 + which) * D + c];
  lds[w][threadIdx.x % kWave] = s;
  __syncthreads();
  if (w != 0 || c >= D) return;
  for (int i = 1; i < kColumnWaves; ++i) s += lds[i][threadIdx.x];
  if (which == 0) {
    if (a.dw_pre) a.dw_pre[c] = s;
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
// launch: kThreads x kVec x kPer covers a row (at most LLEP_MAX_NORM_DIM = 8192 elements)
// ---------------------------------------------------------------------------

template <typename T, int kThreads, int kVec, int kPer>
hipError_t run_norm(const NormArgs &a, hipStream_t stream) {
  constexpr int kRows = kThreads < kRowWg ? kRowWg / kThreads : 1;
  const int64_t grid = std::min((a.T + kRows - 1) / kRows, kNormGrid);
  hipLaunchKernelGGL((block_norm_kernel<T, kThreads, kVec, kPer>), dim3(uint32_t(grid)),
                     dim3(kRows * kThreads), 0, stream, a);
  return hipGetLastError();
}

bool rows_aligned(int32_t D, std::initializer_list<const void *> ps) {
  uintptr_t u = 0;
  for (const void *p : ps) u |= reinterpret_cast<uintptr_t>(p);
  return D % 8 == 0 && (u & 15) == 0;
}

template <typename T>
hipError_t launch_norm_t(const NormArgs &a, hipStream_t stream) {
  const int32_t D = a.D;
  if (rows_aligned(D, {a.x, a.b, a.gate_shape == LLEP_GATE_TOKEN ? nullptr : a.gate, a.w_post,
                       a.w_pre, a.r, a.h})) {
    if (D <= 2048) return run_norm<T, 256, 8, 1>(a, stream);
    if (D <= 4096) return run_norm<T, 256, 8, 2>(a, stream);
    return run_norm<T, 256, 8, 4>(a, stream);
  }
  if (D <= 1024) return run_norm<T, 256, 1, 4>(a, stream);
  return run_norm<T, 1024, 1, 8>(a, stream);
}

hipError_t launch_block_norm(const NormArgs &a, hipStream_t stream) {
  if (a.T == 0) return hipSuccess;
  return a.dtype == LLEP_BF16 ? launch_norm_t<uint16_t>(a, stream) : launch_norm_t<float>(a, stream);
}

size_t norm_bwd_workspace_bytes(int64_t T, int32_t D) {
  return size_t(std::min<int64_t>(T, kNormBwdGrid)) * 2 * size_t(D) * 4;
}

template <typename T, int kThreads, int kVec, int kPer>
hipError_t run_norm_bwd(const NormBwdArgs &a, hipStream_t stream) {
  const int grid = int(std::min<int64_t>(a.n.T, kNormBwdGrid));
  if (grid > 0) {
    hipLaunchKernelGGL((block_norm_bwd_kernel<T, kThreads, kVec, kPer>), dim3(grid), dim3(kThreads),
                       0, stream, a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  if (a.dw_pre || a.column_sums)  // with no rows: zeros
    hipLaunchKernelGGL((norm_columns_kernel<T>), dim3((a.n.D + kWave - 1) / kWave, 2),
                       dim3(kColumnWaves * kWave), 0, stream, a, grid);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_norm_bwd_t(const NormBwdArgs &a, hipStream_t stream) {
  const int32_t D = a.n.D;
  if (rows_aligned(D, {a.r, a.n.b, a.n.gate_shape == LLEP_GATE_TOKEN ? nullptr : a.n.gate,
                       a.n.w_post, a.n.w_pre, a.d_r, a.d_h, a.dx, a.db,
                       a.n.gate_shape == LLEP_GATE_FULL ? a.d_gate : nullptr})) {
    if (D <= 2048) return run_norm_bwd<T, 256, 8, 1>(a, stream);
    if (D <= 4096) return run_norm_bwd<T, 256, 8, 2>(a, stream);
    return run_norm_bwd<T, 1024, 8, 1>(a, stream);
  }
  if (D <= 1024) return run_norm_bwd<T, 256, 1, 4>(a, stream);
  return run_norm_bwd<T, 512, 1, 16>(a, stream);
}

hipError_t launch_block_norm_backward(const NormBwdArgs &a, hipStream_t stream) {
  return a.n.dtype == LLEP_BF16 ? launch_norm_bwd_t<uint16_t>(a, stream)
                                : launch_norm_bwd_t<float>(a, stream);
}

}  // namespace llep
