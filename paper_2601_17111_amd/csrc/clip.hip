// The norm over all gradients of a step, and their clipping
// (llep_gradient_norm, llep_clip_gradients).
//
// ||g|| = sqrt(sum of g^2 over every tensor), out = g min(1, max_norm / ||g||).
// Bound by HBM: every element is read twice and written once. Tensors are cut
// into pieces of kPieceElems elements that the workgroups take in turn,
// whatever tensor they are of, so one launch serves kMostTensors tensors of
// any sizes (their table is the kernel's argument: nothing is copied to the
// device or kept). Squares are summed in 64 bits, which holds the squares of
// all float32 values, by a fixed order: per thread, per workgroup (a part in
// the workspace), then over the parts, which every workgroup of the second
// launch adds up for itself. That launch takes the pieces in the other
// direction: what the first one read last is still in the cache. 398 M float32
// elements: 243 us for the norm (6.6 TB/s) and 576 for the rest; 61 tensors of
// 22 M elements in all 15 and 24.
#include <algorithm>

#include "kernels.h"
#include "rows.h"

namespace llep {

constexpr int kClipThreads = 256;
constexpr int kMostTensors = 96;     // per launch: 3.1 KB of arguments
constexpr int64_t kPieceElems = 16384;

struct ClipTable {
  const void *data[kMostTensors];
  void *out[kMostTensors];
  int64_t n[kMostTensors];
  int32_t first[kMostTensors + 1];  // first piece of each tensor; the number of pieces
  uint8_t bf16[kMostTensors], vec[kMostTensors];  // type; whether 16-byte accesses fit
  int32_t count;
};
static_assert(sizeof(ClipTable) <= 3584, "kernel arguments");

// The tensor of piece p: the last one whose first piece is at most p.
__device__ __forceinline__ int tensor_of(const ClipTable &t, int p) {
  int lo = 0, hi = t.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (t.first[mid] <= p)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Sum over the workgroup in every thread, in a fixed order.
__device__ __forceinline__ double clip_sum(double v, double *lds) {
#pragma unroll
  for (int o = kWave / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  if (lane_id() == 0) lds[threadIdx.x / kWave] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < kClipThreads / kWave; ++w) v += lds[w];
  return v;
}

// A piece's elements as 16-byte vectors, kClipAhead of them requested together
// (f takes the vector's place and its elements), then the last ones, or all of
// a tensor that does not start on a 16-byte boundary, one by one.
constexpr int kClipAhead = 2;

template <typename T, class F>
__device__ __forceinline__ void for_piece(const T *p, int64_t n, bool vec, F f) {
  constexpr int kE = 16 / sizeof(T), kStep = kClipThreads * kE;
  const int64_t whole = vec ? n / kE * kE : 0;
  for (int64_t c = int64_t(threadIdx.x) * kE; c < whole; c += kStep * kClipAhead) {
    RawVec<T, kE> v[kClipAhead];
#pragma unroll
    for (int u = 0; u < kClipAhead; ++u)
      if (c + u * kStep < whole) v[u].load(p + c + u * kStep);
#pragma unroll
    for (int u = 0; u < kClipAhead; ++u)
      if (c + u * kStep < whole) f(c + u * kStep, v[u]);
  }
  for (int64_t c = whole + threadIdx.x; c < n; c += kClipThreads) {
    RawVec<T, 1> v;
    v.load(p + c);
    f(c, v);
  }
}

template <typename T>
__device__ __forceinline__ double piece_squares(const void *data, int64_t at, int64_t n, bool vec) {
  double s = 0.0;
  for_piece(static_cast<const T *>(data) + at, n, vec, [&](int64_t, const auto &v) {
#pragma unroll
    for (int i = 0; i < v.kElems; ++i) s = fma(double(v[i]), double(v[i]), s);
  });
  return s;
}

// fresh: the parts' first launch of a call (they are written, not added to)
__global__ __launch_bounds__(kClipThreads) void squares_kernel(ClipTable t, double *parts,
                                                               bool fresh) {
  __shared__ double lds[kClipThreads / kWave];
  double s = 0.0;
  for (int p = blockIdx.x; p < t.first[t.count]; p += gridDim.x) {
    const int i = tensor_of(t, p);
    const int64_t at = (p - t.first[i]) * kPieceElems, n = min(kPieceElems, t.n[i] - at);
    s += t.bf16[i] ? piece_squares<uint16_t>(t.data[i], at, n, t.vec[i])
                   : piece_squares<float>(t.data[i], at, n, t.vec[i]);
  }
  s = clip_sum(s, lds);
  if (threadIdx.x == 0) parts[blockIdx.x] = fresh ? s : parts[blockIdx.x] + s;
}

// The sum of the parts, the same in every workgroup.
__device__ __forceinline__ double parts_sum(const double *parts, int n_parts, double *lds) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n_parts; i += kClipThreads) s += parts[i];
  return clip_sum(s, lds);
}

__global__ __launch_bounds__(kClipThreads) void grad_norm_kernel(const double *parts, int n_parts,
                                                                 float *norm) {
  __shared__ double lds[kClipThreads / kWave];
  const double s = parts_sum(parts, n_parts, lds);
  if (threadIdx.x == 0) *norm = float(sqrt(s));
}

// (stored past the caches: what is left of the first pass in them stays for the
// pieces still to come; 398 M float32 elements 889 -> 834 us for the call)
template <typename T>
__device__ __forceinline__ void piece_scale(const void *data, void *out, int64_t at, int64_t n,
                                            bool vec, float f) {
  T *o = static_cast<T *>(out) + at;
  for_piece(static_cast<const T *>(data) + at, n, vec, [&](int64_t c, const auto &v) {
    constexpr int kE = std::remove_reference_t<decltype(v)>::kElems;
    float x[kE];
#pragma unroll
    for (int i = 0; i < kE; ++i) x[i] = v[i] * f;
    if constexpr (kE == 1) {
      store_vec<T, 1>(o + c, x);
    } else if constexpr (sizeof(T) == 2) {
      i32x4 q;
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = int32_t(pack_bf16x2(x[2 * i], x[2 * i + 1]));
      __builtin_nontemporal_store(q, reinterpret_cast<i32x4 *>(o + c));
    } else {
      const f32x4 q = {x[0], x[1], x[2], x[3]};
      __builtin_nontemporal_store(q, reinterpret_cast<f32x4 *>(o + c));
    }
  });
}

__global__ __launch_bounds__(kClipThreads) void clip_kernel(ClipTable t, const double *parts,
                                                            int n_parts, float max_norm,
                                                            float *norm) {
  __shared__ double lds[kClipThreads / kWave];
  const double all = sqrt(parts_sum(parts, n_parts, lds));
  // at most max_norm, NaN or infinite (in 32 bits, as the caller sees it): 1
  const float f = all > double(max_norm) && all <= 3.4028234663852886e38
                      ? float(double(max_norm) / all) : 1.0f;
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = float(all);
  const int pieces = t.first[t.count];
  for (int q = blockIdx.x; q < pieces; q += gridDim.x) {
    const int p = pieces - 1 - q, i = tensor_of(t, p);
    if (f == 1.0f && t.out[i] == t.data[i]) continue;
    const int64_t at = (p - t.first[i]) * kPieceElems, n = min(kPieceElems, t.n[i] - at);
    if (t.bf16[i])
      piece_scale<uint16_t>(t.data[i], t.out[i], at, n, t.vec[i], f);
    else
      piece_scale<float>(t.data[i], t.out[i], at, n, t.vec[i], f);
  }
}

// Tables of up to kMostTensors tensors with elements, from tensor `i` on;
// a tensor of more pieces than a launch can count is cut.
struct ClipWalk {
  const ClipArgs &a;
  int i = 0;
  int64_t done = 0;  // elements of tensor i in earlier tables
  explicit ClipWalk(const ClipArgs &a_) : a(a_) {}
  bool next(ClipTable &t) {
    constexpr int64_t kMostPieces = int64_t(1) << 30;
    t.count = 0;
    int64_t pieces = 0;
    while (i < a.n && t.count < kMostTensors && pieces < kMostPieces) {
      const llep_gradient &g = a.grads[i];
      const int64_t n = std::min(g.n - done, (kMostPieces - pieces) * kPieceElems);
      if (n > 0) {
        const int size = g.dtype == LLEP_BF16 ? 2 : 4;
        const int k = t.count++;
        t.data[k] = static_cast<const char *>(g.data) + done * size;
        t.out[k] = a.scale ? static_cast<char *>(g.out) + done * size : nullptr;
        t.n[k] = n;
        t.bf16[k] = g.dtype == LLEP_BF16;
        t.vec[k] = ((reinterpret_cast<uintptr_t>(t.data[k]) |
                     (a.scale ? reinterpret_cast<uintptr_t>(t.out[k]) : 0)) & 15) == 0;
        t.first[k] = int32_t(pieces);
        pieces += (n + kPieceElems - 1) / kPieceElems;
        done += n;
      }
      if (done == g.n) {
        ++i;
        done = 0;
      }
    }
    t.first[t.count] = int32_t(pieces);
    return t.count > 0;
  }
};

hipError_t launch_clip(const ClipArgs &a, hipStream_t stream) {
  ClipTable t;
  // the parts: as many as the largest table has workgroups
  int n_parts = 1;
  for (ClipWalk w(a); w.next(t);) n_parts = std::max(n_parts, std::min(t.first[t.count], kClipParts));
  bool fresh = true;
  ClipWalk w(a);
  do {
    if (!w.next(t) && !fresh) break;  // no tensors: the parts are zeros
    const int grid = fresh ? n_parts : std::min(t.first[t.count], kClipParts);
    hipLaunchKernelGGL(squares_kernel, dim3(grid), dim3(kClipThreads), 0, stream, t, a.parts, fresh);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    fresh = false;
  } while (t.count > 0);
  if (a.scale) {
    bool any = false;
    for (ClipWalk s(a); s.next(t); any = true) {
      hipLaunchKernelGGL(clip_kernel, dim3(std::min(t.first[t.count], kClipParts)),
                         dim3(kClipThreads), 0, stream, t, a.parts, n_parts, a.max_norm, a.norm);
      const hipError_t err = hipGetLastError();
      if (err != hipSuccess) return err;
    }
    if (any) return hipSuccess;
  }
  hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kClipThreads), 0, stream, a.parts, n_parts,
                     a.norm);
  return hipGetLastError();
}

}  // namespace llep
