// Rows and products of 4-bit floating point with a power of two for every 32
// values (llep_quantize_rows_mxfp4, llep_dequantize_rows_mxfp4,
// llep_pack_mxfp4, llep_mxfp4_matmul, llep_grouped_ffn_mxfp4):
//   C[m][n] = sum_b 2^(sa[m][b] + sb[n][b]) sum_{k in block b} A[m][k] B[n][k].
// The matrix cores take the exponents with the operands (v_mfma_scale_f32_*):
// the products of a block are exact, sums over blocks are of 32 bits.
//
// 64 bytes of a row are a slice of 128 k with the four exponents that belong to
// it. Weights are packed (llep_pack_mxfp4) in blocks of 16 rows x one slice, 1 KB
// each, 16 bytes of each row after another, so that lane l of a wavefront that
// reads a block in order has its operand; the exponents of 16 rows lie in blocks
// of four slices, 64 bytes each, 4 bytes a row.
#include <algorithm>
#include <cmath>

#include "mx_tiles.h"
#include "rows.h"

namespace llep {

constexpr int kSliceK = 128;     // values of a row in a slice
constexpr int kBlockK = 32;      // that share an exponent
constexpr int kScaleSlices = 4;  // slices whose exponents lie together
static int32_t mx_slices(int32_t K) { return (K + kSliceK - 1) / kSliceK; }
static int32_t mx_row_bytes(int32_t K) { return mx_slices(K) * 64; }
static int32_t mx_scale_bytes(int32_t K) { return (mx_slices(K) + kScaleSlices - 1) / kScaleSlices * 16; }
int32_t mxfp4_row_bytes(int32_t K) { return mx_row_bytes(K); }
int32_t mxfp4_scale_bytes(int32_t K) { return mx_scale_bytes(K); }

// ---------------------------------------------------------------------------
// rows: a wavefront per 512 values of a row, 8 per lane, so that a block's
// largest is found among four lanes next to each other and the exponents are a
// 16-byte piece
// ---------------------------------------------------------------------------

struct MxRowsArgs {
  int64_t R;
  int32_t D, q_pitch, s_pitch;
  const void *x;
  void *out;
  uint8_t *q, *scale;
};

constexpr int kMxRowWaves = 4;

// A wavefront's items (row, part of it), one after another
struct MxRowItems {
  int64_t row, rows_on;
  int part, parts_on, parts;
  __device__ __forceinline__ explicit MxRowItems(int D) {
    parts = (D + 511) / 512;
    const uint32_t first = blockIdx.x * kMxRowWaves +
                           __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t step = gridDim.x * kMxRowWaves;
    row = first / uint32_t(parts), part = int(first % uint32_t(parts));
    rows_on = step / uint32_t(parts), parts_on = int(step % uint32_t(parts));
  }
  __device__ __forceinline__ void next() {
    row += rows_on, part += parts_on;
    if (part >= parts) part -= parts, ++row;
  }
};

// kPast: values of more than the 256 MB cache behind the L2s, which loads and stores go
// past (92160 x 2880 132 -> 119 us, and 136 -> 101 for the values back; both, on buffers
// in turn, 260 with the 4-bit rows through the cache, 249 past it, though on the same
// buffers again and again 221 and 248). With less, the call that reads the results takes
// longer for it than these save (8192 x 2880 and 2880 x 2880 weights 63 -> 71; values
// back and a read of them 26.7 -> 28.4).
template <typename T, bool kOdd, bool kPast>
__global__ __launch_bounds__(kMxRowWaves * kWave) void mx_quantize_kernel(MxRowsArgs a) {
  const int lane = lane_id();
  const int q_bytes = (a.D + kSliceK - 1) / kSliceK * 64;
  for (MxRowItems it(a.D); it.row < a.R; it.next()) {
    const int64_t row = it.row;
    const int part = it.part, c = part * 512 + lane * 8;
    RawVec<T, 8> in;
    in.zero();
    if (c < a.D) {
      const T *p = static_cast<const T *>(a.x) + row * a.D + c;
      if constexpr (kOdd)
        in.load_any(p, a.D - c);
      else if constexpr (kPast)
#pragma unroll
        for (int j = 0; j < RawVec<T, 8>::kWords; ++j)
          in.w[j] = __builtin_nontemporal_load(reinterpret_cast<const i32x4 *>(p) + j);
      else
        in.load(p);
    }
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(in[j]) & 0x7fffffffu);
    most = max(most, dpp<0xb1, 0xf>(most));  // quad_perm: lanes 1, 0, 3, 2; then 2, 3, 0, 1
    most = max(most, dpp<0x4e, 0xf>(most));
    const uint32_t e = mx_exponent(most);
    const float step = mx_step(e);
    if (c / 2 < q_bytes) {
      const uint32_t v = mx_pack4(in[0], in[1], in[2], in[3], step) |
                         (mx_pack4(in[4], in[5], in[6], in[7], step) << 16);
      uint32_t *to = reinterpret_cast<uint32_t *>(a.q + row * a.q_pitch + c / 2);
      if constexpr (kPast)
        __builtin_nontemporal_store(v, to);
      else
        *to = v;
    }
    uint32_t w = e | (dpp<0x104, 0xf>(e) << 8);  // row_shl:4, :8: four blocks of 16 lanes
    w |= dpp<0x108, 0xf>(w) << 16;
    if ((lane & 15) == 0)
      *reinterpret_cast<uint32_t *>(a.scale + row * a.s_pitch + part * 16 + (lane >> 2)) = w;
  }
}

// kN values of a lane at a time, so that a wavefront's stores are whole pieces of the
// row: 8 of bfloat16, 4 of float32 (20000 x 7168 175 -> 147 us).
template <typename T, bool kPast>
__global__ __launch_bounds__(kMxRowWaves * kWave) void mx_dequantize_kernel(MxRowsArgs a) {
  constexpr int kN = 16 / sizeof(T);
  using Word = std::conditional_t<kN == 8, uint32_t, uint16_t>;
  const int lane = lane_id();
  const bool whole = a.D % 8 == 0 && (reinterpret_cast<uintptr_t>(a.out) & 15) == 0;
  for (MxRowItems it(a.D); it.row < a.R; it.next()) {
#pragma unroll
    for (int part = 0; part < 8 / kN; ++part) {
      const int c = it.part * 512 + (part * kWave + lane) * kN;
      if (c >= a.D) continue;
      const uint32_t w = *reinterpret_cast<const Word *>(a.q + it.row * a.q_pitch + c / 2);
      const uint32_t e = a.scale[it.row * a.s_pitch + c / kBlockK];
      // 2^-127 is below the normal range: half of it times two
      const float step = e == 0 ? 0x1p-126f : mx_step(e);
      float v[kN];
#pragma unroll
      for (int j = 0; j < kN; j += 2) {
        const auto two = j == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, step, 0)
                         : j == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, step, 1)
                         : j == 4 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, step, 2)
                                  : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, step, 3);
        v[j] = two[0], v[j + 1] = two[1];
      }
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        if (e == 0) v[j] *= 0.5f;
        if (e == 255) v[j] = __uint_as_float(0x7fc00000u);
      }
      T *p = static_cast<T *>(a.out) + it.row * a.D + c;
      if (whole) {
        i32x4 u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (kN == 8)
            u[j] = int32_t(pack_bf16x2(v[2 * j], v[2 * j + 1]));
          else
            u[j] = __float_as_int(v[j]);
        }
        if constexpr (kPast)
          __builtin_nontemporal_store(u, reinterpret_cast<i32x4 *>(p));
        else
          *reinterpret_cast<i32x4 *>(p) = u;
      } else {
        store_any<T, kN>(p, v, a.D - c);
      }
    }
  }
}

static dim3 mx_rows_grid(const MxRowsArgs &a) {
  const int64_t items = a.R * ((a.D + 511) / 512);
  return dim3(uint32_t(std::min<int64_t>((items + kMxRowWaves - 1) / kMxRowWaves, 256 * 8 * 4)));
}

static bool mx_past_cache(int64_t bytes) { return bytes > (int64_t(256) << 20); }

hipError_t launch_quantize_mxfp4(int64_t R, int32_t D, llep_dtype dtype, const void *x, uint8_t *q,
                                 int32_t q_pitch, uint8_t *scale, int32_t s_pitch,
                                 hipStream_t stream) {
  if (R == 0) return hipSuccess;
  const MxRowsArgs a = {R, D, q_pitch, s_pitch, x, nullptr, q, scale};
  const bool whole = D % 8 == 0 && (reinterpret_cast<uintptr_t>(x) & 15) == 0;
  const dim3 grid = mx_rows_grid(a), threads(kMxRowWaves * kWave);
  if (dtype == LLEP_BF16) {
    if (whole && mx_past_cache(R * D * 2))
      hipLaunchKernelGGL((mx_quantize_kernel<uint16_t, false, true>), grid, threads, 0, stream, a);
    else if (whole)
      hipLaunchKernelGGL((mx_quantize_kernel<uint16_t, false, false>), grid, threads, 0, stream, a);
    else
      hipLaunchKernelGGL((mx_quantize_kernel<uint16_t, true, false>), grid, threads, 0, stream, a);
  } else {
    if (whole)
      hipLaunchKernelGGL((mx_quantize_kernel<float, false, false>), grid, threads, 0, stream, a);
    else
      hipLaunchKernelGGL((mx_quantize_kernel<float, true, false>), grid, threads, 0, stream, a);
  }
  return hipGetLastError();
}

hipError_t launch_dequantize_mxfp4(int64_t R, int32_t D, llep_dtype dtype, const uint8_t *q,
                                   int32_t q_pitch, const uint8_t *scale, int32_t s_pitch,
                                   void *out, hipStream_t stream) {
  if (R == 0) return hipSuccess;
  const MxRowsArgs a = {R,   D, q_pitch, s_pitch, nullptr, out, const_cast<uint8_t *>(q),
                        const_cast<uint8_t *>(scale)};
  const dim3 grid = mx_rows_grid(a), threads(kMxRowWaves * kWave);
  const bool past = mx_past_cache(R * D * (dtype == LLEP_BF16 ? 2 : 4));
  if (dtype == LLEP_BF16) {
    if (past)
      hipLaunchKernelGGL((mx_dequantize_kernel<uint16_t, true>), grid, threads, 0, stream, a);
    else
      hipLaunchKernelGGL((mx_dequantize_kernel<uint16_t, false>), grid, threads, 0, stream, a);
  } else {
    if (past)
      hipLaunchKernelGGL((mx_dequantize_kernel<float, true>), grid, threads, 0, stream, a);
    else
      hipLaunchKernelGGL((mx_dequantize_kernel<float, false>), grid, threads, 0, stream, a);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// packing: 16 bytes of a packed row, or the exponents of four rows in a slice, per
// thread
// ---------------------------------------------------------------------------

struct MxPackArgs {
  int64_t E;
  int32_t N, K, Np, nk, nq, w_bytes, s_bytes;
  const uint8_t *w0, *s0, *w1, *s1;
  uint8_t *out;
};

__global__ __launch_bounds__(256) void mx_pack_kernel(MxPackArgs a) {
  const int64_t data = int64_t(a.Np / 16) * a.nk * 64, scales = int64_t(a.Np / 16) * a.nq * 16;
  const int64_t per = data + scales;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < a.E * per;
       i += int64_t(gridDim.x) * 256) {
    const int64_t e = i / per, u = i - e * per;
    const bool is_data = u < data;
    const int64_t at = is_data ? u : u - data;
    const int in = int(at & (is_data ? 63 : 15));
    const int64_t blk = at >> (is_data ? 6 : 4);
    const int cols = is_data ? a.nk : a.nq;
    const int kb = int(blk % cols);
    int n = int(blk / cols) * 16 + (is_data ? in & 15 : (in & 3) * 4);
    // two matrices: 32 rows of the first, then the matching 32 of the second
    const uint8_t *w = a.w0, *s = a.s0;
    if (a.w1) {
      if (n & 32) w = a.w1, s = a.s1;
      n = (n >> 6) * 32 + (n & 31);
    }
    uint32_t v[4] = {0u, 0u, 0u, 0u};
    if (is_data) {
      const int k = kb * kSliceK + (in >> 4) * 32;  // the first of 32 values
      const int left = n < a.N ? a.K - k : 0;
      if (left > 0) {
        const uint8_t *p = w + (e * a.N + n) * a.w_bytes + k / 2;
        if (left >= 32 && ((reinterpret_cast<uintptr_t>(w) | a.w_bytes) & 15) == 0) {
          const uint4 q = *reinterpret_cast<const uint4 *>(p);
          v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
        } else {
#pragma unroll
          for (int b = 0; b < 16; ++b) {
            const int have = left - 2 * b;  // values from this byte on
            if (have > 0) v[b / 4] |= (uint32_t(p[b]) & (have > 1 ? 255u : 15u)) << (8 * (b % 4));
          }
        }
      }
    } else {
      const int blocks = (a.K + kBlockK - 1) / kBlockK, c0 = kb * 16 + (in >> 2) * 4;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint8_t *p = s + (e * a.N + min(n + r, a.N - 1)) * a.s_bytes;
#pragma unroll
        for (int b = 0; b < 4; ++b)
          v[r] |= (n + r < a.N && c0 + b < blocks ? uint32_t(p[c0 + b]) : 127u) << (8 * b);
      }
    }
    reinterpret_cast<uint4 *>(a.out)[i] = make_uint4(v[0], v[1], v[2], v[3]);
  }
}

size_t packed_mxfp4_bytes(int32_t N, int32_t K) {
  return (size_t(N) + 15) / 16 * 16 * (mx_row_bytes(K) + mx_scale_bytes(K));
}

hipError_t launch_pack_mxfp4(int32_t E, int32_t N, int32_t K, const uint8_t *w0, const uint8_t *s0,
                             const uint8_t *w1, const uint8_t *s1, int32_t w_bytes, int32_t s_bytes,
                             uint8_t *out, hipStream_t stream) {
  MxPackArgs a = {};
  a.E = E;
  a.N = N;
  a.K = K;
  a.Np = w1 ? 2 * N : (N + 15) / 16 * 16;
  a.nk = mx_slices(K);
  a.nq = mx_scale_bytes(K) / 16;
  a.w_bytes = w_bytes;
  a.s_bytes = s_bytes;
  a.w0 = w0, a.s0 = s0, a.w1 = w1, a.s1 = s1;
  a.out = out;
  const int64_t units = a.E * (int64_t(a.Np) * (a.nk * 4 + a.nq));
  hipLaunchKernelGGL(mx_pack_kernel, dim3(uint32_t(std::min<int64_t>((units + 255) / 256, 65536))),
                     dim3(256), 0, stream, a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------

// Stream: few rows. An item is up to 16 kMB rows of one group (of A, dense) by
// 16 kNB packed rows of the weights; a workgroup of kWaves wavefronts takes one
// item at a time, each wavefront a part of k, and adds the parts up through
// LDS, in the order of the wavefronts. v_mfma_scale_f32_16x16x128 takes a 1 KB
// block of the weights as its first operand (lane l: row l % 16, block of 32 k
// l / 16), 16 rows of A as its second; lane l then holds, of row l % 16 of A, the
// columns 4 (l / 16) .. + 3. Every XCD (workgroups are dealt round-robin over
// the 8) takes a contiguous eighth of the items: dense ones with the row tiles of
// a weight unit next to each other, grouped ones with the units of a row tile.
template <int kMB, int kNB, int kWaves, bool kGrouped, bool kSwigluOut>
__global__ __launch_bounds__(kWaves * kWave) void mx_stream_kernel(MxGemmArgs g) {
  constexpr int kBlocks = kMB * kNB;
  constexpr int kRound = kBlocks >= 16 ? 8 : kBlocks;
  constexpr int kUnroll = kMB * kNB <= 8 ? 4 : 2;  // slices
  __shared__ f32x4 part[kWaves][kRound][kWave];
  static_assert(!kSwigluOut || kNB == 4, "32 gate columns and the matching up columns");
  static_assert(kBlocks % kRound == 0 && kRound % kNB == 0, "rounds of whole rows of blocks");
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int nk = g.Kdim / 32;
  const int n_blk = (g.N + 15) / 16;
  const int n_unit = (n_blk + kNB - 1) / kNB;
  const int n_mt = kGrouped ? *g.n_mtiles : int((g.M + 16 * kMB - 1) / (16 * kMB));
  const int kb0 = nk * wave / kWaves, kb1 = nk * (wave + 1) / kWaves;
  const int64_t items = int64_t(n_mt) * n_unit;
  const int xcd = blockIdx.x % 8;
  const int64_t end = items * (xcd + 1) / 8;
  const int shift = 8 * (lane >> 4);
  for (int64_t item = items * xcd / 8 + blockIdx.x / 8; item < end; item += gridDim.x / 8) {
    const int mt = int(kGrouped ? item / n_unit : item % n_mt);
    const int unit = int(kGrouped ? item % n_unit : item / n_mt);
    int e = 0;
    int64_t row0 = int64_t(mt) * 16 * kMB;
    int rows;
    if (kGrouped) {
      const int4 te = g.tiles[mt];
      const int32_t *gr = g.groups + 4 * te.x;
      e = gr[1];
      row0 = int64_t(gr[2]) + te.y * 16 * kMB;
      rows = min(16 * kMB, gr[3] - te.y * 16 * kMB);
    } else {
      rows = int(min<int64_t>(16 * kMB, g.M - row0));
    }
    const char *A = reinterpret_cast<const char *>(g.A) + row0 * g.lda;
    const uint8_t *As = g.a_scale + row0 * g.a_scale_pitch;
    const int blk0 = unit * kNB;
    const char *Be = reinterpret_cast<const char *>(g.B) + e * g.b_expert_stride;
    const char *B = Be + int64_t(blk0) * g.b_blk_stride;
    const char *Bs = Be + g.b_scale_at + int64_t(blk0) * g.b_scale_blk_stride;
    uint32_t offA[kMB], offAs[kMB], offB[kNB], offBs[kNB];
#pragma unroll
    for (int m = 0; m < kMB; ++m) {  // past the last row: the last one again, not stored
      const uint32_t r = uint32_t(min(m * 16 + (lane & 15), rows - 1));
      offA[m] = r * uint32_t(g.lda) + (lane >> 4) * 16;
      offAs[m] = r * uint32_t(g.a_scale_pitch);
    }
#pragma unroll
    for (int n = 0; n < kNB; ++n) {  // and past the last block
      const uint32_t b = uint32_t(min(n, n_blk - 1 - blk0));
      offB[n] = b * uint32_t(g.b_blk_stride) + lane * 16;
      offBs[n] = b * uint32_t(g.b_scale_blk_stride) + (lane & 15) * 4;
    }
    f32x4 acc[kMB][kNB];
#pragma unroll
    for (int m = 0; m < kMB; ++m)
#pragma unroll
      for (int n = 0; n < kNB; ++n) acc[m][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // kU slices at a time, all of their loads under way together
    auto steps = [&](auto count, int kb) {
      constexpr int kU = decltype(count)::value;
      i32x4 fa[kU][kMB], fb[kU][kNB];
      int sa[kU][kMB], sb[kU][kNB];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int k = kb + u;
#pragma unroll
        for (int n = 0; n < kNB; ++n) {
          fb[u][n] = *reinterpret_cast<const i32x4 *>(B + int64_t(k) * 1024 + offB[n]);
          sb[u][n] = *reinterpret_cast<const int32_t *>(Bs + k * 64 + offBs[n]);
        }
#pragma unroll
        for (int m = 0; m < kMB; ++m) {
          fa[u][m] = *reinterpret_cast<const i32x4 *>(A + k * 64 + offA[m]);
          sa[u][m] = *reinterpret_cast<const int32_t *>(As + k * 4 + offAs[m]);
        }
      }
      // (the lane's 32 values have byte lane / 16 of the four)
#pragma unroll
      for (int u = 0; u < kU; ++u) {
#pragma unroll
        for (int n = 0; n < kNB; ++n) sb[u][n] = int(uint32_t(sb[u][n]) >> shift);
#pragma unroll
        for (int m = 0; m < kMB; ++m) {
          sa[u][m] = int(uint32_t(sa[u][m]) >> shift);
#pragma unroll
          for (int n = 0; n < kNB; ++n)
            acc[m][n] = mx_mfma<0>(fb[u][n], fa[u][m], acc[m][n], sb[u][n], sa[u][m]);
        }
      }
    };
    int kb = kb0;
    for (; kb + kUnroll <= kb1; kb += kUnroll) steps(std::integral_constant<int, kUnroll>{}, kb);
    // the rest together: one wait, not one for each
    switch (kb1 - kb) {
      case 3: steps(std::integral_constant<int, 3>{}, kb); break;
      case 2: steps(std::integral_constant<int, 2>{}, kb); break;
      case 1: steps(std::integral_constant<int, 1>{}, kb); break;
      default: break;
    }
#pragma unroll
    for (int b0 = 0; b0 < kBlocks; b0 += kRound) {
#pragma unroll
      for (int b = 0; b < kRound; ++b) part[wave][b][lane] = acc[(b0 + b) / kNB][(b0 + b) % kNB];
      __syncthreads();
      auto total = [&](int b) {
        f32x4 s = part[0][b][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) s += part[w][b][lane];
        return s;
      };
      if constexpr (kSwigluOut) {
        for (int m = wave; m < kRound / kNB; m += kWaves) {
          const int r = (b0 / kNB + m) * 16 + (lane & 15);
          float v[8];
          uint32_t most = 0;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const f32x4 gate = total(m * kNB + half), up = total(m * kNB + 2 + half);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              v[half * 4 + i] = mx_swiglu(gate[i], up[i]);
              most = max(most, __float_as_uint(v[half * 4 + i]) & 0x7fffffffu);
            }
          }
          most = max(most, uint32_t(__shfl_xor(int(most), 16)));
          most = max(most, uint32_t(__shfl_xor(int(most), 32)));
          const uint32_t x = mx_exponent(most);
          const float step = mx_step(x);
          if (r < rows) {
            uint8_t *q = g.act + (row0 + r) * g.ldc + unit * 16 + (lane >> 4) * 2;
            *reinterpret_cast<uint16_t *>(q) = uint16_t(mx_pack4(v[0], v[1], v[2], v[3], step));
            *reinterpret_cast<uint16_t *>(q + 8) = uint16_t(mx_pack4(v[4], v[5], v[6], v[7], step));
            if (lane < 16) {
              uint8_t *s = g.act_scale + (row0 + r) * g.ldc;
              s[unit] = uint8_t(x);
              if (unit == n_unit - 1) mx_pad_scales(s, n_unit, g.act_blocks);
            }
          }
        }
      } else {
        for (int q = wave; q < kRound; q += kWaves) {
          const int m = q / kNB, n = q % kNB;
          const int r = (b0 / kNB + m) * 16 + (lane & 15);
          const int col = (unit * kNB + n) * 16 + (lane >> 4) * 4;
          if (r >= rows || col >= g.N) continue;
          const f32x4 v = total(q);
          if (g.f32_out)
            int8_store4(reinterpret_cast<float *>(g.C) + (row0 + r) * g.ldc, col, g.N, v);
          else
            int8_store4(g.C + (row0 + r) * g.ldc, col, g.N, v);
        }
      }
      __syncthreads();  // the parts are read before the next ones
    }
  }
}

template <int kMB, int kNB, int kWaves, bool kGrouped, bool kSwigluOut>
hipError_t run_mx_stream(const MxGemmArgs &g, int64_t mtiles, hipStream_t stream) {
  const int64_t items = mtiles * ((g.N + 16 * kNB - 1) / (16 * kNB));
  const int grid = int(std::min<int64_t>((items + 7) / 8 * 8, 16384));
  hipLaunchKernelGGL((mx_stream_kernel<kMB, kNB, kWaves, kGrouped, kSwigluOut>), dim3(grid),
                     dim3(kWaves * kWave), 0, stream, g);
  return hipGetLastError();
}

// BM x BM tiles: 256 rows by eight wavefronts, one workgroup on a compute unit,
// or 128 by four, two workgroups; two wavefronts per SIMD either way.
template <int BM, int WAVES_M, int WAVES_N, int kEpi, bool kGrouped>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N) __attribute__((amdgpu_waves_per_eu(2, 2)))
void mx_tiles_kernel(MxGemmArgs g) {
  __shared__ __attribute__((aligned(1024))) char smem[mx_ring_bytes<BM, BM>()];
  std::conditional_t<kGrouped, LaunchSched<BM, BM>, DenseSched<BM, BM>> sched(g);
  TileCoord t;
  if (!sched.first(t)) return;
  mx_tiles<BM, WAVES_M, WAVES_N, kEpi>(g, smem, t, sched);
}

template <int BM, int kEpi, bool kGrouped>
hipError_t run_mx_tiles(const MxGemmArgs &g, hipStream_t stream) {
  constexpr int WAVES_M = 2, WAVES_N = BM / 64;
  int64_t most = cu_count() * (BM == 256 ? 1 : 2);
  if (!kGrouped) most = std::min(most, (g.M + BM - 1) / BM * ((g.N + BM - 1) / BM));
  const int grid = int((most + 7) / 8 * 8);
  hipLaunchKernelGGL((mx_tiles_kernel<BM, WAVES_M, WAVES_N, kEpi, kGrouped>), dim3(grid),
                     dim3(64 * WAVES_M * WAVES_N), 0, stream, g);
  return hipGetLastError();
}

// outputs in bfloat16 or float32
template <int BM, bool kGrouped>
hipError_t run_mx_tiles_out(const MxGemmArgs &g, hipStream_t stream) {
  return g.f32_out ? run_mx_tiles<BM, kMxF32, kGrouped>(g, stream)
                   : run_mx_tiles<BM, kMxBf16, kGrouped>(g, stream);
}

static MxGemmArgs mx_weights(const uint8_t *w, int32_t N, int32_t K) {
  MxGemmArgs g = {};
  g.B = reinterpret_cast<const uint16_t *>(w);
  g.b_expert_stride = int64_t(packed_mxfp4_bytes(N, K));
  g.b_blk_stride = int64_t(mx_slices(K)) * 1024;
  g.b_scale_at = int64_t((N + 15) / 16) * g.b_blk_stride;
  g.b_scale_blk_stride = int64_t(mx_scale_bytes(K)) * 16;
  g.N = N;
  g.Kdim = mx_slices(K) * 32;
  return g;
}

hipError_t launch_mxfp4_matmul(const MxMatmulArgs &a, hipStream_t stream) {
  if (a.M == 0) return hipSuccess;
  MxGemmArgs g = mx_weights(a.w, a.N, a.K);
  g.A = reinterpret_cast<const uint16_t *>(a.x);
  g.lda = a.x_pitch;
  g.a_scale = a.x_scale;
  g.a_scale_pitch = a.s_pitch;
  g.C = static_cast<uint16_t *>(a.out);
  g.ldc = a.N;
  g.M = a.M;
  g.f32_out = a.dtype == LLEP_F32;
  // The least of what the ways take in us, about: the stream with 32 or 64 rows
  // and columns an item, by rounds of 256 items, the tiles by rounds of as many as
  // the chip has room for (of 128 x 128 two on a compute unit).
  // Stream of 32 / of 64 / tiles of 128 / of 256, M x N x K:
  //   32 x 2880 x 2880 5.6 / 7.8 / 12.6 / -, 64 x 7168 x 2048 7.7 / 8.8 / 10.5 / 13.6,
  //   128 x 2048 x 7168 11.2 / 20.6 / 27.7 / 37, 256 x 4096 x 4096 22.8 / 13.8 / 17.8 / -,
  //   256 x 7168 x 2048 23.4 / 16.7 / 11.2 / 16.7, 512 x 2048 x 7168 36 / 21 / 28 / 42,
  //   512 x 4096 x 4096 42 / 26 / 18 / -, 1024 x 7168 x 2048 64 / 53 / 14.8 / 17.8,
  //   2000 x 4096 x 768 34 / 35 / 9.6 / 11.6, 4096 x 2880 x 2880 - / 108 / 38 / 26,
  //   8192 x 7168 x 2048 - / - / 96 / 83, 8192^3 - / - / 356 / 262
  const double k = a.K;
  auto items = [&](int64_t n) { return double((a.M + n - 1) / n) * double((a.N + n - 1) / n); };
  const double stream32 =
      2.3 + 1.25e-3 * k + std::max(0.0, items(32) / 256 - 1) * (0.8 + 1.05e-3 * k);
  const double stream64 = (4.5 + 2.2e-3 * k) * std::ceil(items(64) / 256);
  const double cus = cu_count();
  const double ring128 = items(128) <= cus ? 4.5 + 3.2e-3 * k
                                           : (3 + 5.1e-3 * k) * std::ceil(items(128) / (2 * cus));
  const double ring256 = items(256) <= cus / 2 ? 5.5 + 5.2e-3 * k
                                               : (6 + 7.3e-3 * k) * std::ceil(items(256) / cus);
  const double best = std::min(std::min(stream32, stream64), std::min(ring128, ring256));
  // up to 16 rows: units of 16 columns, more of which are at work (1 row, 16 / 32 / 64
  // columns: 7168 x 2048 3.8 / 3.5 / 4.2, 768 x 7168 4.1 / 5.4 / 7.7, 16384^2 22 / 25 / 27)
  if (a.M <= 16) return run_mx_stream<1, 1, 8, false, false>(g, 1, stream);
  if (best == stream32) {
    // few items: more wavefronts for k (32 x 2048 x 7168 11.1 -> 7.3, 64 rows 11.0 -> 7.5,
    // but 64 x 4096 x 4096 7.8 -> 10.8)
    const int64_t mt = (a.M + 31) / 32;
    if (mt * ((a.N + 15) / 16) <= 256) return run_mx_stream<2, 1, 16, false, false>(g, mt, stream);
    return run_mx_stream<2, 2, 8, false, false>(g, mt, stream);
  }
  if (best == stream64) return run_mx_stream<4, 4, 8, false, false>(g, (a.M + 63) / 64, stream);
  return best == ring128 ? run_mx_tiles_out<128, false>(g, stream)
                         : run_mx_tiles_out<256, false>(g, stream);
}

// Workspace of the grouped FFN: the tile count (int at 0), the tile list, and
// the activation's rows with their exponents.
struct MxWs {
  size_t tiles, act, total;
};
static int32_t mx_pair_bytes(int32_t D) { return mx_row_bytes(D) + mx_scale_bytes(D); }
static MxWs mx_ws(int64_t R, int32_t E, int32_t P, int32_t F) {
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  MxWs w;
  w.tiles = 256;
  // the shortest tiles have 16 rows
  w.act = w.tiles + up(size_t(R / 16 + 2 * int64_t(E) + P + 1) * 16);
  w.total = w.act + up(size_t(R) * mx_pair_bytes(F));
  return w;
}
size_t ffn_mxfp4_workspace_bytes(int64_t R, int32_t E, int32_t P, int32_t F) {
  return mx_ws(R, E, P, F).total;
}

// Rows of a tile, by the rows per expert on average (the routing is not known
// here): the stream's 16, or tiles of 128 or 256. Whole layers in us, uniform
// routing unless "hot" (60% of the pairs on four experts):
//   2880 x 2880, 32 experts, 4 of them a token, 16 / 128 / 256 rows:
//     8 tokens 68 / 72 / -, 64 hot 121 / 125 / -, 128 135 / 115 / 120,
//     and 128 / 256: 250 tokens 128 / 125, 400 hot 159 / 153, 1000 204 / 173,
//     8192 hot 902 / 688
//   2048 x 768, 128 experts, 8: 16 tokens 55 / 64 / -, 128 96 / 93 / -,
//     700 - / 121 / 122, 1531 - / 158 / 148, 2200 hot - / 200 / 201, 4096 - / 316 / 282
//   1024 x 768, 16 experts, 2: 100 tokens 30 / 38 / -, 300 36 / 40 / 41,
//     700 47 / 43 / 45, 2000 - / 50 / 59
// (With 32 or 64 rows the stream is slower than the better of these in all of them
// but 300 tokens of the last, 35.)
static int ffn_mxfp4_rows(const FfnMxArgs &a) {
  const int64_t R = a.R, E = a.E, weight = int64_t(a.D) * a.F;
  if (R <= 8 * E || weight * R <= int64_t(500000000)) return 16;
  // 256 rows where many would be valid, and a few rounds of such tiles
  const int64_t tiles = (R / 256 + E) * ((a.F + 127) / 128);
  return R > 30 * E && tiles >= 512 ? 256 : 128;
}

hipError_t launch_ffn_mxfp4(const FfnMxArgs &a, hipStream_t stream) {
  if (a.R == 0) return hipSuccess;
  const MxWs w = mx_ws(a.R, a.E, a.P, a.F);
  char *ws = static_cast<char *>(a.ws);
  int32_t *n_mtiles = reinterpret_cast<int32_t *>(ws);
  int4 *tiles = reinterpret_cast<int4 *>(ws + w.tiles);
  uint8_t *act = reinterpret_cast<uint8_t *>(ws + w.act);
  const int rows = ffn_mxfp4_rows(a);
  hipError_t err = launch_tile_table(a.groups, a.group_begin, 2 * a.E + a.P, a.device, a.P, rows,
                                     tiles, n_mtiles, stream);
  if (err != hipSuccess) return err;
  const int64_t mt_most = a.R / rows + std::min<int64_t>(a.R, 2 * int64_t(a.E) + a.P);
  MxGemmArgs g = mx_weights(a.w_gate_up, 2 * a.F, a.D);
  g.A = reinterpret_cast<const uint16_t *>(a.x_perm);
  g.lda = g.a_scale_pitch = mx_pair_bytes(a.D);
  g.a_scale = a.x_perm + mx_row_bytes(a.D);
  g.groups = a.groups;
  g.tiles = tiles;
  g.n_mtiles = n_mtiles;
  g.act = act;
  g.act_scale = act + mx_row_bytes(a.F);
  g.act_blocks = mx_slices(a.F) * 4;
  g.ldc = mx_pair_bytes(a.F);
  err = rows == 16    ? run_mx_stream<1, 4, 4, true, true>(g, mt_most, stream)
        : rows == 128 ? run_mx_tiles<128, kMxSwiglu, true>(g, stream)
                      : run_mx_tiles<256, kMxSwiglu, true>(g, stream);
  if (err != hipSuccess) return err;
  MxGemmArgs d = mx_weights(a.w_down, a.D, a.F);
  d.A = reinterpret_cast<const uint16_t *>(act);
  d.lda = d.a_scale_pitch = mx_pair_bytes(a.F);
  d.a_scale = act + mx_row_bytes(a.F);
  d.groups = a.groups;
  d.tiles = tiles;
  d.n_mtiles = n_mtiles;
  d.C = static_cast<uint16_t *>(a.out_perm);
  d.ldc = a.D;
  d.f32_out = a.f32_out;
  return rows == 16    ? run_mx_stream<1, 4, 4, true, false>(d, mt_most, stream)
         : rows == 128 ? run_mx_tiles_out<128, true>(d, stream)
                       : run_mx_tiles_out<256, true>(d, stream);
}

}  // namespace llep
