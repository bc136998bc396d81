// Products of 8-bit integers with a scale per token and per channel
// (llep_quantize_rows, llep_int8_matmul, llep_grouped_ffn_int8):
//   C[m][n] = s_a[m] s_b[n] sum_k A[m][k] B[n][k],
// the sum exact in 32-bit integers, so that a result does not depend on which
// kernel ran or how k was split.
//
// Weights are packed (llep_pack_int8) in blocks of 16 rows x 64 k, 1 KB each,
// 16 bytes of each row after another: lane l of a wavefront that reads a block
// in order has what it needs as a matrix-core operand of 16 rows. Two kernels:
//   - tiles (gemm.h): 256 x 256 or 128 x 128 outputs per workgroup, operands
//     through a ring in LDS, bound by the matrix cores, which are 85% busy at the
//     clock that the power limit leaves them (8192^3 490 us, 2240 TOP/s; 8192 x
//     7168 x 2048 131 us; the gate/up and down products of 32768 rows over 32
//     experts of 2880 x 2880 575 and, with float32 outputs, 320 us);
//   - stream (below): the wavefronts of a workgroup split k, for few rows, where
//     reading the weights once is the work (8 tokens, 15 such experts: 66 us,
//     5.7 TB/s).
#include <algorithm>
#include <cmath>

#include "gemm.h"
#include "rows.h"

namespace llep {

// ---------------------------------------------------------------------------
// 8-bit rows: bound by HBM, and read once (8192 x 2880 bf16 16 us, 4.4 TB/s; 32768 x
// 2880 float32 85 us, 5.5 TB/s)
// ---------------------------------------------------------------------------

struct QuantArgs {
  int64_t R;
  int32_t D, q_bytes;
  const void *x;
  int8_t *q;
  float *scale;
  // grouped: the rows of `device`'s groups (or of all), R of them at most
  const int32_t *groups, *group_begin;
  int32_t device, P;
};

// kOdd: rows that are not whole 16-byte vectors, or not on 16-byte boundaries
// (8192 x 2879 bf16 22 us; element by element, twice over the row, 50).
template <typename T, int kPer, bool kOne, bool kOdd>
__global__ __launch_bounds__(kOne ? kRowWaves * kWave : 1024) void quantize_rows_kernel(
    QuantArgs a) {
  constexpr int kVec = 8;
  __shared__ double lds[RowReduce<kOne>::kLds];
  RowReduce<kOne> red(lds);
  const uint32_t n = kOne ? kWave : blockDim.x, t = kOne ? threadIdx.x % kWave : threadIdx.x;
  const uint32_t D = a.D;
  int64_t r0 = 0, r1 = a.R;
  if (a.groups) {
    const int lo = a.device < 0 ? a.group_begin[0] : a.group_begin[a.device];
    const int hi = a.device < 0 ? a.group_begin[a.P] : a.group_begin[a.device + 1];
    r0 = lo < hi ? a.groups[4 * lo + 2] : 0;
    r1 = lo < hi ? a.groups[4 * (hi - 1) + 2] + a.groups[4 * (hi - 1) + 3] : 0;
  }
  const int64_t step = int64_t(gridDim.x) * (kOne ? kRowWaves : 1);
  int64_t row = r0 + (kOne ? int64_t(blockIdx.x) * kRowWaves +
                                 __builtin_amdgcn_readfirstlane(threadIdx.x / kWave)
                           : blockIdx.x);
  RawVec<T, kVec> next[kPer];
  auto request = [&]() {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t c = (j * n + t) * kVec;
      next[j].zero();
      if (c >= D) continue;
      const T *p = static_cast<const T *>(a.x) + row * D + c;
      if constexpr (kOdd)
        next[j].load_any(p, int(D - c));
      else
        next[j].load(p);
    }
  };
  constexpr bool kAhead = kPer == 1;  // else there are no registers for it
  if (kAhead && row < r1) request();
  while (row < r1) {
    if (!kAhead) request();
    float v[kPer][kVec];
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        v[j][i] = next[j][i];
        most = max(most, __float_as_uint(fabsf(v[j][i])));
      }
    const int64_t at = row;
    row += step;
    if (kAhead && row < r1) request();  // the next row, while this one is worked on
    const RowScale s = row_scale(red.max_bits(most));
    store_int8_row<kVec, kPer>(a.q + at * a.q_bytes, D, a.q_bytes, t, n, v, s);
    if (t == 0) a.scale[at] = s.scale;
  }
}

constexpr int kQuantWaves = 24;  // of a compute unit that the grid is sized for

template <typename T, int kPer, bool kOne, bool kOdd>
hipError_t run_quantize(const QuantArgs &a, hipStream_t stream) {
  const int threads = kOne ? kRowWaves * kWave : row_threads(a.D, 8, kPer);
  const int64_t wgs = kOne ? (a.R + kRowWaves - 1) / kRowWaves : a.R;
  const int64_t grid = std::min<int64_t>(wgs, 256 * std::max(1, kQuantWaves * kWave / threads));
  hipLaunchKernelGGL((quantize_rows_kernel<T, kPer, kOne, kOdd>), dim3(uint32_t(grid)), dim3(threads), 0,
                     stream, a);
  return hipGetLastError();
}

template <typename T>
hipError_t quantize_t(const QuantArgs &a, hipStream_t stream) {
  if (a.R == 0) return hipSuccess;
  const bool whole = a.D % 8 == 0 && (reinterpret_cast<uintptr_t>(a.x) & 15) == 0;
  static_assert(LLEP_MAX_FFN_DIM == 1024 * 8 * 8, "a row fits a workgroup");
  if (a.D <= 512)
    return whole ? run_quantize<T, 1, true, false>(a, stream)
                 : run_quantize<T, 1, true, true>(a, stream);
  if (a.D <= 8192)
    return whole ? run_quantize<T, 1, false, false>(a, stream)
                 : run_quantize<T, 1, false, true>(a, stream);
  return whole ? run_quantize<T, 8, false, false>(a, stream)
               : run_quantize<T, 8, false, true>(a, stream);
}

hipError_t launch_quantize_rows(int64_t R, int32_t D, llep_dtype dtype, const void *x, int8_t *q,
                                int32_t q_bytes, float *scale, hipStream_t stream) {
  QuantArgs a = {};
  a.R = R;
  a.D = D;
  a.q_bytes = q_bytes;
  a.x = x;
  a.q = q;
  a.scale = scale;
  return dtype == LLEP_BF16 ? quantize_t<uint16_t>(a, stream) : quantize_t<float>(a, stream);
}

// ---------------------------------------------------------------------------
// packing: 16 bytes of a packed row per thread
// ---------------------------------------------------------------------------

__global__ __launch_bounds__(256) void pack_int8_kernel(const int8_t *__restrict__ w0,
                                                        const int8_t *__restrict__ w1, int64_t E,
                                                        int32_t N, int32_t K, int32_t Np,
                                                        int32_t Kp, int8_t *__restrict__ out) {
  const int64_t chunks = E * (int64_t(Np) * Kp / 16);
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < chunks;
       i += int64_t(gridDim.x) * 256) {
    const int64_t blk = i >> 6;
    const int kbs = Kp / 64;
    const int kb = int(blk % kbs), nb = int(blk / kbs % (Np / 16));
    const int64_t e = blk / kbs / (Np / 16);
    int n = nb * 16 + (int(i) & 15);
    const int k = kb * 64 + (int(i) >> 4 & 3) * 16;
    // two matrices: 32 rows of the first, then the matching 32 of the second
    const int8_t *src = w0;
    bool ok = n < N;
    if (w1) {
      src = n & 32 ? w1 : w0;
      n = (n >> 6) * 32 + (n & 31);
      ok = n < N;
    }
    uint32_t v[4] = {0u, 0u, 0u, 0u};
    if (ok) {
      const int8_t *p = src + (e * N + n) * K + k;
      if (K % 16 == 0 && (reinterpret_cast<uintptr_t>(src) & 15) == 0) {
        if (k < K) {
          const uint4 q = *reinterpret_cast<const uint4 *>(p);
          v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
        }
      } else {
#pragma unroll
        for (int b = 0; b < 16; ++b)
          if (k + b < K) v[b / 4] |= (uint32_t(p[b]) & 255u) << (8 * (b % 4));
      }
    }
    reinterpret_cast<uint4 *>(out)[i] = make_uint4(v[0], v[1], v[2], v[3]);
  }
}

hipError_t launch_pack_int8(int32_t E, int32_t N, int32_t K, const int8_t *w0, const int8_t *w1,
                            int8_t *out, hipStream_t stream) {
  const int32_t Np = w1 ? 2 * N : (N + 15) / 16 * 16, Kp = (K + 63) / 64 * 64;
  const int64_t blocks = (E * (int64_t(Np) * Kp / 16) + 255) / 256;
  hipLaunchKernelGGL(pack_int8_kernel, dim3(uint32_t(std::min<int64_t>(blocks, 65536))), dim3(256),
                     0, stream, w0, w1, int64_t(E), N, K, Np, Kp, out);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// stream: few rows
//
// An item is up to 16 kMB rows of one group (of A, dense) by 16 kNB packed
// rows of the weights; a workgroup of kWaves wavefronts takes one item at a
// time, each wavefront a part of k, and adds the parts up through LDS.
// v_mfma_i32_16x16x64_i8 takes a 1 KB block of the weights as its first
// operand (lane l: row l % 16, bytes 16 (l / 16) .. + 15 of its 64: the block in
// order; rows of 64 bytes one after another took 10% longer), 16 rows of A as
// its second; lane l then holds, of row l % 16 of A, the columns
// 4 (l / 16) .. + 3. Every XCD (workgroups are dealt round-robin over the 8)
// takes a contiguous eighth of the items: dense ones with the row tiles of a
// weight unit next to each other, so that its weights come to one L2 once;
// grouped ones with the units of a row tile next to each other.
// ---------------------------------------------------------------------------

template <int kMB, int kNB, int kWaves, bool kGrouped, bool kSwigluOut, bool kOnce>
__global__ __launch_bounds__(kWaves * kWave) void int8_stream_kernel(Int8GemmArgs g) {
  constexpr int kBlocks = kMB * kNB;
  // With more than 16 rows, A goes through LDS (kStaged): a wavefront that
  // reads 16 rows for an operand touches 16 lines with every quarter of its
  // lanes, four times the work of the same bytes in order.
  constexpr bool kStaged = kMB > 1;
  // blocks of k requested together (two where all of the chip's wavefronts are
  // at work: more of them fit; an expert layer of 8 tokens, 15 experts of 2880 x
  // 2880, 97.5 -> 95.7 us), and 16 x 16 blocks of the outputs whose parts are in
  // LDS at a time
  constexpr int kUnroll = kStaged ? 1 : kOnce ? 2 : 4;
  constexpr int kRound = kBlocks >= 16 ? 8 : kBlocks;
  constexpr int kStage = kUnroll * kMB * 1024;  // bytes of A per wavefront, twice
  constexpr int kLdsBytes = kStaged && 2 * kStage > kRound * 1024 ? 2 * kStage : kRound * 1024;
  __shared__ __attribute__((aligned(1024))) char lds[kWaves * kLdsBytes];
  i32x4 (*part)[kRound][kWave] = reinterpret_cast<i32x4 (*)[kRound][kWave]>(lds);
  static_assert(!kSwigluOut || kNB == 4 || kNB == 2, "gate blocks and the matching up blocks");
  static_assert(kBlocks % kRound == 0 && kRound % kNB == 0, "rounds of whole rows of blocks");
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int nkb = g.Kdim / 32;               // blocks of 64 k
  const int n_blk = (g.N + 15) / 16;         // blocks of 16 packed rows
  const int n_unit = (n_blk + kNB - 1) / kNB;
  const int n_mt = kGrouped ? *g.n_mtiles : int((g.M + 16 * kMB - 1) / (16 * kMB));
  const int kb0 = nkb * wave / kWaves, kb1 = nkb * (wave + 1) / kWaves;
  const int64_t items = int64_t(n_mt) * n_unit;
  const int xcd = blockIdx.x % 8;
  const int64_t end = items * (xcd + 1) / 8;
  for (int64_t item = items * xcd / 8 + blockIdx.x / 8; item < end; item += gridDim.x / 8) {
    const int mt = int(kGrouped ? item / n_unit : item % n_mt);
    const int unit = int(kGrouped ? item % n_unit : item / n_mt);
    int e = 0;
    int64_t row0 = int64_t(mt) * 16 * kMB;
    int rows;
    bool lone = n_mt == 1;  // no other row tile of the same weights
    if (kGrouped) {
      const int4 te = g.tiles[mt];
      const int32_t *gr = g.groups + 4 * te.x;
      e = gr[1];
      row0 = int64_t(gr[2]) + te.y * 16 * kMB;
      rows = min(16 * kMB, gr[3] - te.y * 16 * kMB);
      lone = __builtin_amdgcn_readfirstlane(gr[3]) <= 16 * kMB;
    } else {
      rows = int(min<int64_t>(16 * kMB, g.M - row0));
    }
    const int8_t *A = reinterpret_cast<const int8_t *>(g.A) + row0 * g.lda * 2;
    // first packed block of the unit, and from one of its blocks to the next:
    // with two blocks a unit is 16 gate rows and the matching up rows
    constexpr int kApart = kSwigluOut && kNB == 2 ? 2 : 1;
    const int blk0 = kApart == 2 ? 4 * (unit >> 1) + (unit & 1) : unit * kNB;
    const int8_t *B = reinterpret_cast<const int8_t *>(g.B) + e * g.b_expert_stride * 2 +
                      int64_t(blk0) * g.b_blk_stride;
    uint32_t offA[kMB], offB[kNB];
#pragma unroll
    for (int m = 0; m < kMB; ++m)  // past the last row: the last one again, not stored
      offA[m] = uint32_t(min(m * 16 + (lane & 15), rows - 1)) * uint32_t(g.lda * 2) + (lane >> 4) * 16;
#pragma unroll
    for (int n = 0; n < kNB; ++n)  // and past the last block
      offB[n] = uint32_t(min(n * kApart, n_blk - 1 - blk0)) * uint32_t(g.b_blk_stride) +
                lane * 16;
    i32x4 acc[kMB][kNB];
#pragma unroll
    for (int m = 0; m < kMB; ++m)
#pragma unroll
      for (int n = 0; n < kNB; ++n) acc[m][n] = i32x4{0, 0, 0, 0};
    // past: the weights are read past the caches
    auto product = [&](auto past) {
      auto load_weights = [](const int8_t *p) {
        if constexpr (decltype(past)::value)
          return __builtin_nontemporal_load(reinterpret_cast<const i32x4 *>(p));
        else
          return *reinterpret_cast<const i32x4 *>(p);
      };
      if constexpr (kStaged) {
        // One step of kUnroll blocks of k ahead: its rows of A on their way to
        // the wavefront's other half of LDS (lane l: row l / 4 of 16, 16 bytes of
        // it), its weights to registers; the wait at the top of a step is for
        // everything, so both are there. No barrier: each wavefront has its own
        // part of LDS. Blocks past the last one are the last again, not used.
        const char *stage = lds + wave * kLdsBytes;
        const uint32_t stage_at = lds_addr(lds) + wave * kLdsBytes;
        int32_t offS[kMB];
#pragma unroll
        for (int m = 0; m < kMB; ++m)
          offS[m] = min(m * 16 + (lane >> 2), rows - 1) * int32_t(g.lda * 2) +
                    (((lane & 3) ^ ((lane >> 4) & 3)) << 4);
        i32x4 fb[kUnroll][kNB];
        auto request = [&](int kb, int half) {
#pragma unroll
          for (int u = 0; u < kUnroll; ++u) {
            const int k = min(kb + u, kb1 - 1);
#pragma unroll
            for (int m = 0; m < kMB; ++m)
              dma16(reinterpret_cast<const char *>(A) + k * 64, offS[m],
                    stage_at + half * kStage + (u * kMB + m) * 1024);
#pragma unroll
            for (int n = 0; n < kNB; ++n)
              fb[u][n] = load_weights(B + int64_t(k) * 1024 + offB[n]);
          }
        };
        if (kb0 < kb1) request(kb0, 0);
        int half = 0;
        for (int kb = kb0; kb < kb1; kb += kUnroll) {
          asm volatile("" ::: "memory");
          wait_cnt<0, 0>();
          asm volatile("" ::: "memory");
          i32x4 now[kUnroll][kNB];
#pragma unroll
          for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int n = 0; n < kNB; ++n) now[u][n] = fb[u][n];
          if (kb + kUnroll < kb1) request(kb + kUnroll, half ^ 1);
#pragma unroll
          for (int u = 0; u < kUnroll; ++u) {
            if (kb + u >= kb1) break;
#pragma unroll
            for (int m = 0; m < kMB; ++m) {
              const int r = lane & 15;
              const i32x4 fa = *reinterpret_cast<const i32x4 *>(
                  stage + half * kStage + (u * kMB + m) * 1024 + r * 64 +
                  (((lane >> 4) ^ ((r >> 2) & 3)) << 4));
#pragma unroll
              for (int n = 0; n < kNB; ++n)
                acc[m][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(now[u][n], fa, acc[m][n], 0, 0, 0);
            }
          }
          half ^= 1;
        }
        // the parts below go over the stages: every wavefront's reads are done
        asm volatile("" ::: "memory");
        wait_cnt<0, 0>();
        __syncthreads();
      } else {
        auto steps = [&](auto count, int kb) {
          constexpr int kU = decltype(count)::value;
          i32x4 fa[kU][kMB], fb[kU][kNB];
#pragma unroll
          for (int u = 0; u < kU; ++u) {
#pragma unroll
            for (int n = 0; n < kNB; ++n)
              fb[u][n] = load_weights(B + int64_t(kb + u) * 1024 + offB[n]);
#pragma unroll
            for (int m = 0; m < kMB; ++m)
              fa[u][m] = *reinterpret_cast<const i32x4 *>(A + (kb + u) * 64 + offA[m]);
          }
#pragma unroll
          for (int u = 0; u < kU; ++u)
#pragma unroll
            for (int m = 0; m < kMB; ++m)
#pragma unroll
              for (int n = 0; n < kNB; ++n)
                acc[m][n] =
                    __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[u][n], fa[u][m], acc[m][n], 0, 0, 0);
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
      }
    };
    if (kOnce && lone)
      product(std::true_type{});
    else
      product(std::false_type{});
#pragma unroll
    for (int b0 = 0; b0 < kBlocks; b0 += kRound) {
#pragma unroll
      for (int b = 0; b < kRound; ++b)
        part[wave][b][lane] = acc[(b0 + b) / kNB][(b0 + b) % kNB];
      __syncthreads();
      // the sum over the wavefronts of a block
      auto total = [&](int b) {
        i32x4 s = part[0][b][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) s += part[w][b][lane];
        return s;
      };
      if constexpr (kSwigluOut) {
        constexpr int kHalf = kNB / 2;  // blocks of 16 activation columns
        const int F = g.N / 2;
        for (int q = wave; q < kRound / 2; q += kWaves) {
          const int m = q / kHalf, half = q % kHalf;
          const int r = (b0 / kNB + m) * 16 + (lane & 15);
          const int col = unit * kHalf * 16 + half * 16 + (lane >> 4) * 4;
          if (r >= rows) continue;
          const i32x4 sg = total(m * kNB + half), su = total(m * kNB + kHalf + half);
          const float sa = int8_row_scale(g, row0 + r);
          const f32x4 cg = int8_col_scales(g.b_scale + e * g.scale_stride, col, F);
          const f32x4 cu = int8_col_scales(g.b_scale2 + e * g.scale_stride, col, F);
          f32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            v[i] = int8_swiglu(int8_value(sg[i], sa, cg[i]), int8_value(su[i], sa, cu[i]));
          *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(g.C) + (row0 + r) * F + col) = v;
        }
      } else {
        for (int q = wave; q < kRound; q += kWaves) {
          const int m = q / kNB, n = q % kNB;
          const int r = (b0 / kNB + m) * 16 + (lane & 15);
          const int col = (unit * kNB + n) * 16 + (lane >> 4) * 4;
          if (r >= rows || col >= g.N) continue;
          const i32x4 s = total(q);
          const float sa = int8_row_scale(g, row0 + r);
          const f32x4 cb = int8_col_scales(g.b_scale + e * g.scale_stride, col, g.N);
          f32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = int8_value(s[i], sa, cb[i]);
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

// ---------------------------------------------------------------------------
// tiles
// ---------------------------------------------------------------------------

// BM x BN tiles: 256 rows by eight wavefronts, one workgroup on a compute unit,
// or 128 x 128 by four, two workgroups; two wavefronts per SIMD either way.
template <int BM, int BN, int WAVES_M, int WAVES_N, int kEpi, bool kGrouped>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N) __attribute__((amdgpu_waves_per_eu(2, 2)))
void int8_tiles_kernel(Int8GemmArgs g) {
  __shared__ __attribute__((aligned(1024))) char smem[ring_bytes<BN, BM>()];
  std::conditional_t<kGrouped, LaunchSched<BM, BN>, DenseSched<BM, BN>> sched(g);
  TileCoord t;
  if (!sched.first(t)) return;
  gemm_tiles<BN, WAVES_M, WAVES_N, kEpi, false, false>(g, smem, t, sched);
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int kEpi, bool kGrouped>
hipError_t run_int8_tiles(const Int8GemmArgs &g, hipStream_t stream) {
  int64_t most = cu_count() * (BM == 256 ? 1 : 2);
  // few dense tiles: as many workgroups, so that all XCDs have as many of them
  // (2048^3 in 256 tiles 24 -> 15 us)
  if (!kGrouped) most = std::min(most, (g.M + BM - 1) / BM * ((g.N + BN - 1) / BN));
  const int grid = int((most + 7) / 8 * 8);
  hipLaunchKernelGGL((int8_tiles_kernel<BM, BN, WAVES_M, WAVES_N, kEpi, kGrouped>), dim3(grid),
                     dim3(64 * WAVES_M * WAVES_N), 0, stream, g);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// launch
// ---------------------------------------------------------------------------

template <int kMB, int kNB, int kWaves, bool kGrouped, bool kSwigluOut, bool kOnce>
hipError_t run_int8_stream(const Int8GemmArgs &g, int64_t mtiles, hipStream_t stream) {
  const int64_t items = mtiles * ((g.N + 16 * kNB - 1) / (16 * kNB));
  const int grid = int(std::min<int64_t>((items + 7) / 8 * 8, 16384));
  hipLaunchKernelGGL((int8_stream_kernel<kMB, kNB, kWaves, kGrouped, kSwigluOut, kOnce>),
                     dim3(grid), dim3(kWaves * kWave), 0, stream, g);
  return hipGetLastError();
}

// The stream for `mtiles` row tiles (at most) of at most `rows` rows: 16, 32 or
// (dense) 64; bytes: of the weights that the call reads, at most (grouped: as
// many experts as there are rows, or all; the routing is not known here).
// - With up to 256 units of 64 columns k is split over eight wavefronts (4 / 8:
//   64 x 7168 x 2048 7.0 / 6.5 us, 32 x 7168 x 7168 15.7 / 12.9, but 333 x 2880 x
//   1024, 270 units, 7.5 / 9.3). With many, a workgroup takes 64 x 128 outputs,
//   with fewer bytes from the L2 per product (2048^3 26 / 22 us, 512 x 7168 x
//   2048 21 / 18).
// - Up to 16 rows, with few weights, k is split so that about 1024 wavefronts
//   are at work (1 row, N x K = 7168 x 2048 with 4 / 8 / 16: 5.6 / 3.8 / 4.7 us;
//   768 x 7168: 9.4 / - / 4.9 us).
// - Weights of more than half of the 256 MB cache behind the L2s are read past
//   the caches by row tiles that have them to themselves, and for 16 rows in
//   units of 32 packed rows, whose last ones end together (15 experts of 2880 x
//   2880 in use, 376 MB: 105 -> 98 -> 94 us; 32 rows, 32 such experts 195 -> 174;
//   but 4 of them, 100 MB, the same four in every call: 44 -> 49 us, which a
//   hot call, or one device's share, of a layer with many experts takes too).
template <bool kGrouped, bool kSwigluOut>
hipError_t launch_int8_stream(const Int8GemmArgs &g, int rows, int64_t mtiles, int64_t bytes,
                              hipStream_t stream) {
  constexpr bool G = kGrouped, S = kSwigluOut;
  const int64_t units = mtiles * ((g.N + 63) / 64);  // of 64 packed rows
  if constexpr (!G)
    if (rows > 32) {
      if (units >= 800) return run_int8_stream<4, 8, 4, G, S, false>(g, mtiles, stream);
      return units <= 256 ? run_int8_stream<4, 4, 8, G, S, false>(g, mtiles, stream)
                          : run_int8_stream<4, 4, 4, G, S, false>(g, mtiles, stream);
    }
  const bool once = bytes > (int64_t(128) << 20);
  if (rows > 16 && G && once) return run_int8_stream<2, 4, 4, G, S, G>(g, mtiles, stream);
  if (rows > 16)
    return units <= 256 ? run_int8_stream<2, 4, 8, G, S, false>(g, mtiles, stream)
                        : run_int8_stream<2, 4, 4, G, S, false>(g, mtiles, stream);
  if (units * 4 >= 1024)
    return once ? run_int8_stream<1, 2, 4, G, S, true>(g, mtiles, stream)
                : run_int8_stream<1, 4, 4, G, S, false>(g, mtiles, stream);
  if (S || units * 16 >= 1024) return run_int8_stream<1, 2, 8, G, S, false>(g, mtiles, stream);
  if constexpr (!S) return run_int8_stream<1, 1, 16, G, S, false>(g, mtiles, stream);
  return hipErrorInvalidValue;
}

hipError_t launch_int8_matmul(const Int8MatmulArgs &a, hipStream_t stream) {
  if (a.M == 0) return hipSuccess;
  Int8GemmArgs g = {};
  const int32_t Kp = (a.K + 63) / 64 * 64;
  g.A = reinterpret_cast<const uint16_t *>(a.x);
  g.lda = a.x_bytes / 2;
  g.B = reinterpret_cast<const uint16_t *>(a.w);
  g.b_blk_stride = int64_t(Kp) * 16;
  g.C = static_cast<uint16_t *>(a.out);
  g.ldc = a.N;
  g.N = a.N;
  g.Kdim = Kp / 2;
  g.a_scale = a.x_scale;
  g.b_scale = a.w_scale;
  g.M = a.M;
  g.f32_out = a.dtype == LLEP_F32;
  // The least of what the three ways take in us, about: the stream by its
  // multiply-adds (rows in 64s) and outputs, the tiles by 64-byte slices of k and
  // rounds of as many workgroups as the chip has room for (128 x 128 tiles: two
  // on a compute unit, which take twice as long as one). Stream / 128 / 256 rows:
  //   2048^3 21 / 15 / 25, 512 x 2048 x 7168 18 / 31 / 60, 512 x 7168 x 2048
  //   17 / 14 / 24, 1024 x 7168 x 2048 30 / 22 / 26, 2048 x 2880 x 2880 35 / 26 / 32,
  //   2000 x 4096 x 768 20 / 13 / 16, 6000 x 768 x 2048 28 / 20 / 25,
  //   2048 x 7168 x 2048 57 / 42 / 33, 4096 x 2880 x 2880 66 / 55 / 38,
  //   8192 x 7168 x 2048 220 / 146 / 131, 200 x 7168 x 7168 25 / 32 / 60
  const double slices = Kp / 64, cus = cu_count(), m64 = double((a.M + 63) / 64 * 64);
  auto tiles = [&](int64_t n) { return double((a.M + n - 1) / n) * double((a.N + n - 1) / n); };
  const double streamed = 3 + m64 * double(a.N) * (1.0e-6 + 1.8e-9 * double(Kp));
  const double ring128 = tiles(128) <= cus ? 5.5 + 0.25 * slices
                                           : (4.5 + 0.5 * slices) * std::ceil(tiles(128) / (2 * cus));
  const double ring256 = (12 + 0.65 * slices) * std::ceil(tiles(256) / cus);
  if (a.M <= 64 || streamed < std::min(ring128, ring256)) {
    const int rows = a.M <= 16 ? 16 : a.M <= 32 ? 32 : 64;
    return launch_int8_stream<false, false>(g, rows, (a.M + rows - 1) / rows,
                                            int64_t(a.N) * Kp, stream);
  }
  if (ring128 < ring256) return run_int8_tiles<128, 128, 2, 2, kEpiInt8, false>(g, stream);
  return run_int8_tiles<256, 256, kWavesM, kWavesN, kEpiInt8, false>(g, stream);
}

// Workspace of the grouped FFN: the tile count (int at 0), the tile list, the
// rows' activation scales, the activations in float32 and then in 8 bits.
struct Int8Ws {
  size_t tiles, scale, act, act_q, total;
};
static Int8Ws int8_ws(int64_t R, int32_t E, int32_t P, int32_t F) {
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  Int8Ws w;
  w.tiles = 256;
  // the shortest tiles have 16 rows
  w.scale = w.tiles + up(size_t(R / 16 + 2 * int64_t(E) + P + 1) * 16);
  w.act = w.scale + up(size_t(R) * 4);
  w.act_q = w.act + up(size_t(R) * F * 4);
  w.total = w.act_q + up(size_t(R) * F);
  return w;
}

size_t ffn_int8_workspace_bytes(int64_t R, int32_t E, int32_t P, int32_t F) {
  return int8_ws(R, E, P, F).total;
}

// Rows of a tile, by the rows per expert on average (the routing is not known
// here): the stream's 16 or 32, or 128 or 256 rows through the ring. Whole
// layers (float32 outputs of the experts) in us, uniform routing unless "hot"
// (60% of the pairs on four experts; "warm": on 16):
//   2880 x 2880, 32 experts, 4 of them a token, 16 / 32 / 128 / 256 rows:
//     32 tokens 147 / 153 / 178 / 180, 128 tokens 198 / 167 / 193 / 189,
//     and 32 / 128 / 256: 250 tokens 233 / 204 / 217, 400 tokens 295 / 227 / 217,
//     hot 272 / 251 / 251, 1000 tokens hot 529 / 322 / 298
//   2048 x 768, 128 experts, 8, 32 / 128 / 256 rows: 400 tokens 158 / 159 / 161,
//     700 tokens 208 / 175 / 179, 1531 tokens warm 308 / 249 / 271,
//     2200 tokens hot 397 / 274 / 295, 3000 tokens 487 / 325 / 307
//   1024 x 768, 16 experts, 2: 300 tokens 41 / 50 / 51, 700 tokens 48 / 56 / 57,
//     1200 tokens hot 61 / 61 / 70, 2000 tokens 72 / 62 / 76
static int ffn_int8_rows(const FfnInt8Args &a) {
  const int64_t R = a.R, E = a.E, weight = int64_t(a.D) * a.F;
  if (R <= 8 * E) return 16;
  // up to 24 rows an expert the weights are most of the work; small layers have
  // too few tiles for the chip
  if (R <= 24 * E || weight * R <= int64_t(1500000000)) return 32;
  // 256 rows where most would be valid (long products: fewer), and a few rounds
  // of such tiles
  const int64_t tiles = (R / 256 + E) * ((a.F + 127) / 128);
  return (R > 128 * E || (weight > 2000000 && R > 40 * E)) && tiles >= 512 ? 256 : 128;
}

hipError_t launch_ffn_int8(const FfnInt8Args &a, hipStream_t stream) {
  if (a.R == 0) return hipSuccess;
  const Int8Ws w = int8_ws(a.R, a.E, a.P, a.F);
  char *ws = static_cast<char *>(a.ws);
  int32_t *n_mtiles = reinterpret_cast<int32_t *>(ws);
  int4 *tiles = reinterpret_cast<int4 *>(ws + w.tiles);
  float *act = reinterpret_cast<float *>(ws + w.act);
  int8_t *act_q = reinterpret_cast<int8_t *>(ws + w.act_q);
  float *act_scale = reinterpret_cast<float *>(ws + w.scale);
  const int rows = ffn_int8_rows(a);
  const bool streams = rows <= 32;
  const int64_t bytes = 3 * std::min<int64_t>(a.R, a.E) * a.D * a.F;  // of the weights, at most
  hipError_t err = launch_tile_table(a.groups, a.group_begin, 2 * a.E + a.P, a.device, a.P, rows,
                                     tiles, n_mtiles, stream);
  if (err != hipSuccess) return err;
  const int64_t mt_most = a.R / rows + std::min<int64_t>(a.R, 2 * int64_t(a.E) + a.P);
  Int8GemmArgs g = {};
  g.A = reinterpret_cast<const uint16_t *>(a.x_perm);
  g.lda = a.D / 2;
  g.B = reinterpret_cast<const uint16_t *>(a.w_gate_up);
  g.b_expert_stride = int64_t(a.F) * a.D;
  g.b_blk_stride = int64_t(a.D) * 16;
  g.C = reinterpret_cast<uint16_t *>(act);
  g.ldc = a.F;
  g.groups = a.groups;
  g.tiles = tiles;
  g.n_mtiles = n_mtiles;
  g.N = 2 * a.F;
  g.Kdim = a.D / 2;
  g.a_scale = a.x_scale;
  g.row_pair = a.row_pair;
  g.K = a.K;
  g.b_scale = a.gate_scale;
  g.b_scale2 = a.up_scale;
  g.scale_stride = a.F;
  if (streams) {
    err = launch_int8_stream<true, true>(g, rows, mt_most, bytes, stream);
  } else {
    err = rows == 128 ? run_int8_tiles<128, 128, 2, 2, kEpiInt8Swiglu, true>(g, stream)
                      : run_int8_tiles<256, 256, kWavesM, kWavesN, kEpiInt8Swiglu, true>(g, stream);
  }
  if (err != hipSuccess) return err;
  QuantArgs q = {};
  q.R = a.R;
  q.D = q.q_bytes = a.F;
  q.x = act;
  q.q = act_q;
  q.scale = act_scale;
  // all devices: every row, without a look at the groups (a row that a bad id
  // leaves empty is not read afterwards)
  q.groups = a.device < 0 ? nullptr : a.groups;
  q.group_begin = a.group_begin;
  q.device = a.device;
  q.P = a.P;
  if ((err = quantize_t<float>(q, stream)) != hipSuccess) return err;
  Int8GemmArgs d = g;
  d.A = reinterpret_cast<const uint16_t *>(act_q);
  d.lda = a.F / 2;
  d.B = reinterpret_cast<const uint16_t *>(a.w_down);
  d.b_expert_stride = int64_t(a.D) * a.F / 2;
  d.b_blk_stride = int64_t(a.F) * 16;
  d.C = static_cast<uint16_t *>(a.out_perm);
  d.ldc = a.D;
  d.N = a.D;
  d.Kdim = a.F / 2;
  d.a_scale = act_scale;
  d.row_pair = nullptr;
  d.b_scale = a.down_scale;
  d.scale_stride = a.D;
  d.f32_out = a.f32_out;
  if (streams) return launch_int8_stream<true, false>(d, rows, mt_most, bytes, stream);
  if (a.f32_out)
    return rows == 128 ? run_int8_tiles<128, 128, 2, 2, kEpiInt8F32, true>(d, stream)
                       : run_int8_tiles<256, 256, kWavesM, kWavesN, kEpiInt8F32, true>(d, stream);
  if (rows == 128) return run_int8_tiles<128, 128, 2, 2, kEpiInt8, true>(d, stream);
  return run_int8_tiles<256, 256, kWavesM, kWavesN, kEpiInt8, true>(d, stream);
}

}  // namespace llep
