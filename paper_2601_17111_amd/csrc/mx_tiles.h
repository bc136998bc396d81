// Tiles of 4-bit products (mxfp4.hip): C[m][n] = sum over slices of A[m] B_e[n],
// BM x BN outputs per workgroup.
//
// As in gemm.h, operands go global -> LDS by DMA through a ring of slices (64
// bytes of a row: 128 values), the matrix cores' operands are read from LDS one
// step ahead, and half of the wavefronts issue the DMA. The other half requests
// the exponents, 16 bytes of every row for four slices at a time, into one of two
// buffers behind the ring: they have no other loads in flight, so that waiting
// for the exponents, four slices after they were asked for, is waiting for
// everything, and the counts of the first half's DMA stay constant. (The four bytes
// of a slice are read 16 bytes apart for A, 8 cycles a wavefront where 2 are possible;
// with words next to each other, requested as words or written by the scale waves,
// the products took 3 to 6% longer.)
//
// What bounds them: 8192^3 takes 258 to 274 us by the card, 4.0 to 4.3 PFLOP/s; the
// matrix instructions are at work 61% of the time, at the 1.6 GHz that the chip's power
// leaves (of 2.4: matrix instructions alone, on random operands, reach 6.2 PFLOP/s). A
// tile's epilogue is 4.5 us of 21 (K = 2048). Requests into the L2 four to eight slices
// further ahead made products 5 to 10% slower, half tiles in a last round that leaves
// workgroups idle were no faster.
#pragma once

#include "gemm.h"

namespace llep {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------------------
// 4-bit values: sign, two bits of exponent, one of fraction (0, 0.5, 1, 1.5, 2,
// 3, 4, 6). The exponent of a block whose largest magnitude has the (biased)
// exponent field e is e - 2 (4 = 2^2 is the largest power of two among the
// values), at least 1; a block with an infinity or a NaN gets 255, which makes
// all of it NaN. Values are rounded to the nearest, ties to the even one, and
// are at most 6.
// ---------------------------------------------------------------------------

__device__ __forceinline__ uint32_t mx_exponent(uint32_t most_bits) {
  const uint32_t e = most_bits >> 23;
  return e == 255u ? 255u : uint32_t(max(int(e) - 2, 1));
}
// the power of two (of 255: any number, the values do not matter)
__device__ __forceinline__ float mx_step(uint32_t exponent) {
  return __uint_as_float(min(exponent, 254u) << 23);
}
// four values in 16 bits
__device__ __forceinline__ uint32_t mx_pack4(float a, float b, float c, float d, float step) {
  uint32_t v = 0;
  v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, a, b, step, 0);
  v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, c, d, step, 1);
  return v;
}

// A: rows of lda bytes (64 a slice) with their exponents a_scale_pitch bytes
// apart; of the base, lda and b_expert_stride count bytes here, Kdim 32 a slice.
struct MxGemmArgs : GemmArgs {
  const uint8_t *a_scale;
  int64_t a_scale_pitch;
  int64_t b_scale_at;          // of an expert's exponents behind its values, bytes
  int64_t b_scale_blk_stride;  // bytes per 16-row block across all of K
  int64_t M;                   // dense: rows of A
  bool f32_out;
  // SwiGLU: rows of ldc bytes of values, and their exponents
  uint8_t *act, *act_scale;
  int32_t act_blocks;          // exponents of a row that a product reads
};

// The operand of 32 values is 16 bytes (the builtin's other half is not read).
__device__ __forceinline__ i32x8 mx_operand(const i32x4 v) {
  return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1);
}
// the exponents are bytes kSel of the two scale operands
template <int kSel>
__device__ __forceinline__ f32x4 mx_mfma(const i32x4 b, const i32x4 a, const f32x4 c, int sb, int sa) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(b), mx_operand(a), c, 4, 4,
                                                          kSel, sb, kSel, sa);
}
template <int kSel>
__device__ __forceinline__ f32x16 mx_mfma(const i32x4 b, const i32x4 a, const f32x16 c, int sb, int sa) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_operand(b), mx_operand(a), c, 4, 4,
                                                         kSel, sb, kSel, sa);
}
__device__ __forceinline__ float mx_swiglu(float g, float u) {
  return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u;
}
// the exponents behind a row's last block, up to those that a product reads
__device__ __forceinline__ void mx_pad_scales(uint8_t *row, int blocks, int read) {
  for (int b = blocks; b < read; ++b) row[b] = 127;
}

constexpr int kMxAhead = 3;  // slices requested ahead of the one being read
constexpr int kMxStages = kMxAhead + 1;

template <int BM, int BN>
constexpr uint32_t mx_ring_bytes() {
  return uint32_t(kMxStages) * (BM + BN) * 64 + 2 * (BM + BN) * 16;
}

// What becomes of the outputs.
enum MxEpilogue : int { kMxBf16 = 0, kMxF32 = 1, kMxSwiglu = 2 };

template <int BN, int WAVES_M, int WAVES_N, int kEpi, class Sched>
__device__ __forceinline__ void mx_tiles(const MxGemmArgs g, char *smem, TileCoord t, Sched &sched) {
  constexpr int BM = Sched::kBM;
  constexpr int NW = WAVES_M * WAVES_N, NWD = NW / 2;
  constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N;
  constexpr int TM = WM / 32, TN = WN / 32;
  constexpr int A_PER_WAVE = BM / 16 / NWD, B_PER_WAVE = BN / 16 / NWD;
  constexpr int PER_STAGE = A_PER_WAVE + B_PER_WAVE;
  constexpr uint32_t A_STAGE = BM * 64, STAGE = (BM + BN) * 64;
  constexpr uint32_t SCALES = kMxStages * STAGE, SCALE_BUF = (BM + BN) * 16;
  static_assert(BM == 64 * (NW - NWD) && BN == BM, "a scale wave asks for 64 rows of A and of B");
  static_assert(BM / 16 % NWD == 0 && BN / 16 % NWD == 0, "DMA split");
  static_assert(WM % 32 == 0 && WN == 64, "wave tile");
  static_assert(SCALES + 2 * SCALE_BUF == mx_ring_bytes<BM, BN>(), "ring size");
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WAVES_N, wn = wave % WAVES_N;
  const bool dma = wave < NWD;
  const uint32_t lds0 = lds_addr(smem);

  const char *Ab, *Bb, *Asb, *Bsb;
  int32_t offA[A_PER_WAVE];  // of a scale wave: [0] and [1], of the exponents of A and B
  int32_t blkB[B_PER_WAVE];  // (the lane's part of B's offsets is 16 bytes a lane)
  auto setup = [&](const TileCoord &c) {
    int ln = lane;
    asm volatile("" : "+v"(ln));
    // rows and columns past the tile's valid ones re-read its last valid ones
    const int64_t row = int64_t(c.row0) + c.m0;
    Ab = reinterpret_cast<const char *>(g.A) + row * g.lda;
    Asb = reinterpret_cast<const char *>(g.a_scale) + row * g.a_scale_pitch;
    const char *Be = reinterpret_cast<const char *>(g.B) + int64_t(c.e) * g.b_expert_stride;
    Bb = Be + (c.n0 >> 4) * g.b_blk_stride;
    Bsb = Be + g.b_scale_at + (c.n0 >> 4) * g.b_scale_blk_stride;
    const int last_row = c.rows_valid - 1, last_blk = (c.cols_valid - 1) >> 4;
    if (dma) {
      const int kc = (ln & 3) ^ ((ln >> 4) & 3);
#pragma unroll
      for (int j = 0; j < A_PER_WAVE; ++j)
        offA[j] = int32_t(__umul24(uint32_t(min((wave + NWD * j) * 16 + (ln >> 2), last_row)),
                                   uint32_t(g.lda)) + uint32_t(kc * 16));
#pragma unroll
      for (int j = 0; j < B_PER_WAVE; ++j)
        blkB[j] = int32_t(min(wave + NWD * j, last_blk) * g.b_blk_stride);
    } else {
      const int r = (wave - NWD) * 64 + ln;
      offA[0] = int32_t(__umul24(uint32_t(min(r, last_row)), uint32_t(g.a_scale_pitch)));
      const int blk = (wave - NWD) * 4 + ((ln >> 2) & 3);
      offA[1] = int32_t(min(blk, last_blk) * g.b_scale_blk_stride + (ln >> 4) * 64 + (ln & 3) * 16);
    }
  };
  auto request_one = [&](int st, int kt, int d) {  // DMA d of slice kt
    const uint32_t at = lds0 + st * STAGE;
    if (d < A_PER_WAVE)
      dma16(Ab + kt * 64, offA[d], at + (wave + NWD * d) * 1024);
    else
      dma16(Bb + blkB[d - A_PER_WAVE] + kt * 1024, lane * 16,
            at + A_STAGE + (wave + NWD * (d - A_PER_WAVE)) * 1024);
  };
  auto request = [&](int st, int kt) {
#pragma unroll
    for (int d = 0; d < PER_STAGE; ++d) request_one(st, kt, d);
  };
  // Exponents of slices 4 s .. 4 s + 3: of A 16 bytes of a row, of B those of 64 rows for
  // slice after slice.
  auto request_scales = [&](int s) {
    const uint32_t at = lds0 + SCALES + (s & 1) * SCALE_BUF + (wave - NWD) * 1024;
    dma16(Asb + s * 16, offA[0], at);
    dma16(Bsb + s * 256, offA[1], at + BM * 16);
  };
  auto prologue = [&]() {
    if (dma) {
#pragma unroll
      for (int k = 0; k < kMxAhead; ++k)
        if (k < t.nk) request(k, k);
    } else {
      request_scales(0);
    }
  };
  setup(t);
  prologue();
  using Frag = i32x4;
  auto read_a = [&](int st, int ks, int i) {
    const int row = wm * WM + i * 32 + (lane & 31), kc = ks * 2 + h;
    return *reinterpret_cast<const Frag *>(smem + st * STAGE + row * 64 +
                                           ((kc ^ ((row >> 2) & 3)) << 4));
  };
  auto read_b = [&](int st, int ks, int j) {
    const int row = wn * WN + j * 32 + (lane & 31), kc = ks * 2 + h;
    return *reinterpret_cast<const Frag *>(smem + st * STAGE + A_STAGE + (row >> 4) * 1024 +
                                           kc * 256 + (row & 15) * 16);
  };
  // the four exponents of a row in slice kt (i < TM: of A, then of B)
  auto read_scale = [&](int kt, int i) {
    const char *p = smem + SCALES + ((kt >> 2) & 1) * SCALE_BUF;
    if (i < TM)
      p += (wm * WM + i * 32 + (lane & 31)) * 16 + (kt & 3) * 4;
    else
      p += BM * 16 + wn * 1024 + (kt & 3) * 256 + ((i - TM) * 32 + (lane & 31)) * 4;
    return *reinterpret_cast<const uint32_t *>(p);
  };
  static_assert(TN == 2, "side work after the first of two blocks");
  constexpr int NR = TM + TN;
  constexpr int D0 = PER_STAGE / 2;
  auto next_stage = [](int st) { return st + 1 == kMxStages ? 0 : st + 1; };

  // One step (64 values of k) of matrix instructions with the side work spread
  // between them: the operands of the next step (those of A in place, each after
  // its last use: a second set would not fit the registers), with them (kNewSlice)
  // the exponents of its slice, and part of a slice's DMA.
  auto step = [&](auto sel, auto dma_wave, auto new_slice, f32x16 (&acc)[TM][TN], Frag (&fa)[TM],
                  const Frag (&fb)[TN], const uint32_t (&sc)[NR], Frag (&fb_next)[TN],
                  uint32_t (&sc_next)[NR], int st_next, int kt_next, int st_dma, int kt_dma) {
    constexpr bool kDma = decltype(dma_wave)::value, kNewSlice = decltype(new_slice)::value;
    constexpr int kSel = decltype(sel)::value;
    constexpr int ks_next = kNewSlice ? 0 : 1;
    constexpr int NSC = kNewSlice ? NR : 0;
    constexpr int dma_lo = kNewSlice ? D0 : 0, dma_n = kDma ? (kNewSlice ? PER_STAGE - D0 : D0) : 0;
    constexpr int NS = TN + NSC + dma_n;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        acc[i][j] = mx_mfma<kSel>(fb[j], fa[i], acc[i][j], int(sc[TM + j]), int(sc[i]));
        __builtin_amdgcn_sched_barrier(0);
        if (j == TN - 1) {
          fa[i] = read_a(st_next, ks_next, i);
          __builtin_amdgcn_sched_barrier(0);
        } else {
#pragma unroll
          for (int q = 0; q < NS; ++q) {
            if (q * TM >= i * NS && q * TM < (i + 1) * NS) {
              if (q < TN)
                fb_next[q] = read_b(st_next, ks_next, q);
              else if (q < TN + NSC)
                sc_next[q - TN] = read_scale(kt_next, q - TN);
              else
                request_one(st_dma, kt_dma, dma_lo + q - TN - NSC);
              __builtin_amdgcn_sched_barrier(0);
            }
          }
        }
      }
    }
  };
  std::integral_constant<int, 0> sel0;
  std::integral_constant<int, 2> sel2;
  auto wait_scales = [&](int kt) {  // a scale wave at the barrier before slice kt + 1
    if ((kt & 3) == 3) wait_vmcnt<0>();
    wait_and_sync<63>();
  };
  // everything is requested, `left` slices beyond the next one
  auto wait_tail = [&](int left) {
    if (!dma || left < 1)
      wait_vmcnt<0>();
    else
      wait_vmcnt<PER_STAGE>();
    wait_and_sync<63>();
  };

  for (;;) {
    const int nk = t.nk;
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.0f;
    // (a wave whose outputs all lie past the tile's last valid row or column runs
    // the same loop without LDS reads and matrix instructions)
    const int active =
        __builtin_amdgcn_readfirstlane(int(t.rows_valid > wm * WM && t.cols_valid > wn * WN));
    // slice 0, and the first exponents
    // (behind a tile's stores, which are waited for as well: counted past, 8192 x 8192 x
    // 2048 took 87 us for 84)
    if (dma && nk >= kMxAhead)
      wait_vmcnt<(kMxAhead - 1) * PER_STAGE>();
    else
      wait_vmcnt<0>();
    wait_and_sync<63>();
    int st = 0, kt = 0, st_req = kMxAhead % kMxStages;
    // the whole of k, one copy for the DMA waves and one for the others
    auto work = [&](auto dma_wave) {
      constexpr bool kDma = decltype(dma_wave)::value;
      Frag fa[TM], fb0[TN], fb1[TN];
      uint32_t sc[NR], raw[NR];
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[i] = read_a(0, 0, i);
#pragma unroll
      for (int j = 0; j < TN; ++j) fb0[j] = read_b(0, 0, j);
#pragma unroll
      for (int i = 0; i < NR; ++i) raw[i] = read_scale(0, i);
      // bytes 0 and 2 of sc: the lane's half of the first and the second step
      auto take_scales = [&]() {
#pragma unroll
        for (int i = 0; i < NR; ++i) sc[i] = raw[i] >> (8 * h);
      };
#pragma clang loop unroll(disable)
      for (; kt < nk - kMxAhead; ++kt) {
        take_scales();
        if (!kDma && (kt & 3) == 0 && kt + 4 < nk) request_scales((kt >> 2) + 1);
        step(sel0, dma_wave, std::false_type{}, acc, fa, fb0, sc, fb1, raw, st, kt, st_req,
             kt + kMxAhead);
        if (kDma) {
          wait_vmcnt<(kMxAhead - 2) * PER_STAGE + D0>();
          wait_and_sync<63>();
        } else {
          wait_scales(kt);
        }
        st = next_stage(st);
        step(sel2, dma_wave, std::true_type{}, acc, fa, fb1, sc, fb0, raw, st, kt + 1, st_req,
             kt + kMxAhead);
        st_req = next_stage(st_req);
      }
#pragma clang loop unroll(disable)
      for (; kt < nk - 1; ++kt) {
        take_scales();
        step(sel0, std::false_type{}, std::false_type{}, acc, fa, fb0, sc, fb1, raw, st, kt, 0, 0);
        wait_tail(nk - 2 - kt);
        st = next_stage(st);
        step(sel2, std::false_type{}, std::true_type{}, acc, fa, fb1, sc, fb0, raw, st, kt + 1, 0,
             0);
      }
      take_scales();
      step(sel0, std::false_type{}, std::false_type{}, acc, fa, fb0, sc, fb1, raw, st, kt, 0, 0);
      // the last step
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = mx_mfma<2>(fb1[j], fa[i], acc[i][j], int(sc[TM + j]), int(sc[i]));
    };
    if (active) {
      if (dma)
        work(std::true_type{});
      else
        work(std::false_type{});
    } else {
      for (; kt < nk - kMxAhead; ++kt) {
        if (dma) {
          request(st_req, kt + kMxAhead);
          wait_vmcnt<(kMxAhead - 1) * PER_STAGE>();
          wait_and_sync<63>();
        } else {
          if ((kt & 3) == 0 && kt + 4 < nk) request_scales((kt >> 2) + 1);
          wait_scales(kt);
        }
        st_req = next_stage(st_req);
      }
      for (; kt < nk - 1; ++kt) wait_tail(nk - 2 - kt);
    }
    // every wave is done with the ring before the next tile's slices land
    __syncthreads();
    const TileCoord c = t;
    const bool more = sched.next(t);
    // the next tile's first slices load during the epilogue, whose staging area
    // is the last stage
    if (more) {
      setup(t);
      prologue();
    }

    // Epilogue: lane l holds, of a 32 x 32 block, output row l % 32 and in slots 4 q ..
    // 4 q + 3 the columns 8 q + 4 (l / 32) + 0..3.
    // (the lane is hidden from hoisting: what is derived from it holds no register
    // in the main loop)
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int el = ln & 31, eh = ln >> 5;
    constexpr uint32_t STAGING = STAGE / NW;  // bytes per wave
    char *stg = smem + (kMxStages - 1) * STAGE + wave * STAGING;
    const int rows_w = c.rows_valid - wm * WM;  // valid rows of this wave's part
    const bool all_staged = kEpi == kMxSwiglu || !Sched::kAnyC || (g.N & (kEpi == kMxF32 ? 3 : 7)) == 0;
    const int64_t row_w = int64_t(c.row0) + c.m0 + wm * WM;
    const int ncol0 = c.n0 + wn * WN;
    if constexpr (kEpi == kMxSwiglu) {
      // 32 gate columns and the matching up columns: one block of 32 activations
      // of a row, between lanes l and l + 32
      const int f = ncol0 >> 1;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (i * 32 >= rows_w || ncol0 >= g.N) break;
        float v[16];
        uint32_t most = 0;
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          v[q] = mx_swiglu(acc[i][0][q], acc[i][1][q]);
          most = max(most, __float_as_uint(v[q]) & 0x7fffffffu);
        }
        uint32_t other = most;
        swap_halves(most, other);
        most = max(most, other);
        const uint32_t x = mx_exponent(most);
        const float scale = mx_step(x);
        uint32_t lo = mx_pack4(v[0], v[1], v[2], v[3], scale) |
                      (mx_pack4(v[4], v[5], v[6], v[7], scale) << 16);
        uint32_t hi = mx_pack4(v[8], v[9], v[10], v[11], scale) |
                      (mx_pack4(v[12], v[13], v[14], v[15], scale) << 16);
        // columns 8 q + 4 h: after the exchange lane l has the row's first 8 bytes,
        // lane l + 32 the last
        swap_halves(lo, hi);
        if (i * 32 + el < rows_w) {
          const int64_t row = row_w + i * 32 + el;
          *reinterpret_cast<uint2 *>(g.act + row * g.ldc + f / 2 + 8 * eh) =
              make_uint2((lo & 0xffffu) | (hi << 16), (lo >> 16) | (hi & 0xffff0000u));
          if (eh == 0) {
            uint8_t *s = g.act_scale + row * g.ldc;
            s[f >> 5] = uint8_t(x);
            if (2 * f + 64 == g.N) mx_pad_scales(s, (f >> 5) + 1, g.act_blocks);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      // rows of whole 16-byte vectors go through the staging area, 32 rows at a
      // time, as runs of a row; others from the registers. Stores go past the caches (a
      // product and a read of its outputs: 16384 x 4096 x 1024 105 -> 97 us, 32768 x 7168 x
      // 1024 in float32 559 -> 535, but 8192 x 7168 x 2048 120 -> 124)
      constexpr bool kF32 = kEpi == kMxF32;
      const bool staged = all_staged;
      // columns of a piece: its rows are 128 bytes, whose 16-byte chunks are
      // XORed with the row
      constexpr int EB = kF32 ? 4 : 2, PW = 128 / EB;
      static_assert(32 * 128 <= int(STAGING), "staging");
      const int r = el;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (i * 32 >= rows_w) break;
        const int64_t row = row_w + i * 32 + min(r, rows_w - i * 32 - 1);
#pragma unroll
        for (int p = 0; p < WN; p += PW) {
          if (ncol0 + p >= g.N) continue;
#pragma unroll
          for (int c4 = 0; c4 < PW / 8; ++c4) {
            const int j = (p / 8 + c4) / 4, q = c4 % 4, col = 8 * c4 + 4 * eh;
            const f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2],
                             acc[i][j][4 * q + 3]};
            if (staged) {
              char *s = stg + r * 128 + (((col * EB >> 4) ^ (r & 7)) << 4) + (col * EB & 15);
              if constexpr (kF32)
                *reinterpret_cast<f32x4 *>(s) = v;
              else
                *reinterpret_cast<uint2 *>(s) =
                    make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
            } else if (i * 32 + r < rows_w) {
              if constexpr (kF32)
                int8_store4(reinterpret_cast<float *>(g.C) + row * g.ldc, ncol0 + p + col, g.N, v);
              else
                int8_store4(g.C + row * g.ldc, ncol0 + p + col, g.N, v);
            }
          }
          if (staged) {
            char *crow = reinterpret_cast<char *>(g.C) + ((row_w + i * 32) * g.ldc + ncol0 + p) * EB;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
              const int rr = n * 8 + (ln >> 3), ch = ln & 7;
              if (i * 32 + rr < rows_w && ncol0 + p + ch * (16 / EB) < g.N)
                __builtin_nontemporal_store(
                    *reinterpret_cast<const i32x4 *>(stg + rr * 128 + ((ch ^ (rr & 7)) << 4)),
                    reinterpret_cast<i32x4 *>(crow + int64_t(rr) * g.ldc * EB + ch * 16));
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if (!more) break;
  }
}

}  // namespace llep
