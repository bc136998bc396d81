// Internal launch interface between the C ABI (abi.cpp) and the kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "llep.h"

namespace llep {

constexpr int kMaxChunks = 2 * LLEP_MAX_EXPERTS + LLEP_MAX_DEVICES;

// Internal status bit: the plan tables overflowed (never expected; the chunk
// count is bounded by 2E + P).
constexpr int32_t kStatusPlanOverflow = 1 << 30;

// Pairs are counted in tiles of kRankTile pairs (one workgroup each), and
// per slice of kRankSub pairs (a wave's share of a tile); they are ranked
// slice by slice (one workgroup per slice, 64 pairs per wave). rank_base
// holds one row of E counts (then exclusive bases) per tile, a bad-id flag
// per tile, and a row of E counts per slice.
constexpr int kRankTile = 1024;
constexpr int kRankWaves = 4;
constexpr int kRankSub = kRankTile / kRankWaves;

int64_t rank_tiles(int64_t R);

struct PlanArgs {
  int64_t R;
  int32_t E, P, M, min_chunk, mode;
  int64_t cap;
  double lambda;
  int32_t n_tiles;
  const int32_t *ids;
  llep_plan_buffers buf;
};
hipError_t launch_plan(const PlanArgs &a, hipStream_t stream);

struct PermuteArgs {
  int64_t T, R;
  int32_t K, E, D;
  int32_t max_chunks;  // 2E + P: rows of the plan's chunk table
  int32_t n_tiles;
  int32_t elem_bytes;
  const int32_t *ids;
  const float *gates;
  const void *x;
  void *x_perm;
  float *gate_perm;
  int32_t *row_pair, *pair_row;
  llep_plan_buffers plan;
};
hipError_t launch_permute(const PermuteArgs &a, hipStream_t stream);

struct CombineArgs {
  int64_t T;
  int32_t K, D;
  llep_dtype dtype;
  const void *out_perm;
  const int32_t *pair_row;
  const float *gates;
  void *y;
  bool bf16_y;  // float32 out_perm: whether y is bfloat16 all the same
};
hipError_t launch_combine(const CombineArgs &a, hipStream_t stream);

struct FfnArgs {
  int64_t R;
  int64_t device_rows;  // rows that one device can be expected to hold at most
  int32_t P, E, D, F, device;
  llep_dtype dtype;
  const int32_t *groups, *group_begin;
  const void *x_perm, *w_gate_up, *w_down;
  void *out_perm;
  void *gate_up_out;  // training forward: raw gate / up values per x_perm row; null: none
  void *ws;
  size_t ws_bytes;
  int32_t *status;  // the plan's status word (LLEP_STATUS_FFN_WAIT)
};
size_t ffn_workspace_bytes(int64_t R, int32_t E, int32_t P, int32_t F,
                           llep_dtype dtype);
hipError_t launch_grouped_ffn(const FfnArgs &a, hipStream_t stream);
// The bf16 forward of calls of few rows (stream_ffn.hip), at most kStreamRows
// over all devices; act: the workspace's activation.
constexpr int kStreamRows = 4096;
bool use_stream_ffn(const FfnArgs &a);
hipError_t launch_stream_ffn(const FfnArgs &a, void *act, hipStream_t stream);
// The float32 forward and backward (ffn_f32.hip); act [R][F] and dgu [R][2F]
// by x_perm row, in the workspace.
struct FfnBwdArgs;
hipError_t launch_ffn_f32(const FfnArgs &a, void *act, hipStream_t stream);
hipError_t launch_ffn_f32_backward(const FfnBwdArgs &a, float *dgu, float *act,
                                   hipStream_t stream);
// Address on the current GPU of the library's LLEP_NOALLOC_SCRATCH_BYTES
// workspace array (looked up once per GPU, then cached).
hipError_t ffn_scratch_address(void **ptr);

struct FfnBwdArgs {
  int64_t R;
  int32_t P, E, D, F, device;
  llep_dtype dtype;
  const int32_t *groups, *group_begin;
  const void *x_perm, *d_out_perm, *w_gate_up, *w_gate_up_t, *w_down_t;
  const void *gate_up;  // saved by the training forward; null: recompute
  void *dx_perm;
  float *dw_gate, *dw_up, *dw_down;
  void *ws;
};
size_t ffn_backward_workspace_bytes(int64_t R, int32_t E, int32_t P, int32_t D, int32_t F,
                                    llep_dtype dtype);
// whether R rows are within the call's documented limit
bool ffn_backward_rows_ok(int64_t R, int32_t E, int32_t P);
hipError_t launch_grouped_ffn_backward(const FfnBwdArgs &a, hipStream_t stream);
// zeros for the weight gradients of the experts without rows in the range
hipError_t launch_zero_absent(const FfnBwdArgs &a, hipStream_t stream);
hipError_t launch_pack_backward(int32_t E, int32_t D, int32_t F, llep_dtype dtype, const void *w_gate,
                                const void *w_up, const void *w_down, void *gut, void *dnt,
                                hipStream_t stream);

struct CombineBwdArgs {
  int64_t T;
  int32_t K, D;
  llep_dtype dtype;
  const void *out_perm, *dy;
  const int32_t *pair_row;
  const float *gates;
  void *d_out_perm;
  float *d_gates;
};
hipError_t launch_combine_backward(const CombineBwdArgs &a, hipStream_t stream);

// Norms around a block (norm.hip); b, gate, w_post, w_pre, r, h, h_q may be null.
struct NormArgs {
  int64_t T;
  int32_t D;
  llep_dtype dtype;
  llep_gate_shape gate_shape;
  float alpha, eps;
  const void *x, *b, *gate, *w_post, *w_pre;
  void *r, *h;
  int8_t *h_q;
  float *h_scale;
  int32_t q_bytes;  // of a row of h_q
};
hipError_t launch_block_norm(const NormArgs &a, hipStream_t stream);

// workgroups of the backward at most (rows of column sums in the workspace)
constexpr int kNormBwdGrid = 1024;
struct NormBwdArgs {
  NormArgs n;  // the forward's b, gate, weights and numbers
  const void *r, *d_r, *d_h;
  void *dx, *db;
  float *d_gate, *dw_post, *dw_pre;
  float *parts;      // [workgroups][2][D]
  bool column_sums;  // whether d w_post or d g is summed over the rows
};
size_t norm_bwd_workspace_bytes(int64_t T, int32_t D);
hipError_t launch_block_norm_backward(const NormBwdArgs &a, hipStream_t stream);

// 8-bit rows and products (int8.hip).
hipError_t launch_quantize_rows(int64_t R, int32_t D, llep_dtype dtype, const void *x, int8_t *q,
                                int32_t q_bytes, float *scale, hipStream_t stream);
// w1: null, or the up weights whose rows alternate with those of w0 by 32
hipError_t launch_pack_int8(int32_t E, int32_t N, int32_t K, const int8_t *w0, const int8_t *w1,
                            int8_t *out, hipStream_t stream);
struct Int8MatmulArgs {
  int64_t M;
  int32_t N, K, x_bytes;
  llep_dtype dtype;  // of out
  const int8_t *x, *w;
  const float *x_scale, *w_scale;
  void *out;
};
hipError_t launch_int8_matmul(const Int8MatmulArgs &a, hipStream_t stream);
struct FfnInt8Args {
  int64_t R;
  int32_t P, E, D, F, K, device;
  const int32_t *groups, *group_begin, *row_pair;
  const int8_t *x_perm, *w_gate_up, *w_down;
  const float *x_scale, *gate_scale, *up_scale, *down_scale;
  void *out_perm, *ws;
  bool f32_out;  // out_perm is float32, else bfloat16
};
size_t ffn_int8_workspace_bytes(int64_t R, int32_t E, int32_t P, int32_t F);
hipError_t launch_ffn_int8(const FfnInt8Args &a, hipStream_t stream);
// The list of tiles of BM rows of a range's groups (grouped_ffn.hip).
hipError_t launch_tile_table(const int32_t *groups, const int32_t *group_begin, int32_t cap,
                             int32_t device, int32_t P, int32_t BM, int4 *tiles, int32_t *n_tiles,
                             hipStream_t stream);

// Gradient norm and clipping (clip.hip).
struct ClipArgs {
  int32_t n;
  const llep_gradient *grads;  // host
  float max_norm;
  bool scale;  // whether the gradients are clipped, or only their norm taken
  float *norm;
  double *parts;  // [kClipParts]
};
constexpr int kClipParts = 1024;
hipError_t launch_clip(const ClipArgs &a, hipStream_t stream);

hipError_t launch_pack(int32_t E, int32_t D, int32_t F, llep_dtype dtype,
                       const void *w_gate, const void *w_up,
                       const void *w_down, void *gu, void *dn,
                       hipStream_t stream);

}  // namespace llep
