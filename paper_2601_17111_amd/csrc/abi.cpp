// C ABI of the LLEP hot path: argument checks on the host, then launches.
// No entry point allocates, synchronizes or keeps state between calls, apart
// from the calling thread's last error text and the per-GPU address of the
// library's workspace array (llep_grouped_ffn_noalloc), looked up once.
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <string>

#include "kernels.h"
#include "llep.h"

namespace {

thread_local std::string g_last_error;

int fail(int code, const std::string &msg) {
  g_last_error = msg;
  return code;
}

int ok() {
  g_last_error.clear();
  return LLEP_OK;
}

int hip_result(hipError_t err, const char *where) {
  if (err == hipSuccess) return ok();
  return fail(LLEP_E_HIP, std::string(where) + ": " + hipGetErrorString(err));
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_params(const llep_plan_params *p) {
  if (!p) return fail(LLEP_E_ARG, "params is null");
  if (p->T < 0) return fail(LLEP_E_ARG, "T < 0");
  if (p->K < 1) return fail(LLEP_E_ARG, "K < 1");
  if (p->E < 1 || p->E > LLEP_MAX_EXPERTS) return fail(LLEP_E_ARG, "E outside [1, LLEP_MAX_EXPERTS]");
  if (p->P < 1 || p->P > LLEP_MAX_DEVICES) return fail(LLEP_E_ARG, "P outside [1, LLEP_MAX_DEVICES]");
  if (p->E % p->P != 0) return fail(LLEP_E_ARG, "E % P != 0");
  if (p->T > int64_t(INT32_MAX) / p->K) return fail(LLEP_E_ARG, "T * K >= 2^31");
  if (p->capacity < 1) return fail(LLEP_E_ARG, "capacity < 1");
  if (p->mode != LLEP_MODE_LLEP && p->mode != LLEP_MODE_EP) return fail(LLEP_E_ARG, "unknown mode");
  if (p->reserved != 0) return fail(LLEP_E_ARG, "reserved field is not 0");
  return LLEP_OK;
}

int check_plan_buffers(const llep_plan_buffers *b) {
  if (!b) return fail(LLEP_E_ARG, "plan buffers are null");
  if (!b->loads || !b->chunks || !b->chunk_row || !b->expert_chunk_begin || !b->groups ||
      !b->group_begin || !b->device_rows || !b->xfers || !b->rank_base || !b->info)
    return fail(LLEP_E_ARG, "a plan buffer pointer is null");
  return LLEP_OK;
}

int elem_bytes(llep_dtype d) { return d == LLEP_BF16 ? 2 : (d == LLEP_F32 ? 4 : 0); }

int check_rows(int32_t D, llep_dtype dtype) {
  const int eb = elem_bytes(dtype);
  if (eb == 0) return fail(LLEP_E_DTYPE, "unknown dtype");
  if (D < 1) return fail(LLEP_E_ARG, "D < 1");
  if (D % 8 != 0) return fail(LLEP_E_ARG, "D % 8 != 0 (rows must be whole 16-byte vectors)");
  return LLEP_OK;
}

int check_ffn_dims(int32_t D, int32_t F, llep_dtype dtype) {
  if (elem_bytes(dtype) == 0) return fail(LLEP_E_DTYPE, "unknown dtype");
  if (D < 64 || D % 64 != 0) return fail(LLEP_E_ARG, "D must be a positive multiple of 64");
  if (F < 64 || F % 64 != 0) return fail(LLEP_E_ARG, "F must be a positive multiple of 64");
  // the GEMMs address a tile's operand rows with 32-bit byte offsets
  if (D > LLEP_MAX_FFN_DIM || F > LLEP_MAX_FFN_DIM)
    return fail(LLEP_E_ARG, "D and F must be at most LLEP_MAX_FFN_DIM");
  return LLEP_OK;
}

bool aligned_to(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// the arguments that the block norm and its backward share
int check_norm(int64_t T, int32_t D, llep_dtype dtype, const void *b, const void *gate,
               llep_gate_shape gate_shape, const void *w_post, const void *w_pre, float eps) {
  const size_t eb = elem_bytes(dtype);
  if (eb == 0) return fail(LLEP_E_DTYPE, "unknown dtype");
  if (T < 0) return fail(LLEP_E_ARG, "T < 0");
  if (D < 1 || D > LLEP_MAX_NORM_DIM) return fail(LLEP_E_ARG, "D outside [1, LLEP_MAX_NORM_DIM]");
  if (!(eps >= 0.0f)) return fail(LLEP_E_ARG, "eps < 0");
  if (gate_shape < LLEP_GATE_NONE || gate_shape > LLEP_GATE_FULL)
    return fail(LLEP_E_ARG, "unknown gate shape");
  if ((gate != nullptr) != (gate_shape != LLEP_GATE_NONE) &&
      !(T == 0 && gate_shape > LLEP_GATE_CHANNEL))
    return fail(LLEP_E_ARG, "gate and gate_shape do not agree");
  if (!b && T > 0 && (gate_shape != LLEP_GATE_NONE || w_post))
    return fail(LLEP_E_ARG, "a gate or w_post without b");
  if (!aligned_to(b, eb) || !aligned_to(gate, eb) || !aligned_to(w_post, eb) ||
      !aligned_to(w_pre, eb))
    return fail(LLEP_E_ARG, "data not aligned to its type");
  return LLEP_OK;
}

int check_gradients(int32_t n, const llep_gradient *grads, bool scale, const float *norm,
                    const void *workspace, size_t workspace_bytes) {
  if (n < 0) return fail(LLEP_E_ARG, "n < 0");
  if (n > 0 && !grads) return fail(LLEP_E_ARG, "grads is null");
  if (!norm || !aligned_to(norm, 4)) return fail(LLEP_E_ARG, "norm is null or not aligned");
  for (int32_t i = 0; i < n; ++i) {
    const llep_gradient &g = grads[i];
    const size_t eb = elem_bytes(llep_dtype(g.dtype));
    if (eb == 0) return fail(LLEP_E_DTYPE, "unknown dtype");
    if (g.n < 0) return fail(LLEP_E_ARG, "a tensor of fewer than 0 elements");
    if (g.reserved != 0) return fail(LLEP_E_ARG, "reserved field is not 0");
    if (g.n > 0 && (!g.data || (scale && !g.out))) return fail(LLEP_E_ARG, "a data pointer is null");
    if (!aligned_to(g.data, eb) || (scale && !aligned_to(g.out, eb)))
      return fail(LLEP_E_ARG, "data not aligned to its type");
  }
  if (!workspace || workspace_bytes < llep_clip_gradients_workspace_bytes())
    return fail(LLEP_E_WORKSPACE,
                "workspace missing or smaller than llep_clip_gradients_workspace_bytes");
  if (!aligned16(workspace)) return fail(LLEP_E_WORKSPACE, "workspace not 16-byte aligned");
  return LLEP_OK;
}

int check_route(const llep_route_params *p, llep_dtype dtype) {
  if (!p) return fail(LLEP_E_ARG, "params is null");
  if (elem_bytes(dtype) == 0) return fail(LLEP_E_DTYPE, "unknown dtype");
  if (p->T < 0) return fail(LLEP_E_ARG, "T < 0");
  if (p->E < 1 || p->E > LLEP_MAX_EXPERTS) return fail(LLEP_E_ARG, "E outside [1, LLEP_MAX_EXPERTS]");
  if (p->K < 1 || p->K > LLEP_MAX_ROUTE_TOPK)
    return fail(LLEP_E_ARG, "K outside [1, LLEP_MAX_ROUTE_TOPK]");
  if (p->T > int64_t(INT32_MAX) / p->K) return fail(LLEP_E_ARG, "T * K >= 2^31");
  if (p->score != LLEP_SCORE_SOFTMAX && p->score != LLEP_SCORE_SIGMOID)
    return fail(LLEP_E_ARG, "unknown score");
  if (p->groups < 1 || p->groups > LLEP_MAX_ROUTE_GROUPS || p->E % p->groups != 0)
    return fail(LLEP_E_ARG, "groups must divide E and be in [1, LLEP_MAX_ROUTE_GROUPS]");
  if (p->top_groups < 1 || p->top_groups > p->groups)
    return fail(LLEP_E_ARG, "top_groups outside [1, groups]");
  if (p->K > p->E / p->groups * p->top_groups)
    return fail(LLEP_E_ARG, "K is more than the experts of top_groups groups");
  if (p->group_score != LLEP_GROUP_MAX && p->group_score != LLEP_GROUP_TOP2)
    return fail(LLEP_E_ARG, "unknown group score");
  if (p->renormalize != 0 && p->renormalize != 1) return fail(LLEP_E_ARG, "renormalize is 0 or 1");
  if (!(p->scale > 0.0f) || p->scale > 3.4028234e38f)
    return fail(LLEP_E_ARG, "scale must be finite and above 0");
  return LLEP_OK;
}

llep::RouteArgs route_args(const llep_route_params *p, llep_dtype dtype) {
  llep::RouteArgs a = {};
  a.T = p->T;
  a.K = p->K;
  a.E = p->E;
  a.groups = p->top_groups < p->groups ? p->groups : 1;  // all of them: no choice
  a.top_groups = p->top_groups;
  a.score = p->score;
  a.group_score = p->group_score;
  a.renormalize = p->renormalize != 0;
  a.scale = p->scale;
  a.dtype = dtype;
  return a;
}

// 4-bit rows of K values that a call reads or writes
int check_mxfp4_rows(int64_t R, int32_t K, const uint8_t *q, int32_t q_pitch, const uint8_t *scale,
                     int32_t scale_pitch) {
  if (R < 0) return fail(LLEP_E_ARG, "fewer than 0 rows");
  if (K < 1 || K > LLEP_MAX_FFN_DIM)
    return fail(LLEP_E_ARG, "values of a row outside [1, LLEP_MAX_FFN_DIM]");
  if (q_pitch % 16 != 0 || q_pitch < llep::mxfp4_row_bytes(K) || q_pitch > LLEP_MAX_FFN_DIM)
    return fail(LLEP_E_ARG, "q_pitch must be a multiple of 16 from llep_mxfp4_row_bytes on, at most "
                            "LLEP_MAX_FFN_DIM");
  if (scale_pitch % 16 != 0 || scale_pitch < llep::mxfp4_scale_bytes(K) ||
      scale_pitch > LLEP_MAX_FFN_DIM)
    return fail(LLEP_E_ARG, "scale_pitch must be a multiple of 16 from llep_mxfp4_scale_bytes on, at "
                            "most LLEP_MAX_FFN_DIM");
  if (R > 0 && (!q || !scale)) return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned16(q) || !aligned16(scale)) return fail(LLEP_E_ARG, "4-bit rows not 16-byte aligned");
  return LLEP_OK;
}

}  // namespace

extern "C" {

const char *llep_last_error(void) { return g_last_error.c_str(); }

int32_t llep_plan_max_chunks(const llep_plan_params *params) {
  if (check_params(params) != LLEP_OK) return -1;
  return 2 * params->E + params->P;
}

int64_t llep_plan_rank_base_elems(const llep_plan_params *params) {
  if (check_params(params) != LLEP_OK) return -1;
  const int64_t tiles = llep::rank_tiles(params->T * params->K);
  // per tile: E counts (then bases), a bad-id flag, E counts per slice
  return tiles * params->E + tiles + tiles * llep::kRankWaves * params->E;
}

int llep_plan(const llep_plan_params *params, const int32_t *topk_ids,
              const llep_plan_buffers *out, hipStream_t stream) {
  int rc = check_params(params);
  if (rc != LLEP_OK) return rc;
  if ((rc = check_plan_buffers(out)) != LLEP_OK) return rc;
  const int64_t R = params->T * params->K;
  if (R > 0 && !topk_ids) return fail(LLEP_E_ARG, "topk_ids is null");
  llep::PlanArgs a;
  a.R = R;
  a.E = params->E;
  a.P = params->P;
  a.M = params->E / params->P;
  a.min_chunk = params->min_chunk < 1 ? 1 : params->min_chunk;
  a.mode = params->mode;
  a.cap = params->capacity;
  a.lambda = params->lambda;
  a.n_tiles = int32_t(llep::rank_tiles(R));
  a.ids = topk_ids;
  a.buf = *out;
  return hip_result(llep::launch_plan(a, stream), "llep_plan");
}

int llep_permute(const llep_plan_params *params, const llep_plan_buffers *plan,
                 const int32_t *topk_ids, const float *topk_gates, const void *x, int32_t D,
                 llep_dtype dtype, void *x_perm, float *gate_perm, int32_t *row_pair,
                 int32_t *pair_row, hipStream_t stream) {
  int rc = check_params(params);
  if (rc != LLEP_OK) return rc;
  if ((rc = check_plan_buffers(plan)) != LLEP_OK) return rc;
  if ((rc = check_rows(D, dtype)) != LLEP_OK) return rc;
  if (params->T > 0 &&
      (!topk_ids || !topk_gates || !x || !x_perm || !gate_perm || !row_pair || !pair_row))
    return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned16(x) || !aligned16(x_perm)) return fail(LLEP_E_ARG, "x / x_perm not 16-byte aligned");
  llep::PermuteArgs a;
  a.T = params->T;
  a.R = params->T * params->K;
  a.K = params->K;
  a.E = params->E;
  a.max_chunks = 2 * params->E + params->P;
  a.D = D;
  a.n_tiles = int32_t(llep::rank_tiles(a.R));
  a.elem_bytes = elem_bytes(dtype);
  a.ids = topk_ids;
  a.gates = topk_gates;
  a.x = x;
  a.x_perm = x_perm;
  a.gate_perm = gate_perm;
  a.row_pair = row_pair;
  a.pair_row = pair_row;
  a.plan = *plan;
  return hip_result(llep::launch_permute(a, stream), "llep_permute");
}

size_t llep_packed_gate_up_bytes(int32_t E, int32_t D, int32_t F, llep_dtype dtype) {
  if (E < 1 || D < 1 || F < 1 || elem_bytes(dtype) == 0) return 0;
  return size_t(E) * 2 * size_t(F) * size_t(D) * elem_bytes(dtype);
}

size_t llep_packed_down_bytes(int32_t E, int32_t D, int32_t F, llep_dtype dtype) {
  if (E < 1 || D < 1 || F < 1 || elem_bytes(dtype) == 0) return 0;
  return size_t(E) * size_t(D) * size_t(F) * elem_bytes(dtype);
}

int llep_pack_weights(int32_t E, int32_t D, int32_t F, llep_dtype dtype, const void *w_gate,
                      const void *w_up, const void *w_down, void *w_gate_up_packed,
                      void *w_down_packed, hipStream_t stream) {
  if (E < 1 || E > LLEP_MAX_EXPERTS) return fail(LLEP_E_ARG, "E outside [1, LLEP_MAX_EXPERTS]");
  int rc = check_ffn_dims(D, F, dtype);
  if (rc != LLEP_OK) return rc;
  if (!w_gate || !w_up || !w_down || !w_gate_up_packed || !w_down_packed)
    return fail(LLEP_E_ARG, "a weight pointer is null");
  if (!aligned16(w_gate) || !aligned16(w_up) || !aligned16(w_down) ||
      !aligned16(w_gate_up_packed) || !aligned16(w_down_packed))
    return fail(LLEP_E_ARG, "weights not 16-byte aligned");
  return hip_result(llep::launch_pack(E, D, F, dtype, w_gate, w_up, w_down, w_gate_up_packed,
                                      w_down_packed, stream),
                    "llep_pack_weights");
}

size_t llep_grouped_ffn_workspace_bytes(const llep_plan_params *params, int32_t F,
                                        llep_dtype dtype) {
  if (check_params(params) != LLEP_OK || F < 1 || elem_bytes(dtype) == 0) return 0;
  return llep::ffn_workspace_bytes(params->T * params->K, params->E, params->P, F, dtype);
}

static int grouped_ffn(const llep_plan_params *params, const llep_plan_buffers *plan,
                       int32_t device, const void *x_perm, const void *w_gate_up_packed,
                       const void *w_down_packed, int32_t D, int32_t F, llep_dtype dtype,
                       void *out_perm, void *gate_up, void *workspace, size_t workspace_bytes,
                       hipStream_t stream, const char *name) {
  int rc = check_params(params);
  if (rc != LLEP_OK) return rc;
  if ((rc = check_plan_buffers(plan)) != LLEP_OK) return rc;
  if ((rc = check_ffn_dims(D, F, dtype)) != LLEP_OK) return rc;
  if (device < -1 || device >= params->P) return fail(LLEP_E_ARG, "device outside [-1, P)");
  if (!x_perm || !w_gate_up_packed || !w_down_packed || !out_perm)
    return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned16(x_perm) || !aligned16(w_gate_up_packed) || !aligned16(w_down_packed) ||
      !aligned16(out_perm))
    return fail(LLEP_E_ARG, "data not 16-byte aligned");
  const size_t need = llep::ffn_workspace_bytes(params->T * params->K, params->E, params->P, F, dtype);
  if (!workspace || workspace_bytes < need)
    return fail(LLEP_E_WORKSPACE, "workspace missing or smaller than llep_grouped_ffn_workspace_bytes");
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
    return fail(LLEP_E_WORKSPACE, "workspace not 256-byte aligned");
  llep::FfnArgs a = {};
  a.R = params->T * params->K;
  a.device_rows = params->mode == LLEP_MODE_LLEP ? std::min(a.R, params->capacity) : a.R;
  a.P = params->P;
  a.E = params->E;
  a.D = D;
  a.F = F;
  a.device = device;
  a.dtype = dtype;
  a.groups = plan->groups;
  a.group_begin = plan->group_begin;
  a.x_perm = x_perm;
  a.w_gate_up = w_gate_up_packed;
  a.w_down = w_down_packed;
  a.out_perm = out_perm;
  a.gate_up_out = gate_up;
  a.ws = workspace;
  a.ws_bytes = workspace_bytes;
  a.status = &plan->info->status;
  return hip_result(llep::launch_grouped_ffn(a, stream), name);
}

int llep_grouped_ffn(const llep_plan_params *params, const llep_plan_buffers *plan,
                     int32_t device, const void *x_perm, const void *w_gate_up_packed,
                     const void *w_down_packed, int32_t D, int32_t F, llep_dtype dtype,
                     void *out_perm, void *workspace, size_t workspace_bytes,
                     hipStream_t stream) {
  return grouped_ffn(params, plan, device, x_perm, w_gate_up_packed, w_down_packed, D, F, dtype,
                     out_perm, nullptr, workspace, workspace_bytes, stream, "llep_grouped_ffn");
}

int llep_grouped_ffn_train(const llep_plan_params *params, const llep_plan_buffers *plan,
                           int32_t device, const void *x_perm, const void *w_gate_up_packed,
                           const void *w_down_packed, int32_t D, int32_t F, llep_dtype dtype,
                           void *out_perm, void *gate_up, void *workspace,
                           size_t workspace_bytes, hipStream_t stream) {
  if (!gate_up) return fail(LLEP_E_ARG, "gate_up is null");
  if (!aligned16(gate_up)) return fail(LLEP_E_ARG, "gate_up not 16-byte aligned");
  return grouped_ffn(params, plan, device, x_perm, w_gate_up_packed, w_down_packed, D, F, dtype,
                     out_perm, gate_up, workspace, workspace_bytes, stream,
                     "llep_grouped_ffn_train");
}

int llep_grouped_ffn_noalloc(const llep_plan_params *params, const llep_plan_buffers *plan,
                             int32_t device, const void *x_perm, const void *w_gate_up_packed,
                             const void *w_down_packed, int32_t D, int32_t F, llep_dtype dtype,
                             void *out_perm, hipStream_t stream) {
  int rc = check_params(params);
  if (rc != LLEP_OK) return rc;
  if (F < 1 || elem_bytes(dtype) == 0) return check_ffn_dims(D, F, dtype);
  const size_t need = llep::ffn_workspace_bytes(params->T * params->K, params->E, params->P, F, dtype);
  if (need > size_t(LLEP_NOALLOC_SCRATCH_BYTES))
    return fail(LLEP_E_WORKSPACE,
                "llep_grouped_ffn_noalloc: this layer needs " + std::to_string(need) +
                    " bytes of workspace, more than the library's LLEP_NOALLOC_SCRATCH_BYTES = " +
                    std::to_string(size_t(LLEP_NOALLOC_SCRATCH_BYTES)) +
                    "; use llep_grouped_ffn with a caller workspace");
  void *ws = nullptr;
  const hipError_t err = llep::ffn_scratch_address(&ws);
  if (err != hipSuccess) return hip_result(err, "llep_grouped_ffn_noalloc (scratch address)");
  return grouped_ffn(params, plan, device, x_perm, w_gate_up_packed, w_down_packed, D, F, dtype,
                     out_perm, nullptr, ws, size_t(LLEP_NOALLOC_SCRATCH_BYTES), stream,
                     "llep_grouped_ffn_noalloc");
}

static int combine(const llep_plan_params *params, const void *out_perm, const int32_t *pair_row,
                   const float *topk_gates, int32_t D, llep_dtype dtype, void *y, bool bf16_y,
                   hipStream_t stream, const char *name) {
  int rc = check_params(params);
  if (rc != LLEP_OK) return rc;
  if ((rc = check_rows(D, dtype)) != LLEP_OK) return rc;
  // topk_gates == nullptr: every gate is 1 (sums the pairs' input gradients)
  if (params->T > 0 && (!out_perm || !pair_row || !y))
    return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned16(out_perm) || !aligned16(y)) return fail(LLEP_E_ARG, "out_perm / y not 16-byte aligned");
  llep::CombineArgs a = {};
  a.bf16_y = bf16_y;
  a.T = params->T;
  a.K = params->K;
  a.D = D;
  a.dtype = dtype;
  a.out_perm = out_perm;
  a.pair_row = pair_row;
  a.gates = topk_gates;
  a.y = y;
  return hip_result(llep::launch_combine(a, stream), name);
}

int llep_combine(const llep_plan_params *params, const void *out_perm, const int32_t *pair_row,
                 const float *topk_gates, int32_t D, llep_dtype dtype, void *y,
                 hipStream_t stream) {
  return combine(params, out_perm, pair_row, topk_gates, D, dtype, y, false, stream,
                 "llep_combine");
}

int llep_combine_to_bf16(const llep_plan_params *params, const float *out_perm,
                         const int32_t *pair_row, const float *topk_gates, int32_t D, void *y,
                         hipStream_t stream) {
  return combine(params, out_perm, pair_row, topk_gates, D, LLEP_F32, y, true, stream,
                 "llep_combine_to_bf16");
}

int llep_combine_backward(const llep_plan_params *params, const void *out_perm,
                          const int32_t *pair_row, const float *topk_gates, const void *dy,
                          int32_t D, llep_dtype dtype, void *d_out_perm, float *d_gates,
                          hipStream_t stream) {
  int rc = check_params(params);
  if (rc != LLEP_OK) return rc;
  if ((rc = check_rows(D, dtype)) != LLEP_OK) return rc;
  if (params->T > 0 && (!out_perm || !pair_row || !topk_gates || !dy || !d_out_perm || !d_gates))
    return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned16(out_perm) || !aligned16(dy) || !aligned16(d_out_perm))
    return fail(LLEP_E_ARG, "out_perm / dy / d_out_perm not 16-byte aligned");
  llep::CombineBwdArgs a;
  a.T = params->T;
  a.K = params->K;
  a.D = D;
  a.dtype = dtype;
  a.out_perm = out_perm;
  a.dy = dy;
  a.pair_row = pair_row;
  a.gates = topk_gates;
  a.d_out_perm = d_out_perm;
  a.d_gates = d_gates;
  return hip_result(llep::launch_combine_backward(a, stream), "llep_combine_backward");
}

int llep_pack_weights_backward(int32_t E, int32_t D, int32_t F, llep_dtype dtype,
                               const void *w_gate, const void *w_up, const void *w_down,
                               void *w_gate_up_t_packed, void *w_down_t_packed,
                               hipStream_t stream) {
  if (E < 1 || E > LLEP_MAX_EXPERTS) return fail(LLEP_E_ARG, "E outside [1, LLEP_MAX_EXPERTS]");
  int rc = check_ffn_dims(D, F, dtype);
  if (rc != LLEP_OK) return rc;
  if (!w_gate || !w_up || !w_down || !w_gate_up_t_packed || !w_down_t_packed)
    return fail(LLEP_E_ARG, "a weight pointer is null");
  if (!aligned16(w_gate_up_t_packed) || !aligned16(w_down_t_packed))
    return fail(LLEP_E_ARG, "packed weights not 16-byte aligned");
  return hip_result(llep::launch_pack_backward(E, D, F, dtype, w_gate, w_up, w_down,
                                               w_gate_up_t_packed, w_down_t_packed, stream),
                    "llep_pack_weights_backward");
}

size_t llep_grouped_ffn_backward_workspace_bytes(const llep_plan_params *params, int32_t D,
                                                 int32_t F, llep_dtype dtype) {
  if (check_params(params) != LLEP_OK || D < 1 || F < 1 || elem_bytes(dtype) == 0) return 0;
  return llep::ffn_backward_workspace_bytes(params->T * params->K, params->E, params->P, D, F,
                                            dtype);
}

int llep_grouped_ffn_backward(const llep_plan_params *params, const llep_plan_buffers *plan,
                              int32_t device, const void *x_perm, const void *d_out_perm,
                              const void *w_gate_up_packed, const void *w_gate_up_t_packed,
                              const void *w_down_t_packed, const void *gate_up, int32_t D,
                              int32_t F, llep_dtype dtype, void *dx_perm, float *dw_gate,
                              float *dw_up, float *dw_down, void *workspace,
                              size_t workspace_bytes, hipStream_t stream) {
  int rc = check_params(params);
  if (rc != LLEP_OK) return rc;
  if ((rc = check_plan_buffers(plan)) != LLEP_OK) return rc;
  if ((rc = check_ffn_dims(D, F, dtype)) != LLEP_OK) return rc;
  if (device < -1 || device >= params->P) return fail(LLEP_E_ARG, "device outside [-1, P)");
  if (!x_perm || !d_out_perm || !w_gate_up_packed || !w_gate_up_t_packed || !w_down_t_packed ||
      !dx_perm || !dw_gate || !dw_up || !dw_down)
    return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned16(x_perm) || !aligned16(d_out_perm) || !aligned16(w_gate_up_packed) ||
      !aligned16(w_gate_up_t_packed) || !aligned16(w_down_t_packed) || !aligned16(dx_perm) ||
      !aligned16(dw_gate) || !aligned16(dw_up) || !aligned16(dw_down) || !aligned16(gate_up))
    return fail(LLEP_E_ARG, "data not 16-byte aligned");
  if (!llep::ffn_backward_rows_ok(params->T * params->K, params->E, params->P))
    return fail(LLEP_E_ARG, "T * K too large for the backward (about 4 M pairs at most)");
  const size_t need =
      llep::ffn_backward_workspace_bytes(params->T * params->K, params->E, params->P, D, F, dtype);
  if (!workspace || workspace_bytes < need)
    return fail(LLEP_E_WORKSPACE,
                "workspace missing or smaller than llep_grouped_ffn_backward_workspace_bytes");
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
    return fail(LLEP_E_WORKSPACE, "workspace not 256-byte aligned");
  llep::FfnBwdArgs a = {};
  a.R = params->T * params->K;
  a.P = params->P;
  a.E = params->E;
  a.D = D;
  a.F = F;
  a.device = device;
  a.dtype = dtype;
  a.groups = plan->groups;
  a.group_begin = plan->group_begin;
  a.x_perm = x_perm;
  a.d_out_perm = d_out_perm;
  a.w_gate_up = w_gate_up_packed;
  a.w_gate_up_t = w_gate_up_t_packed;
  a.w_down_t = w_down_t_packed;
  a.gate_up = gate_up;
  a.dx_perm = dx_perm;
  a.dw_gate = dw_gate;
  a.dw_up = dw_up;
  a.dw_down = dw_down;
  a.ws = workspace;
  return hip_result(llep::launch_grouped_ffn_backward(a, stream), "llep_grouped_ffn_backward");
}

int llep_zero_absent_gradients(const llep_plan_params *params, const llep_plan_buffers *plan,
                               int32_t device, int32_t D, int32_t F, float *dw_gate,
                               float *dw_up, float *dw_down, hipStream_t stream) {
  int rc = check_params(params);
  if (rc != LLEP_OK) return rc;
  if ((rc = check_plan_buffers(plan)) != LLEP_OK) return rc;
  if ((rc = check_ffn_dims(D, F, LLEP_F32)) != LLEP_OK) return rc;
  if (device < -1 || device >= params->P) return fail(LLEP_E_ARG, "device outside [-1, P)");
  if (!dw_gate || !dw_up || !dw_down) return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned16(dw_gate) || !aligned16(dw_up) || !aligned16(dw_down))
    return fail(LLEP_E_ARG, "data not 16-byte aligned");
  llep::FfnBwdArgs a = {};
  a.P = params->P;
  a.E = params->E;
  a.D = D;
  a.F = F;
  a.device = device;
  a.groups = plan->groups;
  a.group_begin = plan->group_begin;
  a.dw_gate = dw_gate;
  a.dw_up = dw_up;
  a.dw_down = dw_down;
  return hip_result(llep::launch_zero_absent(a, stream), "llep_zero_absent_gradients");
}

int llep_block_norm(int64_t T, int32_t D, llep_dtype dtype, const void *x, const void *b,
                    const void *gate, llep_gate_shape gate_shape, const void *w_post,
                    const void *w_pre, float alpha, float eps, void *r, void *h, int8_t *h_q,
                    float *h_scale, int32_t q_bytes, hipStream_t stream) {
  int rc = check_norm(T, D, dtype, b, gate, gate_shape, w_post, w_pre, eps);
  if (rc != LLEP_OK) return rc;
  if ((h || h_q) && !w_pre) return fail(LLEP_E_ARG, "h or h_q without w_pre");
  if ((h_q != nullptr) != (h_scale != nullptr)) return fail(LLEP_E_ARG, "h_q without h_scale");
  if (h_q && (q_bytes < D || q_bytes % 64 != 0))
    return fail(LLEP_E_ARG, "q_bytes must be a multiple of 64, at least D");
  if (h_q && (!aligned16(h_q) || !aligned_to(h_scale, 4)))
    return fail(LLEP_E_ARG, "h_q / h_scale not aligned");
  const size_t eb = elem_bytes(dtype);
  if (!aligned_to(x, eb) || !aligned_to(r, eb) || !aligned_to(h, eb))
    return fail(LLEP_E_ARG, "data not aligned to its type");
  if (T > 0 && !x) return fail(LLEP_E_ARG, "x is null");
  if (T > 0 && !r && !h && !h_q) return fail(LLEP_E_ARG, "no output");
  llep::NormArgs a = {};
  a.T = T;
  a.D = D;
  a.dtype = dtype;
  a.gate_shape = gate_shape;
  a.alpha = alpha;
  a.eps = eps;
  a.x = x;
  a.b = b;
  a.gate = gate;
  a.w_post = w_post;
  a.w_pre = h || h_q ? w_pre : nullptr;
  a.r = r;
  a.h = h;
  a.h_q = h_q;
  a.h_scale = h_scale;
  a.q_bytes = q_bytes;
  return hip_result(llep::launch_block_norm(a, stream), "llep_block_norm");
}

size_t llep_block_norm_backward_workspace_bytes(int64_t T, int32_t D) {
  if (T < 0 || D < 1 || D > LLEP_MAX_NORM_DIM) return 0;
  return llep::norm_bwd_workspace_bytes(T, D);
}

int llep_block_norm_backward(int64_t T, int32_t D, llep_dtype dtype, const void *r, const void *b,
                             const void *gate, llep_gate_shape gate_shape, const void *w_post,
                             const void *w_pre, float alpha, float eps, const void *d_r,
                             const void *d_h, void *dx, void *db, float *d_gate, float *dw_post,
                             float *dw_pre, void *workspace, size_t workspace_bytes,
                             hipStream_t stream) {
  int rc = check_norm(T, D, dtype, b, gate, gate_shape, w_post, w_pre, eps);
  if (rc != LLEP_OK) return rc;
  const size_t eb = elem_bytes(dtype);
  if (T > 0 && (!d_r || !dx)) return fail(LLEP_E_ARG, "d_r or dx is null");
  if (T > 0 && (w_pre != nullptr) != (d_h != nullptr))
    return fail(LLEP_E_ARG, "d_h and w_pre: both or none");
  if (T > 0 && w_pre && !r) return fail(LLEP_E_ARG, "r is null");
  if (T > 0 && (b != nullptr) != (db != nullptr)) return fail(LLEP_E_ARG, "db and b: both or none");
  if ((w_pre != nullptr) != (dw_pre != nullptr) || (w_post != nullptr) != (dw_post != nullptr))
    return fail(LLEP_E_ARG, "dw_pre (dw_post) and w_pre (w_post): both or none");
  if ((gate_shape == LLEP_GATE_NONE) != (d_gate == nullptr) &&
      !(T == 0 && gate_shape > LLEP_GATE_CHANNEL))
    return fail(LLEP_E_ARG, "d_gate and gate_shape do not agree");
  if (!aligned_to(r, eb) || !aligned_to(d_r, eb) || !aligned_to(d_h, eb) || !aligned_to(dx, eb) ||
      !aligned_to(db, eb) || !aligned_to(d_gate, 4) || !aligned_to(dw_post, 4) ||
      !aligned_to(dw_pre, 4))
    return fail(LLEP_E_ARG, "data not aligned to its type");
  if (workspace_bytes < llep_block_norm_backward_workspace_bytes(T, D) || (T > 0 && !workspace))
    return fail(LLEP_E_WORKSPACE,
                "workspace missing or smaller than llep_block_norm_backward_workspace_bytes");
  if (!aligned16(workspace)) return fail(LLEP_E_WORKSPACE, "workspace not 16-byte aligned");
  llep::NormBwdArgs a = {};
  a.n.T = T;
  a.n.D = D;
  a.n.dtype = dtype;
  a.n.gate_shape = gate_shape;
  a.n.alpha = alpha;
  a.n.eps = eps;
  a.n.b = b;
  a.n.gate = gate;
  a.n.w_post = w_post;
  a.n.w_pre = w_pre;
  a.r = r;
  a.d_r = d_r;
  a.d_h = d_h;
  a.dx = dx;
  a.db = db;
  a.d_gate = d_gate;
  a.dw_post = dw_post;
  a.dw_pre = dw_pre;
  a.parts = static_cast<float *>(workspace);
  a.column_sums = dw_post || gate_shape == LLEP_GATE_CHANNEL;
  return hip_result(llep::launch_block_norm_backward(a, stream), "llep_block_norm_backward");
}

size_t llep_clip_gradients_workspace_bytes(void) { return llep::kClipParts * sizeof(double); }

int llep_gradient_norm(int32_t n, const llep_gradient *grads, float *norm, void *workspace,
                       size_t workspace_bytes, hipStream_t stream) {
  const int rc = check_gradients(n, grads, false, norm, workspace, workspace_bytes);
  if (rc != LLEP_OK) return rc;
  llep::ClipArgs a = {n, grads, 0.0f, false, norm, static_cast<double *>(workspace)};
  return hip_result(llep::launch_clip(a, stream), "llep_gradient_norm");
}

int llep_clip_gradients(int32_t n, const llep_gradient *grads, float max_norm, float *norm,
                        void *workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!(max_norm >= 0.0f)) return fail(LLEP_E_ARG, "max_norm < 0");
  const int rc = check_gradients(n, grads, true, norm, workspace, workspace_bytes);
  if (rc != LLEP_OK) return rc;
  llep::ClipArgs a = {n, grads, max_norm, true, norm, static_cast<double *>(workspace)};
  return hip_result(llep::launch_clip(a, stream), "llep_clip_gradients");
}

int32_t llep_int8_row_bytes(int32_t D) {
  if (D < 1 || D > LLEP_MAX_FFN_DIM) return -1;
  return (D + 63) / 64 * 64;
}

int llep_quantize_rows(int64_t R, int32_t D, llep_dtype dtype, const void *x, int8_t *q,
                       int32_t q_bytes, float *scale, hipStream_t stream) {
  const size_t eb = elem_bytes(dtype);
  if (eb == 0) return fail(LLEP_E_DTYPE, "unknown dtype");
  if (R < 0) return fail(LLEP_E_ARG, "R < 0");
  if (D < 1 || D > LLEP_MAX_FFN_DIM) return fail(LLEP_E_ARG, "D outside [1, LLEP_MAX_FFN_DIM]");
  if (q_bytes < D || q_bytes % 64 != 0)
    return fail(LLEP_E_ARG, "q_bytes must be a multiple of 64, at least D");
  if (R > 0 && (!x || !q || !scale)) return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned_to(x, eb) || !aligned16(q) || !aligned_to(scale, 4))
    return fail(LLEP_E_ARG, "x, q or scale not aligned");
  return hip_result(llep::launch_quantize_rows(R, D, dtype, x, q, q_bytes, scale, stream),
                    "llep_quantize_rows");
}

size_t llep_packed_int8_bytes(int32_t E, int32_t N, int32_t K) {
  if (E < 1 || E > LLEP_MAX_EXPERTS || N < 1 || N > LLEP_MAX_INT8_COLUMNS || K < 1 ||
      K > LLEP_MAX_FFN_DIM)
    return 0;
  return size_t(E) * ((size_t(N) + 15) / 16 * 16) * ((size_t(K) + 63) / 64 * 64);
}

int llep_pack_int8(int32_t E, int32_t N, int32_t K, const int8_t *w, const int8_t *w_up,
                   int8_t *packed, hipStream_t stream) {
  if (llep_packed_int8_bytes(E, N, K) == 0)
    return fail(LLEP_E_ARG, "E, N or K outside its range");
  if (w_up && (N % 32 != 0 || N > LLEP_MAX_FFN_DIM))
    return fail(LLEP_E_ARG, "gate and up rows: N must be a multiple of 32, at most LLEP_MAX_FFN_DIM");
  if (!w || !packed) return fail(LLEP_E_ARG, "a weight pointer is null");
  if (!aligned16(packed)) return fail(LLEP_E_ARG, "packed weights not 16-byte aligned");
  return hip_result(llep::launch_pack_int8(E, N, K, w, w_up, packed, stream), "llep_pack_int8");
}

size_t llep_int8_matmul_workspace_bytes(int64_t M, int32_t N, int32_t K) {
  // no kernel of this version needs one, for any sizes
  (void)M, (void)N, (void)K;
  return 0;
}

int llep_int8_matmul(int64_t M, int32_t N, int32_t K, const int8_t *x, int32_t x_bytes,
                     const float *x_scale, const int8_t *w_packed, const float *w_scale,
                     llep_dtype dtype, void *out, void *workspace, size_t workspace_bytes,
                     hipStream_t stream) {
  const size_t eb = elem_bytes(dtype);
  if (eb == 0) return fail(LLEP_E_DTYPE, "unknown dtype");
  if (M < 0 || M > LLEP_MAX_INT8_ROWS) return fail(LLEP_E_ARG, "M outside [0, LLEP_MAX_INT8_ROWS]");
  if (llep_packed_int8_bytes(1, N, K) == 0) return fail(LLEP_E_ARG, "N or K outside its range");
  if (x_bytes % 64 != 0 || x_bytes < llep_int8_row_bytes(K) || x_bytes > LLEP_MAX_FFN_DIM)
    return fail(LLEP_E_ARG, "x_bytes must be a multiple of 64 from llep_int8_row_bytes(K) on");
  if (!w_packed || !w_scale || (M > 0 && (!x || !x_scale || !out)))
    return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned16(x) || !aligned16(w_packed) || !aligned16(w_scale) || !aligned16(out) ||
      !aligned_to(x_scale, 4))
    return fail(LLEP_E_ARG, "data not 16-byte aligned");
  const size_t need = llep_int8_matmul_workspace_bytes(M, N, K);
  if (workspace_bytes < need || (need > 0 && !workspace))
    return fail(LLEP_E_WORKSPACE,
                "workspace missing or smaller than llep_int8_matmul_workspace_bytes");
  if (!aligned_to(workspace, 256)) return fail(LLEP_E_WORKSPACE, "workspace not 256-byte aligned");
  llep::Int8MatmulArgs a = {};
  a.M = M;
  a.N = N;
  a.K = K;
  a.x_bytes = x_bytes;
  a.dtype = dtype;
  a.x = x;
  a.w = w_packed;
  a.x_scale = x_scale;
  a.w_scale = w_scale;
  a.out = out;
  return hip_result(llep::launch_int8_matmul(a, stream), "llep_int8_matmul");
}

size_t llep_grouped_ffn_int8_workspace_bytes(const llep_plan_params *params, int32_t F) {
  if (check_params(params) != LLEP_OK || F < 1 || F > LLEP_MAX_FFN_DIM) return 0;
  return llep::ffn_int8_workspace_bytes(params->T * params->K, params->E, params->P, F);
}

static int grouped_ffn_int8(const llep_plan_params *params, const llep_plan_buffers *plan,
                            int32_t device, const int8_t *x_perm, const float *x_scale,
                            const int32_t *row_pair, const int8_t *w_gate_up_packed,
                            const float *gate_scale, const float *up_scale,
                            const int8_t *w_down_packed, const float *down_scale, int32_t D,
                            int32_t F, void *out_perm, bool f32_out, void *workspace,
                            size_t workspace_bytes, hipStream_t stream, const char *name) {
  int rc = check_params(params);
  if (rc != LLEP_OK) return rc;
  if ((rc = check_plan_buffers(plan)) != LLEP_OK) return rc;
  if ((rc = check_ffn_dims(D, F, LLEP_BF16)) != LLEP_OK) return rc;
  if (device < -1 || device >= params->P) return fail(LLEP_E_ARG, "device outside [-1, P)");
  // (arrays of no rows may have no address)
  if (!w_gate_up_packed || !gate_scale || !up_scale || !w_down_packed || !down_scale ||
      (params->T > 0 && (!x_perm || !x_scale || !out_perm)))
    return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned16(x_perm) || !aligned16(w_gate_up_packed) || !aligned16(w_down_packed) ||
      !aligned16(gate_scale) || !aligned16(up_scale) || !aligned16(down_scale) ||
      !aligned16(out_perm) || !aligned_to(x_scale, 4) || !aligned_to(row_pair, 4))
    return fail(LLEP_E_ARG, "data not 16-byte aligned");
  const size_t need = llep_grouped_ffn_int8_workspace_bytes(params, F);
  if (!workspace || workspace_bytes < need)
    return fail(LLEP_E_WORKSPACE,
                "workspace missing or smaller than llep_grouped_ffn_int8_workspace_bytes");
  if (!aligned_to(workspace, 256)) return fail(LLEP_E_WORKSPACE, "workspace not 256-byte aligned");
  llep::FfnInt8Args a = {};
  a.R = params->T * params->K;
  a.P = params->P;
  a.E = params->E;
  a.D = D;
  a.F = F;
  a.K = params->K;
  a.device = device;
  a.groups = plan->groups;
  a.group_begin = plan->group_begin;
  a.row_pair = row_pair;
  a.x_perm = x_perm;
  a.w_gate_up = w_gate_up_packed;
  a.w_down = w_down_packed;
  a.x_scale = x_scale;
  a.gate_scale = gate_scale;
  a.up_scale = up_scale;
  a.down_scale = down_scale;
  a.out_perm = out_perm;
  a.f32_out = f32_out;
  a.ws = workspace;
  return hip_result(llep::launch_ffn_int8(a, stream), name);
}

int llep_grouped_ffn_int8(const llep_plan_params *params, const llep_plan_buffers *plan,
                          int32_t device, const int8_t *x_perm, const float *x_scale,
                          const int32_t *row_pair, const int8_t *w_gate_up_packed,
                          const float *gate_scale, const float *up_scale,
                          const int8_t *w_down_packed, const float *down_scale, int32_t D,
                          int32_t F, void *out_perm, void *workspace, size_t workspace_bytes,
                          hipStream_t stream) {
  return grouped_ffn_int8(params, plan, device, x_perm, x_scale, row_pair, w_gate_up_packed,
                          gate_scale, up_scale, w_down_packed, down_scale, D, F, out_perm, false,
                          workspace, workspace_bytes, stream, "llep_grouped_ffn_int8");
}

int llep_grouped_ffn_int8_f32(const llep_plan_params *params, const llep_plan_buffers *plan,
                              int32_t device, const int8_t *x_perm, const float *x_scale,
                              const int32_t *row_pair, const int8_t *w_gate_up_packed,
                              const float *gate_scale, const float *up_scale,
                              const int8_t *w_down_packed, const float *down_scale, int32_t D,
                              int32_t F, float *out_perm, void *workspace, size_t workspace_bytes,
                              hipStream_t stream) {
  return grouped_ffn_int8(params, plan, device, x_perm, x_scale, row_pair, w_gate_up_packed,
                          gate_scale, up_scale, w_down_packed, down_scale, D, F, out_perm, true,
                          workspace, workspace_bytes, stream, "llep_grouped_ffn_int8_f32");
}

int llep_route(const llep_route_params *params, llep_dtype dtype, const void *logits,
               const float *bias, int32_t *ids, float *gates, hipStream_t stream) {
  const int rc = check_route(params, dtype);
  if (rc != LLEP_OK) return rc;
  if (params->T > 0 && (!logits || !ids || !gates)) return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned_to(logits, elem_bytes(dtype)) || !aligned_to(bias, 4) || !aligned_to(ids, 4) ||
      !aligned_to(gates, 4))
    return fail(LLEP_E_ARG, "data not aligned to its type");
  llep::RouteArgs a = route_args(params, dtype);
  a.logits = logits;
  a.bias = bias;
  a.ids = ids;
  a.gates = gates;
  return hip_result(llep::launch_route(a, false, stream), "llep_route");
}

int llep_route_backward(const llep_route_params *params, llep_dtype dtype, const void *logits,
                        const int32_t *ids, const float *gates, const float *d_gates,
                        void *d_logits, hipStream_t stream) {
  const int rc = check_route(params, dtype);
  if (rc != LLEP_OK) return rc;
  const bool reads = params->score != LLEP_SCORE_SOFTMAX || !params->renormalize;
  if (params->T > 0 && ((reads && !logits) || !ids || !gates || !d_gates || !d_logits))
    return fail(LLEP_E_ARG, "a data pointer is null");
  const size_t eb = elem_bytes(dtype);
  if (!aligned_to(logits, eb) || !aligned_to(d_logits, eb) || !aligned_to(ids, 4) ||
      !aligned_to(gates, 4) || !aligned_to(d_gates, 4))
    return fail(LLEP_E_ARG, "data not aligned to its type");
  llep::RouteArgs a = route_args(params, dtype);
  a.logits = logits;
  a.ids = const_cast<int32_t *>(ids);
  a.gates = const_cast<float *>(gates);
  a.d_gates = d_gates;
  a.d_logits = d_logits;
  return hip_result(llep::launch_route(a, true, stream), "llep_route_backward");
}

int32_t llep_mxfp4_row_bytes(int32_t D) {
  return D < 1 || D > LLEP_MAX_FFN_DIM ? -1 : llep::mxfp4_row_bytes(D);
}

int32_t llep_mxfp4_scale_bytes(int32_t D) {
  return D < 1 || D > LLEP_MAX_FFN_DIM ? -1 : llep::mxfp4_scale_bytes(D);
}

int llep_quantize_rows_mxfp4(int64_t R, int32_t D, llep_dtype dtype, const void *x, uint8_t *q,
                             int32_t q_pitch, uint8_t *scale, int32_t scale_pitch,
                             hipStream_t stream) {
  const size_t eb = elem_bytes(dtype);
  if (eb == 0) return fail(LLEP_E_DTYPE, "unknown dtype");
  const int rc = check_mxfp4_rows(R, D, q, q_pitch, scale, scale_pitch);
  if (rc != LLEP_OK) return rc;
  if (R > 0 && !x) return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned_to(x, eb)) return fail(LLEP_E_ARG, "x not aligned to its type");
  return hip_result(
      llep::launch_quantize_mxfp4(R, D, dtype, x, q, q_pitch, scale, scale_pitch, stream),
      "llep_quantize_rows_mxfp4");
}

int llep_dequantize_rows_mxfp4(int64_t R, int32_t D, llep_dtype dtype, const uint8_t *q,
                               int32_t q_pitch, const uint8_t *scale, int32_t scale_pitch,
                               void *out, hipStream_t stream) {
  const size_t eb = elem_bytes(dtype);
  if (eb == 0) return fail(LLEP_E_DTYPE, "unknown dtype");
  const int rc = check_mxfp4_rows(R, D, q, q_pitch, scale, scale_pitch);
  if (rc != LLEP_OK) return rc;
  if (R > 0 && !out) return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned_to(out, eb)) return fail(LLEP_E_ARG, "out not aligned to its type");
  return hip_result(
      llep::launch_dequantize_mxfp4(R, D, dtype, q, q_pitch, scale, scale_pitch, out, stream),
      "llep_dequantize_rows_mxfp4");
}

size_t llep_packed_mxfp4_bytes(int32_t E, int32_t N, int32_t K) {
  if (E < 1 || E > LLEP_MAX_EXPERTS || N < 1 || N > LLEP_MAX_MXFP4_COLUMNS || K < 1 ||
      K > LLEP_MAX_FFN_DIM)
    return 0;
  return size_t(E) * llep::packed_mxfp4_bytes(N, K);
}

int llep_pack_mxfp4(int32_t E, int32_t N, int32_t K, const uint8_t *w, const uint8_t *scale,
                    const uint8_t *w_up, const uint8_t *up_scale, int32_t w_bytes,
                    int32_t scale_bytes, uint8_t *packed, hipStream_t stream) {
  if (llep_packed_mxfp4_bytes(E, N, K) == 0) return fail(LLEP_E_ARG, "E, N or K outside its range");
  if ((w_up != nullptr) != (up_scale != nullptr))
    return fail(LLEP_E_ARG, "w_up and up_scale: both or none");
  if (w_up && (N % 32 != 0 || N > LLEP_MAX_FFN_DIM))
    return fail(LLEP_E_ARG, "gate and up rows: N must be a multiple of 32, at most LLEP_MAX_FFN_DIM");
  if (w_bytes < (K + 1) / 2 || scale_bytes < (K + 31) / 32)
    return fail(LLEP_E_ARG, "w_bytes or scale_bytes below those of K values");
  if (!w || !scale || !packed) return fail(LLEP_E_ARG, "a weight pointer is null");
  if (!aligned16(packed)) return fail(LLEP_E_ARG, "packed weights not 16-byte aligned");
  return hip_result(llep::launch_pack_mxfp4(E, N, K, w, scale, w_up, up_scale, w_bytes, scale_bytes,
                                            packed, stream),
                    "llep_pack_mxfp4");
}

int llep_mxfp4_matmul(int64_t M, int32_t N, int32_t K, const uint8_t *x, int32_t q_pitch,
                      const uint8_t *x_scale, int32_t scale_pitch, const uint8_t *w_packed,
                      llep_dtype dtype, void *out, hipStream_t stream) {
  if (elem_bytes(dtype) == 0) return fail(LLEP_E_DTYPE, "unknown dtype");
  if (llep_packed_mxfp4_bytes(1, N, K) == 0) return fail(LLEP_E_ARG, "N or K outside its range");
  if (M > LLEP_MAX_MXFP4_ROWS) return fail(LLEP_E_ARG, "M above LLEP_MAX_MXFP4_ROWS");
  const int rc = check_mxfp4_rows(M, K, x, q_pitch, x_scale, scale_pitch);
  if (rc != LLEP_OK) return rc;
  if (!w_packed || (M > 0 && !out)) return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned16(w_packed) || !aligned16(out)) return fail(LLEP_E_ARG, "data not 16-byte aligned");
  llep::MxMatmulArgs a = {};
  a.M = M;
  a.N = N;
  a.K = K;
  a.x_pitch = q_pitch;
  a.s_pitch = scale_pitch;
  a.dtype = dtype;
  a.x = x;
  a.x_scale = x_scale;
  a.w = w_packed;
  a.out = out;
  return hip_result(llep::launch_mxfp4_matmul(a, stream), "llep_mxfp4_matmul");
}

size_t llep_grouped_ffn_mxfp4_workspace_bytes(const llep_plan_params *params, int32_t F) {
  if (check_params(params) != LLEP_OK || F < 1 || F > LLEP_MAX_FFN_DIM) return 0;
  return llep::ffn_mxfp4_workspace_bytes(params->T * params->K, params->E, params->P, F);
}

int llep_grouped_ffn_mxfp4(const llep_plan_params *params, const llep_plan_buffers *plan,
                           int32_t device, const uint8_t *x_perm, const uint8_t *w_gate_up_packed,
                           const uint8_t *w_down_packed, int32_t D, int32_t F, llep_dtype dtype,
                           void *out_perm, void *workspace, size_t workspace_bytes,
                           hipStream_t stream) {
  int rc = check_params(params);
  if (rc != LLEP_OK) return rc;
  if ((rc = check_plan_buffers(plan)) != LLEP_OK) return rc;
  if ((rc = check_ffn_dims(D, F, dtype)) != LLEP_OK) return rc;
  if (device < -1 || device >= params->P) return fail(LLEP_E_ARG, "device outside [-1, P)");
  // (arrays of no rows may have no address)
  if (!w_gate_up_packed || !w_down_packed || (params->T > 0 && (!x_perm || !out_perm)))
    return fail(LLEP_E_ARG, "a data pointer is null");
  if (!aligned16(x_perm) || !aligned16(w_gate_up_packed) || !aligned16(w_down_packed) ||
      !aligned16(out_perm))
    return fail(LLEP_E_ARG, "data not 16-byte aligned");
  const size_t need = llep_grouped_ffn_mxfp4_workspace_bytes(params, F);
  if (!workspace || workspace_bytes < need)
    return fail(LLEP_E_WORKSPACE,
                "workspace missing or smaller than llep_grouped_ffn_mxfp4_workspace_bytes");
  if (!aligned_to(workspace, 256)) return fail(LLEP_E_WORKSPACE, "workspace not 256-byte aligned");
  llep::FfnMxArgs a = {};
  a.R = params->T * params->K;
  a.P = params->P;
  a.E = params->E;
  a.D = D;
  a.F = F;
  a.device = device;
  a.groups = plan->groups;
  a.group_begin = plan->group_begin;
  a.x_perm = x_perm;
  a.w_gate_up = w_gate_up_packed;
  a.w_down = w_down_packed;
  a.out_perm = out_perm;
  a.f32_out = dtype == LLEP_F32;
  a.ws = workspace;
  return hip_result(llep::launch_ffn_mxfp4(a, stream), "llep_grouped_ffn_mxfp4");
}

}  // extern "C"
