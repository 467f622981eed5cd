// C ABI of the windowed attention: argument checks and launches.
#include <math.h>

#include "heads.h"
#include "window_args.h"

using namespace elasto;

namespace {

// A copy with the window no wider than any sequence; false and the error set on a bad one.
bool check_desc(const elasto_window_t* d, elasto_window_t* a) {
  if (!d) return fail(ELASTO_ERR_INVALID_ARG, "window attention: NULL description"), false;
  *a = *d;
  if (a->dtype != ELASTO_BF16 && a->dtype != ELASTO_FP32)
    return fail(ELASTO_ERR_INVALID_ARG, "bad dtype %d", a->dtype), false;
  if (a->head_dim != 64 && a->head_dim != 128)
    return fail(ELASTO_ERR_INVALID_ARG, "window attention needs head_dim 64 or 128, not %d", a->head_dim), false;
  if (a->batch < 0 || a->q_tokens < 0 || a->k_tokens < 0 || a->k_tokens > (1 << 29) || a->heads < 1 ||
      a->kv_heads < 1 || a->heads % a->kv_heads ||
      (int64_t)a->q_tokens * (a->heads / a->kv_heads) > (1 << 29) ||
      (int64_t)a->batch * a->heads > (1 << 29))
    return fail(ELASTO_ERR_INVALID_ARG, "window attention: bad batch, tokens or heads"), false;
  if (a->window < 1) return fail(ELASTO_ERR_INVALID_ARG, "window %d is below 1", a->window), false;
  if (a->sinks < 0 || a->sinks > kMaxSinks)
    return fail(ELASTO_ERR_INVALID_ARG, "sinks %d outside [0, %d]", a->sinks, kMaxSinks), false;
  if (!(a->scale >= 1e-30f) || !(a->scale <= 1e30f))
    return fail(ELASTO_ERR_INVALID_ARG, "window attention: scale must be positive, within [1e-30, 1e30]"), false;
  if (!aligned(a->q_lens, 4) || !aligned(a->k_lens, 4))
    return fail(ELASTO_ERR_INVALID_ARG, "window attention: misaligned lengths"), false;
  // No distance between a query and a key of one sequence reaches 2^30.
  a->window = a->window < (1 << 30) ? a->window : (1 << 30);
  a->causal = a->causal != 0;
  return true;
}

bool set_view(const char* name, const elasto_window_t& a, const elasto_heads_t* t, int64_t tokens,
              int heads, bool written, View* v) {
  return take_view("window attention", name, t, a.batch, tokens, heads, a.head_dim,
                   a.dtype == ELASTO_BF16 ? 2 : 4, written, v);
}

// Tiles of up to 64 tokens (of `heads` heads together) are loaded at 32-bit
// offsets from their first row; a single head is reached by its address.
bool check_reach(const char* name, const View& v, int heads) {
  const int64_t limit = kReach;
  const int64_t sh = heads > 1 ? v.sh : 0;
  if (v.st > limit || sh > limit || 64 * v.st + (heads - 1) * sh + 512 >= limit)
    return fail(ELASTO_ERR_INVALID_ARG, "window attention: 64 tokens of %s span nearly 4 GiB or more", name), false;
  return true;
}

bool check_ws(const void* ws, int64_t have, int64_t need) {
  if (need == 0) return true;
  if (!ws || have < need)
    return fail(ELASTO_ERR_INVALID_ARG, "window attention: the workspace holds %lld of %lld bytes",
                (long long)(ws ? have : 0), (long long)need), false;
  if (!aligned(ws, 256)) return fail(ELASTO_ERR_INVALID_ARG, "the workspace must be 256-byte aligned"), false;
  return true;
}

// The launchers refuse grids that a launch does not hold before they launch any.
elasto_status_t launch_error(hipError_t e) {
  if (e == hipErrorInvalidConfiguration)
    return fail(ELASTO_ERR_INVALID_ARG, "window attention: more than %lld workgroups", (long long)kMaxBlocks - 1);
  return fail(ELASTO_ERR_HIP, "window attention: %s", hipGetErrorString(e));
}

}  // namespace

extern "C" {

elasto_status_t elasto_window_attention_workspace(const elasto_window_t* desc, int32_t backward,
                                                  int64_t* bytes) {
  if (!bytes) return fail(ELASTO_ERR_INVALID_ARG, "NULL argument");
  elasto_window_t a;
  if (!check_desc(desc, &a)) return ELASTO_ERR_INVALID_ARG;
  *bytes = a.batch == 0 ? 0 : backward ? window_bwd_workspace(a) : a.q_tokens == 0 ? 0 : window_fwd_workspace(a);
  return ELASTO_OK;
}

elasto_status_t elasto_op_window_attention(const elasto_window_t* desc, const elasto_heads_t* q,
                                           const elasto_heads_t* k, const elasto_heads_t* v,
                                           const elasto_heads_t* o, float* lse, void* workspace,
                                           int64_t workspace_bytes, void* hip_stream) {
  elasto_window_t a;
  if (!check_desc(desc, &a)) return ELASTO_ERR_INVALID_ARG;
  if (a.batch == 0 || a.q_tokens == 0) return ELASTO_OK;
  WindowTensors t = {};
  if (!set_view("q", a, q, a.q_tokens, a.heads, false, &t.q) ||
      !set_view("k", a, k, a.k_tokens, a.kv_heads, false, &t.k) ||
      !set_view("v", a, v, a.k_tokens, a.kv_heads, false, &t.v) ||
      !set_view("o", a, o, a.q_tokens, a.heads, true, &t.o) || !check_reach("k", t.k, 1) ||
      !check_reach("v", t.v, 1))
    return ELASTO_ERR_INVALID_ARG;
  if (!aligned(lse, 4)) return fail(ELASTO_ERR_INVALID_ARG, "window attention: misaligned lse");
  if (!check_ws(workspace, workspace_bytes, window_fwd_workspace(a))) return ELASTO_ERR_INVALID_ARG;
  t.lse = lse;
  const hipError_t e = launch_window_fwd(a, t, workspace, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return launch_error(e);
  return ELASTO_OK;
}

elasto_status_t elasto_op_window_attention_bwd(const elasto_window_t* desc, const elasto_heads_t* q,
                                               const elasto_heads_t* k, const elasto_heads_t* v,
                                               const elasto_heads_t* o, const float* lse,
                                               const elasto_heads_t* dout, const elasto_heads_t* dq,
                                               const elasto_heads_t* dk, const elasto_heads_t* dv,
                                               void* workspace, int64_t workspace_bytes,
                                               void* hip_stream) {
  elasto_window_t a;
  if (!check_desc(desc, &a)) return ELASTO_ERR_INVALID_ARG;
  if (a.batch == 0 || (a.q_tokens == 0 && a.k_tokens == 0)) return ELASTO_OK;
  WindowTensors t = {};
  if (!set_view("q", a, q, a.q_tokens, a.heads, false, &t.q) ||
      !set_view("k", a, k, a.k_tokens, a.kv_heads, false, &t.k) ||
      !set_view("v", a, v, a.k_tokens, a.kv_heads, false, &t.v) ||
      !set_view("o", a, o, a.q_tokens, a.heads, false, &t.o) ||
      !set_view("dout", a, dout, a.q_tokens, a.heads, false, &t.dout) ||
      !set_view("dq", a, dq, a.q_tokens, a.heads, true, &t.dq) ||
      !set_view("dk", a, dk, a.k_tokens, a.kv_heads, true, &t.dk) ||
      !set_view("dv", a, dv, a.k_tokens, a.kv_heads, true, &t.dv) || !check_reach("k", t.k, 1) ||
      !check_reach("v", t.v, 1) || !check_reach("q", t.q, a.heads / a.kv_heads) ||
      !check_reach("dout", t.dout, a.heads / a.kv_heads))
    return ELASTO_ERR_INVALID_ARG;
  if (a.q_tokens > 0 && (!lse || !aligned(lse, 4)))
    return fail(ELASTO_ERR_INVALID_ARG, "window attention: lse is NULL or misaligned");
  if (!check_ws(workspace, workspace_bytes, window_bwd_workspace(a))) return ELASTO_ERR_INVALID_ARG;
  t.lse = const_cast<float*>(lse);
  const hipError_t e = launch_window_bwd(a, t, workspace, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return launch_error(e);
  return ELASTO_OK;
}

}  // extern "C"
