// The context behind the C ABI and the argument checks its entry points share.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include <exception>
#include <string>
#include <vector>

#include "vp.h"
#include "vp_attend.h"
#include "vp_cache4.h"
#include "vp_internal.h"

struct vp_ctx {
  vp_config cfg;
  int device = 0;
  int num_sms = 0;
  vp::WsLayout lay;
  void* ws = nullptr;
  size_t ws_bytes = 0;
  float* z_ws = nullptr;
  float* split_st = nullptr;
  float* split_o = nullptr;
  float* gpart_o = nullptr;
  float* gpart_st = nullptr;
  float* mt_o = nullptr;
  float* mt_st = nullptr;
  float* hmax = nullptr;
  float diag_delta = 0.f;          // diagnostics (vp_set_diagnostics)
  int32_t* diag_n_act = nullptr;
  uint32_t* diag_bits = nullptr;
  int32_t score_path = VP_SCORE_AUTO;  // vp_set_score_path
  unsigned* tickets = nullptr;
  unsigned* err = nullptr;
  std::string last_error;
  std::vector<cudaEvent_t> tev;  // stage-timing events, 4 per slot
  int32_t tslots = 0;
  int64_t tcalls = 0;
  int32_t last_score_path = 0;  // vp_last_launch: score kernel and kernel count of the last call
  int32_t last_kernels = 0;
  void* new_ws = nullptr;  // workspace of vp_attend_new (vp_reserve_new)
  vp::NewLayout new_lay;
  void* ws4 = nullptr;  // workspace of vp_attend4 (vp_reserve4)
  vp::Layout4 lay4;
};

namespace vp {

inline vp_status fail(vp_ctx* ctx, vp_status st, const std::string& msg) {
  if (ctx) ctx->last_error = msg;
  else context_free_error() = msg;
  return st;
}

inline vp_status cuda_fail(vp_ctx* ctx, const char* what, cudaError_t e) {
  return fail(ctx, VP_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline bool kv_ok(const vp_ctx* ctx, const vp_kv* kv, const char* name, std::string* why) {
  const size_t esz = ctx->cfg.dtype == VP_BF16 ? 2 : 4;
  char buf[160];
  if (!kv || !kv->data) { snprintf(buf, sizeof buf, "%s: NULL cache", name); *why = buf; return false; }
  if (!aligned16(kv->data)) { snprintf(buf, sizeof buf, "%s: data must be 16-byte aligned", name); *why = buf; return false; }
  const int64_t strides[3] = {kv->stride_b, kv->stride_h, kv->stride_t};
  for (int64_t s : strides) {
    if (s < 0 || ((uint64_t)s * esz) % 16 != 0) {
      snprintf(buf, sizeof buf, "%s: strides must be >= 0 and multiples of 16 bytes", name); *why = buf; return false;
    }
  }
  if (ctx->cfg.paged) {
    if (!kv->block_table || kv->max_pages < 1 || kv->num_pages < 1) {
      snprintf(buf, sizeof buf, "%s: paged cache needs block_table, max_pages >= 1, num_pages >= 1", name);
      *why = buf; return false;
    }
  } else if (kv->block_table) {
    snprintf(buf, sizeof buf, "%s: block_table given but the context is not paged", name); *why = buf; return false;
  }
  return true;
}

inline KvView view(const vp_kv& c) {
  return KvView{c.data, c.stride_b, c.stride_h, c.stride_t, c.block_table, c.max_pages, c.num_pages};
}

inline bool rows_ok(const vp_ctx* ctx, const vp_rows* r, const char* name, std::string* why) {
  const size_t esz = ctx->cfg.dtype == VP_BF16 ? 2 : 4;
  if (!r || !r->data) { *why = std::string(name) + ": NULL"; return false; }
  if (!aligned16(r->data)) { *why = std::string(name) + ": data must be 16-byte aligned"; return false; }
  for (int64_t s : {r->stride_b, r->stride_n, r->stride_h})
    if (s < 0 || ((uint64_t)s * esz) % 16 != 0) {
      *why = std::string(name) + ": strides must be >= 0 and multiples of 16 bytes";
      return false;
    }
  return true;
}

// No exception may cross the C ABI (a failed allocation of an error text), and
// nothing is allocated or launched on another device than the context's.
template <typename F>
vp_status guarded(vp_ctx* ctx, const char* name, F&& f) {
  if (!ctx) return VP_ERR_NOT_INITIALIZED;
  try {
    ctx->last_error.clear();
    int device = 0;
    const cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return cuda_fail(ctx, name, e);
    if (device != ctx->device)
      return fail(ctx, VP_ERR_INVALID_ARG, std::string(name) + ": the current device is " + std::to_string(device) +
                  ", the context's is " + std::to_string(ctx->device));
    return f();
  } catch (const std::exception&) {
    return VP_ERR_CUDA;
  }
}

}  // namespace vp
