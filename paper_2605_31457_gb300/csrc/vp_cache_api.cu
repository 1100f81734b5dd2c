// Host side of vp_reserve_new, vp_attend_new and vp_evict: argument checks,
// workspace ownership and launches.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <cmath>
#include <string>

#include "vp.h"
#include "vp_attend.h"
#include "vp_ctx.h"
#include "vp_internal.h"

using vp::aligned16;
using vp::cuda_fail;
using vp::fail;
using vp::guarded;
using vp::kv_ok;
using vp::rows_ok;
using vp::view;

namespace {

constexpr int kMaxGridY = 65535;  // sequences of a call of vp_evict

bool weights_ok(const vp_weights* w, const char* name, std::string* why) {
  if (!w->data || (reinterpret_cast<uintptr_t>(w->data) & 3u)) {
    *why = std::string(name) + ": data must be non-NULL and 4-byte aligned";
    return false;
  }
  if (w->stride_b < 0 || w->stride_h < 0) { *why = std::string(name) + ": strides must be >= 0"; return false; }
  return true;
}

bool same_cache(const vp_kv& a, const vp_kv& b) {
  return a.data == b.data && a.stride_b == b.stride_b && a.stride_h == b.stride_h && a.stride_t == b.stride_t &&
         a.block_table == b.block_table && a.max_pages == b.max_pages && a.num_pages == b.num_pages;
}

// Two caches in one pool whose pages the caller keeps apart (a block table each).
bool other_pages(const vp_kv& a, const vp_kv& b) {
  return a.block_table && b.block_table && a.block_table != b.block_table;
}

vp_status reserve_new(vp_ctx* ctx, int32_t max_new, int32_t max_weight_new) {
  const vp_config& c = ctx->cfg;
  if (max_new < 1 || max_new > c.max_seq)
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_reserve_new: max_new must lie in [1, max_seq]");
  if (max_weight_new < 0 || max_weight_new > max_new)
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_reserve_new: max_weight_new must lie in [0, max_new]");
  const int G = c.num_q_heads / c.num_kv_heads;
  if ((int64_t)max_weight_new * G > vp::kNewWeightRows)
    return fail(ctx, VP_ERR_UNSUPPORTED, "vp_reserve_new: weights need max_weight_new * G <= 128");
  if ((int64_t)max_new * G >= (1 << 28))
    return fail(ctx, VP_ERR_UNSUPPORTED, "vp_reserve_new: max_new * G is too large");
  cudaError_t e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return cuda_fail(ctx, "vp_reserve_new", e);
  if (ctx->new_ws) cudaFree(ctx->new_ws);
  ctx->new_ws = nullptr;
  ctx->new_lay = vp::NewLayout();
  const vp::NewLayout lay = vp::new_layout(c.max_batch, c.num_q_heads, c.num_kv_heads, c.head_dim, c.max_seq, max_new,
                                           max_weight_new, ctx->num_sms);
  e = vp::configure_attend();
  if (e == cudaSuccess) e = cudaMalloc(&ctx->new_ws, lay.total);
  if (e == cudaSuccess) {
    e = cudaMemset(static_cast<char*>(ctx->new_ws) + lay.o_tk, 0, lay.o_lse - lay.o_tk);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) cudaFree(ctx->new_ws);
  }
  if (e != cudaSuccess) {
    ctx->new_ws = nullptr;
    cudaGetLastError();
    return cuda_fail(ctx, "vp_reserve_new: workspace", e);
  }
  ctx->new_lay = lay;
  return VP_OK;
}

vp_status attend_new(vp_ctx* ctx, int32_t batch, int32_t n_new, const vp_rows* q, const vp_kv* k_cache,
                     const vp_kv* v_cache, const int32_t* seq_len, const int32_t* new_len, const vp_visible* visible,
                     const vp_rows* out, float* lse, const vp_weights* weight_in, const vp_weights* weight_out,
                     void* cuda_stream) {
  const vp_config& c = ctx->cfg;
  if (batch < 0) return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend_new: batch < 0");
  if (batch > c.max_batch) return fail(ctx, VP_ERR_CAPACITY, "vp_attend_new: batch exceeds max_batch");
  if (n_new < 0) return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend_new: n_new < 0");
  if (!visible) return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend_new: visible is NULL");
  if (visible->window < VP_NO_WINDOW || visible->sinks < 0)
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend_new: window must be >= 0 or VP_NO_WINDOW, sinks >= 0");
  if (!(visible->scale >= 0.f) || !std::isfinite(visible->scale))
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend_new: scale must be finite and >= 0");
  if (weight_in && !weight_out)
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend_new: weight_in needs weight_out");
  const int H = c.num_q_heads, Hkv = c.num_kv_heads, G = H / Hkv;
  if (weight_out && (int64_t)n_new * G > vp::kNewWeightRows)
    return fail(ctx, VP_ERR_UNSUPPORTED, "vp_attend_new: weights need n_new * G <= 128");
  if (n_new > ctx->new_lay.max_new || (weight_out && n_new > ctx->new_lay.max_weight_new))
    return fail(ctx, VP_ERR_CAPACITY, "vp_attend_new: vp_reserve_new has not reserved for " + std::to_string(n_new) +
                " new tokens" + (weight_out ? " with weights" : ""));
  if (batch == 0 || n_new == 0) return VP_OK;
  std::string why;
  if (!seq_len) return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend_new: seq_len is NULL");
  if (!rows_ok(ctx, q, "q", &why) || !rows_ok(ctx, out, "out", &why) || !kv_ok(ctx, k_cache, "k_cache", &why) ||
      !kv_ok(ctx, v_cache, "v_cache", &why) || (weight_in && !weights_ok(weight_in, "weight_in", &why)) ||
      (weight_out && !weights_ok(weight_out, "weight_out", &why)))
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend_new: " + why);

  vp::AttendParams p;
  memset(&p, 0, sizeof p);
  p.dtype = c.dtype;
  p.B = batch; p.H = H; p.Hkv = Hkv; p.G = G; p.D = c.head_dim; p.max_seq = c.max_seq;
  p.paged = c.paged; p.page_size = c.paged ? c.page_size : 1;
  while ((1 << p.page_shift) < p.page_size) ++p.page_shift;
  p.n_new = n_new; p.R = n_new * G;
  p.g_mul = G == 1 ? 0u : (uint32_t)((1ull << 32) / (unsigned)G + 1);
  p.q = vp::RowView{q->data, q->stride_b, q->stride_n, q->stride_h};
  p.out = vp::RowView{out->data, out->stride_b, out->stride_n, out->stride_h};
  p.k = view(*k_cache); p.v = view(*v_cache);
  p.seq_len = seq_len; p.new_len = new_len;
  p.window = visible->window; p.sinks = visible->sinks;
  p.c_log2 = (visible->scale > 0.f ? visible->scale : 1.0f / sqrtf((float)c.head_dim)) * 1.4426950408889634f;
  p.lse = lse;
  p.weigh = weight_out != nullptr;
  if (weight_in) p.w_in = vp::WeightView{weight_in->data, weight_in->stride_b, weight_in->stride_h};
  if (weight_out) p.w_out = vp::WeightView{weight_out->data, weight_out->stride_b, weight_out->stride_h};
  char* ws = static_cast<char*>(ctx->new_ws);
  p.part_st = reinterpret_cast<float*>(ws + ctx->new_lay.o_st);
  p.part_o = reinterpret_cast<float*>(ws + ctx->new_lay.o_o);
  p.z = reinterpret_cast<float*>(ws + ctx->new_lay.o_z);
  p.z_row = ctx->new_lay.z_row;
  p.err = ctx->err;
  p.num_sms = ctx->num_sms;
  p.tickets = reinterpret_cast<unsigned*>(ws + ctx->new_lay.o_tk);
  p.lse2 = reinterpret_cast<float*>(ws + ctx->new_lay.o_lse);
  vp::plan_attend(p);
  const cudaError_t e = vp::launch_attend(p, static_cast<cudaStream_t>(cuda_stream));
  if (e != cudaSuccess) return cuda_fail(ctx, "vp_attend_new: launch", e);
  return VP_OK;
}

vp_status evict(vp_ctx* ctx, int32_t batch, const vp_kv* k_src, const vp_kv* v_src, const int32_t* seq_len,
                const vp_evict_policy* policy, const vp_kv* k_dst, const vp_kv* v_dst, const vp_weights* weight,
                const vp_weights* weight_dst, int32_t* kept_idx, int32_t kept_cap, int32_t* new_len,
                void* cuda_stream) {
  const vp_config& c = ctx->cfg;
  if (batch < 0) return fail(ctx, VP_ERR_INVALID_ARG, "vp_evict: batch < 0");
  if (batch > c.max_batch) return fail(ctx, VP_ERR_CAPACITY, "vp_evict: batch exceeds max_batch");
  if (batch > kMaxGridY) return fail(ctx, VP_ERR_UNSUPPORTED, "vp_evict: batch above 65535 is not supported");
  if (!policy) return fail(ctx, VP_ERR_INVALID_ARG, "vp_evict: policy is NULL");
  if (policy->keep < 1 || policy->sinks < 0 || policy->recent < 0 ||
      (int64_t)policy->sinks + policy->recent > policy->keep)
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_evict: needs keep >= 1, sinks >= 0, recent >= 0, sinks + recent <= keep");
  if (policy->granularity != 0 && policy->granularity != 1)
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_evict: granularity must be 0 or 1");
  if (kept_cap < policy->keep)
    return fail(ctx, VP_ERR_CAPACITY, "vp_evict: kept_cap " + std::to_string(kept_cap) + " is below keep " +
                std::to_string(policy->keep));
  if (batch == 0) return VP_OK;
  std::string why;
  if (!seq_len || !kept_idx || !new_len || !weight) return fail(ctx, VP_ERR_INVALID_ARG, "vp_evict: NULL argument");
  if (!kv_ok(ctx, k_src, "k_src", &why) || !kv_ok(ctx, v_src, "v_src", &why) || !weights_ok(weight, "weight", &why) ||
      (weight_dst && !weights_ok(weight_dst, "weight_dst", &why)))
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_evict: " + why);
  const size_t esz = c.dtype == VP_BF16 ? 2 : 4;
  for (const vp_kv* d : {k_dst, v_dst}) {
    if (!d || !d->data || !aligned16(d->data))
      return fail(ctx, VP_ERR_INVALID_ARG, "vp_evict: a destination needs 16-byte-aligned data");
    for (int64_t s : {d->stride_b, d->stride_h, d->stride_t})
      if (s < 0 || ((uint64_t)s * esz) % 16 != 0)
        return fail(ctx, VP_ERR_INVALID_ARG, "vp_evict: destination strides must be >= 0 and multiples of 16 bytes");
    if (d->block_table && (!c.paged || d->max_pages < 1 || d->num_pages < 1))
      return fail(ctx, VP_ERR_INVALID_ARG, "vp_evict: a paged destination needs a paged context, max_pages >= 1 and "
                  "num_pages >= 1");
  }
  const bool in_place = same_cache(*k_src, *k_dst);
  if (in_place != same_cache(*v_src, *v_dst) ||
      (!in_place && ((k_src->data == k_dst->data && !other_pages(*k_src, *k_dst)) ||
                     (v_src->data == v_dst->data && !other_pages(*v_src, *v_dst)))))
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_evict: the destinations must be the sources themselves or not overlap them");
  if (weight_dst) {
    // In place the freed entries up to seq_len are cleared, which only weight itself has room for.
    const bool same = weight_dst->data == weight->data;
    if (in_place ? !same || weight_dst->stride_b != weight->stride_b || weight_dst->stride_h != weight->stride_h : same)
      return fail(ctx, VP_ERR_INVALID_ARG, "vp_evict: weight_dst must be weight itself in place, and must not overlap it "
                  "otherwise");
  }
  vp::EvictParams p;
  memset(&p, 0, sizeof p);
  p.esz = (int)esz;
  p.B = batch; p.Hkv = c.num_kv_heads; p.D = c.head_dim; p.max_seq = c.max_seq;
  p.page_size = c.paged ? c.page_size : 1;
  while ((1 << p.page_shift) < p.page_size) ++p.page_shift;
  p.ks = view(*k_src); p.vs = view(*v_src); p.kd = view(*k_dst); p.vd = view(*v_dst);
  p.in_place = in_place;
  p.seq_len = seq_len;
  p.keep = policy->keep; p.sinks = policy->sinks; p.recent = policy->recent; p.granularity = policy->granularity;
  p.w = vp::WeightView{weight->data, weight->stride_b, weight->stride_h};
  if (weight_dst) p.wd = vp::WeightView{weight_dst->data, weight_dst->stride_b, weight_dst->stride_h};
  p.kept_idx = kept_idx; p.kept_cap = kept_cap; p.new_len = new_len;
  p.err = ctx->err;
  p.num_sms = ctx->num_sms;
  const cudaError_t e = vp::launch_evict(p, static_cast<cudaStream_t>(cuda_stream));
  if (e != cudaSuccess) return cuda_fail(ctx, "vp_evict: launch", e);
  return VP_OK;
}

}  // namespace

extern "C" {

vp_status vp_reserve_new(vp_ctx* ctx, int32_t max_new, int32_t max_weight_new) {
  return guarded(ctx, "vp_reserve_new", [&] { return reserve_new(ctx, max_new, max_weight_new); });
}

vp_status vp_attend_new(vp_ctx* ctx, int32_t batch, int32_t n_new, const vp_rows* q,
                        const vp_kv* k_cache, const vp_kv* v_cache,
                        const int32_t* seq_len, const int32_t* new_len, const vp_visible* visible,
                        const vp_rows* out, float* lse,
                        const vp_weights* weight_in, const vp_weights* weight_out, void* cuda_stream) {
  return guarded(ctx, "vp_attend_new", [&] {
    return attend_new(ctx, batch, n_new, q, k_cache, v_cache, seq_len, new_len, visible, out, lse, weight_in,
                      weight_out, cuda_stream);
  });
}

vp_status vp_evict(vp_ctx* ctx, int32_t batch, const vp_kv* k_src, const vp_kv* v_src,
                   const int32_t* seq_len, const vp_evict_policy* policy,
                   const vp_kv* k_dst, const vp_kv* v_dst,
                   const vp_weights* weight, const vp_weights* weight_dst,
                   int32_t* kept_idx, int32_t kept_cap, int32_t* new_len, void* cuda_stream) {
  return guarded(ctx, "vp_evict", [&] {
    return evict(ctx, batch, k_src, v_src, seq_len, policy, k_dst, v_dst, weight, weight_dst, kept_idx, kept_cap,
                 new_len, cuda_stream);
  });
}

}  // extern "C"
