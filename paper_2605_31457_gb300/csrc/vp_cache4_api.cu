// Host side of vp_append, vp_append4, vp_reserve4 and vp_attend4: argument checks,
// workspace ownership and launches.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <cmath>
#include <string>
#include <type_traits>

#include "vp.h"
#include "vp_cache4.h"
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

vp::RowView view(const vp_rows& r) { return vp::RowView{r.data, r.stride_b, r.stride_n, r.stride_h}; }
vp::Kv4View view(const vp_kv4& c) {
  return vp::Kv4View{static_cast<uint8_t*>(c.codes), static_cast<uint16_t*>(c.scales),
                     c.code_stride_b, c.code_stride_h, c.code_stride_t,
                     c.scale_stride_b, c.scale_stride_h, c.scale_stride_t,
                     c.block_table, c.max_pages, c.num_pages};
}

bool kv4_ok(const vp_ctx* ctx, const vp_kv4* kv, const char* name, std::string* why) {
  const int per = ctx->cfg.head_dim / vp::kGroup4;  // scales of a row
  if (!kv || !kv->codes || !kv->scales) { *why = std::string(name) + ": NULL cache"; return false; }
  if (!aligned16(kv->codes) || (reinterpret_cast<uintptr_t>(kv->scales) % (2 * per)) != 0) {
    *why = std::string(name) + ": codes must be 16-byte aligned, scales " + std::to_string(2 * per) + "-byte aligned";
    return false;
  }
  for (int64_t s : {kv->code_stride_b, kv->code_stride_h, kv->code_stride_t})
    if (s < 0 || s % 16 != 0) { *why = std::string(name) + ": code strides must be >= 0 and multiples of 16"; return false; }
  for (int64_t s : {kv->scale_stride_b, kv->scale_stride_h, kv->scale_stride_t})
    if (s < 0 || s % per != 0) {
      *why = std::string(name) + ": scale strides must be >= 0 and multiples of " + std::to_string(per);
      return false;
    }
  if (ctx->cfg.paged) {
    if (!kv->block_table || kv->max_pages < 1 || kv->num_pages < 1) {
      *why = std::string(name) + ": paged cache needs block_table, max_pages >= 1, num_pages >= 1";
      return false;
    }
  } else if (kv->block_table) {
    *why = std::string(name) + ": block_table given but the context is not paged";
    return false;
  }
  return true;
}

bool rotation_ok(const vp_ctx* ctx, const vp_rotation& r, std::string* why) {
  if (!r.cos_sin || !aligned16(r.cos_sin)) { *why = "rotation: cos_sin must be non-NULL and 16-byte aligned"; return false; }
  if (r.max_pos < 1) { *why = "rotation: max_pos must be >= 1"; return false; }
  if (r.rot_dim < 16 || r.rot_dim % 16 != 0 || r.rot_dim > ctx->cfg.head_dim) {
    *why = "rotation: rot_dim must be a multiple of 16 in [16, head_dim]";
    return false;
  }
  if (r.interleaved != 0 && r.interleaved != 1) { *why = "rotation: interleaved must be 0 or 1"; return false; }
  if (r.axes < 1 || r.axes > 3 || (r.axes > 1 && !r.pos)) {
    *why = "rotation: axes must lie in [1, 3], and be 1 without pos";
    return false;
  }
  if (r.axes > 1) {
    int64_t sum = 0;
    for (int a = 0; a < r.axes; ++a) {
      if (r.sections[a] < 0) { *why = "rotation: sections must be >= 0"; return false; }
      sum += r.sections[a];
    }
    if (sum != r.rot_dim / 2) { *why = "rotation: the axes' sections must add up to rot_dim / 2"; return false; }
  }
  return true;
}

// Rows that a call writes: no two of them overlap.
bool apart_ok(const vp_ctx* ctx, const vp_rows& r, int batch, int n_new, int heads, const char* name, std::string* why) {
  if (vp::rows_apart(r.stride_b, r.stride_h, r.stride_n, batch, heads, n_new, ctx->cfg.head_dim)) return true;
  *why = std::string(name) + ": rows that are written need strides of at least head_dim";
  return false;
}
// The same of a cache: its strides, its sequences or pages, elements of a row.
bool apart_ok(const vp_ctx* ctx, int64_t sb, int64_t sh, int64_t st, int64_t lead, int64_t row, const char* name,
              std::string* why) {
  const vp_config& c = ctx->cfg;
  if (vp::rows_apart(sb, sh, st, lead, c.num_kv_heads, c.paged ? c.page_size : c.max_seq, row)) return true;
  *why = std::string(name) + ": a cache that is written needs strides of at least a row";
  return false;
}
bool apart_ok(const vp_ctx* ctx, const vp_kv& kv, int batch, const char* name, std::string* why) {
  return apart_ok(ctx, kv.stride_b, kv.stride_h, kv.stride_t, ctx->cfg.paged ? kv.num_pages : batch, ctx->cfg.head_dim,
                  name, why);
}
bool apart_ok(const vp_ctx* ctx, const vp_kv4& kv, int batch, const char* name, std::string* why) {
  const int64_t lead = ctx->cfg.paged ? kv.num_pages : batch, D = ctx->cfg.head_dim;
  return apart_ok(ctx, kv.code_stride_b, kv.code_stride_h, kv.code_stride_t, lead, D / 2, name, why) &&
         apart_ok(ctx, kv.scale_stride_b, kv.scale_stride_h, kv.scale_stride_t, lead, D / vp::kGroup4, name, why);
}

// Kv: vp_kv or vp_kv4.
template <typename Kv>
vp_status append(vp_ctx* ctx, const char* name, int32_t batch, int32_t n_new, const vp_rows* q, const vp_rows* k,
                 const vp_rows* v, const int32_t* seq_len, const int32_t* new_len, const vp_rotation* rotation,
                 const vp_rows* q_out, const Kv* k_cache, const Kv* v_cache, const vp_rows* k_held,
                 const vp_rows* v_held, void* cuda_stream) {
  constexpr bool kFour = std::is_same<Kv, vp_kv4>::value;
  const vp_config& c = ctx->cfg;
  const std::string at = std::string(name) + ": ";
  if (batch < 0) return fail(ctx, VP_ERR_INVALID_ARG, at + "batch < 0");
  if (batch > c.max_batch) return fail(ctx, VP_ERR_CAPACITY, at + "batch exceeds max_batch");
  if (n_new < 0) return fail(ctx, VP_ERR_INVALID_ARG, at + "n_new < 0");
  if (n_new > c.max_seq) return fail(ctx, VP_ERR_CAPACITY, at + "n_new exceeds max_seq");
  if ((q == nullptr) != (q_out == nullptr)) return fail(ctx, VP_ERR_INVALID_ARG, at + "q and q_out go together");
  if ((int64_t)batch * n_new * (c.num_q_heads + 2 * c.num_kv_heads) > INT32_MAX)
    return fail(ctx, VP_ERR_UNSUPPORTED, at + "more than 2^31 - 1 rows");
  std::string why;
  if (rotation && !rotation_ok(ctx, *rotation, &why)) return fail(ctx, VP_ERR_INVALID_ARG, at + why);
  if (batch == 0 || n_new == 0) return VP_OK;
  if (!seq_len) return fail(ctx, VP_ERR_INVALID_ARG, at + "seq_len is NULL");
  if ((q && (!rows_ok(ctx, q, "q", &why) || !rows_ok(ctx, q_out, "q_out", &why) ||
             !apart_ok(ctx, *q_out, batch, n_new, c.num_q_heads, "q_out", &why))) ||
      !rows_ok(ctx, k, "k", &why) || !rows_ok(ctx, v, "v", &why))
    return fail(ctx, VP_ERR_INVALID_ARG, at + why);
  for (const vp_rows* held : {k_held, v_held})
    if (held && (!rows_ok(ctx, held, "k_held, v_held", &why) ||
                 !apart_ok(ctx, *held, batch, n_new, c.num_kv_heads, "k_held, v_held", &why)))
      return fail(ctx, VP_ERR_INVALID_ARG, at + why);
  if (q && q->data == q_out->data &&
      (q->stride_b != q_out->stride_b || q->stride_n != q_out->stride_n || q->stride_h != q_out->stride_h))
    return fail(ctx, VP_ERR_INVALID_ARG, at + "q_out must be q itself or not overlap it");

  vp::AppendParams p = {};
  if constexpr (kFour) {
    if (!kv4_ok(ctx, k_cache, "k_cache", &why) || !kv4_ok(ctx, v_cache, "v_cache", &why) ||
        !apart_ok(ctx, *k_cache, batch, "k_cache", &why) || !apart_ok(ctx, *v_cache, batch, "v_cache", &why))
      return fail(ctx, VP_ERR_INVALID_ARG, at + why);
    p.kc4 = view(*k_cache);
    p.vc4 = view(*v_cache);
  } else {
    if (!kv_ok(ctx, k_cache, "k_cache", &why) || !kv_ok(ctx, v_cache, "v_cache", &why) ||
        !apart_ok(ctx, *k_cache, batch, "k_cache", &why) || !apart_ok(ctx, *v_cache, batch, "v_cache", &why))
      return fail(ctx, VP_ERR_INVALID_ARG, at + why);
    p.kc = vp::view(*k_cache);
    p.vc = vp::view(*v_cache);
  }
  p.B = batch; p.n_new = n_new; p.H = q ? c.num_q_heads : 0; p.Hkv = c.num_kv_heads; p.max_seq = c.max_seq;
  p.paged = c.paged; p.page_size = c.paged ? c.page_size : 1;
  while ((1 << p.page_shift) < p.page_size) ++p.page_shift;
  if (q) { p.q = view(*q); p.q_out = view(*q_out); }
  p.k = view(*k); p.v = view(*v);
  if (k_held) p.k_held = view(*k_held);
  if (v_held) p.v_held = view(*v_held);
  p.seq_len = seq_len; p.new_len = new_len;
  if (rotation) {
    const vp_rotation& r = *rotation;
    const int s0 = r.axes > 1 ? r.sections[0] : r.rot_dim / 2, s1 = r.axes > 1 ? r.sections[1] : 0;
    p.rot = vp::RotView{r.cos_sin, r.max_pos, r.rot_dim, r.interleaved, r.pos, r.axes, s0, s0 + s1};
  }
  p.err = ctx->err;
  const cudaError_t e = vp::launch_append(p, c.dtype, c.head_dim, kFour, ctx->num_sms, static_cast<cudaStream_t>(cuda_stream));
  if (e != cudaSuccess) return cuda_fail(ctx, (at + "launch").c_str(), e);
  return VP_OK;
}

vp_status reserve4(vp_ctx* ctx, int32_t max_new) {
  const vp_config& c = ctx->cfg;
  if (max_new < 1 || max_new > c.max_seq)
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_reserve4: max_new must lie in [1, max_seq]");
  if ((int64_t)max_new * (c.num_q_heads / c.num_kv_heads) >= (1 << 28))
    return fail(ctx, VP_ERR_UNSUPPORTED, "vp_reserve4: max_new * G is too large");
  cudaError_t e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return cuda_fail(ctx, "vp_reserve4", e);
  if (ctx->ws4) cudaFree(ctx->ws4);
  ctx->ws4 = nullptr;
  ctx->lay4 = vp::Layout4();
  const vp::Layout4 lay = vp::layout4(c.max_batch, c.num_q_heads, c.num_kv_heads, c.head_dim, c.max_seq, max_new, c.dtype,
                                      c.paged, c.page_size, ctx->num_sms);
  e = vp::configure_attend4();
  if (e == cudaSuccess && lay.seqs > 0) e = vp::configure_attend();
  if (e == cudaSuccess) e = cudaMalloc(&ctx->ws4, lay.total);
  if (e == cudaSuccess) {
    e = cudaMemset(static_cast<char*>(ctx->ws4) + lay.o_tk, 0, lay.o_lse - lay.o_tk);
    if (e == cudaSuccess && lay.seqs > 0) {  // pages that no call has filled are not mapped
      e = cudaMemset(static_cast<char*>(ctx->ws4) + lay.o_table, 0xff, lay.total - lay.o_table);
    }
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) cudaFree(ctx->ws4);
  }
  if (e != cudaSuccess) {
    ctx->ws4 = nullptr;
    cudaGetLastError();
    return cuda_fail(ctx, "vp_reserve4: workspace", e);
  }
  ctx->lay4 = lay;
  return VP_OK;
}

// The call by way of bf16 caches of the workspace, a group of sequences at a time.
cudaError_t staged(const vp::Attend4Params& all, const vp::Layout4& lay, char* ws, cudaStream_t st) {
  const int64_t row = (int64_t)lay.rows * all.D;  // elements of a staged (sequence, kv-head)
  const int64_t page = (int64_t)all.page_size * all.D;
  for (int b0 = 0; b0 < all.B; b0 += lay.seqs) {
    vp::Attend4Params p = all;
    p.B = all.B - b0 < lay.seqs ? all.B - b0 : lay.seqs;
    p.q.data = static_cast<uint16_t*>(all.q.data) + b0 * all.q.sb;
    p.out.data = static_cast<uint16_t*>(all.out.data) + b0 * all.out.sb;
    p.seq_len = all.seq_len + b0;
    if (all.new_len) p.new_len = all.new_len + b0;
    if (all.lse) p.lse = all.lse + (int64_t)b0 * all.n_new * all.H;
    vp::Unpack4Params u = {};
    u.B = p.B; u.Hkv = p.Hkv; u.D = p.D; u.max_seq = p.max_seq; u.n_new = p.n_new;
    u.paged = p.paged; u.page_size = p.page_size; u.page_shift = p.page_shift;
    u.k4 = all.k4; u.v4 = all.v4;
    for (vp::Kv4View* x : {&u.k4, &u.v4}) {
      if (p.paged) {
        x->block_table += (int64_t)b0 * x->max_pages;
      } else {
        x->codes += b0 * x->cb;
        x->scales += b0 * x->sb;
      }
    }
    u.k = ws + lay.o_k; u.v = ws + lay.o_v;
    u.rows = lay.rows; u.pages = lay.pages;
    u.table = reinterpret_cast<int32_t*>(ws + lay.o_table);
    u.seq_len = p.seq_len; u.new_len = p.new_len;
    u.window = p.window; u.sinks = p.sinks;
    u.err = p.err; u.num_sms = p.num_sms;
    cudaError_t e = vp::launch_unpack4(u, st);
    if (e != cudaSuccess) return e;
    if (p.paged)
      p.k = vp::KvView{u.k, p.Hkv * page, page, p.D, u.table, lay.pages, lay.seqs * lay.pages};
    else
      p.k = vp::KvView{u.k, p.Hkv * row, row, p.D, nullptr, 0, 0};
    p.v = p.k;
    p.v.data = u.v;
    vp::plan_attend(p);
    e = vp::launch_attend(p, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

vp_status attend4(vp_ctx* ctx, int32_t batch, int32_t n_new, const vp_rows* q, const vp_kv4* k_cache,
                  const vp_kv4* v_cache, const int32_t* seq_len, const int32_t* new_len, const vp_visible* visible,
                  const vp_rows* out, float* lse, void* cuda_stream) {
  const vp_config& c = ctx->cfg;
  if (batch < 0) return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend4: batch < 0");
  if (batch > c.max_batch) return fail(ctx, VP_ERR_CAPACITY, "vp_attend4: batch exceeds max_batch");
  if (n_new < 0) return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend4: n_new < 0");
  if (!visible) return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend4: visible is NULL");
  if (visible->window < VP_NO_WINDOW || visible->sinks < 0)
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend4: window must be >= 0 or VP_NO_WINDOW, sinks >= 0");
  if (!(visible->scale >= 0.f) || !std::isfinite(visible->scale))
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend4: scale must be finite and >= 0");
  if (n_new > ctx->lay4.max_new)
    return fail(ctx, VP_ERR_CAPACITY, "vp_attend4: vp_reserve4 has not reserved for " + std::to_string(n_new) + " new tokens");
  if (batch == 0 || n_new == 0) return VP_OK;
  std::string why;
  if (!seq_len) return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend4: seq_len is NULL");
  if (!rows_ok(ctx, q, "q", &why) || !rows_ok(ctx, out, "out", &why) ||
      !apart_ok(ctx, *out, batch, n_new, c.num_q_heads, "out", &why) || !kv4_ok(ctx, k_cache, "k_cache", &why) ||
      !kv4_ok(ctx, v_cache, "v_cache", &why))
    return fail(ctx, VP_ERR_INVALID_ARG, "vp_attend4: " + why);
  for (const vp_kv4* kv : {k_cache, v_cache})
    for (int64_t s : {kv->code_stride_t, kv->scale_stride_t, c.paged ? kv->code_stride_b : 0, c.paged ? kv->scale_stride_b : 0})
      if (s > INT32_MAX) return fail(ctx, VP_ERR_UNSUPPORTED, "vp_attend4: token and page strides must be below 2^31");

  vp::Attend4Params p = {};
  const int H = c.num_q_heads, Hkv = c.num_kv_heads, G = H / Hkv;
  p.dtype = c.dtype;
  p.B = batch; p.H = H; p.Hkv = Hkv; p.G = G; p.D = c.head_dim; p.max_seq = c.max_seq;
  p.paged = c.paged; p.page_size = c.paged ? c.page_size : 1;
  while ((1 << p.page_shift) < p.page_size) ++p.page_shift;
  p.n_new = n_new; p.R = n_new * G;
  p.g_mul = G == 1 ? 0u : (uint32_t)((1ull << 32) / (unsigned)G + 1);
  p.q = view(*q); p.out = view(*out);
  p.k4 = view(*k_cache); p.v4 = view(*v_cache);
  p.seq_len = seq_len; p.new_len = new_len;
  p.window = visible->window; p.sinks = visible->sinks;
  p.c_log2 = (visible->scale > 0.f ? visible->scale : 1.0f / sqrtf((float)c.head_dim)) * 1.4426950408889634f;
  p.lse = lse;
  char* ws = static_cast<char*>(ctx->ws4);
  p.part_st = reinterpret_cast<float*>(ws + ctx->lay4.o_st);
  p.part_o = reinterpret_cast<float*>(ws + ctx->lay4.o_o);
  p.tickets = reinterpret_cast<unsigned*>(ws + ctx->lay4.o_tk);
  p.err = ctx->err;
  p.num_sms = ctx->num_sms;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaSuccess;
  if (vp::stages(p.dtype, p.paged, p.page_size, p.R)) {
    e = staged(p, ctx->lay4, ws, st);
  } else {
    vp::plan_attend4(p);
    if (vp::line_bound((int64_t)p.B * p.Hkv * p.nqt, p.max_seq, p.fixed) > INT32_MAX)
      return fail(ctx, VP_ERR_UNSUPPORTED, "vp_attend4: batch * Hkv * n_new * G * max_seq is too large for one call");
    e = vp::launch_attend4(p, st);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, "vp_attend4: launch", e);
  return VP_OK;
}

}  // namespace

extern "C" {

vp_status vp_append(vp_ctx* ctx, int32_t batch, int32_t n_new, const vp_rows* q, const vp_rows* k, const vp_rows* v,
                    const int32_t* seq_len, const int32_t* new_len, const vp_rotation* rotation,
                    const vp_rows* q_out, const vp_kv* k_cache, const vp_kv* v_cache, void* cuda_stream) {
  return guarded(ctx, "vp_append", [&] {
    return append<vp_kv>(ctx, "vp_append", batch, n_new, q, k, v, seq_len, new_len, rotation, q_out, k_cache, v_cache,
                         nullptr, nullptr, cuda_stream);
  });
}

vp_status vp_append4(vp_ctx* ctx, int32_t batch, int32_t n_new, const vp_rows* q, const vp_rows* k, const vp_rows* v,
                     const int32_t* seq_len, const int32_t* new_len, const vp_rotation* rotation,
                     const vp_rows* q_out, const vp_kv4* k_cache, const vp_kv4* v_cache,
                     const vp_rows* k_held, const vp_rows* v_held, void* cuda_stream) {
  return guarded(ctx, "vp_append4", [&] {
    return append<vp_kv4>(ctx, "vp_append4", batch, n_new, q, k, v, seq_len, new_len, rotation, q_out, k_cache, v_cache,
                          k_held, v_held, cuda_stream);
  });
}

vp_status vp_reserve4(vp_ctx* ctx, int32_t max_new) {
  return guarded(ctx, "vp_reserve4", [&] { return reserve4(ctx, max_new); });
}

vp_status vp_attend4(vp_ctx* ctx, int32_t batch, int32_t n_new, const vp_rows* q,
                     const vp_kv4* k_cache, const vp_kv4* v_cache,
                     const int32_t* seq_len, const int32_t* new_len, const vp_visible* visible,
                     const vp_rows* out, float* lse, void* cuda_stream) {
  return guarded(ctx, "vp_attend4", [&] {
    return attend4(ctx, batch, n_new, q, k_cache, v_cache, seq_len, new_len, visible, out, lse, cuda_stream);
  });
}

}  // extern "C"
