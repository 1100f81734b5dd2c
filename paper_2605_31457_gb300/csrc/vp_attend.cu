// Attention of newly appended tokens over a cache (vp_attend_new): causal, with
// an optional sliding window and sink tokens, for a decode step, a few drafted
// tokens or a prompt.
//
// For new token i of sequence b at position t_i and query head h of kv-head g,
// over the tokens j that t_i sees (V_i: j <= t_i and j > t_i - window or
// j < sinks):
//   z_j = scale <q_ih, k_gj>,  lse = log sum_j exp z_j,  out = sum_j exp(z_j - lse) v_gj,
//   weight_g[j] += sum_{i, h of g} exp(z_j - lse).
// One pass over the cache: a running maximum m, l = sum exp(z - m) and
// o = sum exp(z - m) v, rescaled when m rises; partials (m, l, o) over disjoint
// parts of V_i join as m = max m_p, l = sum l_p e^(m_p - m), o likewise.
// Logits are carried in log2 units (one exp2 each).
//
//   k_att_dec   (vp_attend_dec.cu) bf16, up to 64 query rows per kv-head;
//   k_att_tc    (vp_attend_tc.cu) bf16, more rows;
//   k_att_any   fp32 caches, and bf16 caches of any layout;
//   k_att_weights  the accumulated weights, from the logits the others stored.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include "vp_attend.h"
#include "vp_attend_device.h"
#include "vp_device.h"

namespace vp {
namespace {

// Row of (sequence b, kv-head g, token j); NULL where the block table maps it
// to no page of the pool.
template <typename T>
__device__ __forceinline__ const T* cache_row(const KvView& kv, int paged, int page_shift, int b, int g, int j) {
  const T* base = static_cast<const T*>(kv.data);
  if (!paged) return base + (int64_t)b * kv.sb + (int64_t)g * kv.sh + (int64_t)j * kv.st;
  const int lp = j >> page_shift;
  if (lp >= kv.max_pages) return nullptr;
  const int page = __ldg(kv.block_table + (int64_t)b * kv.max_pages + lp);
  if (page < 0 || page >= kv.num_pages) return nullptr;
  return base + (int64_t)page * kv.sb + (int64_t)g * kv.sh + (int64_t)(j & ((1 << page_shift) - 1)) * kv.st;
}

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  float4 f;
  bf2(u.x, f.x, f.y);
  bf2(u.y, f.z, f.w);
  return f;
}

// ---------------------------------------------------------------------------
// k_att_any: one CTA of 128 threads per (sequence, kv-head, row block, split).  A CTA takes
// 4 * RPW query rows over its share of the tiles of 32 tokens that those rows
// see.  Per tile: K and V rows (any layout; a row that no query of the CTA
// sees is taken as zeros) go to shared memory in 32 bits; a thread forms the
// logits of one token (its lane) and the RPW rows of its warp; the softmax of
// a row is a warp reduction; for P.V a lane holds D / 32 dimensions.  Bound by
// the FMA pipes and shared-memory reads, which suits its use: fp32 caches
// (which must not be rounded to a tensor-core type) and layouts that a tensor
// map cannot describe.
// ---------------------------------------------------------------------------
template <int D, int RPW>
struct AnySmem {
  float q[4 * RPW][D];
  float k[kAnyTile][D + 4];  // padded: lanes read one row each, 16 bytes at a time
  float v[kAnyTile][D];
  float z[4 * RPW][kAnyTile];
};

template <typename T, int D, int RPW>
__global__ void __launch_bounds__(128) k_att_any(const __grid_constant__ AttendParams p) {
  constexpr int RB = 4 * RPW, C4 = D / 4, DL = D / 32;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  AnySmem<D, RPW>& sm = *reinterpret_cast<AnySmem<D, RPW>*>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int blocks = (p.R + RB - 1) / RB;
  const int s = blockIdx.x % p.ns, rb = blockIdx.x / p.ns % blocks, bg = blockIdx.x / p.ns / blocks;
  const int r0 = rb * RB, b = bg / p.Hkv, g = bg % p.Hkv;
  pdl_wait();
  pdl_trigger();
  const NewSeq sq = load_new(p, b, s == 0 && rb == 0 && g == 0);
  const int t_first = sq.len - sq.n;                    // position of new token 0
  const int rows = min(p.R, sq.n * p.G);                // live query rows of the sequence
  const int r1 = min(rows, r0 + RB);
  SeenRange sr{0, 0, 0};
  if (r0 < r1) sr = seen_range(t_first + r0 / p.G, t_first + (r1 - 1) / p.G, p.window, p.sinks);
  const TileList tl = tile_list(sr, kAnyTile);
  const int per = (tl.n + p.ns - 1) / p.ns;
  const int u0 = min(tl.n, s * per), u1 = min(tl.n, u0 + per);

  for (int i = tid; i < RB * C4; i += 128) {
    const int r = i / C4, c = i % C4, row = r0 + r;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row < r1)
      x = load4(static_cast<const T*>(p.q.data) + (int64_t)b * p.q.sb + (int64_t)(row / p.G) * p.q.sn +
                (int64_t)(g * p.G + row % p.G) * p.q.sh + 4 * c);
    *reinterpret_cast<float4*>(&sm.q[r][4 * c]) = x;
  }
  float m[RPW], l[RPW], acc[RPW][DL];
  int t[RPW];  // position of the row's token; -1: no row
#pragma unroll
  for (int i = 0; i < RPW; ++i) {
    const int row = r0 + warp * RPW + i;
    m[i] = -CUDART_INF_F;
    l[i] = 0.f;
    t[i] = row < r1 ? t_first + row / p.G : -1;
#pragma unroll
    for (int d = 0; d < DL; ++d) acc[i][d] = 0.f;
  }
  unsigned err = 0;
  for (int u = u0; u < u1; ++u) {
    const int j0 = tl.tile(u) * kAnyTile;
    __syncthreads();
    bool bad = false;
    for (int i = tid; i < kAnyTile * C4; i += 128) {
      const int r = i / C4, c = i % C4, j = j0 + r;
      float4 kx = make_float4(0.f, 0.f, 0.f, 0.f), vx = kx;
      if (j < sr.s_end || (j >= sr.lo && j < sr.hi)) {
        const T* kr = cache_row<T>(p.k, p.paged, p.page_shift, b, g, j);
        const T* vr = cache_row<T>(p.v, p.paged, p.page_shift, b, g, j);
        if (kr && vr) {
          kx = load4(kr + 4 * c);
          vx = load4(vr + 4 * c);
        } else {
          bad = true;
        }
      }
      *reinterpret_cast<float4*>(&sm.k[r][4 * c]) = kx;
      *reinterpret_cast<float4*>(&sm.v[r][4 * c]) = vx;
    }
    if (bad) err |= ERR_PAGE;
    __syncthreads();
    const int j = j0 + lane;
    bool mapped = true;  // only a page of the pool is part of the attention
    if (p.paged && (j < sr.s_end || (j >= sr.lo && j < sr.hi)))
      mapped = cache_row<T>(p.k, 1, p.page_shift, b, g, j) && cache_row<T>(p.v, 1, p.page_shift, b, g, j);
    float z[RPW];
#pragma unroll
    for (int i = 0; i < RPW; ++i) z[i] = 0.f;
#pragma unroll 8
    for (int c = 0; c < C4; ++c) {
      const float4 kx = *reinterpret_cast<const float4*>(&sm.k[lane][4 * c]);
#pragma unroll
      for (int i = 0; i < RPW; ++i) {
        const float4 qx = *reinterpret_cast<const float4*>(&sm.q[warp * RPW + i][4 * c]);
        z[i] = fmaf(qx.x, kx.x, z[i]);
        z[i] = fmaf(qx.y, kx.y, z[i]);
        z[i] = fmaf(qx.z, kx.z, z[i]);
        z[i] = fmaf(qx.w, kx.w, z[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < RPW; ++i) {
      const bool see = mapped && sees(j, t[i], p.window, p.sinks);
      z[i] = see ? z[i] * p.c_log2 : -CUDART_INF_F;
      if (p.weigh && t[i] >= 0 && j < p.z_row)
        p.z[((int64_t)bg * p.R + r0 + warp * RPW + i) * p.z_row + j] = z[i];
      const float mn = fmaxf(m[i], warp_max(z[i]));
      const float mu = mn == -CUDART_INF_F ? 0.f : mn;
      const float pe = exp2f(z[i] - mu), f = exp2f(m[i] - mu);
      l[i] = fmaf(l[i], f, warp_sum(pe));
#pragma unroll
      for (int d = 0; d < DL; ++d) acc[i][d] *= f;
      m[i] = mn;
      sm.z[warp * RPW + i][lane] = pe;
    }
    __syncwarp();
#pragma unroll 4
    for (int jj = 0; jj < kAnyTile; ++jj) {
      float vx[DL];
#pragma unroll
      for (int d = 0; d < DL; ++d) vx[d] = sm.v[jj][32 * d + lane];
#pragma unroll
      for (int i = 0; i < RPW; ++i) {
        const float pe = sm.z[warp * RPW + i][jj];
#pragma unroll
        for (int d = 0; d < DL; ++d) acc[i][d] = fmaf(pe, vx[d], acc[i][d]);
      }
    }
  }
  if (err) atomicOr(p.err, err);
  if (p.ns == 1) {
#pragma unroll
    for (int i = 0; i < RPW; ++i) {
      const int row = r0 + warp * RPW + i;
      if (row >= p.R) continue;
      const float inv = l[i] > 0.f ? 1.f / l[i] : 0.f;
      T* o = out_row<T>(p, b, g, row);
#pragma unroll
      for (int d = 0; d < DL; ++d) o[32 * d + lane] = from_f<T>(acc[i][d] * inv);
      if (lane == 0) store_lse(p, b, g, row, m[i], l[i]);
    }
    return;
  }
  const int unit = bg * blocks + rb;
#pragma unroll
  for (int i = 0; i < RPW; ++i) {
    const int64_t at = ((int64_t)unit * p.ns + s) * RB + warp * RPW + i;
    if (lane == 0) *reinterpret_cast<float2*>(p.part_st + 2 * at) = make_float2(m[i], l[i]);
#pragma unroll
    for (int d = 0; d < DL; ++d) p.part_o[at * D + 32 * d + lane] = acc[i][d];
  }
  __shared__ int flag;
  if (last_to_arrive(p.tickets + unit, p.ns, tid, &flag, [] { __syncthreads(); }))
    join_records<T, D, 128>(p, b, g, r0, min(RB, p.R - r0), p.ns, RB, [&](int k) { return unit * p.ns + k; }, tid);
}

// ---------------------------------------------------------------------------
// k_att_weights: weight_out = weight_in + sum over the query rows of
// exp2(z - lse), from the logits that the attention kernel stored; a thread per
// four cached tokens of one (sequence, kv-head).  Bound by reading the logits
// (4 R bytes per token and kv-head, from L2 where they fit).
// ---------------------------------------------------------------------------
constexpr int kWeightThreads = 128, kWeightTokens = 4 * kWeightThreads;

__global__ void __launch_bounds__(kWeightThreads) k_att_weights(const __grid_constant__ AttendParams p) {
  __shared__ float lse_s[kNewWeightRows];
  const int tid = threadIdx.x;
  pdl_wait();
  const int chunks = (p.max_seq + kWeightTokens - 1) / kWeightTokens;
  const int bg = blockIdx.x / chunks, b = bg / p.Hkv, g = bg % p.Hkv;
  const NewSeq sq = load_new(p, b, false);
  const int rows = sq.n * p.G, t_first = sq.len - sq.n;
  const int j = (blockIdx.x % chunks) * kWeightTokens + 4 * tid;
  if (tid < rows) lse_s[tid] = __ldcg(p.lse2 + (int64_t)bg * p.R + tid);
  __syncthreads();
  if (j >= sq.len) return;
  float w[4] = {0.f, 0.f, 0.f, 0.f};
  const float* z = p.z + (int64_t)bg * p.R * p.z_row + j;
  for (int n = 0; n < sq.n; ++n) {
    const int t = t_first + n;
    bool see[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) see[k] = sees(j + k, t, p.window, p.sinks);
    if (!(see[0] || see[1] || see[2] || see[3])) continue;
#pragma unroll 4
    for (int row = n * p.G; row < (n + 1) * p.G; ++row) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(z + (int64_t)row * p.z_row));
      const float s = lse_s[row];
      if (see[0]) w[0] += exp2f(x.x - s);
      if (see[1]) w[1] += exp2f(x.y - s);
      if (see[2]) w[2] += exp2f(x.z - s);
      if (see[3]) w[3] += exp2f(x.w - s);
    }
  }
  const float* win = p.w_in.data ? p.w_in.data + (int64_t)b * p.w_in.sb + (int64_t)g * p.w_in.sh : nullptr;
  float* wout = p.w_out.data + (int64_t)b * p.w_out.sb + (int64_t)g * p.w_out.sh;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (j + k < sq.len) wout[j + k] = win ? win[j + k] + w[k] : w[k];
}

template <typename T, int D>
cudaError_t launch_any(const AttendParams& p, cudaStream_t st) {
  const int rb = any_rows(p.R);
  const int64_t ctas = (int64_t)p.B * p.Hkv * ((p.R + rb - 1) / rb) * p.ns;
  if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)ctas);
  if (rb == 4) return launch_dep(k_att_any<T, D, 1>, grid, 128, sizeof(AnySmem<D, 1>), st, p);
  if (rb == 8) return launch_dep(k_att_any<T, D, 2>, grid, 128, sizeof(AnySmem<D, 2>), st, p);
  return launch_dep(k_att_any<T, D, 4>, grid, 128, sizeof(AnySmem<D, 4>), st, p);
}

}  // namespace

cudaError_t configure_attend() {
  const cudaError_t e = configure_dec();
  return e == cudaSuccess ? configure_tc() : e;
}

void plan_attend(AttendParams& p) {
  p.kind = ATT_ANY;
  p.ns = any_splits(p.B, p.Hkv, p.R, any_rows(p.R), p.n_new, p.window, p.sinks, p.max_seq, p.num_sms);
  // The tensor cores read bf16, and boxes of fewer than 8 rows would split the
  // swizzle's 1024-byte atoms.
  if (p.dtype != 0 || (p.paged && p.page_size < 8)) return;
  const KvShape shape{p.D, p.Hkv, p.B, p.paged, p.page_size, p.max_seq};
  const int rows = p.paged && p.page_size < kTcTile ? p.page_size : kTcTile;
  int vt = 0, vg = 0, vb = 0;
  if (!encode_kv_map(p.k, shape, &p.tmk, &p.tpos, &p.gpos, &p.bpos, rows) ||
      !encode_kv_map(p.v, shape, &p.tmv, &vt, &vg, &vb, rows) || vt != p.tpos || vg != p.gpos || vb != p.bpos)
    return;
  p.kind = p.R <= kDecRows ? ATT_DEC : p.R <= kTcTile ? ATT_TC1 : ATT_TC2;
  p.block = p.kind == ATT_TC2 ? 2 * kTcTile : p.R;
  p.nqt = (p.R + p.block - 1) / p.block;
  p.fixed = (p.kind == ATT_DEC ? 1 : 2) * kTileUnits;
  if (line_bound((int64_t)p.B * p.Hkv * p.nqt, p.max_seq, p.fixed) > INT32_MAX) {
    p.kind = ATT_ANY;
    return;
  }
  p.grid = p.kind == ATT_DEC && p.R <= 16 ? 2 * p.num_sms : p.num_sms;  // CTAs per SM
}

cudaError_t launch_attend(const AttendParams& p, cudaStream_t st) {
  cudaError_t e;
  if (p.kind == ATT_DEC) e = launch_dec(p, st);
  else if (p.kind != ATT_ANY) e = launch_tc(p, st);
  else if (p.dtype == 0) e = p.D == 128 ? launch_any<__nv_bfloat16, 128>(p, st) : launch_any<__nv_bfloat16, 64>(p, st);
  else e = p.D == 128 ? launch_any<float, 128>(p, st) : launch_any<float, 64>(p, st);
  if (e != cudaSuccess || !p.weigh) return e;
  const int64_t ctas = (int64_t)p.B * p.Hkv * ((p.max_seq + kWeightTokens - 1) / kWeightTokens);
  if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
  return launch_dep(k_att_weights, dim3((unsigned)ctas), kWeightThreads, 0, st, p);
}

}  // namespace vp
