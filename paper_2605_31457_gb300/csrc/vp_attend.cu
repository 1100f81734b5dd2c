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

#include <type_traits>

#include "vp_attend.h"
#include "vp_attend_device.h"
#include "vp_device.h"

namespace vp {
namespace {

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  float4 f;
  bf2(u.x, f.x, f.y);
  bf2(u.y, f.z, f.w);
  return f;
}
// N (2 or 4) elements in 32 bits.
template <int N, typename T>
__device__ __forceinline__ void load_n(const T* p, float* x) {
  if constexpr (N == 4) {
    const float4 f = load4(p);
    x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
  } else if constexpr (sizeof(T) == 4) {
    const float2 f = *reinterpret_cast<const float2*>(p);
    x[0] = f.x; x[1] = f.y;
  } else {
    bf2(*reinterpret_cast<const uint32_t*>(p), x[0], x[1]);
  }
}
// 16 bytes to shared memory, or 16 zero bytes.
__device__ __forceinline__ void copy16(void* dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(live ? 16 : 0)
               : "memory");
}

// ---------------------------------------------------------------------------
// k_att_any: one CTA of 128 threads per (sequence, kv-head, block of RB = 4 RG
// query rows, split), over its share of the tiles of 32 tokens that those rows
// see.  K and V rows (any layout; a row that no query of the CTA sees, or that
// lies on no page of the pool, as zeros) are copied to shared memory
// asynchronously, up to `stages - 1` tiles ahead.  Per tile:
//   S    a lane holds 4 rows x RG tokens of S and a warp a quarter of the head's
//        dimensions, so that 16 RG products come from 4 + RG 16-byte reads;
//   P    the warps take RG rows each, a token per lane: the four parts of a
//        logit are added, the row's maximum is a warp reduction, its sum stays a
//        part per lane;
//   P.V  a warp takes 8 tokens, a lane 4 rows x D RG / 32 dimensions.  The four
//        warps' sums meet once, at the end.
// Row r of the block is lane group r % RG's, its slot in P and in the state is
// 4 (r % RG) + r / RG.  Serves fp32 caches (which must not be rounded to a
// tensor-core type) and layouts that a tensor map cannot describe.
// Up to 8 rows it is bound by the cache's bytes, above by the FMA pipes and the
// latency of two warps per scheduler.  fp32, D = 128: 64 sequences of 1500 to
// 5000 tokens, 32/8 heads, with weights 325 us (5.3 TB/s); 8 sequences of 5000
// to 12000 tokens, one kv-head, 64 query rows 135 us (16 TFLOP/s); a prompt of
// 3857 tokens, 28/4 heads, 4.26 ms (25 TFLOP/s).  The form before it, a
// token per lane with all of K's row and loads between barriers, took 1076 and
// 210 us.
// ---------------------------------------------------------------------------
template <typename T, int D, int RG>
struct AnySmem {
  static constexpr int RB = 4 * RG, kStages = D == 128 ? 2 : 4;
  // Four row groups write to different banks; with two, three CTAs still fit an SM.
  static constexpr int kZPitch = RG == 4 ? 34 : RG == 2 ? 33 : 32;
  static constexpr int kPitch = D + 16 / (int)sizeof(T);  // a K row per lane: all on different banks
  struct Stage {
    T k[kAnyTile][kPitch];
    T v[kAnyTile][D];
  };
  Stage st[kStages];
  float q[RB][D + 4];
  float z[4][RB][kZPitch];
  float p[kAnyTile][RB == 4 ? 4 : RB + 4];
  float f[RB], m[RB], l[RB];
  unsigned char ok[kStages][kAnyTile];
  int flag;
  // The warps' outputs, where the tiles were.
  __device__ float* sum() { return reinterpret_cast<float*>(st); }
  static_assert(sizeof(Stage) * kStages >= 4 * RB * D * sizeof(float), "the sums overlay the tiles");
};

template <typename T, int D, int RG>
__global__ void __launch_bounds__(128) k_att_any(const __grid_constant__ AttendParams p) {
  using Smem = AnySmem<T, D, RG>;
  constexpr int RB = Smem::RB, NS = Smem::kStages, C4 = D / 4;
  constexpr int TL = 32 / RG;                 // lanes of a row group: over tokens (S), over dimensions (P.V)
  constexpr int DT = D / TL, VW = DT < 4 ? DT : 4;
  constexpr int CH = D * (int)sizeof(T) / 16; // 16-byte pieces of a cache row
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rg = lane / TL, ln = lane % TL;
  const int blocks = (p.R + RB - 1) / RB;
  const int s = blockIdx.x % p.ns, rb = blockIdx.x / p.ns % blocks, bg = blockIdx.x / p.ns / blocks;
  const int r0 = rb * RB, b = bg / p.Hkv, g = bg % p.Hkv;
  pdl_wait();
  pdl_trigger();
  const NewSeq sq = load_new(p, b, s == 0 && rb == 0 && g == 0);
  const int t_first = sq.len - sq.n;                    // position of new token 0
  const int r1 = min(min(p.R, sq.n * p.G), r0 + RB);    // end of the block's live query rows
  SeenRange sr{0, 0, 0};
  if (r0 < r1) sr = seen_range(t_first + row_token(p, r0), t_first + row_token(p, r1 - 1), p.window, p.sinks);
  const TileList tl = tile_list(sr, kAnyTile);
  const int per = (tl.n + p.ns - 1) / p.ns;
  const int u0 = min(tl.n, s * per), u1 = min(tl.n, u0 + per);

  // Lane i copies for row 8 * warp + i % 8 of a tile; its pages are looked up a
  // tile before they are needed.
  const int cr = 8 * warp + (lane & 7);
  int page_k = 0, page_v = 0;
  auto look_up = [&](int u) {
    if (!p.paged || u >= u1) return;
    const int lp = (tl.tile(u) * kAnyTile + cr) >> p.page_shift;
    page_k = lp < p.k.max_pages ? __ldg(p.k.block_table + (int64_t)b * p.k.max_pages + lp) : -1;
    page_v = lp < p.v.max_pages ? __ldg(p.v.block_table + (int64_t)b * p.v.max_pages + lp) : -1;
  };
  unsigned err = 0;
  auto copy_tile = [&](int u) {
    if (u < u1) {
      const int j = tl.tile(u) * kAnyTile + cr, stage = (u - u0) % NS;
      const bool need = j < sr.s_end || (j >= sr.lo && j < sr.hi);
      const bool ok = need && (!p.paged || (page_k >= 0 && page_k < p.k.num_pages && page_v >= 0 && page_v < p.v.num_pages));
      if (need && !ok) err |= ERR_PAGE;
      const int64_t jj = p.paged ? j & ((1 << p.page_shift) - 1) : j;
      const T* kr = static_cast<const T*>(p.k.data);
      const T* vr = static_cast<const T*>(p.v.data);
      if (ok) {
        kr += (p.paged ? page_k : b) * p.k.sb + g * p.k.sh + jj * p.k.st;
        vr += (p.paged ? page_v : b) * p.v.sb + g * p.v.sh + jj * p.v.st;
      }
      if (lane < 8) sm.ok[stage][cr] = ok;
#pragma unroll
      for (int i = 0; i < 8; i += 32 / CH) {
        const int r = i + lane / CH, c = lane % CH * (16 / (int)sizeof(T));
        const T* ks = reinterpret_cast<const T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(kr), r));
        const T* vs = reinterpret_cast<const T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(vr), r));
        const bool live = __shfl_sync(0xffffffffu, (int)ok, r);
        copy16(&sm.st[stage].k[8 * warp + r][c], ks + c, live);
        copy16(&sm.st[stage].v[8 * warp + r][c], vs + c, live);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    look_up(u + 1);
  };
  look_up(u0);
#pragma unroll
  for (int i = 0; i < NS - 1; ++i) copy_tile(u0 + i);

  for (int i = tid; i < RB * C4; i += 128) {
    const int r = i / C4, c = i % C4, row = r0 + r;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row < r1) {
      const int tok = row_token(p, row);
      x = load4(static_cast<const T*>(p.q.data) + (int64_t)b * p.q.sb + (int64_t)tok * p.q.sn +
                (int64_t)(g * p.G + row - tok * p.G) * p.q.sh + 4 * c);
    }
    *reinterpret_cast<float4*>(&sm.q[r][4 * c]) = x;
  }
  // Softmax state of this warp's RG slots; l is this lane's part of the sum.
  float m[RG], l[RG];
  int t[RG], zr[RG];  // position of the row's token (-1: no row); the row
#pragma unroll
  for (int k = 0; k < RG; ++k) {
    const int slot = warp * RG + k, row = r0 + slot / 4 + RG * (slot % 4);
    m[k] = -CUDART_INF_F;
    l[k] = 0.f;
    t[k] = row < r1 ? t_first + row_token(p, row) : -1;
    zr[k] = row;
  }
  float acc[4][DT];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[i][d] = 0.f;

  for (int u = u0; u < u1; ++u) {
    const int stage = (u - u0) % NS;
    asm volatile("cp.async.wait_group %0;" ::"n"(NS - 2) : "memory");
    __syncthreads();  // tile u is there, tile u - 1 is done with
    copy_tile(u + NS - 1);
    {
      float z[4][RG];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < RG; ++k) z[i][k] = 0.f;
#pragma unroll 4
      for (int c = warp * (C4 / 4); c < (warp + 1) * (C4 / 4); ++c) {
        float4 kx[RG];
#pragma unroll
        for (int k = 0; k < RG; ++k) kx[k] = load4(&sm.st[stage].k[ln + TL * k][4 * c]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 qx = load4(&sm.q[rg + RG * i][4 * c]);
#pragma unroll
          for (int k = 0; k < RG; ++k) {
            z[i][k] = fmaf(qx.x, kx[k].x, z[i][k]);
            z[i][k] = fmaf(qx.y, kx[k].y, z[i][k]);
            z[i][k] = fmaf(qx.z, kx[k].z, z[i][k]);
            z[i][k] = fmaf(qx.w, kx[k].w, z[i][k]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < RG; ++k) sm.z[warp][4 * rg + i][ln + TL * k] = z[i][k];
    }
    __syncthreads();
    {
      const int j = tl.tile(u) * kAnyTile + lane;
      const bool ok = sm.ok[stage][lane];
      float pe[RG], mx[RG];
#pragma unroll
      for (int k = 0; k < RG; ++k) {
        const int slot = warp * RG + k;
        const float z = (sm.z[0][slot][lane] + sm.z[1][slot][lane]) + (sm.z[2][slot][lane] + sm.z[3][slot][lane]);
        pe[k] = ok && sees(j, t[k], p.window, p.sinks) ? z * p.c_log2 : -CUDART_INF_F;
        if (p.weigh && t[k] >= 0 && j < p.z_row) p.z[((int64_t)bg * p.R + zr[k]) * p.z_row + j] = pe[k];
        mx[k] = fmaxf(m[k], warp_max(pe[k]));
      }
#pragma unroll
      for (int k = 0; k < RG; ++k) {
        const float mu = mx[k] == -CUDART_INF_F ? 0.f : mx[k];
        const float f = exp2f(m[k] - mu);
        pe[k] = exp2f(pe[k] - mu);
        l[k] = fmaf(l[k], f, pe[k]);
        m[k] = mx[k];
        sm.p[lane][warp * RG + k] = pe[k];
        if (lane == 0) sm.f[warp * RG + k] = f;
      }
    }
    __syncthreads();
    const float4 f = load4(&sm.f[4 * rg]);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      acc[0][d] *= f.x;
      acc[1][d] *= f.y;
      acc[2][d] *= f.z;
      acc[3][d] *= f.w;
    }
#pragma unroll 4
    for (int jj = 8 * warp; jj < 8 * warp + 8; ++jj) {
      const float4 pe = load4(&sm.p[jj][4 * rg]);
#pragma unroll
      for (int d = 0; d < DT; d += VW) {
        float vx[VW];
        load_n<VW>(&sm.st[stage].v[jj][VW * (ln + TL * (d / VW))], vx);
#pragma unroll
        for (int e = 0; e < VW; ++e) {
          acc[0][d + e] = fmaf(pe.x, vx[e], acc[0][d + e]);
          acc[1][d + e] = fmaf(pe.y, vx[e], acc[1][d + e]);
          acc[2][d + e] = fmaf(pe.z, vx[e], acc[2][d + e]);
          acc[3][d + e] = fmaf(pe.w, vx[e], acc[3][d + e]);
        }
      }
    }
  }
  if (err) atomicOr(p.err, err);

  __syncthreads();  // the tiles are done with; no copy is in flight
  float* sum = sm.sum();
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int d = 0; d < DT; ++d)
      sum[(warp * RB + rg + RG * i) * D + VW * (ln + TL * (d / VW)) + d % VW] = acc[i][d];
#pragma unroll
  for (int k = 0; k < RG; ++k) {
    const float all = warp_sum(l[k]);
    if (lane == 0) {
      sm.m[zr[k] - r0] = m[k];
      sm.l[zr[k] - r0] = all;
    }
  }
  __syncthreads();
  const int unit = bg * blocks + rb;
  const int64_t rec = ((int64_t)unit * p.ns + s) * RB;
  for (int i = tid; i < RB * C4; i += 128) {
    const int r = i / C4, d = 4 * (i % C4);
    float4 o = load4(sum + r * D + d);
#pragma unroll
    for (int w = 1; w < 4; ++w) {
      const float4 x = load4(sum + (w * RB + r) * D + d);
      o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
    }
    if (p.ns > 1) {
      *reinterpret_cast<float4*>(p.part_o + (rec + r) * D + d) = o;
      if (d == 0) *reinterpret_cast<float2*>(p.part_st + 2 * (rec + r)) = make_float2(sm.m[r], sm.l[r]);
    } else if (r0 + r < p.R) {
      const float inv = sm.l[r] > 0.f ? 1.f / sm.l[r] : 0.f;
      store4(out_row<T>(p, b, g, r0 + r) + d, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
      if (d == 0) store_lse(p, b, g, r0 + r, sm.m[r], sm.l[r]);
    }
  }
  if (p.ns > 1 && last_to_arrive(p.tickets + unit, p.ns, tid, &sm.flag, [] { __syncthreads(); }))
    join_records<T, D, 128, 1, 16>(p, b, g, r0, min(RB, p.R - r0), p.ns, RB, [&](int k) { return unit * p.ns + k; }, tid);
}

// ---------------------------------------------------------------------------
// k_att_weights: weight_out = weight_in + sum over the query rows of
// exp2(z - lse), from the logits that the attention kernel stored; a thread per
// four cached tokens of one (sequence, kv-head).  Bound by reading the logits
// (4 R bytes per token and kv-head, from L2 where they fit): 9.5 us for 8 sequences
// of 20480 tokens and 7 rows (18 MB).
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

// f(kernel, shared bytes) for the instance of a type, dimension and block.
template <typename F>
cudaError_t with_any(int dtype, int D, int rows, F&& f) {
  auto typed = [&](auto zero, auto dim) {
    using T = decltype(zero);
    constexpr int N = decltype(dim)::value;
    if (rows == 4) return f(k_att_any<T, N, 1>, sizeof(AnySmem<T, N, 1>));
    if (rows == 8) return f(k_att_any<T, N, 2>, sizeof(AnySmem<T, N, 2>));
    return f(k_att_any<T, N, 4>, sizeof(AnySmem<T, N, 4>));
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (dtype == 0) return D == 128 ? typed(__nv_bfloat16(), D128()) : typed(__nv_bfloat16(), D64());
  return D == 128 ? typed(0.f, D128()) : typed(0.f, D64());
}

}  // namespace

cudaError_t configure_attend() {
  cudaError_t e = configure_dec();
  if (e == cudaSuccess) e = configure_tc();
  for (int dtype : {0, 1})
    for (int D : {64, 128})
      for (int rows : {4, 8, 16})
        if (e == cudaSuccess)
          e = with_any(dtype, D, rows, [](auto kernel, size_t smem) {
            return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
          });
  return e;
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
  else {
    const int rb = any_rows(p.R);
    const int64_t ctas = (int64_t)p.B * p.Hkv * ((p.R + rb - 1) / rb) * p.ns;
    if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
    e = with_any(p.dtype, p.D, rb, [&](auto kernel, size_t smem) {
      return launch_dep(kernel, dim3((unsigned)ctas), 128, smem, st, p);
    });
  }
  if (e != cudaSuccess || !p.weigh) return e;
  const int64_t ctas = (int64_t)p.B * p.Hkv * ((p.max_seq + kWeightTokens - 1) / kWeightTokens);
  if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
  return launch_dep(k_att_weights, dim3((unsigned)ctas), kWeightThreads, 0, st, p);
}

}  // namespace vp
