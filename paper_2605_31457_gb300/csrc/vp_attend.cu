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
//   k_att_tc    (vp_attend_tc.cu) tensor-core kernel: bf16;
//   k_att_any   FFMA kernel: fp32 caches, and bf16 caches of any layout;
//   k_att_join  joins partials into out and lse, and adds the weights;
//   k_att_join_cut  joins the prompt items that k_att_tc cut between CTAs.
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

// Writes N consecutive output values of a row, rounded once to the cache type.
template <int N>
__device__ __forceinline__ void store_row(float* p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = v[i];
}
template <int N>
__device__ __forceinline__ void store_row(__nv_bfloat16* p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = __float2bfloat16_rn(v[i]);
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
#pragma unroll
  for (int i = 0; i < RPW; ++i) {
    const int row = r0 + warp * RPW + i;
    if (row >= p.R) continue;
    if (p.ns > 1 || p.weigh) {  // partials, joined by k_att_join
      const int64_t pr = ((int64_t)bg * p.ns + s) * p.R + row;
      if (lane == 0) *reinterpret_cast<float2*>(p.part_st + 2 * pr) = make_float2(m[i], l[i]);
#pragma unroll
      for (int d = 0; d < DL; ++d) p.part_o[pr * D + 32 * d + lane] = acc[i][d];
    } else {
      const int n = row / p.G, h = g * p.G + row % p.G;
      const float inv = l[i] > 0.f ? 1.f / l[i] : 0.f;
      T* o = static_cast<T*>(p.out.data) + (int64_t)b * p.out.sb + (int64_t)n * p.out.sn + (int64_t)h * p.out.sh;
#pragma unroll
      for (int d = 0; d < DL; ++d) o[32 * d + lane] = from_f<T>(acc[i][d] * inv);
      if (p.lse && lane == 0)
        p.lse[((int64_t)b * p.n_new + n) * p.H + h] = l[i] > 0.f ? (m[i] + log2f(l[i])) * kLn2 : -CUDART_INF_F;
    }
  }
}

// ---------------------------------------------------------------------------
// The partials of one query row: n records (those that are not live were never
// written).  k_att_any leaves one per split; k_att_tc, in its one-row-block
// form, one per part of the item and softmax group with tiles.
// ---------------------------------------------------------------------------
struct Partials {
  int64_t first;     // record of entry 0
  int n, stride;     // entries; records between them
  int64_t W, p0, p1; // k_att_tc: total work, the item's tiles on it
  int nc, c0;
};
__device__ __forceinline__ int part_tiles(const Partials& q, int c) {
  const int64_t a = cut(q.W, q.nc, c), z = cut(q.W, q.nc, c + 1);
  return (int)(min(z, q.p1) - max(a, q.p0));
}
__device__ __forceinline__ Partials partials_of(const AttendParams& p, int b, int g) {
  Partials q;
  q.stride = p.R;
  if (p.kind == ATT_ANY) {
    q.first = (int64_t)(b * p.Hkv + g) * p.ns * p.R;
    q.n = p.ns;
    return q;
  }
  const int total = __ldcg(p.prefix + p.B), at = __ldcg(p.prefix + b), next = __ldcg(p.prefix + b + 1);
  q.W = (int64_t)total * p.Hkv;
  q.nc = (int)min((int64_t)p.grid, q.W);
  q.p0 = (int64_t)g * total + at + kItemCost;
  q.p1 = (int64_t)g * total + next;
  q.n = 0;
  if (q.p1 > q.p0) {
    q.c0 = owner(q.W, q.nc, q.p0);
    q.n = 2 * (owner(q.W, q.nc, q.p1 - 1) - q.c0 + 1);
    q.first = (int64_t)(g * p.B + b + q.c0) * 2 * p.R;
  }
  return q;
}
__device__ __forceinline__ bool partial_live(const AttendParams& p, const Partials& q, int i) {
  return p.kind == ATT_ANY || part_tiles(q, q.c0 + (i >> 1)) > (i & 1);
}
__device__ __forceinline__ float2 partial_stat(const AttendParams& p, const Partials& q, int i, int row) {
  if (!partial_live(p, q, i)) return make_float2(-CUDART_INF_F, 0.f);
  return __ldcg(reinterpret_cast<const float2*>(p.part_st) + q.first + (int64_t)i * q.stride + row);
}

// ---------------------------------------------------------------------------
// k_att_join: 128 threads.  Blocks below B * Hkv * R join the partials of one
// query row into out and lse; the others (when weights are asked for) add the
// weights of 512 cached tokens of one (sequence, kv-head), from the stored
// logits and the rows' joined maxima and sums.
// ---------------------------------------------------------------------------
constexpr int kJoinTokens = 512;

template <typename T, int D>
__global__ void __launch_bounds__(128) k_att_join(const __grid_constant__ AttendParams p) {
  constexpr int DL = D / 32;
  __shared__ float red[4];
  __shared__ float osum[4][D];
  __shared__ float lse_s[kNewWeightRows];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  const int64_t nrows = (int64_t)p.B * p.Hkv * p.R;
  if (blockIdx.x < nrows) {
    const int row = blockIdx.x % p.R, bg = blockIdx.x / p.R, b = bg / p.Hkv, g = bg % p.Hkv;
    const NewSeq sq = load_new(p, b, false);
    const int n = row / p.G, h = g * p.G + row % p.G;
    const Partials q = partials_of(p, b, g);
    const int parts = n < sq.n ? q.n : 0;
    float m = -CUDART_INF_F;
    for (int i = tid; i < parts; i += 128) m = fmaxf(m, partial_stat(p, q, i, row).x);
    m = warp_max(m);
    if (lane == 0) red[warp] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float l = 0.f, acc[DL];
#pragma unroll
    for (int d = 0; d < DL; ++d) acc[d] = 0.f;
    for (int i = warp; i < parts; i += 4) {
      const float2 st = partial_stat(p, q, i, row);
      if (st.x == -CUDART_INF_F) continue;
      const float f = exp2f(st.x - m);
      const float* po = p.part_o + (q.first + (int64_t)i * q.stride + row) * D + lane;
      l = fmaf(st.y, f, l);
#pragma unroll
      for (int d = 0; d < DL; ++d) acc[d] = fmaf(f, __ldcg(po + 32 * d), acc[d]);
    }
    __syncthreads();
    if (lane == 0) red[warp] = l;
#pragma unroll
    for (int d = 0; d < DL; ++d) osum[warp][32 * d + lane] = acc[d];
    __syncthreads();
    l = (red[0] + red[1]) + (red[2] + red[3]);
    const float inv = l > 0.f ? 1.f / l : 0.f;
    T* o = static_cast<T*>(p.out.data) + (int64_t)b * p.out.sb + (int64_t)n * p.out.sn + (int64_t)h * p.out.sh;
    if (tid < D) o[tid] = from_f<T>(((osum[0][tid] + osum[1][tid]) + (osum[2][tid] + osum[3][tid])) * inv);
    if (p.lse && tid == 0)
      p.lse[((int64_t)b * p.n_new + n) * p.H + h] = l > 0.f ? (m + log2f(l)) * kLn2 : -CUDART_INF_F;
    return;
  }
  const int64_t wi = blockIdx.x - nrows;
  const int chunks = (p.max_seq + kJoinTokens - 1) / kJoinTokens;
  const int bg = (int)(wi / chunks), b = bg / p.Hkv, g = bg % p.Hkv, j0 = (int)(wi % chunks) * kJoinTokens;
  const NewSeq sq = load_new(p, b, false);
  if (j0 >= sq.len) return;
  const int rows = sq.n * p.G;
  const Partials q = partials_of(p, b, g);
  for (int row = warp; row < rows; row += 4) {
    float m = -CUDART_INF_F, l = 0.f;
    for (int i = lane; i < q.n; i += 32) m = fmaxf(m, partial_stat(p, q, i, row).x);
    m = warp_max(m);
    for (int i = lane; i < q.n; i += 32) {
      const float2 st = partial_stat(p, q, i, row);
      if (st.x != -CUDART_INF_F) l = fmaf(st.y, exp2f(st.x - m), l);
    }
    l = warp_sum(l);
    if (lane == 0) lse_s[row] = l > 0.f ? m + log2f(l) : CUDART_INF_F;  // log2 units
  }
  __syncthreads();
  const int t_first = sq.len - sq.n;
  const float* win = p.w_in.data ? p.w_in.data + (int64_t)b * p.w_in.sb + (int64_t)g * p.w_in.sh : nullptr;
  float* wout = p.w_out.data + (int64_t)b * p.w_out.sb + (int64_t)g * p.w_out.sh;
  for (int j = j0 + tid; j < min(sq.len, j0 + kJoinTokens); j += 128) {
    float w = 0.f;
    for (int row = 0; row < rows; ++row)
      if (sees(j, t_first + row / p.G, p.window, p.sinks))
        w += exp2f(__ldcg(p.z + ((int64_t)bg * p.R + row) * p.z_row + j) - lse_s[row]);
    wout[j] = win ? win[j] + w : w;
  }
}

// ---------------------------------------------------------------------------
// k_att_join_cut: the items of the two-group form of k_att_tc that were cut
// between CTAs.  Blocks (c, x) with the cut before CTA c the first one inside
// its item join 32 of its 256 query rows, a warp per row; the other blocks
// leave at once.
// ---------------------------------------------------------------------------
template <int D>
__global__ void __launch_bounds__(128) k_att_join_cut(const __grid_constant__ AttendParams p) {
  constexpr int DL = D / 32, kRows = 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  const int pairs = p.B * p.nqt, c = blockIdx.y + 1;
  const int total = __ldcg(p.prefix + pairs);
  const int64_t W = (int64_t)total * p.Hkv;
  const int nc = (int)min((int64_t)p.grid, W);
  if (c >= nc) return;
  const int64_t x = cut(W, nc, c);
  const int g = (int)(x / total), at = (int)(x - (int64_t)g * total);
  int lo = 0, hi = pairs;  // the pair that holds position `at`
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldcg(p.prefix + mid) <= at) lo = mid;
    else hi = mid;
  }
  const int64_t p0 = (int64_t)g * total + __ldcg(p.prefix + lo), p1 = (int64_t)g * total + __ldcg(p.prefix + lo + 1);
  if (x == p0 || cut(W, nc, c - 1) > p0) return;  // no item is cut here, or it was cut before
  const int b = lo / p.nqt, qt = lo % p.nqt, last = owner(W, nc, p1 - 1);
  const NewSeq sq = load_new(p, b, false);
  for (int r = blockIdx.x * kRows + warp; r < (blockIdx.x + 1) * kRows; r += 4) {
    const int row = qt * 2 * kTcTile + r;
    if (row >= p.R) return;
    const int n = row / p.G, h = g * p.G + row % p.G;
    // CTA c - 1 began the item (its second record); the later ones went on with it.
    auto rec = [&](int k) { return (int64_t)(k < c ? 2 * k + 1 : 2 * k) * 2 * kTcTile + r; };
    auto live = [&](int k) {
      return min(cut(W, nc, k + 1), p1) > max(cut(W, nc, k), p0 + kItemCost);
    };
    float m = -CUDART_INF_F, l = 0.f, acc[DL];
#pragma unroll
    for (int d = 0; d < DL; ++d) acc[d] = 0.f;
    if (n < sq.n) {
      for (int k = c - 1; k <= last; ++k)
        if (live(k)) m = fmaxf(m, __ldcg(p.part_st + 2 * rec(k)));
      for (int k = c - 1; k <= last; ++k) {
        if (!live(k)) continue;
        const float2 st = __ldcg(reinterpret_cast<const float2*>(p.part_st) + rec(k));
        if (st.x == -CUDART_INF_F) continue;
        const float f = exp2f(st.x - m);
        const float* po = p.part_o + rec(k) * D + lane;
        l = fmaf(st.y, f, l);
#pragma unroll
        for (int d = 0; d < DL; ++d) acc[d] = fmaf(f, __ldcg(po + 32 * d), acc[d]);
      }
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    __nv_bfloat16* o = static_cast<__nv_bfloat16*>(p.out.data) + (int64_t)b * p.out.sb + (int64_t)n * p.out.sn +
                       (int64_t)h * p.out.sh;
#pragma unroll
    for (int d = 0; d < DL; ++d) o[32 * d + lane] = __float2bfloat16_rn(acc[d] * inv);
    if (p.lse && lane == 0)
      p.lse[((int64_t)b * p.n_new + n) * p.H + h] = l > 0.f ? (m + log2f(l)) * kLn2 : -CUDART_INF_F;
  }
}

template <typename T, int D>
cudaError_t launch_join(const AttendParams& p, cudaStream_t st) {
  const int64_t chunks = p.weigh ? (p.max_seq + kJoinTokens - 1) / kJoinTokens : 0;
  const int64_t joins = (int64_t)p.B * p.Hkv * (p.R + chunks);
  if (joins > INT32_MAX) return cudaErrorInvalidConfiguration;
  return launch_dep(k_att_join<T, D>, dim3((unsigned)joins), 128, 0, st, p);
}

template <int D>
cudaError_t launch_tensor(const AttendParams& p, cudaStream_t st) {
  const cudaError_t e = launch_tc(p, st);
  if (e != cudaSuccess) return e;
  if (p.kind == ATT_TC1) return launch_join<__nv_bfloat16, D>(p, st);
  return p.grid > 1 ? launch_dep(k_att_join_cut<D>, dim3(2 * kTcTile / 32, p.grid - 1), 128, 0, st, p) : cudaSuccess;
}

template <typename T, int D>
cudaError_t launch_any(const AttendParams& p, cudaStream_t st) {
  const int rb = any_rows(p.R);
  const int64_t ctas = (int64_t)p.B * p.Hkv * ((p.R + rb - 1) / rb) * p.ns;
  if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)ctas);
  cudaError_t e;
  if (rb == 4) e = launch_dep(k_att_any<T, D, 1>, grid, 128, sizeof(AnySmem<D, 1>), st, p);
  else if (rb == 8) e = launch_dep(k_att_any<T, D, 2>, grid, 128, sizeof(AnySmem<D, 2>), st, p);
  else e = launch_dep(k_att_any<T, D, 4>, grid, 128, sizeof(AnySmem<D, 4>), st, p);
  if (e != cudaSuccess || (p.ns == 1 && !p.weigh)) return e;
  return launch_join<T, D>(p, st);
}

}  // namespace

cudaError_t configure_attend() { return configure_tc(); }

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
  p.kind = p.R <= kTcTile ? ATT_TC1 : ATT_TC2;
  p.nqt = p.kind == ATT_TC1 ? 1 : (p.R + 2 * kTcTile - 1) / (2 * kTcTile);
  p.grid = p.num_sms;
  p.stream_once = p.kind == ATT_TC1;
}

cudaError_t launch_attend(const AttendParams& p, cudaStream_t st) {
  if (p.kind != ATT_ANY) return p.D == 128 ? launch_tensor<128>(p, st) : launch_tensor<64>(p, st);
  if (p.dtype == 0)
    return p.D == 128 ? launch_any<__nv_bfloat16, 128>(p, st) : launch_any<__nv_bfloat16, 64>(p, st);
  return p.D == 128 ? launch_any<float, 128>(p, st) : launch_any<float, 64>(p, st);
}

}  // namespace vp
