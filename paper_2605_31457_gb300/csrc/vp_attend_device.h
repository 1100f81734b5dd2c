// Device and launch helpers shared by the kernels of vp_attend_new.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include "vp_attend.h"
#include "vp_device.h"

namespace vp {

constexpr float kLn2 = 0.6931471805599453f;

// Live tokens of a sequence and how many of them are new.
struct NewSeq {
  int len, n;
};
__device__ __forceinline__ NewSeq load_new(const AttendParams& p, int b, bool report) {
  NewSeq s;
  s.len = __ldcg(p.seq_len + b);
  unsigned e = 0;
  if (s.len < 0 || s.len > p.max_seq) { e |= ERR_LEN; s.len = min(max(s.len, 0), p.max_seq); }
  s.n = p.new_len ? __ldcg(p.new_len + b) : (s.len > 0 ? p.n_new : 0);
  const int most = min(p.n_new, s.len);
  if (s.n < 0 || s.n > most) { e |= ERR_NEW; s.n = min(max(s.n, 0), most); }
  if (e && report) atomicOr(p.err, e);
  return s;
}

// The new token of a query row, row / G, by a multiplication (rows < 2^28).
__device__ __forceinline__ int row_token(const AttendParams& p, int row) { return token_of_row(row, p.G, p.g_mul); }
// Output row (new token row / G, query head g * G + row % G) of sequence b.
template <typename T>
__device__ __forceinline__ T* out_row(const AttendParams& p, int b, int g, int row) {
  const int tok = row_token(p, row);
  return static_cast<T*>(p.out.data) + (int64_t)b * p.out.sb + (int64_t)tok * p.out.sn +
         (int64_t)(g * p.G + row - tok * p.G) * p.out.sh;
}
// The log-sum-exp of a row from its maximum (log2 units) and sum: a sum of 0 is a
// row that sees nothing, one that is not a number stays that.
__device__ __forceinline__ void store_lse(const AttendParams& p, int b, int g, int row, float m, float l) {
  const float x = l == 0.f ? -CUDART_INF_F : m + log2f(l);
  const int tok = row_token(p, row);
  if (p.lse) p.lse[((int64_t)b * p.n_new + tok) * p.H + g * p.G + row - tok * p.G] = x * kLn2;
  if (p.weigh) p.lse2[(int64_t)(b * p.Hkv + g) * p.R + row] = l == 0.f ? CUDART_INF_F : x;
}

// ---- The line of work of the tensor-core kernels (AttItem, LineCut).

// A CTA's place on it: the item (kv-head g, pair = sequence * nqt + row block)
// and the position within the item, its position on the line, positions left.
// With `shares` set the CTA has one part, share_at of an item's `shares`.
struct Walk {
  int g, pair, off;
  int pos, left;
  int shares, share_at;
  NewSeq sq;        // of the first item
  bool known;
  LineCut lc;
};
// The next item a CTA does, or its share of it (the same in every lane of a
// converged warp, which calls it together): tiles [u0, u1) of the list.
struct Part {
  int g, b, u0, u1;
  bool owner;       // this CTA holds the item's first position: it answers for an item without tiles
  int c0, parts;    // the item's tiles lie with CTAs [c0, c0 + parts)
  NewSeq sq;
  AttItem it;
  __device__ bool whole() const { return u0 == 0 && u1 == it.tl.n; }
};
__device__ __forceinline__ bool next_part(const AttendParams& p, Walk& w, Part& q) {
  if (w.left <= 0) return false;
  q.g = w.g;
  q.b = p.nqt == 1 ? w.pair : w.pair / p.nqt;
  if (!w.known) w.sq = load_new(p, q.b, false);
  w.known = false;
  q.sq.len = uniform(w.sq.len);
  q.sq.n = uniform(w.sq.n);
  q.it = att_item(q.sq.len, q.sq.n, p.G, p.block, w.pair - q.b * p.nqt, p.window, p.sinks, p.g_mul);
  const int cost = q.it.cost(p.fixed), end = min(cost, w.off + w.left), done = end - w.off;
  q.u0 = q.it.tiles_before(w.off, p.fixed);
  q.u1 = q.it.tiles_before(end, p.fixed);
  q.owner = w.off == 0;
  if (w.shares) {
    q.c0 = blockIdx.x - w.share_at;
    q.parts = w.shares;
  } else if (q.whole()) {
    q.c0 = blockIdx.x;
    q.parts = 1;
  } else {
    const int first = w.pos - w.off + p.fixed;
    q.c0 = w.lc.owner(first);
    q.parts = w.lc.owner(first + (q.it.tl.n - 1) * q.it.unit()) - q.c0 + 1;
  }
  w.left -= done;
  w.pos += done;
  w.off = 0;
  if (++w.pair == p.B * p.nqt) { w.pair = 0; ++w.g; }
  return true;
}
// The sum over the block's NT threads before this one, and over all of them.
template <int NT>
__device__ __forceinline__ int block_scan(int x, int* warps, int& total) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();
  if (lane == 31) warps[warp] = incl;
  __syncthreads();
  const int w = lane < NT / 32 ? warps[lane] : 0;
  total = __reduce_add_sync(0xffffffffu, w);
  return incl - x + __reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
}
// Finds this CTA's start: each thread sums the costs of a run of pairs, a block
// scan gives their places.  misc: NT / 32 + 7 ints of shared memory.
template <int NT>
__device__ __forceinline__ Walk line_start(const AttendParams& p, int* misc) {
  const int tid = threadIdx.x, ctas = gridDim.x;
  const int pairs = p.B * p.nqt, run = (pairs + NT - 1) / NT;
  const int i0 = min(pairs, tid * run), i1 = min(pairs, i0 + run);
  int* found = misc + NT / 32;
  NewSeq sq{0, 0};  // of the last pair looked at
  auto pair_cost = [&](int i, bool report) {
    const int b = p.nqt == 1 ? i : i / p.nqt;
    sq = load_new(p, b, report && blockIdx.x == 0 && i == b * p.nqt);
    return att_item(sq.len, sq.n, p.G, p.block, i - b * p.nqt, p.window, p.sinks, p.g_mul).cost(p.fixed);
  };
  int mine = 0;
#pragma unroll 1
  for (int i = i0; i < i1; ++i) mine += pair_cost(i, true);
  int total;
  int before = block_scan<NT>(mine, misc, total);
  Walk w{0, 0, 0, 0, 0, 0, 0, {0, 0}, true, LineCut()};
  if (pairs * p.Hkv <= ctas / 4 && run == 1) {
    // Few items: the smallest share that leaves no more shares than CTAs, found
    // in a few tries between the even share and one that surely does.
    const int all = total * p.Hkv, low = (all + ctas - 1) / ctas;
    const int high = (all + ctas - pairs * p.Hkv - 1) / (ctas - pairs * p.Hkv);
    int per, m = 0, heads;
#pragma unroll 1
    for (int t = 0; t < 4; ++t) {
      per = max(min_share(p.fixed), low + (high - low) * t / 3);
      m = tid < pairs ? share_count(mine, per) : 0;
      before = block_scan<NT>(m, misc, heads);
      if (heads * p.Hkv <= ctas) break;
    }
    w.g = blockIdx.x / heads;
    const int at = blockIdx.x - w.g * heads;
    if (tid < pairs && at >= before && at < before + m) {
      const int k = at - before;
      found[0] = tid;
      found[1] = mine * k / m;
      found[2] = sq.len;
      found[3] = sq.n;
      found[4] = m;
      found[5] = mine * (k + 1) / m - mine * k / m;
      found[6] = k;
    }
    __syncthreads();
    if (w.g < p.Hkv) {
      w.left = uniform(found[5]);
      w.shares = uniform(found[4]);
      w.share_at = uniform(found[6]);
    }
  } else {
    total = uniform(total);
    w.lc = LineCut(total * p.Hkv, ctas);
    if ((int)blockIdx.x < w.lc.nc) {
      w.pos = w.lc.start(blockIdx.x);
      w.left = w.lc.start(blockIdx.x + 1) - w.pos;
      w.g = w.pos / total;
    }
    const int at = w.pos - w.g * total;
    if (at >= before && at < before + mine) {
      int sum = before, i = i0;
      if (run > 1) {
#pragma unroll 1
        for (;; ++i) {
          const int cost = pair_cost(i, false);
          if (at < sum + cost) break;
          sum += cost;
        }
      }
      found[0] = i;
      found[1] = at - sum;
      found[2] = sq.len;
      found[3] = sq.n;
    }
    __syncthreads();
  }
  w.pair = uniform(found[0]);
  w.off = uniform(found[1]);
  w.sq = NewSeq{found[2], found[3]};
  return w;
}

// ---- Joining records.  A record holds, for RS query rows, the maximum and sum
// (part_st) and the unnormalised output (part_o) of one share of an item.

// Called by the NT threads of `bar` after their record is written: true for the
// group that is the last of `expected` to arrive at the ticket.
template <typename Sync>
__device__ __forceinline__ bool last_to_arrive(unsigned* ticket, unsigned expected, int tid, int* flag, Sync&& sync) {
  sync();
  if (tid == 0) {
    __threadfence();  // orders what the barrier made this thread see, too
    const bool last = atomicAdd(ticket, 1u) == expected - 1;
    if (last) *ticket = 0;  // for the next call
    *flag = last;
  }
  sync();
  const bool last = *flag != 0;
  if (last) __threadfence();
  return last;
}

// Four values of a row, 8 or 16 bytes at once.
__device__ __forceinline__ void store4(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 x) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
}
// Joins records rec(0) .. rec(n - 1) of rows [row0, row0 + rows) into out and
// lse.  A thread takes EU groups of four dimensions of a row and has KU records in
// flight (a round trip to L2 each time: the join is bound by their number): many
// records of few rows want EU = 1 and KU = 16, few records of many rows EU = KU = 4
// (two sequences, 400 new tokens of 1000, 28/4 heads of 128: 49 us a call against
// 100).
template <typename T, int D, int NT, int EU, int KU, typename Rec>
__device__ __forceinline__ void join_records(const AttendParams& p, int b, int g, int row0, int rows, int n, int RS,
                                             Rec&& rec, int tid) {
  constexpr int C = D / 4 / EU;  // threads per row, their groups C apart
#pragma unroll 1
  for (int e = tid; e < rows * C; e += NT) {
    const int r = e / C, d = 4 * (e % C);
    float m = -CUDART_INF_F, l = 0.f;
    float4 o[EU];
#pragma unroll
    for (int i = 0; i < EU; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int k0 = 0; k0 < n; k0 += KU) {
      float2 st[KU];
      float4 x[KU][EU];
#pragma unroll
      for (int k = 0; k < KU; ++k) {
        st[k] = make_float2(-CUDART_INF_F, 0.f);
#pragma unroll
        for (int i = 0; i < EU; ++i) x[k][i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k0 + k < n) {
          const int at = rec(k0 + k) * RS + r;  // at most 4 records per SM of up to 128 rows
          st[k] = __ldcg(reinterpret_cast<const float2*>(p.part_st) + at);
#pragma unroll
          for (int i = 0; i < EU; ++i)
            x[k][i] = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * D + d + 4 * C * i));
        }
      }
      float mn = m;
#pragma unroll
      for (int k = 0; k < KU; ++k) mn = fmaxf(mn, st[k].x);
      const float mu = mn == -CUDART_INF_F ? 0.f : mn;
      const float f = exp2f(m - mu);
      l *= f;
#pragma unroll
      for (int i = 0; i < EU; ++i) { o[i].x *= f; o[i].y *= f; o[i].z *= f; o[i].w *= f; }
#pragma unroll
      for (int k = 0; k < KU; ++k) {
        const float w = exp2f(st[k].x - mu);
        l = fmaf(w, st[k].y, l);
#pragma unroll
        for (int i = 0; i < EU; ++i) {
          o[i].x = fmaf(w, x[k][i].x, o[i].x);
          o[i].y = fmaf(w, x[k][i].y, o[i].y);
          o[i].z = fmaf(w, x[k][i].z, o[i].z);
          o[i].w = fmaf(w, x[k][i].w, o[i].w);
        }
      }
      m = mn;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    T* out = out_row<T>(p, b, g, row0 + r) + d;
#pragma unroll
    for (int i = 0; i < EU; ++i)
      store4(out + 4 * C * i, make_float4(o[i].x * inv, o[i].y * inv, o[i].z * inv, o[i].w * inv));
    if (d == 0) store_lse(p, b, g, row0 + r, m, l);
  }
}

inline cudaError_t launch_dep(void (*kernel)(AttendParams), dim3 grid, int threads, size_t smem, cudaStream_t st,
                              const AttendParams& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace vp
