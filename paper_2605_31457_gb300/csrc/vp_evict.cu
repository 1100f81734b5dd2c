// Eviction from a cache by accumulated attention weight (vp_evict).
//
//   k_evict_select  which tokens stay: the first `sinks`, the last `recent` and
//                   the largest weights between them; writes the kept positions
//                   in ascending order, the new length and the kept weights;
//   k_evict_move    moves the kept rows of K and V to the front, into other
//                   caches or in place.
#include <cuda_runtime.h>
#include <stdint.h>

#include "vp_attend.h"
#include "vp_device.h"

namespace vp {
namespace {

constexpr int kSelThreads = 1024, kSelWarps = kSelThreads / 32;
constexpr int kMoveThreads = 256;
constexpr int kMoveRows = 64;       // destination rows per CTA of k_evict_move, out of place
constexpr int kInPlaceRows = 8;     // rows a thread of it holds at a time, in place
constexpr int kBins = 2048;         // 11-bit digits

// Weights as integers in the same order; -0 equals +0 and NaN ranks below all.
__device__ __forceinline__ uint32_t order_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ int live_len(const EvictParams& p, int b, bool report) {
  const int t = __ldcg(p.seq_len + b);
  if (t >= 0 && t <= p.max_seq) return t;
  if (report) atomicOr(p.err, ERR_LEN);
  return min(max(t, 0), p.max_seq);
}

// Sum over the block; every thread gets it.  red: one int per warp.
__device__ __forceinline__ int block_sum(int x, int* red) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  x = __reduce_add_sync(0xffffffffu, x);
  __syncthreads();
  if (lane == 0) red[warp] = x;
  __syncthreads();
  return __reduce_add_sync(0xffffffffu, red[lane]);
}

// ---------------------------------------------------------------------------
// k_evict_select: one CTA of 1024 threads per (kept set, sequence).  The m-th
// largest key of the middle is found by radix select, three passes of 11, 11
// and 10 bits over the weights (in L2 after the first), a histogram of 2048
// bins in shared memory each; keys above it stay, and of the equal ones the
// first in position, so the result does not depend on any order of atomics.
// Two passes over contiguous warp segments then count and write the kept
// positions.  Bound by latency: five passes over T weights by one SM.
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(kSelThreads) k_evict_select(const __grid_constant__ EvictParams p) {
  __shared__ int hist[kBins];
  __shared__ int red[kSelWarps];
  __shared__ int seg_kept[kSelWarps], seg_eq[kSelWarps];
  __shared__ int bin_s, above_s;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g0 = p.granularity ? blockIdx.x : 0, b = blockIdx.y;
  const int T = live_len(p, b, blockIdx.x == 0);
  int32_t* kept = p.kept_idx + ((int64_t)b * (p.granularity ? p.Hkv : 1) + g0) * p.kept_cap;
  const int K = min(T, p.keep);
  for (int i = K + tid; i < p.kept_cap; i += kSelThreads) kept[i] = -1;
  const float* w0 = p.w.data + (int64_t)b * p.w.sb + (int64_t)g0 * p.w.sh;
  auto key_of = [&](int j) {
    float w = w0[j];
    if (!p.granularity)
      for (int g = 1; g < p.Hkv; ++g) w += w0[(int64_t)g * p.w.sh + j];
    return order_key(w);
  };
  if (T <= p.keep) {
    for (int i = tid; i < T; i += kSelThreads) kept[i] = i;
  } else {
    const int lo = p.sinks, hi = T - p.recent;
    int m = p.keep - p.sinks - p.recent;  // to choose of the hi - lo > m tokens between
    uint32_t prefix = 0, mask = 0;        // digits of the threshold found so far
    int equal = 0;                        // of the keys equal to the threshold, how many stay
    if (m > 0) {
      for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t digits = pass == 2 ? 1023u : 2047u;
        for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
        __syncthreads();
        for (int j = lo + tid; j < hi; j += kSelThreads) {
          const uint32_t k = key_of(j);
          if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & digits], 1);
        }
        __syncthreads();
        // The bin that holds the m-th largest: thread i owns bins 2i, 2i + 1
        // counted from the top.
        const int top = kBins - 1 - 2 * tid;
        const int h1 = hist[top], h0 = hist[top - 1];
        int incl = h1 + h0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += y;
        }
        if (lane == 31) red[warp] = incl;
        __syncthreads();
        const int before = __reduce_add_sync(0xffffffffu, lane < warp ? red[lane] : 0);
        const int ex = before + incl - h1 - h0;  // keys in higher bins
        if (ex < m && m <= ex + h1) { bin_s = top; above_s = ex; }
        else if (ex + h1 < m && m <= ex + h1 + h0) { bin_s = top - 1; above_s = ex + h1; }
        __syncthreads();
        m -= above_s;
        prefix |= (uint32_t)bin_s << shift;
        mask |= digits << shift;
        __syncthreads();
      }
      equal = m;
    }
    // Each warp takes a contiguous segment: counts, block scan, then writes.
    const int seg = ((T + kSelThreads - 1) / kSelThreads) * 32;
    const int a = min(T, warp * seg), z = min(T, a + seg);
    const bool any = p.keep > p.sinks + p.recent;
    auto classify = [&](int j, bool& above, bool& eq) {
      above = eq = false;
      if (j >= z) return;
      if (j < lo || j >= hi) { above = true; return; }
      if (!any) return;
      const uint32_t k = key_of(j);
      above = k > prefix;
      eq = k == prefix;
    };
    int ng = 0, ne = 0;
    for (int j = a + lane; j - lane < z; j += 32) {
      bool above, eq;
      classify(j, above, eq);
      ng += __popc(__ballot_sync(0xffffffffu, above));
      ne += __popc(__ballot_sync(0xffffffffu, eq));
    }
    if (lane == 0) { seg_kept[warp] = ng; seg_eq[warp] = ne; }
    __syncthreads();
    int eq_before = __reduce_add_sync(0xffffffffu, lane < warp ? seg_eq[lane] : 0);
    int at = __reduce_add_sync(0xffffffffu, lane < warp ? seg_kept[lane] : 0) + min(eq_before, equal);
    for (int j = a + lane; j - lane < z; j += 32) {
      bool above, eq;
      classify(j, above, eq);
      const unsigned me = __ballot_sync(0xffffffffu, eq), below = (1u << lane) - 1u;
      const bool stay = above || (eq && eq_before + __popc(me & below) < equal);
      const unsigned ms = __ballot_sync(0xffffffffu, stay);
      if (stay) kept[at + __popc(ms & below)] = j;
      at += __popc(ms);
      eq_before += __popc(me);
    }
  }
  if (!p.wd.data) return;
  // The kept weights, moved towards the front: a round's reads come before its
  // writes, and later rounds read beyond them (kept[i] >= i), so it may be in
  // place.
  __syncthreads();
  const int ng = p.granularity ? 1 : p.Hkv;
  for (int g = 0; g < ng; ++g) {
    const float* src = w0 + (int64_t)g * p.w.sh;
    float* dst = p.wd.data + (int64_t)b * p.wd.sb + (int64_t)(g0 + g) * p.wd.sh;
    for (int i0 = 0; i0 < K; i0 += kSelThreads) {
      const int i = i0 + tid;
      float x = 0.f;
      if (i < K) x = src[kept[i]];
      __syncthreads();
      if (i < K) dst[i] = x;
    }
    if (p.in_place)
      for (int i = K + tid; i < T; i += kSelThreads) dst[i] = 0.f;
  }
}

// Bytes of row (b, g, j) of a cache; NULL where its page is unmapped.
__device__ __forceinline__ char* row_bytes(const EvictParams& p, const KvView& kv, int b, int g, int j) {
  char* base = static_cast<char*>(const_cast<void*>(kv.data));
  int64_t off;
  if (!kv.block_table) {
    off = (int64_t)b * kv.sb + (int64_t)g * kv.sh + (int64_t)j * kv.st;
  } else {
    const int lp = j >> p.page_shift;
    const int page = lp < kv.max_pages ? __ldg(kv.block_table + (int64_t)b * kv.max_pages + lp) : -1;
    if (page < 0 || page >= kv.num_pages) return nullptr;
    off = (int64_t)page * kv.sb + (int64_t)g * kv.sh + (int64_t)(j & (p.page_size - 1)) * kv.st;
  }
  return base + off * p.esz;
}

// ---------------------------------------------------------------------------
// k_evict_move: one (sequence, kv-head, K or V) per group of CTAs; each thread
// copies 16-byte pieces.  Out of place a CTA takes 64 destination rows.  In
// place a CTA takes a column slice of every row, in rounds of destination rows
// in ascending order: a round's reads come before its writes (a barrier
// between), and kept[i] >= i, so no row is overwritten before it is read.
// Bound by HBM: each kept row is read and written once.
// ---------------------------------------------------------------------------
template <bool IN_PLACE>
__global__ void __launch_bounds__(kMoveThreads) k_evict_move(const __grid_constant__ EvictParams p, int slices,
                                                             int chunks) {
  // No early trigger: the next call may read these caches before its own wait.
  pdl_wait();
  const int tid = threadIdx.x;
  const int per = IN_PLACE ? slices : chunks;
  const int part = blockIdx.x % per;
  int rest = blockIdx.x / per;
  const int is_v = rest & 1;
  rest >>= 1;
  const int g = rest % p.Hkv, b = rest / p.Hkv;
  const KvView& src = is_v ? p.vs : p.ks;
  const KvView& dst = is_v ? p.vd : p.kd;
  // new_len may be seq_len itself, written below by another CTA: either value
  // gives the same K, and everything else comes from the kept list.
  const int K = min(live_len(p, b, false), p.keep);
  const int32_t* kept = p.kept_idx + ((int64_t)b * (p.granularity ? p.Hkv : 1) + (p.granularity ? g : 0)) * p.kept_cap;
  const int pieces = p.D * p.esz / 16;
  unsigned err = 0;
  if (!IN_PLACE) {
    const int step = kMoveThreads / pieces, r1 = min(K, (part + 1) * kMoveRows);
    for (int i = part * kMoveRows + tid / pieces; i < r1; i += step) {
      const char* s = row_bytes(p, src, b, g, __ldcg(kept + i));
      char* d = row_bytes(p, dst, b, g, i);
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (s) x = *(reinterpret_cast<const uint4*>(s) + tid % pieces);
      if (d) *(reinterpret_cast<uint4*>(d) + tid % pieces) = x;
      if (!s || !d) err |= ERR_PAGE;
    }
  } else if (K > 0 && __ldcg(kept + K - 1) != K - 1) {  // else every row stays where it is
    const int mine = pieces / slices, step = kMoveThreads / mine;
    const int piece = part * mine + tid % mine, r = tid / mine;
    for (int i0 = 0; i0 < K; i0 += step * kInPlaceRows) {
      uint4 x[kInPlaceRows];
      bool moved[kInPlaceRows];
#pragma unroll
      for (int k = 0; k < kInPlaceRows; ++k) {
        const int i = i0 + k * step + r;
        const int j = i < K ? __ldcg(kept + i) : i;
        x[k] = make_uint4(0u, 0u, 0u, 0u);
        moved[k] = j != i;
        if (!moved[k]) continue;
        const char* s = row_bytes(p, src, b, g, j);
        if (s) x[k] = *(reinterpret_cast<const uint4*>(s) + piece);
        else err |= ERR_PAGE;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kInPlaceRows; ++k) {
        if (!moved[k]) continue;
        char* d = row_bytes(p, dst, b, g, i0 + k * step + r);
        if (d) *(reinterpret_cast<uint4*>(d) + piece) = x[k];
        else err |= ERR_PAGE;
      }
    }
  }
  if (err) atomicOr(p.err, err);
  if (g == 0 && is_v == 0 && part == 0 && tid == 0) p.new_len[b] = K;
}

template <typename... Args>
cudaError_t launch_dep(void (*kernel)(Args...), dim3 grid, int threads, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace

cudaError_t launch_evict(const EvictParams& p, cudaStream_t st) {
  cudaError_t e = launch_dep(k_evict_select, dim3(p.granularity ? p.Hkv : 1, p.B), kSelThreads, st, p);
  if (e != cudaSuccess) return e;
  const int64_t units = (int64_t)p.B * p.Hkv * 2;
  // In place: column slices of at least 32 bytes (a sector), as many as it
  // takes for two CTAs per SM.
  const int pieces = p.D * p.esz / 16;
  int slices = 1;
  while (slices * 2 <= pieces / 2 && units * slices < 2 * p.num_sms) slices *= 2;
  const int rows = p.keep < p.max_seq ? p.keep : p.max_seq;
  const int chunks = (rows + kMoveRows - 1) / kMoveRows;
  const int64_t ctas = units * (p.in_place ? slices : chunks);
  if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
  if (ctas == 0) return cudaSuccess;
  return launch_dep(p.in_place ? k_evict_move<true> : k_evict_move<false>, dim3((unsigned)ctas), kMoveThreads, st, p,
                    slices, chunks);
}

}  // namespace vp
