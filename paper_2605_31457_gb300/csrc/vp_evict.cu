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
constexpr int kMoveThreads = 128, kMoveWarps = kMoveThreads / 32;
constexpr int kMoveLoads = 4;       // 16-byte pieces a lane of k_evict_move has in flight, out of place
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

// ---------------------------------------------------------------------------
// k_evict_select<KR>: one CTA of 1024 threads per (kept set, sequence).  Each
// warp owns a contiguous segment of the tokens, each thread every 32nd token of
// it; their keys are formed once and held, KR per thread in registers or (KR =
// 0) in shared memory, up to kSelShared of them (KR < 0, longer caches: formed
// again in every pass).  The m-th largest key of the middle is found by radix
// select in three passes of 11, 11 and 10 bits, a histogram of 2048 bins each.
// After the first one a thread holds, a bit per token, which stay for sure and
// which are in the threshold's bin; only the latter, a few in a hundred, are
// looked at again.  Keys above the threshold stay, and of the equal ones the
// first in position, so the result does not depend on any order of atomics.
// Bound by instructions and barriers on one SM: a call on one sequence of 3857
// tokens takes 9.2 us with the move, on 8 of 20480 tokens 38 us.  Slower were: 256 bins with a
// column per lane against queues at one address and four passes (3857 tokens:
// 10.0 against 7.6 us), one addition per bin and warp after matching the lanes
// (10.4 us), clusters of eight CTAs that share their histograms through
// distributed shared memory (20480 tokens: 44 us).
// ---------------------------------------------------------------------------
constexpr int kSelShared = 32 * kSelThreads;  // keys held in shared memory, at most: a bit of a word each

template <int KR>
__global__ void __launch_bounds__(kSelThreads) k_evict_select(const __grid_constant__ EvictParams p) {
  extern __shared__ uint32_t keys_s[];
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
  const float* w0 = p.w.data + (int64_t)b * p.w.sb + (int64_t)g0 * p.w.sh;
  float* wd0 = p.wd.data + (int64_t)b * p.wd.sb + (int64_t)g0 * p.wd.sh;
#pragma unroll 1
  for (int i = K + tid; i < p.kept_cap; i += kSelThreads) kept[i] = -1;
  if (T <= p.keep) {  // every token stays where it is
#pragma unroll 1
    for (int j = tid; j < T; j += kSelThreads) kept[j] = j;
    if (p.wd.data && !p.in_place)
      for (int g = 0; g < (p.granularity ? 1 : p.Hkv); ++g)
#pragma unroll 1
        for (int j = tid; j < T; j += kSelThreads) wd0[(int64_t)g * p.wd.sh + j] = w0[(int64_t)g * p.w.sh + j];
    return;
  }
  const int steps = KR > 0 ? KR : (T + kSelThreads - 1) / kSelThreads;
  const int a = warp * steps * 32 + lane;  // the thread's first token
  const int lo = p.sinks, hi = T - p.recent;  // the middle to choose from
  const int heads = p.granularity ? 1 : p.Hkv;
  // The weights of tokens j, j + 32, ..., summed over the heads of the set; 0 past the end.
  auto weights_at = [&](int j, auto& w) {
    constexpr int N = sizeof(w) / sizeof(float);
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = j + 32 * i < T ? w0[j + 32 * i] : 0.f;
#pragma unroll 1
    for (int g = 1; g < heads; ++g) {
      float x[N];
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = j + 32 * i < T ? w0[(int64_t)g * p.w.sh + j + 32 * i] : 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] += x[i];
    }
  };
  auto weight_at = [&](int j) {
    float w[1];
    weights_at(j, w);
    return w[0];
  };
  float held[KR > 0 ? KR : 1];
  if constexpr (KR > 0) {
    weights_at(a, held);
  } else if constexpr (KR == 0) {  // a thread reads back only what it wrote
#pragma unroll 1
    for (int i0 = 0; i0 < steps; i0 += 8) {
      float w[8];
      weights_at(a + 32 * i0, w);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (i0 + k < steps && a + 32 * (i0 + k) < T) keys_s[a + 32 * (i0 + k)] = order_key(w[k]);
    }
  }
  // This thread's steps, a bit each, whose token lies in front of x (KR >= 0: at most
  // 32 steps).
  auto in_front = [&](int x) {
    const int n = min((x - a + 31) >> 5, steps);
    return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u;
  };
  // Calls f(step, key) for this thread's tokens of the middle; KR >= 0: for those in
  // `bits`, most of them or (few) a few.
  auto each = [&](uint32_t bits, bool few, auto&& f) {
    if constexpr (KR > 0) {
#pragma unroll
      for (int i = 0; i < KR; ++i)
        if ((bits >> i) & 1u) f(i, order_key(held[i]));
    } else if constexpr (KR == 0) {
      if (!few) {
#pragma unroll 4
        for (int i = 0; i < steps; ++i)
          if ((bits >> i) & 1u) f(i, keys_s[a + 32 * i]);
      } else {
#pragma unroll 1
        for (uint32_t c = bits; c; c &= c - 1) {
          const int i = __ffs(c) - 1;
          f(i, keys_s[a + 32 * i]);
        }
      }
    } else {
      for (int i = 0; i < steps; ++i) {
        const int j = a + 32 * i;
        if (j >= lo && j < hi) f(i, order_key(weight_at(j)));
      }
    }
  };
  int m = p.keep - p.sinks - p.recent;  // how many of the middle stay
  uint32_t prefix = 0, mask = 0;        // digits of the threshold found so far
  // A bit per step: stays for sure; may be equal to the threshold.
  uint32_t up = 0, cand = in_front(hi) & ~in_front(lo);
  const bool any = m > 0;
  if (any) {
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t digits = pass == 2 ? 1023u : 2047u;
      for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
      __syncthreads();
      each(cand, pass > 0, [&](int, uint32_t k) {
        if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & digits], 1);
      });
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
      if constexpr (KR >= 0) {
        uint32_t in = 0;
        each(cand, pass > 0, [&](int i, uint32_t k) {
          const uint32_t d = k & mask;
          if (d > prefix) up |= 1u << i;
          if (d == prefix) in |= 1u << i;
        });
        cand = in;
      }
    }
  } else {
    cand = 0;
  }
  const int equal = any ? m : 0;  // of the keys equal to the threshold, how many stay
  // Counts per segment, their scan, then the kept positions in order.
  auto stays = [&](int j, bool& eq) {  // KR < 0: without ties; eq: equal to the threshold
    const bool mid = j >= lo && j < hi;
    const uint32_t k = mid && any ? order_key(weight_at(j)) : 0u;
    eq = mid && any && k == prefix;
    return (mid && any && k > prefix) || (j < T && !mid);
  };
  if constexpr (KR >= 0) up |= (in_front(lo) | ~in_front(hi)) & in_front(T);
  int ng = __popc(up), ne = __popc(cand);
  if constexpr (KR < 0) {
    ng = ne = 0;
    for (int i = 0; i < steps; ++i) {
      bool eq;
      ng += stays(a + 32 * i, eq);
      ne += eq;
    }
  }
  ng = __reduce_add_sync(0xffffffffu, ng);
  ne = __reduce_add_sync(0xffffffffu, ne);
  if (lane == 0) { seg_kept[warp] = ng; seg_eq[warp] = ne; }
  __syncthreads();
  int eq_before = __reduce_add_sync(0xffffffffu, lane < warp ? seg_eq[lane] : 0);
  int at = __reduce_add_sync(0xffffffffu, lane < warp ? seg_kept[lane] : 0) + min(eq_before, equal);
  // Usually the equal ones all stay; only a tie that is split asks for their order.
  const bool tie = KR < 0 || __reduce_add_sync(0xffffffffu, seg_eq[lane]) != equal;
  if (!tie) up |= cand;
  // One kept set per kv-head: the weights go along, from registers (every one
  // has been read, so also in place) or, out of place, read again.
  const bool along = p.granularity && p.wd.data && (KR > 0 || !p.in_place);
  auto emit = [&](int i, int j, float w) {
    const unsigned below = (1u << lane) - 1u;
    bool stay = (up >> i) & 1u;
    if (tie) {
      bool eq = (cand >> i) & 1u;
      if constexpr (KR < 0) stay = stays(j, eq);
      const unsigned me = __ballot_sync(0xffffffffu, eq);
      stay = stay || (eq && eq_before + __popc(me & below) < equal);
      eq_before += __popc(me);
    }
    const unsigned ms = __ballot_sync(0xffffffffu, stay);
    const int to = at + __popc(ms & below);
    if (stay && to < K) {
      kept[to] = j;
      if (along) wd0[to] = w;
    }
    at += __popc(ms);
  };
  if constexpr (KR > 0) {
#pragma unroll
    for (int i = 0; i < KR; ++i) emit(i, a + 32 * i, held[i]);
  } else {
#pragma unroll 1
    for (int i0 = 0; i0 < steps; i0 += 4) {
      float w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = along && i0 + k < steps && a + 32 * (i0 + k) < T ? w0[a + 32 * (i0 + k)] : 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i0 + k < steps) emit(i0 + k, a + 32 * (i0 + k), w[k]);
    }
  }
  if (!p.wd.data) return;
  // Other forms: the kept weights move towards the front; a round's reads come
  // before its writes, and later rounds read beyond them (kept[i] >= i), so it
  // may be in place.
  __syncthreads();
#pragma unroll 1
  for (int g = 0; g < heads; ++g) {
    const float* src = w0 + (int64_t)g * p.w.sh;
    float* dst = wd0 + (int64_t)g * p.wd.sh;
#pragma unroll 1
    for (int i0 = 0; i0 < (along ? 0 : K); i0 += kSelThreads) {
      const int i = i0 + tid;
      float x = 0.f;
      if (i < K) x = src[kept[i]];
      __syncthreads();
      if (i < K) dst[i] = x;
    }
    if (p.in_place)
#pragma unroll 1
      for (int i = K + tid; i < T; i += kSelThreads) dst[i] = 0.f;
  }
}

// The page of token j of sequence b, -1 where the block table maps it to none;
// 0 in a contiguous cache.
__device__ __forceinline__ int page_of(const EvictParams& p, const KvView& kv, int b, int j) {
  if ((unsigned)j >= (unsigned)p.max_seq) return -1;  // no position of a kept list lies there
  if (!kv.block_table) return 0;
  const int lp = j >> p.page_shift;
  const int page = lp < kv.max_pages ? __ldg(kv.block_table + (int64_t)b * kv.max_pages + lp) : -1;
  return page < kv.num_pages ? page : -1;
}
// Bytes of row (b, g, j) of a cache, its page known; NULL for page -1.
__device__ __forceinline__ char* row_bytes(const EvictParams& p, const KvView& kv, int b, int g, int j, int page) {
  if (page < 0) return nullptr;
  const int64_t off = kv.block_table
      ? (int64_t)page * kv.sb + (int64_t)g * kv.sh + (int64_t)(j & (p.page_size - 1)) * kv.st
      : (int64_t)b * kv.sb + (int64_t)g * kv.sh + (int64_t)j * kv.st;
  return static_cast<char*>(const_cast<void*>(kv.data)) + off * p.esz;
}

// ---------------------------------------------------------------------------
// k_evict_move: one (sequence, kv-head, K or V) per group of CTAs.  Out of place
// a warp takes a run of up to 32 destination rows: lane i looks up where row i
// comes from and goes to, then the rows are moved 16 bytes a lane, their addresses
// passed by shuffles (every lane finding its own rows' addresses, four rows each,
// it was bound by those instructions: 119 against 91 us a call with 512 MB to move).
// In place a CTA takes a column slice of every row, in rounds of destination rows
// in ascending order: a round's reads come before its writes (a barrier between),
// and kept[i] >= i, so no row is
// overwritten before it is read.  Bound by HBM: each kept row is read and written
// once (a call with 512 MB of 256-byte rows in pages of 16: 91 us, 5.6 TB/s with the
// selection).  In place the same call takes 281 us, 240 without pages, bound by
// latency (kept position, page, row, barrier in every round: 15% of DRAM's rate).
// ---------------------------------------------------------------------------
template <bool IN_PLACE>
__global__ void __launch_bounds__(kMoveThreads) k_evict_move(const __grid_constant__ EvictParams p, int slices,
                                                             int chunks, int run) {
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
    // Lane i of a warp finds where row i of its `run` rows comes from and goes to;
    // then `pieces` lanes move a row together.
    const int lane = tid & 31, i = (part * kMoveWarps + (tid >> 5)) * run + lane;
    const char* from = nullptr;
    char* to = nullptr;
    if (lane < run && i < K) {
      const int j = __ldcg(kept + i);
      from = row_bytes(p, src, b, g, j, page_of(p, src, b, j));
      to = row_bytes(p, dst, b, g, i, page_of(p, dst, b, i));
      if (!from || !to) err |= ERR_PAGE;
    }
    const int step = 32 / pieces, r = lane / pieces, at = lane % pieces * 16;
    auto pointer = [](const char* x, int lane) {
      return reinterpret_cast<char*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(x), lane));
    };
#pragma unroll 1
    for (int r0 = r; r0 - r < run; r0 += kMoveLoads * step) {
      uint4 x[kMoveLoads];
#pragma unroll
      for (int k = 0; k < kMoveLoads; ++k) {
        const char* s = pointer(from, r0 + k * step);
        x[k] = make_uint4(0u, 0u, 0u, 0u);
        if (s && r0 + k * step < run) x[k] = __ldcs(reinterpret_cast<const uint4*>(s + at));
      }
#pragma unroll
      for (int k = 0; k < kMoveLoads; ++k) {
        char* d = pointer(to, r0 + k * step);
        if (d && r0 + k * step < run) __stcs(reinterpret_cast<uint4*>(d + at), x[k]);
      }
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
        const char* s = row_bytes(p, src, b, g, j, page_of(p, src, b, j));
        if (s) x[k] = *(reinterpret_cast<const uint4*>(s) + piece);
        else err |= ERR_PAGE;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kInPlaceRows; ++k) {
        if (!moved[k]) continue;
        const int i = i0 + k * step + r;
        char* d = row_bytes(p, dst, b, g, i, page_of(p, dst, b, i));
        if (d) *(reinterpret_cast<uint4*>(d) + piece) = x[k];
        else err |= ERR_PAGE;
      }
    }
  }
  if (err) atomicOr(p.err, err);
  if (g == 0 && is_v == 0 && part == 0 && tid == 0) p.new_len[b] = K;
}

template <typename... Args>
cudaError_t launch_dep(void (*kernel)(Args...), dim3 grid, int threads, size_t smem, cudaStream_t st, Args... args) {
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
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace

cudaError_t configure_evict() {
  return cudaFuncSetAttribute(k_evict_select<0>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelShared * 4);
}

cudaError_t launch_evict(const EvictParams& p, cudaStream_t st) {
  const dim3 sets(p.granularity ? p.Hkv : 1, p.B);
  cudaError_t e;
  if (p.max_seq <= 4 * kSelThreads) e = launch_dep(k_evict_select<4>, sets, kSelThreads, 0, st, p);
  else if (p.max_seq <= 8 * kSelThreads) e = launch_dep(k_evict_select<8>, sets, kSelThreads, 0, st, p);
  else if (p.max_seq <= kSelShared) e = launch_dep(k_evict_select<0>, sets, kSelThreads, (size_t)p.max_seq * 4, st, p);
  else e = launch_dep(k_evict_select<-1>, sets, kSelThreads, 0, st, p);
  if (e != cudaSuccess) return e;
  const int64_t units = (int64_t)p.B * p.Hkv * 2;
  // In place: column slices of at least 32 bytes (a sector), as many as it
  // takes for two CTAs per SM.
  const int pieces = p.D * p.esz / 16;
  int slices = 1;
  while (slices * 2 <= pieces / 2 && units * slices < 2 * p.num_sms) slices *= 2;
  const int rows = p.keep < p.max_seq ? p.keep : p.max_seq;
  // Rows of a warp, out of place: 16, or 8 where that leaves fewer than four CTAs
  // per SM (one sequence, 2048 rows kept: 9.4 us a call with 8, 10.0 with 16; 32
  // sequences, 4096 rows: 97 with 8, 91 with 16).
  const int64_t wide = units * ((rows + 16 * kMoveWarps - 1) / (16 * kMoveWarps));
  const int run = wide >= 4 * p.num_sms ? 16 : 8, per_cta = kMoveWarps * run;
  const int chunks = (rows + per_cta - 1) / per_cta;
  const int64_t grid = units * (p.in_place ? slices : chunks);
  if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
  if (grid == 0) return cudaSuccess;
  return launch_dep(p.in_place ? k_evict_move<true> : k_evict_move<false>, dim3((unsigned)grid), kMoveThreads, 0, st, p,
                    slices, chunks, run);
}

}  // namespace vp
