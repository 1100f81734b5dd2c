// k_att_tc: attention of newly appended tokens on the fifth-generation tensor
// cores (vp_attend_new, bf16 caches that a tensor map describes).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include "vp_attend.h"
#include "vp_attend_device.h"
#include "vp_device.h"

namespace vp {
namespace {

// ---------------------------------------------------------------------------
// k_att_tc<D, NQ>: one CTA per SM, 352 threads in four roles.
//   warps 0-3, 4-7  two softmax groups, a thread per query row;
//   warp 8          copies tiles of 128 K or V rows into a ring (4-D bulk-tensor
//                   copies, 128-byte swizzle);
//   warps 9, 10     one lane each issues tcgen05.mma for one of the groups: S =
//                   Q K^T (M = 128 query rows, N = 128 tokens, K = D) and, half
//                   a tile at a time, O += P V (M = 128, N = D, K = 64) with P
//                   in TMEM.
// Query rows are the (new token, head of the kv-head) pairs, so a group of G
// heads shares every K and V row that is copied.  Each softmax group has its
// own S and O in TMEM (4 x 128 columns = all 512 at D = 128); P overwrites S.
// The groups take turns: while one turns its S into P the tensor cores work for
// the other.
//   NQ = 1 (65 to 128 rows): both groups hold the same queries and take alternate
//          tiles; each writes its own record, also of an item that the CTA does
//          alone.
//   NQ = 2 (prompts): the groups hold 128 query rows each and both read every
//          tile.
// The work is a line of tiles cut evenly over the CTAs (vp_attend.h): an item
// cut between CTAs leaves a record (m, l, O) per CTA, and the last CTA to finish
// joins them; the two records of an item that one CTA has alone (NQ = 1) are
// joined in it, between two barriers of the groups.
//
// Prompts are bound by two chains that take turns, not by a pipe: per half tile
// a softmax thread spends its time on 64 exponentials, the two terms of P, and
// waits, TMEM loads and arrivals, and a product warp on issuing 16 products (S
// from 64 tokens reads 6 KB of shared memory for 32 clocks of tensor work).  28/4
// heads of 128: 3857 tokens in 147 us (725 TFLOP/s); 32/8 heads, 12289 tokens with
// a window of 2048 and 4 sinks in 463 us (818 TFLOP/s).  112 rows (NQ = 1): 64
// sequences of 700 to 6400 tokens, 28/4 heads, 16 new tokens each in 126 us (3.7
// TB/s of cache), or 400 us with weights, when it writes 407 MB of logits that their
// kernel reads.  When long ranges had P in
// one term (see below), slower were: two warps for every 32 rows,
// 32 columns each (16 softmax warps of 96 registers; 533 against 447 us at the
// time); S's second half loaded during the first's exponentials (461 against 420);
// the next step's S fetched before a P is announced (491 against 419).  What
// helped most was less code: instructions fetched from L2 cost more than the
// work outside the tile loop (211 -> 90 KB of code, 526 -> 420 us with the next
// part's queries loaded during this one's output), and joins with more loads in
// flight (419 -> 388).
//
// Softmax: a row's reference m is the largest logit of the first 64 tokens it
// sees, and is raised, O rescaled in TMEM, only when P = exp2(z - m) passes 2^64:
// up to there P has bf16's and float's full precision all the same, and S is
// read once.  P goes to the tensor cores as two bf16 terms, hi + lo (2^-16 of it
// at most is lost); l sums the unrounded values in 32 bits.  With one term the two
// prompts above take 123 and 380 us, but its error does not average out: over 4096 to 16384 tokens it is 1.4 times that of a rounded
// exact result where the weight is spread (2.3e-3 of the output's rms against
// 1.7e-3) and 7 to 18 times where one token has nearly all of it (1.5e-3 against
// 0.8e-4 to 2e-4), whatever the range.
//
// Rows of a tile that nobody sees may hold anything: their logits are masked,
// and their V rows are zeroed in shared memory before the product (0 x NaN is
// not 0); pages that hold only such rows are not copied at all.
//
// Waits are bounded: a role whose wait gives up stops working, still meets
// every barrier of its group, and the error word reports it.
// ---------------------------------------------------------------------------
constexpr int kAttThreads = 352;
constexpr int kSub = 64;       // tokens of a softmax step: half a tile
constexpr float kPMost = 18446744073709551616.f;  // 2^64
constexpr int kMaskRing = 16;  // tiles between the copy warp and the softmax groups, at most

template <int D, int NQ>
struct TcCfg2 {
  static constexpr int HALF = kTcTile * 128;            // 128 rows x 64 dimensions, swizzled
  static constexpr int HALVES = D / 64;
  static constexpr int SLOT = HALVES * HALF;            // a tile of K or of V, or 128 query rows
  static constexpr int S = D == 128 ? 7 - NQ : 8;       // ring slots
  static constexpr int LA = NQ == 1 ? 2 : 1;            // tiles whose S is ahead of the P.V product
  static constexpr int OFF_Q = S * SLOT;
  static constexpr int OFF_BAR = OFF_Q + NQ * SLOT;
  static constexpr int NBAR = 2 * S + 18;               // full, empty, s_full, p_full, pv_done, o_free, q_full, done
  static constexpr int OFF_BAD = OFF_BAR + NBAR * 8;    // unmapped boxes of a tile, one bit each
  static constexpr int OFF_MISC = OFF_BAD + kMaskRing * 4;  // int [16]: scan, start, TMEM base
  static constexpr size_t SMEM = 1024 + (size_t)OFF_MISC + 24 * 4;
  static_assert(SMEM <= 232448, "227 KB of shared memory");
  static_assert(S >= 2 * LA, "the K tiles ahead and a V tile fit the ring");
};

// Instruction descriptor: bf16 x bf16 -> f32, M = 128, N = n, A K-major, B
// K-major or (b_mn) MN-major.
__host__ __device__ constexpr uint32_t att_idesc(int n, int b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(128 >> 4) << 24);
}

// The first n of 32 bits.
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }
// Which of the 32 tokens from jb on (columns k .. k + 31 of their tile) a row at
// position t sees whose window begins after `low`; bad: the tile's unmapped boxes
// of 1 << box rows.
__device__ __forceinline__ uint32_t seen_bits(int jb, int t, int low, int sinks, uint32_t bad, int k, int box) {
  uint32_t see = low_bits(t + 1 - jb) & (~low_bits(low + 1 - jb) | low_bits(sinks - jb));
  if (bad) {
#pragma unroll 1
    for (int x = 0; x < 32; ++x)
      if ((bad >> ((k + x) >> box)) & 1u) see &= ~(1u << x);
  }
  return see;
}
// The 32 tokens' logits that `see` lacks become -infinity.
__device__ __forceinline__ void mask_cols(float (&x)[32], uint32_t see) {
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = (see >> i) & 1u ? x[i] : -CUDART_INF_F;
}
// Four 16-byte pieces per lane: piece j of lane i of a quad goes to piece i of lane j.
__device__ __forceinline__ void quad_transpose(uint4 (&v)[4], int lane) {
  auto swap = [](uint4& a, uint4& b, bool upper, int x) {  // a of the upper lane and b of the lower one
    const uint4 send = upper ? a : b;
    uint4 got;
    got.x = __shfl_xor_sync(0xffffffffu, send.x, x);
    got.y = __shfl_xor_sync(0xffffffffu, send.y, x);
    got.z = __shfl_xor_sync(0xffffffffu, send.z, x);
    got.w = __shfl_xor_sync(0xffffffffu, send.w, x);
    if (upper) a = got;
    else b = got;
  };
  swap(v[0], v[1], lane & 1, 1);
  swap(v[2], v[3], lane & 1, 1);
  swap(v[0], v[2], lane & 2, 2);
  swap(v[1], v[3], lane & 2, 2);
}
template <int D, int NQ>
__global__ void __launch_bounds__(kAttThreads, 1) k_att_tc(const __grid_constant__ AttendParams p) {
  using C = TcCfg2<D, NQ>;
  constexpr int S = C::S, LA = C::LA;
  constexpr uint32_t kIdQK = att_idesc(kSub, 0), kIdPV = att_idesc(D, 1);
  extern __shared__ __align__(16) unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);  // [S] a slot's copies landed
  uint64_t* empty = full + S;                                        // [S] a slot's tile was read
  uint64_t* s_full = full + 2 * S;                                   // [2][2] half a tile's S of a group written
  uint64_t* p_full = s_full + 4;                                     // [2][2] its P written (an arrival per warp)
  uint64_t* pv_done = s_full + 8;                                    // [2][2] its P.V complete
  uint64_t* o_free = s_full + 12;                                    // [2] O of the last part read (128)
  uint64_t* q_full = s_full + 14;                                    // [2] a group's queries loaded (128; NQ = 1: 256)
  uint64_t* done = s_full + 16;                                      // [2] every product of a group complete
  volatile uint32_t* bad_ring = reinterpret_cast<uint32_t*>(smem + C::OFF_BAD);
  int* misc = reinterpret_cast<int*>(smem + C::OFF_MISC);            // [0, 18) line_start; [18, 19] flags; [20] TMEM

  if (tid == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, 2);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(s_full + i, 1);
      mbar_init(p_full + i, 4);
      mbar_init(pv_done + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(o_free + i, 128);
      mbar_init(q_full + i, NQ == 1 ? 256 : 128);
      mbar_init(done + i, 1);
    }
    mbar_fence_init();
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&p.tmk)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&p.tmv)) : "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(misc + 20))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  pdl_wait();
  pdl_trigger();
  tc_fence_before();
  Walk walk = line_start<kAttThreads>(p, misc);  // passes the CTA-wide barrier
  tc_fence_after();
  Part q;
  const unsigned tmem = (unsigned)uniform(misc[20]);  // columns [0, 128), [128, 256): S / P; from 256: O of the groups
  const int R2 = p.paged ? min(kTcTile, p.page_size) : kTcTile;  // rows per copied box
  const int box = 31 - __clz(R2), nb = kTcTile / R2;
  unsigned err = 0;
  bool timed_out = false;

  if (warp == 8) {
    // -------------------------------------------------------------- copies
    // Pieces in the order the tensor cores read them: K of the first LA
    // tiles, then V of a tile and K of the tile LA later.  Lane HALVES * x + hh
    // copies half hh of box x.
    const int x = lane / C::HALVES, hh = lane % C::HALVES;
    int pc = 0, tiles = 0;
    auto lookup = [&](const Part& q, int u, int& kp, int& vp) {  // pages of this lane's box of tile u; -2: not needed
      kp = vp = -2;
      if (x >= nb) return;
      const int j0 = q.it.tl.tile(u) * kTcTile + x * R2, j1 = j0 + R2;
      const SeenRange& sr = q.it.sr;
      if (!(j0 < sr.s_end || max(j0, sr.lo) < min(j1, sr.hi))) return;
      if (!p.paged) { kp = vp = q.b; return; }
      const int lp = j0 >> p.page_shift;
      int a = -1, c = -1;
      if (lp < p.k.max_pages) a = __ldg(p.k.block_table + (int64_t)q.b * p.k.max_pages + lp);
      if (lp < p.v.max_pages) c = __ldg(p.v.block_table + (int64_t)q.b * p.v.max_pages + lp);
      const bool ok = a >= 0 && a < p.k.num_pages && c >= 0 && c < p.v.num_pages;
      kp = ok ? a : -1;
      vp = ok ? c : -1;
    };
    auto issue = [&](const Part& q, int u, const CUtensorMap* map, int page) {
      const int sl = pc % S;
      if (!__all_sync(0xffffffffu, mbar_wait(empty + sl, ((pc / S) & 1) ^ 1))) return false;
      const bool live = page >= 0;
      const unsigned n_live = __popc(__ballot_sync(0xffffffffu, live));
      if (lane == 0) mbar_expect_tx(full + sl, n_live * (unsigned)R2 * 128u);
      __syncwarp();
      if (live) {
        const int j = q.it.tl.tile(u) * kTcTile + x * R2;
        const int row = p.paged ? j & (p.page_size - 1) : j;
        auto crd = [&](int axis) { return axis == p.tpos ? row : axis == p.gpos ? q.g : page; };
        const unsigned dst = smem_u32(smem + sl * C::SLOT) + hh * C::HALF + x * R2 * 128;
        if (NQ == 1) tma_load_4d(dst, map, 64 * hh, crd(1), crd(2), crd(3), full + sl);
        else tma_load_4d_keep(dst, map, 64 * hh, crd(1), crd(2), crd(3), full + sl);
      }
      ++pc;
      return true;
    };
    while (!timed_out && next_part(p, walk, q)) {
      const int n = q.u1 - q.u0;
      int kp = -2, vp = -2, kn, vn;   // pages of tile i, looked up one tile ahead
      int vq[LA];                     // V pages of the tiles whose V is due
      if (n > 0) lookup(q, q.u0, kp, vp);
#pragma unroll 1
      for (int i = 0; i < n + LA && n > 0; ++i) {
        kn = vn = -2;
        if (i + 1 < n) lookup(q, q.u0 + i + 1, kn, vn);
        if (i >= LA && !issue(q, q.u0 + i - LA, &p.tmv, vq[LA - 1])) { timed_out = true; break; }
        if (i < n) {
          const unsigned bad = __ballot_sync(0xffffffffu, kp == -1 && hh == 0);
          unsigned boxes = 0;  // bit of box x instead of lane HALVES * x
#pragma unroll
          for (int y = 0; y < 32 / C::HALVES; ++y) boxes |= ((bad >> (C::HALVES * y)) & 1u) << y;
          if (bad) err |= ERR_PAGE;
          if (lane == 0) bad_ring[tiles % kMaskRing] = boxes;
          ++tiles;
          if (!issue(q, q.u0 + i, &p.tmk, kp)) { timed_out = true; break; }
        }
#pragma unroll
        for (int y = LA - 1; y > 0; --y) vq[y] = vq[y - 1];
        vq[0] = vp;
        kp = kn;
        vp = vn;
      }
    }
    // Copies still in flight (only after a timeout can any be unread) land
    // before the CTA's shared memory is released.
#pragma unroll 1
    for (int k = max(0, pc - S); k < pc; ++k) mbar_wait(full + k % S, (k / S) & 1);
  } else if (warp >= 9) {
    // ------------------------------- tensor cores, a warp for each group s
    // Half a tile at a time: S of the next tile's half follows P.V of this
    // tile's same half, whose columns it takes, so that the softmax threads have
    // the next S while they form a P.  One warp for both
    // groups spent more time waiting at barriers than the products took.
    auto wait = [&](uint64_t* bar, unsigned parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)); };
    const int leader = elect_one();
    const int s = uniform(warp - 9);
    const unsigned o = tmem + 256 + D * s, pa = tmem + 128 * s;
    int slot = 0, tiles = 0;                   // the ring's next piece; tiles of the parts before
    unsigned phase = 0, parts = 0, tp = 0;     // of the ring; parts with tiles of this group, its tiles before
    // The next piece of the ring.  Every one is waited for, in order, and released
    // by both warps, the group's own or not: a warp that left some out could take
    // a later phase of a slot's barrier for the one it waits for.
    auto take = [&](int& sl) {
      sl = slot;
      const bool ok = wait(full + slot, phase);
      if (++slot == S) { slot = 0; phase ^= 1; }
      return ok;
    };
    auto qk = [&](int half, int ks) {  // by the leader: S of half a tile
      const uint32_t kd = umma_desc_lo(smem_u32(smem + ks * C::SLOT) + half * kSub * 128, 16);
      const uint32_t qd = umma_desc_lo(smem_u32(smem + C::OFF_Q + (NQ == 1 ? 0 : s) * C::SLOT), 16);
      umma_ss<kIdQK, 0>(pa + kSub * half, qd, kd);
#pragma unroll
      for (int x = 1; x < D / 16; ++x) {  // 16 dimensions: 32 bytes, every fourth step the next half
        const uint32_t at = (x >> 2) * (C::HALF / 16) + (x & 3) * 2;
        umma_ss<kIdQK, 1>(pa + kSub * half, qd + at, kd + at);
      }
      umma_commit(s_full + 2 * s + half);
    };
    while (!timed_out && next_part(p, walk, q)) {
      const int n = q.u1 - q.u0;
      if (n <= 0) continue;
      const int two = NQ == 2 && q.it.rows > kTcTile;  // the second group has rows
      auto own = [&](int t) { return NQ == 2 ? s == 0 || two : (t & 1) == s; };  // tile t is this group's
      if (NQ == 2 ? s == 0 || two : n > s) {  // it has tiles in this part
        if (!wait(q_full + s, parts & 1)) { timed_out = true; break; }
        ++parts;
      }
      // The copy warp's order: K of the first LA tiles, then V of a tile and K of
      // the tile LA later.
#pragma unroll 1
      for (int t = 0; t < min(LA, n); ++t) {
        int ks;
        if (!take(ks)) { timed_out = true; break; }
        if (leader) {
          if (own(t)) {
            qk(0, ks);
            qk(1, ks);
          }
          umma_commit(empty + ks);
        }
        __syncwarp();
      }
      int mine = 0;  // tiles of this group so far
#pragma unroll 1
      for (int t = 0; t < n && !timed_out; ++t) {
        int vs, ks = -1;
        if (!take(vs) || (t + LA < n && !take(ks))) { timed_out = true; break; }
        if (!own(t)) {
          if (leader) {
            umma_commit(empty + vs);
            if (ks >= 0) umma_commit(empty + ks);
          }
          __syncwarp();
          continue;
        }
        // V rows that no row of the item sees, or of unmapped pages: zero them
        // before the product reads them (both warps, where both do).
        const int j0 = q.it.tl.tile(q.u0 + t) * kTcTile;
        const uint32_t bad = p.paged ? bad_ring[(tiles + t) % kMaskRing] : 0u;
        const SeenRange& sr = q.it.sr;
        if (bad || !((j0 >= sr.lo && j0 + kTcTile <= sr.hi) || j0 + kTcTile <= sr.s_end)) {
#pragma unroll 1
          for (int r = lane; r < kTcTile; r += 32) {
            const int j = j0 + r;
            if ((j < sr.s_end || (j >= sr.lo && j < sr.hi)) && !((bad >> (r >> box)) & 1u)) continue;
            unsigned char* vr = smem + vs * C::SLOT + r * 128;
#pragma unroll
            for (int x = 0; x < C::HALVES * 8; ++x)
              *reinterpret_cast<uint4*>(vr + (x >> 3) * C::HALF + (x & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_proxy_async();
          __syncwarp();
        }
        if (mine == 0 && !wait(o_free + s, parts & 1)) { timed_out = true; break; }
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          if (!wait(p_full + 2 * s + half, tp & 1)) { timed_out = true; break; }
          tc_fence_after();
          if (leader) {
            const uint32_t vd = umma_desc_lo(smem_u32(smem + vs * C::SLOT) + half * kSub * 128, C::HALF);
            const unsigned ph = pa + kSub * half;
            // 16 tokens a product: 2048 bytes of V
            if (mine == 0 && half == 0) umma_ts<kIdPV, 0>(o, ph, vd);
            else umma_ts<kIdPV, 1>(o, ph, vd);
            umma_ts<kIdPV, 1>(o, ph + 8, vd + 128);
            umma_ts<kIdPV, 1>(o, ph + 32, vd + 256);
            umma_ts<kIdPV, 1>(o, ph + 40, vd + 384);
            umma_ts<kIdPV, 1>(o, ph + 16, vd);
            umma_ts<kIdPV, 1>(o, ph + 24, vd + 128);
            umma_ts<kIdPV, 1>(o, ph + 48, vd + 256);
            umma_ts<kIdPV, 1>(o, ph + 56, vd + 384);
            umma_commit(pv_done + 2 * s + half);
            if (ks >= 0) qk(half, ks);
            if (half) {
              umma_commit(empty + vs);
              if (ks >= 0) umma_commit(empty + ks);
            }
          }
          __syncwarp();
        }
        ++mine;
        ++tp;
      }
      tiles += n;
    }
    if (leader) umma_commit(done + s);  // after every product issued above
    __syncwarp();
    if (!mbar_wait(done + s, 0)) timed_out = true;
  } else {
    // ------------------------------------------- softmax, one row a thread
    const int s = warp >> 2, r = tid & 127;
    const unsigned taddr = tmem + ((unsigned)((warp & 3) * 32) << 16) + 128 * s, oaddr = taddr + 256 + (D - 128) * s;
    const float c = p.c_log2;
    bool dead = false;            // a wait of this thread gave up: skip the work, keep the barriers
    int ns = 0, tiles = 0;        // steps of this group done, tiles of the parts before
    auto wait = [&](uint64_t* bar, unsigned parity) {
      if (!__all_sync(0xffffffffu, !dead && mbar_wait(bar, parity))) dead = true;
      tc_fence_after();
      return !dead;
    };
    // A group without rows takes no part: it must not arrive at q_full, whose
    // phases nobody would wait for (nor, with NQ = 1, for a part without tiles).
    auto takes_part = [&](const Part& q) { return q.u1 > q.u0 && (NQ == 1 || s == 0 || q.it.rows > kTcTile); };
    // Queries of a part into shared memory, asynchronously: once S of the last
    // tile of the part before is there, its products no longer read them.  In the
    // one-row-block form both groups load half of the rows, when neither waits
    // for an S any more.
    auto load_queries = [&](const Part& q) {
      if (!takes_part(q)) return;
      if (NQ == 1) asm volatile("barrier.cta.sync 1, 256;\n" ::: "memory");
      constexpr int P16 = D / 8, kStep = NQ == 1 ? 256 : 128;  // 16-byte pieces of a row; threads
      const int first = q.it.row0 + (NQ == 1 ? 0 : s * kTcTile), rows_q = min(kTcTile, q.it.row0 + q.it.rows - first);
      const __nv_bfloat16* qb = static_cast<const __nv_bfloat16*>(p.q.data) + (int64_t)q.b * p.q.sb;
      const unsigned qs = smem_u32(smem + C::OFF_Q + (NQ == 1 ? 0 : s) * C::SLOT);
      const int cc = tid % P16;
#pragma unroll 4
      for (int rr = (NQ == 1 ? tid : r) / P16; rr < rows_q; rr += kStep / P16) {
        const int tok = row_token(p, first + rr);
        const __nv_bfloat16* src = qb + (int64_t)tok * p.q.sn + (int64_t)(q.g * p.G + first + rr - tok * p.G) * p.q.sh + 8 * cc;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(
                         qs + (cc >> 3) * C::HALF + rr * 128 + (((cc & 7) ^ (rr & 7)) << 4)),
                     "l"(src)
                     : "memory");
      }
    };
    auto queries_there = [&](const Part& q) {
      if (!takes_part(q)) return;
      asm volatile("cp.async.wait_all;" ::: "memory");
      fence_proxy_async();  // read by the tensor core
      if (NQ == 2) {
        mbar_arrive(q_full + s);
      } else {
        mbar_arrive(q_full);
        if (q.u1 - q.u0 > 1) mbar_arrive(q_full + 1);
      }
    };
    // Each turn does part q and gets the queries of the next; in the first turn q
    // is empty.  (One copy of the code for both: cold instructions cost more than
    // the empty turn.)
    q = Part();
    for (;;) {
      const int n = q.u1 - q.u0;
      const int row_s = q.it.row0 + (NQ == 2 ? s * kTcTile : 0), row = row_s + r;  // query row of the kv-head
      const bool valid = row < q.it.row0 + q.it.rows;
      const bool rows_here = __any_sync(0xffffffffu, valid);
      const int t = valid ? q.sq.len - q.sq.n + row_token(p, row) : -1;  // its position
      const int low = p.window < 0 ? -1 : t - p.window;                  // the window sees j > low
      // Tiles inside [all_lo, all_hi), or below both all_hi and the sinks' end, are
      // seen whole by every row of the group.
      const int last = min(row_s + kTcTile, q.it.row0 + q.it.rows) - 1;
      const int all_hi = q.sq.len - q.sq.n + row_token(p, row_s) + 1;
      const int all_lo = p.window < 0 ? 0 : q.sq.len - q.sq.n + row_token(p, max(last, 0)) - p.window + 1;
      float m = -CUDART_INF_F, l = 0.f;
      bool have = false;  // O holds something
      const bool group = NQ == 1 || s == 0 || q.it.rows > kTcTile;
#pragma unroll 1
      for (int i = NQ == 1 ? s : 0; i < n && group; i += NQ == 1 ? 2 : 1) {
        const int j0 = q.it.tl.tile(q.u0 + i) * kTcTile;
        wait(s_full + 2 * s, (ns >> 1) & 1);
        const uint32_t bad = p.paged ? bad_ring[(tiles + i) % kMaskRing] : 0u;
        const bool masked = bad || j0 + kTcTile > all_hi || (j0 < all_lo && j0 + kTcTile > p.sinks);
        float* zr = NQ == 1 && p.weigh && valid ? p.z + ((int64_t)(q.b * p.Hkv + q.g) * p.R + row) * p.z_row + j0 : nullptr;
#pragma unroll 1
        for (int k0 = 0; k0 < kTcTile; k0 += kSub) {
          const int half = k0 / kSub;
          if (half) wait(s_full + 2 * s + 1, (ns >> 1) & 1);
          if (rows_here && !dead) {
            // 64 columns of the row of S.  P = exp2(c z - m) goes over them:
            // columns [k, k + 16), k = 0 and 32, take hi of tokens k .. k + 31
            // and the next 16 lo.  A P past 2^64 shows in their sum,
            // so no maximum is formed unless the reference must be set or raised;
            // S is then read again.  Loops stay rolled and each piece of code
            // single: eleven warps run different code at once.
            float x[64];
            float (&xa)[32] = *reinterpret_cast<float (*)[32]>(x), (&xb)[32] = *reinterpret_cast<float (*)[32]>(x + 32);
            uint32_t hi[32];
            float sum;
            for (bool again = false;; again = true) {
              tmem_ld_start(taddr + k0, xa);
              tmem_ld_start(taddr + k0 + 32, xb);
              tmem_ld_wait(xa);
              tmem_ld_wait(xb);
              if (masked) {
                mask_cols(xa, seen_bits(j0 + k0, t, low, p.sinks, bad, k0, box));
                mask_cols(xb, seen_bits(j0 + k0 + 32, t, low, p.sinks, bad, k0 + 32, box));
              }
              if (again) {
                float top = x[0];
#pragma unroll
                for (int k = 1; k < kSub; ++k) top = fmaxf(top, x[k]);
                const float mn = fmaxf(m, top * c), f = m == -CUDART_INF_F ? 0.f : fexp2(m - mn);
                m = mn;
                l *= f;
                // O holds the products of this group's steps so far: rescale it
                // once the last of them is complete.
                if (have && wait(pv_done + 2 * s + ((ns - 1) & 1), ((ns - 1) >> 1) & 1)) {
#pragma unroll 1
                  for (int e = 0; e < D; e += 16) {
                    float o[16];
                    tmem_ld16(oaddr + e, o);
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] *= f;
                    tmem_st16(oaddr + e, o);
                  }
                }
              } else if (zr) {
#pragma unroll
                for (int k = 0; k < kSub; k += 4)
                  *reinterpret_cast<float4*>(zr + k0 + k) =
                      make_float4(x[k] * c, x[k + 1] * c, x[k + 2] * c, x[k + 3] * c);
              }
              const float mu = m == -CUDART_INF_F ? 0.f : m;
              const float2 c2 = make_float2(c, c), mu2 = make_float2(-mu, -mu);
              float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
              for (int k = 0; k < 32; ++k) {
                float2 e = fma2(make_float2(x[2 * k], x[2 * k + 1]), c2, mu2);
                e.x = fexp2(e.x);
                e.y = fexp2(e.y);
                if (k & 1) s1 = add2(s1, e);
                else s0 = add2(s0, e);
                hi[k] = pack_bf16(e.x, e.y);
                x[2 * k] = e.x;
                x[2 * k + 1] = e.y;
              }
              sum = (s0.x + s0.y) + (s1.x + s1.y);
              if (again || !__any_sync(0xffffffffu, valid && (m == -CUDART_INF_F || sum > kPMost))) break;
            }
            l += sum;
            tmem_st(taddr + k0, *reinterpret_cast<uint32_t (*)[16]>(hi));
            tmem_st(taddr + k0 + 32, *reinterpret_cast<uint32_t (*)[16]>(hi + 16));
            __syncwarp();  // no lo before the last hi is stored: both at once do not fit the registers
#pragma unroll
            for (int k = 0; k < 32; ++k) {
              float2 h;
              bf2(hi[k], h.x, h.y);
              const float2 d = add2(make_float2(x[2 * k], x[2 * k + 1]), make_float2(-h.x, -h.y));
              hi[k] = pack_bf16(d.x, d.y);
            }
            tmem_st(taddr + k0 + 16, *reinterpret_cast<uint32_t (*)[16]>(hi));
            tmem_st(taddr + k0 + 48, *reinterpret_cast<uint32_t (*)[16]>(hi + 16));
            tmem_st_wait();
          }
          have = true;
          ++ns;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full + 2 * s + half);
        }
      }
      tiles += max(0, n);
      Part next;
      const bool more = next_part(p, walk, next);
      if (more) load_queries(next);
      // ---- rows that see nothing: padding, or all of an item without tiles
      if (q.owner && (NQ == 2 || s == 0) && row < min(p.R, q.it.row0 + p.block) && (!valid || q.it.tl.n == 0)) {
        uint4* o = reinterpret_cast<uint4*>(out_row<__nv_bfloat16>(p, q.b, q.g, row));
#pragma unroll
        for (int k = 0; k < D / 8; ++k) o[k] = make_uint4(0u, 0u, 0u, 0u);
        store_lse(p, q.b, q.g, row, 0.f, 0.f);
      }
      // ---- the others' output, or this CTA's record of it
      const bool direct = NQ == 2 && !by_ticket(q.parts);
      const int c0 = q.c0;
      auto rec_of = [&](int c, int grp) { return record_of(c, c0) * 2 + grp; };
      if (have) wait(pv_done + 2 * s + ((ns - 1) & 1), ((ns - 1) >> 1) & 1);
      if (rows_here && n > 0 && group) {
        float* po = nullptr;
        __nv_bfloat16* out = nullptr;
        if (valid && direct) {
          out = out_row<__nv_bfloat16>(p, q.b, q.g, row);
          store_lse(p, q.b, q.g, row, m, l);
        } else if (valid) {
          const int64_t at = (int64_t)rec_of(blockIdx.x, s) * kTcTile + r;
          *reinterpret_cast<float2*>(p.part_st + 2 * at) = make_float2(m, l);
          po = p.part_o + at * D;
        }
        const float inv = l > 0.f ? 1.f / l : 0.f;
        __nv_bfloat16* outs[4];  // the rows of this lane's quad
#pragma unroll
        for (int x = 0; x < 4; ++x)
          outs[x] = reinterpret_cast<__nv_bfloat16*>(
              __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(out), (lane & ~3) + x));
#pragma unroll 1
        for (int k = 0; k < D; k += 32) {
          float o[32];
          if (have && !dead) {
            tmem_ld(oaddr + k, o);
          } else {
#pragma unroll
            for (int x = 0; x < 32; ++x) o[x] = 0.f;
          }
          if (po) {
#pragma unroll
            for (int x = 0; x < 32; x += 4)
              *reinterpret_cast<float4*>(po + k + x) = make_float4(o[x], o[x + 1], o[x + 2], o[x + 3]);
          }
          if (direct) {
            // A quad's lanes write 64 bytes of a row together.
            uint4 v[4];
#pragma unroll
            for (int x = 0; x < 4; ++x)
              v[x] = make_uint4(pack_bf16(o[8 * x] * inv, o[8 * x + 1] * inv), pack_bf16(o[8 * x + 2] * inv, o[8 * x + 3] * inv),
                                pack_bf16(o[8 * x + 4] * inv, o[8 * x + 5] * inv),
                                pack_bf16(o[8 * x + 6] * inv, o[8 * x + 7] * inv));
            quad_transpose(v, lane);
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (outs[x]) *reinterpret_cast<uint4*>(outs[x] + k + 8 * (lane & 3)) = v[x];
          }
        }
      }
      if (have) {
        tc_fence_before();
        mbar_arrive(o_free + s);
      }
      if (more) queries_there(next);
      // NQ = 1: the records of both groups of every CTA; NQ = 2: this group's rows.
      const int parts = q.parts;
      auto sync = [&] { asm volatile("barrier.cta.sync %0, 128;\n" ::"r"(2 + s) : "memory"); };
      // NQ = 1, an item of this CTA alone: its groups' records meet at a barrier
      // of the two, the first group joins them, and at a second one both know that
      // the records may be written again (for the CTA's next item).
      const bool meet = NQ == 1 && n > 0 && !by_ticket(parts);
      bool join = false;
      if (meet) {
        asm volatile("barrier.cta.sync 1, 256;\n" ::: "memory");
        join = s == 0;
      } else if (!direct && n > 0 && group) {
        join = last_to_arrive(p.tickets + 2 * c0 + (NQ == 2 ? s : 0), NQ == 1 ? 2 * parts : parts, r, misc + 18 + s, sync);
      }
      if (join) {
        if (NQ == 1)
          join_records<__nv_bfloat16, D, 128, 4, 4>(p, q.b, q.g, 0, q.it.rows, 2 * parts, kTcTile,
                                              [&](int k) { return rec_of(c0 + (k >> 1), k & 1); }, r);
        else
          join_records<__nv_bfloat16, D, 128, 4, 4>(p, q.b, q.g, row_s, min(kTcTile, q.it.rows - s * kTcTile), parts, kTcTile,
                                              [&](int k) { return rec_of(c0 + k, s); }, r);
      }
      if (meet) asm volatile("barrier.cta.sync 1, 256;\n" ::: "memory");
      if (!more) break;
      q = next;
    }
    if (dead) timed_out = true;
  }
  if (timed_out) err |= ERR_TIMEOUT;
  if (err) atomicOr(p.err, err);
  // Every copy has landed and every tensor-core operation is complete (warps 8
  // to 10 waited for them, bounded); free the columns.
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem) : "memory");
  }
}

template <int D, int NQ>
cudaError_t launch_tc_d(const AttendParams& p, cudaStream_t st) {
  return launch_dep(k_att_tc<D, NQ>, dim3(p.grid), kAttThreads, TcCfg2<D, NQ>::SMEM, st, p);
}

template <int D, int NQ>
cudaError_t set_tc_smem() {
  return cudaFuncSetAttribute(k_att_tc<D, NQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TcCfg2<D, NQ>::SMEM);
}

}  // namespace

cudaError_t configure_tc() {
  cudaError_t e = set_tc_smem<128, 1>();
  if (e == cudaSuccess) e = set_tc_smem<128, 2>();
  if (e == cudaSuccess) e = set_tc_smem<64, 1>();
  if (e == cudaSuccess) e = set_tc_smem<64, 2>();
  return e;
}

cudaError_t launch_tc(const AttendParams& p, cudaStream_t st) {
  if (p.kind == ATT_TC1) return p.D == 128 ? launch_tc_d<128, 1>(p, st) : launch_tc_d<64, 1>(p, st);
  return p.D == 128 ? launch_tc_d<128, 2>(p, st) : launch_tc_d<64, 2>(p, st);
}

}  // namespace vp
