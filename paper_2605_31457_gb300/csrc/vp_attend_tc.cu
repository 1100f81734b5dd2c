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
// k_att_tc<D, NQ>: one CTA per SM, 320 threads in four roles.
//   warps 0-3, 4-7  two softmax groups, a thread per query row;
//   warp 8          copies tiles of 128 K or V rows into a ring (4-D bulk-tensor
//                   copies, 128-byte swizzle);
//   warp 9          one lane issues tcgen05.mma: S = Q K^T (M = 128 query rows,
//                   N = 128 tokens, K = D) and O += P V (M = 128, N = D, K =
//                   128 tokens) with P in TMEM.
// Query rows are the (new token, head of the kv-head) pairs, so a group of G
// heads shares every K and V row that is copied.  Each softmax group has its
// own S and O in TMEM (4 x 128 columns = all 512 at D = 128); P, rounded to
// bf16, overwrites S.  The groups take turns: while one turns its S into P the
// tensor cores work for the other.
//   NQ = 1 (decode, drafted tokens: at most 128 rows): both groups hold the
//          same queries and take alternate tiles; each writes its own partial.
//          Bound by HBM: 64 KB per tile at D = 128 against 0.25 us of tensor
//          work, which is why M = 128 may stand mostly empty at G = 7 rows.
//   NQ = 2 (prompts): the groups hold 128 query rows each and both read every
//          tile.  Bound by the tensor cores and, close behind, by the
//          exponentials: 128 x 128 of them per 2 x 128 x 128 x D MACs.
// The work is a line of tiles cut evenly over the CTAs (vp_attend.h): an item
// cut between CTAs leaves partials (m, l, O) that k_att_join merges.
//
// Softmax: a row's reference maximum is raised only when a logit passes it by
// more than 8 (log2 units), when O is rescaled in TMEM; P then stays below 2^8
// and the sums, in 32 bits, mean the same.  P is rounded to bf16 for the tensor
// cores (the caches are bf16 themselves); l sums the unrounded values.
//
// Rows of a tile that nobody sees may hold anything: their logits are masked,
// and their V rows are zeroed in shared memory before the product (0 x NaN is
// not 0); pages that hold only such rows are not copied at all.
//
// Waits are bounded: a role whose wait gives up stops working, still meets
// every barrier of its group, and the error word reports it.
// ---------------------------------------------------------------------------
constexpr int kAttThreads = 320;
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
  static constexpr int NBAR = 2 * S + 11;               // full, empty, s_full, p_full, pv_done, o_free, q_full, done
  static constexpr int OFF_BAD = OFF_BAR + NBAR * 8;    // unmapped boxes of a tile, one bit each
  static constexpr int OFF_MISC = OFF_BAD + kMaskRing * 4;  // int [16]: scan, start, TMEM base
  static constexpr size_t SMEM = 1024 + (size_t)OFF_MISC + 16 * 4;
  static_assert(SMEM <= 232448, "227 KB of shared memory");
  static_assert(S >= 2 * LA, "the K tiles ahead and a V tile fit the ring");
};

// Instruction descriptor: bf16 x bf16 -> f32, M = 128, N = n, A K-major, B
// K-major or (b_mn) MN-major.
__host__ __device__ constexpr uint32_t att_idesc(int n, int b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(128 >> 4) << 24);
}

template <int D, int NQ>
__global__ void __launch_bounds__(kAttThreads, 1) k_att_tc(const __grid_constant__ AttendParams p) {
  using C = TcCfg2<D, NQ>;
  constexpr int S = C::S, LA = C::LA;
  constexpr uint32_t kIdQK = att_idesc(128, 0), kIdPV = att_idesc(D, 1);
  extern __shared__ __align__(16) unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);  // [S] a slot's copies landed
  uint64_t* empty = full + S;                                        // [S] a slot's tile was read
  uint64_t* s_full = full + 2 * S;                                   // [2] S of a group written
  uint64_t* p_full = s_full + 2;                                     // [2] P written (128 arrivals)
  uint64_t* pv_done = s_full + 4;                                    // [2] P.V complete
  uint64_t* o_free = s_full + 6;                                     // [2] O of the last part read (128)
  uint64_t* q_full = s_full + 8;                                     // [2] queries loaded (128; NQ = 1: [0], 256)
  uint64_t* done = s_full + 10;                                      // every tensor-core operation complete
  volatile uint32_t* bad_ring = reinterpret_cast<uint32_t*>(smem + C::OFF_BAD);
  int* misc = reinterpret_cast<int*>(smem + C::OFF_MISC);            // [0..11] line_start; [12, 13] flags; [15] TMEM

  if (tid == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + i, 1);
      mbar_init(p_full + i, 128);
      mbar_init(pv_done + i, 1);
      mbar_init(o_free + i, 128);
      mbar_init(q_full + i, NQ == 1 ? 256 : 128);
    }
    mbar_init(done, 1);
    mbar_fence_init();
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&p.tmk)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&p.tmv)) : "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(misc + 15))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  pdl_wait();
  pdl_trigger();
  LineCut lc;
  tc_fence_before();
  Walk walk = line_start<kAttThreads>(p, misc, lc);  // passes the CTA-wide barrier
  tc_fence_after();
  Part q;
  const unsigned tmem = (unsigned)misc[15];  // columns [0, 128), [128, 256): S / P; from 256: O of the groups
  const int R2 = p.paged ? min(kTcTile, p.page_size) : kTcTile;  // rows per copied box
  const int nb = kTcTile / R2;
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
    for (int k = max(0, pc - S); k < pc; ++k) mbar_wait(full + k % S, (k / S) & 1);
  } else if (warp == 9) {
    // -------------------------------------------------------- tensor cores
    auto wait_all = [&](uint64_t* bar, unsigned parity) {
      const bool ok = __all_sync(0xffffffffu, mbar_wait(bar, parity));
      tc_fence_after();
      return ok;
    };
    int pc = 0, parts = 0, parts2 = 0;         // pieces; parts with tiles, of them with rows of the second group
    int np[2] = {0, 0}, no[2] = {0, 0};        // per group: P read, parts with tiles
    auto qk = [&](int s, int sl) {
      if (lane == 0) {
        const unsigned kb = smem_u32(smem + sl * C::SLOT), qb = smem_u32(smem + C::OFF_Q + (NQ == 1 ? 0 : s) * C::SLOT);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
          umma(tmem + 128 * s, umma_desc(qb + (ks >> 2) * C::HALF + (ks & 3) * 32, 16, 1024),
               umma_desc(kb + (ks >> 2) * C::HALF + (ks & 3) * 32, 16, 1024), kIdQK, ks > 0);
        umma_commit(s_full + s);
      }
      __syncwarp();
    };
    auto pv = [&](int s, int sl, bool first) {
      if (first && !wait_all(o_free + s, (no[s] & 1) ^ 1)) return false;
      if (first) ++no[s];
      if (!wait_all(p_full + s, np[s] & 1)) return false;
      ++np[s];
      if (lane == 0) {
        const unsigned vb = smem_u32(smem + sl * C::SLOT);
#pragma unroll
        for (int ks = 0; ks < kTcTile / 16; ++ks)
          umma_ts(tmem + 256 + D * s, tmem + 128 * s + 8 * ks, umma_desc(vb + ks * 2048, C::HALF, 1024), kIdPV,
                  !first || ks > 0);
#pragma unroll
        for (int ks = 0; ks < kTcTile / 16; ++ks)
          umma_ts(tmem + 256 + D * s, tmem + 128 * s + 64 + 8 * ks, umma_desc(vb + ks * 2048, C::HALF, 1024), kIdPV, true);
        umma_commit(pv_done + s);
      }
      __syncwarp();
      return true;
    };
    auto release = [&](int sl) {
      if (lane == 0) umma_commit(empty + sl);
      __syncwarp();
    };
    while (!timed_out && next_part(p, walk, q)) {
      const int n = q.u1 - q.u0;
      if (n <= 0) continue;
      const bool two = NQ == 2 && q.it.rows > kTcTile;  // the second group has rows
      if (!wait_all(q_full, parts & 1) || (two && !wait_all(q_full + 1, parts2 & 1))) { timed_out = true; break; }
      ++parts;
      parts2 += two;
      for (int i = 0; i < n + LA; ++i) {
        int vs = 0, ks = 0;
        if (i >= LA) {
          vs = pc % S;
          if (!wait_all(full + vs, (pc / S) & 1)) { timed_out = true; break; }
          ++pc;
          const int j = i - LA;
          if (!pv(NQ == 1 ? j & 1 : 0, vs, NQ == 1 ? j < 2 : j == 0)) { timed_out = true; break; }
          if (!two) release(vs);
        }
        if (i < n) {
          ks = pc % S;
          if (!wait_all(full + ks, (pc / S) & 1)) { timed_out = true; break; }
          ++pc;
          qk(NQ == 1 ? i & 1 : 0, ks);
          if (!two) release(ks);
        }
        if (two) {
          if (i >= LA) {
            if (!pv(1, vs, i == LA)) { timed_out = true; break; }
            release(vs);
          }
          if (i < n) {
            qk(1, ks);
            release(ks);
          }
        }
      }
    }
    if (lane == 0) umma_commit(done);  // after every operation issued above
    __syncwarp();
    if (!mbar_wait(done, 0)) timed_out = true;
  } else {
    // ------------------------------------------- softmax, one row a thread
    const int s = warp >> 2, r = tid & 127;
    const unsigned taddr = tmem + ((unsigned)((warp & 3) * 32) << 16) + 128 * s, oaddr = taddr + 256 + (D - 128) * s;
    const float c = p.c_log2;
    bool dead = false;            // a wait of this thread gave up: skip the work, keep the barriers
    int ns = 0, pc = 0, tiles = 0;  // S buffers of this group read; pieces and tiles of the parts before
    auto wait = [&](uint64_t* bar, unsigned parity) {
      if (!__all_sync(0xffffffffu, !dead && mbar_wait(bar, parity))) dead = true;
      tc_fence_after();
      return !dead;
    };
    while (next_part(p, walk, q)) {
      const int n = q.u1 - q.u0;
      const SeenRange sr = q.it.sr;
      const int row_s = q.it.row0 + (NQ == 2 ? s * kTcTile : 0), row = row_s + r;  // query row of the kv-head
      const bool valid = row < q.it.row0 + q.it.rows;
      const bool rows_here = __any_sync(0xffffffffu, valid);
      const int t = valid ? q.sq.len - q.sq.n + row / p.G : -1;      // its position
      const int low = p.window < 0 ? -1 : t - p.window;              // the window sees j > low
      float m = -CUDART_INF_F, l = 0.f;
      bool have = false;  // O holds something
      // A group without rows takes no part: it must not arrive at q_full, whose
      // phases nobody would wait for.
      const bool group = NQ == 1 || s == 0 || q.it.rows > kTcTile;
      if (n > 0 && group) {
        // Queries: in the one-row-block form both groups load half of the rows,
        // once neither reads the last part's S any more (its products with
        // the old queries are then complete).
        if (NQ == 1) asm volatile("barrier.cta.sync 1, 256;\n" ::: "memory");
        constexpr int P16 = D / 8;  // 16-byte pieces of a row
        const int rows_q = NQ == 1 ? q.it.rows : min(kTcTile, max(0, q.it.rows - s * kTcTile));
        const __nv_bfloat16* qb = static_cast<const __nv_bfloat16*>(p.q.data) + (int64_t)q.b * p.q.sb;
        unsigned char* qs = smem + C::OFF_Q + (NQ == 1 ? 0 : s) * C::SLOT;
        for (int i = NQ == 1 ? tid : r; i < rows_q * P16; i += NQ == 1 ? 256 : 128) {
          const int rr = i / P16, cc = i % P16, qrow = q.it.row0 + (NQ == 2 ? s * kTcTile : 0) + rr;
          const uint4 v = *reinterpret_cast<const uint4*>(qb + (int64_t)(qrow / p.G) * p.q.sn +
                                                          (int64_t)(q.g * p.G + qrow % p.G) * p.q.sh + 8 * cc);
          *reinterpret_cast<uint4*>(qs + (cc >> 3) * C::HALF + rr * 128 + (((cc & 7) ^ (rr & 7)) << 4)) = v;
        }
        fence_proxy_async();  // read by the tensor core
        mbar_arrive(q_full + (NQ == 1 ? 0 : s));
      }
      for (int i = NQ == 1 ? s : 0; i < n && group; i += NQ == 1 ? 2 : 1) {
        const int j0 = q.it.tl.tile(q.u0 + i) * kTcTile;
        wait(s_full + s, ns & 1);
        const uint32_t bad = bad_ring[(tiles + i) % kMaskRing];
        // Rows of the tile that no row of the item sees, or of unmapped pages:
        // zero their V before the product reads it.
        const bool clean = bad == 0 && ((j0 >= sr.lo && j0 + kTcTile <= sr.hi) || j0 + kTcTile <= sr.s_end);
        if (!clean && (NQ == 1 || s == 0)) {
          const int vp = pc + min(i + LA, n) + i, sl = vp % S;  // the tile's V among the pieces
          if (wait(full + sl, (vp / S) & 1)) {
            const int j = j0 + r;
            if (!(j < sr.s_end || (j >= sr.lo && j < sr.hi)) || ((bad >> (r / R2)) & 1u)) {
              unsigned char* vr = smem + sl * C::SLOT + r * 128;
#pragma unroll
              for (int k = 0; k < C::HALVES * 8; ++k)
                *reinterpret_cast<uint4*>(vr + (k >> 3) * C::HALF + (k & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            fence_proxy_async();
          }
        }
        if (rows_here && !dead) {
          float z[128];
          tmem_ld(taddr, z);
          const bool all = !valid || (bad == 0 && j0 + kTcTile - 1 <= t && (j0 > low || j0 + kTcTile <= p.sinks));
          if (!__all_sync(0xffffffffu, all)) {
#pragma unroll
            for (int k = 0; k < 128; ++k) {
              const int j = j0 + k;
              if (!(j <= t && (j > low || j < p.sinks))) z[k] = -CUDART_INF_F;
            }
            if (bad) {
#pragma unroll
              for (int k = 0; k < 128; ++k)
                if ((bad >> (k / R2)) & 1u) z[k] = -CUDART_INF_F;
            }
          }
          if (p.weigh && valid) {
            float4* zr = reinterpret_cast<float4*>(
                p.z + ((int64_t)(q.b * p.Hkv + q.g) * p.R + row) * p.z_row + j0);
#pragma unroll
            for (int k = 0; k < 32; ++k) zr[k] = make_float4(z[4 * k] * c, z[4 * k + 1] * c, z[4 * k + 2] * c, z[4 * k + 3] * c);
          }
          float mx = z[0];
#pragma unroll
          for (int k = 1; k < 128; ++k) mx = fmaxf(mx, z[k]);
          mx *= c;
          if (!have) {
            m = mx;
          } else if (__any_sync(0xffffffffu, valid && mx > m + 8.f)) {
            // O holds the products of this group's tiles so far: rescale it
            // once the last of them is complete.
            const float mn = fmaxf(m, mx), f = m == -CUDART_INF_F ? 0.f : fexp2(m - mn);
            m = mn;
            l *= f;
            if (wait(pv_done + s, (ns - 1) & 1)) {
#pragma unroll
              for (int k = 0; k < D; k += 32) {
                float o[32];
                tmem_ld(oaddr + k, o);
#pragma unroll
                for (int x = 0; x < 32; ++x) o[x] *= f;
                tmem_st(oaddr + k, o);
              }
              tmem_st_wait();
            }
          }
          const float mu = m == -CUDART_INF_F ? 0.f : m;
          float l0 = 0.f, l1 = 0.f;
#pragma unroll
          for (int k = 0; k < 128; k += 32) {
            uint32_t hi[16], lo[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) {
              const float a = fexp2(fmaf(z[k + 2 * x], c, -mu)), b = fexp2(fmaf(z[k + 2 * x + 1], c, -mu));
              l0 += a;
              l1 += b;
              hi[x] = pack_bf16(a, b);
              float ah, bh;
              bf2(hi[x], ah, bh);
              lo[x] = pack_bf16(a - ah, b - bh);
            }
            tmem_st(taddr + k / 2, hi);
            tmem_st(taddr + 64 + k / 2, lo);
          }
          l += l0 + l1;
          tmem_st_wait();
        }
        have = true;
        ++ns;
        tc_fence_before();
        mbar_arrive(p_full + s);
      }
      pc += 2 * max(0, n);
      tiles += max(0, n);
      // ---- rows that see nothing: padding, or all of an item without tiles
      if (q.owner && (NQ == 2 || s == 0) && row < min(p.R, q.it.row0 + p.block) && (!valid || q.it.tl.n == 0)) {
        uint4* o = reinterpret_cast<uint4*>(out_row<__nv_bfloat16>(p, q.b, q.g, row));
#pragma unroll
        for (int k = 0; k < D / 8; ++k) o[k] = make_uint4(0u, 0u, 0u, 0u);
        store_lse(p, q.b, q.g, row, 0.f, 0.f);
      }
      if (n <= 0 || !group) continue;
      // ---- the others' output, or this CTA's record of it
      const bool direct = NQ == 2 && q.whole();
      const int c0 = lc.owner(q.first);
      auto rec_of = [&](int c, int grp) { return (2 * c + (c == c0 ? 1 : 0)) * 2 + grp; };
      if (have) wait(pv_done + s, (ns - 1) & 1);
      if (rows_here) {
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
#pragma unroll
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
          if (out) {
#pragma unroll
            for (int x = 0; x < 32; x += 8) {
              uint4 v;
              v.x = pack_bf16(o[x] * inv, o[x + 1] * inv);
              v.y = pack_bf16(o[x + 2] * inv, o[x + 3] * inv);
              v.z = pack_bf16(o[x + 4] * inv, o[x + 5] * inv);
              v.w = pack_bf16(o[x + 6] * inv, o[x + 7] * inv);
              *reinterpret_cast<uint4*>(out + k + x) = v;
            }
          }
        }
      }
      if (have) {
        tc_fence_before();
        mbar_arrive(o_free + s);
      }
      if (direct) continue;
      // NQ = 1: the records of both groups of every CTA; NQ = 2: this group's rows.
      const int parts = lc.owner(q.first + q.it.tl.n - 1) - c0 + 1;
      auto sync = [&] { asm volatile("barrier.cta.sync %0, 128;\n" ::"r"(2 + s) : "memory"); };
      if (last_to_arrive(p.tickets + 2 * c0 + (NQ == 2 ? s : 0), NQ == 1 ? 2 * parts : parts, r, misc + 12 + s, sync)) {
        if (NQ == 1)
          join_records<__nv_bfloat16, D, 128>(p, q.b, q.g, 0, q.it.rows, 2 * parts, kTcTile,
                                              [&](int k) { return rec_of(c0 + (k >> 1), k & 1); }, r);
        else
          join_records<__nv_bfloat16, D, 128>(p, q.b, q.g, row_s, min(kTcTile, q.it.rows - s * kTcTile), parts, kTcTile,
                                              [&](int k) { return rec_of(c0 + k, s); }, r);
      }
    }
    if (dead) timed_out = true;
  }
  if (timed_out) err |= ERR_TIMEOUT;
  if (err) atomicOr(p.err, err);
  // Every copy has landed and every tensor-core operation is complete (warps 8
  // and 9 waited for them, bounded); free the columns.
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
