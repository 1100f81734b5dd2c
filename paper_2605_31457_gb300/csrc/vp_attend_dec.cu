// k_att_dec: attention of one or a few new tokens over a long cache on the
// fifth-generation tensor cores (vp_attend_new, bf16, up to 64 query rows).
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
// k_att_dec<D, GM>: up to GM (8, 16, 32 or 64) query rows of a (sequence,
// kv-head), in three roles, two CTAs per SM (one from GM = 32 on):
//   warp 0     copies tiles of 128 K or V rows into a ring (4-D bulk-tensor
//              copies, 128-byte swizzle, evict-first in L2: each is read once);
//   warp 1     one lane issues tcgen05.mma with the cache as the M side, so
//              that few query rows do not leave the accumulators empty:
//              S = K Q^T (M = 128 tokens, N = query rows, K = D) and
//              O += V^T P^T (M = D, N = 2 GM, K = 128 tokens);
//   groups of four warps, one for every 16 query rows: a thread per token reads
//              its 16 columns of S, forms P and writes it, transposed, to shared
//              memory.
// P enters the product as two bf16 terms, P = hi + lo, in columns [0, GM) and
// [GM, 2 GM) of P^T; the two halves of O are added at the end.  P's rounding
// (2^-16 of it) then vanishes beside the output's, at no cost: the kernel is
// bound by HBM, 64 KB per tile at D = 128, and for few or short sequences by its
// start and end (about 10 us: the line's cut, the first tiles, the records and
// their join).  D = 128: 64 sequences of 17408 tokens, 32/8 heads, in 627 us (7.3
// TB/s); 16 of 2305 to 9001 tokens with five new tokens each in 68 us (5.4 TB/s);
// one of 3857 tokens, 28/4 heads, in 13.3 us.  With the queries as the M side and
// a join kernel of its own (k_att_tc's first form, which served these calls before)
// the first took 904 us against 639 and the last 28 us against 16.
//
// A row's reference is the largest logit of the first tile it sees and is raised
// only when a logit passes it by more than 64 (log2 units), when O and the sums
// are rescaled, so most tiles need no exchange between the threads; P <= 2^64
// has bf16's and float's full precision all the same.  The work is a line of
// tiles cut evenly over the CTAs (AttItem, LineCut): an item whose tiles lie with
// several CTAs leaves a record per CTA, and the last CTA to finish joins them.
//
// Rows of a tile that nobody sees may hold anything: their logits are masked,
// and their V rows are zeroed in shared memory before the product (0 x NaN is
// not 0); pages that hold only such rows are not copied at all.
// Waits are bounded: a thread whose wait gives up stops its work, still passes
// every barrier of its group, and the error word reports it.
// ---------------------------------------------------------------------------
constexpr float kDecRaise = 64.f;
constexpr int kBadRing = 16;  // more than the tiles between the copy warp and the others

template <int D, int GM>
struct DecCfg {
  static constexpr int HALF = kTcTile * 128;           // 128 rows x 64 dimensions, swizzled
  static constexpr int HALVES = D / 64;
  static constexpr int SLOT = HALVES * HALF;           // a tile of K or of V
  static constexpr int CPS = GM >= 32 ? 1 : 2;         // CTAs per SM
  static constexpr int S = GM == 64 ? (D == 128 ? 5 : 8) : (D == 128 ? 6 : 10) / CPS;  // ring slots
  static constexpr int GR = GM < 16 ? GM : 16;         // query rows of a softmax group
  static constexpr int SG = GM / GR;                   // softmax groups
  static constexpr int THREADS = 64 + 128 * SG;
  static constexpr int NQ = GM < 16 ? 16 : GM;         // query rows of the QK product
  static constexpr int NP = 2 * GM;                    // columns of P^T: hi, lo
  static constexpr int PB = GM == 8 ? 2 : 1;           // P buffers
  static constexpr int QHALF = NQ * 128;               // NQ rows x 64 dimensions
  static constexpr int PHALF = NP * 128;               // NP rows x 64 tokens
  static constexpr int PBUF = 2 * PHALF;
  static constexpr int OFF_Q = S * SLOT;
  static constexpr int OFF_P = OFF_Q + HALVES * QHALF;
  static constexpr int OFF_BAR = OFF_P + PB * PBUF;
  static constexpr int NBAR = 2 * S + 2 + 2 + PB + PB + 3;  // full, empty, s_full, s_free, p_full, pv_done, q_full, o_free, done
  static constexpr int OFF_BAD = OFF_BAR + NBAR * 8;   // unmapped boxes of a tile, one bit each
  static constexpr int LINE = THREADS / 32 + 7;        // ints of line_start
  static constexpr int OFF_MISC = OFF_BAD + kBadRing * 4;     // int: line_start, flags, TMEM base
  static constexpr int OFF_RED = OFF_MISC + (LINE + SG + 1) * 4;  // float [SG][5][GR]: maxima, then sums, of 4 warps; references
  static constexpr size_t SMEM = 1024 + (size_t)OFF_RED + 5 * GM * 4;
  static constexpr int O_COL = 2 * NQ;                 // TMEM columns: two S buffers, then O
  static constexpr int COLS = O_COL + NP <= 64 ? 64 : O_COL + NP <= 128 ? 128 : 256;
  static_assert(O_COL + NP <= COLS, "TMEM columns");
  static_assert(SMEM <= 232448 / CPS - (CPS > 1 ? 1024 : 0), "shared memory of the CTAs of an SM");
  static_assert(PHALF % 1024 == 0 && QHALF % 1024 == 0, "swizzle atoms stay aligned");
};

// Instruction descriptor: bf16 x bf16 -> f32; A K-major or (a_mn) MN-major, B K-major.
__host__ __device__ constexpr uint32_t dec_idesc(int m, int n, int a_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(m >> 4) << 24);
}

template <int D, int GM>
__global__ void __launch_bounds__(DecCfg<D, GM>::THREADS, DecCfg<D, GM>::CPS) k_att_dec(const __grid_constant__ AttendParams p) {
  using C = DecCfg<D, GM>;
  constexpr int S = C::S, PB = C::PB, GR = C::GR;
  constexpr uint32_t kIdQK = dec_idesc(128, C::NQ, 0), kIdPV = dec_idesc(D, C::NP, 1);
  extern __shared__ __align__(16) unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);  // [S] a slot's copies landed
  uint64_t* empty = full + S;                                        // [S] a slot's tile was read
  uint64_t* s_full = full + 2 * S;                                   // [2] S buffer written
  uint64_t* s_free = s_full + 2;                                     // [2] S buffer read (an arrival per softmax warp)
  uint64_t* p_full = s_full + 4;                                     // [PB] P buffer written (likewise)
  uint64_t* pv_done = p_full + PB;                                   // [PB] P.V of that buffer complete
  uint64_t* q_full = pv_done + PB;                                   // queries loaded (likewise)
  uint64_t* o_free = q_full + 1;                                     // O of the last part read (likewise)
  uint64_t* done = q_full + 2;                                       // every tensor-core operation complete
  volatile uint32_t* bad_ring = reinterpret_cast<uint32_t*>(smem + C::OFF_BAD);
  int* misc = reinterpret_cast<int*>(smem + C::OFF_MISC);            // [0, LINE) line_start; [LINE, LINE + SG) flags; then TMEM
  float* red = reinterpret_cast<float*>(smem + C::OFF_RED);

  if (tid == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + i, 1);
      mbar_init(s_free + i, 4 * C::SG);
    }
    for (int i = 0; i < PB; ++i) {
      mbar_init(p_full + i, 4 * C::SG);
      mbar_init(pv_done + i, 1);
    }
    mbar_init(q_full, 4 * C::SG);
    mbar_init(o_free, 4 * C::SG);
    mbar_init(done, 1);
    mbar_fence_init();
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&p.tmk)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&p.tmv)) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(misc + C::LINE + C::SG)),
                 "n"(C::COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  pdl_wait();
  pdl_trigger();
  tc_fence_before();
  Walk walk = line_start<C::THREADS>(p, misc);  // passes the CTA-wide barrier
  tc_fence_after();
  Part q;
  const unsigned tmem = (unsigned)misc[C::LINE + C::SG];
  const int R2 = p.paged ? min(kTcTile, p.page_size) : kTcTile;  // rows per copied box
  const int nb = kTcTile / R2;
  unsigned err = 0;
  bool timed_out = false;

  if (warp == 0) {
    // -------------------------------------------------------------- copies
    // Pieces in the order the tensor cores read them: K of tile i, then V of
    // tile i - 1.  Lane HALVES * x + hh copies half hh of box x.
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
        tma_load_4d(smem_u32(smem + sl * C::SLOT) + hh * C::HALF + x * R2 * 128, map, 64 * hh, crd(1), crd(2), crd(3),
                    full + sl);
      }
      ++pc;
      return true;
    };
    while (!timed_out && next_part(p, walk, q)) {
      const int n = q.u1 - q.u0;
      if (n <= 0) continue;
      int kp, vp, kn = -2, vn = -2, vd = -2;  // pages of tile i, of tile i + 1 (looked up ahead), V page due
      lookup(q, q.u0, kp, vp);
#pragma unroll 1
      for (int i = 0; i <= n; ++i) {
        if (i + 1 < n) lookup(q, q.u0 + i + 1, kn, vn);
        if (i < n) {
          const unsigned bad = __ballot_sync(0xffffffffu, kp == -1 && hh == 0);
          unsigned boxes = 0;  // bit of box x instead of lane HALVES * x
#pragma unroll
          for (int y = 0; y < 32 / C::HALVES; ++y) boxes |= ((bad >> (C::HALVES * y)) & 1u) << y;
          if (bad) err |= ERR_PAGE;
          if (lane == 0) bad_ring[tiles % kBadRing] = boxes;
          ++tiles;
          if (!issue(q, q.u0 + i, &p.tmk, kp)) { timed_out = true; break; }
        }
        if (i > 0 && !issue(q, q.u0 + i - 1, &p.tmv, vd)) { timed_out = true; break; }
        vd = vp;
        kp = kn;
        vp = vn;
      }
    }
    // Copies still in flight (only after a timeout can any be unread) land
    // before the CTA's shared memory is released.
#pragma unroll 1
    for (int k = max(0, pc - S); k < pc; ++k) mbar_wait(full + k % S, (k / S) & 1);
  } else if (warp == 1) {
    // -------------------------------------------------------- tensor cores
    // Tile i's QK is issued before tile i - 1's P.V, so that the softmax
    // threads find S(i) ready when they finish P(i - 1).
    auto wait_all = [&](uint64_t* bar, unsigned parity) {
      const bool ok = __all_sync(0xffffffffu, mbar_wait(bar, parity));
      tc_fence_after();
      return ok;
    };
    const int leader = elect_one();
    int pc = 0, parts = 0, ks = 0, ps = 0, tiles = 0;  // pieces, parts with tiles, QK and P.V products, tiles before
    while (!timed_out && next_part(p, walk, q)) {
      const int n = q.u1 - q.u0;
      if (n <= 0) continue;
      if (!wait_all(q_full, parts & 1)) { timed_out = true; break; }
#pragma unroll 1
      for (int i = 0; i <= n; ++i) {
        if (i < n) {
          const int sl = pc % S, sb = ks & 1;
          if (!wait_all(full + sl, (pc / S) & 1) || !wait_all(s_free + sb, ((ks >> 1) & 1) ^ 1)) {
            timed_out = true;
            break;
          }
          if (leader) {
            const uint32_t kd = umma_desc_lo(smem_u32(smem + sl * C::SLOT), 16);
            const uint32_t qd = umma_desc_lo(smem_u32(smem + C::OFF_Q), 16);
            umma_ss<kIdQK, 0>(tmem + C::NQ * sb, kd, qd);
#pragma unroll
            for (int k = 1; k < D / 16; ++k)  // 16 dimensions: 32 bytes, every fourth step the next half
              umma_ss<kIdQK, 1>(tmem + C::NQ * sb, kd + (k >> 2) * (C::HALF / 16) + (k & 3) * 2,
                                qd + (k >> 2) * (C::QHALF / 16) + (k & 3) * 2);
            umma_commit(s_full + sb);
            umma_commit(empty + sl);
          }
          __syncwarp();
          ++pc;
          ++ks;
        }
        if (i > 0) {
          const int sl = pc % S, pb = ps % PB;
          if (!wait_all(full + sl, (pc / S) & 1)) { timed_out = true; break; }
          // V rows that nobody sees, or of unmapped pages: zero them.
          const int j0 = q.it.tl.tile(q.u0 + i - 1) * kTcTile;
          const uint32_t bad = p.paged ? bad_ring[(tiles + i - 1) % kBadRing] : 0u;
          const SeenRange& sr = q.it.sr;
          if (bad || !((j0 >= sr.lo && j0 + kTcTile <= sr.hi) || j0 + kTcTile <= sr.s_end)) {
#pragma unroll 1
            for (int r = lane; r < kTcTile; r += 32) {
              const int j = j0 + r;
              if ((j < sr.s_end || (j >= sr.lo && j < sr.hi)) && !((bad >> (r / R2)) & 1u)) continue;
              unsigned char* vr = smem + sl * C::SLOT + r * 128;
#pragma unroll
              for (int k = 0; k < C::HALVES * 8; ++k)
                *reinterpret_cast<uint4*>(vr + (k >> 3) * C::HALF + (k & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            fence_proxy_async();
          }
          __syncwarp();
          if (i == 1 && !wait_all(o_free, (parts & 1) ^ 1)) { timed_out = true; break; }
          if (!wait_all(p_full + pb, (ps / PB) & 1)) { timed_out = true; break; }
          if (leader) {
            const uint32_t vd = umma_desc_lo(smem_u32(smem + sl * C::SLOT), C::HALF);
            const uint32_t pd = umma_desc_lo(smem_u32(smem + C::OFF_P + pb * C::PBUF), 16);
            if (i == 1) umma_ss<kIdPV, 0>(tmem + C::O_COL, vd, pd);
            else umma_ss<kIdPV, 1>(tmem + C::O_COL, vd, pd);
#pragma unroll
            for (int k = 1; k < kTcTile / 16; ++k)  // 16 tokens: 2048 bytes of V
              umma_ss<kIdPV, 1>(tmem + C::O_COL, vd + k * 128, pd + (k >> 2) * (C::PHALF / 16) + (k & 3) * 2);
            umma_commit(pv_done + pb);
            umma_commit(empty + sl);
          }
          __syncwarp();
          ++pc;
          ++ps;
        }
      }
      ++parts;
      tiles += n;
    }
    if (leader) umma_commit(done);  // after every operation issued above
    __syncwarp();
    if (!mbar_wait(done, 0)) timed_out = true;
  } else {
    // ------------------------------------------- softmax, one token a thread
    const int sg = C::SG == 1 ? 0 : (tid - 64) >> 7, wq = warp & 3;  // group; its warp's TMEM lanes are [32 wq, 32 wq + 32)
    const int r = wq * 32 + lane, st = (tid - 64) & 127;  // token row of a tile; index within the group
    const int h0 = sg * GR;                         // the group's query rows are [h0, h0 + GR)
    const unsigned taddr = tmem + ((unsigned)(wq * 32) << 16);
    const unsigned scol = taddr + h0, ocol = taddr + C::O_COL + h0;
    float* redg = red + sg * 5 * GR;
    const float c = p.c_log2;
    const int G = p.G;
    auto sync = [&] { asm volatile("barrier.cta.sync %0, 128;\n" ::"r"(1 + sg) : "memory"); };
    auto arrive = [&](uint64_t* bar) {  // for this warp
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    bool dead = false;  // a wait of this thread gave up: skip the work, keep the barriers
    auto wait = [&](uint64_t* bar, unsigned parity) {
      if (!__all_sync(0xffffffffu, !dead && mbar_wait(bar, parity))) dead = true;
      tc_fence_after();
      return !dead;
    };
    int ks = 0, tiles = 0;  // tiles done by this CTA, of the parts before
    while (next_part(p, walk, q)) {
      const int n = q.u1 - q.u0;
      const int rows = min(GR, max(0, q.it.rows - h0));  // of the group
      // ---- rows that see nothing: padding, or all of an item without tiles
      if (q.owner) {
        const int first = q.it.tl.n == 0 ? 0 : rows;
#pragma unroll 1
        for (int i = st; i < (min(GR, p.R - h0) - first) * (D / 8); i += 128) {
          const int row = h0 + first + i / (D / 8);
          reinterpret_cast<uint4*>(out_row<__nv_bfloat16>(p, q.b, q.g, row))[i % (D / 8)] = make_uint4(0u, 0u, 0u, 0u);
          if (i % (D / 8) == 0) store_lse(p, q.b, q.g, row, 0.f, 0.f);
        }
      }
      if (n <= 0) continue;
      // ---- the group's queries, K-major and swizzled.  The products with the
      // last part's are complete: this thread has waited for their S.
#pragma unroll 1
      for (int i = st; i < rows * (D / 8); i += 128) {
        const int rr = h0 + i / (D / 8), cc = i % (D / 8), tok = row_token(p, rr);
        const uint4 v = *reinterpret_cast<const uint4*>(
            static_cast<const __nv_bfloat16*>(p.q.data) + (int64_t)q.b * p.q.sb + (int64_t)tok * p.q.sn +
            (int64_t)(q.g * G + rr - tok * G) * p.q.sh + 8 * cc);
        *reinterpret_cast<uint4*>(smem + C::OFF_Q + (cc >> 3) * C::QHALF + rr * 128 + (((cc & 7) ^ (rr & 7)) << 4)) = v;
      }
      fence_proxy_async();  // read by the tensor core
      arrive(q_full);
      const int base = q.sq.len - q.sq.n;          // position of new token 0
      const int t0 = base + row_token(p, h0), t1 = base + row_token(p, h0 + max(0, rows - 1));  // of the group's rows
      float mref[GR], l[GR];
#pragma unroll
      for (int h = 0; h < GR; ++h) {
        mref[h] = -CUDART_INF_F;
        l[h] = 0.f;
      }
#pragma unroll 1
      for (int i = 0; i < n; ++i, ++ks) {
        const int sb = ks & 1, pb = ks % PB;
        const int j0 = q.it.tl.tile(q.u0 + i) * kTcTile, j = j0 + r;
        // Which rows see this thread's token, a bit each.
        uint32_t see = (1u << rows) - 1u;
        const bool part = j0 + kTcTile - 1 > t0 || !(p.window < 0 || j0 > t1 - p.window || j0 + kTcTile <= p.sinks);
        if (part) {
          uint32_t seen = 0;
#pragma unroll 1
          for (int h = 0; h < rows; ++h)
            if (sees(j, base + row_token(p, h0 + h), p.window, p.sinks)) seen |= 1u << h;
          see = seen;
        }
        float z[16];
        if (wait(s_full + sb, (ks >> 1) & 1) && rows > 0) {
          tmem_ld16(scol + C::NQ * sb, z);
        } else {
#pragma unroll
          for (int h = 0; h < 16; ++h) z[h] = 0.f;
        }
        tc_fence_before();
        arrive(s_free + sb);
        if (p.paged && ((bad_ring[(tiles + i) % kBadRing] >> (r / R2)) & 1u)) see = 0;
        if (p.weigh && !dead) {
          float* zr = p.z + ((int64_t)(q.b * p.Hkv + q.g) * p.R + h0) * p.z_row + j;
#pragma unroll
          for (int h = 0; h < GR; ++h)
            if (h < rows) zr[(int64_t)h * p.z_row] = (see >> h) & 1u ? z[h] * c : -CUDART_INF_F;
        }
        bool need = false;
#pragma unroll
        for (int h = 0; h < GR; ++h) {
          z[h] = (see >> h) & 1u ? z[h] * c : -CUDART_INF_F;
          need |= z[h] > mref[h] + kDecRaise;
        }
        int raise;
        asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 p, %1, 0;\n barrier.cta.red.or.pred q, %2, 128, p;\n selp.s32 %0, 1, 0, q;\n}\n"
                     : "=r"(raise) : "r"((int)need), "r"(1 + sg) : "memory");
        if (raise) {
#pragma unroll
          for (int h = 0; h < GR; ++h) {
            const float m = warp_max_now(z[h]);
            if (lane == 0) redg[wq * GR + h] = m;
          }
          sync();
          // O holds the products of this part's tiles so far: rescale it once
          // the last of them is complete.
          const bool fix = i > 0 && wait(pv_done + (ks - 1) % PB, ((ks - 1) / PB) & 1);
          float f[GR];
#pragma unroll
          for (int h = 0; h < GR; ++h) {
            const float mn = fmaxf(fmaxf(mref[h], fmaxf(redg[h], redg[GR + h])), fmaxf(redg[2 * GR + h], redg[3 * GR + h]));
            f[h] = mref[h] == -CUDART_INF_F ? 0.f : fexp2(mref[h] - mn);
            l[h] *= f[h];
            mref[h] = mn;
          }
          if (fix) {
#pragma unroll
            for (int k = 0; k < 2 * GR; k += 16) {  // GR = 8: hi and lo side by side
              float o[16];
              tmem_ld16(ocol + (k / GR) * GM, o);
#pragma unroll
              for (int h = 0; h < 16; ++h) o[h] *= f[h % GR];
              tmem_st16(ocol + (k / GR) * GM, o);
            }
          }
          sync();  // redg is read before its next use
        }
        if (ks >= PB && !dead) wait(pv_done + pb, ((ks / PB) & 1) ^ 1);  // P buffer free
        if (rows > 0) {
          unsigned char* pt = smem + C::OFF_P + pb * C::PBUF + (r >> 6) * C::PHALF + h0 * 128 + (r & 7) * 2;
#pragma unroll
          for (int h = 0; h < GR; ++h) {
            const float mu = mref[h] == -CUDART_INF_F ? 0.f : mref[h];
            const float pe = fexp2(z[h] - mu);
            l[h] += pe;
            const __nv_bfloat16 hi = __float2bfloat16_rn(pe), lo = __float2bfloat16_rn(pe - __bfloat162float(hi));
            const unsigned col = (((r & 63) >> 3) ^ (h & 7)) << 4;
            *reinterpret_cast<__nv_bfloat16*>(pt + h * 128 + col) = hi;
            *reinterpret_cast<__nv_bfloat16*>(pt + (GM + h) * 128 + col) = lo;
          }
        }
        fence_proxy_async();
        tc_fence_before();
        arrive(p_full + pb);
      }
      tiles += n;
      // ---- the rows' sums over the threads, then their output or this CTA's
      // record of it.  A thread holds dimension d of O.
      sync();
#pragma unroll
      for (int h = 0; h < GR; ++h) {
        const float s = warp_sum(l[h]);
        if (lane == 0) redg[wq * GR + h] = s;
      }
      // They go through the group's rows of a P buffer, which no product reads any
      // more, so that a thread writes 16 bytes: dimensions 32 x to 32 x + 31 of a
      // row take the 128 bytes of its hi (x < 2) or lo values of half x & 1.
      auto staged = [&](int h, int d) {
        return reinterpret_cast<float*>(smem + C::OFF_P + ((d >> 5) & 1) * C::PHALF + ((d >> 6) * GM + h0 + h) * 128 +
                                        (d & 31) * 4);
      };
      // D = 64: an M = 64 accumulator holds rows 16 w .. 16 w + 15 in the first
      // 16 lanes of warp w.
      const int dim = D == 128 ? r : 16 * wq + (lane & 15);
      if (st == 0) {
#pragma unroll
        for (int h = 0; h < GR; ++h) redg[4 * GR + h] = mref[h];
      }
      const bool there = wait(pv_done + (ks - 1) % PB, ((ks - 1) / PB) & 1);
      if (rows > 0) {
        float o[2 * GR];  // hi, lo
        if (there) {
#pragma unroll
          for (int k = 0; k < 2 * GR; k += 16) tmem_ld16(ocol + (k / GR) * GM, *reinterpret_cast<float (*)[16]>(o + k));
        } else {
#pragma unroll
          for (int k = 0; k < 2 * GR; ++k) o[k] = 0.f;
        }
        if (D == 128 || lane < 16) {
#pragma unroll
          for (int h = 0; h < GR; ++h) *staged(h, dim) = o[h] + o[GR + h];
        }
      }
      tc_fence_before();
      arrive(o_free);
      sync();
      if (rows <= 0) continue;
      const bool direct = !by_ticket(q.parts);
      const int c0 = q.c0;
      auto rec_of = [&](int cta) { return record_of(cta, c0) * C::SG + sg; };
#pragma unroll 1
      for (int i = st; i < rows * (D / 8); i += 128) {
        const int h = i / (D / 8), d = 8 * (i % (D / 8));
        const float sum = (redg[h] + redg[GR + h]) + (redg[2 * GR + h] + redg[3 * GR + h]);
        const float4 x = *reinterpret_cast<const float4*>(staged(h, d)), y = *reinterpret_cast<const float4*>(staged(h, d + 4));
        if (direct) {
          const float inv = sum > 0.f ? 1.f / sum : 0.f;
          *reinterpret_cast<uint4*>(out_row<__nv_bfloat16>(p, q.b, q.g, h0 + h) + d) =
              make_uint4(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv),
                         pack_bf16(y.x * inv, y.y * inv), pack_bf16(y.z * inv, y.w * inv));
          if (d == 0) store_lse(p, q.b, q.g, h0 + h, redg[4 * GR + h], sum);
        } else {
          const int at = rec_of(blockIdx.x) * GR + h;
          *reinterpret_cast<float4*>(p.part_o + at * D + d) = x;
          *reinterpret_cast<float4*>(p.part_o + at * D + d + 4) = y;
          if (d == 0) *reinterpret_cast<float2*>(p.part_st + 2 * at) = make_float2(redg[4 * GR + h], sum);
        }
      }
      if (direct) continue;
      if (last_to_arrive(p.tickets + c0 * C::SG + sg, q.parts, st, misc + C::LINE + sg, sync))
        join_records<__nv_bfloat16, D, 128, 1, 16>(p, q.b, q.g, h0, rows, q.parts, GR, [&](int k) { return rec_of(c0 + k); }, st);
    }
    if (dead) timed_out = true;
  }
  if (timed_out) err |= ERR_TIMEOUT;
  if (err) atomicOr(p.err, err);
  // Every copy has landed and every tensor-core operation is complete (warps 0
  // and 1 waited for them, bounded); free the columns.
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "n"(C::COLS) : "memory");
  }
}

template <int D, int GM>
cudaError_t launch_dec_d(const AttendParams& p, cudaStream_t st) {
  return launch_dep(k_att_dec<D, GM>, dim3(p.grid), DecCfg<D, GM>::THREADS, DecCfg<D, GM>::SMEM, st, p);
}

template <int D>
cudaError_t launch_dec_r(const AttendParams& p, cudaStream_t st) {
  if (p.R <= 8) return launch_dec_d<D, 8>(p, st);
  if (p.R <= 16) return launch_dec_d<D, 16>(p, st);
  if (p.R <= 32) return launch_dec_d<D, 32>(p, st);
  return launch_dec_d<D, 64>(p, st);
}

template <int D, int GM>
cudaError_t set_dec_smem() {
  return cudaFuncSetAttribute(k_att_dec<D, GM>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)DecCfg<D, GM>::SMEM);
}

}  // namespace

cudaError_t configure_dec() {
  cudaError_t e = set_dec_smem<128, 8>();
  if (e == cudaSuccess) e = set_dec_smem<128, 16>();
  if (e == cudaSuccess) e = set_dec_smem<128, 32>();
  if (e == cudaSuccess) e = set_dec_smem<128, 64>();
  if (e == cudaSuccess) e = set_dec_smem<64, 64>();
  if (e == cudaSuccess) e = set_dec_smem<64, 8>();
  if (e == cudaSuccess) e = set_dec_smem<64, 16>();
  if (e == cudaSuccess) e = set_dec_smem<64, 32>();
  return e;
}

cudaError_t launch_dec(const AttendParams& p, cudaStream_t st) {
  return p.D == 128 ? launch_dec_r<128>(p, st) : launch_dec_r<64>(p, st);
}

}  // namespace vp
