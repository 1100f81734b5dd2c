// k_att4: attention of newly appended tokens over a cache held in 4 bits
// (vp_attend4).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include <type_traits>

#include "vp_attend_device.h"
#include "vp_cache4.h"
#include "vp_codes4.h"
#include "vp_device.h"

namespace vp {
namespace {

// ---------------------------------------------------------------------------
// k_att4<T, D, NT>: up to 8 NT query rows of a (sequence, kv-head).  A warp takes
// 32 of the 128 tokens of a tile, with softmax statistics and an output of its
// own; the warps' are joined at the end of a CTA's part of an item.
//
// Codes are not turned into values one by one, but into the whole numbers code - 8
// in fp16, two at a time: a mask puts four bits into the mantissa of 1024, and one
// operation takes the 1032 off.  (Left in the mantissa of a subnormal number they
// would need no operation, but the tensor cores align a subnormal factor by its
// exponent field and lose up to ten bits of the sum.)  The products on the tensor
// cores (mma.sync):
//   S^T = K Q^T   (M = 16 tokens, N = 8 query rows, K = 16 dimensions): the sum of
//         a group of 32 dimensions is scaled by the token's scale in float;
//   O^T = V^T P^T (M = 16 dimensions, N = 8 rows, K = 16 tokens): the scale of the
//         group's dimensions, one a token, goes into P.
// The order of a group's dimensions within a product is that of the masks, four
// bits here and sixteen higher, so that no value is moved.
// A query row in fp16 is scaled by a power of two so that its largest magnitude
// lies in [2^13, 2^14): a bf16 number fits exactly (what is more than 2^30 times
// smaller than the row's largest is rounded), a float takes two terms.  P enters in
// one fp16 term for bf16 outputs: its rounding and that of its product with the
// scale are 2^-11 each of a term, an eighth of the output's own each.  Float
// outputs: two terms.
//
// P = exp2(z - reference).  The reference is 10 (log2 units) below the largest
// logit that raised it, and is raised when a logit is more than 14 above it, so
// P <= 2^14.  V's scales are taken in units, a power of two for each group of
// dimensions (and so is the group's output): a turn's scales lie within [2^-7, 2) of
// theirs, so that P * scale < 2^15, and below 2^-14, where fp16's step is fixed, only
// for a P more than 2^17 below the row's largest: 2^-28 of that at worst (a second
// term is held times 2^11: 2^-39).  Each lane puts one token's scales into their
// units, in the ring, where they are read eight times.  When a turn does not fit,
// units follow the largest scales, up or down; where a group's scales lie further
// apart than that, the turn is done again for those that were left out, until none is.
//
// Float outputs: the tensor cores cut what they add to a sum, so 16 tokens' products
// are summed by themselves and added in float; bf16 outputs, whose rounding is far
// larger, are summed in the accumulators (2^-24 of the sum per 16 tokens of a warp).
//
// Tokens that no row sees are not copied: the ring gets zeros for them, their scales
// among these, and their logits are masked.
//
// A warp's ring is filled by its own asynchronous copies, two or three turns ahead, so
// warps need no barrier until a part ends; a part's first copies run while the part
// before it is joined (where shared memory holds both: up to 16 rows of 128 dimensions).
// mma.sync takes its operands from registers, where the codes are converted.  For
// tcgen05 they would first be written to shared memory (512 bytes for every 144 that are
// read) or, K's, to tensor memory.  For 8 rows that is more than the products themselves;
// a form that converts each tile once for all of 9 to 128 rows has not been built, and
// this one converts it again for every 32.
//
// Bound by issue slots: 337 instructions of a warp for 16 tokens of K and V with 8
// rows, 144 of them the conversion, at 60% of the issue rate; at the measured copy rate
// an SM gets these tokens' bytes in the time of 390.
// Heads of 128, 32/8: 64 sequences of 17408 tokens in 247 us (5.2 TB/s); 16 of 2305 to
// 9001 with five new tokens in 53 us; 28/4: 32 of 2816 to 6400 in 29 us, one of 3857 in
// 9.7 us.  fp32: the first of these in 380 us.  Units of V's scales cost 7 instructions
// of those 337 (243, 51, 28 and 9.3 us without; scales put into them behind the logits
// instead of before, 255 us).  Slower, against 243: 16 tokens a turn and 8 warps a CTA (304 us), 16
// warps per SM at 128 registers (250), constants of the conversion left to the compiler,
// which loads them again for every use (348).  Two warps sharing 24 rows' registers,
// with two barriers a turn, took 68 us for the drafted tokens (then 55).
// ---------------------------------------------------------------------------
constexpr float kAbove4 = 10.f, kRaise4 = 4.f;
constexpr uint32_t kLeastUnit4 = 0x7800;  // 2^15, one over the least unit, in fp16
constexpr float kSecond4 = 2048.f;        // a second term is held times this
constexpr float kLowest4 = -3e38f;  // the reference of a row that has seen nothing
constexpr int kWarps4 = 4, kThreads4 = 32 * kWarps4;
constexpr int kStep4 = kTcTile / kWarps4;  // tokens of a warp's turn: a row's lane looks up its page

template <typename T, int D, int NT>
struct Cfg4 {
  static constexpr int TERMS = std::is_same<T, float>::value ? 2 : 1;
  static constexpr int GROUPS = D / kGroup4;
  static constexpr int CPS = NT * TERMS == 1 ? 3 : 2;   // CTAs per SM
  static constexpr int RS = 8 * NT;                     // query rows of an item
  static constexpr int CODES = kStep4 * D / 2;          // a stage: codes of a turn's tokens, then their scales, of K and of V
  static constexpr int SCALES = kStep4 * GROUPS * 2;
  static constexpr int STAGE = 2 * (CODES + SCALES);
  // Stages of a warp's ring (three also for 32 rows: 64 us against 67 with four and 74
  // with two; 24 rows: 51 with four, 55 with three).
  static constexpr int S = CPS == 3 || NT == 4 ? 3 : 4;
  // A warp's ring, and behind it its output to be joined, float [RS][D] (in the ring where there is no room).
  static constexpr int RING = S * STAGE;
  static constexpr int OUT = RS * D * 4;
  static constexpr bool APART = kWarps4 * (RING + OUT) <= 232448 / CPS - 4096 - NT * TERMS * GROUPS * 512;
  static constexpr int WARP = APART ? RING + OUT : RING > OUT ? RING : OUT;
  static constexpr int OFF_O = APART ? RING : 0;
  // The queries as the products take them: in registers, or uint4 [NT][TERMS][GROUPS][32] and float [RS] factors.
  static constexpr bool Q_REGS = NT * TERMS == 1;
  static constexpr int OFF_Q = kWarps4 * WARP;
  static constexpr int OFF_FAC = OFF_Q + (Q_REGS ? 0 : NT * TERMS * GROUPS * 512);
  static constexpr int OFF_ML = OFF_FAC + RS * 4;              // float2 [warps][RS]
  static constexpr int OFF_MASK = OFF_ML + kWarps4 * RS * 8;   // unsigned [warps][S]: tokens copied
  static constexpr int OFF_MISC = OFF_MASK + kWarps4 * S * 4;  // int: line_start, a flag
  static constexpr int LINE = kWarps4 + 7;
  static constexpr size_t SMEM = OFF_MISC + (LINE + 1) * 4;
  static_assert(SMEM <= 232448 / CPS - (CPS > 1 ? 1024 : 0), "shared memory of the CTAs of an SM");
  static_assert(STAGE % 128 == 0 && WARP % 128 == 0, "rows keep their banks");
  static_assert(2 * CPS * RS <= kPartRows && CPS <= kTickets, "two records and a ticket of a CTA");
};

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// D = A * B.
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                              uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// The transpose of an 8x8 matrix of 16-bit values held as two a lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t mul_f16(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// A group's unit from one over it (a power of two, the low or high half of a register).
__device__ __forceinline__ float unit_of(uint32_t one_over, int high) {
  const float2 x = unpack_f16(one_over);
  return __uint_as_float((254u << 23) - __float_as_uint(high ? x.y : x.x));
}
// A copy of N bytes, or N zeros.
template <int N>
__device__ __forceinline__ void cp_async_or_zero(unsigned dst, const void* src, bool copy) {
  const int n = copy ? N : 0;
  if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(n) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;\n" ::"r"(dst), "l"(src), "r"(n), "n"(N) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }

// Byte offset of 16-byte chunk `ch` of token `row` in a stage's codes: the chunks
// are exchanged so that eight rows' same chunk lies in different banks.
template <int D>
__device__ __forceinline__ int code_at(int row, int ch) {
  return D == 128 ? row * 64 + ((ch ^ ((row >> 1) & 3)) << 4) : row * 32 + ((ch ^ ((row >> 2) & 1)) << 4);
}

// True for the CTA that is the last of `expected` to arrive at the ticket, its record
// written.  One atomic operation releases that record and acquires the others', for
// the whole CTA by way of the barriers around it.
__device__ __forceinline__ bool last_of(unsigned* ticket, unsigned expected, int tid, int* flag) {
  __syncthreads();
  if (tid == 0) {
    unsigned before;
    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;\n" : "=r"(before) : "l"(ticket) : "memory");
    const bool last = before == expected - 1;
    if (last) *ticket = 0;  // for the next call
    *flag = last;
  }
  __syncthreads();
  return *flag != 0;
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kThreads4, Cfg4<T, D, NT>::CPS) k_att4(const __grid_constant__ Attend4Params p) {
  using C = Cfg4<T, D, NT>;
  constexpr int S = C::S, NG = C::GROUPS, TERMS = C::TERMS, RS = C::RS;
  extern __shared__ __align__(128) unsigned char smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int r = lane >> 2, c = lane & 3;
  float2* ml_all = reinterpret_cast<float2*>(smem + C::OFF_ML);
  unsigned* masks = reinterpret_cast<unsigned*>(smem + C::OFF_MASK) + warp * S;
  int* misc = reinterpret_cast<int*>(smem + C::OFF_MISC);
  unsigned char* const mine = smem + warp * C::WARP;
  const unsigned ring = smem_u32(mine);
  pdl_wait();
  pdl_trigger();
  Walk walk = line_start<kThreads4>(p, misc);
  Part q;
  unsigned err = 0;
  const Codes codes;

  // Addresses of this lane's matrix rows within a stage (ldmatrix: lane l gives
  // row l % 8 of matrix l / 8; matrices: tokens 0-7 and 8-15 of one group, then
  // of the next).
  const int m_off = code_at<D>((lane & 7) + ((lane >> 3) & 1) * 8, lane >> 4);  // of groups 0 and 1
  // Copies: 16-byte chunks of a row of codes, rows copied at once, this lane's.
  constexpr int CH = D / 32, ROWS = 32 / CH;
  const int crow = lane / CH, cch = lane % CH;
  const unsigned c_to = ring + code_at<D>(crow, cch);  // ROWS further rows have their chunks exchanged alike
  const unsigned s_to = ring + 2 * C::CODES + lane * 2 * NG;
  // Token and page strides are below 2^31 (vp_attend4 checks them).
  const int kt = (int)p.k4.ct, vt = (int)p.v4.ct, kst = (int)p.k4.st, vst = (int)p.v4.st;
  const int kpage = (int)p.k4.cb, vpage = (int)p.v4.cb, kspage = (int)p.k4.sb, vspage = (int)p.v4.sb;
  const int in_page = p.paged ? p.page_size - 1 : -1;
  const bool dense = kt == D / 2 && vt == D / 2;  // a token's codes lie next to the next one's

  uint4* const q_smem = reinterpret_cast<uint4*>(smem + C::OFF_Q) + lane;
  float* const fac_smem = reinterpret_cast<float*>(smem + C::OFF_FAC);
  // The part whose output is still to be joined.
  int d_b = 0, d_g = 0, d_row0 = 0, d_rows = 0, d_c0 = 0, d_parts = 0;

  for (bool more = true; more;) {
    more = next_part(p, walk, q);
    const int rows = more ? q.it.rows : 0;
    if (!more) q.u0 = q.u1 = 0;
    const int n = q.u1 - q.u0;
    // ---- rows that see nothing: padding, or all of an item without tiles
    if (more && q.owner) {
      const int first = q.it.tl.n == 0 ? 0 : rows;
#pragma unroll 1
      for (int i = tid; i < (min(p.block, p.R - q.it.row0) - first) * (D / 4); i += kThreads4) {
        const int row = q.it.row0 + first + i / (D / 4);
        store4(out_row<T>(p, q.b, q.g, row) + 4 * (i % (D / 4)), make_float4(0.f, 0.f, 0.f, 0.f));
        if (i % (D / 4) == 0) store_lse(p, q.b, q.g, row, 0.f, 0.f);
      }
    }
    if (more && n <= 0) continue;
    const SeenRange& sr = q.it.sr;
    auto first_token = [&](int u) { return q.it.tl.tile(u) * kTcTile + kStep4 * warp; };

    // ---- copies of the warp's 32 tokens of tile u, into stage u % S
    const unsigned char* k_lane = p.k4.codes + q.g * p.k4.ch + (int64_t)crow * kt + 16 * cch;
    const unsigned char* v_lane = p.v4.codes + q.g * p.v4.ch + (int64_t)crow * vt + 16 * cch;
    const uint16_t *ks_lane = p.k4.scales + q.g * p.k4.sh, *vs_lane = p.v4.scales + q.g * p.v4.sh;
    if (!p.paged) {
      k_lane += q.b * p.k4.cb;
      v_lane += q.b * p.v4.cb;
      ks_lane += q.b * p.k4.sb;
      vs_lane += q.b * p.v4.sb;
    }
    int kn = 0, vn = 0;   // page ids of the next turn to be copied
    unsigned partly = 0;  // bit of a stage: masks has which of its tokens were copied; else all of them
    auto lookup = [&](int u) {  // page ids of token `lane` of tile u
      if (!p.paged || u >= q.u1) return;
      const int lp = (first_token(u) + lane) >> p.page_shift;
      kn = lp < p.k4.max_pages ? __ldg(p.k4.block_table + (int64_t)q.b * p.k4.max_pages + lp) : -1;
      vn = lp < p.v4.max_pages ? __ldg(p.v4.block_table + (int64_t)q.b * p.v4.max_pages + lp) : -1;
    };
    auto issue = [&](int u) {
      if (u < q.u1) {
        const int st = (unsigned)(u - q.u0) % S;
        const unsigned to = c_to + st * C::STAGE, s_st = s_to + st * C::STAGE;
        const int j0 = first_token(u), j = j0 + lane;
        const bool whole = (j0 >= sr.lo && j0 + kStep4 <= sr.hi) || j0 + kStep4 <= sr.s_end;
        unsigned mask = 0xffffffffu;
        if (!whole || p.paged) {
          const bool ok = !p.paged || ((unsigned)kn < (unsigned)p.k4.num_pages && (unsigned)vn < (unsigned)p.v4.num_pages);
          bool live = j < sr.s_end || (j >= sr.lo && j < sr.hi);
          if (live && !ok) err |= ERR_PAGE;
          live = live && ok;
          mask = __ballot_sync(0xffffffffu, live);
        }
        if (whole && !p.paged) {
          partly &= ~(1u << st);
          const unsigned char *kc = k_lane + (int64_t)j0 * kt, *vc = v_lane + (int64_t)j0 * vt;
          if (dense) {
#pragma unroll
            for (int i = 0; i < kStep4; i += ROWS) {
              cp_async16(to + i * (D / 2), kc + i * (D / 2));
              cp_async16(to + C::CODES + i * (D / 2), vc + i * (D / 2));
            }
          } else {
#pragma unroll
            for (int i = 0; i < kStep4; i += ROWS) {
              cp_async16(to + i * (D / 2), kc + (int64_t)i * kt);
              cp_async16(to + C::CODES + i * (D / 2), vc + (int64_t)i * vt);
            }
          }
          cp_async_or_zero<2 * NG>(s_st, ks_lane + (int64_t)j * kst, true);
          cp_async_or_zero<2 * NG>(s_st + C::SCALES, vs_lane + (int64_t)j * vst, true);
        } else if (mask == 0xffffffffu && p.page_size >= 16) {
          partly &= ~(1u << st);
#pragma unroll
          for (int h = 0; h < kStep4; h += 16) {
            const int at = (j0 + h) & in_page;
            const unsigned char* kc = k_lane + (int64_t)__shfl_sync(0xffffffffu, kn, h) * kpage + (int64_t)at * kt;
            const unsigned char* vc = v_lane + (int64_t)__shfl_sync(0xffffffffu, vn, h) * vpage + (int64_t)at * vt;
#pragma unroll
            for (int i = 0; i < 16; i += ROWS) {
              cp_async16(to + (h + i) * (D / 2), kc + (dense ? (int64_t)(i * (D / 2)) : (int64_t)i * kt));
              cp_async16(to + C::CODES + (h + i) * (D / 2), vc + (dense ? (int64_t)(i * (D / 2)) : (int64_t)i * vt));
            }
          }
          const int at = j & in_page;
          cp_async_or_zero<2 * NG>(s_st, ks_lane + (int64_t)kn * kspage + (int64_t)at * kst, true);
          cp_async_or_zero<2 * NG>(s_st + C::SCALES, vs_lane + (int64_t)vn * vspage + (int64_t)at * vst, true);
        } else {
          // A row's page is known to its lane.  A token that is not copied leaves
          // zeros, its scale's among them.
          partly |= 1u << st;
          if (lane == 0) masks[st] = mask;
#pragma unroll 1
          for (int i = 0; i < kStep4; i += ROWS) {
            const int row = crow + i;
            const int kr = __shfl_sync(0xffffffffu, kn, row), vr = __shfl_sync(0xffffffffu, vn, row);
            const bool copy = (mask >> row) & 1u;
            const int64_t at = ((j0 + row) & in_page) - crow;  // k_lane is of row crow
            cp_async_or_zero<16>(to + i * (D / 2), copy ? k_lane + (int64_t)kr * kpage + at * kt : p.k4.codes, copy);
            cp_async_or_zero<16>(to + C::CODES + i * (D / 2), copy ? v_lane + (int64_t)vr * vpage + at * vt : p.v4.codes, copy);
          }
          const bool live = (mask >> lane) & 1u;
          const int64_t at = j & in_page;
          cp_async_or_zero<2 * NG>(s_st, live ? ks_lane + (int64_t)kn * kspage + at * kst : p.k4.scales, live);
          cp_async_or_zero<2 * NG>(s_st + C::SCALES, live ? vs_lane + (int64_t)vn * vspage + at * vst : p.v4.scales, live);
        }
        lookup(u + 1);
      }
      cp_async_commit();
    };
    auto begin = [&] {
      lookup(q.u0);
#pragma unroll 1
      for (int v = 0; v < S - 1; ++v) issue(q.u0 + v);
    };
    // The first copies are on their way while the last part's output is joined
    // (unless that lies in the ring).
    if (C::APART && more) begin();
    if (d_parts > 0) {
      // ---- the warps' outputs become rows of out or a record
      __syncthreads();
      const bool direct = !by_ticket(d_parts);
      const int rec = record_of(blockIdx.x, d_c0) * RS;
#pragma unroll 1
      for (int i = tid; i < d_rows * (D / 4); i += kThreads4) {
        const int row = i / (D / 4), d = 4 * (i % (D / 4));
        float m = -CUDART_INF_F;
#pragma unroll
        for (int w = 0; w < kWarps4; ++w) m = fmaxf(m, ml_all[w * RS + row].x);
        const float mu = m == -CUDART_INF_F ? 0.f : m;
        float sum = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps4; ++w) {
          const float2 st = ml_all[w * RS + row];
          const float f = exp2f(st.x - mu);
          const float4 y = *reinterpret_cast<const float4*>(smem + w * C::WARP + C::OFF_O + 4 * (row * D + d));
          sum = fmaf(st.y, f, sum);
          x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w);
        }
        if (direct) {
          const float inv = sum > 0.f ? 1.f / sum : 0.f;
          store4(out_row<T>(p, d_b, d_g, d_row0 + row) + d, make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv));
          if (d == 0) store_lse(p, d_b, d_g, d_row0 + row, m, sum);
        } else {
          *reinterpret_cast<float4*>(p.part_o + (int64_t)(rec + row) * D + d) = x;
          if (d == 0) *reinterpret_cast<float2*>(p.part_st + 2 * (rec + row)) = make_float2(m, sum);
        }
      }
      if (direct) __syncthreads();  // the outputs are read before their next use
      else if (last_of(p.tickets + d_c0, d_parts, tid, misc + C::LINE))
        join_records<T, D, kThreads4, NT == 1 ? 2 : 4, 8>(p, d_b, d_g, d_row0, d_rows, d_parts, RS,
                                             [&](int k) { return record_of(d_c0 + k, d_c0); }, tid);
    }
    if (!more) break;
    if (!C::APART) begin();
    // ---- queries: 8 dimensions of each group a lane, in the order of the codes
    uint4 q_regs[C::Q_REGS ? NG : 1] = {};
    float fac[NT][2];
    int tq[NT][2];
    const int base = q.sq.len - q.sq.n;
#pragma unroll 1
    for (int t = C::Q_REGS ? 0 : warp; t < NT; t += kWarps4) {  // a warp of the CTA does a tile of 8 rows for all of them
      const int row = 8 * t + r;
      float x[NG][8];
      float top = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[g][e] = 0.f;
        if (row < rows) {
          const int tok = row_token(p, q.it.row0 + row);
          const T* src = static_cast<const T*>(p.q.data) + (int64_t)q.b * p.q.sb + (int64_t)tok * p.q.sn +
                         (int64_t)(q.g * p.G + q.it.row0 + row - tok * p.G) * p.q.sh + 32 * g + 8 * c;
          if constexpr (TERMS == 1) {
            const uint4 v = __ldcg(reinterpret_cast<const uint4*>(src));
            bf2(v.x, x[g][0], x[g][1]); bf2(v.y, x[g][2], x[g][3]); bf2(v.z, x[g][4], x[g][5]); bf2(v.w, x[g][6], x[g][7]);
          } else {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(src)), w = __ldcg(reinterpret_cast<const float4*>(src) + 1);
            x[g][0] = v.x; x[g][1] = v.y; x[g][2] = v.z; x[g][3] = v.w;
            x[g][4] = w.x; x[g][5] = w.y; x[g][6] = w.z; x[g][7] = w.w;
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[g][e]));
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // 2^k and 2^-k, the largest magnitude times 2^k in [2^13, 2^14)
      const int field = min(267 - (int)(__float_as_uint(top) >> 23), 253);
      const float up = __uint_as_float((unsigned)field << 23), down = __uint_as_float((unsigned)(254 - field) << 23);
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {  // dimensions k and k + 4 meet one mask
          const float a = x[g][k] * up, b = x[g][k + 4] * up;
          hi[k] = pack_f16(a, b);
          const float2 h = unpack_f16(hi[k]);
          lo[k] = pack_f16(a - h.x, b - h.y);
        }
        if constexpr (C::Q_REGS) {
          q_regs[g] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        } else {
          q_smem[(t * TERMS * NG + g) * 32] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          if constexpr (TERMS == 2) q_smem[(t * TERMS * NG + NG + g) * 32] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
      }
      const float f = fmaxf(down * p.c_log2, 1e-37f);  // above 0: masked logits are multiplied by it
      if constexpr (C::Q_REGS) {
        fac[0][0] = __shfl_sync(0xffffffffu, f, 8 * c);
        fac[0][1] = __shfl_sync(0xffffffffu, f, 8 * c + 4);
      } else if (c == 0) {
        fac_smem[row] = f;
      }
    }
    if constexpr (!C::Q_REGS) __syncthreads();  // (the last part's were read before the barrier behind it)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if constexpr (!C::Q_REGS) fac[t][k] = fac_smem[8 * t + 2 * c + k];
        tq[t][k] = base + row_token(p, q.it.row0 + min(8 * t + 2 * c + k, rows - 1));
      }
    const int t0 = base + row_token(p, q.it.row0);
    const int t1 = base + row_token(p, q.it.row0 + rows - 1);
    auto query = [&](int t, int m, int g) {
      if constexpr (C::Q_REGS) return q_regs[g];
      else return q_smem[((t * TERMS + m) * NG + g) * 32];
    };

    float o[NT][NG][2][4], ref[NT][2], l[NT][2];
    // One over the groups' units, two of them in a register; what is left of the turn's
    // scales, this lane's token's, when it is done again.
    uint32_t one_over[NG / 2], left[NG / 2];
    bool again = false;
#pragma unroll
    for (int m = 0; m < NG / 2; ++m) {
      one_over[m] = 0x3c003c00;
      left[m] = 0;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      ref[t][0] = ref[t][1] = kLowest4;
      l[t][0] = l[t][1] = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < 4; ++k) o[t][g][h][k] = 0.f;
    }

#pragma unroll 1
    for (int u = q.u0; u < q.u1; u += again ? 0 : 1) {
      const bool repeat = again;
      again = false;
      cp_async_wait<S - 2>();
      __syncwarp();
      if (!repeat) issue(u + S - 1);  // into the stage that the last turn read
      const int st = (unsigned)(u - q.u0) % S;
      const unsigned turn = (partly >> st) & 1u ? masks[st] : 0xffffffffu;
      const int jt = first_token(u);
      const bool all_see = turn == 0xffffffffu && jt + kStep4 - 1 <= t0 &&
                           (p.window < 0 || jt > t1 - p.window || jt + kStep4 <= p.sinks);
      const unsigned at = ring + st * C::STAGE;
      unsigned char* const scales = mine + st * C::STAGE + 2 * C::CODES;

      // ---- V's scales of token `lane`, in their units
      uint32_t* const of_mine = reinterpret_cast<uint32_t*>(scales + C::SCALES + lane * 2 * NG);
      uint32_t held[NG / 2], out_of = 0;
#pragma unroll
      for (int m = 0; m < NG / 2; ++m) held[m] = repeat ? left[m] : of_mine[m];
#pragma unroll
      for (int m = 0; m < NG / 2; ++m) {
        const uint32_t in_units = mul_f16(held[m], one_over[m]);
        of_mine[m] = in_units;
        out_of |= in_units ^ 0x20002000;
      }
      const bool off = (out_of & 0x60006000) != 0;  // an exponent is not one of 2^-7 to 2^0

      // ---- logits, over the row's factor: tokens r and r + 8 of each half, query rows 2c and 2c + 1
      float z[2][NT][4];
      uint32_t kscale[2][2][NG / 2];  // half, tokens: two groups' scales each
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const unsigned char* const of = scales + (16 * h + 8 * k + r) * 2 * NG;
          if constexpr (NG == 4) {
            const uint2 v = *reinterpret_cast<const uint2*>(of);
            kscale[h][k][0] = v.x;
            kscale[h][k][1] = v.y;
          } else {
            kscale[h][k][0] = *reinterpret_cast<const uint32_t*>(of);
          }
        }
#pragma unroll
      for (int gp = 0; gp < NG; gp += 2) {
        uint32_t kw[2][2][2];  // half, group, tokens 0-7 or 8-15
        float2 ks[2][2];       // half, tokens: the two groups' scales
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          ldsm_x4(at + (m_off ^ (16 * gp)) + 8 * D * h, kw[h][0][0], kw[h][0][1], kw[h][1][0], kw[h][1][1]);
#pragma unroll
          for (int k = 0; k < 2; ++k)
            ks[h][k] = unpack_f16(kscale[h][k][gp / 2]);
        }
#pragma unroll
        for (int gg = 0; gg < 2; ++gg) {
          const int g = gp + gg;
          uint32_t a[2][8];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const uint32_t x = kw[h][gg][k], y = x >> 8;
              a[h][k] = codes.low(x);
              a[h][2 + k] = codes.high(x);
              a[h][4 + k] = codes.low(y);
              a[h][6 + k] = codes.high(y);
            }
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const uint4 b = query(t, 0, g);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float s[4];
              mma_f16_first(s, a[h][0], a[h][1], a[h][2], a[h][3], b.x, b.y);
              mma_f16(s, a[h][4], a[h][5], a[h][6], a[h][7], b.z, b.w);
              if constexpr (TERMS == 2) {
                const uint4 d = query(t, TERMS - 1, g);
                mma_f16(s, a[h][0], a[h][1], a[h][2], a[h][3], d.x, d.y);
                mma_f16(s, a[h][4], a[h][5], a[h][6], a[h][7], d.z, d.w);
              }
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float step = gg ? ks[h][k >> 1].y : ks[h][k >> 1].x;
                z[h][t][k] = g == 0 ? s[k] * step : fmaf(s[k], step, z[h][t][k]);
              }
            }
          }
        }
      }
      if (!all_see) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int row = 16 * h + r + 8 * (k >> 1);
              if (!((turn >> row) & 1u) || !sees(jt + row, tq[t][k & 1], p.window, p.sinks)) z[h][t][k] = -CUDART_INF_F;
            }
      }

      // ---- the references and units
      bool need = false;
      auto largest = [&](int t, int k) { return fmaxf(fmaxf(z[0][t][k], z[0][t][2 + k]), fmaxf(z[1][t][k], z[1][t][2 + k])); };
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int k = 0; k < 2; ++k) need |= fmaf(largest(t, k), fac[t][k], -ref[t][k]) > kAbove4 + kRaise4;
      if (__any_sync(0xffffffffu, need || off)) {
        float change[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) change[g] = 1.f;
        if (__any_sync(0xffffffffu, off)) {
          uint32_t rest = 0;
#pragma unroll
          for (int m = 0; m < NG / 2; ++m) {
            uint32_t next = one_over[m];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const uint32_t top = __reduce_max_sync(0xffffffffu, (held[m] >> (16 * x)) & 0x7fff);
              const uint32_t field = top >> 10;
              const float was = unit_of(one_over[m], x), size = __half2float(__ushort_as_half((unsigned short)top));
              if (top != 0 && !(size >= 0.0078125f * was && size < 2.f * was)) {  // it becomes the unit that is next below
                const float unit = __uint_as_float((min(field, 30u) + 112u) << 23);
                change[2 * m + x] = was * (1.f / unit);
                const uint32_t bits = __half_as_ushort(__float2half_rn(1.f / unit));
                next = x ? prmt(next, bits, 0x5410) : prmt(next, bits, 0x3254);
              }
            }
            one_over[m] = next;
            uint32_t in_units = mul_f16(held[m], next);
            // What lies below the unit's reach is left for later, unless there is no smaller unit; the
            // group's largest never is, so that passes end.
            const uint32_t small = __hlt2_mask(__habs2(*reinterpret_cast<const __half2*>(&in_units)),
                                               __float2half2_rn(0.0078125f)) &
                                   ~((next & 0xffff) == kLeastUnit4 ? 0xffffu : 0u) &
                                   ~((next >> 16) == kLeastUnit4 ? 0xffff0000u : 0u);
            left[m] = held[m] & small;
            of_mine[m] = in_units & ~small;
            rest |= left[m] & 0x7fff7fff;
          }
          again = __any_sync(0xffffffffu, rest != 0);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float next = fmaxf(ref[t][k], fmaf(group_max(largest(t, k)), fac[t][k], -kAbove4));
            const float f = fexp2(ref[t][k] - next);
            ref[t][k] = next;
            l[t][k] *= f;
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                o[t][g][h][k] *= f * change[g];
                o[t][g][h][2 + k] *= f * change[g];
              }
          }
      }
      __syncwarp();

#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // ---- probabilities, transposed: query row r, tokens 2c, 2c + 1 and 2c + 8, 2c + 9
        uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          float e[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) e[k] = fexp2(fmaf(z[h][t][k], fac[t][k & 1], -ref[t][k & 1]));
          if (!repeat) {
            l[t][0] += e[0] + e[2];
            l[t][1] += e[1] + e[3];
          }
          const uint32_t h0 = pack_f16(e[0], e[1]), h1 = pack_f16(e[2], e[3]);
          ph[t][0] = transpose8(h0);
          ph[t][1] = transpose8(h1);
          if constexpr (TERMS == 2) {
            const float2 f0 = unpack_f16(h0), f1 = unpack_f16(h1);
            pl[t][0] = transpose8(pack_f16((e[0] - f0.x) * kSecond4, (e[1] - f0.y) * kSecond4));
            pl[t][1] = transpose8(pack_f16((e[2] - f1.x) * kSecond4, (e[3] - f1.y) * kSecond4));
          }
        }

        // ---- V's scales of those tokens, two of a group in a register
        uint32_t sc[NG][2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t w[NG];
          const unsigned char* const two = scales + C::SCALES + (16 * h + 8 * k + 2 * c) * 2 * NG;
          if constexpr (NG == 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(two);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
          } else {
            const uint2 v = *reinterpret_cast<const uint2*>(two);
            w[0] = v.x; w[1] = v.y;
          }
#pragma unroll
          for (int g = 0; g < NG; g += 2) {
            sc[g][k] = prmt(w[g / 2], w[NG / 2 + g / 2], 0x5410);
            sc[g + 1][k] = prmt(w[g / 2], w[NG / 2 + g / 2], 0x7632);
          }
        }

        // ---- output: dimensions 32 g + 4 r + 2 x and the next, query rows 2c, 2c + 1
#pragma unroll
        for (int gp = 0; gp < NG; gp += 2) {
          uint32_t vw[2][2];
          ldsm_x4_t(at + (m_off ^ (16 * gp)) + C::CODES + 8 * D * h, vw[0][0], vw[0][1], vw[1][0], vw[1][1]);
#pragma unroll
          for (int gg = 0; gg < 2; ++gg) {
            const int g = gp + gg;
            uint32_t a[8];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const uint32_t x = vw[gg][k], y = x >> 8;
              a[2 * k] = codes.low(x);
              a[2 * k + 1] = codes.high(x);
              a[4 + 2 * k] = codes.low(y);
              a[5 + 2 * k] = codes.high(y);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              if constexpr (TERMS == 1) {
                const uint32_t w0 = mul_f16(ph[t][0], sc[g][0]), w1 = mul_f16(ph[t][1], sc[g][1]);
                mma_f16(o[t][g][0], a[0], a[1], a[2], a[3], w0, w1);
                mma_f16(o[t][g][1], a[4], a[5], a[6], a[7], w0, w1);
              } else {
                uint32_t hi[2], lo[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const float2 x = unpack_f16(ph[t][k]), y = unpack_f16(pl[t][k]), s = unpack_f16(sc[g][k]);
                  const float ea = fmaf(y.x, 1.f / kSecond4, x.x) * s.x, eb = fmaf(y.y, 1.f / kSecond4, x.y) * s.y;
                  hi[k] = pack_f16(ea, eb);
                  const float2 f = unpack_f16(hi[k]);
                  lo[k] = pack_f16((ea - f.x) * kSecond4, (eb - f.y) * kSecond4);
                }
                // The tensor cores cut what they add to a sum, which over a long range adds up:
                // sixteen tokens' products are summed by themselves, and added in float.
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                  float sum[4], second[4];
                  mma_f16_first(sum, a[4 * x], a[4 * x + 1], a[4 * x + 2], a[4 * x + 3], hi[0], hi[1]);
                  mma_f16_first(second, a[4 * x], a[4 * x + 1], a[4 * x + 2], a[4 * x + 3], lo[0], lo[1]);
#pragma unroll
                  for (int k = 0; k < 4; ++k) o[t][g][x][k] += fmaf(second[k], 1.f / kSecond4, sum[k]);
                }
              }
            }
          }
        }
      }
    }
    cp_async_wait<0>();
    __syncwarp();
    // ---- this warp's output, to be joined with the others'
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int row = 8 * t + 2 * c + k;
        const float sum = group_sum(l[t][k]);
        if (r == 0) ml_all[warp * RS + row] = make_float2(ref[t][k], sum);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const float unit = unit_of(one_over[g / 2], g & 1);
          *reinterpret_cast<float4*>(mine + C::OFF_O + 4 * (row * D + 32 * g + 4 * r)) =
              make_float4(o[t][g][0][k] * unit, o[t][g][0][2 + k] * unit, o[t][g][1][k] * unit, o[t][g][1][2 + k] * unit);
        }
      }
    d_b = q.b; d_g = q.g; d_row0 = q.it.row0; d_rows = rows; d_c0 = q.c0; d_parts = q.parts;
  }
  if (err) atomicOr(p.err, err);
}


// f(kernel, shared bytes, rows, CTAs per SM) for the instance that serves R query rows.
template <typename F>
auto with_att4(int dtype, int D, int R, F&& f) {
  auto inst = [&](auto zero, auto dim, auto tiles) {
    using T = decltype(zero);
    using C = Cfg4<T, decltype(dim)::value, decltype(tiles)::value>;
    return f(k_att4<T, decltype(dim)::value, decltype(tiles)::value>, C::SMEM, C::RS, C::CPS);
  };
  auto sized = [&](auto zero, auto dim) {
    if (R <= 8) return inst(zero, dim, std::integral_constant<int, 1>());
    if (R <= 16 || sizeof(zero) == 4) return inst(zero, dim, std::integral_constant<int, 2>());
    if constexpr (sizeof(zero) == 2) {
      return R <= 24 ? inst(zero, dim, std::integral_constant<int, 3>()) : inst(zero, dim, std::integral_constant<int, 4>());
    } else return inst(zero, dim, std::integral_constant<int, 2>());
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (dtype == 0) return D == 128 ? sized(__nv_bfloat16(), D128()) : sized(__nv_bfloat16(), D64());
  return D == 128 ? sized(0.f, D128()) : sized(0.f, D64());
}

}  // namespace

cudaError_t configure_attend4() {
  cudaError_t e = cudaSuccess;
  for (int dtype : {0, 1})
    for (int D : {64, 128})
      for (int R : {8, 16, 24, 32})
        if (e == cudaSuccess)
          e = with_att4(dtype, D, R, [](auto kernel, size_t smem, int, int) {
            return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
          });
  return e;
}

void plan_attend4(Attend4Params& p) {
  p.block = with_att4(p.dtype, p.D, p.R, [](auto, size_t, int rows, int) { return rows; });
  p.nqt = (p.R + p.block - 1) / p.block;
  // No more CTAs than shares of two tiles: idle ones cost a microsecond (one sequence of
  // 3857 tokens, 4 kv-heads: 11.0 us with 456 CTAs, 9.3 with 152).
  const int64_t items = p.B * (int64_t)p.nqt * p.Hkv;
  int64_t span = p.max_seq;
  if (p.window >= 0 && (int64_t)p.window + p.n_new + p.sinks + 2 * kTcTile < span)
    span = (int64_t)p.window + p.n_new + p.sinks + 2 * kTcTile;
  const int64_t shares = items * ((span + 2 * kTcTile - 1) / (2 * kTcTile)), waves = (shares + p.num_sms - 1) / p.num_sms;
  const int cps = with_att4(p.dtype, p.D, p.R, [](auto, size_t, int, int cps) { return cps; });
  p.grid = p.num_sms * (int)(waves < cps ? waves : cps);
  // An item's start and end take about as long as two tiles; where every item has
  // CTAs of its own, the least share of one follows from it (min_share).
  p.fixed = items <= p.grid / 4 ? 2 : 6;
}

cudaError_t launch_attend4(const Attend4Params& p, cudaStream_t st) {
  return with_att4(p.dtype, p.D, p.R, [&](auto kernel, size_t smem, int, int) {
    return launch_dep(kernel, dim3(p.grid), kThreads4, smem, st, p);
  });
}

}  // namespace vp
