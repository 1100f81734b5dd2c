// k_unpack4: the tokens of 4-bit caches that a call of vp_attend4 sees, as bf16 rows
// of the workspace.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "vp_attend_device.h"
#include "vp_cache4.h"
#include "vp_codes4.h"
#include "vp_device.h"

namespace vp {
namespace {

// ---------------------------------------------------------------------------
// k_unpack4<D>: (code - 8) * scale, rounded to bf16 where it is not one already.
// D / 8 lanes a row, 8 values each; a CTA takes 64 tokens of one (sequence,
// kv-head) at a time.  Rows that no new token sees are left as they are.  Of a
// paged cache the staged pages' table has -1 for those that are not mapped, which
// the attention kernel leaves out and reports.  144 bytes are read and 512 written per
// token and kv-head at D = 128, the latter into L2 where they fit: one sequence of
// 12289 tokens, 8 kv-heads, in 15 us of a call of 219.
// ---------------------------------------------------------------------------
constexpr int kUnpackThreads = 256, kUnpackTokens = 64;

__device__ __forceinline__ uint4 values(const Codes& codes, uint32_t x, uint16_t scale) {
  const float s = __half2float(__ushort_as_half(scale));
  const uint32_t y = x >> 8;
  // Dimensions k and k + 4 meet one mask.
  const float2 a = unpack_f16(codes.low(x)), b = unpack_f16(codes.high(x)), c = unpack_f16(codes.low(y)), d = unpack_f16(codes.high(y));
  return make_uint4(pack_bf16(a.x * s, b.x * s), pack_bf16(c.x * s, d.x * s), pack_bf16(a.y * s, b.y * s), pack_bf16(c.y * s, d.y * s));
}

template <int D>
__global__ void __launch_bounds__(kUnpackThreads) k_unpack4(const __grid_constant__ Unpack4Params p) {
  constexpr int L = D / 8, ROWS = kUnpackThreads / L;
  const int chunk = threadIdx.x % L, slot = threadIdx.x / L;
  const Codes codes;
  pdl_wait();
  pdl_trigger();
  const int blocks = (p.max_seq + kUnpackTokens - 1) / kUnpackTokens;
#pragma unroll 1
  for (int64_t x = blockIdx.x; x < (int64_t)p.B * p.Hkv * blocks; x += gridDim.x) {
    const int bg = (int)(x / blocks), j0 = (int)(x - (int64_t)bg * blocks) * kUnpackTokens, b = bg / p.Hkv, g = bg - b * p.Hkv;
    const NewSeq sq = load_new(p, b, false);
    if (sq.n <= 0) continue;
    const SeenRange sr = seen_range(sq.len - sq.n, sq.len - 1, p.window, p.sinks);
    if (j0 >= sr.hi || (j0 >= sr.s_end && j0 + kUnpackTokens <= sr.lo)) continue;
#pragma unroll 4
    for (int t = slot; t < kUnpackTokens; t += ROWS) {
      const int j = j0 + t;
      if (!(j < sr.s_end || (j >= sr.lo && j < sr.hi))) continue;
      int64_t kat = b, vat = b, row = j, to = ((int64_t)b * p.Hkv + g) * p.rows + j;
      if (p.paged) {
        const int lp = j >> p.page_shift;
        kat = lp < p.k4.max_pages ? __ldg(p.k4.block_table + (int64_t)b * p.k4.max_pages + lp) : -1;
        vat = lp < p.v4.max_pages ? __ldg(p.v4.block_table + (int64_t)b * p.v4.max_pages + lp) : -1;
        const bool ok = kat >= 0 && kat < p.k4.num_pages && vat >= 0 && vat < p.v4.num_pages;
        const int64_t page = (int64_t)b * p.pages + lp;
        // Every lane of a page's seen rows writes the same entry.
        if (g == 0 && chunk == 0) p.table[page] = ok ? (int)page : -1;
        if (!ok) continue;
        row = j & (p.page_size - 1);
        to = (page * p.Hkv + g) * p.page_size + row;
      }
      const uint32_t kc = __ldcs(reinterpret_cast<const uint32_t*>(p.k4.codes + kat * p.k4.cb + g * p.k4.ch + row * p.k4.ct) + chunk);
      const uint32_t vc = __ldcs(reinterpret_cast<const uint32_t*>(p.v4.codes + vat * p.v4.cb + g * p.v4.ch + row * p.v4.ct) + chunk);
      const uint16_t ks = __ldg(p.k4.scales + kat * p.k4.sb + g * p.k4.sh + row * p.k4.st + chunk / 4);
      const uint16_t vs = __ldg(p.v4.scales + vat * p.v4.sb + g * p.v4.sh + row * p.v4.st + chunk / 4);
      static_cast<uint4*>(p.k)[to * L + chunk] = values(codes, kc, ks);
      static_cast<uint4*>(p.v)[to * L + chunk] = values(codes, vc, vs);
    }
  }
}

}  // namespace

cudaError_t launch_unpack4(const Unpack4Params& p, cudaStream_t st) {
  const int64_t all = (int64_t)p.B * p.Hkv * ((p.max_seq + kUnpackTokens - 1) / kUnpackTokens);
  const int64_t most = 8 * (int64_t)p.num_sms;
  const dim3 grid((unsigned)(all < most ? all : most));
  return p.D == 128 ? launch_dep(k_unpack4<128>, grid, kUnpackThreads, 0, st, p)
                    : launch_dep(k_unpack4<64>, grid, kUnpackThreads, 0, st, p);
}

}  // namespace vp
