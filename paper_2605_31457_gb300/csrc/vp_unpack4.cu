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
// kv-head) at a time, every `splits`-th such tile.  Rows that no new token sees are left as they are.  Of a
// paged cache the staged pages' table has -1 for those that are not mapped, which
// the attention kernel leaves out and reports.  144 bytes are read and 512 written per
// token and kv-head at D = 128, the latter into L2 where they fit: one sequence of
// 12289 tokens, 8 kv-heads, in 14 us of a call of 219.
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
  constexpr int L = D / 8, ROWS = kUnpackThreads / L, RPT = kUnpackTokens / ROWS;
  const int chunk = threadIdx.x % L, slot = threadIdx.x / L;
  const Codes codes;
  pdl_wait();
  pdl_trigger();
  const int bg = blockIdx.x / p.splits, b = bg / p.Hkv, g = bg - b * p.Hkv;
  const NewSeq sq = load_new(p, b, false);
  if (sq.n <= 0) return;
  const SeenRange sr = seen_range(sq.len - sq.n, sq.len - 1, p.window, p.sinks);
  const TileList tl = tile_list(sr, kUnpackTokens);
#pragma unroll 1
  for (int u = blockIdx.x - bg * p.splits; u < tl.n; u += p.splits) {
    const int j0 = tl.tile(u) * kUnpackTokens;
    uint32_t kc[RPT], vc[RPT];
    uint16_t ks[RPT], vs[RPT];
    int64_t to[RPT];  // the staged row; < 0: none
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const int j = j0 + slot + i * ROWS;
      to[i] = -1;
      kc[i] = vc[i] = 0;
      ks[i] = vs[i] = 0;
      if (!(j < sr.s_end || (j >= sr.lo && j < sr.hi))) continue;
      int64_t kat = b, vat = b, row = j;
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
        to[i] = (page * p.Hkv + g) * p.page_size + row;
      } else {
        to[i] = ((int64_t)b * p.Hkv + g) * p.rows + j;
      }
      kc[i] = __ldcs(reinterpret_cast<const uint32_t*>(p.k4.codes + kat * p.k4.cb + g * p.k4.ch + row * p.k4.ct) + chunk);
      vc[i] = __ldcs(reinterpret_cast<const uint32_t*>(p.v4.codes + vat * p.v4.cb + g * p.v4.ch + row * p.v4.ct) + chunk);
      ks[i] = __ldg(p.k4.scales + kat * p.k4.sb + g * p.k4.sh + row * p.k4.st + chunk / 4);
      vs[i] = __ldg(p.v4.scales + vat * p.v4.sb + g * p.v4.sh + row * p.v4.st + chunk / 4);
    }
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      if (to[i] < 0) continue;
      static_cast<uint4*>(p.k)[to[i] * L + chunk] = values(codes, kc[i], ks[i]);
      static_cast<uint4*>(p.v)[to[i] * L + chunk] = values(codes, vc[i], vs[i]);
    }
  }
}

}  // namespace

cudaError_t launch_unpack4(Unpack4Params& p, cudaStream_t st) {
  const int tiles = (p.max_seq + kUnpackTokens - 1) / kUnpackTokens, want = 16 * p.num_sms / (p.B * p.Hkv);
  p.splits = want < 1 ? 1 : want < tiles ? want : tiles;
  const int64_t ctas = (int64_t)p.B * p.Hkv * p.splits;
  if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)ctas);
  return p.D == 128 ? launch_dep(k_unpack4<128>, grid, kUnpackThreads, 0, st, p)
                    : launch_dep(k_unpack4<64>, grid, kUnpackThreads, 0, st, p);
}

}  // namespace vp
