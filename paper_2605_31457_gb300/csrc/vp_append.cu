// k_append: the position rotation of new queries and keys, and the new keys and
// values appended to their caches, in the context's type or in 4 bits (vp_append,
// vp_append4).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "vp_attend_device.h"
#include "vp_cache4.h"
#include "vp_device.h"

namespace vp {
namespace {

// ---------------------------------------------------------------------------
// k_append<T, D, Q4>: a row (D values of a query head, key or value) is D / 8
// lanes of a warp, 8 values each.  A pair (a, b) with the angle's cosine c and
// sine s becomes (a c - b s, b c + a s) in float, every operation rounded by
// itself; with pairs half the rotated dimensions apart the partner's values come
// from another lane by shuffles.  Rows come out rounded once to T.
//
// Q4: 32 values (4 lanes) share a scale, the least number of four significant
// bits that is not below 1 / 7.5 of their largest magnitude, so that a held value
// (code - 8) * scale, a 4-bit whole number times 4 significant bits, is exact in
// bf16.  A code is the value times the scale's rounded reciprocal, rounded to
// the nearest whole number (ties to even).  A NaN makes its group's scale NaN.
//
// Bound by memory for prompts and by the launch for tokens.  A CTA serves rows
// of one token, so that its threads hold one set of cosines and sines; tokens are
// few at a decode step, when several CTAs share one token's rows (AppendParams
// ::parts).  Nothing triggers the next kernel early: what follows may read the
// caches before it waits.
// ---------------------------------------------------------------------------
constexpr int kAppendThreads = 128;

template <typename T> struct Raw8;  // eight values as 32-bit words
template <> struct Raw8<__nv_bfloat16> {
  static constexpr int N = 4;
  uint32_t w[4];
  __device__ void floats(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) bf2(w[i], f[2 * i], f[2 * i + 1]);
  }
  __device__ void set(const float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
  }
};
template <> struct Raw8<float> {
  static constexpr int N = 8;
  uint32_t w[8];
  __device__ void floats(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
  }
  __device__ void set(const float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(f[i]);
  }
};
template <typename T>
__device__ __forceinline__ void load_raw(Raw8<T>& r, const T* p) {
#pragma unroll
  for (int i = 0; i < Raw8<T>::N; i += 4) {
    const uint4 v = __ldcg(reinterpret_cast<const uint4*>(p) + i / 4);
    r.w[i] = v.x; r.w[i + 1] = v.y; r.w[i + 2] = v.z; r.w[i + 3] = v.w;
  }
}
template <typename T>
__device__ __forceinline__ void store_raw(T* p, const Raw8<T>& r) {
#pragma unroll
  for (int i = 0; i < Raw8<T>::N; i += 4)
    reinterpret_cast<uint4*>(p)[i / 4] = make_uint4(r.w[i], r.w[i + 1], r.w[i + 2], r.w[i + 3]);
}

// The cosine and signed sine of each of this lane's 8 values: value e becomes
// x c + partner s, the partner the pair's other value.
// at: the token's positions on the axes.
__device__ __forceinline__ void load_angles(const RotView& r, const int (&at)[3], int chunk, float (&c)[8], float (&s)[8],
                                            unsigned& err) {
  const int pairs = r.rot / 2;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    c[e] = 1.f;
    s[e] = 0.f;
  }
  if (8 * chunk >= r.rot) return;
  auto row = [&](int f) {  // the table's row for pair f
    int x = f < r.end0 ? at[0] : f < r.end1 ? at[1] : at[2];
    if (x < 0 || x >= r.max_pos) {
      err |= ERR_POS;
      x = x < 0 ? 0 : r.max_pos - 1;
    }
    return r.cos_sin + (int64_t)x * r.rot;
  };
  auto one_axis = [&](int f0, int f1) {
    return (f0 < r.end0) == (f1 < r.end0) && (f0 < r.end1) == (f1 < r.end1);
  };
  if (r.interleaved) {
    const int f0 = 4 * chunk;
    float x[4], y[4];
    if (one_axis(f0, f0 + 3)) {
      const float* t = row(f0) + f0;
      load_f(t, x);
      load_f(t + pairs, y);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float* t = row(f0 + k) + f0 + k;
        x[k] = __ldg(t);
        y[k] = __ldg(t + pairs);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      c[2 * k] = c[2 * k + 1] = x[k];
      s[2 * k] = -y[k];
      s[2 * k + 1] = y[k];
    }
  } else {
    const bool second = 8 * chunk >= pairs;
    const int f0 = 8 * chunk - (second ? pairs : 0);
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
      float x[4], y[4];
      if (one_axis(f0 + h, f0 + h + 3)) {
        const float* t = row(f0 + h) + f0 + h;
        load_f(t, x);
        load_f(t + pairs, y);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float* t = row(f0 + h + k) + f0 + h + k;
          x[k] = __ldg(t);
          y[k] = __ldg(t + pairs);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        c[h + k] = x[k];
        s[h + k] = second ? y[k] : -y[k];
      }
    }
  }
}

// Eight values of a row in 4 bits, their group in this lane and the three beside
// it (called by the whole warp): the scale, the codes of the values, the first in
// the lowest bits, and in x what they stand for.
__device__ __forceinline__ uint32_t quantise(float (&x)[8], __half& scale) {
  uint32_t top = 0;  // the magnitude's bits: NaN above everything
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const bool nan = top > 0x7f800000u;
  const uint32_t t = __float_as_uint(__fmul_rn(__uint_as_float(top), (float)(1 / 7.5)));
  const float up = __uint_as_float((t + 0xfffffu) & ~0xfffffu);
  const float step = nan ? 1.f : fminf(fmaxf(up, kLeastStep4), kMostStep4);
  scale = nan ? __ushort_as_half(0x7fff) : __float2half_rn(step);
  const float inv = __frcp_rn(step), held = nan ? __uint_as_float(0x7fffffffu) : step;
  // Rounding to whole numbers by an addition: floats in [2^23, 2^24) are those, and
  // 8 more than 1.5 * 2^23 leaves the code in the lowest bits.
  constexpr float kWhole = 12582920.f;
  uint32_t codes = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float whole = __fadd_rn(fminf(fmaxf(__fmul_rn(x[e], inv), -8.f), 7.f), kWhole);
    codes |= (__float_as_uint(whole) & 15u) << (4 * e);
    x[e] = (whole - kWhole) * held;
  }
  return codes;
}

template <typename T, int D, bool Q4>
__global__ void __launch_bounds__(kAppendThreads) k_append(const __grid_constant__ AppendParams p) {
  constexpr int L = D / 8, SLOTS = kAppendThreads / L;  // lanes of a row, rows at a time
  const int chunk = threadIdx.x % L, slot = threadIdx.x / L;
  constexpr int U = 24 / Raw8<T>::N;  // rows of a thread in flight: 48 (D = 128, bf16) of a CTA
  pdl_wait();
  const int token = blockIdx.x / p.parts, part = blockIdx.x - token * p.parts;
  const int b = token / p.n_new, i = token - b * p.n_new;
  const int rows = p.H + 2 * p.Hkv;
  Raw8<T> x[U];
  auto load = [&](int r0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * p.parts * SLOTS + slot;
      if (r >= rows) continue;
      const bool is_q = r < p.H, is_k = r < p.H + p.Hkv;
      const RowView& in = is_q ? p.q : is_k ? p.k : p.v;
      const int g = is_q ? r : is_k ? r - p.H : r - p.H - p.Hkv;
      load_raw(x[u], static_cast<const T*>(in.data) + (int64_t)b * in.sb + (int64_t)i * in.sn + (int64_t)g * in.sh + 8 * chunk);
    }
  };
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < Raw8<T>::N; ++k) x[u].w[k] = 0;
  load(part * SLOTS);  // on their way while lengths, pages and angles are looked up
  unsigned err = 0;
  int at[3] = {0, 0, 0};
  if (p.rot.pos) {
#pragma unroll
    for (int a = 0; a < 3; ++a)
      if (a < p.rot.axes) at[a] = __ldg(p.rot.pos + ((int64_t)a * p.B + b) * p.n_new + i);
  }
  const int len = __ldcg(p.seq_len + b);
  int n = p.new_len ? __ldcg(p.new_len + b) : len > 0 ? p.n_new : 0;
  if (len < 0 || len > p.max_seq) err |= ERR_LEN;
  else if (n < 0 || n > min(p.n_new, len)) err |= ERR_NEW;
  if (err) n = 0;  // nothing of this sequence is appended
  if (i < n) {
    const int place = len - n + i;
    int64_t kat = b, vat = b;  // sequence or page of the new rows; < 0: nowhere
    int row = place;
    if (p.paged) {
      const int lp = place >> p.page_shift;
      const int32_t *kt = Q4 ? p.kc4.block_table : p.kc.block_table, *vt = Q4 ? p.vc4.block_table : p.vc.block_table;
      const int kmax = Q4 ? p.kc4.max_pages : p.kc.max_pages, vmax = Q4 ? p.vc4.max_pages : p.vc.max_pages;
      const int kn = Q4 ? p.kc4.num_pages : p.kc.num_pages, vn = Q4 ? p.vc4.num_pages : p.vc.num_pages;
      kat = lp < kmax ? __ldg(kt + (int64_t)b * kmax + lp) : -1;
      vat = lp < vmax ? __ldg(vt + (int64_t)b * vmax + lp) : -1;
      if (kat < 0 || kat >= kn) kat = -1;
      if (vat < 0 || vat >= vn) vat = -1;
      if (kat < 0 || vat < 0) err |= ERR_PAGE;
      row = place & (p.page_size - 1);
    }
    float c[8], s[8];
    if (!p.rot.pos) at[0] = place;
    if (p.rot.cos_sin) load_angles(p.rot, at, chunk, c, s, err);
    const int pairs = p.rot.rot / 2;
    // The lane that holds the partners of this lane's values.
    const int lane = threadIdx.x & 31;
    const int other = 8 * chunk >= p.rot.rot ? lane : 8 * chunk >= pairs ? lane - pairs / 8 : lane + pairs / 8;
    for (int r0 = part * SLOTS; r0 < rows; r0 += U * p.parts * SLOTS) {
      if (r0 != part * SLOTS) load(r0);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = r0 + u * p.parts * SLOTS + slot;
        const bool is_q = r < p.H, is_k = !is_q && r < p.H + p.Hkv, is_v = !is_q && !is_k && r < rows;
        const int g = is_q ? r : is_k ? r - p.H : r - p.H - p.Hkv;
        if (p.rot.cos_sin && __any_sync(0xffffffffu, is_q || is_k)) {
          float f[8], o[8];
          x[u].floats(f);
          if (p.rot.interleaved) {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = f[e ^ 1];
          } else {
            Raw8<T> y;
#pragma unroll
            for (int k = 0; k < Raw8<T>::N; ++k) y.w[k] = __shfl_sync(0xffffffffu, x[u].w[k], other);
            y.floats(o);
          }
          if ((is_q || is_k) && 8 * chunk < p.rot.rot) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __fadd_rn(__fmul_rn(f[e], c[e]), __fmul_rn(o[e], s[e]));
            x[u].set(f);
          }
        }
        if (is_q)
          store_raw(static_cast<T*>(p.q_out.data) + (int64_t)b * p.q_out.sb + (int64_t)i * p.q_out.sn +
                        (int64_t)g * p.q_out.sh + 8 * chunk, x[u]);
        const int64_t to_b = is_k ? kat : vat;
        if constexpr (Q4) {
          if (__any_sync(0xffffffffu, is_k || is_v)) {
            float f[8];
            x[u].floats(f);
            __half scale;
            const uint32_t codes = quantise(f, scale);
            if (is_k || is_v) {
              if (to_b >= 0) {
                const Kv4View& to = is_k ? p.kc4 : p.vc4;
                *reinterpret_cast<uint32_t*>(to.codes + to_b * to.cb + (int64_t)g * to.ch + (int64_t)row * to.ct + 4 * chunk) = codes;
                if (chunk % 4 == 0)
                  to.scales[to_b * to.sb + (int64_t)g * to.sh + (int64_t)row * to.st + chunk / 4] = __half_as_ushort(scale);
              }
              const RowView& held = is_k ? p.k_held : p.v_held;
              if (held.data) {
                x[u].set(f);
                store_raw(static_cast<T*>(held.data) + (int64_t)b * held.sb + (int64_t)i * held.sn +
                              (int64_t)g * held.sh + 8 * chunk, x[u]);
              }
            }
          }
        } else if ((is_k || is_v) && to_b >= 0) {
          const KvView& to = is_k ? p.kc : p.vc;
          store_raw(static_cast<T*>(const_cast<void*>(to.data)) + to_b * to.sb + (int64_t)g * to.sh + (int64_t)row * to.st + 8 * chunk,
                    x[u]);
        }
      }
    }
  }
  if (err) atomicOr(p.err, err);
}

template <typename T, int D, bool Q4>
cudaError_t launch(const AppendParams& p, cudaStream_t st) {
  const int64_t ctas = (int64_t)p.B * p.n_new * p.parts;
  if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
  return launch_dep(k_append<T, D, Q4>, dim3((unsigned)ctas), kAppendThreads, 0, st, p);
}

}  // namespace

cudaError_t launch_append(AppendParams& p, int dtype, int D, bool four, int num_sms, cudaStream_t st) {
  const int slots = kAppendThreads / (D / 8), most = (p.H + 2 * p.Hkv + slots - 1) / slots;
  const int64_t tokens = (int64_t)p.B * p.n_new, want = 8 * (int64_t)num_sms / tokens;
  p.parts = want < 1 ? 1 : want > most ? most : (int)want;
  auto typed = [&](auto zero) {
    using T = decltype(zero);
    if (D == 128) return four ? launch<T, 128, true>(p, st) : launch<T, 128, false>(p, st);
    return four ? launch<T, 64, true>(p, st) : launch<T, 64, false>(p, st);
  };
  return dtype == 0 ? typed(__nv_bfloat16()) : typed(0.f);
}

}  // namespace vp
