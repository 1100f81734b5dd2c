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
// Bound by the launch for tokens and by memory and issue slots for prompts.  A warp
// serves rows of one token, so that its lanes hold one set of cosines and sines and of
// addresses; where tokens are few, several warps share one token's rows (AppendParams
// ::parts).  Its turns are of one kind each, queries, keys or values, so that nothing
// is chosen per lane, and the loads of four rows are on their way while lengths, pages
// and angles are looked up.  In a graph, heads of 128: one token of 32 sequences, 28/4,
// in 2.8 us (4 bits: 3.1); a prompt of 3857, 28/4, in 15.5 us (4.7 TB/s; 12.1 us time
// after time on one set of inputs, half of which stays in L2), where the loads of the next
// four rows wait for the stores of these; four of up to
// 2305, 32/8, in 4 bits in 43 us (4.6 TB/s; three quarters of the issue slots).  A CTA
// per token took 17.1 and 52 us, six rows in flight 15.5 and 50.
// Nothing triggers the next kernel early: what follows may read the caches before it
// waits.
// ---------------------------------------------------------------------------
constexpr int kAppendThreads = 128;
constexpr int kAppendWarps = 16;  // warps per SM that a call is spread over

template <typename T> struct Raw8;  // eight values as 32-bit words; get and set: the i-th two of them
template <> struct Raw8<__nv_bfloat16> {
  static constexpr int N = 4;
  uint32_t w[4];
  __device__ float2 get(int i) const {
    float2 f;
    bf2(w[i], f.x, f.y);
    return f;
  }
  __device__ void set(int i, float2 f) { w[i] = pack_bf16(f.x, f.y); }
};
template <> struct Raw8<float> {
  static constexpr int N = 8;
  uint32_t w[8];
  __device__ float2 get(int i) const { return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])); }
  __device__ void set(int i, float2 f) {
    w[2 * i] = __float_as_uint(f.x);
    w[2 * i + 1] = __float_as_uint(f.y);
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
  auto larger = [](float a, float b) {  // of magnitudes; NaN above everything
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
  };
  float top = fabsf(x[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) top = larger(top, fabsf(x[e]));
  top = larger(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = larger(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const bool nan = isnan(top);
  const float t = __fmul_rn(top, (float)(1 / 7.5));
  const float up = __uint_as_float((__float_as_uint(t) + 0xfffffu) & ~0xfffffu);
  const float step = nan ? 1.f : fminf(fmaxf(up, kLeastStep4), kMostStep4);
  scale = nan ? __ushort_as_half(0x7fff) : __float2half_rn(step);
  const float inv = __frcp_rn(step), held = nan ? __uint_as_float(0x7fffffffu) : step;
  if (up > kMostStep4) {  // cut to what the largest scale holds
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = fminf(fmaxf(x[e], -8.f * kMostStep4), 8.f * kMostStep4);
  }
  // Rounding to whole numbers by an addition, floats from 2^23 to 2^24 being those;
  // |x / step| <= 7.5 (a little more by rounding) leaves at least -8.
  constexpr float kWhole = 12582912.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = __fadd_rn(fminf(__fmul_rn(x[e], inv), 7.f), kWhole) - kWhole;
  // Four codes side by side, 8 added to each: a whole number below 2^16.
  auto four = [&](int e) {
    return __float_as_uint(fmaf(fmaf(x[e + 3], 16.f, x[e + 2]), 256.f, fmaf(x[e + 1], 16.f, x[e])) + (8388608.f + 34952.f));
  };
  const uint32_t codes = prmt(four(0), four(4), 0x5410);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= held;
  return codes;
}

template <typename T, int D, bool Q4>
__global__ void __launch_bounds__(kAppendThreads, Q4 ? 7 : 6) k_append(const __grid_constant__ AppendParams p) {
  constexpr int L = D / 8, SLOTS = 32 / L;  // lanes of a row, rows of a warp at a time
  constexpr int U = 16 / Raw8<T>::N;        // of a lane in flight
  const int lane = threadIdx.x & 31, chunk = lane % L, slot = lane / L;
  pdl_wait();
  const unsigned unit = uniform(blockIdx.x * (kAppendThreads / 32) + threadIdx.x / 32);
  const unsigned token = unit / (unsigned)p.parts, part = unit - token * p.parts;
  const int b = token / (unsigned)p.n_new, i = token - b * p.n_new;
  if (b >= p.B) return;
  // Turns: SLOTS rows of queries each, then of keys, then of values.
  const int nq = (p.H + SLOTS - 1) / SLOTS, nk = (p.Hkv + SLOTS - 1) / SLOTS, turns = nq + 2 * nk;
  struct Turn {
    bool is_q, is_k;
    int first;  // its first row
  };
  auto turn = [&](int t) {
    Turn x;
    x.is_q = t < nq;
    x.is_k = !x.is_q && t < nq + nk;
    x.first = (x.is_q ? t : x.is_k ? t - nq : t - nq - nk) * SLOTS;
    return x;
  };
  // This lane's chunk of row `slot`, where it comes from and goes to.
  auto from = [&](const RowView& v) {
    return static_cast<T*>(v.data) + (int64_t)b * v.sb + (int64_t)i * v.sn + (int64_t)slot * v.sh + 8 * chunk;
  };
  const T *q_in = from(p.q), *k_in = from(p.k), *v_in = from(p.v);
  Raw8<T> x[U];
  auto load = [&](int t0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * p.parts;
      if (t >= turns) break;
      const Turn w = turn(t);
      if (w.first + slot < (w.is_q ? p.H : p.Hkv))
        load_raw(x[u], (w.is_q ? q_in : w.is_k ? k_in : v_in) + w.first * (w.is_q ? p.q.sh : w.is_k ? p.k.sh : p.v.sh));
    }
  };
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < Raw8<T>::N; ++k) x[u].w[k] = 0;
  load(part);  // on their way while lengths, pages and angles are looked up
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
    const bool turned = p.rot.cos_sin && 8 * chunk < p.rot.rot;
    const int other = !turned ? lane : 8 * chunk >= pairs ? lane - pairs / 8 : lane + pairs / 8;
    auto turn2 = [&](float2 a, float2 z, int k) {  // products two at a time, sums apart (as pairs they would be fused)
      const float2 x = mul2(a, make_float2(c[2 * k], c[2 * k + 1])), y = mul2(z, make_float2(s[2 * k], s[2 * k + 1]));
      return make_float2(__fadd_rn(x.x, y.x), __fadd_rn(x.y, y.y));
    };
    auto rotate = [&](Raw8<T>& y) {
      if (!p.rot.cos_sin) return;
      if (p.rot.interleaved) {
        if (!turned) return;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 a = y.get(k);
          y.set(k, turn2(a, make_float2(a.y, a.x), k));
        }
        return;
      }
      Raw8<T> o;
#pragma unroll
      for (int k = 0; k < Raw8<T>::N; ++k) o.w[k] = __shfl_sync(0xffffffffu, y.w[k], other);
      if (!turned) return;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        y.set(k, turn2(y.get(k), o.get(k), k));
      }
    };
    T* const q_out = from(p.q_out);
    // The new token's rows of the caches, in T or as codes with their scale.
    T *k_to = nullptr, *v_to = nullptr, *k_held = nullptr, *v_held = nullptr;
    uint8_t *k_codes = nullptr, *v_codes = nullptr;
    uint16_t *k_scale = nullptr, *v_scale = nullptr;
    if constexpr (Q4) {
      k_codes = p.kc4.codes + kat * p.kc4.cb + row * p.kc4.ct + slot * p.kc4.ch + 4 * chunk;
      v_codes = p.vc4.codes + vat * p.vc4.cb + row * p.vc4.ct + slot * p.vc4.ch + 4 * chunk;
      k_scale = p.kc4.scales + kat * p.kc4.sb + row * p.kc4.st + slot * p.kc4.sh + chunk / 4;
      v_scale = p.vc4.scales + vat * p.vc4.sb + row * p.vc4.st + slot * p.vc4.sh + chunk / 4;
      k_held = from(p.k_held);
      v_held = from(p.v_held);
    } else {
      k_to = static_cast<T*>(const_cast<void*>(p.kc.data)) + kat * p.kc.sb + row * p.kc.st + slot * p.kc.sh + 8 * chunk;
      v_to = static_cast<T*>(const_cast<void*>(p.vc.data)) + vat * p.vc.sb + row * p.vc.st + slot * p.vc.sh + 8 * chunk;
    }
#pragma unroll 1
    for (int t0 = part; t0 < turns; t0 += U * p.parts) {
      if (t0 != (int)part) load(t0);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = t0 + u * p.parts;
        if (t >= turns) break;
        const Turn w = turn(t);
        const bool there = w.first + slot < (w.is_q ? p.H : p.Hkv);
        Raw8<T>& y = x[u];
        if (w.is_q) {
          rotate(y);
          if (there) store_raw(q_out + w.first * p.q_out.sh, y);
          continue;
        }
        if (w.is_k) rotate(y);
        const bool mapped = there && (w.is_k ? kat : vat) >= 0;
        if constexpr (Q4) {
          float f[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 a = y.get(k);
            f[2 * k] = a.x;
            f[2 * k + 1] = a.y;
          }
          __half scale;
          const uint32_t codes = quantise(f, scale);
          if (mapped) {
            *reinterpret_cast<uint32_t*>((w.is_k ? k_codes : v_codes) + w.first * (w.is_k ? p.kc4.ch : p.vc4.ch)) = codes;
            if (chunk % 4 == 0)
              (w.is_k ? k_scale : v_scale)[w.first * (w.is_k ? p.kc4.sh : p.vc4.sh)] = __half_as_ushort(scale);
          }
          if (there && (w.is_k ? p.k_held.data : p.v_held.data) != nullptr) {
#pragma unroll
            for (int k = 0; k < 4; ++k) y.set(k, make_float2(f[2 * k], f[2 * k + 1]));
            store_raw((w.is_k ? k_held : v_held) + w.first * (w.is_k ? p.k_held.sh : p.v_held.sh), y);
          }
        } else if (mapped) {
          store_raw((w.is_k ? k_to : v_to) + w.first * (w.is_k ? p.kc.sh : p.vc.sh), y);
        }
      }
    }
  }
  if (err) atomicOr(p.err, err);
}

template <typename T, int D, bool Q4>
cudaError_t launch(const AppendParams& p, cudaStream_t st) {
  constexpr int kUnits = kAppendThreads / 32;
  const int64_t ctas = ((int64_t)p.B * p.n_new * p.parts + kUnits - 1) / kUnits;
  if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
  return launch_dep(k_append<T, D, Q4>, dim3((unsigned)ctas), kAppendThreads, 0, st, p);
}

}  // namespace

cudaError_t launch_append(AppendParams& p, int dtype, int D, bool four, int num_sms, cudaStream_t st) {
  const int slots = 256 / D, most = (p.H + slots - 1) / slots + 2 * ((p.Hkv + slots - 1) / slots);
  const int64_t tokens = (int64_t)p.B * p.n_new, want = kAppendWarps * (int64_t)num_sms / tokens;
  p.parts = want < 1 ? 1 : want > most ? most : (int)want;
  auto typed = [&](auto zero) {
    using T = decltype(zero);
    if (D == 128) return four ? launch<T, 128, true>(p, st) : launch<T, 128, false>(p, st);
    return four ? launch<T, 64, true>(p, st) : launch<T, 64, false>(p, st);
  };
  return dtype == 0 ? typed(__nv_bfloat16()) : typed(0.f);
}

}  // namespace vp
