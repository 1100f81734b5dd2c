// Definitions of vp_append, vp_append4 and vp_attend4 shared by the host side
// (vp_cache4_api.cu) and the kernels (vp_append.cu, vp_attend4.cu), and the form
// of a cache held in 4 bits.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "vp_attend.h"
#include "vp_internal.h"

namespace vp {

constexpr int kGroup4 = 32;  // values that share a scale
// Scales are fp16 numbers in [kLeastStep4, kMostStep4].
constexpr float kLeastStep4 = 6.103515625e-05f, kMostStep4 = 61440.f;

// A 4-bit cache (vp_kv4): rows of D / 2 bytes of codes and of D / 32 fp16 scales;
// code strides in bytes, scale strides in scales.
struct Kv4View {
  uint8_t* codes;
  uint16_t* scales;
  int64_t cb, ch, ct;
  int64_t sb, sh, st;
  const int32_t* block_table;
  int32_t max_pages, num_pages;
};

// Rotation of the rows that vp_append writes (vp_rotation).  Pair f of a row turns
// by the angle of its axis' position: axis 0 for f < end0, 1 for f < end1, else 2.
struct RotView {
  const float* cos_sin;  // [max_pos][rot]: rot / 2 cosines, then the sines; NULL: no rotation
  int max_pos, rot, interleaved;
  const int32_t* pos;    // [axes][B][n_new], or NULL: the token's place in its sequence
  int axes, end0, end1;  // axes 1: end0 = rot / 2
};

// Whether rows of `row` elements do not overlap: nb, nh and nt of them along axes of
// these strides.  (An axis of one element may have any stride.)
inline bool rows_apart(int64_t sb, int64_t sh, int64_t st, int64_t nb, int64_t nh, int64_t nt, int64_t row) {
  return (nb <= 1 || sb >= row) && (nh <= 1 || sh >= row) && (nt <= 1 || st >= row);
}

struct AppendParams {
  int B, n_new, H, Hkv, max_seq;  // H: query heads to rotate; 0: none
  int paged, page_size, page_shift;
  RowView q, k, v, q_out;
  RowView k_held, v_held;         // data may be NULL
  KvView kc, vc;                  // vp_append
  Kv4View kc4, vc4;               // vp_append4
  const int32_t* seq_len;
  const int32_t* new_len;         // or NULL
  RotView rot;
  unsigned* err;
  int parts;                      // warps of a token
};

cudaError_t launch_append(AppendParams& p, int dtype, int D, bool four, int num_sms, cudaStream_t s);

// vp_attend4.  AttendParams' k and v are not used.
struct Attend4Params : AttendParams {
  Kv4View k4, v4;
};

// Calls of many query rows unpack the tokens that they see into bf16 caches of the
// workspace (exactly, for vp_append4's scales) and run the kernels of vp_attend_new
// on those: a group of sequences at a time, as many as the workspace holds (which follows
// from max_seq, not from their lengths).  The rule goes by rows alone: where there are
// few items, as with one sequence, k_att4 is still the faster way somewhat above it.  Measured,
// 32/8 heads of 128, k_att4 against this way: one sequence of 9001 tokens, 128 rows
// 35 us against 97, 256 rows 60 against 72; four of up to 9001, 128 rows 65 against
// 93, 192 rows 94 against 89; 16 of them, 128 rows 227 against 255, 160 rows 283
// against 265.
constexpr int kStageRows = 128;  // more query rows than this per (sequence, kv-head)
constexpr size_t kStageBytes = (size_t)1 << 30;
inline bool stages(int dtype, int paged, int page_size, int64_t R) {
  return dtype == 0 && (!paged || page_size >= 8) && R > kStageRows;
}

// The workspace of vp_attend4 (vp_reserve4): that of vp_attend_new, then the staged
// caches, K and V each [seqs][Hkv][rows][D] or, paged, [seqs * pages][Hkv][page_size][D]
// with their block table [seqs][pages].
struct Layout4 : NewLayout {
  int seqs = 0, rows = 0, pages = 0;
  size_t o_k = 0, o_v = 0, o_table = 0;
};
inline Layout4 layout4(int max_batch, int H, int Hkv, int D, int max_seq, int max_new, int dtype, int paged, int page_size,
                       int num_sms) {
  Layout4 w;
  static_cast<NewLayout&>(w) = new_layout(max_batch, H, Hkv, D, max_seq, max_new, 0, num_sms);
  if (!stages(dtype, paged, page_size, (int64_t)max_new * (H / Hkv))) return w;
  const int unit = paged ? page_size : kTcTile;
  w.pages = (max_seq + unit - 1) / unit;
  w.rows = w.pages * unit;
  const size_t one = (size_t)Hkv * w.rows * D * 2;  // bytes of a sequence's K or V
  const size_t fit = kStageBytes / (2 * one);
  w.seqs = fit < 1 ? 1 : fit < (size_t)max_batch ? (int)fit : max_batch;
  w.o_k = w.total;
  w.o_v = ws_round(w.o_k + w.seqs * one);
  w.o_table = ws_round(w.o_v + w.seqs * one);
  w.total = ws_round(w.o_table + (paged ? (size_t)w.seqs * w.pages * 4 : 0));
  return w;
}

struct Unpack4Params {
  int B, Hkv, D, max_seq, n_new;
  int paged, page_size, page_shift;
  Kv4View k4, v4;
  void *k, *v;         // staged caches
  int rows, pages;     // Layout4's
  int32_t* table;      // paged
  const int32_t* seq_len;
  const int32_t* new_len;
  int window, sinks;
  unsigned* err;
  int num_sms;
  int splits;          // CTAs of a (sequence, kv-head), set by launch_unpack4
};
cudaError_t launch_unpack4(Unpack4Params& p, cudaStream_t s);

void plan_attend4(Attend4Params& p);
cudaError_t configure_attend4();
cudaError_t launch_attend4(const Attend4Params& p, cudaStream_t s);

}  // namespace vp
