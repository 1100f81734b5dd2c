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
// The workspace of vp_attend4 (vp_reserve4) is that of vp_attend_new.
void plan_attend4(Attend4Params& p);
cudaError_t configure_attend4();
cudaError_t launch_attend4(const Attend4Params& p, cudaStream_t s);

}  // namespace vp
