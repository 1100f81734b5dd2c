// Device and launch helpers shared by the kernels of vp_attend_new.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "vp_attend.h"

namespace vp {

constexpr float kLn2 = 0.6931471805599453f;

// Live tokens of a sequence and how many of them are new.
struct NewSeq {
  int len, n;
};
__device__ __forceinline__ NewSeq load_new(const AttendParams& p, int b, bool report) {
  NewSeq s;
  s.len = __ldcg(p.seq_len + b);
  unsigned e = 0;
  if (s.len < 0 || s.len > p.max_seq) { e |= ERR_LEN; s.len = min(max(s.len, 0), p.max_seq); }
  s.n = p.new_len ? __ldcg(p.new_len + b) : (s.len > 0 ? p.n_new : 0);
  const int most = min(p.n_new, s.len);
  if (s.n < 0 || s.n > most) { e |= ERR_NEW; s.n = min(max(s.n, 0), most); }
  if (e && report) atomicOr(p.err, e);
  return s;
}

inline cudaError_t launch_dep(void (*kernel)(AttendParams), dim3 grid, int threads, size_t smem, cudaStream_t st,
                       const AttendParams& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace vp
