// Device helpers of the kernels that read caches held in 4 bits: codes as fp16
// numbers.
#pragma once

#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace vp {

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 unpack_f16(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }

// The whole numbers code - 8 of the codes in bits 0-3 and 16-19 (low), and of
// those in bits 4-7 and 20-23 (high), in the widely published way: the bits become the
// mantissa of 1024 and an addition takes the offset off, for the high ones with a factor
// of 1/16; the constants follow from fp16's format.  They are kept in registers: a mask
// and the exponent are one operation then.
struct Codes {
  uint32_t mask, mask_high, k1024, k1032, sixteenth, k72;
  __device__ __forceinline__ Codes() {
    asm volatile("mov.b32 %0, 0x000f000f;\n mov.b32 %1, 0x00f000f0;\n mov.b32 %2, 0x64006400;\n"
                 "mov.b32 %3, 0xe408e408;\n mov.b32 %4, 0x2c002c00;\n mov.b32 %5, 0xd480d480;\n"
                 : "=r"(mask), "=r"(mask_high), "=r"(k1024), "=r"(k1032), "=r"(sixteenth), "=r"(k72));
  }
  __device__ __forceinline__ uint32_t low(uint32_t x) const {
    uint32_t r;
    asm("{\n .reg .b32 y;\n lop3.b32 y, %1, %2, %3, 0xea;\n add.f16x2 %0, y, %4;\n}\n"  // 1024 + code
        : "=r"(r) : "r"(x), "r"(mask), "r"(k1024), "r"(k1032));
    return r;
  }
  __device__ __forceinline__ uint32_t high(uint32_t x) const {
    uint32_t r;
    asm("{\n .reg .b32 y;\n lop3.b32 y, %1, %2, %3, 0xea;\n fma.rn.f16x2 %0, y, %4, %5;\n}\n"  // 1024 + 16 code
        : "=r"(r) : "r"(x), "r"(mask_high), "r"(k1024), "r"(sixteenth), "r"(k72));
    return r;
  }
};

}  // namespace vp
