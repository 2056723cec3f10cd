// What the int8 product's kernels share (gemm_int8.hip, gemm_int8_wide.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "internal.h"

namespace pgsr {

// Up to three products of the same X; their tile columns are numbered through.
struct Int8Args {
  int m, k, count;
  const uint8_t* x;
  const float* xs;
  const uint8_t* w[kGemmMulti];
  const float* ws[kGemmMulti];
  const uint16_t* r[kGemmMulti];
  uint16_t* y[kGemmMulti];
  int n[kGemmMulti];
};

// The product that a workgroup's tile column belongs to (columns of BN outputs, the
// products' numbered through); tn becomes the column within it.  Selects at constant
// places keep the pointers in scalar registers, which the requests need.
struct Int8Side {
  const uint8_t* w;
  const float* ws;
  const uint16_t* r;
  uint16_t* y;
  int n;
};
template <int BN>
__device__ __forceinline__ Int8Side int8_side(const Int8Args& a, int& tn) {
  Int8Side p{a.w[0], a.ws[0], a.r[0], a.y[0], a.n[0]};
#pragma unroll
  for (int i = 1; i < kGemmMulti; ++i)
    if (i < a.count && tn >= (p.n + BN - 1) / BN) {
      tn -= (p.n + BN - 1) / BN;
      p = Int8Side{a.w[i], a.ws[i], a.r[i], a.y[i], a.n[i]};
    }
  return p;
}

// One wave per SIMD and 256 x 256 tiles: K a multiple of 128.
hipError_t launch_gemm_int8_wide(const Int8Args& a, hipStream_t s);

}  // namespace pgsr
