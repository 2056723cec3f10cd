// What the int8 product's kernels share (gemm_int8.hip, gemm_int8_ring.hip,
// gemm_int8_wide.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <utility>

#include "elementwise.h"
#include "internal.h"

namespace pgsr {

namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kSub = 128;              // k of an image row (bytes)

template <class F, int... I>
__device__ __forceinline__ void static_for(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

// swizzle of the 16-byte chunk slot within a 128-byte image row
__device__ __forceinline__ int gsw(int row) { return (row >> 1) & 7; }

// all but this wave's latest N requests, and its LDS reads, complete
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// Four outputs of a row: the sums times their scales, plus four bf16 residuals.  Two
// roundings to fp32 in every kernel (left alone, some tiles' code fuses them into one,
// and a row's bits would depend on how many rows share its call).
__device__ __forceinline__ bf16x4 scaled(i32x4 sum, f32x4 scale, bool add, u32x2 r) {
#pragma clang fp contract(off)
  f32x4 v = __builtin_convertvector(sum, f32x4) * scale;
  if (add) v += f32x4{lo_bf16(r[0]), hi_bf16(r[0]), lo_bf16(r[1]), hi_bf16(r[1])};
  return __builtin_convertvector(v, bf16x4);
}

}  // namespace

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

// Tiles of 128 x 64, 128 x 128 and 256 x 128 (bm x bn), eight waves.
hipError_t launch_gemm_int8_ring(const Int8Args& a, int bm, int bn, hipStream_t s);
// One wave per SIMD and tiles of 256 x bn, bn 128 or 256: K a multiple of 128.
hipError_t launch_gemm_int8_wide(const Int8Args& a, int bn, hipStream_t s);

}  // namespace pgsr
