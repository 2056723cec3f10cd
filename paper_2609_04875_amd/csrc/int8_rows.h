// A row of an int8 KV cache from bf16 values (the formulas at the top of kv_int8.hip):
// the append kernel's and, for single tokens, the decode kernel's.
#pragma once

#include "attn_common.h"

namespace pgsr {
namespace {

constexpr int kExpLo = -100, kExpHi = 100;

// What eight values of a row give: the largest magnitude's bits, and whether one is NaN.
struct RowMax {
  uint32_t bits = 0;      // of |x|, an integer order
  bool nan = false;
};

__device__ inline void row_max(const uint16_t (&x)[8], RowMax& m) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t b = x[j] & 0x7FFFu;
    if (b > 0x7F80u) m.nan = true;
    else m.bits = max(m.bits, b);
  }
}

// e of a row whose largest magnitude has these bf16 bits
__device__ inline int row_exp(uint32_t bits) {
  return min(max((int)(bits >> 7) - 127 - 6, kExpLo), kExpHi);   // zeros and subnormals: the lowest
}

// Eight codes of x 2^-e, in element order.
__device__ inline u32x2 codes8(const uint16_t (&x)[8], int e, bool none) {
  const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
  u32x2 r = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float f = __uint_as_float((uint32_t)x[j] << 16) * inv;
    const float c = fminf(fmaxf(__builtin_rintf(f), -127.f), 127.f);
    const int code = none || f != f ? 0 : (int)c;
    r[j / 4] |= (uint32_t)(uint8_t)code << (8 * (j % 4));
  }
  return r;
}

// Over the lanes of C consecutive ones that hold a row of K and of V each: both maxima
// and the flag.  Magnitudes have 15 bits, so both go through one word.
template <int C>
__device__ inline uint32_t rows_max(const RowMax& k, const RowMax& v, int& nan) {
  uint32_t both = k.bits | (v.bits << 16);
  nan = k.nan || v.nan;
#pragma unroll
  for (int off = C / 2; off >= 1; off >>= 1) {
    const uint32_t o = __shfl_xor(both, off);
    both = max(both & 0xFFFFu, o & 0xFFFFu) | (max(both >> 16, o >> 16) << 16);
    nan |= __shfl_xor(nan, off);
  }
  return both;
}

__device__ inline void halves(const u32x4& w, uint16_t (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = (uint16_t)(w[j / 2] >> (16 * (j % 2)));
}

}  // namespace
}  // namespace pgsr
