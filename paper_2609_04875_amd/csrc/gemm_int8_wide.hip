// Dense int8 projection, large-product path: one wave per SIMD, each owning a 128 x
// 128 block of a 256 x 256 output tile (8 x 8 sub-tiles of 16 x 16, 256 int32
// accumulators in AGPRs).  The formula, the bits and the operand layout are those of
// gemm_int8.hip; the step's schedule is that of the bf16 kernel of the same tile
// (gemm_bf16_wide.hip), whose byte counts and issue slots an i8 product shares: it
// takes the same 16 bytes a lane of both operands and the same cycles.
//
// K advances 128 at a time.  A step needs a 256 x 128 tile of X and one of W (32 KB
// each, one 64 KB LDS buffer); two buffers alternate.  128 issue slots to a step (one
// product each): slots 0-31 read the operands of the step's second half, at slot 40 the
// wave waits for its requests of step kt + 1 and the workgroup meets at the step's one
// barrier, slots 40-100 issue the 16 requests of step kt + 2 into the buffer just read,
// slots 64-94 read the first operands of step kt + 1.
//
// Bound by the matrix units at the clock they leave (8192 x 8192 x 8192: 393 us, 2.8
// POP/s; the eight-wave 256 x 128 tiles of gemm_int8.hip 516) and, where K is short, by
// the stores of the tile, which all CUs send at once (7 of 54 us a tile at K = 4096).
#include <hip/hip_runtime.h>

#include <utility>

#include "gemm_int8.h"
#include "internal.h"

// The requests write M0 (the LDS address of a global->LDS load) from inline
// assembly that lists it as clobbered; nothing else in this file uses M0.
#pragma clang diagnostic ignored "-Winline-asm"

namespace pgsr {

namespace {

constexpr int kGB = 256;               // output tile edge (M and N)
constexpr int kGK = 128;               // K step (bytes of an image row)
constexpr int kGNB = 2;                // LDS buffers
constexpr int kGImg = kGB * kGK;       // bytes of one X or W image
constexpr int kGBuf = 2 * kGImg;       // bytes of one buffer (X image, then W image)
constexpr int kGRuns = 8;              // 1 KB runs per wave and image per step
constexpr int kGGroupM = 4;            // tile rows per group of the tile order

template <class F, int... I>
__device__ __forceinline__ void static_for(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

// swizzle of the 16-byte chunk slot within a 128-byte image row
__device__ __forceinline__ int gsw(int row) { return (row >> 1) & 7; }

__global__ void __launch_bounds__(256, 1)
gemm_int8_wide_kernel(Int8Args a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[kGNB * kGBuf];

  // output tile of this workgroup: XCD x = blockIdx % 8 takes tiles
  // [x * per_xcd, (x + 1) * per_xcd), in groups of kGGroupM tile rows
  const int M = a.m, K = a.k;
  const int n_tm = (M + kGB - 1) / kGB;
  int n_tn = 0;
#pragma unroll
  for (int i = 0; i < kGemmMulti; ++i) n_tn += i < a.count ? (a.n[i] + kGB - 1) / kGB : 0;
  const int per_xcd = (n_tm * n_tn + 7) / 8;
  const int t = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
  if (t >= n_tm * n_tn) return;
  const int grp = t / (kGGroupM * n_tn), first_m = grp * kGGroupM;
  const int gsize = min(n_tm - first_m, kGGroupM);
  const int idx = t - grp * kGGroupM * n_tn;
  const int m0 = (first_m + idx % gsize) * kGB;
  int tn = idx / gsize;
  const Int8Side p = int8_side<kGB>(a, tn);
  const int N = p.n, n0 = tn * kGB;

  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int wm = (w & 1) * 128, wn = (w >> 1) * 128;

  // Requests: wave w takes runs w, w + 4, ..., w + 28 of each image; run q =
  // rows 8 q .. 8 q + 7, lane l -> row 8 q + l / 8, slot l % 8, chunk
  // (l % 8) ^ gsw(row).  Rows past M or N read row M-1 or N-1 (their outputs
  // are never stored).  Byte offsets from the tile's first row.
  const char* const X0 = (const char*)a.x + (int64_t)m0 * K;
  const char* const W0 = (const char*)p.w + (int64_t)n0 * K;
  uint32_t xoff[kGRuns], woff[kGRuns];
#pragma unroll
  for (int j = 0; j < kGRuns; ++j) {
    const int row = 8 * (w + 4 * j) + lane / 8;
    const int c = (lane & 7) ^ gsw(row);
    xoff[j] = (uint32_t)(min(m0 + row, M - 1) - m0) * (uint32_t)K + 16u * c;
    woff[j] = (uint32_t)(min(n0 + row, N - 1) - n0) * (uint32_t)K + 16u * c;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)&lds[0] + 1024u * w;
  const int nk = K / kGK;
  // request q (0..15) of step kt: X run q (q < 8) or W run q - 8, into buffer
  // kt mod kGNB; steps past the last read the last step again (its buffer is
  // never read), so every step issues the same number of requests
  auto request = [&](int kt, int q) {
    const int ks = min(kt, nk - 1);
    const char* src = (q < 8 ? X0 : W0) + (int64_t)ks * kGK;
    const uint32_t img = lds0 + (uint32_t)((kt % kGNB) * kGBuf + (q < 8 ? 0 : kGImg)) + 4096u * (q & 7);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 :: "v"(q < 8 ? xoff[q & 7] : woff[q & 7]), "s"(src), "s"(img) : "memory", "m0");
  };

  // Operand reads: 16 rows x 64 k (slice ks) of rows base + r16, lane l ->
  // row l % 16, k group l / 16 (16 codes): chunk 4 ks + l / 16 of the row,
  // at slot (4 ks + l / 16) ^ gsw(r16) (every base is a multiple of 16)
  const int r16 = lane & 15, g4 = lane >> 4;
  int soff[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) soff[ks] = r16 * kGK + (((4 * ks + g4) ^ gsw(r16)) << 4);
  i32x4 wa[2][8], xb[2][8];
  // operand u (0..15) of slice ks: W sub-tile u / 2 (even u), X sub-tile u / 2 (odd u)
  auto read_op = [&](int buf, int ks, int u) {
    const uint8_t* img = &lds[buf * kGBuf + ((u & 1) ? 0 : kGImg)];
    const int base = ((u & 1) ? wm : wn) + 16 * (u >> 1);
    const i32x4 v = *(const i32x4*)&img[base * kGK + soff[ks]];
    if (u & 1) xb[ks][u >> 1] = v;
    else wa[ks][u >> 1] = v;
  };

  i32x4 acc[8][8];      // [n sub-tile][m sub-tile], element (n, m)
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = i32x4{};

  // prologue: steps 0 and 1 requested, step 0 landed, its slice-0 operands read
#pragma unroll
  for (int q = 0; q < 16; ++q) request(0, q);
#pragma unroll
  for (int q = 0; q < 16; ++q) request(1, q);
  asm volatile("s_waitcnt vmcnt(16)\n\ts_barrier" ::: "memory");
#pragma unroll
  for (int u = 0; u < 16; ++u) read_op(0, 0, u);

  // step kt with its buffer parity CUR known at compile time, so that every
  // operand address is a loop-invariant register plus an immediate
  auto step = [&](auto cur_c, int kt) {
    constexpr int cur = decltype(cur_c)::value, nxt = 1 - cur;
    auto slot = [&](auto ic) {
      constexpr int s = decltype(ic)::value;
      constexpr int ks = s / 64, i = (s / 8) % 8, j = s % 8;
      if constexpr (s == 40) {
        // step kt + 1 landed (this wave's requests, and the barrier for the
        // other waves'), and every wave has read all of step kt's buffer,
        // which the requests below refill with step kt + 2
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      }
      if constexpr (s < 32 && s % 2 == 0) read_op(cur, 1, s / 2);
      else if constexpr (s >= 64 && s < 96 && s % 2 == 0) read_op(nxt, 0, (s - 64) / 2);
      if constexpr (s >= 40 && s < 104 && s % 4 == 0) request(kt + 2, (s - 40) / 4);
      asm("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc[i][j]) : "v"(wa[ks][i]), "v"(xb[ks][j]));
      __builtin_amdgcn_sched_barrier(0);
    };
    static_for(slot, std::make_integer_sequence<int, 128>{});
  };
  int kt = 0;
  for (; kt + 1 < nk; kt += 2) {
    step(std::integral_constant<int, 0>{}, kt);
    step(std::integral_constant<int, 1>{}, kt + 1);
  }
  if (kt < nk) step(std::integral_constant<int, 0>{}, kt);
  // 19 wait states before any VALU read of the accumulators (the epilogue
  // reads each m sub-tile's after an assembly statement ordered after this)
  asm volatile("s_nop 15\n\ts_nop 3" ::: "memory");
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // requests past the end, before LDS is handed on

  // acc[i][j] lane l, register q: n = wn + 16 i + 4 (l / 16) + q, m = wm + 16 j + l % 16.
  // Scales, and a row's residuals, are asked for ahead of the stores that could (as far
  // as the compiler knows) change them: one at a time the tile's epilogue took 20 us.
  const int nb = n0 + wn + 4 * g4;                 // N is a multiple of 8: whole groups in or out
  f32x4 wsc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) wsc[i] = *(const f32x4*)(p.ws + min(nb + 16 * i, N - 4));
  float xsc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) xsc[j] = a.xs[min(m0 + wm + 16 * j + r16, M - 1)];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    // one m sub-tile's accumulators at a time: they count as written here, so
    // their reads cannot move above the previous sub-tile's stores
    asm volatile("" : "+a"(acc[0][j]), "+a"(acc[1][j]), "+a"(acc[2][j]), "+a"(acc[3][j]),
                 "+a"(acc[4][j]), "+a"(acc[5][j]), "+a"(acc[6][j]), "+a"(acc[7][j]) :: "memory");
    const int m = m0 + wm + 16 * j + r16;
    if (m >= M) continue;
    const int64_t row = (int64_t)m * N;
    u32x2 rb[8];
    if (p.r) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (nb + 16 * i < N) rb[i] = *(const u32x2*)(p.r + row + nb + 16 * i);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (nb + 16 * i >= N) continue;
      *(bf16x4*)(p.y + row + nb + 16 * i) = scaled(acc[i][j], xsc[j] * wsc[i], p.r != nullptr, rb[i]);
    }
  }
}

}  // namespace

hipError_t launch_gemm_int8_wide(const Int8Args& a, hipStream_t s) {
  if (a.k <= 0 || a.k % kGK != 0) return hipErrorInvalidValue;
  int64_t cols = 0;
  for (int i = 0; i < a.count; ++i) cols += (a.n[i] + kGB - 1) / kGB;
  const int64_t tiles = (int64_t)((a.m + kGB - 1) / kGB) * cols;
  hipLaunchKernelGGL(gemm_int8_wide_kernel, dim3((unsigned)(8 * ((tiles + 7) / 8))), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace pgsr
