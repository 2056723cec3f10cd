// Dense int8 projection, large-product path: one wave per SIMD, each owning 128 rows and
// half the columns of a 256 x 256 output tile (8 x 8 sub-tiles of 16 x 16, 256 int32
// accumulators in AGPRs) or of a 256 x 128 one (8 x 4).  The formula, the bits and the
// operand layout are those of gemm_int8.hip; the step's schedule is that of the bf16
// kernel of the same tile (gemm_bf16_wide.hip), whose byte counts and issue slots an i8
// product shares: it takes the same 16 bytes a lane of both operands and the same cycles.
//
// K advances 128 at a time.  A step needs a 256 x 128 image of X and one of W (64 KB
// with 256 columns, two buffers alternate; 48 KB with 128, three).  A step has an issue
// slot for each product, 128 or 64: the first ones read the operands of the step's second
// half, at slot 40 (26) the wave waits for its requests of step kt + 1 and the workgroup
// meets at the step's one barrier, then it issues its 16 (12) requests of the step that
// takes the buffer just read, and from the middle on it reads the first operands of step
// kt + 1.  With 128 columns a request has two steps of 64 products to land instead of
// one of 128: the same time.
//
// Bound by the matrix units at the clock they leave (8192 x 8192 x 8192: 383 us, 2.9
// POP/s; eight waves on 256 x 128 516) and, where K is short, by the stores of the tile,
// which all CUs send at once (7 of 54 us a tile at K = 4096).  256 x 128 where that fills
// the CUs and 256 x 256 does not: 2048 x 3584 x 18944 116 us (eight waves 138, 256 x 256
// 180), 2048 x 4096 x 14336 95 (116, 143), 2048 x 4096 x 4096 32.7 (37, 45); a CU then
// takes 48 KB a step in 780 ns, about what it can have on its way (gemm_int8.hip).
#include <hip/hip_runtime.h>

#include <utility>

#include "gemm_int8.h"
#include "internal.h"

// The requests write M0 (the LDS address of a global->LDS load) from inline
// assembly that lists it as clobbered; nothing else in this file uses M0.
#pragma clang diagnostic ignored "-Winline-asm"

namespace pgsr {

namespace {

constexpr int kGM = 256;               // tile rows
constexpr int kXImg = kGM * kSub;      // bytes of an X image
constexpr int kXRuns = kGM / 32;       // its 1 KB runs per wave and step
constexpr int kGGroupM = 4;            // tile rows per group of the tile order

template <int BN>
__global__ void __launch_bounds__(256, 1)
gemm_int8_wide_kernel(Int8Args a) {
  constexpr int TN = BN / 32;                      // n sub-tiles of a wave (and 8 m sub-tiles)
  constexpr int WR = BN / 32;                      // 1 KB runs of W per wave and step
  constexpr int NB = BN == 256 ? 2 : 3;            // LDS buffers
  constexpr int BUF = kXImg + BN * kSub;           // bytes of one (X image, then W image)
  constexpr int RPS = kXRuns + WR;                 // requests of a wave and step
  constexpr int OPS = 8 + TN;                      // operands of a slice
  constexpr int SLOTS = 2 * 8 * TN;                // products of a step
  constexpr int MEET = BN == 256 ? 40 : 26;        // slot of the barrier
  constexpr int GAP = BN == 256 ? 4 : 3;           // slots from request to request
  static_assert(2 * OPS <= MEET && MEET + GAP * (RPS - 1) < SLOTS && 2 * OPS <= SLOTS / 2, "slots of a step");
  __shared__ __attribute__((aligned(16))) uint8_t lds[NB * BUF];

  // output tile of this workgroup: XCD x = blockIdx % 8 takes tiles
  // [x * per_xcd, (x + 1) * per_xcd), in groups of kGGroupM tile rows
  const int M = a.m, K = a.k;
  const int n_tm = (M + kGM - 1) / kGM;
  int n_tn = 0;
#pragma unroll
  for (int i = 0; i < kGemmMulti; ++i) n_tn += i < a.count ? (a.n[i] + BN - 1) / BN : 0;
  const int per_xcd = (n_tm * n_tn + 7) / 8;
  const int t = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
  if (t >= n_tm * n_tn) return;
  const int grp = t / (kGGroupM * n_tn), first_m = grp * kGGroupM;
  const int gsize = min(n_tm - first_m, kGGroupM);
  const int idx = t - grp * kGGroupM * n_tn;
  const int m0 = (first_m + idx % gsize) * kGM;
  int tn = idx / gsize;
  const Int8Side p = int8_side<BN>(a, tn);
  const int N = p.n, n0 = tn * BN;

  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int wm = (w & 1) * 128, wn = (w >> 1) * (BN / 2);

  // Requests: wave w takes runs w, w + 4, ... of each image; run q = rows 8 q ..
  // 8 q + 7, lane l -> row 8 q + l / 8, slot l % 8, chunk (l % 8) ^ gsw(row).  Rows
  // past M or N read row M-1 or N-1 (their outputs are never stored).  Byte offsets
  // from the tile's first row.
  const char* const X0 = (const char*)a.x + (int64_t)m0 * K;
  const char* const W0 = (const char*)p.w + (int64_t)n0 * K;
  uint32_t xoff[kXRuns], woff[WR];
#pragma unroll
  for (int j = 0; j < kXRuns; ++j) {
    const int row = 8 * (w + 4 * j) + lane / 8;
    const uint32_t c = 16u * ((lane & 7) ^ gsw(row));
    xoff[j] = (uint32_t)(min(m0 + row, M - 1) - m0) * (uint32_t)K + c;
    if (j < WR) woff[j] = (uint32_t)(min(n0 + row, N - 1) - n0) * (uint32_t)K + c;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)&lds[0] + 1024u * w;
  const int nk = K / kSub;
  // request q of step kt: X run q or W run q - kXRuns, into buffer `buf` = kt mod NB;
  // steps past the last read the last step again (its buffer is never read), so every
  // step issues the same number of requests
  auto request = [&](int kt, int buf, int q) {
    const bool x = q < kXRuns;
    const int j = x ? q : q - kXRuns;
    const char* src = (x ? X0 : W0) + (int64_t)min(kt, nk - 1) * kSub;
    const uint32_t img = lds0 + (uint32_t)(buf * BUF + (x ? 0 : kXImg)) + 4096u * j;
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 :: "v"(x ? xoff[j] : woff[x ? 0 : j]), "s"(src), "s"(img) : "memory", "m0");
  };

  // Operand reads: 16 rows x 64 k (slice ks) of rows base + r16, lane l ->
  // row l % 16, k group l / 16 (16 codes): chunk 4 ks + l / 16 of the row,
  // at slot (4 ks + l / 16) ^ gsw(r16) (every base is a multiple of 16)
  const int r16 = lane & 15, g4 = lane >> 4;
  int soff[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) soff[ks] = r16 * kSub + (((4 * ks + g4) ^ gsw(r16)) << 4);
  i32x4 wa[2][TN], xb[2][8];
  // operand u of slice ks: W and X sub-tiles in turn, then the rest of X
  auto read_op = [&](int buf, int ks, int u) {
    const bool x = u >= 2 * TN || (u & 1);
    const int j = u >= 2 * TN ? u - TN : u / 2;
    const uint8_t* img = &lds[buf * BUF + (x ? 0 : kXImg)];
    const i32x4 v = *(const i32x4*)&img[((x ? wm : wn) + 16 * j) * kSub + soff[ks]];
    if (x) xb[ks][j] = v;
    else wa[ks][x ? 0 : j] = v;
  };

  i32x4 acc[TN][8];     // [n sub-tile][m sub-tile], element (n, m)
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = i32x4{};

  // prologue: the first NB steps requested, step 0 landed, its slice-0 operands read
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int q = 0; q < RPS; ++q) request(b, b, q);
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(RPS * (NB - 1)) : "memory");
#pragma unroll
  for (int u = 0; u < OPS; ++u) read_op(0, 0, u);

  // step kt with its buffer CUR known at compile time, so that every operand address
  // is a loop-invariant register plus an immediate
  auto step = [&](auto cur_c, int kt) __attribute__((always_inline)) {
    constexpr int cur = decltype(cur_c)::value, nxt = cur + 1 == NB ? 0 : cur + 1;
    auto slot = [&](auto ic) __attribute__((always_inline)) {
      constexpr int s = decltype(ic)::value, half = SLOTS / 2;
      constexpr int ks = s / half, i = (s / 8) % TN, j = s % 8;
      if constexpr (s == MEET) {
        // step kt + 1 landed (this wave's requests but for the later steps', and the
        // barrier for the other waves'), and every wave has read all of step kt's
        // buffer, which the requests below refill with step kt + NB
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(RPS * (NB - 2)) : "memory");
      }
      if constexpr (s < 2 * OPS && s % 2 == 0) read_op(cur, 1, s / 2);
      else if constexpr (s >= half && s < half + 2 * OPS && s % 2 == 0) read_op(nxt, 0, (s - half) / 2);
      if constexpr (s >= MEET && s < MEET + GAP * RPS && (s - MEET) % GAP == 0) request(kt + NB, cur, (s - MEET) / GAP);
      asm("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc[i][j]) : "v"(wa[ks][i]), "v"(xb[ks][j]));
      __builtin_amdgcn_sched_barrier(0);
    };
    static_for(slot, std::make_integer_sequence<int, SLOTS>{});
  };
  int kt = 0;
  for (; kt + NB <= nk; kt += NB) {
    step(std::integral_constant<int, 0>{}, kt);
    step(std::integral_constant<int, 1>{}, kt + 1);
    if constexpr (NB == 3) step(std::integral_constant<int, 2>{}, kt + 2);
  }
  if (kt < nk) step(std::integral_constant<int, 0>{}, kt);
  if constexpr (NB == 3)
    if (kt + 1 < nk) step(std::integral_constant<int, 1>{}, kt + 1);
  // 19 wait states before any VALU read of the accumulators (the epilogue
  // reads each m sub-tile's after an assembly statement ordered after this)
  asm volatile("s_nop 15\n\ts_nop 3" ::: "memory");
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // requests past the end, before LDS is handed on

  // acc[i][j] lane l, register q: n = wn + 16 i + 4 (l / 16) + q, m = wm + 16 j + l % 16.
  // Scales, and a row's residuals, are asked for ahead of the stores that could (as far
  // as the compiler knows) change them: one at a time the tile's epilogue took 20 us.
  const int nb = n0 + wn + 4 * g4;                 // N is a multiple of 8: whole groups in or out
  f32x4 wsc[TN];
#pragma unroll
  for (int i = 0; i < TN; ++i) wsc[i] = *(const f32x4*)(p.ws + min(nb + 16 * i, N - 4));
  float xsc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) xsc[j] = a.xs[min(m0 + wm + 16 * j + r16, M - 1)];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    // one m sub-tile's accumulators at a time: they count as written here, so
    // their reads cannot move above the previous sub-tile's stores
#pragma unroll
    for (int i = 0; i < TN; ++i) asm volatile("" : "+a"(acc[i][j])::"memory");
    const int m = m0 + wm + 16 * j + r16;
    if (m >= M) continue;
    const int64_t row = (int64_t)m * N;
    u32x2 rb[TN];
    if (p.r) {
#pragma unroll
      for (int i = 0; i < TN; ++i)
        if (nb + 16 * i < N) rb[i] = *(const u32x2*)(p.r + row + nb + 16 * i);
    }
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      if (nb + 16 * i >= N) continue;
      *(bf16x4*)(p.y + row + nb + 16 * i) = scaled(acc[i][j], xsc[j] * wsc[i], p.r != nullptr, rb[i]);
    }
  }
}

}  // namespace

hipError_t launch_gemm_int8_wide(const Int8Args& a, int bn, hipStream_t s) {
  if (a.k <= 0 || a.k % kSub != 0) return hipErrorInvalidValue;
  int64_t cols = 0;
  for (int i = 0; i < a.count; ++i) cols += (a.n[i] + bn - 1) / bn;
  const int64_t tiles = (int64_t)((a.m + kGM - 1) / kGM) * cols;
  const dim3 grid((unsigned)(8 * ((tiles + 7) / 8)));
  if (bn == 256) hipLaunchKernelGGL(gemm_int8_wide_kernel<256>, grid, dim3(256), 0, s, a);
  else if (bn == 128) hipLaunchKernelGGL(gemm_int8_wide_kernel<128>, grid, dim3(256), 0, s, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pgsr
