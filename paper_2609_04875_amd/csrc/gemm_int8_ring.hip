// Int8 product, middle sizes: eight waves share 128 x 64 to 256 x 128 outputs.  The
// formula, the bits and the operand layout are those of gemm_int8.hip.
//
// X and W come to LDS by global->LDS loads through a ring of NST stages, in the scheme
// of the bf16 kernels (gemm_bf16_dma.hip): a stage is KSUB images of 128 k (128-byte
// rows of X, then of W), a request 8 rows x 128 bytes with chunk c of row j in slot
// c ^ ((j / 2) mod 8); a wave waits for its own requests of the next stage (vmcnt,
// exact), meets the others at one barrier, reads the next operand group and refills the
// slot that the barrier freed, ahead of the products of the operands in registers.  An
// instruction takes the same bytes of both operands and the same cycles as the bf16 one
// and does twice the work, so a stage of 128 k costs what one of 64 k costs there.
// Bound like gemm_int8.hip by the lines a CU can have on their way (333 x 3584 x 18944:
// 55 us, 24 KB of both operands a 128-k step in 348 ns).
#include <hip/hip_runtime.h>

#include <utility>

#include "gemm_int8.h"
#include "internal.h"

// The requests write M0 (the LDS address of a global->LDS load) from inline
// assembly that lists it as clobbered; nothing else in this file uses M0.
#pragma clang diagnostic ignored "-Winline-asm"

namespace pgsr {

namespace {

// ONCE: one tile row, so no other tile reads this W: non-temporal requests.
template <int BM, int BN, int WGM, int WGN, int KSUB, int NST, int GS, int GM, bool ONCE>
__global__ void __launch_bounds__(WGM * WGN * 64, 1) gemm_int8_ring_kernel(Int8Args a) {
  constexpr int NW = WGM * WGN;
  constexpr int TM = BM / WGM / 16, TN = BN / WGN / 16;
  constexpr int XR = BM / 8 / NW, WR = BN / 8 / NW;       // 1 KB runs per wave and sub-image
  static_assert(XR * NW * 8 == BM && WR * NW * 8 == BN, "runs split evenly over the waves");
  constexpr int RPW = KSUB * (XR + WR);                    // requests per wave and stage
  static_assert(RPW * (NST - 1) <= 63, "vmcnt range");
  constexpr int SUBE = (BM + BN) * kSub, STE = KSUB * SUBE;   // bytes of a sub-image pair, a stage
  constexpr int KST = kSub * KSUB;                         // k of a stage
  constexpr int NKS = 2 * KSUB;                            // k slices of 64 per stage
  constexpr int NG = NKS / GS;                             // operand groups of GS slices per stage
  static_assert(NKS % GS == 0 && (NG == 1 || NG % 2 == 0), "operand groups");
  __shared__ __attribute__((aligned(16))) uint8_t lds[NST * STE];

  // output tile of this workgroup: XCD x = blockIdx % 8 takes tiles
  // [x * per_xcd, (x + 1) * per_xcd), in groups of GM tile rows (the tile rows
  // of one W panel run side by side on one XCD, so its L2 takes W once)
  const int M = a.m, K = a.k;
  const int n_tm = (M + BM - 1) / BM;
  int n_tn = 0;
#pragma unroll
  for (int i = 0; i < kGemmMulti; ++i) n_tn += i < a.count ? (a.n[i] + BN - 1) / BN : 0;
  const int per_xcd = (n_tm * n_tn + 7) / 8;
  const int t = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
  if (t >= n_tm * n_tn) return;
  const int grp = t / (GM * n_tn), first_m = grp * GM;
  const int gsize = min(n_tm - first_m, GM);
  const int idx = t - grp * GM * n_tn;
  const int m0 = (first_m + idx % gsize) * BM;
  int tn = idx / gsize;
  const Int8Side p = int8_side<BN>(a, tn);
  const int N = p.n;
  const int n0 = tn * BN;

  const int tid = threadIdx.x;
  const int w = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, r16 = lane & 15, g4 = lane >> 4;
  const int wm = (w % WGM) * TM * 16, wn = (w / WGM) * TN * 16;

  // This lane's requests: run j holds rows 8 (w + NW j) + lane / 8; rows past M or
  // N read row M-1 or N-1 (never stored).  Offsets from the tile's first row.
  const char* const X0 = (const char*)a.x + (int64_t)m0 * K;
  const char* const W0 = (const char*)p.w + (int64_t)n0 * K;
  uint32_t xrow[XR], wrow[WR];
  int xc[XR], wc[WR];                              // chunk of the image row this lane fetches
#pragma unroll
  for (int j = 0; j < XR; ++j) {
    const int row = 8 * (w + NW * j) + lane / 8;
    xrow[j] = (uint32_t)(min(m0 + row, M - 1) - m0) * (uint32_t)K;
    xc[j] = (lane & 7) ^ gsw(row);
  }
#pragma unroll
  for (int j = 0; j < WR; ++j) {
    const int row = 8 * (w + NW * j) + lane / 8;
    wrow[j] = (uint32_t)(min(n0 + row, N - 1) - n0) * (uint32_t)K;
    wc[j] = (lane & 7) ^ gsw(row);
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)&lds[0] + 1024u * w;
  const int nst = (K + KST - 1) / KST;
  const int last_chunks = (K - (nst - 1) * KST) / 16;      // of the last stage, 1 .. 8 KSUB
  auto request = [&](int st, int slot) {
    const char* xs = X0 + (int64_t)st * KST;
    const char* ws = W0 + (int64_t)st * KST;
    const uint32_t img = lds0 + (uint32_t)(slot * STE);
    const int most = (st == nst - 1 ? last_chunks : 8 * KSUB) - 1;
#pragma unroll
    for (int sub = 0; sub < KSUB; ++sub) {
#pragma unroll
      for (int j = 0; j < WR; ++j) {
        const uint32_t off = wrow[j] + 16u * (uint32_t)min(8 * sub + wc[j], most);
        if constexpr (ONCE)
          asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt"
                       ::"v"(off), "s"(ws), "s"(img + (uint32_t)(sub * SUBE + BM * kSub) + 1024u * NW * j)
                       : "memory", "m0");
        else
          asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                       ::"v"(off), "s"(ws), "s"(img + (uint32_t)(sub * SUBE + BM * kSub) + 1024u * NW * j)
                       : "memory", "m0");
      }
#pragma unroll
      for (int j = 0; j < XR; ++j) {
        const uint32_t off = xrow[j] + 16u * (uint32_t)min(8 * sub + xc[j], most);
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                     ::"v"(off), "s"(xs), "s"(img + (uint32_t)(sub * SUBE) + 1024u * NW * j)
                     : "memory", "m0");
      }
    }
  };
  // this wave's requests complete but for those of the latest `ahead` stages
  // (its LDS reads too), and every other wave's at the barrier
  auto landed = [&](int ahead) {
    if (ahead >= NST - 2) wait_loads<RPW * (NST - 2)>();
    else
      static_for([&](auto ic) { if (ahead == decltype(ic)::value) wait_loads<RPW * decltype(ic)::value>(); },
                 std::make_integer_sequence<int, (NST > 2 ? NST - 2 : 1)>{});
    if constexpr (NW > 1) asm volatile("s_barrier" ::: "memory");
  };

  // operand = 16 rows x 64 k: lane l -> row l % 16, chunk l / 16 of the slice
  int soff[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) soff[h] = r16 * kSub + (((4 * h + g4) ^ gsw(r16)) << 4);
  i32x4 wa[2][GS][TN], xb[2][GS][TM];
  // operand group grp of the stage in `slot`; `last`: its chunks of X past K are cleared
  auto read_ops = [&](int slot, int grp, bool last, auto set_c) {
    constexpr int set = decltype(set_c)::value;
#pragma unroll
    for (int h = 0; h < GS; ++h) {
      const int ks = grp * GS + h;
      const uint8_t* img = &lds[slot * STE + (ks / 2) * SUBE];
#pragma unroll
      for (int i = 0; i < TN; ++i) wa[set][h][i] = *(const i32x4*)&img[(BM + wn + 16 * i) * kSub + soff[ks & 1]];
#pragma unroll
      for (int j = 0; j < TM; ++j) xb[set][h][j] = *(const i32x4*)&img[(wm + 16 * j) * kSub + soff[ks & 1]];
    }
    if (last) {
#pragma unroll
      for (int h = 0; h < GS; ++h) {
        const bool in = 4 * (grp * GS + h) + g4 < last_chunks;
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) xb[set][h][j][q] = in ? xb[set][h][j][q] : 0;
      }
    }
  };

  i32x4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = i32x4{};

  const bool ragged = last_chunks != 8 * KSUB;
#pragma unroll
  for (int st = 0; st < NST - 1; ++st)
    if (st < nst) request(st, st);
  landed(min(NST - 1, nst) - 1);
  if (NST - 1 < nst) request(NST - 1, NST - 1);
  read_ops(0, 0, ragged && nst == 1, std::integral_constant<int, 0>{});

  int slot = 0;
  // stage s from ring slot `slot`, its first operand group in set par
  auto stage = [&](int s, auto par_c) {
    constexpr int par = decltype(par_c)::value;
    const int nslot = slot + 1 == NST ? 0 : slot + 1;
    static_for([&](auto gc) {
      constexpr int g = decltype(gc)::value, cur = (par + g) & 1;
      if constexpr (g < NG - 1) {
        read_ops(slot, g + 1, ragged && s == nst - 1, std::integral_constant<int, 1 - cur>{});
      } else if (s + 1 < nst) {
        landed(min(NST - 2, nst - 2 - s));
        read_ops(nslot, 0, ragged && s == nst - 2, std::integral_constant<int, 1 - cur>{});
        if (s + NST < nst) request(s + NST, slot);
      }
#pragma unroll
      for (int h = 0; h < GS; ++h)
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int j = 0; j < TM; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wa[cur][h][i], xb[cur][h][j], acc[i][j], 0, 0, 0);
    }, std::make_integer_sequence<int, NG>{});
    slot = nslot;
  };
  int s = 0;
  for (; s + 1 < nst; s += 2) {
    stage(s, std::integral_constant<int, 0>{});
    stage(s + 1, std::integral_constant<int, NG & 1>{});
  }
  if (s < nst) stage(s, std::integral_constant<int, 0>{});

  // acc[i][j] lane l, register q: n = wn + 16 i + 4 (l / 16) + q, m = wm + 16 j + l % 16.
  // Scales, and a row's residuals, are asked for ahead of the stores that could (as far
  // as the compiler knows) change them.
  const int nb = n0 + wn + 4 * g4;                 // N is a multiple of 8: whole groups in or out
  f32x4 wsc[TN];
#pragma unroll
  for (int i = 0; i < TN; ++i) wsc[i] = *(const f32x4*)(p.ws + min(nb + 16 * i, N - 4));
  float xsc[TM];
#pragma unroll
  for (int j = 0; j < TM; ++j) xsc[j] = a.xs[min(m0 + wm + 16 * j + r16, M - 1)];
#pragma unroll
  for (int j = 0; j < TM; ++j) {
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

template <int BM, int BN, int WGM, int WGN, int KSUB, int NST, int GS, int GM>
void launch_tile(const Int8Args& a, hipStream_t s) {
  int64_t cols = 0;
  for (int i = 0; i < a.count; ++i) cols += (a.n[i] + BN - 1) / BN;
  const int64_t tiles = (int64_t)((a.m + BM - 1) / BM) * cols;
  const dim3 grid((unsigned)(8 * ((tiles + 7) / 8))), blk(WGM * WGN * 64);
  if (a.m <= BM)
    hipLaunchKernelGGL((gemm_int8_ring_kernel<BM, BN, WGM, WGN, KSUB, NST, GS, GM, true>), grid, blk, 0, s, a);
  else
    hipLaunchKernelGGL((gemm_int8_ring_kernel<BM, BN, WGM, WGN, KSUB, NST, GS, GM, false>), grid, blk, 0, s, a);
}

}  // namespace

hipError_t launch_gemm_int8_ring(const Int8Args& a, int bm, int bn, hipStream_t s) {
  if (bm == 128 && bn == 64) launch_tile<128, 64, 4, 2, 2, 3, 2, 8>(a, s);
  else if (bm == 128 && bn == 128) launch_tile<128, 128, 4, 2, 1, 4, 1, 8>(a, s);
  else if (bm == 256 && bn == 128) launch_tile<256, 128, 4, 2, 1, 3, 1, 4>(a, s);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pgsr
