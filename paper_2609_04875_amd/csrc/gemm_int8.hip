// Dense int8 projection Y = (Xq Wq^T) * xs * ws (+ R): codes with a scale for each
// token (row of X) and each output channel (row of W, [n][k]), exact int32 sums on
// v_mfma_i32_16x16x64_i8, one rounding to bf16.
//
//   Y[m][n] = bf16(float(sum_k Xq[m][k] Wq[n][k]) * (xs[m] * ws[n]) + R[m][n])
//
// |sum| <= 127^2 k stays below 2^31 for k up to 133144, which the host checks; the
// conversion to fp32 rounds sums past 2^24 by half a step of fp32.  Integer sums have no
// order, so a result depends on no tile, and rows not on which rows share the launch.
//
// This file: the choice of the tile, and the kernel of tiles from 16 x 16 to 96 x 64.
// Its four waves share the tile's outputs and split K: wave w takes the 128-k stages
// w, w + 4, ... through a ring of its own in LDS (global->LDS loads: a request is 8 rows
// x 128 bytes, chunk c of row j in slot c ^ ((j / 2) mod 8)), waits for its own requests
// alone, and meets the others at the end, where they add up their sums.  No barrier in
// the loop, each byte read from LDS once, and four stages of K at a time from a handful
// of rows: against four waves that split the outputs, 1 x 3584 x 18944 17.2 -> 12.4 us,
// 1 x 28672 x 4096 22.8 -> 19.5, 102 x 4096 x 14336 24.4 -> 23.7, 200 rows 30.3 -> 28.5.
// (96 x 64, all of the LDS: 316 rows 34.1, the ring of 128 x 64 tiles 41.5.)
// Few rows stream W from HBM once.  From 64 rows on what bounds it is the lines that a
// CU can have on their way: about 100 of 128 bytes, each 370 to 490 cycles on average
// where a quarter come from HBM (102 x 3584 x 18944: 70 GB/s a CU; 125 with every line
// in L2), so larger tiles pay as soon as they fill the CUs, and LDS or the products do
// not.
//
// K any multiple of 16: the last stage clamps the chunks past K to the row's last
// one, and their operands of X are cleared in registers (W's may hold anything:
// integers times 0).  Addresses are a 64-bit tile origin and 32-bit offsets inside the
// tile, so sizes are bounded by memory alone.
#include <hip/hip_runtime.h>

#include <cmath>
#include <utility>

#include "gemm_int8.h"
#include "internal.h"

// The requests write M0 (the LDS address of a global->LDS load) from inline
// assembly that lists it as clobbered; nothing else in this file uses M0.
#pragma clang diagnostic ignored "-Winline-asm"

namespace pgsr {

namespace {

constexpr int kCus = 256;
constexpr int kWaves = 4;
constexpr int kGroupM = 8;             // tile rows per group of the tile order

// ONCE: one tile row, so no other tile reads this W: non-temporal requests.
template <int BM, int BN, int NST, bool ONCE>
__global__ void __launch_bounds__(kWaves * 64, 1) gemm_int8_kernel(Int8Args a) {
  constexpr int TM = BM / 16, TN = BN / 16;
  constexpr int XR = BM / 8, WR = BN / 8;                  // requests of 8 rows x 128 bytes
  constexpr int RPS = XR + WR;                             // a wave's, of one stage
  static_assert(RPS * (NST - 1) <= 63, "vmcnt range");
  constexpr int STE = (BM + BN) * kSub;                    // bytes of a stage: rows of X, then of W
  constexpr int RING = kWaves * NST * STE, SUMS = TM * TN * kWaves * 1024;
  __shared__ __attribute__((aligned(16))) uint8_t lds[RING > SUMS ? RING : SUMS];

  // output tile of this workgroup: XCD x = blockIdx % 8 takes tiles
  // [x * per_xcd, (x + 1) * per_xcd), in groups of kGroupM tile rows (the tile rows
  // of one W panel run side by side on one XCD, so its L2 takes W once)
  const int M = a.m, K = a.k;
  const int n_tm = (M + BM - 1) / BM;
  int n_tn = 0;
#pragma unroll
  for (int i = 0; i < kGemmMulti; ++i) n_tn += i < a.count ? (a.n[i] + BN - 1) / BN : 0;
  const int per_xcd = (n_tm * n_tn + 7) / 8;
  const int t = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
  if (t >= n_tm * n_tn) return;
  const int grp = t / (kGroupM * n_tn), first_m = grp * kGroupM;
  const int gsize = min(n_tm - first_m, kGroupM);
  const int idx = t - grp * kGroupM * n_tn;
  const int m0 = (first_m + idx % gsize) * BM;
  int tn = idx / gsize;
  const Int8Side p = int8_side<BN>(a, tn);
  const int N = p.n;
  const int n0 = tn * BN;

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, r16 = lane & 15, g4 = lane >> 4;

  // This lane's requests: run j holds rows 8 j + lane / 8; rows past M or N read row
  // M-1 or N-1 (never stored).  Offsets from the tile's first row.
  const char* const X0 = (const char*)a.x + (int64_t)m0 * K;
  const char* const W0 = (const char*)p.w + (int64_t)n0 * K;
  uint32_t xrow[XR], wrow[WR];
#pragma unroll
  for (int j = 0; j < XR; ++j) xrow[j] = (uint32_t)(min(m0 + 8 * j + lane / 8, M - 1) - m0) * (uint32_t)K;
#pragma unroll
  for (int j = 0; j < WR; ++j) wrow[j] = (uint32_t)(min(n0 + 8 * j + lane / 8, N - 1) - n0) * (uint32_t)K;
  // chunk of the image row this lane fetches, even and odd runs
  const int chunk[2] = {(lane & 7) ^ gsw(lane / 8), (lane & 7) ^ gsw(8 + lane / 8)};
  const uint32_t lds0 = (uint32_t)(uintptr_t)&lds[0] + (uint32_t)(w * NST * STE);
  const int nst = (K + kSub - 1) / kSub;
  const int last_chunks = (K - (nst - 1) * kSub) / 16;     // of the last stage, 1 .. 8
  const int mine = (nst - w + kWaves - 1) / kWaves;        // this wave's stages: w, w + kWaves, ..
  auto request = [&](int i, int slot) {
    const int st = w + kWaves * i;
    const char* xs = X0 + (int64_t)st * kSub;
    const char* ws = W0 + (int64_t)st * kSub;
    const uint32_t img = lds0 + (uint32_t)(slot * STE);
    const int most = (st == nst - 1 ? last_chunks : 8) - 1;
    const uint32_t c[2] = {16u * (uint32_t)min(chunk[0], most), 16u * (uint32_t)min(chunk[1], most)};
#pragma unroll
    for (int j = 0; j < WR; ++j) {
      if constexpr (ONCE)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt"
                     ::"v"(wrow[j] + c[j & 1]), "s"(ws), "s"(img + (uint32_t)(BM * kSub + 1024 * j)) : "memory", "m0");
      else
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                     ::"v"(wrow[j] + c[j & 1]), "s"(ws), "s"(img + (uint32_t)(BM * kSub + 1024 * j)) : "memory", "m0");
    }
#pragma unroll
    for (int j = 0; j < XR; ++j)
      asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                   ::"v"(xrow[j] + c[j & 1]), "s"(xs), "s"(img + (uint32_t)(1024 * j)) : "memory", "m0");
  };
  // this wave's requests complete but for those of the latest `ahead` stages
  auto landed = [&](int ahead) {
    static_for([&](auto ic) { if (ahead == decltype(ic)::value) wait_loads<RPS * decltype(ic)::value>(); },
               std::make_integer_sequence<int, NST>{});
  };

  i32x4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = i32x4{};

#pragma unroll
  for (int i = 0; i < NST; ++i)
    if (i < mine) request(i, i);
  int slot = 0;
  for (int i = 0; i < mine; ++i) {
    landed(min(NST - 1, mine - 1 - i));
    // operand = 16 rows x 64 k: lane l -> row l % 16, chunk l / 16 of the slice
    const uint8_t* img = &lds[(w * NST + slot) * STE];
    i32x4 wa[2][TN], xb[2][TM];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int off = r16 * kSub + (((4 * h + g4) ^ gsw(r16)) << 4);
#pragma unroll
      for (int q = 0; q < TN; ++q) wa[h][q] = *(const i32x4*)&img[(BM + 16 * q) * kSub + off];
#pragma unroll
      for (int q = 0; q < TM; ++q) xb[h][q] = *(const i32x4*)&img[16 * q * kSub + off];
    }
    if (last_chunks != 8 && w + kWaves * i == nst - 1) {   // chunks of X past K are cleared
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < TM; ++q)
#pragma unroll
          for (int c = 0; c < 4; ++c) xb[h][q][c] = 4 * h + g4 < last_chunks ? xb[h][q][c] : 0;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the slot is read: it takes stage i + NST
    if (i + NST < mine) request(i + NST, slot);
    slot = slot + 1 == NST ? 0 : slot + 1;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < TN; ++q)
#pragma unroll
        for (int j = 0; j < TM; ++j)
          acc[q][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wa[h][q], xb[h][j], acc[q][j], 0, 0, 0);
  }

  // The waves' sums: sub-tile u is added up and stored by wave u % kWaves, which takes
  // the others' from LDS (every ring is read: the barrier).
  __syncthreads();
#pragma unroll
  for (int u = 0; u < TN * TM; ++u)
    if (w != u % kWaves) *(i32x4*)&lds[(u * kWaves + w) * 1024 + lane * 16] = acc[u / TM][u % TM];
  // acc[i][j] lane l, register q: n = 16 i + 4 (l / 16) + q, m = 16 j + l % 16.
  // Scales and residuals are asked for ahead of the stores that could (as far as the
  // compiler knows) change them.
  constexpr int OWN = (TN * TM + kWaves - 1) / kWaves;
  f32x4 wsc[OWN];
  float xsc[OWN];
  u32x2 rb[OWN];
  const int nb = n0 + 4 * g4;                      // N is a multiple of 8: whole groups in or out
#pragma unroll
  for (int v = 0; v < OWN; ++v) {
    const int u = v * kWaves + w, n = nb + 16 * (u / TM), m = m0 + 16 * (u % TM) + r16;
    wsc[v] = *(const f32x4*)(p.ws + min(n, N - 4));
    xsc[v] = a.xs[min(m, M - 1)];
    if (p.r && u < TN * TM && m < M && n < N) rb[v] = *(const u32x2*)(p.r + (int64_t)m * N + n);
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < TN * TM; ++u) {
    if (w != u % kWaves) continue;
    i32x4 sum = acc[u / TM][u % TM];
#pragma unroll
    for (int o = 1; o < kWaves; ++o) sum += *(const i32x4*)&lds[(u * kWaves + (u + o) % kWaves) * 1024 + lane * 16];
    const int n = nb + 16 * (u / TM), m = m0 + 16 * (u % TM) + r16;
    if (m >= M || n >= N) continue;
    *(bf16x4*)(p.y + (int64_t)m * N + n) =
        scaled(sum, xsc[u / kWaves] * wsc[u / kWaves], p.r != nullptr, rb[u / kWaves]);
  }
}

template <int BM, int BN, int NST>
void launch_tile(const Int8Args& a, hipStream_t s) {
  int64_t cols = 0;
  for (int i = 0; i < a.count; ++i) cols += (a.n[i] + BN - 1) / BN;
  const int64_t tiles = (int64_t)((a.m + BM - 1) / BM) * cols;
  const dim3 grid((unsigned)(8 * ((tiles + 7) / 8))), blk(kWaves * 64);
  if (a.m <= BM) hipLaunchKernelGGL((gemm_int8_kernel<BM, BN, NST, true>), grid, blk, 0, s, a);
  else hipLaunchKernelGGL((gemm_int8_kernel<BM, BN, NST, false>), grid, blk, 0, s, a);
}

// Tile choice: the time of a launch is close to
//   max(1, 0.36 r + 0.64 ceil(r)) * (K / 128 * step + fix),   r = tiles / 256 CUs
// (a partly filled last round costs most of a whole one): one 128-k step of one tile
// per CU, and a tile's prologue and epilogue.  step and fix are fitted to 602 products
// (M 1 to 6000; N and K of three models' projections, W out of the caches, and drawn
// ones from 8 and 16 on), where the tile it picks is 0.5% slower than the fastest of the
// twelve on average and 13% at most (64 x 6144 x 4096 in 64 x 32 tiles 10.2 us, 32 x 32
// 9.2).  A wave of 16 x 16 tiles has a ring of four stages where they are few, two
// workgroups to a CU, and K is long or W large enough to come from HBM (1 x 3584 x 18944
// 12.4 us, two stages 16.5; 1 x 32 x 11904 7.3, 10.0), of two else, five to a CU (1 x
// 28672 x 4096 19.5 us, four stages 22.3; 83 x 416 x 3456 4.1, 4.4).
struct TileCost {
  int bm, bn;
  double step_ns, fix_ns;
};
constexpr TileCost kTiles[] = {{16, 16, 54, 892},   {16, 16, 50, 380},      {32, 16, 63, 719},     {32, 32, 99, 788},
                               {64, 32, 164, 1921}, {64, 64, 218, 3230},    {96, 64, 319, 2763},   {128, 64, 354, 1809},
                               {128, 128, 582, 1585}, {256, 128, 1051, 1148}, {256, 128, 863, 3144}, {256, 256, 1529, 2340}};
constexpr int kDeep = 0, kShallow = 1; // 16 x 16
constexpr int kDeepK = 8192;
constexpr double kDeepBytes = 8e6;
constexpr int kWide = 10;               // from here on gemm_int8_wide.hip: K a multiple of 128

int pick_tile(int m, int k, int count, const int* n) {
  int best = -1;
  double best_cost = 0, bytes = 0;
  for (int j = 0; j < count; ++j) bytes += (double)n[j] * k;
  for (int i = 0; i < (k % 128 == 0 ? kWide + 2 : kWide); ++i) {
    const TileCost& t = kTiles[i];
    double cols = 0;
    for (int j = 0; j < count; ++j) cols += ((int64_t)n[j] + t.bn - 1) / t.bn;
    const double tiles = (double)(((int64_t)m + t.bm - 1) / t.bm) * cols, r = tiles / kCus;
    if (i <= kShallow && (i == kDeep) != (tiles <= 2 * kCus && (k >= kDeepK || bytes >= kDeepBytes))) continue;
    if (tiles * 512 >= 4294967296.0) continue;     // a launch counts its threads in 32 bits
    const double cost = (r <= 1.0 ? 1.0 : 0.36 * r + 0.64 * ceil(r)) * ((k + 127) / 128 * t.step_ns + t.fix_ns);
    if (best < 0 || cost < best_cost) {
      best = i;
      best_cost = cost;
    }
  }
  return best;
}

hipError_t run_tile(int tile, const Int8Args& a, hipStream_t s) {
  switch (tile) {
    case kDeep: launch_tile<16, 16, 4>(a, s); break;
    case kShallow: launch_tile<16, 16, 2>(a, s); break;
    case 2: launch_tile<32, 16, 3>(a, s); break;
    case 3: launch_tile<32, 32, 2>(a, s); break;
    case 4: launch_tile<64, 32, 3>(a, s); break;
    case 5: launch_tile<64, 64, 2>(a, s); break;
    case 6: launch_tile<96, 64, 2>(a, s); break;
    case 7:
    case 8:
    case 9: return launch_gemm_int8_ring(a, kTiles[tile].bm, kTiles[tile].bn, s);
    default: return launch_gemm_int8_wide(a, kTiles[tile].bn, s);
  }
  return hipGetLastError();
}

}  // namespace

// m * n below 2^34 in whole tiles of 256 x 128, which leaves 2^19 of those: one tile at
// least that any such size can take in one launch.
bool gemm_int8_fits(int m, int count, const int* n) {
  double cols = 0;
  for (int i = 0; i < count; ++i) cols += ((int64_t)n[i] + 127) / 128;
  return (double)(((int64_t)m + 255) / 256) * cols < 524288.0;
}

hipError_t launch_gemm_int8(int m, int k, int count, const int* n, const void* x, const float* xs,
                            const void* const* w, const float* const* ws, const void* r, void* const* y, hipStream_t s) {
  Int8Args a{};
  a.m = m;
  a.k = k;
  a.x = (const uint8_t*)x;
  a.xs = xs;
  for (int i = 0; i < count; ++i) {
    if (n[i] <= 0) continue;
    a.w[a.count] = (const uint8_t*)w[i];
    a.ws[a.count] = ws[i];
    a.y[a.count] = (uint16_t*)y[i];
    a.n[a.count++] = n[i];
  }
  if (m <= 0 || a.count == 0) return hipSuccess;
  a.r[0] = (const uint16_t*)r;
  return run_tile(pick_tile(m, k, a.count, a.n), a, s);
}

}  // namespace pgsr
