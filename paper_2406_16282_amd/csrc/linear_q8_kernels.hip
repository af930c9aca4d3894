// Linear layers of 8-bit rows and 8-bit weights, forward, for gfx950.
//
//   y = (sum_k q[m, k] w[n, k]) scale[m] w_scale[n] + bias[n]
//
// The sums are whole numbers in 32 bits and exact for up to kQ8MaxDepth products (128 * 128 *
// kQ8MaxDepth < 2^31); one conversion to fp32, one product of the scales, one fused
// multiply-add with the bias, one rounding to the output's type.
//
// What bounds it. Many rows: the card's power. A loop of nothing but 16x16x64 products of random
// bytes runs at 3404 TOPS, of 32x32x32 ones at 3087 (4419 and 3986 on zeros), so the smaller shape
// is taken although it needs as many operand reads. [8192 x 4096] x 11008 takes 305 to 340 us by the
// card's state (2170 to 2420 TOPS; the library's int8 product without scales 392 to 413, its bf16
// product 686 to 704, in the same runs), 8192^3 392 to 437 us (2510 to 2806; library 430 to 453):
// matrix cores busy 63 to 67% of the cycles, no bank conflicts, a clock of 1.6 to 1.85 GHz. Few rows:
// the weight's bytes. One row of 11008 x 4096 9.1 us with weights that the caches do not hold
// (5.0 TB/s; one load's way and the launch are 3 of them), 16384 x 16384 40 us (6.7 TB/s), 16 rows
// of the first 12.5 us.
//
// Tiles (product_tile). The loop is that of the bf16 layers (linear_kernels.hip): K in steps of
// 128 bytes, each in two half steps; a ring of slots of half a step's operands (half of every wave's
// rows of x and of W), filled straight from memory by buffer loads into LDS that return zeros past
// the operands' ends; a half step multiplies fragments in registers, reads the next ones and loads
// into the slot that was read before, with one barrier and a wait that leaves kRing - 2 slots in
// flight. An LDS row is 128 bytes = eight 16-byte units, unit u of row r at u ^ swz(r), so that the
// 16 rows of a read fall into distinct banks: (r >> 1) % 8 for x, bit 1 and bits 3, 4 of r for W.
// Blocks are persistent and the loads run on from one tile into the next. MFMA rows are rows of W,
// dealt to the tiles so that a lane ends with 16 consecutive columns of a row: whole vectors are
// stored from registers. The tiles' scales travel with the operands, in LDS.
// Tried on 8192 rows of 11008 x 4096 without gain: the MFMAs in a fixed order with the reads and
// loads between them (2 to 5% faster as long as it spilled two registers, slower without), 256 x 256
// by 4 waves.
//
// Some rows (product_rows). Too few tiles to fill the card: a block takes 16, 32 or 64 rows and 32
// columns, its four waves the K steps in turn, each through a ring of its own without barriers.
// 16 rows, us: rings of two steps 13.3 (11008 x 4096) and 15.9 (4096 x 11008), of three 13.8 and 16.0; 64
// columns to a block 12.9 and 21.6 (768 x 768 4.7 against 3.9).
//
// One or two rows (product_few). Dot products: the matrix form would load as much and compute 16
// rows; 9.1 us against 11.7 for 11008 x 4096 (2 rows: 10.0 and 12.0). Reloading each piece as soon as it
// is used instead of four at a time gave nothing (one row) or cost 10% (two).
#include "linear_q8_device.hpp"

#include <algorithm>

namespace lmbp {
namespace lq8 {

constexpr int kBK = 128;   // K step in bytes: an LDS row

// MINW: waves per SIMD that the registers are budgeted for (blocks per CU follow from it).
template <int BM_, int BN_, int WM_, int WN_, int MINW_, int RING_ = 4>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, kMinWaves = MINW_;
  static constexpr int kWaves = WM * WN, kThreads = kWaves * kWave;
  static constexpr int HM = BM / WM / 2, HN = BN / WN / 2;   // half of a wave's rows, columns
  static constexpr int TMH = HM / 16, TNH = HN / 16;         // MFMA tiles per half
  static constexpr int TM = 2 * TMH, TN = 2 * TNH;
  static constexpr int kSlot = (BM + BN) / 2 * kBK;          // one ring slot: half of A and of B
  static constexpr int kRing = RING_;
  static constexpr int kBlocksPerCu = kMinWaves * 4 / kWaves;
  static constexpr int kLA = BM / 16 / kWaves, kLB = BN / 16 / kWaves;   // 1 KiB loads per wave
  static constexpr int kSide = 4 * (BM + BN) * 4;            // the scales of four tiles
  static constexpr int kLdsBytes = kRing * kSlot + kSide;
  static_assert(HN % 32 == 0 && HM % 16 == 0, "wave tile");
  static_assert(kLA >= 1 && kLB >= 1 && (BM / 16) % kWaves == 0 && (BN / 16) % kWaves == 0, "loads");
  static_assert(kLdsBytes * kBlocksPerCu <= 160 * 1024, "LDS per CU");
};

// 16 consecutive results of a row from column `col` on; those from N on are not stored.
template <class OUT>
__device__ inline void store16(const Args& a, int64_t row, int64_t col, const float (&f)[16]) {
  constexpr int E = OUT::kPerVec;
  const int64_t base = row * a.N + col;
  int left = int(a.N - col);   // columns that there are; new in every call: 16 masks kept would be spilled
  asm volatile("" : "+v"(left));
#pragma unroll
  for (int p = 0; p < 16; p += E) {
    if (p + E <= left) {
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = f[p + e];
      store_16(elem<OUT>(a.y, base + p), OUT::pack(v));
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (p + e < left) OUT::store1(a.y, base + p + e, f[p + e]);
    }
  }
}

template <class C, class OUT>
__global__ __launch_bounds__(C::kThreads, C::kMinWaves) void product_tile(Args a) {
  constexpr int BM = C::BM, BN = C::BN, TM = C::TM, TN = C::TN, TMH = C::TMH, TNH = C::TNH;
  constexpr int HM = C::HM, HN = C::HN, kWaves = C::kWaves;
  constexpr int kLA = C::kLA, kLB = C::kLB, kL = kLA + kLB, kSlot = C::kSlot, kRing = C::kRing;
  const uint32_t M = uint32_t(a.M), N = uint32_t(a.N), K = uint32_t(a.K);   // below 2^31
  extern __shared__ __attribute__((aligned(16))) int8_t lds[];
  float* const as_lds = reinterpret_cast<float*>(lds + kRing * kSlot);
  float* const bs_lds = as_lds + 4 * BM;
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = wave_in_block();
  const int wm = wave / C::WN, wn = wave % C::WN;
  const uint32_t tiles = a.map.tiles;
  const int kt_count = int((K + kBK - 1) / kBK);   // K > 0

  // ---- load side: byte offsets of this lane's chunks at K step 0, for both halves
  uint32_t ld_a[2][kLA], ld_b[2][kLB];
  uint32_t kc_a[kLA], kc_b[kLB];
  const int r_in = lane / 8, u_in = lane % 8;
#pragma unroll
  for (int q = 0; q < kLA; ++q) {
    const int lr = (wave + kWaves * q) * 8 + r_in;
    kc_a[q] = (u_in ^ ((lr >> 1) & 7)) * 16;
#pragma unroll
    for (int h = 0; h < 2; ++h) ld_a[h][q] = uint32_t((lr / HM) * 2 * HM + h * HM + lr % HM) * K + kc_a[q];
  }
#pragma unroll
  for (int q = 0; q < kLB; ++q) {
    const int lr = (wave + kWaves * q) * 8 + r_in;
    kc_b[q] = (u_in ^ (((lr >> 1) & 1) | (((lr >> 3) & 3) << 1))) * 16;
#pragma unroll
    for (int h = 0; h < 2; ++h) ld_b[h][q] = uint32_t((lr / 8) * 16 + h * 8 + lr % 8) * K + kc_b[q];
  }
  // Load cursor: tile l_tile (l_seq-th of this block), K step l_k. Past the last tile the
  // resources are empty and the loads read zeros into slots that nothing reads.
  uint32_t l_tile = blockIdx.x;
  int l_seq = 0, l_k = 0;
  __amdgpu_buffer_rsrc_t ra, rb;
  auto enter_tile = [&]() {
    uint32_t tm = 0, tn = 0;
    const bool in = l_tile < tiles;
    if (in) tile_of(l_tile, a.map, tm, tn);
    const uint32_t m0 = tm * BM, n0 = tn * BN;
    const uint32_t rows_a = !in ? 0u : (M - m0 < BM) ? M - m0 : BM;
    const uint32_t rows_b = !in ? 0u : (N - n0 < BN) ? N - n0 : BN;
    ra = make_rsrc(a.a + uint64_t(m0) * K, rows_a * K);
    rb = make_rsrc(a.b + uint64_t(n0) * K, rows_b * K);
    // The tile's scales, into one of four places: the cursor runs at most two tiles ahead of
    // the tile being computed. Issued before the tile's first operands, they have landed when
    // those have.
    for (int v = wave; v < BM / 64; v += kWaves)
      load_lds4(make_rsrc(a.a_scale + m0, rows_a * 4), as_lds + (l_seq & 3) * BM + v * 64, uint32_t(v * 256 + lane * 4));
    for (int v = wave; v < BN / 64; v += kWaves)
      load_lds4(make_rsrc(a.b_scale + n0, rows_b * 4), bs_lds + (l_seq & 3) * BN + v * 64, uint32_t(v * 256 + lane * 4));
  };
  auto issue = [&](int h, int8_t* S) {
    const uint32_t k0 = uint32_t(l_k) * kBK;
#pragma unroll
    for (int q = 0; q < kLA; ++q)
      load_lds16(ra, S + (wave + kWaves * q) * 1024, k0 + kc_a[q] < K ? ld_a[h][q] + k0 : kOutOfRange);
#pragma unroll
    for (int q = 0; q < kLB; ++q)
      load_lds16(rb, S + BM / 2 * kBK + (wave + kWaves * q) * 1024, k0 + kc_b[q] < K ? ld_b[h][q] + k0 : kOutOfRange);
  };
  auto advance = [&]() {
    if (++l_k == kt_count) {
      l_k = 0;
      l_tile += gridDim.x;
      ++l_seq;
      enter_tile();
    }
  };

  // ---- compute side
  const int a_off = (wm * HM + (lane & 15)) * kBK;
  const int b_off = BM / 2 * kBK + (wn * HN + ((lane & 15) >> 2) * 8 + (lane & 3)) * kBK;
  const int swa = (lane & 15) >> 1;
  const int swb = ((lane >> 1) & 1) | (((lane >> 2) & 3) << 1);
  const int ua[2] = {((lane >> 4) ^ swa) * 16, ((4 + (lane >> 4)) ^ swa) * 16};
  const int ub[2] = {((lane >> 4) ^ swb) * 16, ((4 + (lane >> 4)) ^ swb) * 16};
  i32x4 fa[2][TMH][2], fb[2][TNH][2];
  auto read_a = [&](const int8_t* S, int h) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < TMH; ++i) fa[h][i][kk] = *reinterpret_cast<const i32x4*>(S + a_off + i * 16 * kBK + ua[kk]);
  };
  auto read_b = [&](const int8_t* S, int h) {   // tile j: columns 4 (j % 2) of the wave's (j / 2)-th 64
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int j = 0; j < TNH; ++j)
        fb[h][j][kk] = *reinterpret_cast<const i32x4*>(S + b_off + ((j / 2) * 32 + (j % 2) * 4) * kBK + ub[kk]);
  };
  i32x4 acc[TM][TN];
  auto quad = [&](int ha, int hb) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < TMH; ++i)
#pragma unroll
        for (int j = 0; j < TNH; ++j)
          acc[ha * TMH + i][hb * TNH + j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
              fb[hb][j][kk], fa[ha][i][kk], acc[ha * TMH + i][hb * TNH + j], 0, 0, 0);
  };
  constexpr int MF = TMH * TNH * 2, RA = TMH * 2, RB = TNH * 2;

  // An odd ring has its second-half slots loaded in first half steps and the other way round.
  enter_tile();
  constexpr bool kOdd = kRing % 2 != 0;
#pragma unroll
  for (int d = 0; d < kRing; ++d) {
    issue(d & 1, lds + d * kSlot);
    if (d & 1) advance();
  }
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"((kRing - 2) * kL) : "memory");
  asm volatile("s_barrier" ::: "memory");

  int slot = 0;   // of the half step's first data unit
  auto next = [&](int v, int d) { v += d; return v >= kRing ? v - kRing : v; };
  int seq = 0;
  for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x, ++seq) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    // The tile's first fragments; no wave may load over them before all have read them.
    read_a(lds + slot * kSlot, 0);
    read_b(lds + slot * kSlot, 0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    asm volatile("s_barrier" ::: "memory");

    for (int kt = 0; kt < kt_count; ++kt) {
      int8_t* S = lds + slot * kSlot;
      int8_t* S1 = lds + next(slot, 1) * kSlot;
      slot = next(slot, 2);
      int8_t* Sn = lds + slot * kSlot;
      __builtin_amdgcn_s_setprio(1);
      issue(kOdd ? 1 : 0, S);
      read_b(S1, 1);
      read_a(S1, 1);
      quad(0, 0);
      quad(0, 1);
      spread<2 * MF, kL, RA + RB>();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(0);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      asm volatile("s_waitcnt vmcnt(%0)" :: "n"((kRing - 2) * kL) : "memory");
      asm volatile("s_barrier" ::: "memory");
      if constexpr (kOdd) advance();
      issue(kOdd ? 0 : 1, S1);
      read_a(Sn, 0);
      quad(1, 0);
      spread<MF, kL, RA>();
      __builtin_amdgcn_sched_barrier(0);
      read_b(Sn, 0);
      quad(1, 1);
      spread<MF, 0, RB>();
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      asm volatile("s_waitcnt vmcnt(%0)" :: "n"((kRing - 2) * kL) : "memory");
      asm volatile("s_barrier" ::: "memory");
      if constexpr (!kOdd) advance();
    }

    // ---- epilogue; no ring slot is touched, so the next tile's loads run on
    uint32_t tm, tn;
    tile_of(tile, a.map, tm, tn);
    const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN;
    int lane_e = lane;   // new in every tile: addresses formed from it ahead of the loop would be spilled
    asm volatile("" : "+v"(lane_e));
    const int g = lane_e >> 4;
    const float* const as = as_lds + (seq & 3) * BM;
#pragma unroll
    for (int gr = 0; gr < HN / 32; ++gr) {
      const int in_tile = wn * 2 * HN + gr * 64 + g * 16;
      const int64_t col = n0 + in_tile;
      float ws[16], b[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        ws[e] = bs_lds[(seq & 3) * BN + in_tile + e];
        b[e] = 0.0f;
      }
      if (a.bias != nullptr) {
#pragma unroll
        for (int e = 0; e < 16; ++e) b[e] = col + e < N ? OUT::load1(a.bias, col + e) : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int row = wm * 2 * HM + i * 16 + (lane_e & 15);
        const float sc = as[row];
        float f[16];
#pragma unroll
        for (int e = 0; e < 16; ++e)   // column 4 j + r of the 16: j = e / 4, half j / 2, tile j % 2 of the half
          f[e] = __builtin_fmaf(float(acc[i][(e / 8) * TNH + gr * 2 + (e / 4) % 2][e % 4]), sc * ws[e], b[e]);
        if (m0 + row < M) store16<OUT>(a, m0 + row, col, f);
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load into LDS outlives the block
}

template <class C, class OUT>
hipError_t launch_tile(Args a, int dev, int cus, hipStream_t s) {
  if (!map_tiles(a, C::BM, C::BN)) return hipErrorInvalidValue;
  const hipError_t e = allow_lds<product_tile<C, OUT>>(dev, C::kLdsBytes);
  if (e != hipSuccess) return e;
  const uint32_t slots = uint32_t(cus) * C::kBlocksPerCu;
  hipLaunchKernelGGL((product_tile<C, OUT>), dim3(a.map.tiles < slots ? a.map.tiles : slots), dim3(C::kThreads),
                     C::kLdsBytes, s, a);
  return hipGetLastError();
}

using BigTile = Tile<256, 256, 2, 4, 2>;      // one block of 8 waves per CU
using MidTile = Tile<128, 256, 1, 4, 2, 3>;   // two blocks of 4 waves
using SmallTile = Tile<128, 128, 2, 2, 2>;    // two blocks of 4 waves
using LowTile = Tile<64, 128, 2, 2, 3>;       // three blocks of 4 waves

// Few rows: a block of 4 waves takes MT x 16 rows of x and NB x 16 of W; its waves take the K
// steps in turn, each through an LDS ring of its own, and the partial sums meet in LDS.
constexpr int kRowsWaves = 4;
template <int MT, int NB, int D>
constexpr int kRowsLds = kRowsWaves * D * (NB + MT) * 16 * kBK;

template <int MT, int NB, int D, bool NT, class OUT>
__global__ __launch_bounds__(kRowsWaves * kWave) void product_rows(Args a) {
  constexpr int kWaves = kRowsWaves, kRows = MT * 16, kOut = NB * 16;
  constexpr int kTiles = MT * NB, kSumWaves = kTiles < kWaves ? kTiles : kWaves;
  static_assert(kTiles % kSumWaves == 0 && kRowsLds<MT, NB, D> <= 160 * 1024, "result tiles per wave; LDS");
  static_assert(kRowsLds<MT, NB, D> >= kWaves * kTiles * 1024, "room for the partial sums");
  const int64_t M = a.M, N = a.N;
  const uint32_t K = uint32_t(a.K);
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = wave_in_block();
  // Row blocks of one column block run on one XCD, next to each other.
  const uint32_t b = blockIdx.x;
  const uint32_t id = (b < a.map.per_xcd * kXcds) ? (b % kXcds) * a.map.per_xcd + b / kXcds : b;
  const int64_t m0 = int64_t(id % a.map.tiles_m) * kRows, n0 = int64_t(id / a.map.tiles_m) * kOut;
  const int64_t rows_a = (M - m0 < kRows) ? M - m0 : kRows, rows_b = (N - n0 < kOut) ? N - n0 : kOut;
  const auto ra = make_rsrc(a.a + m0 * K, rows_a * K), rb = make_rsrc(a.b + n0 * K, rows_b * K);
  const int g = lane >> 4;
  // This wave's ring: D steps of kOut rows of W and kRows of x. No other wave touches it: no
  // barrier in the K loop.
  constexpr int kStep = (kOut + kRows) * kBK, kLoads = 2 * (NB + MT);
  extern __shared__ __attribute__((aligned(16))) int8_t lds[];
  int8_t* const ring = lds + wave * D * kStep;
  const int r_in = lane / 8;   // rows 8 q + r_in of the load q: even and odd q differ in their swizzle
  const uint32_t kc[2] = {uint32_t((lane % 8) ^ (r_in >> 1)) * 16, uint32_t((lane % 8) ^ (4 + (r_in >> 1))) * 16};
  const uint32_t off[2] = {r_in * K + kc[0], (8 + r_in) * K + kc[1]}, tile_off = 16 * K;
  auto load = [&](int step, int d) {
    int8_t* S = ring + d * kStep;
    const uint32_t k0 = uint32_t(step) * kBK;
#pragma unroll
    for (int q = 0; q < 2 * NB; ++q)
      load_lds16<NT ? 2 : 0>(rb, S + q * 1024, k0 + kc[q % 2] < K ? off[q % 2] + k0 + (q / 2) * tile_off : kOutOfRange);
#pragma unroll
    for (int q = 0; q < 2 * MT; ++q)
      load_lds16(ra, S + kOut * kBK + q * 1024, k0 + kc[q % 2] < K ? off[q % 2] + k0 + (q / 2) * tile_off : kOutOfRange);
  };
  i32x4 acc[MT][NB];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  const int steps = int((K + kBK - 1) / kBK);
#pragma unroll
  for (int d = 0; d < D; ++d) load(wave + d * kWaves, d);   // steps past the end read zeros
  const int frag = (lane & 15) * kBK, sw = (lane & 15) >> 1;
  const int u[2] = {(g ^ sw) * 16, ((4 + g) ^ sw) * 16};
  int d = 0;
  for (int st = wave; st < steps; st += kWaves) {
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"((D - 1) * kLoads) : "memory");
    const int8_t* S = ring + d * kStep + frag;
    i32x4 fw[NB][2], fx[MT][2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
      for (int j = 0; j < NB; ++j) fw[j][kk] = *reinterpret_cast<const i32x4*>(S + j * 16 * kBK + u[kk]);
#pragma unroll
      for (int i = 0; i < MT; ++i) fx[i][kk] = *reinterpret_cast<const i32x4*>(S + (NB + i) * 16 * kBK + u[kk]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before it is loaded over
    load(st + D * kWaves, d);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[j][kk], fx[i][kk], acc[i][j], 0, 0, 0);
    d = d + 1 == D ? 0 : d + 1;
  }
  // The rings' place holds the sums from here on: no load may still land there (a barrier
  // alone does not promise that), and every ring must have been read.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  auto part = reinterpret_cast<i32x4 (*)[MT][NB][kWave]>(lds);
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) part[wave][i][j][lane] = acc[i][j];
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kTiles / kSumWaves; ++q) {
    const int tile = wave + q * kSumWaves, i = tile / NB, j = tile % NB;
    if (tile >= kTiles) return;
    i32x4 v = part[0][i][j][lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += part[w][i][j][lane];
    const int64_t row = m0 + i * 16 + (lane & 15), col = n0 + j * 16 + g * 4;
    if (row >= M) continue;
    const float sc = a.a_scale[row];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < N)
        OUT::store1(a.y, row * N + col + e,
                    __builtin_fmaf(float(v[e]), sc * a.b_scale[col + e], a.bias != nullptr ? OUT::load1(a.bias, col + e) : 0.0f));
  }
}

template <int MT, int NB, int D, bool NT, class OUT>
hipError_t launch_rows(Args a, int dev, hipStream_t s) {
  if (!map_tiles(a, MT * 16, NB * 16) || a.map.tiles > most_blocks(kRowsWaves * kWave)) return hipErrorInvalidValue;
  const hipError_t e = allow_lds<product_rows<MT, NB, D, NT, OUT>>(dev, kRowsLds<MT, NB, D>);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((product_rows<MT, NB, D, NT, OUT>), dim3(a.map.tiles), dim3(kRowsWaves * kWave), (kRowsLds<MT, NB, D>),
                     s, a);
  return hipGetLastError();
}

// One or two rows: a wave takes R rows of W, 1 KiB of each at a time (16 bytes to a lane), against
// the same pieces of all MT rows of x, and adds up its lanes' sums at the end.
constexpr int kFewWaves = 4;
template <int MT, int R, class OUT>
__global__ __launch_bounds__(kFewWaves * kWave) void product_few(Args a) {
  constexpr int kDeep = 4 / R;   // pieces of a row in flight
  const uint32_t K = uint32_t(a.K);
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t n0 = ((int64_t(a.first) + blockIdx.x) * kFewWaves + wave_in_block()) * R;
  if (n0 >= a.N) return;
  const int rows_b = a.N - n0 < R ? int(a.N - n0) : R;
  const auto rb = make_rsrc(a.b + n0 * K, int64_t(rows_b) * K), ra = make_rsrc(a.a, a.M * K);
  int sum[R][MT];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < MT; ++i) sum[r][i] = 0;
  for (uint32_t k0 = 0; k0 < K; k0 += kDeep * 1024) {
    u32x4 w[kDeep][R], x[kDeep][MT];
#pragma unroll
    for (int p = 0; p < kDeep; ++p) {
      const uint32_t k = k0 + p * 1024 + lane * 16;
#pragma unroll
      for (int r = 0; r < R; ++r)
        w[p][r] = __builtin_amdgcn_raw_buffer_load_b128(rb, k < K ? r * K + k : kOutOfRange, 0, 2);
#pragma unroll
      for (int i = 0; i < MT; ++i)
        x[p][i] = __builtin_amdgcn_raw_buffer_load_b128(ra, k < K ? i * K + k : kOutOfRange, 0, 0);
    }
#pragma unroll
    for (int p = 0; p < kDeep; ++p)
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sum[r][i] = __builtin_amdgcn_sdot4(int(w[p][r][e]), int(x[p][i][e]), sum[r][i], false);
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) sum[r][i] += __shfl_xor(sum[r][i], off, kWave);
      const int64_t n = n0 + r;
      if (lane == r * MT + i && i < a.M && n < a.N)
        OUT::store1(a.y, i * a.N + n,
                    __builtin_fmaf(float(sum[r][i]), a.a_scale[i] * a.b_scale[n],
                                   a.bias != nullptr ? OUT::load1(a.bias, n) : 0.0f));
    }
}

template <int MT, class OUT>
hipError_t launch_few(Args a, hipStream_t s) {
  auto launch = [&](auto kernel, int rows) {
    const int64_t per = int64_t(kFewWaves) * rows;
    return in_parts((a.N + per - 1) / per, most_blocks(kFewWaves * kWave), [&](int64_t first, int64_t count) {
      a.first = uint32_t(first);
      hipLaunchKernelGGL(kernel, dim3(unsigned(count)), dim3(kFewWaves * kWave), 0, s, a);
    });
  };
  // Two rows of W to a wave where they are short. One row of x, two against one: 11008 x 1024 4.65 and
  // 6.1 us, 11008 x 2048 6.0 and 7.0; 11008 x 4096 9.8 and 9.1 (two rows of x: 10.6 and 10.0). Four were
  // never the best (11008 x 1024 4.72, 4096 x 1024 3.64 against 3.40).
  return a.K <= 2048 ? launch(product_few<MT, 2, OUT>, 2) : launch(product_few<MT, 1, OUT>, 1);
}

// The form by estimated times (linear_q8_device.hpp), their constants fitted to the times of every
// form at 420 sizes of 15 layers. The choice is 0.8% slower than the best form on average and 27% at
// worst (0.9% on layers that were left out of the fit). Both sides, us: 11008 x 4096 at 16 rows
// rows16 12.5, 64x128 tiles 19.8; at 32 rows rows32 15.3, 64x128 20.0; at 128 rows rows64 30, 64x128
// 20.7; 197 rows 64x128 26.5, 128x128 23.5; 512 rows 128x128 38.4, 128x256 36.5; 2048 rows 128x256 91,
// 256x256 105; 4096 rows 174 and 163; 8192 rows 318 and 318. 768 x 768 at 1576 rows 64x128 6.4, 128x128
// 7.4, 256x256 14.8. 4096 x 11008 at 128 rows rows64 22.7, 64x128 43.9; 8192 rows 128x256 298, 256x256 281.
enum Form { kFew, kRows16, kRows32, kRows64, kLow, kSmall, kMid, kBig, kForms };

constexpr RowsCost kRows16Cost = {2.685f, 0.2485f, 0.2127f, 0.578f, 0.001916f, 0.009501f, 0.0643f, 1.986f, 0, 0};
constexpr RowsCost kRows32Cost = {3.018f, 0.2897f, 0.338f, 0.4889f, 0.003409f, 0.009262f, 0.04509f, 1.318f, 0, 0};
constexpr RowsCost kRows64Cost = {3.573f, 0.4323f, 0.1489f, 0.6175f, 0.003602f, 0.005212f, 0.01158f, 2.154f, 0, 0};
constexpr TileCost kLowCost = {3.156f, 0.8615f, 0.3726f, 0.1655f, 0.3679f, 0.08068f, 0.2468f};
constexpr TileCost kSmallCost = {3.676f, 0.8739f, 0.4877f, 0.312f, 0, 0.05597f, 0.2539f};
constexpr TileCost kMidCost = {4.706f, 1.471f, 0.7827f, 0.561f, 0, 0.08527f, 0.2501f};
constexpr TileCost kBigCost = {5.923f, 1.435f, 1.257f, 0, 0, 0.003937f, 0.2741f};

Form choose_form(int64_t M, int64_t N, int64_t K, int cus, float* time = nullptr) {
  // Two rows of x take twice the loads of x against each of W; with large weights (which the caches do not
  // hold) the matrix form is ahead: 13824 x 5120 19.3 and 15.5 us, 5120 x 13824 17.3 and 16.6, but 11008 x 4096
  // 10.3 and 12.3, 4096 x 11008 12.6 and 14.2.
  if (M == 1 || (M == 2 && N * K <= (int64_t(56) << 20))) {
    if (time) *time = 3.2f + float(N) * float(K) * (1.0f / 5.5e6f);
    return kFew;
  }
  auto rows = [&](int bm, int blocks_per_cu, const RowsCost& c) {
    return M <= 2048 ? rows_cost(M, N, K, bm, 32, kBK, blocks_per_cu, 1, cus, c) : INFINITY;
  };
  const float t[kForms] = {INFINITY,
                           rows(16, 3, kRows16Cost),
                           rows(32, 2, kRows32Cost),
                           rows(64, 1, kRows64Cost),
                           tile_cost<LowTile>(M, N, K, kBK, 1, cus, kLowCost),
                           tile_cost<SmallTile>(M, N, K, kBK, 1, cus, kSmallCost),
                           tile_cost<MidTile>(M, N, K, kBK, 1, cus, kMidCost),
                           tile_cost<BigTile>(M, N, K, kBK, 1, cus, kBigCost)};
  const float* const least = std::min_element(t, t + kForms);
  if (time) *time = *least;
  return Form(least - t);
}

// Whether a layer's rows, of both operands, are copied to aligned ones first (pad_pays).
bool pads(int64_t M, int64_t N, int64_t K, int cus) {
  if (K % 16 == 0 || M == 0 || N == 0) return false;
  float fast;
  choose_form(M, N, padded(K), cus, &fast);
  return pad_pays(M, N, K, M + N, K, fast);
}

template <class OUT>
hipError_t launch_fwd(const Args& a, hipStream_t s) {
  const bool aligned = a.K > 0 && a.K % 16 == 0 && reinterpret_cast<uintptr_t>(a.a) % 16 == 0 &&
                       reinterpret_cast<uintptr_t>(a.b) % 16 == 0;
  if (!aligned) return launch_any<OUT, false>(a, s);
  int dev = 0, cus = 0;
  const hipError_t e = current_device(dev, cus);
  if (e != hipSuccess) return e;
  // Weights by non-temporal loads where one row block reads them and they are more than the caches are
  // likely to hold until the next call. 16 rows, without and with, weights cold / in the caches: 11008 x
  // 4096 14.1 and 12.7 / 10.4 and 10.6 us, 16384 x 16384 51 and 44 / 40 and 43; 8192 x 4096 (32 MiB) 9.7 and
  // 8.9 / 5.8 and 6.3.
  const bool nt = a.N * a.K > (int64_t(32) << 20);
  switch (choose_form(a.M, a.N, a.K, cus)) {
    case kFew: return a.M == 1 ? launch_few<1, OUT>(a, s) : launch_few<2, OUT>(a, s);
    case kRows16:
      return nt && a.M <= 16 ? launch_rows<1, 2, 2, true, OUT>(a, dev, s) : launch_rows<1, 2, 2, false, OUT>(a, dev, s);
    case kRows32: return launch_rows<2, 2, 2, false, OUT>(a, dev, s);
    case kRows64: return launch_rows<4, 2, 2, false, OUT>(a, dev, s);
    case kLow: return launch_tile<LowTile, OUT>(a, dev, cus, s);
    case kSmall: return launch_tile<SmallTile, OUT>(a, dev, cus, s);
    case kMid: return launch_tile<MidTile, OUT>(a, dev, cus, s);
    default: return launch_tile<BigTile, OUT>(a, dev, cus, s);
  }
}

}  // namespace lq8

LinearQ8Form linear_q8_fwd_form(int64_t M, int64_t N, int64_t K) {
  int dev = 0, cus = 256;
  if (current_device(dev, cus) != hipSuccess) cus = 256;   // no device here
  const bool copies = lq8::pads(M, N, K, cus);
  if (K == 0 || (K % 16 != 0 && !copies)) return {8, 1, false};
  return {int(lq8::choose_form(M, N, lq8::padded(K), cus)), 1, copies};
}

size_t linear_q8_fwd_workspace(int64_t M, int64_t N, int64_t K) {
  int dev = 0, cus = 256;
  if (current_device(dev, cus) != hipSuccess) cus = 256;   // no device here
  return lq8::pads(M, N, K, cus) ? size_t(M + N) * size_t(lq8::padded(K)) : 0;
}

hipError_t launch_linear_q8_fwd(bool bf16, int64_t M, int64_t N, int64_t K, const int8_t* q, const float* scale,
                                const int8_t* w, const float* w_scale, const void* bias, void* y, void* workspace,
                                hipStream_t s) {
  lq8::Args a{q, w, scale, w_scale, bias, nullptr, y, M, N, K, K, K, nullptr, 0, 0, {}, 0};
  int dev = 0, cus = 0;
  hipError_t e = current_device(dev, cus);
  if (e != hipSuccess) return e;
  if (lq8::pads(M, N, K, cus)) {   // zeros behind the rows add nothing to the sums
    a.K = a.a_pitch = a.b_pitch = lq8::padded(K);
    int8_t* const rows = static_cast<int8_t*>(workspace);
    e = lq8::launch_pad(q, M, w, N, K, rows, a.K, s);
    if (e != hipSuccess) return e;
    a.a = rows;
    a.b = rows + M * a.K;
  }
  return bf16 ? lq8::launch_fwd<BF16>(a, s) : lq8::launch_fwd<F32>(a, s);
}

}  // namespace lmbp
