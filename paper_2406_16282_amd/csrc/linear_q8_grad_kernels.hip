// Input gradient of the linear layers of 8-bit rows and 8-bit weights, for gfx950.
//
//   dx = (sum_n p[m, n] w[n, k]) p_scale[m] + add,  p and p_scale the rows of dy[m, n] w_scale[n]
//                                                   in 8 bits (q8_kernels.hip)
//
// Here the product is y = a b with a = p [M x K], b = w [K x N]: K stands for the layer's output
// features, N for its input features. The sums are exact, as the forward's.
//
// What bounds it. Many rows: the card's power, as the forward; 8192 rows of 11008 x 4096 355 us, 44 of
// them dy to 8 bits (270 MB, 6.1 TB/s) and 311 the product (2380 TOPS); with its operands laid out this
// way the library's int8 product takes 475 to 496 us. 2000 rows of 4096 x 11008 97 us in a row, 114
// from memory: 688 tiles of 128 x 256 on 512 places. Few rows: the weight's bytes and the chain of K steps.
//
// b's columns are K-strided: its rows are staged as they lie in memory and read with the transposing
// LDS read (8 bytes to a lane). A ring slot holds 64 products, whole (that read wants 8 rows of each
// column), and a step has four segments of MFMAs with the loads of a later slot and the reads of the
// next fragments between them. After LDS loads issued by the compiler's builtin it waits for all of
// them before each such read; the loads are written as asm for that reason (they have no output
// registers, and every wait is written out). bf16 results are exchanged between neighbouring lane groups, so
// that a lane stores 8 consecutive ones.
//
// dy is brought to 8 bits by a kernel of its own: a row's scale is known only after the whole row,
// and every tile of columns needs the row. add (the other layers' gradients) is read in the epilogue.
#include "linear_q8_device.hpp"

#include <type_traits>

namespace lmbp {
namespace lq8 {
namespace tr {

using lin::lds_addr;
using lin::load_lds16_asm;
using lin::rsrc_words;

// 4 consecutive elements at any element's address.
template <class IO>
__device__ inline void load4(const void* p, int64_t i, float (&f)[4]) {
  if constexpr (IO::kBytes == 4) {
    const u32x4 v = *reinterpret_cast<const u32x4_at2*>(elem<IO>(p, i));
    F32::unpack(v, f);
  } else {
    const u32x2_at2 v = *reinterpret_cast<const u32x2_at2*>(elem<IO>(p, i));
    f[0] = __uint_as_float(v[0] << 16);
    f[1] = __uint_as_float(v[0] & 0xffff0000u);
    f[2] = __uint_as_float(v[1] << 16);
    f[3] = __uint_as_float(v[1] & 0xffff0000u);
  }
}
template <class IO>
__device__ inline void store4(void* p, int64_t i, const float (&f)[4]) {
  if constexpr (IO::kBytes == 4) store_16(elem<IO>(p, i), F32::pack(f));
  else *reinterpret_cast<u32x2_at2*>(elem<IO>(p, i)) = u32x2_at2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
}

// Results of a row at 4 columns from `col` on, f = sum * scale + add; columns from N on are 0.
template <class OUT>
__device__ inline void results4(const Args& a, int64_t row, int64_t col, const i32x4& v, float sc, float (&f)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = 0.0f;
  if (a.add != nullptr) {
    if (col + 4 <= a.N) load4<OUT>(a.add, row * a.N + col, f);
    else
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = col + e < a.N ? OUT::load1(a.add, row * a.N + col + e) : 0.0f;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = __builtin_fmaf(float(v[e]), sc, f[e]);
}
// The same, stored.
template <class OUT>
__device__ inline void finish4(const Args& a, int64_t row, int64_t col, const i32x4& v, float sc) {
  float f[4];
  results4<OUT>(a, row, col, v, sc, f);
  if (col + 4 <= a.N) {
    store4<OUT>(a.y, row * a.N + col, f);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < a.N) OUT::store1(a.y, row * a.N + col + e, f[e]);
  }
}

// Scheduling groups: DS LDS reads spread over the first half of MF MFMAs.
template <int MF, int DS, int I = 0>
__device__ inline void spread_reads() {
  if constexpr (I < MF) {
    constexpr int W = MF / 2 < 1 ? 1 : MF / 2;
    constexpr int ds = I < W ? DS * (I + 1) / W - DS * I / W : 0;
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if constexpr (ds > 0) __builtin_amdgcn_sched_group_barrier(0x100, ds, 0);
    spread_reads<MF, DS, I + 1>();
  }
}

constexpr int kTrStep = 64;   // products per ring slot
template <int BM_, int BN_, int WM_, int WN_, int MINW_, int RING_ = 4>
struct TrTile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, kMinWaves = MINW_;
  static constexpr int kWaves = WM * WN, kThreads = kWaves * kWave;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
  static constexpr int kSlot = (BM + BN) * kTrStep;
  static constexpr int kRing = RING_;
  static constexpr int kBlocksPerCu = kMinWaves * 4 / kWaves;
  static constexpr int kLA = BM / 16 / kWaves, kLB = BN / 16 / kWaves;
  static constexpr int kLdsBytes = kRing * kSlot;
  static_assert(TN == 4 && (BN == 128 || BN == 256), "wave tile; swizzle of b");
  static_assert(kLA >= 1 && kLB >= 1 && (BM / 16) % kWaves == 0 && (BN / 16) % kWaves == 0, "loads");
  static_assert(kLdsBytes * kBlocksPerCu <= 160 * 1024, "LDS per CU");
};

// SPLIT: a share of K per blockIdx.y, the sums to a.part.
template <class C, bool SPLIT, class OUT>
__global__ __launch_bounds__(C::kThreads, C::kMinWaves) void product_tr_tile(Args a) {
  constexpr int BM = C::BM, BN = C::BN, TM = C::TM, TN = C::TN, kWaves = C::kWaves;
  constexpr int kLA = C::kLA, kLB = C::kLB, kL = kLA + kLB, kRing = C::kRing, kSlot = C::kSlot;
  constexpr int kUnits = BN / 16;   // 16-byte units in a row of b's slot
  const int64_t M = a.M, N = a.N;
  const uint32_t pitch = uint32_t(a.b_pitch);
  extern __shared__ __attribute__((aligned(16))) int8_t lds[];
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = wave_in_block();
  const int wm = wave / C::WN, wn = wave % C::WN;
  const uint32_t tiles = a.map.tiles;
  const int first = SPLIT ? int(blockIdx.y) * a.share : 0, all_steps = int((a.K + kTrStep - 1) / kTrStep);
  const int steps = SPLIT && all_steps - first > a.share ? a.share : all_steps - first;   // of this share
  // Unit u of row r of the slot is stored at u ^ swz(r): no read meets a bank conflict (bits 2 and 3 of r
  // for a cost one more pass in each of its reads, 364 us instead of 355 for 8192 rows of 11008 x 4096).
  auto swz_a = [](int r) { return (r >> 1) & 3; };
  auto swz_b = [](int r) { return BN == 256 ? (r & 7) | (((r >> 4) & 1) << 3) : ((r >> 1) & 3) | (((r >> 4) & 1) << 2); };
  uint32_t ld_a[kLA], ld_b[kLB];
#pragma unroll
  for (int q = 0; q < kLA; ++q) {
    const int p = (wave + kWaves * q) * 64 + lane, r = p / 4;
    ld_a[q] = uint32_t(r) * uint32_t(a.a_pitch) + ((p % 4) ^ swz_a(r)) * 16;
  }
#pragma unroll
  for (int q = 0; q < kLB; ++q) {
    const int p = (wave + kWaves * q) * 64 + lane, r = p / kUnits;
    ld_b[q] = uint32_t(r) * pitch + ((p % kUnits) ^ swz_b(r)) * 16;
  }
  // Load cursor: slots of the tile still to load.
  uint32_t l_tile = blockIdx.x;
  int l_slots = 0;
  uint64_t pa = 0, pb = 0;
  uint32_t na = 0, nb = 0;   // records: bytes in range
  const uint32_t nb_step = kTrStep * pitch;
  const int64_t rows_left = a.K - int64_t(first + steps - 1) * kTrStep;
  const int last_rows = rows_left < kTrStep ? int(rows_left) : kTrStep;
  auto enter = [&]() {
    uint32_t tm = 0, tn = 0;
    const bool in = l_tile < tiles;   // past the last tile: zeros
    if (in) tile_of(l_tile, a.map, tm, tn);
    const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN;
    const uint32_t left = uint32_t(M - m0);   // M < 2^31
    pa = reinterpret_cast<uint64_t>(a.a + m0 * a.a_pitch) + uint64_t(first) * kTrStep;
    pb = reinterpret_cast<uint64_t>(a.b + n0) + uint64_t(first) * nb_step;
    na = in ? (left < uint32_t(BM) ? left : uint32_t(BM)) * uint32_t(a.a_pitch) - uint32_t(first) * kTrStep : 0u;
    nb = in ? uint32_t(steps == 1 ? last_rows : kTrStep) * pitch - uint32_t(n0) : 0u;
    l_slots = in ? steps : 0x7fffffff;
  };
  auto load = [&](uint32_t S, int q) {
    if (q < kLA) load_lds16_asm(rsrc_words(pa, na), S + (wave + kWaves * q) * 1024, ld_a[q < kLA ? q : 0]);
    else load_lds16_asm(rsrc_words(pb, nb), S + BM * kTrStep + (wave + kWaves * (q - kLA)) * 1024, ld_b[q < kLA ? 0 : q - kLA]);
  };
  auto advance = [&]() {
    if (--l_slots == 0) {
      l_tile += gridDim.x;
      enter();
    } else if (l_tile < tiles) {
      pa += kTrStep;
      na -= kTrStep;   // the rows are padded to whole slots
      pb += nb_step;
      if (l_slots == 1) nb -= uint32_t(kTrStep - last_rows) * pitch;
    }
  };

  const int g = lane >> 4, i16 = lane & 15;
  int a_at[TM], b_at[TN][2];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int r = (wm * TM + i) * 16 + i16;
    a_at[i] = r * kTrStep + (g ^ swz_a(r)) * 16;
  }
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = 16 * g + 8 * h + (i16 >> 1);
      b_at[j][h] = BM * kTrStep + r * BN + ((wn * TN + j) ^ swz_b(r)) * 16 + (i16 & 1) * 8;
    }
  i32x4 fa[2][TM], fb[2][TN];
  auto read_b = [&](const int8_t* S, int buf, int j) {
    const i32x2 lo = read_tr8(S + b_at[j][0]), hi = read_tr8(S + b_at[j][1]);
    fb[buf][j] = i32x4{lo[0], lo[1], hi[0], hi[1]};
  };
  auto read_a = [&](const int8_t* S, int buf, int i) { fa[buf][i] = *reinterpret_cast<const i32x4*>(S + a_at[i]); };
  i32x4 acc[TM][TN];
  // One slot: 4 segments of MFMAs of the fragments in buf, with the loads into slot `fill` and
  // the reads of the next fragments from slot S spread over them.
  auto segment = [&](auto number, int buf, uint32_t fill, const int8_t* S) {
    constexpr int sg = decltype(number)::value;
#pragma unroll
    for (int q = 0; q < kL; ++q)
      if (q * 4 / kL == sg) load(fill, q);
    if constexpr (sg == 0) {
#pragma unroll
      for (int j = 0; j < TN; ++j) read_b(S, buf ^ 1, j);
    } else if constexpr (sg < 3) {
#pragma unroll
      for (int i = (sg - 1) * TM / 2; i < sg * TM / 2; ++i) read_a(S, buf ^ 1, i);
    }
#pragma unroll
    for (int t = sg * TM * TN / 4; t < (sg + 1) * TM * TN / 4; ++t)
      acc[t / TN][t % TN] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[buf][t % TN], fa[buf][t / TN], acc[t / TN][t % TN], 0, 0, 0);
    spread_reads<TM * TN / 4, sg == 0 ? 2 * TN : sg < 3 ? TM / 2 : 0>();
    __builtin_amdgcn_sched_barrier(0);
  };
  auto half = [&](int buf, uint32_t fill, const int8_t* S) {
    segment(std::integral_constant<int, 0>{}, buf, fill, S);
    segment(std::integral_constant<int, 1>{}, buf, fill, S);
    segment(std::integral_constant<int, 2>{}, buf, fill, S);
    segment(std::integral_constant<int, 3>{}, buf, fill, S);
  };
  auto sync = [&]() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"((kRing - 2) * kL) : "memory");
    asm volatile("s_barrier" ::: "memory");
  };
  auto next = [&](int v, int d) { v += d; return v >= kRing ? v - kRing : v; };

  const uint32_t lds0 = lds_addr(lds);
  enter();
#pragma unroll
  for (int d = 0; d < kRing; ++d) {
#pragma unroll
    for (int q = 0; q < kL; ++q) load(lds0 + d * kSlot, q);
    advance();
  }
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"((kRing - 2) * kL) : "memory");
  asm volatile("s_barrier" ::: "memory");
  int slot = 0;
  for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < TN; ++j) read_b(lds + slot * kSlot, 0, j);
#pragma unroll
    for (int i = 0; i < TM; ++i) read_a(lds + slot * kSlot, 0, i);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    asm volatile("s_barrier" ::: "memory");
    for (int st = 0; st < steps; st += 2) {
      half(0, lds0 + slot * kSlot, lds + next(slot, 1) * kSlot);
      slot = next(slot, 1);
      advance();
      sync();
      if (st + 1 < steps) {
        half(1, lds0 + slot * kSlot, lds + next(slot, 1) * kSlot);
        slot = next(slot, 1);
        advance();
        sync();
      }
    }
    // Epilogue. The lane holds row lane % 16 and columns 4 g + 0 .. 3 of each 16 x 16 results.
    uint32_t tm, tn;
    tile_of(tile, a.map, tm, tn);
    const int64_t m0 = int64_t(tm) * BM + wm * TM * 16, n0 = int64_t(tn) * BN + wn * TN * 16;
    int lane_e = lane;
    asm volatile("" : "+v"(lane_e));
    if constexpr (SPLIT) {
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int64_t row = m0 + i * 16 + (lane_e & 15);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const int64_t col = n0 + j * 16 + (lane_e >> 4) * 4;
          if (row < M && col < N)
            *reinterpret_cast<i32x4*>(a.part + (int64_t(blockIdx.y) * M + row) * a.part_pitch + col) = acc[i][j];
        }
      }
      continue;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t row = m0 + i * 16 + (lane_e & 15);
      const float sc = row < M ? a.a_scale[row] : 0.0f;
      if constexpr (OUT::kBytes == 4) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
          if (row < M) finish4<OUT>(a, row, n0 + j * 16 + (lane_e >> 4) * 4, acc[i][j], sc);
      } else {   // neighbouring lane groups exchange halves: 8 consecutive columns to a lane
#pragma unroll
        for (int j = 0; j < TN; j += 2) {
          uint32_t v[2][2];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (row < M) results4<OUT>(a, row, n0 + (j + t) * 16 + (lane_e >> 4) * 4, acc[i][j + t], sc, f);
            v[t][0] = pack_bf16x2(f[0], f[1]);
            v[t][1] = pack_bf16x2(f[2], f[3]);
          }
          const auto s0 = __builtin_amdgcn_permlane16_swap(v[0][0], v[1][0], false, false);
          const auto s1 = __builtin_amdgcn_permlane16_swap(v[0][1], v[1][1], false, false);
          const int g4 = lane_e >> 4;
          const int64_t col = n0 + (j + (g4 & 1)) * 16 + (g4 >> 1) * 8;
          const u32x4 out = {s0[0], s1[0], s0[1], s1[1]};
          if (row < M) {
            if (col + 8 <= N) {
              store_16(elem<OUT>(a.y, row * N + col), out);
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (col + e < N) static_cast<uint16_t*>(a.y)[row * N + col + e] = uint16_t(out[e / 2] >> (16 * (e % 2)));
            }
          }
        }
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load into LDS outlives the block
}

// The shares' sums, added up in order (4 columns to a thread).
template <class OUT>
__global__ __launch_bounds__(256) void add_shares(Args a, int shares) {
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4, all = a.M * a.part_pitch;
  if (i >= all) return;
  i32x4 v = {0, 0, 0, 0};
  for (int p = 0; p < shares; ++p) v += *reinterpret_cast<const i32x4*>(a.part + p * all + i);
  const int64_t row = i / a.part_pitch;
  finish4<OUT>(a, row, i - row * a.part_pitch, v, a.a_scale[row]);
}
template <class OUT>
hipError_t launch_add_shares(const Args& a, int shares, hipStream_t s) {
  const int64_t blocks = (a.M * a.part_pitch + 1023) / 1024;
  hipLaunchKernelGGL((add_shares<OUT>), dim3(unsigned(blocks)), dim3(256), 0, s, a, shares);
  return hipGetLastError();
}

template <class C, bool SPLIT, class OUT>
hipError_t launch_tile(Args a, int shares, int dev, int cus, hipStream_t s) {
  if (!map_tiles(a, C::BM, C::BN)) return hipErrorInvalidValue;
  const hipError_t e = allow_lds<product_tr_tile<C, SPLIT, OUT>>(dev, C::kLdsBytes);
  if (e != hipSuccess) return e;
  shares = share_out(a, int((a.K + kTrStep - 1) / kTrStep), shares);
  const uint32_t slots = uint32_t(cus) * C::kBlocksPerCu;
  hipLaunchKernelGGL((product_tr_tile<C, SPLIT, OUT>), dim3(a.map.tiles < slots ? a.map.tiles : slots, unsigned(shares)),
                     dim3(C::kThreads), C::kLdsBytes, s, a);
  return SPLIT ? launch_add_shares<OUT>(a, shares, s) : hipGetLastError();
}

using BigTile = TrTile<256, 256, 2, 4, 2>;      // one block of 8 waves per CU
using MidTile = TrTile<128, 256, 1, 4, 2, 3>;   // two blocks of 4 waves
using SmallTile = TrTile<128, 128, 2, 2, 2>;    // two blocks of 4 waves
using LowTile = TrTile<64, 128, 2, 2, 3>;       // three blocks of 4 waves

// Few rows: a block of 4 waves takes MT x 16 rows of a and 64 columns of b, its waves the steps of
// 64 products in turn, each through an LDS ring of its own; the partial sums meet in LDS. With 16 rows,
// us, dy's rows and the shares' sum included: 11008 x 4096 22.5, with 128 columns to a block 21.5; 4096 x 4096
// 12.5 and 13.1, 768 x 768 7.0 and 7.9; rings of four steps instead of two 22.7, 13.0 and 7.7.
constexpr int kRowsWaves = 4;
template <int MT, int D>
constexpr int kTrRowsLds = kRowsWaves * D * (MT * 16 + 64) * kTrStep;

template <int MT, int D, class OUT>
__global__ __launch_bounds__(kRowsWaves * kWave) void product_tr_rows(Args a) {
  constexpr int kWaves = kRowsWaves, kRows = MT * 16, NB = 4;
  static_assert(kTrRowsLds<MT, D> <= 160 * 1024 && kTrRowsLds<MT, D> >= kWaves * MT * NB * 1024, "LDS; the partial sums");
  const int64_t M = a.M, N = a.N;
  const uint32_t pitch = uint32_t(a.b_pitch);
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = wave_in_block();
  const uint32_t blk = blockIdx.x, split = blockIdx.y;
  const uint32_t id = (blk < a.map.per_xcd * kXcds) ? (blk % kXcds) * a.map.per_xcd + blk / kXcds : blk;
  const int64_t m0 = int64_t(id % a.map.tiles_m) * kRows, n0 = int64_t(id / a.map.tiles_m) * 64;
  const uint32_t rows_a = uint32_t(M - m0 < kRows ? M - m0 : kRows);
  const int all_steps = int((a.K + kTrStep - 1) / kTrStep), first = int(split) * a.share;
  const int steps = all_steps < first + a.share ? all_steps : first + a.share;   // this share's end
  constexpr int kStep = (kRows + 64) * kTrStep, kLoads = MT + 4;
  extern __shared__ __attribute__((aligned(16))) int8_t lds[];
  int8_t* const ring = lds + wave * D * kStep;
  const uint32_t ring_at = lds_addr(lds) + wave * D * kStep;
  // Unit u (of 4) of row r at u ^ swz(r), 16 rows of 64 bytes to a load.
  auto swz_a = [](int r) { return (r >> 1) & 3; };
  auto swz_b = [](int r) { return ((r >> 2) & 1) | (((r >> 4) & 1) << 1); };
  uint32_t off_a[MT], off_b[4];
#pragma unroll
  for (int q = 0; q < MT; ++q) {
    const int r = q * 16 + lane / 4;
    off_a[q] = uint32_t(r) * uint32_t(a.a_pitch) + ((lane % 4) ^ swz_a(r)) * 16;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int r = q * 16 + lane / 4;
    off_b[q] = uint32_t(r) * pitch + ((lane % 4) ^ swz_b(r)) * 16;
  }
  const uint64_t pa = reinterpret_cast<uint64_t>(a.a + m0 * a.a_pitch), pb = reinterpret_cast<uint64_t>(a.b + n0);
  auto load = [&](int step, int d) {
    const uint32_t S = ring_at + d * kStep;
    const int64_t left = step < steps ? a.K - int64_t(step) * kTrStep : 0;   // rows of b from this step on
    const uint32_t rows_b = left <= 0 ? 0u : left < kTrStep ? uint32_t(left) : uint32_t(kTrStep);
    const u32x4 ra = rsrc_words(pa + uint64_t(step) * kTrStep, rows_b == 0 ? 0u : rows_a * uint32_t(a.a_pitch) - uint32_t(step) * kTrStep);
    const u32x4 rb = rsrc_words(pb + uint64_t(step) * kTrStep * pitch, rows_b == 0 ? 0u : rows_b * pitch - uint32_t(n0));
#pragma unroll
    for (int q = 0; q < MT; ++q) load_lds16_asm(ra, S + q * 1024, off_a[q]);
#pragma unroll
    for (int q = 0; q < 4; ++q) load_lds16_asm(rb, S + kRows * kTrStep + q * 1024, off_b[q]);
  };
  const int g = lane >> 4, i16 = lane & 15;
  i32x4 acc[MT][NB];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
#pragma unroll
  for (int d = 0; d < D; ++d) load(first + wave + d * kWaves, d);   // steps past the end read zeros
  int d = 0;
  for (int st = first + wave; st < steps; st += kWaves) {
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"((D - 1) * kLoads) : "memory");
    const int8_t* S = ring + d * kStep;
    i32x4 fa[MT], fb[NB];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int r = i * 16 + i16;
      fa[i] = *reinterpret_cast<const i32x4*>(S + r * kTrStep + (g ^ swz_a(r)) * 16);
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int r0 = 16 * g + (i16 >> 1), r1 = r0 + 8;
      const int8_t* B = S + kRows * kTrStep + (i16 & 1) * 8;
      const i32x2 lo = read_tr8(B + r0 * 64 + (j ^ swz_b(r0)) * 16), hi = read_tr8(B + r1 * 64 + (j ^ swz_b(r1)) * 16);
      fb[j] = i32x4{lo[0], lo[1], hi[0], hi[1]};
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before it is loaded over
    __builtin_amdgcn_sched_barrier(0);
    load(st + D * kWaves, d);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    d = d + 1 == D ? 0 : d + 1;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // as in product_rows
  __syncthreads();
  auto part = reinterpret_cast<i32x4 (*)[MT][NB][kWave]>(lds);
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) part[wave][i][j][lane] = acc[i][j];
  __syncthreads();
#pragma unroll
  for (int q = 0; q < (MT * NB + kWaves - 1) / kWaves; ++q) {
    const int tile = wave + q * kWaves, i = tile / NB, j = tile % NB;
    if (tile >= MT * NB) return;
    i32x4 v = part[0][i][j][lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += part[w][i][j][lane];
    const int64_t row = m0 + i * 16 + i16, col = n0 + j * 16 + g * 4;
    if (row >= M || col >= N) continue;
    if (a.part != nullptr) {
      *reinterpret_cast<i32x4*>(a.part + (int64_t(split) * M + row) * a.part_pitch + col) = v;
      continue;
    }
    finish4<OUT>(a, row, col, v, a.a_scale[row]);
  }
}

template <int MT, int D, class OUT>
hipError_t launch_rows(Args a, int shares, hipStream_t s) {
  if (!map_tiles(a, MT * 16, 64) || a.map.tiles > most_blocks(kRowsWaves * kWave)) return hipErrorInvalidValue;
  shares = share_out(a, int((a.K + kTrStep - 1) / kTrStep), shares);
  if (shares == 1) a.part = nullptr;
  static_assert(kTrRowsLds<MT, D> <= 64 * 1024, "no more than is allowed without asking");
  hipLaunchKernelGGL((product_tr_rows<MT, D, OUT>), dim3(a.map.tiles, unsigned(shares)), dim3(kRowsWaves * kWave),
                     (kTrRowsLds<MT, D>), s, a);
  return shares > 1 ? launch_add_shares<OUT>(a, shares, s) : hipGetLastError();
}

enum Form { kRows16, kRows32, kRows64, kLow, kSmall, kMid, kBig, kForms };
struct Plan {
  Form form;
  int shares;   // of K, for the rows forms and the lowest tiles
};

constexpr RowsCost kRows16Cost = {2.6f, 0.2819f, 0.1857f, 0.6247f, 0.002049f, 0.02439f, 0.1592f, 0.7644f, 2.624f, 0.6724f};
constexpr RowsCost kRows32Cost = {3.066f, 0.3273f, 0.2738f, 0.6311f, 0.00255f, 0.02104f, 0.1365f, 0.5573f, 2.53f, 0.5608f};
constexpr RowsCost kRows64Cost = {3.941f, 0.4253f, 0.4258f, 0.6417f, 0.004474f, 0.01234f, 0.07593f, 0.5821f, 2.654f, 0.5531f};
constexpr TileCost kLowCost = {4.0f, 0.5062f, 0.2452f, 0.1427f, 0.1589f, 0.08949f, 0.2922f, 2.38f, 0.4422f};
constexpr TileCost kSmallCost = {5.062f, 0.5398f, 0.3443f, 0.1797f, 0, 0, 0.3102f, 0, 0};
constexpr TileCost kMidCost = {7.429f, 0.8145f, 0.4905f, 0.2797f, 0, 0.006095f, 0.2591f, 0, 0};
constexpr TileCost kBigCost = {8.289f, 0.793f, 0.7208f, 0, 0, 0, 0.2536f, 0, 0};

// The form by the estimates (linear_q8_device.hpp), their constants fitted to 420 sizes of 15 layers as
// the forward's: 0.8% slower than the best on average, 16% at worst (0.8% on layers left out). Both sides,
// us, dy's rows included: 11008 x 4096 at 16 rows 16-row blocks 45.3, K split over 2 of them 29.5, 4 21.3,
// 8 22.9; at 64 rows 64-row blocks 57.7, over 4 26.8, 64x128 tiles over 8 24.1; 128 rows 64-row blocks over
// 2 36.0, 64x128 64.8, over 2 41.1, over 4 29.4; 197 rows 64-row blocks 46.2, 64x128 54.0, over 2 36.8; 1024
// rows 64x128 90, 128x128 80, 128x256 99; 1576 rows 128x128 122, 128x256 107; 8192 rows 128x256 388, 256x256 364.
// 768 x 768 at 1024 rows 32-row blocks 9.9, 64x128 10.3; at 1576 rows 12.5 and 11.3.
// The partial sums of a split K stay below 32 MiB, and K below 1024 is not split (at 16 rows of 768 x 768
// 8.3 us against 6.4). The forward's K is not split over blocks: over the same sizes it gave 0.3%.
Plan make_plan(int64_t M, int64_t N, int64_t K, int cus, float* time = nullptr) {
  Plan best{kLow, 1};
  float least = tile_cost<LowTile>(M, N, K, kTrStep, 1, cus, kLowCost);
  auto take = [&](Form f, int shares, float t) {
    if (t < least) {
      least = t;
      best = {f, shares};
    }
  };
  take(kSmall, 1, tile_cost<SmallTile>(M, N, K, kTrStep, 1, cus, kSmallCost));
  take(kMid, 1, tile_cost<MidTile>(M, N, K, kTrStep, 1, cus, kMidCost));
  take(kBig, 1, tile_cost<BigTile>(M, N, K, kTrStep, 1, cus, kBigCost));
  for (int shares = 1; shares <= 8 && M <= 1024; shares *= 2) {
    if (shares > 1 && (K < 1024 || int64_t(shares) * M * N * 4 > (int64_t(32) << 20))) break;
    take(kRows16, shares, rows_cost(M, N, K, 16, 64, kTrStep, 4, shares, cus, kRows16Cost));
    take(kRows32, shares, rows_cost(M, N, K, 32, 64, kTrStep, 3, shares, cus, kRows32Cost));
    take(kRows64, shares, rows_cost(M, N, K, 64, 64, kTrStep, 2, shares, cus, kRows64Cost));
    if (shares > 1) take(kLow, shares, tile_cost<LowTile>(M, N, K, kTrStep, shares, cus, kLowCost));
  }
  if (time) *time = least;
  return best;
}

// Whether b's rows are copied to aligned ones first.
bool pads(int64_t M, int64_t N, int64_t K, int cus) {
  if (N % 16 == 0 || M == 0 || K == 0 || N >= (1 << 24)) return false;
  float fast;
  make_plan(M, padded(N), K, cus, &fast);
  return pad_pays(M, N, K, K, N, fast);
}

template <class OUT>
hipError_t launch(const Args& a, hipStream_t s) {
  // b's rows start on 16-byte boundaries and a ring slot's 64 rows fit a buffer resource.
  const bool aligned = a.K > 0 && a.b_pitch % 16 == 0 && a.b_pitch <= (1 << 24) && reinterpret_cast<uintptr_t>(a.b) % 16 == 0;
  if (!aligned) return launch_any<OUT, true>(a, s);
  int dev = 0, cus = 0;
  const hipError_t e = current_device(dev, cus);
  if (e != hipSuccess) return e;
  const Plan plan = make_plan(a.M, a.b_pitch, a.K, cus);
  switch (plan.form) {
    case kRows16: return launch_rows<1, 2, OUT>(a, plan.shares, s);
    case kRows32: return launch_rows<2, 2, OUT>(a, plan.shares, s);
    case kRows64: return launch_rows<4, 2, OUT>(a, plan.shares, s);
    case kLow:
      return plan.shares > 1 ? launch_tile<LowTile, true, OUT>(a, plan.shares, dev, cus, s)
                             : launch_tile<LowTile, false, OUT>(a, 1, dev, cus, s);
    case kSmall: return launch_tile<SmallTile, false, OUT>(a, 1, dev, cus, s);
    case kMid: return launch_tile<MidTile, false, OUT>(a, 1, dev, cus, s);
    default: return launch_tile<BigTile, false, OUT>(a, 1, dev, cus, s);
  }
}

// Rows of p start on 128-byte lines and are padded with zeros to whole K steps.
int64_t pitch_of(int64_t n) { return (n + 127) / 128 * 128; }
size_t more_at(int64_t m, int64_t n) { return (size_t(m) * size_t(pitch_of(n)) + size_t(m) * 4 + 15) / 16 * 16; }

}  // namespace tr
}  // namespace lq8

LinearQ8Form linear_q8_bwd_form(int64_t M, int64_t N, int64_t K) {
  int dev = 0, cus = 256;
  if (current_device(dev, cus) != hipSuccess) cus = 256;   // no device here
  const bool copies = lq8::tr::pads(M, K, N, cus);
  if (N == 0 || (K % 16 != 0 && !copies)) return {8, 1, false};
  const lq8::tr::Plan plan = lq8::tr::make_plan(M, lq8::padded(K), N, cus);
  return {int(plan.form) + 1, plan.shares, copies};
}

// p, its scales, the copy of w, and the sums of the shares, 16-byte aligned.
size_t linear_q8_bwd_workspace(int64_t M, int64_t N, int64_t K) {
  int dev = 0, cus = 256;
  if (current_device(dev, cus) != hipSuccess) cus = 256;   // no device here
  const size_t pitch = size_t(lq8::padded(K)), copy = lq8::tr::pads(M, K, N, cus) ? size_t(N) * pitch : 0;
  const lq8::tr::Plan plan = lq8::tr::make_plan(M, int64_t(pitch), N, cus);
  return lq8::tr::more_at(M, N) + copy + (plan.shares > 1 ? size_t(plan.shares) * size_t(M) * pitch * 4 : 0);
}

hipError_t launch_linear_q8_bwd(bool bf16, bool dx_bf16, int64_t M, int64_t N, int64_t K, const void* dy, const int8_t* w,
                                const float* w_scale, const void* add, void* dx, void* workspace, hipStream_t s) {
  const int64_t pitch = lq8::tr::pitch_of(N);
  int8_t* const p = static_cast<int8_t*>(workspace);
  float* const p_scale = reinterpret_cast<float*>(p + M * pitch);
  if (N > 0) {
    const hipError_t e = launch_q8_rows(bf16, M, N, pitch, dy, w_scale, p, p_scale, s);
    if (e != hipSuccess) return e;
  }
  int8_t* more = p + lq8::tr::more_at(M, N);
  lq8::Args a{p, w, N > 0 ? p_scale : nullptr, nullptr, nullptr, add, dx, M, K, N, pitch, K, nullptr, lq8::padded(K), 0, {}, 0};
  int dev = 0, cus = 0;
  const hipError_t e = current_device(dev, cus);
  if (e != hipSuccess) return e;
  if (lq8::tr::pads(M, K, N, cus)) {
    a.b_pitch = lq8::padded(K);
    const hipError_t ep = lq8::launch_pad(w, N, nullptr, 0, K, more, a.b_pitch, s);
    if (ep != hipSuccess) return ep;
    a.b = more;
    more += N * a.b_pitch;
  }
  a.part = reinterpret_cast<int32_t*>(more);
  return dx_bf16 ? lq8::tr::launch<BF16>(a, s) : lq8::tr::launch<F32>(a, s);
}

}  // namespace lmbp
