// The products of 8-bit rows and 8-bit weights: what the forward's and the input gradient's kernels
// share (gfx950).
#pragma once

#include "lmbp_device.hpp"
#include "lmbp_launch.hpp"
#include "tile_device.hpp"

#include <atomic>

namespace lmbp {
namespace lq8 {

using lin::kOutOfRange;
using lin::load_lds16;
using lin::load_lds4;
using lin::make_rsrc;
using lin::spread;
using lin::tile_of;
using lin::TileMap;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_at1 __attribute__((ext_vector_type(4), aligned(1)));

struct Args {
  const int8_t* a;        // [M x K], rows a_pitch bytes apart
  const int8_t* b;        // forward: [N x K]; input gradient (TR): [K x N]
  const float* a_scale;   // per row; null where there is nothing to add up (K = 0)
  const float* b_scale;   // forward: per column of the result
  const void* bias;       // forward: per column, of the result's type, or null
  const void* add;        // input gradient: [M x N] of the result's type, or null; may be y
  void* y;                // [M x N]
  int64_t M, N, K, a_pitch;
  bool vec;               // forward: y takes 16-byte stores
  TileMap map;
};

// 16 bytes of a row from byte k0 on, zeros from byte `end` on; any alignment.
__device__ inline u32x4 row_piece(const int8_t* row, int64_t k0, int64_t end) {
  if (k0 + 16 <= end) return *reinterpret_cast<const u32x4_at1*>(row + k0);
  u32x4 v = {0u, 0u, 0u, 0u};
  for (int i = 0; i < 16 && k0 + i < end; ++i) v[i / 4] |= uint32_t(uint8_t(row[k0 + i])) << (8 * (i % 4));
  return v;
}

// Any sizes and alignments: a block of 4 waves takes 64 x 64 results, 64 products at a time,
// both operands staged through registers into LDS with the products contiguous.
template <class OUT, bool TR>
__global__ __launch_bounds__(256) void product_any(Args a) {
  constexpr int kStep = 64, kRow = kStep + 16;
  __shared__ __attribute__((aligned(16))) int8_t la[64 * kRow], lb[64 * kRow];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = wave_in_block();
  const int64_t tiles_n = (a.N + 63) / 64;
  const int64_t m0 = int64_t(blockIdx.x) / tiles_n * 64, n0 = int64_t(blockIdx.x) % tiles_n * 64;
  i32x4 acc[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = i32x4{0, 0, 0, 0};
  const int r = tid / 4, c = (tid % 4) * 16;
  for (int64_t k0 = 0; k0 < a.K; k0 += kStep) {
    u32x4 va = {0u, 0u, 0u, 0u}, vb = {0u, 0u, 0u, 0u};
    if (m0 + r < a.M) va = row_piece(a.a + (m0 + r) * a.a_pitch, k0 + c, a.K);
    if constexpr (TR) {
      if (k0 + r < a.K) vb = row_piece(a.b + (k0 + r) * a.N, n0 + c, a.N);
    } else {
      if (n0 + r < a.N) vb = row_piece(a.b + (n0 + r) * a.K, k0 + c, a.K);
    }
    __syncthreads();
    *reinterpret_cast<u32x4*>(la + r * kRow + c) = va;
    if constexpr (TR) {
      for (int i = 0; i < 16; ++i) lb[(c + i) * kRow + r] = int8_t(vb[i / 4] >> (8 * (i % 4)));
    } else {
      *reinterpret_cast<u32x4*>(lb + r * kRow + c) = vb;
    }
    __syncthreads();
    const i32x4 fa = *reinterpret_cast<const i32x4*>(la + (wave * 16 + (lane & 15)) * kRow + (lane >> 4) * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const i32x4 fb = *reinterpret_cast<const i32x4*>(lb + (j * 16 + (lane & 15)) * kRow + (lane >> 4) * 16);
      acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb, fa, acc[j], 0, 0, 0);
    }
  }
  // The lane holds row lane % 16 and columns 4 (lane / 16) + 0 .. 3 of each 16 x 16 results.
  const int64_t m = m0 + wave * 16 + (lane & 15);
  if (m >= a.M) return;
  const float as = a.a_scale != nullptr ? a.a_scale[m] : 1.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t n = n0 + j * 16 + (lane >> 4) * 4 + e;
      if (n < a.N) {
        const float sc = TR ? as : as * a.b_scale[n];
        const float more = TR ? (a.add != nullptr ? OUT::load1(a.add, m * a.N + n) : 0.0f)
                              : (a.bias != nullptr ? OUT::load1(a.bias, n) : 0.0f);
        OUT::store1(a.y, m * a.N + n, __builtin_fmaf(float(acc[j][e]), sc, more));
      }
    }
}

template <class OUT, bool TR>
hipError_t launch_any(const Args& a, hipStream_t s) {
  const int64_t blocks = ((a.M + 63) / 64) * ((a.N + 63) / 64);
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((product_any<OUT, TR>), dim3(unsigned(blocks)), dim3(256), 0, s, a);
  return hipGetLastError();
}

// More than 64 KiB of dynamic LDS must be allowed explicitly, per kernel and device: done on the
// first launch on each device.
template <auto Kernel>
hipError_t allow_lds(int dev, int bytes) {
  static std::atomic<bool> done[kMaxDevices];
  if (bytes <= 64 * 1024 || done[dev].load(std::memory_order_acquire)) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(Kernel),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done[dev].store(true, std::memory_order_release);
  return e;
}

// The grid of tiles; false if there are too many.
inline bool map_tiles(Args& a, int bm, int bn) {
  const int64_t tiles_m = (a.M + bm - 1) / bm, tiles_n = (a.N + bn - 1) / bn, tiles = tiles_m * tiles_n;
  if (tiles > 0x3fffffff) return false;
  a.map = {uint32_t(tiles_m), uint32_t(tiles_n), uint32_t(tiles), uint32_t(tiles / kXcds),
           uint32_t((uint64_t(1) << 32) / uint64_t(tiles_n) - (tiles_n == 1))};
  return true;
}

}  // namespace lq8
}  // namespace lmbp
