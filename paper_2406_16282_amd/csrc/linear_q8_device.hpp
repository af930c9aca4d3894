// The products of 8-bit rows and 8-bit weights: what the forward's and the input gradient's kernels
// share (gfx950).
#pragma once

#include "lmbp_device.hpp"
#include "lmbp_launch.hpp"
#include "tile_device.hpp"

#include <algorithm>
#include <atomic>
#include <cmath>

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
  int64_t M, N, K, a_pitch, b_pitch;   // bytes from one row to the next
  int32_t* part;          // [shares][M x part_pitch] sums over shares of K, or null
  int64_t part_pitch;     // N in whole sixteens
  int32_t share;          // steps of K to a share
  TileMap map;
  uint32_t first;         // product_any, product_few: blocks of the launches before (in_parts)
};

// 16 and 8 bytes at any element's address (global memory takes such accesses).
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));
__device__ inline void store_16(void* p, const u32x4& v) { *static_cast<u32x4_at2*>(p) = v; }
template <class IO>
__device__ inline char* elem(const void* p, int64_t i) {
  return const_cast<char*>(static_cast<const char*>(p)) + i * IO::kBytes;
}

// 16 bytes of a matrix of `total` bytes (16 at least) from byte `at` on, at any alignment; those
// that start less than 16 before its end are read from 16 before its end (mend shifts them).
__device__ inline u32x4 fetch(const int8_t* base, int64_t total, int64_t at) {
  return *reinterpret_cast<const u32x4_at1*>(base + (at < total - 16 ? at : total - 16));
}
// What `fetch` read, with byte `at` first and zeros from the count-th on.
__device__ inline u32x4 mend(const u32x4& v, int64_t total, int64_t at, int64_t count) {
  uint64_t lo = uint64_t(v[1]) << 32 | v[0], hi = uint64_t(v[3]) << 32 | v[2];
  const int by = at > total - 16 ? 8 * int(at - (total - 16)) : 0;   // bits
  const int keep = count <= 0 ? 0 : count < 16 ? 8 * int(count) : 128;
  if (by >= 64) {
    lo = by < 128 ? hi >> (by - 64) : 0;
    hi = 0;
  } else if (by > 0) {
    lo = lo >> by | hi << (64 - by);
    hi >>= by;
  }
  if (keep < 64) {
    lo &= (uint64_t(1) << keep) - 1;
    hi = 0;
  } else if (keep < 128) {
    hi &= (uint64_t(1) << (keep - 64)) - 1;
  }
  return u32x4{uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32)};
}
// The same of a matrix of any size.
__device__ inline u32x4 few_bytes(const int8_t* base, int64_t at, int64_t count) {
  u32x4 v = {0u, 0u, 0u, 0u};
  for (int i = 0; i < 16 && i < count; ++i) v[i / 4] |= uint32_t(uint8_t(base[at + i])) << (8 * (i % 4));
  return v;
}

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
// Transposing LDS read: of 16 lanes, lane q passes the address of columns 8 (q % 2) .. + 7 of row
// q / 2 and lane i gets the 8 rows of column i (checked on the hardware).
__device__ inline i32x2 read_tr8(const int8_t* p) {
  return __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(p));
}

// Any sizes and alignments. A block takes 64 x 64 results; its 4 waves take the steps of 64 products
// in turn, each through registers (the next step's loads under way) and LDS of its own, so that the
// loop has no barrier, and the partial sums meet in LDS. Rows that do not start on 16-byte
// boundaries rule out the loads straight into LDS. What bounds it: the chain of loads (0.65 us a
// step) for small sizes, the way through registers for large ones (450 TOPS: 3000 x 3001 x 2999 in
// 127 us). Every load is made, at a clamped address: branches around them let none run ahead.
constexpr int kAnyRow = 80;   // LDS bytes to a row of 64: 16 rows' pieces in distinct banks
template <class OUT, bool TR>
__global__ __launch_bounds__(256) void product_any(Args a) {
  __shared__ __attribute__((aligned(16))) int8_t lds[64 * 1024];
  const int lane = threadIdx.x & (kWave - 1), wave = wave_in_block();
  const int64_t tiles_n = (a.N + 63) / 64;
  const int64_t block = int64_t(a.first) + blockIdx.x, m0 = block / tiles_n * 64, n0 = block % tiles_n * 64;
  int8_t* const la = lds + wave * 2 * 64 * kAnyRow;
  int8_t* const lb = la + 64 * kAnyRow;
  const int r = lane / 4, c = (lane % 4) * 16, g = lane >> 4, i16 = lane & 15;
  const int64_t a_bytes = a.M * a.a_pitch, b_bytes = a.N * a.K;
  const bool tiny = a_bytes < 16 || b_bytes < 16;
  // Rows beyond the matrices are read as their last ones (their results are not stored, and the
  // backward's a holds zeros there), so that every load is made: 8 of them under way, no branch.
  int64_t row_a[4], row_b[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    row_a[q] = std::min<int64_t>(m0 + q * 16 + r, a.M - 1) * a.a_pitch;
    row_b[q] = TR ? 0 : std::min<int64_t>(n0 + q * 16 + r, a.N - 1) * a.K;
  }
  auto at_a = [&](int q, int64_t k0) { return row_a[q] + k0 + c; };
  auto at_b = [&](int q, int64_t k0) {
    return TR ? std::min<int64_t>(k0 + q * 16 + r, a.K - 1) * a.N + n0 + c : row_b[q] + k0 + c;
  };
  u32x4 va[4], vb[4];
  auto load = [&](int64_t k0) {
    if (tiny) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        va[q] = few_bytes(a.a, at_a(q, k0), a.K - k0 - c);
        vb[q] = few_bytes(a.b, at_b(q, k0), TR ? a.N - n0 - c : a.K - k0 - c);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        va[q] = fetch(a.a, a_bytes, at_a(q, k0));
        vb[q] = fetch(a.b, b_bytes, at_b(q, k0));
      }
    }
  };
  i32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  int64_t k0 = int64_t(wave) * 64;
  if (k0 < a.K) load(k0);
  for (; k0 < a.K; k0 += 256) {
    // The step that ends the rows of both, or (TR) that holds rows of b within 16 bytes of its end:
    // one of its last 17 rows, where it is one byte wide.
    if (!tiny && k0 + (TR ? 80 : 64) >= a.K) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        va[q] = mend(va[q], a_bytes, at_a(q, k0), a.K - k0 - c);
        vb[q] = mend(vb[q], b_bytes, at_b(q, k0), TR ? 16 : a.K - k0 - c);
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      *reinterpret_cast<u32x4*>(la + (q * 16 + r) * kAnyRow + c) = va[q];
      *reinterpret_cast<u32x4*>(lb + (q * 16 + r) * kAnyRow + c) = vb[q];
    }
    if (k0 + 256 < a.K) load(k0 + 256);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // written by this wave's other lanes
    i32x4 fa[4], fb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      fa[i] = *reinterpret_cast<const i32x4*>(la + (i * 16 + i16) * kAnyRow + g * 16);
      if constexpr (TR) {
        const int8_t* p = lb + (16 * g + (i16 >> 1)) * kAnyRow + i * 16 + (i16 & 1) * 8;
        const i32x2 lo = read_tr8(p), hi = read_tr8(p + 8 * kAnyRow);
        fb[i] = i32x4{lo[0], lo[1], hi[0], hi[1]};
      } else {
        fb[i] = *reinterpret_cast<const i32x4*>(lb + (i * 16 + i16) * kAnyRow + g * 16);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before it is written over
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
  }
  __syncthreads();
  auto part = reinterpret_cast<i32x4 (*)[4][4][kWave]>(lds);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) part[wave][i][j][lane] = acc[i][j];
  __syncthreads();
  // The lane holds row lane % 16 and columns 4 (lane / 16) + 0 .. 3 of each 16 x 16 results.
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    i32x4 v = part[0][wave][j][lane];
#pragma unroll
    for (int w = 1; w < 4; ++w) v += part[w][wave][j][lane];
    const int64_t m = m0 + wave * 16 + i16;
    if (m >= a.M) return;
    const float as = a.a_scale != nullptr ? a.a_scale[m] : 1.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t n = n0 + j * 16 + g * 4 + e;
      if (n < a.N) {
        // Nothing to add up (K = 0) is 0 whatever the scales are, infinite and NaN ones among them.
        const float sc = a.K == 0 ? 0.0f : TR ? as : as * a.b_scale[n];
        const float more = TR ? (a.add != nullptr ? OUT::load1(a.add, m * a.N + n) : 0.0f)
                              : (a.bias != nullptr ? OUT::load1(a.bias, n) : 0.0f);
        OUT::store1(a.y, m * a.N + n, __builtin_fmaf(float(v[e]), sc, more));
      }
    }
  }
}

template <class OUT, bool TR>
hipError_t launch_any(Args a, hipStream_t s) {
  const int64_t blocks = ((a.M + 63) / 64) * ((a.N + 63) / 64);
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  return in_parts(blocks, most_blocks(256), [&](int64_t first, int64_t count) {
    a.first = uint32_t(first);
    hipLaunchKernelGGL((product_any<OUT, TR>), dim3(unsigned(count)), dim3(256), 0, s, a);
  });
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

// Steps to a share, and the shares that then hold any.
inline int share_out(Args& a, int steps, int shares) {
  a.share = (steps + shares - 1) / shares;
  return (steps + a.share - 1) / a.share;
}

// Rows of `cols` bytes at any address, copied to rows `pitch` (a multiple of 16) bytes apart with
// zeros behind them: those of `src`, then those of `src2`. A wave to a row.
__global__ inline __launch_bounds__(256) void pad_rows(const int8_t* src, int64_t rows, const int8_t* src2, int64_t rows2,
                                                       int64_t cols, int8_t* dst, int64_t pitch, int64_t first) {
  int64_t row = (first + blockIdx.x) * 4 + wave_in_block();
  if (row >= rows + rows2) return;
  int8_t* const to = dst + row * pitch;
  if (row >= rows) {
    row -= rows;
    src = src2;
    rows = rows2;
  }
  const int64_t total = rows * cols;
  for (int64_t k = int64_t(threadIdx.x & (kWave - 1)) * 16; k < pitch; k += kWave * 16) {
    const int64_t at = row * cols + k;
    const u32x4 v = total < 16 ? few_bytes(src, at, cols - k) : mend(fetch(src, total, at), total, at, cols - k);
    *reinterpret_cast<u32x4*>(to + k) = v;
  }
}
inline hipError_t launch_pad(const int8_t* src, int64_t rows, const int8_t* src2, int64_t rows2, int64_t cols, int8_t* dst,
                             int64_t pitch, hipStream_t s) {
  return in_parts((rows + rows2 + 3) / 4, most_blocks(256), [&](int64_t first, int64_t count) {
    hipLaunchKernelGGL(pad_rows, dim3(unsigned(count)), dim3(256), 0, s, src, rows, src2, rows2, cols, dst, pitch, first);
  });
}
inline int64_t padded(int64_t bytes) { return (bytes + 15) / 16 * 16; }

// Whether rows of k bytes that are no multiple of 16 are worth a copy to ones that are: `fast` is the
// estimated time of the product after it, `copied` the rows. The general form takes a chain of K
// steps and 450 TOPS, the copy a launch and 3 TB/s. Both sides, without and with the copy: 333 rows of
// 1001 x 1023 10.9 and 9.0 us, 3000 of 3001 x 2999 127 and 58 (the gradient 123 and 64).
inline bool pad_pays(int64_t M, int64_t N, int64_t K, int64_t copied, int64_t k, float fast) {
  const float any = 5.5f + 0.65f * float((K + 255) / 256) + float(M) * float(N) * float(K) * (2.0f / 450e6f);
  return fast + 2.5f + float(copied) * float(k) * (1.0f / 3e6f) < any;
}

// Estimated times, in us, by which a form is chosen. Tiles: full rounds of the resident blocks and a
// partial one, in which a CU with one block (or two of three) is faster; the bytes of the weight and
// the results. Rows forms: the chain of a wave's K steps, longer where a CU has several blocks, in
// every further round of them, and with a weight that the caches do not hold; the bytes that all
// blocks take in. Both: a second kernel and the partial sums' bytes where K is split over blocks.
struct TileCost {
  float base, step_full, step_first, step_second, step_third, w_mb, out_mb, split, part_mb;
};
template <class C>
float tile_cost(int64_t M, int64_t N, int64_t K, int k_step, int shares, int cus, const TileCost& c) {
  const int64_t tiles = ((M + C::BM - 1) / C::BM) * ((N + C::BN - 1) / C::BN) * shares, slots = int64_t(cus) * C::kBlocksPerCu;
  const int64_t rest = tiles % slots, steps = (K + k_step - 1) / k_step;
  const float per_step = c.step_full * float(tiles / slots) + c.step_first * float(rest > 0) +
                         c.step_second * float(rest > cus) + c.step_third * float(rest > 2 * int64_t(cus));
  const float out = float(M) * float(N);
  return c.base + float((steps + shares - 1) / shares) * per_step + c.w_mb * float(N) * float(K) * 1e-6f + c.out_mb * out * 2e-6f +
         (shares > 1 ? c.split + c.part_mb * float(shares) * out * 4e-6f : 0.0f);
}
struct RowsCost {
  float base, chain, chain_second, chain_round, chain_w, mb, w_mb, out_mb, split, part_mb;
};
// blocks_per_cu: those that fit by their LDS.
inline float rows_cost(int64_t M, int64_t N, int64_t K, int bm, int bn, int k_step, int blocks_per_cu, int shares, int cus,
                       const RowsCost& c) {
  const int64_t tiles = ((M + bm - 1) / bm) * ((N + bn - 1) / bn), steps = (K + k_step - 1) / k_step;
  const float chain = float(((steps + shares - 1) / shares + 3) / 4);   // 4 waves take the steps in turn
  const float per_cu = float(tiles * shares) / float(cus), w_mb = float(N) * float(K) * 1e-6f;
  const float rounds = std::ceil(per_cu / float(blocks_per_cu)) - 1.0f;
  const float out = float(M) * float(N);
  return c.base + chain * (c.chain + c.chain_second * float(per_cu > 1.0f) + c.chain_round * rounds +
                           c.chain_w * std::min(w_mb, 64.0f)) +
         c.mb * float(tiles) * float(steps) * float((bm + bn) * k_step) * 1e-6f + c.w_mb * w_mb + c.out_mb * out * 2e-6f +
         (shares > 1 ? c.split + c.part_mb * float(shares) * out * 4e-6f : 0.0f);
}

}  // namespace lq8
}  // namespace lmbp
