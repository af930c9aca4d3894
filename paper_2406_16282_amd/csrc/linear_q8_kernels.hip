// Linear layers of 8-bit rows and 8-bit weights, for gfx950.
//
//   linear_q8_fwd : y = (sum_k q[m, k] w[n, k]) scale[m] w_scale[n] + bias[n]
//   linear_q8_bwd : dx = (sum_n p[m, n] w[n, k]) p_scale[m], p and p_scale the rows of
//                   dy[m, n] w_scale[n] in 8 bits
//
// The sums are whole numbers in 32 bits and exact for up to kQ8MaxDepth products (128 * 128 *
// kQ8MaxDepth < 2^31); one conversion to fp32, one product of the scales, one fused
// multiply-add with the bias, one rounding to the output's type.
#include "lmbp_device.hpp"
#include "lmbp_launch.hpp"

namespace lmbp {
namespace lq8 {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_at1 __attribute__((ext_vector_type(4), aligned(1)));

struct Args {
  const int8_t* a;        // [M x K], rows a_pitch bytes apart
  const int8_t* b;        // forward: [N x K]; backward (TR): [K x N]
  const float* a_scale;   // per row, or null where there is nothing to add up (K = 0)
  const float* b_scale;   // per column of the result, or null
  const void* bias;       // per column, of the result's type, or null
  void* y;                // [M x N]
  int64_t M, N, K, a_pitch;
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
        const float sc = a.b_scale != nullptr ? as * a.b_scale[n] : as;
        OUT::store1(a.y, m * a.N + n,
                    __builtin_fmaf(float(acc[j][e]), sc, a.bias != nullptr ? OUT::load1(a.bias, n) : 0.0f));
      }
    }
}

template <class OUT, bool TR>
hipError_t launch(const Args& a, hipStream_t s) {
  const int64_t blocks = ((a.M + 63) / 64) * ((a.N + 63) / 64);
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((product_any<OUT, TR>), dim3(unsigned(blocks)), dim3(256), 0, s, a);
  return hipGetLastError();
}

int64_t pitch_of(int64_t n) { return (n + 127) / 128 * 128; }

}  // namespace lq8

hipError_t launch_linear_q8_fwd(bool bf16, int64_t M, int64_t N, int64_t K, const int8_t* q, const float* scale,
                                const int8_t* w, const float* w_scale, const void* bias, void* y, hipStream_t s) {
  const lq8::Args a{q, w, scale, w_scale, bias, y, M, N, K, K};
  return bf16 ? lq8::launch<BF16, false>(a, s) : lq8::launch<F32, false>(a, s);
}

size_t linear_q8_bwd_workspace(int64_t M, int64_t N) {
  return size_t(M) * size_t(lq8::pitch_of(N)) + size_t(M) * 4;
}

hipError_t launch_linear_q8_bwd(bool bf16, int64_t M, int64_t N, int64_t K, const void* dy, const int8_t* w,
                                const float* w_scale, void* dx, void* workspace, hipStream_t s) {
  const int64_t pitch = lq8::pitch_of(N);
  int8_t* const p = static_cast<int8_t*>(workspace);
  float* const p_scale = reinterpret_cast<float*>(p + M * pitch);
  if (N > 0) {
    const hipError_t e = launch_q8_rows(bf16, M, N, pitch, dy, w_scale, p, p_scale, s);
    if (e != hipSuccess) return e;
  }
  const lq8::Args a{p, w, N > 0 ? p_scale : nullptr, nullptr, nullptr, dx, M, K, N, pitch};
  return bf16 ? lq8::launch<BF16, true>(a, s) : lq8::launch<F32, true>(a, s);
}

}  // namespace lmbp
