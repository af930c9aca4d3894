// Gradient of a linear layer's bias, db[n] = sum_m dy[m, n], for gfx950.
//
// What bounds it: memory, dy once. A block takes up to 64 pieces of columns (4 elements to a lane, one
// where n or the address does not allow that) and a group of rows, 256 / pieces of them at a time;
// its sums meet in LDS. With several groups their sums (fp32) are added up by a second launch of the
// same kernel. All orders are fixed by the size, the address of dy and the number of CUs: a column's chain is
// its rows of a thread, then the threads, then the groups. bf16, us: 8192 x 11008 36 (5.0 TB/s), 8192 x 4096 18 (3.7), 12608 x 768 12.7, 1576 x 768 6.8 (two
// launches), 16 x 4096 3.0, 8192 x 11009 (one element to a lane) 68; torch's sum over the same rows 58, 33, 23,
// 12, 3.8 and 135.
#include "lmbp_launch.hpp"

#include "lmbp_device.hpp"

#include <algorithm>

namespace lmbp {
namespace bias {

typedef uint32_t u32x2_v __attribute__((ext_vector_type(2)));

// P (4 or 1) elements from element i on; 4 are aligned to their size.
template <class IO, int P>
__device__ inline void load(const void* p, int64_t i, float (&f)[P]) {
  if constexpr (P == 1) {
    f[0] = IO::load1(p, i);
  } else if constexpr (IO::kBytes == 4) {
    F32::unpack(*reinterpret_cast<const u32x4*>(static_cast<const float*>(p) + i), f);
  } else {
    const u32x2_v v = *reinterpret_cast<const u32x2_v*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      f[2 * k] = __uint_as_float(v[k] << 16);
      f[2 * k + 1] = __uint_as_float(v[k] & 0xffff0000u);
    }
  }
}

// pieces: threads across columns (a power of two up to 64); a group of `share` rows per blockIdx.y,
// its sums to row blockIdx.y of out. first_block: blocks across columns of the launches before.
template <class IO, class OUT, int P>
__global__ __launch_bounds__(256) void column_sums(const void* dy, int64_t m, int64_t n, int pieces, int64_t share, void* out,
                                                   int64_t first_block) {
  __shared__ float lds[256 * P];
  const int tx = threadIdx.x & (pieces - 1), ty = threadIdx.x / pieces, rows = 256 / pieces;
  const int64_t col = ((first_block + blockIdx.x) * pieces + tx) * P;
  const int64_t first = int64_t(blockIdx.y) * share, end = m - first < share ? m : first + share;
  float sum[P];
#pragma unroll
  for (int e = 0; e < P; ++e) sum[e] = 0.0f;
  if (col < n) {
#pragma unroll 4
    for (int64_t r = first + ty; r < end; r += rows) {
      float f[P];
      load<IO, P>(dy, r * n + col, f);
#pragma unroll
      for (int e = 0; e < P; ++e) sum[e] += f[e];
    }
  }
#pragma unroll
  for (int e = 0; e < P; ++e) lds[threadIdx.x * P + e] = sum[e];
  __syncthreads();
  if (ty != 0 || col >= n) return;
  for (int y = 1; y < rows; ++y)
#pragma unroll
    for (int e = 0; e < P; ++e) sum[e] += lds[(y * pieces + tx) * P + e];
#pragma unroll
  for (int e = 0; e < P; ++e) OUT::store1(out, int64_t(blockIdx.y) * n + col + e, sum[e]);
}

struct Plan {
  int p, pieces;
  int64_t blocks, groups, share;
};
// Groups until the card has four blocks to a CU, of 16 rows to a thread at least.
Plan make_plan(int64_t m, int64_t n, bool wide, int cus) {
  Plan a;
  a.p = wide ? 4 : 1;
  const int64_t all = (n + a.p - 1) / a.p;
  a.pieces = 1;
  while (a.pieces < 64 && a.pieces < all) a.pieces *= 2;
  a.blocks = (all + a.pieces - 1) / a.pieces;
  const int64_t per = int64_t(256 / a.pieces) * 16;
  a.groups = std::max<int64_t>(1, std::min((m + per - 1) / per, 4 * int64_t(cus) / a.blocks));
  a.share = std::max<int64_t>(1, (m + a.groups - 1) / a.groups);
  a.groups = std::max<int64_t>(1, (m + a.share - 1) / a.share);
  return a;
}

template <class IO, class OUT>
hipError_t launch(const Plan& a, int64_t m, int64_t n, const void* dy, void* out, hipStream_t s) {
  const auto kernel = a.p == 4 ? column_sums<IO, OUT, 4> : column_sums<IO, OUT, 1>;
  return in_parts(a.blocks, most_blocks(256), [&](int64_t first, int64_t count) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(count), unsigned(a.groups)), dim3(256), 0, s, dy, m, n, a.pieces, a.share, out, first);
  });
}
template <class OUT>
hipError_t launch_from(bool bf16, const Plan& a, int64_t m, int64_t n, const void* dy, void* out, hipStream_t s) {
  return bf16 ? launch<BF16, OUT>(a, m, n, dy, out, s) : launch<F32, OUT>(a, m, n, dy, out, s);
}

}  // namespace bias

// Room for the most groups that any address of dy takes.
size_t linear_bias_grad_workspace(int64_t m, int64_t n) {
  int dev = 0, cus = 256;
  if (current_device(dev, cus) != hipSuccess) cus = 256;   // no device here
  int64_t groups = bias::make_plan(m, n, false, cus).groups;
  if (n % 4 == 0) groups = std::max(groups, bias::make_plan(m, n, true, cus).groups);
  return groups > 1 ? size_t(groups) * size_t(n) * 4 : 0;
}

hipError_t launch_linear_bias_grad(bool bf16, bool db_bf16, int64_t m, int64_t n, const void* dy, void* db, void* workspace,
                                   hipStream_t s) {
  int dev = 0, cus = 0;
  const hipError_t e = current_device(dev, cus);
  if (e != hipSuccess) return e;
  const bool wide = n % 4 == 0 && reinterpret_cast<uintptr_t>(dy) % (bf16 ? 8 : 16) == 0;
  const bias::Plan a = bias::make_plan(m, n, wide, cus);
  if (a.groups == 1)
    return db_bf16 ? bias::launch_from<BF16>(bf16, a, m, n, dy, db, s) : bias::launch_from<F32>(bf16, a, m, n, dy, db, s);
  const hipError_t e1 = bias::launch_from<F32>(bf16, a, m, n, dy, workspace, s);
  if (e1 != hipSuccess) return e1;
  bias::Plan b = bias::make_plan(a.groups, n, n % 4 == 0, cus);
  b.share = a.groups;   // one group
  b.groups = 1;
  return db_bf16 ? bias::launch_from<BF16>(false, b, a.groups, n, workspace, db, s)
                 : bias::launch_from<F32>(false, b, a.groups, n, workspace, db, s);
}

}  // namespace lmbp
