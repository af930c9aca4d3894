// Rows in 8 bits with one scale each, for gfx950: of a tensor as it is (q8_rows), of the
// output of MS-RMSNorm with the residual's addition in front (msrms_q8_fwd), and of a
// gradient times a factor per column (the first half of linear_q8_bwd); the values that such
// rows stand for (q8_values); and MS-RMSNorm's backward from its output in 8 bits
// (msrms_q8_bwd). q8_device.hpp states how a row is brought to 8 bits.
//
// msrms_q8_fwd, per row: s = x + res rounded to the storage type, rstd = 1 / sqrt(p^-1 |s|^2
// + eps), z = s rstd. z is a multiple of s, so q comes from s itself and rstd only enters
// the scale: scale = a rstd / 127 with a the largest |s|.
// msrms_q8_bwd: with z = q scale, dx = rstd (dz - z p^-1 z^T dz) + ds.
#include "lmbp_launch.hpp"
#include "q8_device.hpp"

namespace lmbp {
namespace q8 {

enum { kRows = 0, kColumns = 1, kNorm = 2, kNormRes = 3 };   // what is brought to 8 bits

struct FwdArgs {
  const void* x;
  const void* res;        // kNormRes
  const float* columns;   // kColumns: a factor per column
  void* s;                // kNormRes: x + res
  int8_t* q;
  float* scale;
  float* rstd;            // kNorm, kNormRes
  int64_t rows, cols, pitch;   // pitch: bytes from one row of q to the next, zeros behind the row
  float eps;
};

// Maximum of v and sum of t over the block's 4 waves.
__device__ inline void block_max_sum(uint32_t& v, float& t, uint32_t* most, float* sum) {
  v = wave_umax(v);
  t = wave_sum(t);
  if ((threadIdx.x & (kWave - 1)) == 0) {
    most[threadIdx.x / kWave] = v;
    sum[threadIdx.x / kWave] = t;
  }
  __syncthreads();
  v = umax(umax(most[0], most[1]), umax(most[2], most[3]));
  t = (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// Block per row, any width and alignment; the row is read once per pass.
template <class IO, int MODE>
__global__ __launch_bounds__(256) void fwd_any(FwdArgs a) {
  __shared__ uint32_t most_lds[4];
  __shared__ float sum_lds[4];
  const int64_t row = blockIdx.x, base = row * a.cols;
  const int tid = threadIdx.x;
  uint32_t most = 0;
  float sum = 0.0f;
  for (int64_t k = tid; k < a.cols; k += 256) {
    float f = IO::load1(a.x, base + k);
    if constexpr (MODE == kNormRes) {
      IO::store1(a.s, base + k, f + IO::load1(a.res, base + k));
      f = IO::load1(a.s, base + k);
    }
    if constexpr (MODE == kColumns) f *= a.columns[k];
    most = umax(most, magnitude(f));
    sum = __builtin_fmaf(f, f, sum);
  }
  block_max_sum(most, sum, most_lds, sum_lds);
  const Q8Row w = q8_row(most);
  for (int64_t k = tid; k < a.pitch; k += 256) {
    uint32_t v = 0;
    if (k < a.cols) {
      float f = IO::load1(MODE == kNormRes ? a.s : a.x, base + k);
      if constexpr (MODE == kColumns) f *= a.columns[k];
      v = w.finite ? to_q8(f, w.r) : 0u;
    }
    a.q[row * a.pitch + k] = int8_t(v);
  }
  if (tid == 0) {
    if constexpr (MODE == kNorm || MODE == kNormRes) {
      const float rs = rsqrtf(sum / float(a.cols) + a.eps);
      a.rstd[row] = rs;
      a.scale[row] = w.a * rs / 127.0f;
    } else {
      a.scale[row] = w.a / 127.0f;
    }
  }
}

template <class IO>
__global__ __launch_bounds__(256) void values_any(const int8_t* q, const float* __restrict__ scale, void* v, int64_t cols) {
  const int64_t row = blockIdx.x, base = row * cols;
  const float sc = scale[row];
  for (int64_t k = threadIdx.x; k < cols; k += 256) IO::store1(v, base + k, float(q[base + k]) * sc);
}

template <class IO>
__global__ __launch_bounds__(256) void norm_bwd_any(const void* dz, const int8_t* q, const float* __restrict__ scale,
                                                    const float* __restrict__ rstd, const void* ds, void* dx,
                                                    int64_t cols) {
  __shared__ float red[256 / kWave];
  const int64_t row = blockIdx.x, base = row * cols;
  float s = 0.0f;
  for (int64_t k = threadIdx.x; k < cols; k += 256) s = __builtin_fmaf(float(q[base + k]), IO::load1(dz, base + k), s);
  const float sc = scale[row], rs = rstd[row];
  const float b = sc * (sc * (block_sum(s, red) / float(cols)));
  for (int64_t k = threadIdx.x; k < cols; k += 256) {
    const float g = __builtin_fmaf(-float(q[base + k]), b, IO::load1(dz, base + k));
    IO::store1(dx, base + k, ds != nullptr ? __builtin_fmaf(rs, g, IO::load1(ds, base + k)) : rs * g);
  }
}

template <class IO, int MODE>
hipError_t launch_fwd(const FwdArgs& a, hipStream_t s) {
  if (a.rows > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((fwd_any<IO, MODE>), dim3(unsigned(a.rows)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <class IO>
hipError_t launch_values(int64_t rows, int64_t cols, const int8_t* q, const float* scale, void* v, hipStream_t s) {
  if (rows > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((values_any<IO>), dim3(unsigned(rows)), dim3(256), 0, s, q, scale, v, cols);
  return hipGetLastError();
}

template <class IO>
hipError_t launch_norm_bwd(int64_t rows, int64_t cols, const void* dz, const int8_t* q, const float* scale,
                           const float* rstd, const void* ds, void* dx, hipStream_t s) {
  if (rows > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((norm_bwd_any<IO>), dim3(unsigned(rows)), dim3(256), 0, s, dz, q, scale, rstd, ds, dx, cols);
  return hipGetLastError();
}

}  // namespace q8

hipError_t launch_q8_rows(bool bf16, int64_t rows, int64_t cols, int64_t pitch, const void* x, const float* columns,
                          int8_t* q, float* scale, hipStream_t s) {
  const q8::FwdArgs a{x, nullptr, columns, nullptr, q, scale, nullptr, rows, cols, pitch, 0.0f};
  if (columns != nullptr)
    return bf16 ? q8::launch_fwd<BF16, q8::kColumns>(a, s) : q8::launch_fwd<F32, q8::kColumns>(a, s);
  return bf16 ? q8::launch_fwd<BF16, q8::kRows>(a, s) : q8::launch_fwd<F32, q8::kRows>(a, s);
}

hipError_t launch_q8_values(bool bf16, int64_t rows, int64_t cols, const int8_t* q, const float* scale, void* v,
                            hipStream_t s) {
  return bf16 ? q8::launch_values<BF16>(rows, cols, q, scale, v, s) : q8::launch_values<F32>(rows, cols, q, scale, v, s);
}

hipError_t launch_msrms_q8_fwd(bool bf16, int64_t rows, int64_t cols, float eps, const void* x, const void* res,
                               void* sum, int8_t* q, float* scale, float* rstd, hipStream_t s) {
  const q8::FwdArgs a{x, res, nullptr, sum, q, scale, rstd, rows, cols, cols, eps};
  if (res != nullptr)
    return bf16 ? q8::launch_fwd<BF16, q8::kNormRes>(a, s) : q8::launch_fwd<F32, q8::kNormRes>(a, s);
  return bf16 ? q8::launch_fwd<BF16, q8::kNorm>(a, s) : q8::launch_fwd<F32, q8::kNorm>(a, s);
}

hipError_t launch_msrms_q8_bwd(bool bf16, int64_t rows, int64_t cols, const void* dz, const int8_t* q,
                               const float* scale, const float* rstd, const void* ds, void* dx, hipStream_t s) {
  return bf16 ? q8::launch_norm_bwd<BF16>(rows, cols, dz, q, scale, rstd, ds, dx, s)
              : q8::launch_norm_bwd<F32>(rows, cols, dz, q, scale, rstd, ds, dx, s);
}

}  // namespace lmbp
