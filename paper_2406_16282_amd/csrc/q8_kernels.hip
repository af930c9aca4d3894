// Rows in 8 bits with one scale each, for gfx950: of a tensor as it is (q8_rows), of the
// output of MS-RMSNorm with the residual's addition in front (msrms_q8_fwd), and of a
// gradient times a factor per column (the first half of linear_q8_bwd); the values that such
// rows stand for (q8_values); and MS-RMSNorm's backward from its output in 8 bits
// (msrms_q8_bwd). q8_device.hpp states how a row is brought to 8 bits.
//
// What bounds them: memory. A row is read once and held in registers while its largest value (and
// sum of squares) is found. On [8192 x 4096] bf16: q8_rows 18 us (5.6 TB/s), q8_values 16 (6.35),
// msrms_q8_fwd 18 and with the residual 38 to 40 (5.9 to 6.2), msrms_q8_bwd 27 (6.2) and with ds 35 (6.7); on
// [8192 x 13824] 53 us (6.4), 50 to 58, 54, 128 (6.2), 83 to 91 and 113 to 124; a copy of 1 GiB runs at 6.6 to
// 6.8 TB/s. On [2439 x 1025] fp32, rows at any address: 4.6, 4.5, 5.1, 8.7, 6.8 and 8.2 us. q is stored past the
// caches (about 8% on q8_rows of the first). Pieces of 16 elements instead of 8 were slower; blocks
// that walk the rows no faster than a block for each group of them, but for factors per column: there
// the factors stay in registers over a block's rows ([8192 x 11008] 44 us; read again for every row 161).
//
// msrms_q8_fwd, per row: s = x + res rounded to the storage type, rstd = 1 / sqrt(p^-1 |s|^2
// + eps), z = s rstd. z is a multiple of s, so q comes from s itself and rstd only enters
// the scale: scale = a rstd / 127 with a the largest |s|. Squares that add up to 2^128 or more (a
// value above 2^64, or many near it) are added up again as (s 2^-96)^2, which no row overflows; what
// falls below the smallest number there is less than 2^-60 of the sum. One wave does so for its row,
// from memory and behind everything else: of the pieces in registers it cost every call 10 to 20 registers.
// So do squares whose mean, eps included, is below 2^-90 (no eps in use is that small), as (s 2^60)^2.
// The backward's sum of q dz is formed again of dz 2^-56 in the same case, by each wave for its pieces.
// msrms_q8_bwd: with z = q scale, dx = rstd (dz - z p^-1 z^T dz) + ds.
#include "lmbp_launch.hpp"
#include "q8_device.hpp"

#include <algorithm>
#include <type_traits>

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

// Infinite or NaN, of a sum that is the same in all lanes: a scalar condition, so that the other side of the
// branch costs no registers.
__device__ inline bool overflowed(float sum) {
  return (uint32_t(__builtin_amdgcn_readfirstlane(__float_as_int(sum))) & 0x7f800000u) == 0x7f800000u;
}

// The factor in front of the squares of a row of that mean: 1, or one that keeps them in fp32's range.
__device__ inline float unit_of(float mean) { return overflowed(mean) ? 0x1p-96f : mean < 0x1p-90f ? 0x1p60f : 1.0f; }
__device__ inline float add_square(float v, float unit, float sum) { return __builtin_fmaf(v * unit, v * unit, sum); }
// rstd of a row, and the scale of one whose largest magnitude is a, of its mean square + eps times unit^2.
__device__ inline void store_stats(const FwdArgs& f, int64_t row, float mean, float unit, float a) {
  const float rs = rsqrtf(mean);
  f.rstd[row] = rs * unit;
  f.scale[row] = a * unit * rs / 127.0f;
}

// Threads per block of the register kernels: 256, or one row of WPR waves where that is wider.
template <int WPR>
constexpr int block_of() { return WPR * kWave > 256 ? WPR * kWave : 256; }

// P consecutive elements of a row in storage form; RAGGED: at any element's address.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
template <class IO, int P, bool RAGGED>
struct Piece {
  static constexpr int kVecs = P * IO::kBytes / 16, E = IO::kPerVec;
  u32x4 v[kVecs];
  __device__ inline void clear() {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) v[k] = u32x4{0u, 0u, 0u, 0u};
  }
  __device__ inline void load(const void* base, int64_t elem) {
    const char* p = static_cast<const char*>(base) + elem * IO::kBytes;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      if constexpr (RAGGED) v[k] = reinterpret_cast<const u32x4_any*>(p)[k];
      else v[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p) + k);
    }
  }
  __device__ inline void store(void* base, int64_t elem) const {
    char* p = static_cast<char*>(base) + elem * IO::kBytes;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      if constexpr (RAGGED) reinterpret_cast<u32x4_any*>(p)[k] = v[k];
      else __builtin_nontemporal_store(v[k], reinterpret_cast<u32x4*>(p) + k);
    }
  }
  __device__ inline void get(float (&f)[P]) const {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      float e[E];
      IO::unpack(v[k], e);
#pragma unroll
      for (int i = 0; i < E; ++i) f[k * E + i] = e[i];
    }
  }
  __device__ inline void set(const float (&f)[P]) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      float e[E];
#pragma unroll
      for (int i = 0; i < E; ++i) e[i] = f[k * E + i];
      v[k] = IO::pack(e);
    }
  }
};

// P bytes of q (4 or 8).
template <int P, bool RAGGED>
struct Bytes {
  typedef uint32_t any __attribute__((ext_vector_type(P / 4), aligned(RAGGED ? 1 : P)));
  uint32_t v[P / 4];
  __device__ inline void load(const int8_t* p) {
    const any b = *reinterpret_cast<const any*>(p);
#pragma unroll
    for (int k = 0; k < P / 4; ++k) v[k] = b[k];
  }
  __device__ inline void store(int8_t* p) const {
    any b;
#pragma unroll
    for (int k = 0; k < P / 4; ++k) b[k] = v[k];
    if constexpr (!RAGGED) __builtin_nontemporal_store(b, reinterpret_cast<any*>(p));
    else *reinterpret_cast<any*>(p) = b;
  }
  __device__ inline void get(float (&f)[P]) const {
#pragma unroll
    for (int k = 0; k < P; ++k) f[k] = float(int8_t(v[k / 4] >> (8 * (k % 4))));
  }
  __device__ inline void set(const float (&t)[P], float r) {   // q8_device.hpp
#pragma unroll
    for (int k = 0; k < P / 4; ++k) {
      const uint32_t lo = __builtin_amdgcn_perm(to_q8(t[4 * k + 1], r), to_q8(t[4 * k], r), 0x0c0c0400u);
      const uint32_t hi = __builtin_amdgcn_perm(to_q8(t[4 * k + 3], r), to_q8(t[4 * k + 2], r), 0x04000c0cu);
      v[k] = lo | hi;
    }
  }
};

// Rows in registers: WPR waves to a row, thread t of the row holding pieces t, t + 64 WPR, ...
// (VPL of them); RAGGED rows have fewer than a piece's elements left, one to a thread. With a
// factor per column the blocks walk the rows, each with its columns' factors in registers.
template <class IO, int MODE, int VPL, int WPR, bool RAGGED>
__global__ __launch_bounds__(block_of<WPR>()) void fwd_rows(FwdArgs a) {
  constexpr int P = IO::kPerVec, TPR = kWave * WPR, RPB = block_of<WPR>() / TPR;
  constexpr bool kIsNorm = MODE == kNorm || MODE == kNormRes;
  // Rows of 8 waves and more with many pieces: the waves' sums are read behind the pieces' use, not held in
  // 8 or 16 registers meanwhile ([4096 x 20000] fp32 66.7 us, else 76.9; elsewhere that only ends the block
  // later, [8192 x 4096] fp32 30.1 us against 28.8).
  constexpr bool kSumLate = WPR == 16 || (WPR == 8 && VPL == 4);
  __shared__ uint32_t most_lds[2][block_of<WPR>() / kWave];
  __shared__ float sum_lds[block_of<WPR>() / kWave];
  const int t = threadIdx.x % TPR;
  const int cols = int(a.cols), pieces = cols / P;
  float c[MODE == kColumns ? VPL : 1][P], c_last = 1.0f;
  if constexpr (MODE == kColumns) {
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      Piece<F32, P, true> f;
      f.clear();
      if (j * TPR + t < pieces) f.load(a.columns, (j * TPR + t) * P);
      f.get(c[j]);
    }
    if (RAGGED && pieces * P + t < cols) c_last = a.columns[pieces * P + t];
  }
  const int64_t groups = (a.rows + RPB - 1) / RPB;
  int turn = 0;   // LDS place: a wave can be at most one barrier ahead of another
  for (int64_t group = blockIdx.x; group < groups; group += gridDim.x, turn ^= 1) {
    const int64_t row = group * RPB + wave_in_block() / WPR;
    const bool active = row < a.rows;
    const int64_t base = row * a.cols;
    Piece<IO, P, RAGGED> x[VPL], y[MODE == kNormRes ? VPL : 1];
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      const int idx = j * TPR + t;
      x[j].clear();
      if constexpr (MODE == kNormRes) y[j].clear();
      if (active && idx < pieces) {
        x[j].load(a.x, base + idx * P);
        if constexpr (MODE == kNormRes) y[j].load(a.res, base + idx * P);
      }
    }
    const bool rest = RAGGED && active && pieces * P + t < cols;
    float last = 0.0f;
    if (rest) {
      const int64_t at = base + pieces * P + t;
      last = IO::load1(a.x, at);
      if constexpr (MODE == kNormRes) {
        IO::store1(a.s, at, last + IO::load1(a.res, at));
        last = IO::load1(a.s, at);
      }
      if constexpr (MODE == kColumns) last *= c_last;
    }
    uint32_t most = magnitude(last);
    float sum = last * last;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      float f[P];
      x[j].get(f);
      if constexpr (MODE == kNormRes) {
        float g[P];
        y[j].get(g);
#pragma unroll
        for (int e = 0; e < P; ++e) f[e] += g[e];
        x[j].set(f);
        const int idx = j * TPR + t;
        if (active && idx < pieces) x[j].store(a.s, base + idx * P);
        x[j].get(f);   // as stored
      }
#pragma unroll
      for (int e = 0; e < P; ++e) {
        if constexpr (MODE == kColumns) f[e] *= c[j][e];
        most = umax(most, magnitude(f[e]));
        if constexpr (kIsNorm) sum = __builtin_fmaf(f[e], f[e], sum);
      }
    }
    most = wave_umax(most);
    if constexpr (kIsNorm) sum = wave_sum(sum);
    if constexpr (WPR > 1) {
      const int wave = threadIdx.x / kWave, first = wave / WPR * WPR;
      if ((threadIdx.x & (kWave - 1)) == 0) {
        most_lds[turn][wave] = most;
        if constexpr (kIsNorm) sum_lds[wave] = sum;
      }
      __syncthreads();
      most = 0;
      sum = 0.0f;
#pragma unroll
      for (int k = 0; k < WPR; ++k) {
        most = umax(most, most_lds[turn][first + k]);
        if constexpr (kIsNorm && !kSumLate) sum += sum_lds[first + k];
      }
    }
    if (!active) continue;   // the last group: no barrier follows
    const Q8Row w = q8_row(most);
    int8_t* const q = a.q + row * a.pitch;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      const int idx = j * TPR + t;
      if (idx < pieces) {
        float f[P];
        x[j].get(f);
        if constexpr (MODE == kColumns) {
#pragma unroll
          for (int e = 0; e < P; ++e) f[e] *= c[j][e];
        }
        Bytes<P, RAGGED> b;
        b.set(f, w.r);
#pragma unroll
        for (int k = 0; k < P / 4; ++k) b.v[k] = w.finite ? b.v[k] : 0u;
        b.store(q + idx * P);
      }
    }
    if (rest) q[pieces * P + t] = int8_t(w.finite ? to_q8(last, w.r) : 0u);
    if constexpr (MODE == kColumns) {
      for (int k = cols + t; k < a.pitch; k += TPR) q[k] = 0;
    }
    if constexpr (kIsNorm) {
      if (t < kWave) {   // the row's first wave
        if constexpr (kSumLate) {
          const int first = threadIdx.x / kWave;
#pragma unroll
          for (int k = 0; k < WPR; ++k) sum += sum_lds[first + k];
        }
        float mean = sum / float(cols) + a.eps;
        const float unit = unit_of(mean);
        if (w.finite && unit != 1.0f) {
          __threadfence_block();   // s is read as other lanes and waves stored it
          float again = 0.0f;
#pragma unroll 1
          for (int k = t; k < cols; k += kWave) again = add_square(IO::load1(MODE == kNormRes ? a.s : a.x, base + k), unit, again);
          mean = wave_sum(again) / float(cols) + a.eps * unit * unit;
        }
        if (t == 0) store_stats(a, row, mean, unit, w.a);
      }
    } else if (t == 0) {
      a.scale[row] = w.a / 127.0f;
    }
    if constexpr (MODE != kColumns) return;   // a block for every group
  }
}

template <class IO, int VPL, int WPR, bool RAGGED>
__global__ __launch_bounds__(block_of<WPR>()) void values_rows(const int8_t* q, const float* __restrict__ scale, void* v,
                                                               int64_t rows, int cols) {
  constexpr int P = IO::kPerVec, TPR = kWave * WPR, RPB = block_of<WPR>() / TPR;
  const int t = threadIdx.x % TPR;
  const int64_t row = int64_t(blockIdx.x) * RPB + wave_in_block() / WPR;
  if (row >= rows) return;
  const int pieces = cols / P;
  const int64_t base = row * cols;
  const float sc = scale[row];
  Bytes<P, RAGGED> b[VPL];
#pragma unroll
  for (int j = 0; j < VPL; ++j)
    if (j * TPR + t < pieces) b[j].load(q + base + (j * TPR + t) * P);
#pragma unroll
  for (int j = 0; j < VPL; ++j) {
    const int idx = j * TPR + t;
    if (idx < pieces) {
      float f[P];
      b[j].get(f);
#pragma unroll
      for (int e = 0; e < P; ++e) f[e] *= sc;
      Piece<IO, P, RAGGED> o;
      o.set(f);
      o.store(v, base + idx * P);
    }
  }
  const int at = pieces * P + t;
  if (RAGGED && at < cols) IO::store1(v, base + at, float(q[base + at]) * sc);
}

// b = sc^2 p^-1 sum, the factor of q in z mean(z dz); down: the sum of q (dz kDownDz), for a sum that
// has overflowed.
constexpr float kDownDz = 0x1p-56f;
__device__ inline float along(float sum, float down, int64_t cols, float sc) {
  // A branch: a choice of values takes 7 registers more ([8192 x 11008] bf16 72.5 us against 65.6).
  if (overflowed(sum)) return sc * (sc * (down / float(cols))) / kDownDz;
  return sc * (sc * (sum / float(cols)));
}

struct BwdArgs {
  const void* dz;
  const int8_t* q;
  const float* scale;
  const float* rstd;
  const void* ds;
  void* dx;
  int64_t rows, cols;
};

template <class DZ, class IO, int VPL, int WPR, bool RAGGED>
__global__ __launch_bounds__(block_of<WPR>()) void norm_bwd_rows(BwdArgs a) {
  constexpr int P = IO::kPerVec, TPR = kWave * WPR, RPB = block_of<WPR>() / TPR;
  __shared__ float sum_lds[2][block_of<WPR>() / kWave];
  const int t = threadIdx.x % TPR;
  const int64_t row = int64_t(blockIdx.x) * RPB + wave_in_block() / WPR;
  const bool active = row < a.rows;
  if constexpr (WPR == 1) {
    if (!active) return;
  }
  const int cols = int(a.cols), pieces = cols / P;
  const int64_t base = row * a.cols;
  Piece<DZ, P, RAGGED> dz[VPL];
  Piece<IO, P, RAGGED> ds[VPL];
  Bytes<P, RAGGED> q[VPL];
#pragma unroll
  for (int j = 0; j < VPL; ++j) {
    const int idx = j * TPR + t;
    dz[j].clear();
    ds[j].clear();
#pragma unroll
    for (int k = 0; k < P / 4; ++k) q[j].v[k] = 0u;
    if (active && idx < pieces) {
      dz[j].load(a.dz, base + idx * P);
      q[j].load(a.q + base + idx * P);
      if (a.ds != nullptr) ds[j].load(a.ds, base + idx * P);
    }
  }
  const int at = pieces * P + t;
  const bool rest = RAGGED && active && at < cols;
  const float last_dz = rest ? DZ::load1(a.dz, base + at) : 0.0f, last_q = rest ? float(a.q[base + at]) : 0.0f;
  const float last_ds = rest && a.ds != nullptr ? IO::load1(a.ds, base + at) : 0.0f;
  const float sc = active ? a.scale[row] : 0.0f, rs = active ? a.rstd[row] : 0.0f;
  float sum = last_dz * last_q;
#pragma unroll
  for (int j = 0; j < VPL; ++j) {
    float g[P], z[P];
    dz[j].get(g);
    q[j].get(z);
#pragma unroll
    for (int e = 0; e < P; ++e) sum = __builtin_fmaf(z[e], g[e], sum);
  }
  sum = wave_sum(sum);
  float down = sum * kDownDz;
  if (overflowed(sum)) {
    down = last_dz * kDownDz * last_q;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      float g[P], z[P];
      dz[j].get(g);
      q[j].get(z);
#pragma unroll
      for (int e = 0; e < P; ++e) down = __builtin_fmaf(z[e], g[e] * kDownDz, down);
    }
    down = wave_sum(down);
  }
  if constexpr (WPR > 1) {
    const int wave = threadIdx.x / kWave, first = wave / WPR * WPR;
    if ((threadIdx.x & (kWave - 1)) == 0) {
      sum_lds[0][wave] = sum;
      sum_lds[1][wave] = down;
    }
    __syncthreads();
    sum = 0.0f;
    down = 0.0f;
#pragma unroll
    for (int k = 0; k < WPR; ++k) {
      sum += sum_lds[0][first + k];
      down += sum_lds[1][first + k];
    }
    if (!active) return;
  }
  const float b = along(sum, down, cols, sc);
#pragma unroll
  for (int j = 0; j < VPL; ++j) {
    const int idx = j * TPR + t;
    if (idx < pieces) {
      float g[P], z[P], d[P];
      dz[j].get(g);
      q[j].get(z);
      ds[j].get(d);
#pragma unroll
      for (int e = 0; e < P; ++e) g[e] = __builtin_fmaf(rs, __builtin_fmaf(-z[e], b, g[e]), d[e]);
      Piece<IO, P, RAGGED> o;
      o.set(g);
      o.store(a.dx, base + idx * P);
    }
  }
  if (rest) IO::store1(a.dx, base + at, __builtin_fmaf(rs, __builtin_fmaf(-last_q, b, last_dz), last_ds));
}

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
  float mean = sum / float(a.cols) + a.eps;
  const float unit = unit_of(mean);
  if constexpr (MODE == kNorm || MODE == kNormRes) {
    if (w.finite && unit != 1.0f) {   // for all threads or none
      float again = 0.0f;
      for (int64_t k = tid; k < a.cols; k += 256)
        again = add_square(IO::load1(MODE == kNormRes ? a.s : a.x, base + k), unit, again);
      __syncthreads();   // the sums of before have been read
      block_max_sum(most, again, most_lds, sum_lds);
      mean = again / float(a.cols) + a.eps * unit * unit;
    }
  }
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
    if constexpr (MODE == kNorm || MODE == kNormRes) store_stats(a, row, mean, unit, w.a);
    else a.scale[row] = w.a / 127.0f;
  }
}

template <class IO>
__global__ __launch_bounds__(256) void values_any(const int8_t* q, const float* __restrict__ scale, void* v, int64_t cols) {
  const int64_t row = blockIdx.x, base = row * cols;
  const float sc = scale[row];
  for (int64_t k = threadIdx.x; k < cols; k += 256) IO::store1(v, base + k, float(q[base + k]) * sc);
}

template <class DZ, class IO>
__global__ __launch_bounds__(256) void norm_bwd_any(const void* dz, const int8_t* q, const float* __restrict__ scale,
                                                    const float* __restrict__ rstd, const void* ds, void* dx,
                                                    int64_t cols) {
  __shared__ float red[256 / kWave];
  const int64_t row = blockIdx.x, base = row * cols;
  float s = 0.0f;
  for (int64_t k = threadIdx.x; k < cols; k += 256) s = __builtin_fmaf(float(q[base + k]), DZ::load1(dz, base + k), s);
  const float sc = scale[row], rs = rstd[row];
  const float sum = block_sum(s, red);
  float down = 0.0f;
  if (overflowed(sum)) {   // for all threads or none
    for (int64_t k = threadIdx.x; k < cols; k += 256)
      down = __builtin_fmaf(float(q[base + k]), DZ::load1(dz, base + k) * kDownDz, down);
    down = block_sum(down, red);
  }
  const float b = along(sum, down, cols, sc);
  for (int64_t k = threadIdx.x; k < cols; k += 256) {
    const float g = __builtin_fmaf(-float(q[base + k]), b, DZ::load1(dz, base + k));
    IO::store1(dx, base + k, ds != nullptr ? __builtin_fmaf(rs, g, IO::load1(ds, base + k)) : rs * g);
  }
}

// Launch shapes of the register kernels, by the pieces that they hold: the fewest waves to a row
// that hold it in 3 pieces per thread (4 with 8 waves), or 16 waves with up to MOST (what a kernel
// has registers for). Measured in us as waves x pieces, bf16, 8192 rows, tensors of their own throughout: q8_rows,
// msrms_q8_fwd with a residual, msrms_q8_bwd with ds. 768 columns 1x2 5.4, 10.0, 10.2 and 2x1 7.1, 10.1, 10.1; 4096
// columns 4x2 17.7, 38.6, 35.7, 8x1 21.1, 39.0, 36.1 and 2x4 17.7, 39.8, 36.5; 11008 columns 8x3 43.1, 102.8, 91.3 and
// 16x2 52.2, 103.2, 93.2; 13824 columns 8x4 53.2, 128.5, 114.9, 16x2 60.1, 128.6, 115.6 and 16x3 59.7, 128.6, 148.6 (with
// factors per column 8x4 56.8, 16x2 70). In 32 bits 4096 columns 8x2 28.0, 69.6, 65.0 and 4x4 29.0, 68.3, 65.4; 8192
// columns 8x4 55.4, 137.5, 134.4 and 16x2 56.7, 139.4, 132.2 (with factors 58 and 66).
struct Shape {
  int wpr, vpl;
};
constexpr Shape kShapes[] = {{1, 1}, {1, 2}, {1, 3}, {2, 2},  {2, 3},  {4, 2}, {4, 3},
                             {8, 2}, {8, 3}, {8, 4}, {16, 3}, {16, 4}, {16, 6}, {16, 8}};
constexpr int kNumShapes = sizeof(kShapes) / sizeof(kShapes[0]);

// Calls f(VPL, WPR) for the shape that holds `pieces`; false if none does.
template <int MOST, int I = 0, class F>
bool with_shape(int64_t pieces, F f) {
  if constexpr (I < kNumShapes) {
    constexpr int wpr = kShapes[I].wpr, vpl = kShapes[I].vpl;
    if constexpr (vpl <= MOST) {
      if (pieces <= int64_t(kWave) * wpr * vpl) {
        f(std::integral_constant<int, vpl>{}, std::integral_constant<int, wpr>{});
        return true;
      }
    }
    return with_shape<MOST, I + 1>(pieces, f);
  } else {
    return false;
  }
}

// Blocks for `rows` of them at WPR waves each.
template <int WPR>
int64_t blocks_of(int64_t rows) {
  constexpr int rpb = block_of<WPR>() / (kWave * WPR);
  return (rows + rpb - 1) / rpb;
}
// Rows that one launch takes.
template <int WPR>
constexpr int64_t rows_at_once() { return most_blocks(block_of<WPR>()) * (block_of<WPR>() / (kWave * WPR)); }

bool at16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

template <class T>
T* moved(T* p, int64_t bytes) {   // null stays null
  return p == nullptr ? p : reinterpret_cast<T*>(reinterpret_cast<uintptr_t>(p) + bytes);
}

template <class IO, int MODE>
hipError_t launch_fwd(const FwdArgs& a, hipStream_t s) {
  const bool ragged = a.cols % IO::kPerVec != 0 || !at16(a.x) || (MODE == kNormRes && (!at16(a.res) || !at16(a.s))) ||
                      reinterpret_cast<uintptr_t>(a.q) % IO::kPerVec != 0;
  int dev = 0, cus = 0;
  hipError_t e = hipSuccess;
  if (MODE == kColumns) {
    e = current_device(dev, cus);
    if (e != hipSuccess) return e;
  }
  auto rows_of = [&](int64_t first, int64_t rows) {
    const int64_t at = first * a.cols * IO::kBytes;
    return FwdArgs{moved(a.x, at), moved(a.res, at), a.columns, moved(a.s, at), a.q + first * a.pitch, a.scale + first,
                   moved(a.rstd, first * 4), rows, a.cols, a.pitch, a.eps};
  };
  const bool held = a.cols < (1 << 24) && with_shape<MODE == kColumns && IO::kPerVec == 8 ? 4 : 8>(a.cols / IO::kPerVec, [&](auto vpl, auto wpr) {
    constexpr int V = decltype(vpl)::value, W = decltype(wpr)::value;
    const auto kernel = ragged ? fwd_rows<IO, MODE, V, W, true> : fwd_rows<IO, MODE, V, W, false>;
    // With a factor per column the blocks walk the rows: any number of rows in one launch.
    e = in_parts(a.rows, MODE == kColumns ? a.rows : rows_at_once<W>(), [&](int64_t first, int64_t rows) {
      int64_t blocks = blocks_of<W>(rows);
      if (MODE == kColumns) blocks = std::min<int64_t>(blocks, int64_t(cus) * (1024 / block_of<W>()));
      hipLaunchKernelGGL(kernel, dim3(unsigned(blocks)), dim3(block_of<W>()), 0, s, rows_of(first, rows));
    });
  });
  if (held) return e;
  return in_parts(a.rows, most_blocks(256), [&](int64_t first, int64_t rows) {
    hipLaunchKernelGGL((fwd_any<IO, MODE>), dim3(unsigned(rows)), dim3(256), 0, s, rows_of(first, rows));
  });
}

template <class IO>
hipError_t launch_values(int64_t rows, int64_t cols, const int8_t* q, const float* scale, void* v, hipStream_t s) {
  const bool ragged = cols % IO::kPerVec != 0 || !at16(v) || reinterpret_cast<uintptr_t>(q) % IO::kPerVec != 0;
  hipError_t e = hipSuccess;
  const bool held = cols < (1 << 24) && with_shape<8>(cols / IO::kPerVec, [&](auto vpl, auto wpr) {
    constexpr int V = decltype(vpl)::value, W = decltype(wpr)::value;
    const auto kernel = ragged ? values_rows<IO, V, W, true> : values_rows<IO, V, W, false>;
    e = in_parts(rows, rows_at_once<W>(), [&](int64_t first, int64_t count) {
      hipLaunchKernelGGL(kernel, dim3(unsigned(blocks_of<W>(count))), dim3(block_of<W>()), 0, s, q + first * cols, scale + first,
                         moved(v, first * cols * IO::kBytes), count, int(cols));
    });
  });
  if (held) return e;
  return in_parts(rows, most_blocks(256), [&](int64_t first, int64_t count) {
    hipLaunchKernelGGL((values_any<IO>), dim3(unsigned(count)), dim3(256), 0, s, q + first * cols, scale + first,
                       moved(v, first * cols * IO::kBytes), cols);
  });
}

template <class DZ, class IO>
hipError_t launch_norm_bwd(int64_t rows, int64_t cols, const void* dz, const int8_t* q, const float* scale,
                           const float* rstd, const void* ds, void* dx, hipStream_t s) {
  const bool ragged = cols % IO::kPerVec != 0 || !at16(dz) || !at16(ds) || !at16(dx) ||
                      reinterpret_cast<uintptr_t>(q) % IO::kPerVec != 0;
  hipError_t e = hipSuccess;
  auto rows_of = [&](int64_t first, int64_t count) {
    const int64_t at = first * cols;
    return BwdArgs{moved(dz, at * DZ::kBytes), q + at, scale + first, rstd + first, moved(ds, at * IO::kBytes),
                   moved(dx, at * IO::kBytes), count, cols};
  };
  const bool held = cols < (1 << 24) && with_shape<IO::kPerVec == 8 ? 4 : 8>(cols / IO::kPerVec, [&](auto vpl, auto wpr) {
    constexpr int V = decltype(vpl)::value, W = decltype(wpr)::value;
    const auto kernel = ragged ? norm_bwd_rows<DZ, IO, V, W, true> : norm_bwd_rows<DZ, IO, V, W, false>;
    e = in_parts(rows, rows_at_once<W>(), [&](int64_t first, int64_t count) {
      hipLaunchKernelGGL(kernel, dim3(unsigned(blocks_of<W>(count))), dim3(block_of<W>()), 0, s, rows_of(first, count));
    });
  });
  if (held) return e;
  return in_parts(rows, most_blocks(256), [&](int64_t first, int64_t count) {
    const BwdArgs a = rows_of(first, count);
    hipLaunchKernelGGL((norm_bwd_any<DZ, IO>), dim3(unsigned(count)), dim3(256), 0, s, a.dz, a.q, a.scale, a.rstd, a.ds, a.dx,
                       cols);
  });
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

hipError_t launch_msrms_q8_bwd(bool dz_bf16, bool bf16, int64_t rows, int64_t cols, const void* dz, const int8_t* q,
                               const float* scale, const float* rstd, const void* ds, void* dx, hipStream_t s) {
  if (!bf16) return q8::launch_norm_bwd<F32, F32>(rows, cols, dz, q, scale, rstd, ds, dx, s);
  return dz_bf16 ? q8::launch_norm_bwd<BF16, BF16>(rows, cols, dz, q, scale, rstd, ds, dx, s)
                 : q8::launch_norm_bwd<F32, BF16>(rows, cols, dz, q, scale, rstd, ds, dx, s);
}

}  // namespace lmbp
