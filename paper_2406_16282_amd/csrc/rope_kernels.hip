// Rotary positions of query and key heads, alone or behind MS-RMSNorm of each head, for gfx950.
//
// A head's columns are taken in pairs; pair p of token t turns by freqs[p] times the position of t on the pair's axis.
// The angle is formed in revolutions as a whole number of 2^-64: position times the frequency so held, modulo 2^64, which
// is exact for every position, near or far; a quarter turn is taken off it and sine and cosine come from their
// series on [-pi/4, pi/4] (to r^9 and r^10: within 2e-9 and 2e-10). There is no table, and no position can read out of one.
//
// Norm (per head, D columns): rstd = 1 / sqrt(D^-1 |x|^2 + eps), z = x rstd, y = turn(gain z). The turn keeps lengths and
// products, so without a gain the backward needs no z: with y as it was kept, dx = turn_back(rstd (dy - y D^-1 (y . dy))). With a
// gain g = turn_back(dy), dz = gain g, dx = rstd (dz - z D^-1 (z . dz)), dgain = sum of g z over the rows, from x.
#include "lmbp_device.hpp"
#include "lmbp_launch.hpp"

#include <algorithm>
#include <cmath>

namespace lmbp {
namespace rope {

enum { kTurn = 0, kNorm = 1, kNormBack = 2, kNormBackGain = 3 };

// Queries or keys: one tensor's heads.
struct Side {
  const void* x;      // read: x, or the gradient of y
  void* y;            // written
  const void* kept;   // backward: y without gain, x with
  float* rstd;        // [tokens][heads]; written by the forward
  const void* gain;   // [dim] or null
  int64_t x_row, x_head, y_row, y_head, kept_row, kept_head;
  int heads, shares;  // shares: waves that take a token's heads in turn
};

struct Args {
  Side side[2];
  const void* positions;
  int64_t axis_stride, tokens;
  float* part;        // kNormBackGain: [2][blocks][dim]
  int64_t first;      // token of this launch's first block
  int dim, pairs, lanes, rows;   // lanes to a head (a power of two), heads to a wave at a time
  float eps, sign;
  uint8_t wide, interleaved, gain_bf16;
  uint8_t axis[kRopePairs];
  uint64_t freq[kRopePairs];
};

// This lane's place in a head: E pairs, two pieces of E columns or 2 E single columns.
template <class IO, bool VEC>
struct Place {
  static constexpr int E = IO::kPerVec;
  int pair, a, b;   // first pair; VEC: where the pieces start
  int dim, half;
  bool inside, interleaved;
  __device__ inline Place(const Args& f, int at) {
    dim = f.dim;
    half = f.pairs;
    interleaved = f.interleaved;
    pair = at * E;
    inside = 2 * pair < dim;
    if (interleaved) {
      a = 2 * pair;
      b = a + E;
    } else if (pair < half) {
      a = pair;
      b = pair + half;
    } else {   // columns that do not turn
      a = 2 * half + 2 * (pair - half);
      b = a + E;
    }
  }
  // Not VEC: a copy whose columns are formed again, not held (with their bounds' masks) over the loop.
  __device__ inline Place again() const {
    Place p = *this;
    asm volatile("" : "+v"(p.pair));
    return p;
  }
  // Columns of pair e (not VEC); the second may be past the row.
  __device__ inline int first(int e) const {
    const int p = pair + e;
    return interleaved || p >= half ? 2 * p : p;
  }
  __device__ inline int second(int e) const {
    const int p = pair + e;
    return interleaved || p >= half ? 2 * p + 1 : p + half;
  }
  // v, or 0 for a column past the row: as a mask in a vector register.
  __device__ inline float within(float v, int column) const {
    int m = (column - dim) >> 31;
    asm volatile("" : "+v"(m));
    return __int_as_float(__float_as_int(v) & m);
  }
  __device__ inline void load(const void* row, float (&x)[E], float (&y)[E]) const {
    if constexpr (VEC) {
      u32x4 u = {0u, 0u, 0u, 0u}, v = u;
      if (inside) {
        u = *reinterpret_cast<const u32x4*>(static_cast<const char*>(row) + a * IO::kBytes);
        v = *reinterpret_cast<const u32x4*>(static_cast<const char*>(row) + b * IO::kBytes);
      }
      float s[E], t[E];
      IO::unpack(u, s);
      IO::unpack(v, t);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float left = e < E / 2 ? s[2 * e % E] : t[2 * e % E], right = e < E / 2 ? s[(2 * e + 1) % E] : t[(2 * e + 1) % E];
        x[e] = interleaved ? left : s[e];
        y[e] = interleaved ? right : t[e];
      }
    } else {
      const Place p = again();
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = p.first(e), j = p.second(e);
        x[e] = within(IO::load1(row, i < dim ? i : 0), i);
        y[e] = within(IO::load1(row, j < dim ? j : 0), j);
      }
    }
  }
  __device__ inline void store(void* row, const float (&x)[E], const float (&y)[E]) const {
    if constexpr (VEC) {
      float s[E], t[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        s[e] = interleaved ? (e % 2 ? y[e / 2] : x[e / 2]) : x[e];
        t[e] = interleaved ? (e % 2 ? y[(E + e) / 2] : x[(E + e) / 2]) : y[e];
      }
      if (inside) {
        *reinterpret_cast<u32x4*>(static_cast<char*>(row) + a * IO::kBytes) = IO::pack(s);
        *reinterpret_cast<u32x4*>(static_cast<char*>(row) + b * IO::kBytes) = IO::pack(t);
      }
    } else {
      const Place p = again();
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (p.first(e) < dim) IO::store1(row, p.first(e), x[e]);
        if (p.second(e) < dim) IO::store1(row, p.second(e), y[e]);
      }
    }
  }
  __device__ inline void load_gain(const void* g, bool bf16, float (&x)[E], float (&y)[E]) const {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = column_a(e) < dim ? column_a(e) : 0, j = column_b(e) < dim ? column_b(e) : 0;   // columns past the row hold 0
      x[e] = bf16 ? BF16::load1(g, i) : F32::load1(g, i);
      y[e] = bf16 ? BF16::load1(g, j) : F32::load1(g, j);
    }
  }
  // The columns of pair e.
  __device__ inline int column_a(int e) const { return VEC ? (interleaved ? a + 2 * e : a + e) : first(e); }
  __device__ inline int column_b(int e) const { return VEC ? (interleaved ? a + 2 * e + 1 : b + e) : second(e); }
};

// Cosine and sine of a whole number of 2^-64 revolutions.
__device__ inline void cos_sin(uint64_t turns, float& c, float& s) {
  const uint64_t near = turns + (uint64_t(1) << 61);
  const int quarter = int(near >> 62);
  const int32_t rest = int32_t(uint32_t(turns >> 32) - (uint32_t(quarter) << 30));   // of 2^-32, at most an eighth
  const float r = float(rest) * 1.46291807926715968e-9f;                           // 2 pi 2^-32
  const float q = r * r;
  const float sn = __builtin_fmaf(
      r * q, __builtin_fmaf(q, __builtin_fmaf(q, __builtin_fmaf(q, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -0.166666667f), r);
  const float cs = __builtin_fmaf(
      q, __builtin_fmaf(q, __builtin_fmaf(q, __builtin_fmaf(q, __builtin_fmaf(q, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f), 1.0f);
  const float x = quarter & 1 ? sn : cs, y = quarter & 1 ? cs : sn;
  c = quarter == 1 || quarter == 2 ? -x : x;
  s = quarter >= 2 ? -y : y;
}

template <class IO, bool VEC>
__device__ inline void angles(const Args& f, const Place<IO, VEC>& at, int64_t token, float (&c)[IO::kPerVec], float (&s)[IO::kPerVec]) {
#pragma unroll
  for (int e = 0; e < IO::kPerVec; ++e) {
    c[e] = 1.0f;
    s[e] = 0.0f;
    const int p = at.pair + e;
    if (p < f.pairs) {
      const int64_t i = int64_t(f.axis[p]) * f.axis_stride + token;
      const int64_t pos = f.wide ? static_cast<const int64_t*>(f.positions)[i] : static_cast<const int32_t*>(f.positions)[i];
      cos_sin(uint64_t(pos) * f.freq[p], c[e], s[e]);
      s[e] *= f.sign;
    }
  }
}

__device__ inline float sum_lanes(float v, int lanes) {
  for (int off = lanes >> 1; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  return v;
}

// Blocks of 4 waves, queries (blockIdx.y 0) or keys; `shares` waves take a token's heads in turn, `rows` heads at a time.
template <class IO, int MODE, bool VEC>
__global__ __launch_bounds__(256) void rope_kernel(Args f) {
  constexpr int E = IO::kPerVec;
  const int lane = threadIdx.x & (kWave - 1);
  const Side d = blockIdx.y == 0 ? f.side[0] : f.side[1];
  const Place<IO, VEC> at(f, lane & (f.lanes - 1));
  const int in_step = lane / f.lanes;
  float ga[E], gb[E], sum_a[E], sum_b[E];
  bool gains = false;
  if constexpr (MODE == kNorm || MODE == kNormBackGain) {
    gains = d.gain != nullptr;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      ga[e] = gb[e] = 1.0f;
      sum_a[e] = sum_b[e] = 0.0f;
    }
    if (gains) at.load_gain(d.gain, f.gain_bf16, ga, gb);
  }
  const int64_t units = (f.tokens - f.first) * d.shares;
  for (int64_t u = int64_t(blockIdx.x) * 4 + wave_in_block(); u < units; u += int64_t(gridDim.x) * 4) {
    const int64_t token = f.first + u / d.shares;
    float c[E], s[E];
    angles(f, at, token, c, s);
    for (int head = int(u % d.shares) * f.rows + in_step; head - in_step < d.heads; head += d.shares * f.rows) {
      const bool real = head < d.heads;
      const int h = real ? head : 0;
      const char* x = static_cast<const char*>(d.x) + (token * d.x_row + h * d.x_head) * IO::kBytes;
      char* y = static_cast<char*>(d.y) + (token * d.y_row + h * d.y_head) * IO::kBytes;
      float a[E], b[E];
      at.load(x, a, b);
      if constexpr (MODE == kTurn) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float p = a[e], q = b[e];
          a[e] = __builtin_fmaf(p, c[e], -q * s[e]);
          b[e] = __builtin_fmaf(p, s[e], q * c[e]);
        }
      } else if constexpr (MODE == kNorm) {
        float sq = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) sq = __builtin_fmaf(a[e], a[e], __builtin_fmaf(b[e], b[e], sq));
        float mean = sum_lanes(sq, f.lanes) / float(f.dim) + f.eps, unit_ = 1.0f;
        // squares that fp32 does not hold are added up again as (x unit)^2
        const bool large = !(mean < 3.0e38f), tiny = mean < 0x1p-90f;
        if (__any(large || tiny)) {
          unit_ = large ? 0x1p-96f : tiny ? 0x1p60f : 1.0f;
          sq = 0.0f;
#pragma unroll
          for (int e = 0; e < E; ++e)
            sq = __builtin_fmaf(a[e] * unit_, a[e] * unit_, __builtin_fmaf(b[e] * unit_, b[e] * unit_, sq));
          mean = sum_lanes(sq, f.lanes) / float(f.dim) + f.eps * unit_ * unit_;
        }
        const float r = rsqrtf(mean);
        if (real && (lane & (f.lanes - 1)) == 0) d.rstd[token * d.heads + head] = r * unit_;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float p = a[e] * unit_ * r * ga[e], q = b[e] * unit_ * r * gb[e];
          a[e] = __builtin_fmaf(p, c[e], -q * s[e]);
          b[e] = __builtin_fmaf(p, s[e], q * c[e]);
        }
      } else {
        float p[E], q[E];
        at.load(static_cast<const char*>(d.kept) + (token * d.kept_row + h * d.kept_head) * IO::kBytes, p, q);
        const float r = d.rstd[token * d.heads + h];
        float along = 0.0f;
        if constexpr (MODE == kNormBack) {
#pragma unroll
          for (int e = 0; e < E; ++e) along = __builtin_fmaf(a[e], p[e], __builtin_fmaf(b[e], q[e], along));
          along = sum_lanes(along, f.lanes) / float(f.dim);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float v = r * __builtin_fmaf(-p[e], along, a[e]), w = r * __builtin_fmaf(-q[e], along, b[e]);
            a[e] = __builtin_fmaf(v, c[e], -w * s[e]);
            b[e] = __builtin_fmaf(v, s[e], w * c[e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float v = __builtin_fmaf(a[e], c[e], -b[e] * s[e]), w = __builtin_fmaf(a[e], s[e], b[e] * c[e]);
            p[e] *= r;
            q[e] *= r;
            sum_a[e] = __builtin_fmaf(real ? v : 0.0f, real ? p[e] : 0.0f, sum_a[e]);
            sum_b[e] = __builtin_fmaf(real ? w : 0.0f, real ? q[e] : 0.0f, sum_b[e]);
            a[e] = v * ga[e];
            b[e] = w * gb[e];
            along = __builtin_fmaf(a[e], p[e], __builtin_fmaf(b[e], q[e], along));
          }
          along = sum_lanes(along, f.lanes) / float(f.dim);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            a[e] = r * __builtin_fmaf(-p[e], along, a[e]);
            b[e] = r * __builtin_fmaf(-q[e], along, b[e]);
          }
        }
      }
      if (real) at.store(y, a, b);
    }
  }
  if constexpr (MODE == kNormBackGain) {   // heads of a wave, waves of the block, in order
    __shared__ float lds[4][kRopeDim];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float v = sum_a[e], w = sum_b[e];
      for (int off = f.lanes; off < kWave; off <<= 1) {
        v += __shfl_xor(v, off, kWave);
        w += __shfl_xor(w, off, kWave);
      }
      if (lane < f.lanes) {
        if (at.column_a(e) < f.dim) lds[wave_in_block()][at.column_a(e)] = v;
        if (at.column_b(e) < f.dim) lds[wave_in_block()][at.column_b(e)] = w;
      }
    }
    __syncthreads();
    for (int j = threadIdx.x; j < f.dim; j += 256)
      f.part[(int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * f.dim + j] = (lds[0][j] + lds[1][j]) + (lds[2][j] + lds[3][j]);
  }
}

// Gains' gradients: a block per 4 columns and side, a wave's lanes over the blocks' sums.
__global__ __launch_bounds__(256) void rope_gain_kernel(const float* part, int blocks, int dim, int bf16, void* q, void* k) {
  const int side = blockIdx.y, j = int(blockIdx.x) * 4 + wave_in_block(), lane = threadIdx.x & (kWave - 1);
  void* to = side == 0 ? q : k;
  if (to == nullptr || j >= dim) return;
  float v = 0.0f;
  for (int b = lane; b < blocks; b += kWave) v += part[(int64_t(side) * blocks + b) * dim + j];
  v = wave_sum(v);
  if (lane == 0) {
    if (bf16) BF16::store1(to, j, v);
    else F32::store1(to, j, v);
  }
}

}  // namespace rope

namespace {

constexpr int kGainBlocks = 512;   // of the backward with gains: one sum of each to the workspace

int lanes_of(int64_t dim, int per) {
  int lanes = 1;
  while (int64_t(lanes) * per * 2 < dim) lanes *= 2;
  return lanes;
}

// How a launch is split: a token's heads over more waves while the device has room.
template <class IO>
void plan(rope::Args& f) {
  f.lanes = lanes_of(f.dim, IO::kPerVec);
  f.rows = kWave / f.lanes;
  for (rope::Side& d : f.side) {
    const int steps = (d.heads + f.rows - 1) / f.rows;
    d.shares = 1;
    while (d.shares < steps && f.tokens * d.shares < 4096) d.shares *= 2;
    d.shares = std::max(1, std::min(d.shares, steps));
  }
}
// Blocks for `tokens` tokens of the side that takes more of them.
int64_t blocks_of(const rope::Args& f, int64_t tokens) { return (tokens * std::max(f.side[0].shares, f.side[1].shares) + 3) / 4; }
int gain_blocks(const rope::Args& f) { return int(std::clamp<int64_t>(blocks_of(f, f.tokens), 1, kGainBlocks)); }

template <class IO, int MODE>
hipError_t launch(const rope::Args& f, bool vec, hipStream_t s) {
  if constexpr (MODE == rope::kNormBackGain) {
    const dim3 grid(gain_blocks(f), 2);
    if (vec) rope::rope_kernel<IO, MODE, true><<<grid, 256, 0, s>>>(f);
    else rope::rope_kernel<IO, MODE, false><<<grid, 256, 0, s>>>(f);
    return hipGetLastError();
  } else {
    // tokens to a launch; the kernel takes what lies from its first token on
    const int64_t part = most_blocks(256) / std::max(f.side[0].shares, f.side[1].shares) * 4;
    return in_parts(f.tokens, part, [&](int64_t first, int64_t count) {
      rope::Args g = f;
      g.first = first;
      g.tokens = first + count;
      const dim3 grid(uint32_t(blocks_of(f, count)), f.side[1].heads > 0 ? 2 : 1);
      if (vec) rope::rope_kernel<IO, MODE, true><<<grid, 256, 0, s>>>(g);
      else rope::rope_kernel<IO, MODE, false><<<grid, 256, 0, s>>>(g);
    });
  }
}

rope::Args args_of(const RopePlan& r, bool bf16, bool& vec) {
  rope::Args f{};
  f.positions = r.positions;
  f.axis_stride = r.axis_stride;
  f.tokens = r.tokens;
  f.dim = int(r.dim);
  f.pairs = int(r.pairs);
  f.wide = r.wide;
  f.interleaved = r.interleaved;
  for (int p = 0; p < r.pairs; ++p) {
    f.axis[p] = uint8_t(r.axes ? r.axes[p] : 0);
    // the frequency in revolutions as a whole number of 2^-64: what is lost is below 2^-63 of a turn per position
    const long double turns = static_cast<long double>(r.freqs[p]) / 6.283185307179586476925286766559005768L;
    const long double part = (turns - std::floor(turns)) * 18446744073709551616.0L;
    f.freq[p] = part >= 18446744073709551615.0L ? ~uint64_t(0) : uint64_t(part);
  }
  const int per = bf16 ? 8 : 4;
  vec = r.dim % (2 * per) == 0 && (r.interleaved || r.pairs % per == 0);
  return f;
}

void side_of(rope::Side& d, const HeadsView& x, const HeadsView& y, const HeadsView& kept, float* rstd, const void* gain, int64_t heads,
             bool bf16, bool& vec) {
  d.x = x.p;
  d.y = y.p;
  d.kept = kept.p;
  d.rstd = rstd;
  d.gain = gain;
  d.x_row = x.row, d.x_head = x.head;
  d.y_row = y.row, d.y_head = y.head;
  d.kept_row = kept.row, d.kept_head = kept.head;
  d.heads = int(heads);
  const int per = bf16 ? 8 : 4;
  for (const HeadsView* v : {&x, &y, &kept})
    if (heads > 0 && v->p != nullptr)
      vec = vec && reinterpret_cast<uintptr_t>(v->p) % 16 == 0 && v->row % per == 0 && v->head % per == 0;
}

template <int MODE>
hipError_t launch_type(bool bf16, rope::Args& f, bool vec, hipStream_t s) {
  if (bf16) plan<BF16>(f);
  else plan<F32>(f);
  return bf16 ? launch<BF16, MODE>(f, vec, s) : launch<F32, MODE>(f, vec, s);
}

}  // namespace

size_t msrms_rope_bwd_workspace(int64_t dim) { return size_t(kGainBlocks) * 2 * size_t(dim) * 4; }

hipError_t launch_rope(bool bf16, const RopePlan& r, bool back, const HeadsView (&x)[2], const HeadsView (&y)[2], hipStream_t s) {
  bool vec;
  rope::Args f = args_of(r, bf16, vec);
  f.sign = back ? -1.0f : 1.0f;
  for (int i = 0; i < 2; ++i) side_of(f.side[i], x[i], y[i], HeadsView{}, nullptr, nullptr, r.heads[i], bf16, vec);
  return launch_type<rope::kTurn>(bf16, f, vec, s);
}

hipError_t launch_msrms_rope_fwd(bool bf16, const RopePlan& r, float eps, bool gain_bf16, const void* const (&gain)[2],
                                 const HeadsView (&x)[2], const HeadsView (&y)[2], float* const (&rstd)[2], hipStream_t s) {
  bool vec;
  rope::Args f = args_of(r, bf16, vec);
  f.sign = 1.0f;
  f.eps = eps;
  f.gain_bf16 = gain_bf16;
  for (int i = 0; i < 2; ++i) side_of(f.side[i], x[i], y[i], HeadsView{}, rstd[i], gain[i], r.heads[i], bf16, vec);
  return launch_type<rope::kNorm>(bf16, f, vec, s);
}

hipError_t launch_msrms_rope_bwd(bool bf16, const RopePlan& r, bool gain_bf16, const void* const (&gain)[2], const HeadsView (&dy)[2],
                                 const HeadsView (&kept)[2], const float* const (&rstd)[2], const HeadsView (&dx)[2],
                                 void* const (&dgain)[2], void* workspace, hipStream_t s) {
  bool vec;
  rope::Args f = args_of(r, bf16, vec);
  f.sign = -1.0f;
  f.gain_bf16 = gain_bf16;
  f.part = static_cast<float*>(workspace);
  for (int i = 0; i < 2; ++i)
    side_of(f.side[i], dy[i], dx[i], kept[i], const_cast<float*>(rstd[i]), gain[i], r.heads[i], bf16, vec);
  if (gain[0] == nullptr && gain[1] == nullptr) return launch_type<rope::kNormBack>(bf16, f, vec, s);
  const hipError_t e = launch_type<rope::kNormBackGain>(bf16, f, vec, s);
  if (e != hipSuccess) return e;
  rope::rope_gain_kernel<<<dim3(uint32_t((r.dim + 3) / 4), 2), 256, 0, s>>>(f.part, gain_blocks(f), int(r.dim), gain_bf16, dgain[0], dgain[1]);
  return hipGetLastError();
}

}  // namespace lmbp
