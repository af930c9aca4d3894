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
//
// What bounds it: memory. A wave takes heads of one token, 4 (backward 2) of each lane's at a time whose loads run while the
// angles are formed: each pair's by one lane, handed round through LDS (formed by every lane for its own columns they cost
// 7 us on each pass over the token, 8 us more in all). Loads and stores are non-temporal (52 us without). 8192 tokens of 32 + 32
// heads of 128, bf16: turned 43 to 46 us (5.9 to 6.2 TB/s), norm and turn 48, its backward 64 (6.3); 2, 4 and 8 waves to a token
// instead of one 47 -> 45, 48 -> 48, 67 -> 64. A half that is no multiple of 16 bytes goes in pieces of 8 where that does, else element by element: 1531
// tokens of 12 heads of 72, 18 pairs, fp32, with gains 9.2 us, backward 10.7 and 3.8 for the sum of the gains' gradients (element by
// element 11.5 and 12.1); 8192 of 16 + 16 of 72, bf16, 31 and 32 without gains (45 and 59).
#include "lmbp_device.hpp"
#include "lmbp_launch.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace lmbp {
namespace rope {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

enum { kTurn = 0, kNorm = 1, kNormBack = 2, kNormGain = 3, kNormBackGain = 4 };
enum { kSingle = 0, kHalves = 1, kPairs = 2 };   // element by element; 16- or 8-byte pieces of pairs half apart, side by side

// Queries or keys: one tensor's heads.
struct Side {
  const void* x;      // read: x, or the gradient of y
  void* y;            // written
  const void* kept;   // backward: y without gain, x with
  float* rstd;        // [tokens][heads]; written by the forward
  const void* gain;   // [dim] or null
  int64_t x_row, x_head, y_row, y_head, kept_row, kept_head;
  int heads, steps;   // steps: of `rows` heads
};

struct Args {
  Side side[2];
  const void* positions;
  int64_t axis_stride, tokens;
  float* part;        // kNormBackGain: [2][blocks][dim]
  int64_t first;      // token of this launch's first block
  int dim, pairs, lanes, rows;   // lanes to a head (a power of two), heads to a wave at a time
  int shares;         // waves that take a token's heads in turn
  int blocks;         // kNormBackGain: of each side
  float eps, sign;
  uint8_t wide, interleaved, gain_bf16;
  uint8_t axis[kRopePairs];
  uint64_t freq[kRopePairs];
};

// Pieces of 8 bytes, for heads whose halves are no multiple of 16.
struct BF16Narrow : BF16 {
  static constexpr int kPerVec = 4;
  static __device__ inline void unpack(const u32x2& v, float (&f)[4]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      f[2 * k] = __uint_as_float(v[k] << 16);
      f[2 * k + 1] = __uint_as_float(v[k] & 0xffff0000u);
    }
  }
  static __device__ inline u32x2 pack(const float (&f)[4]) { return u32x2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])}; }
};
struct F32Narrow : F32 {
  static constexpr int kPerVec = 2;
  static __device__ inline void unpack(const u32x2& v, float (&f)[2]) {
    f[0] = __uint_as_float(v[0]);
    f[1] = __uint_as_float(v[1]);
  }
  static __device__ inline u32x2 pack(const float (&f)[2]) { return u32x2{__float_as_uint(f[0]), __float_as_uint(f[1])}; }
};

// This lane's place in a head: E pairs, two pieces of E columns or 2 E single columns.
template <class IO, int FORM>
struct Place {
  static constexpr int E = IO::kPerVec;
  static constexpr bool VEC = FORM != kSingle;
  using Vec = std::conditional_t<E * IO::kBytes == 16, u32x4, u32x2>;
  int pair, a, b;   // first pair; VEC: where the pieces start
  int dim, half;
  bool inside;
  bool interleaved;   // known when compiled but for kSingle
  __device__ inline Place(const Args& f, int at) {
    dim = f.dim;
    half = f.pairs;
    interleaved = FORM == kSingle ? f.interleaved : FORM == kPairs;
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
  // A head's values of this lane as they come from memory, so that several heads' loads run before the first is used.
  struct Raw {
    Vec u, v;               // VEC
    float x[VEC ? 1 : E], y[VEC ? 1 : E];
  };
  __device__ inline void load(const void* row, Raw& r) const {
    if constexpr (VEC) {
      r.u = r.v = Vec{};
      if (inside) {
        r.u = __builtin_nontemporal_load(reinterpret_cast<const Vec*>(static_cast<const char*>(row) + a * IO::kBytes));
        r.v = __builtin_nontemporal_load(reinterpret_cast<const Vec*>(static_cast<const char*>(row) + b * IO::kBytes));
      }
    } else {
      const Place p = again();
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = p.first(e), j = p.second(e);
        r.x[e] = within(IO::load1(row, i < dim ? i : 0), i);
        r.y[e] = within(IO::load1(row, j < dim ? j : 0), j);
      }
    }
  }
  __device__ inline void unpack(const Raw& r, float (&x)[E], float (&y)[E]) const {
    if constexpr (VEC) {
      float s[E], t[E];
      IO::unpack(r.u, s);
      IO::unpack(r.v, t);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float left = e < E / 2 ? s[2 * e % E] : t[2 * e % E], right = e < E / 2 ? s[(2 * e + 1) % E] : t[(2 * e + 1) % E];
        x[e] = interleaved ? left : s[e];
        y[e] = interleaved ? right : t[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        x[e] = r.x[e];
        y[e] = r.y[e];
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
        __builtin_nontemporal_store(IO::pack(s), reinterpret_cast<Vec*>(static_cast<char*>(row) + a * IO::kBytes));
        __builtin_nontemporal_store(IO::pack(t), reinterpret_cast<Vec*>(static_cast<char*>(row) + b * IO::kBytes));
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
  // Pair e turned. Columns behind the pairs are left as they are: not by an angle of 0, since 0 times an infinite neighbour is NaN.
  // AGAIN: asked each time, where held over the loop the answers would take more scalar registers than there are.
  template <bool AGAIN>
  __device__ inline void turn(int e, float p, float q, float c, float s, float& x, float& y) const {
    int p0 = FORM == kHalves ? pair : pair + e;   // halves turn in whole pieces
    if constexpr (AGAIN) asm volatile("" : "+v"(p0));
    const bool turns = p0 < half;
    x = turns ? __builtin_fmaf(p, c, -q * s) : p;
    y = turns ? __builtin_fmaf(p, s, q * c) : q;
  }
  // This lane's pairs turned. VEC: whether all do is asked once. 8192 tokens of 32 + 32 heads of 72, halves, norm and turn 40.4 us, with
  // a select for every pair 43.1; element by element it is the other way round (129 and 122 at 100 columns), and so is the norm's forward
  // with pairs side by side (42.9 and 38.4), which turns them one by one.
  __device__ inline void turn(float (&x)[E], float (&y)[E], const float (&c)[E], const float (&s)[E]) const {
    if (VEC && pair + E <= half) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float p = x[e], q = y[e];
        x[e] = __builtin_fmaf(p, c[e], -q * s[e]);
        y[e] = __builtin_fmaf(p, s[e], q * c[e]);
      }
    } else if constexpr (FORM != kHalves) {
#pragma unroll
      for (int e = 0; e < E; ++e) turn<false>(e, x[e], y[e], c[e], s[e], x[e], y[e]);
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

// Cosines and sines of a token's pairs: each formed once, by one lane of the wave, and handed to the lanes that hold the pair's
// columns through LDS of the wave's own (`table`: kRopePairs cosines, then sines; behind the pairs there are numbers that nothing uses).
template <class IO, int FORM>
__device__ inline void angles(const Args& f, const Place<IO, FORM>& at, int64_t token, float* table, float (&c)[IO::kPerVec],
                              float (&s)[IO::kPerVec]) {
  constexpr int E = IO::kPerVec;
  const int held = f.lanes * E;   // pairs, those behind the row's end included
  __builtin_amdgcn_wave_barrier();   // the last token's have been read (a wave's LDS operations run in order)
  for (int p = threadIdx.x & (kWave - 1); p < held; p += kWave) {
    float co = 1.0f, si = 0.0f;
    if (p < f.pairs) {
      const int64_t i = int64_t(f.axis[p]) * f.axis_stride + token;
      const int64_t pos = f.wide ? static_cast<const int64_t*>(f.positions)[i] : static_cast<const int32_t*>(f.positions)[i];
      cos_sin(uint64_t(pos) * f.freq[p], co, si);
    }
    table[p] = co;
    table[kRopePairs + p] = si * f.sign;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if constexpr (E == 2) {
    const float2 x = *reinterpret_cast<const float2*>(table + at.pair), y = *reinterpret_cast<const float2*>(table + kRopePairs + at.pair);
    c[0] = x.x, c[1] = x.y;
    s[0] = y.x, s[1] = y.y;
    return;
  }
#pragma unroll
  for (int e = 0; e + 4 <= E; e += 4) {
    const float4 x = *reinterpret_cast<const float4*>(table + at.pair + e), y = *reinterpret_cast<const float4*>(table + kRopePairs + at.pair + e);
    c[e] = x.x, c[e + 1] = x.y, c[e + 2] = x.z, c[e + 3] = x.w;
    s[e] = y.x, s[e + 1] = y.y, s[e + 2] = y.z, s[e + 3] = y.w;
  }
}

__device__ inline float sum_lanes(float v, int lanes) {
  for (int off = lanes >> 1; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  return v;
}

// Blocks of 4 waves; `shares` waves take a token's heads in turn, `rows` of the queries' or of the keys' at a time, with the
// token's angles formed once. With gains, which a wave holds over all its tokens (and sums
// their gradients), blocks are the queries' or the keys'.
template <class IO, int MODE, int FORM>
__global__ __launch_bounds__(256) void rope_kernel(Args f) {
  constexpr int E = IO::kPerVec;
  constexpr bool VEC = FORM != kSingle;
  const int lane = threadIdx.x & (kWave - 1);
  const Place<IO, FORM> at(f, lane & (f.lanes - 1));
  const int in_step = lane / f.lanes;
  __shared__ __attribute__((aligned(16))) float tables[4][2 * kRopePairs];
  constexpr bool kGain = MODE == kNormGain || MODE == kNormBackGain, kForward = MODE == kTurn || MODE == kNorm || MODE == kNormGain;
  float ga[E], gb[E], sum_a[E], sum_b[E];
  if constexpr (kGain) {
    at.load_gain(f.side[blockIdx.y].gain, f.gain_bf16, ga, gb);
#pragma unroll
    for (int e = 0; e < E; ++e) sum_a[e] = sum_b[e] = 0.0f;
  }
  const int64_t units = (f.tokens - f.first) * f.shares;
  for (int64_t u = int64_t(blockIdx.x) * 4 + wave_in_block(); u < units; u += int64_t(gridDim.x) * 4) {
    const int64_t token = f.first + u / f.shares;
    int start = int(u % f.shares);   // this wave's first step of the side
    float c[E], s[E];
    bool ready = false;
#pragma unroll 1
    for (int side = kGain ? int(blockIdx.y) : 0; side < (kGain ? int(blockIdx.y) + 1 : 2); ++side) {
      const Side d = side == 0 ? f.side[0] : f.side[1];
      // kBatch heads of each lane at a time: their loads run while the angles are formed
      constexpr int kBatch = !VEC ? 1 : kForward ? 4 : 2;
      const int stride = f.shares * f.rows;
      int group = start * f.rows;
      for (; group < d.heads; group += kBatch * stride) {
        typename Place<IO, FORM>::Raw rx[kBatch], rk[kBatch];
        float rs[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          if (group + j * stride >= d.heads) break;
          const int head = group + j * stride + in_step, h = head < d.heads ? head : 0;
          at.load(static_cast<const char*>(d.x) + (token * d.x_row + h * d.x_head) * IO::kBytes, rx[j]);
          if constexpr (!kForward) {
            if constexpr (!VEC) __builtin_amdgcn_sched_barrier(0);   // masks of one load at a time
            at.load(static_cast<const char*>(d.kept) + (token * d.kept_row + h * d.kept_head) * IO::kBytes, rk[j]);
            rs[j] = d.rstd[token * d.heads + h];
          }
        }
        if (!ready) angles(f, at, token, tables[wave_in_block()], c, s);
        ready = true;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          if (group + j * stride >= d.heads) break;
          const int head = group + j * stride + in_step;
          const bool real = head < d.heads;
          const int h = real ? head : 0;
          char* y = static_cast<char*>(d.y) + (token * d.y_row + h * d.y_head) * IO::kBytes;
          float a[E], b[E];
          at.unpack(rx[j], a, b);
          if constexpr (MODE == kTurn) {
            at.turn(a, b, c, s);
          } else if constexpr (kForward) {
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
              a[e] = a[e] * unit_ * r;
              b[e] = b[e] * unit_ * r;
              if constexpr (kGain) {
                a[e] *= ga[e];
                b[e] *= gb[e];
              }
              if constexpr (FORM == kPairs) at.template turn<false>(e, a[e], b[e], c[e], s[e], a[e], b[e]);
            }
            if constexpr (FORM != kPairs) at.turn(a, b, c, s);
          } else {
            float p[E], q[E];
            at.unpack(rk[j], p, q);
            float r = rs[j], along = 0.0f;
            // a head that is not finite (its rstd is 0 or NaN) and gets no gradient gives none, whatever it holds
            if (__any(!(r > 0.0f))) {
              uint32_t any = 0u;
#pragma unroll
              for (int e = 0; e < E; ++e) any |= (__float_as_uint(a[e]) | __float_as_uint(b[e])) & 0x7fffffffu;
              for (int off = f.lanes >> 1; off > 0; off >>= 1) any |= uint32_t(__shfl_xor(int(any), off, kWave));
              uint32_t keep = r > 0.0f || any != 0u ? ~0u : 0u;   // a mask in a vector register: there is no scalar one left
              asm volatile("" : "+v"(keep));
              r = __uint_as_float(__float_as_uint(r) & keep);
#pragma unroll
              for (int e = 0; e < E; ++e) {
                p[e] = __uint_as_float(__float_as_uint(p[e]) & keep);
                q[e] = __uint_as_float(__float_as_uint(q[e]) & keep);
              }
            }
            if constexpr (MODE == kNormBack) {
#pragma unroll
              for (int e = 0; e < E; ++e) along = __builtin_fmaf(a[e], p[e], __builtin_fmaf(b[e], q[e], along));
              along = sum_lanes(along, f.lanes) / float(f.dim);
#pragma unroll
              for (int e = 0; e < E; ++e) {
                a[e] = r * __builtin_fmaf(-p[e], along, a[e]);
                b[e] = r * __builtin_fmaf(-q[e], along, b[e]);
              }
              at.turn(a, b, c, s);
            } else {
#pragma unroll
              for (int e = 0; e < E; ++e) {   // one by one: the branch of a whole lane takes registers that this kernel has not
                float v, w;
                at.template turn<FORM == kPairs && E < 8>(e, a[e], b[e], c[e], s[e], v, w);
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
      start = (start + f.shares - d.steps % f.shares) % f.shares;
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

constexpr int kGainBlocks = 1024;   // at most, of the backward with gains: one sum of each to the workspace

int lanes_of(int64_t dim, int per) {
  int lanes = 1;
  while (int64_t(lanes) * per * 2 < dim) lanes *= 2;
  return lanes;
}

// How a launch is split: a token's heads over more waves while the device has room.
template <class IO>
void plan(rope::Args& f, bool apart) {
  f.lanes = lanes_of(f.dim, IO::kPerVec);
  f.rows = kWave / f.lanes;
  int steps = 0;   // that a token's waves share
  for (rope::Side& d : f.side) {
    d.steps = (d.heads + f.rows - 1) / f.rows;
    steps = apart ? std::max(steps, d.steps) : steps + d.steps;
  }
  f.shares = 1;
  while (f.shares < steps && f.tokens * f.shares < 32768) f.shares *= 2;
  f.shares = std::min(f.shares, steps);
}
int64_t blocks_of(const rope::Args& f, int64_t tokens) { return (tokens * f.shares + 3) / 4; }
// Blocks of the backward with gains, of each side: about as many as are resident at once, which walk over the tokens. Pieces of 8 bf16 (156
// registers) leave room for 3 to a CU, 384 to a side: 8192 tokens of 32 + 32 heads of 128 85 us (512: 108, 256: 98), of 32 + 8 68 (91, 75).
// The others 4: 4000 tokens of 12 + 12 fp32 heads of 64 22 us (twice as many 25, half 24).
int gain_blocks(const rope::Args& f, bool wide) {
  const int64_t most = (wide ? kGainBlocks / 4 * 3 : kGainBlocks) / (f.side[1].heads > 0 ? 2 : 1);
  return int(std::clamp<int64_t>(blocks_of(f, f.tokens), 1, most));
}

template <class IO, int MODE>
hipError_t launch(rope::Args& f, bool vec, hipStream_t s) {
  auto go = [&](const rope::Args& g, dim3 grid) {
    if (!vec) {
      if constexpr (IO::kPerVec * IO::kBytes == 16) rope::rope_kernel<IO, MODE, rope::kSingle><<<grid, 256, 0, s>>>(g);
    } else if (g.interleaved) rope::rope_kernel<IO, MODE, rope::kPairs><<<grid, 256, 0, s>>>(g);
    else {
      rope::rope_kernel<IO, MODE, rope::kHalves><<<grid, 256, 0, s>>>(g);
    }
  };
  if constexpr (MODE == rope::kNormBackGain || MODE == rope::kNormGain) {
    // Forward: 8192 tokens of 32 + 32 heads of 128, bf16, 59 us; 1280 to a side 62, 640 71, one wave to each unit 83: it reads its gains by
    // single elements, which so far is what many tokens to a wave make up for.
    const int blocks = MODE == rope::kNormGain ? int(std::clamp<int64_t>(blocks_of(f, f.tokens), 1, 2 * kGainBlocks)) : gain_blocks(f, IO::kPerVec == 8);
    f.blocks = blocks;
    go(f, dim3(blocks, f.side[1].heads > 0 ? 2 : 1));
    return hipGetLastError();
  } else {
    // tokens to a launch; the kernel takes what lies from its first token on
    return in_parts(f.tokens, most_blocks(256) / f.shares * 4, [&](int64_t first, int64_t count) {
      rope::Args g = f;
      g.first = first;
      g.tokens = first + count;
      go(g, dim3(uint32_t(blocks_of(f, count))));
    });
  }
}

// A frequency of |f| < 2^52 radians in revolutions modulo 1, as a whole number of 2^-64 (cut off twice, so within 1.5 of them): its 53 bits
// times 1 / (2 pi) to 128 bits. In long double this took 4 us of a call with 64 pairs (10.0 us in all, 6.2 so).
uint64_t turns_of(double f) {
  constexpr uint64_t kInverse[2] = {0x28be60db9391054aull, 0x7f09d5f47d4d3770ull};
  int e = 0;
  const uint64_t m = uint64_t(std::ldexp(std::frexp(std::fabs(f), &e), 53));   // |f| = m 2^(e - 53)
  e -= 53;
  if (e >= 0) {   // more than a turn's bits: what a position turns by is lost in f's own rounding
    const long double t = static_cast<long double>(f) / 6.283185307179586476925286766559005768L;
    const long double part = (t - std::floor(t)) * 18446744073709551616.0L;
    return part >= 18446744073709551615.0L ? ~uint64_t(0) : uint64_t(part);
  }
  using Wide = unsigned __int128;
  const Wide high = Wide(m) * kInverse[0] + uint64_t(Wide(m) * kInverse[1] >> 64);   // m / (2 pi) in 2^-64
  const Wide part = e > -128 ? high >> -e : 0;
  return f < 0 ? -uint64_t(part) : uint64_t(part);
}

rope::Args args_of(const RopePlan& r) {
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
    f.freq[p] = turns_of(r.freqs[p]);
  }
  return f;
}

void side_of(rope::Side& d, const HeadsView& x, const HeadsView& y, const HeadsView& kept, float* rstd, const void* gain, int64_t heads) {
  d.x = x.p;
  d.y = y.p;
  d.kept = kept.p;
  d.rstd = rstd;
  d.gain = gain;
  d.x_row = x.row, d.x_head = x.head;
  d.y_row = y.row, d.y_head = y.head;
  d.kept_row = kept.row, d.kept_head = kept.head;
  d.heads = int(heads);
}

// Whether heads can be taken in pieces of `per` elements.
bool in_pieces(const rope::Args& f, int per, int bytes) {
  if (f.dim % (2 * per) != 0 || f.dim > 2 * per * kWave || (!f.interleaved && f.pairs % per != 0)) return false;
  for (const rope::Side& d : f.side) {
    if (d.heads == 0) continue;
    for (const void* p : {d.x, static_cast<const void*>(d.y), d.kept})
      if (reinterpret_cast<uintptr_t>(p) % uintptr_t(per * bytes) != 0) return false;
    for (int64_t stride : {d.x_row, d.x_head, d.y_row, d.y_head, d.kept_row, d.kept_head})
      if (stride % per != 0) return false;
  }
  return true;
}

template <class IO, class NARROW, int MODE>
hipError_t launch_pieces(rope::Args& f, bool apart, hipStream_t s) {
  const bool wide = in_pieces(f, IO::kPerVec, IO::kBytes);
  if (!wide && in_pieces(f, NARROW::kPerVec, IO::kBytes)) {
    plan<NARROW>(f, apart);
    return launch<NARROW, MODE>(f, true, s);
  }
  plan<IO>(f, apart);
  return launch<IO, MODE>(f, wide, s);
}

template <int MODE>
hipError_t launch_type(bool bf16, rope::Args& f, hipStream_t s) {
  constexpr bool kApart = MODE == rope::kNormBackGain || MODE == rope::kNormGain;   // queries and keys in blocks of their own
  return bf16 ? launch_pieces<BF16, rope::BF16Narrow, MODE>(f, kApart, s) : launch_pieces<F32, rope::F32Narrow, MODE>(f, kApart, s);
}

}  // namespace

size_t msrms_rope_bwd_workspace(int64_t dim) { return size_t(kGainBlocks) * size_t(dim) * 4; }

hipError_t launch_rope(bool bf16, const RopePlan& r, bool back, const HeadsView (&x)[2], const HeadsView (&y)[2], hipStream_t s) {
  rope::Args f = args_of(r);
  f.sign = back ? -1.0f : 1.0f;
  for (int i = 0; i < 2; ++i) side_of(f.side[i], x[i], y[i], HeadsView{}, nullptr, nullptr, r.heads[i]);
  return launch_type<rope::kTurn>(bf16, f, s);
}

hipError_t launch_msrms_rope_fwd(bool bf16, const RopePlan& r, float eps, bool gain_bf16, const void* const (&gain)[2],
                                 const HeadsView (&x)[2], const HeadsView (&y)[2], float* const (&rstd)[2], hipStream_t s) {
  rope::Args f = args_of(r);
  f.sign = 1.0f;
  f.eps = eps;
  f.gain_bf16 = gain_bf16;
  for (int i = 0; i < 2; ++i) side_of(f.side[i], x[i], y[i], HeadsView{}, rstd[i], gain[i], r.heads[i]);
  return gain[0] != nullptr ? launch_type<rope::kNormGain>(bf16, f, s) : launch_type<rope::kNorm>(bf16, f, s);
}

hipError_t launch_msrms_rope_bwd(bool bf16, const RopePlan& r, bool gain_bf16, const void* const (&gain)[2], const HeadsView (&dy)[2],
                                 const HeadsView (&kept)[2], const float* const (&rstd)[2], const HeadsView (&dx)[2],
                                 void* const (&dgain)[2], void* workspace, hipStream_t s) {
  rope::Args f = args_of(r);
  f.sign = -1.0f;
  f.gain_bf16 = gain_bf16;
  f.part = static_cast<float*>(workspace);
  for (int i = 0; i < 2; ++i)
    side_of(f.side[i], dy[i], dx[i], kept[i], const_cast<float*>(rstd[i]), gain[i], r.heads[i]);
  if (gain[0] == nullptr && gain[1] == nullptr) return launch_type<rope::kNormBack>(bf16, f, s);
  const hipError_t e = launch_type<rope::kNormBackGain>(bf16, f, s);
  if (e != hipSuccess) return e;
  rope::rope_gain_kernel<<<dim3(uint32_t((r.dim + 3) / 4), r.heads[1] > 0 ? 2 : 1), 256, 0, s>>>(f.part, f.blocks, int(r.dim), gain_bf16, dgain[0], dgain[1]);
  return hipGetLastError();
}

}  // namespace lmbp
