// Attention backward for gfx950. With P = exp(scale q k^T - lse), D = rowsum(do o), dS = P (do v^T - D):
//
//   dq = scale dS k,  dk = scale dS^T q,  dv = P^T do
//
// Two kernels, each forming the scores again: dq per rows (which also writes each row's lse and D for the other),
// dk and dv per keys. One kernel for all three would have to add dq up with atomics, whose order changes results.
//
// The matrix units bound both: three and four products of the forward's size. P and dS are formed in fp32 and rounded to bf16 once, as
// operands. 16384 tokens of 32 heads on 8, dim 128, causal: dq 2.83 ms (1167 TFLOP/s, matrix units 62% of the cycles), dk and dv 3.93
// (1120, 56%), at the power limit's 1.8 to 1.9 GHz; 4 sequences of 2048, 32 heads: 232 and 304 us. The order of LDS reads, MFMAs and
// exponentials is written out (left to the compiler dk and dv took 4.75 ms). Two waves to a SIMD with 256 registers: one with 512,
// which reads LDS less often, took 4.44 to 5.18, since a lone wave issues too seldom. Narrow heads' dk and dv fit three waves (64
// images of 197, 12 heads of 64: 37.4 us, two 42.6).
#include "attention_device.hpp"

#include <algorithm>
#include <type_traits>

namespace lmbp {
namespace attn {

struct BwdArgs {
  Shape s;
  Heads q, k, v, o, d_o, dq, dk, dv;
  const float* lse;   // [rows][heads]
  float* stats;       // [kv_heads][rows * group][2]: lse in log2, D
  float* part;        // shares > 1: [shares][2][rows of k][kv_heads][dim]: dk, dv
  int shares, share;  // the most shares of a key tile's rows; row tiles that one share should have
  int64_t first;      // block number of this launch's first block
  uint32_t per_xcd;
};

constexpr int kKeys = 64;   // keys to a tile of the dq kernel
constexpr int kRows = 32;   // packed rows to a tile of the dk, dv kernel

template <int D>
struct Queries {
  using T = Tile<D>;
  bf16x8 q[T::kSteps], d_o[T::kSteps];
  f32x16 dq[T::kBlocks];
  float lse, share;   // lse in log2; D
  int limit;

  // P (D less) of value i from its scores.
  __device__ inline void weight(f32x16& x, const f32x16& y, int i, float c) const {
    x[i] = exp2_fast(__builtin_fmaf(x[i], c, -lse)) * (y[i] - share);
  }
  // q k^T and do v^T of 32 keys, the tile's from `first` on; operands are read two steps ahead.
  __device__ inline void scores(f32x16& x, f32x16& y, const uint16_t* K, const uint16_t* V, Reader<D>& rd, int first) const {
    constexpr int kS = T::kSteps, kAhead = 2;
    bf16x8 a[kS], b[kS];
    rd.refresh();
    auto read = [&](int s) {
      a[s] = rd.rows(K, first, s);
      b[s] = rd.rows(V, first, s);
    };
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < kAhead; ++s) read(s);
    x = y = f32x16{};
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      if (s + kAhead < kS) read(s + kAhead);
      x = mfma(a[s], q[s], x);
      y = mfma(b[s], d_o[s], y);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // 32 keys that the whole block sees. Half of the exponentials stand between the MFMAs of the other half's sums.
  __device__ inline void whole(const uint16_t* K, const uint16_t* V, Reader<D>& rd, int first, float c) {
    constexpr int kN = 2 * T::kBlocks, kAhead = 2;
    f32x16 x, y;
    bf16x8 k[kN];
    scores(x, y, K, V, rd, first);
    auto read = [&](int n) { k[n] = rd.across(K, first + 16 * (n / T::kBlocks), n % T::kBlocks); };
#pragma unroll
    for (int n = 0; n < kAhead; ++n) read(n);
#pragma unroll
    for (int i = 0; i < 8; ++i) weight(x, y, i, c);
    bf16x8 ds = pack8(x, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      if (n == T::kBlocks) ds = pack8(x, 8);
      dq[n % T::kBlocks] = mfma(k[n], ds, dq[n % T::kBlocks]);
      if (n + kAhead < kN) read(n + kAhead);
      if (n < T::kBlocks) {
#pragma unroll
        for (int i = 8 + n * 8 / T::kBlocks; i < 8 + (n + 1) * 8 / T::kBlocks; ++i) weight(x, y, i, c);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // 32 keys from key0 on, of which a row sees those below its limit. GUARD: K may hold infinities and NaN.
  template <bool GUARD>
  __device__ inline void masked(const uint16_t* K, const uint16_t* V, Reader<D>& rd, int first, int key0, float c) {
    f32x16 x, y;
    scores(x, y, K, V, rd, first);
    const int left = limit - key0 - 4 * ((threadIdx.x >> 5) & 1);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      weight(x, y, i, c);
      x[i] = 8 * (i / 4) + i % 4 < left ? x[i] : 0.0f;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8 ds = pack8(x, 8 * t);
      if constexpr (GUARD) {
        add_guarded<true, D>(dq, K, rd, first + 16 * t, ds, seen_of(key0 + 16 * t, 0, limit));
      } else {
#pragma unroll
        for (int b = 0; b < T::kBlocks; ++b) dq[b] = mfma(rd.across(K, first + 16 * t, b), ds, dq[b]);
      }
    }
  }
};

// A block of 4 waves: 128 packed rows of one key head against all keys that they see.
template <int D>
__global__ __launch_bounds__(256, 2) void attention_dq_kernel(BwdArgs a) {
  using T = Tile<D>;
  constexpr int kTile = kKeys * D;
  extern __shared__ __attribute__((aligned(16))) uint16_t lds[];   // two slots of K and V
  __shared__ int flags[2];
  if (threadIdx.x < 2) flags[threadIdx.x] = 0;   // a barrier follows in any case
  const Shape& s = a.s;
  const int64_t id = block_number(a.first, a.per_xcd);
  const int head = int(id % s.kv_heads);
  Part p;
  if (!locate<true>(s, id / s.kv_heads, 128, s.group, p)) return;
  const int wave = wave_in_block(), lane = threadIdx.x & (kWave - 1);
  const int tile = s.causal ? p.tiles - 1 - p.tile : p.tile;   // the longest first
  const uint32_t rows = uint32_t(p.q_len) * uint32_t(s.group);
  const uint32_t row = uint32_t(tile) * 128 + wave * 32 + (lane & 31);
  const bool real = row < rows;
  uint32_t token, member;
  split_row(s, real ? row : 0, token, member);
  auto seen = [&](uint32_t r) {
    if (!s.causal) return p.k_len;
    const uint32_t last = r < rows ? r : rows - 1;
    const int n = int(last / uint32_t(s.group)) + 1 + p.k_len - p.q_len;
    return n < 0 ? 0 : n < p.k_len ? n : p.k_len;
  };
  Queries<D> w;
#pragma unroll
  for (int b = 0; b < T::kBlocks; ++b) w.dq[b] = f32x16{};
  w.limit = real ? seen(row) : 0;
  const int whole = uniform(seen(uint32_t(tile) * 128)) / kKeys;   // tiles that need no mask
  const int wave_max = uniform(seen(uint32_t(tile) * 128 + wave * 32 + 31));
  const int end = (uniform(seen(uint32_t(tile) * 128 + 127)) + kKeys - 1) / kKeys;

  const Loader<D, kKeys, 4> ld(wave, s.dim);
  Reader<D> rd;
  const uint32_t lds0 = lds_addr(lds);
  const uint32_t k_pitch = uint32_t(a.k.row * 2), v_pitch = uint32_t(a.v.row * 2);
  const uint64_t kb = reinterpret_cast<uint64_t>(a.k.p + p.k0 * a.k.row + head * a.k.head);
  const uint64_t vb = reinterpret_cast<uint64_t>(a.v.p + p.k0 * a.v.row + head * a.v.head);
  auto fetch = [&](int t, int slot) {
    const int left = p.k_len - t * kKeys;
    ld.load(kb + uint64_t(t) * kKeys * k_pitch, k_pitch, left, lds0 + slot * 4 * kTile);
    ld.load(vb + uint64_t(t) * kKeys * v_pitch, v_pitch, left, lds0 + slot * 4 * kTile + 2 * kTile);
  };
  if (end > 0) fetch(0, 0);

  const int64_t q_head = int64_t(head) * s.group + member, q_row = p.q0 + token;
  load_rows<D>(w.q, real ? a.q.p + q_row * a.q.row + q_head * a.q.head : nullptr, s.dim);
  load_rows<D>(w.d_o, real ? a.d_o.p + q_row * a.d_o.row + q_head * a.d_o.head : nullptr, s.dim);
  bf16x8 o[T::kSteps];
  load_rows<D>(o, real ? a.o.p + q_row * a.o.row + q_head * a.o.head : nullptr, s.dim);
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < T::kSteps; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(float(w.d_o[i][e]), float(o[i][e]), sum);
  w.share = column_sum(sum);
  // A row that sees one key has P = 1 and dS = 0: there D is formed as do v^T is, so that their difference is 0 and not
  // what two orders of the sum leave.
  if (__any(w.limit == 1)) {
    bf16x8 v[T::kSteps];
    load_rows<D>(v, reinterpret_cast<const uint16_t*>(vb), s.dim);
    f32x16 y = f32x16{};
#pragma unroll
    for (int i = 0; i < T::kSteps; ++i) y = mfma(v[i], w.d_o[i], y);
    if (w.limit == 1) w.share = y[0];
  }
  w.lse = real ? a.lse[q_row * s.heads + q_head] * kLog2e : 0.0f;
  if (real && lane < 32) {
    float* st = a.stats + ((int64_t(head) * s.q.rows + p.q0) * s.group + row) * 2;
    st[0] = w.lse;
    st[1] = w.share;
  }
  const float c = s.scale * kLog2e;
  int t = 0;
  auto next = [&]() {   // the tile in LDS
    wait_and_meet();
    if (t + 1 < end) fetch(t + 1, (t + 1) & 1);
    return lds + (t & 1) * 2 * kTile;
  };
  for (; t < end && t < whole; ++t) {
    const uint16_t* K = next();
#pragma unroll
    for (int f = 0; f < kKeys; f += 32) w.whole(K, K + kTile, rd, f, c);
  }
  const uint16_t* K = nullptr;
  bool odd = false;
  for (; t < end; ++t) {
    K = next();
    odd = tile_is_odd<D, kKeys>(K, flags, t & 1);
    if (odd) break;
#pragma unroll 1
    for (int f = 0; f < kKeys && t * kKeys + f < wave_max; f += 32) w.template masked<false>(K, K + kTile, rd, f, t * kKeys + f, c);
  }
  for (; t < end; ++t) {
    if (!odd) K = next();
    odd = false;
#pragma unroll 1
    for (int f = 0; f < kKeys && t * kKeys + f < wave_max; f += 32) w.template masked<true>(K, K + kTile, rd, f, t * kKeys + f, c);
  }
  wait_all();   // no load into LDS outlives the block
  const auto& e = late_args<BwdArgs>();
  const int64_t out_head = int64_t(head) * e.s.group + member, out_row = p.q0 + token;
  store_columns<D>(w.dq, e.s.scale, e.dq.p + out_row * e.dq.row + out_head * e.dq.head, real, e.s.dim);
}

template <int D>
struct Keys {
  using T = Tile<D>;
  bf16x8 k[T::kSteps];
  f32x16 dk[T::kBlocks], dv[T::kBlocks];
  int from, rows;   // packed rows from the first on see this lane's key; all of them

  // The lse and D of this lane's rows 2 i and 2 i + 1 (of its 16).
  static __device__ inline f32x4 stats_of(const float* stats, int i) {
    return *reinterpret_cast<const f32x4*>(stats + (8 * (i / 2) + 4 * ((threadIdx.x >> 5) & 1)) * 2 + 4 * (i % 2));
  }
  // From the scores of values 2 i and 2 i + 1 P and dS.
  static __device__ inline void weights(f32x16& x, f32x16& y, const f32x4& st, int i, float c) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float p = exp2_fast(__builtin_fmaf(x[2 * i + e], c, -st[2 * e]));
      y[2 * i + e] = p * (y[2 * i + e] - st[2 * e + 1]);
      x[2 * i + e] = p;
    }
  }
  // A tile of 32 packed rows that needs no mask. V: the block's values, this wave's from row `mine` on. The order is written out:
  // operands are read a few MFMAs ahead (left to itself the compiler reads each just before its MFMA and waits for
  // LDS every time), and half of the exponentials stand between the sums' MFMAs.
  __device__ inline void whole(const uint16_t* Q, const uint16_t* O, const uint16_t* V, int mine, const float* stats, Reader<D>& rd, float c) {
    constexpr int kS = T::kSteps, kB = T::kBlocks, kAhead = D <= 64 ? 1 : 2;
    bf16x8 a[kS], b[kS], d[kS], fo[2 * kB], fq[2 * kB];
    f32x4 st[8];
    f32x16 x = f32x16{}, y = f32x16{};
    rd.refresh();
    auto scores = [&](int s) {
      a[s] = rd.rows(Q, 0, s);
      b[s] = rd.rows(O, 0, s);
      d[s] = rd.rows(V, mine, s);
    };
    auto sums = [&](int i) {
      fo[i] = rd.across(O, 16 * (i / kB), i % kB);
      fq[i] = rd.across(Q, 16 * (i / kB), i % kB);
    };
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < kAhead; ++s) scores(s);
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      if (s + kAhead < kS) scores(s + kAhead);
      if (s + 2 >= kS) st[s + 2 - kS] = stats_of(stats, s + 2 - kS);
      x = mfma(a[s], k[s], x);
      y = mfma(b[s], d[s], y);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i + 2 < 5) st[i + 2] = stats_of(stats, i + 2);
      if (i >= 4 - kAhead) sums(i + kAhead - 4);
      weights(x, y, st[i], i, c);
      __builtin_amdgcn_sched_barrier(0);
    }
    bf16x8 p = pack8(x, 0), ds = pack8(y, 0);
#pragma unroll
    for (int i = 0; i < 2 * kB; ++i) {
      if (i == kB) {
        p = pack8(x, 8);
        ds = pack8(y, 8);
      }
      dv[i % kB] = mfma(fo[i], p, dv[i % kB]);
      if (i + kAhead < 2 * kB) sums(i + kAhead);
      if (i < kB) {
#pragma unroll
        for (int j = 4 + i * 4 / kB; j < 4 + (i + 1) * 4 / kB; ++j) {
          if (j + 1 < 8) st[j + 1] = stats_of(stats, j + 1);
          weights(x, y, st[j], j, c);
        }
      }
      dk[i % kB] = mfma(fq[i], ds, dk[i % kB]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // A tile that needs a mask; GUARD: q and do may hold infinities and NaN.
  template <bool GUARD>
  __device__ inline void masked(const uint16_t* Q, const uint16_t* O, const uint16_t* V, int mine, const float* stats, Reader<D>& rd, int row0, float c) {
    f32x16 x = f32x16{}, y = f32x16{};
    rd.refresh();
#pragma unroll
    for (int s = 0; s < T::kSteps; ++s) {
      x = mfma(rd.rows(Q, 0, s), k[s], x);
      y = mfma(rd.rows(O, 0, s), rd.rows(V, mine, s), y);
    }
    __builtin_amdgcn_sched_barrier(0);
    // rows behind the last one are zeros, of which a key with an infinity would make NaN
    const int skip = from - row0 - 4 * ((threadIdx.x >> 5) & 1);
    const uint32_t count = uint32_t(rows - from);
#pragma unroll
    for (int i = 0; i < 8; ++i) weights(x, y, stats_of(stats, i), i, c);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const bool sees = uint32_t(8 * (i / 4) + i % 4 - skip) < count;
      x[i] = sees ? x[i] : 0.0f;
      y[i] = sees ? y[i] : 0.0f;
    }
    const bf16x8 p[2] = {pack8(x, 0), pack8(x, 8)}, ds[2] = {pack8(y, 0), pack8(y, 8)};
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll 1
    for (int t = 0; t < 2; ++t) {
      const bf16x8 pt = t == 0 ? p[0] : p[1], dt = t == 0 ? ds[0] : ds[1];
      if constexpr (GUARD) {
        const bf16x8 see = seen_of(row0 + 16 * t, from, rows);
        add_guarded<false, D>(dv, O, rd, 16 * t, pt, see);
        add_guarded<true, D>(dk, Q, rd, 16 * t, dt, see);
      } else {
#pragma unroll
        for (int b = 0; b < T::kBlocks; ++b) {
          dv[b] = mfma(rd.across(O, 16 * t, b), pt, dv[b]);
          dk[b] = mfma(rd.across(Q, 16 * t, b), dt, dk[b]);
        }
      }
    }
  }
};

// The tiles of packed rows that see keys from key0 on, and the shares that they are split into.
struct RowTiles {
  int lowest, all, shares;
};
__device__ inline RowTiles row_tiles(const BwdArgs& a, const Part& p, int key0) {
  const int rows = p.q_len * a.s.group, off = p.k_len - p.q_len;
  RowTiles r;
  const bool any = key0 < p.k_len;   // keys in use
  r.lowest = a.s.causal && any && key0 > off ? (key0 - off) * a.s.group / kRows : 0;
  r.all = any && r.lowest * kRows < rows ? (rows + kRows - 1) / kRows - r.lowest : 0;
  const int want = (r.all + a.share - 1) / a.share;
  r.shares = want < 1 ? 1 : want < a.shares ? want : a.shares;
  return r;
}

// A block of 4 waves: 128 keys of one head, 32 to a wave, against all (or a share of) the packed rows that see them, from the last
// row on: so blocks that run at once read the same rows at the same time.
template <int D>
__global__ __launch_bounds__(256, D <= 64 ? 3 : 2) void attention_dkv_kernel(BwdArgs a) {
  using T = Tile<D>;
  constexpr int kTile = kRows * D;
  extern __shared__ __attribute__((aligned(16))) uint16_t lds[];   // two slots of Q and dO, V, two slots of the rows' values
  constexpr int kV = 4 * kTile;   // elements in front of V
  const uint16_t* V = lds + kV;
  float* stats = reinterpret_cast<float*>(lds + kV + 128 * D);
  const Shape& s = a.s;
  const int64_t id = block_number(a.first, a.per_xcd);
  const int head = int(id % s.kv_heads);
  const int64_t rest = id / s.kv_heads;
  const int part = int(rest % a.shares);
  Part p;
  if (!locate<false>(s, rest / a.shares, 128, 1, p)) return;
  const int wave = wave_in_block(), lane = threadIdx.x & (kWave - 1);
  const int key_b = p.tile * 128, key_w = key_b + wave * 32;
  const int rows = p.q_len * s.group, off = p.k_len - p.q_len;
  // that sees key j; rows of a tile behind the last key stand at it, since times the group's heads they may pass 32 bits
  auto first_row = [&](int j) {
    const int n = (j < p.k_len ? j : p.k_len - 1) - off;
    return s.causal && n > 0 ? n * s.group : 0;
  };
  Keys<D> w;
#pragma unroll
  for (int b = 0; b < T::kBlocks; ++b) w.dk[b] = w.dv[b] = f32x16{};
  {
    const int key = key_w + (lane & 31);
    load_rows<D>(w.k, key < p.k_len ? a.k.p + (p.k0 + key) * a.k.row + head * a.k.head : nullptr, s.dim);
  }
  const RowTiles rt = row_tiles(a, p, key_b);
  if (part >= rt.shares) return;
  const int each = (rt.all + rt.shares - 1) / rt.shares;
  const int begin = uniform(rt.lowest + part * each);
  const int end = uniform(rt.lowest + (part * each + each < rt.all ? part * each + each : rt.all));
  int masked = uniform((first_row(key_b + 127) + kRows - 1) / kRows);   // tiles from it on need no mask

  const Loader<D, kRows, 4> ld(wave, s.dim);
  Reader<D> rd;
  const uint32_t lds0 = lds_addr(lds);
  const int64_t q_head0 = int64_t(head) * s.group;
  const uint64_t qb = reinterpret_cast<uint64_t>(a.q.p + p.q0 * a.q.row + q_head0 * a.q.head);
  const uint64_t ob = reinterpret_cast<uint64_t>(a.d_o.p + p.q0 * a.d_o.row + q_head0 * a.d_o.head);
  const uint64_t sb = reinterpret_cast<uint64_t>(a.stats + (int64_t(head) * s.q.rows + p.q0) * s.group * 2);
  // Where a tile is whole tokens the offsets within it are those of every tile.
  const bool whole_tokens = kRows % s.group == 0;
  const uint32_t q_pitch = uint32_t(a.q.row * 2), q_step = uint32_t(a.q.head * 2), o_pitch = uint32_t(a.d_o.row * 2), o_step = uint32_t(a.d_o.head * 2);
  uint32_t q_off[decltype(ld)::kLoads], o_off[decltype(ld)::kLoads];
  ld.packed(s, q_pitch, q_step, 0, q_off);
  ld.packed(s, o_pitch, o_step, 0, o_off);
  auto fetch = [&](int t, int slot) {
    const uint32_t row0 = uint32_t(t) * kRows;
    if (!whole_tokens) {
      ld.packed(s, q_pitch, q_step, row0, q_off);
      ld.packed(s, o_pitch, o_step, row0, o_off);
    }
    const uint64_t token = uint64_t(row0 / uint32_t(s.group));
    ld.load_at(qb + token * q_pitch, q_off, rows - int(row0), lds0 + slot * 4 * kTile);
    ld.load_at(ob + token * o_pitch, o_off, rows - int(row0), lds0 + slot * 4 * kTile + 2 * kTile);
    if (wave == 0)
      load_lds4_asm(rsrc_words(sb + uint64_t(row0) * 8, kAllRecords), lds0 + 2 * kV + 256 * D + slot * kRows * 8,
                    int(row0) + lane / 2 < rows ? uint32_t(lane) * 4 : kOutOfRange);
  };
  const float c = s.scale * kLog2e;
  int t = end - 1;
  if (begin < end) {
    const Loader<D, 128, 4> lv(wave, s.dim);
    lv.load(reinterpret_cast<uint64_t>(a.v.p + (p.k0 + key_b) * a.v.row + head * a.v.head), uint32_t(a.v.row * 2), p.k_len - key_b,
            lds0 + 2 * kV);
    fetch(t, t & 1);
  }
  auto next = [&]() {   // tile t has landed
    wait_and_meet();
    if (t > begin) fetch(t - 1, (t - 1) & 1);
  };
  auto q_of = [&]() { return lds + (t & 1) * 2 * kTile; };
  auto st_of = [&]() { return stats + (t & 1) * kRows * 2; };
  // Nor do rows behind the last one, zeros that weigh exp(0) and add 0: but where one of the wave's keys holds an infinity they
  // would weigh NaN.
  if (rows % kRows != 0 && any_odd(w.k)) masked = 0x7fffffff;
  for (; t >= begin && t >= masked; --t) {
    next();
    w.whole(q_of(), q_of() + kTile, V, wave * 32, st_of(), rd, c);
  }
  // This lane's key: formed again behind the loop, which has no register for it.
  const int key = key_w + (lane_again() & 31);
  const bool used = key < p.k_len;
  w.from = first_row(key);
  w.rows = rows;
  // A row of q or do that holds an infinity or NaN has such an lse or D (so has one that sees no key): where no row
  // of a tile has, unseen rows' zeros as factors are all that a mask takes.
  bool odd = false;
  for (; t >= begin; --t) {
    next();
    odd = __any((__float_as_uint(st_of()[lane_again()]) & 0x7f800000u) == 0x7f800000u);
    if (odd) break;
    w.template masked<false>(q_of(), q_of() + kTile, V, wave * 32, st_of(), rd, t * kRows, c);
  }
  for (; t >= begin; --t) {
    if (!odd) next();
    odd = false;
    w.template masked<true>(q_of(), q_of() + kTile, V, wave * 32, st_of(), rd, t * kRows, c);
  }
  wait_all();   // no load into LDS outlives the block
  const auto& e = late_args<BwdArgs>();
  // keys that are not in use get zeros where the rows of no sequence do
  const bool real = key < (e.s.fill ? p.k_slot : p.k_len);
  if (rt.shares > 1) {
    if (key >= p.k_len) return;   // the sum takes them as zeros
    const int64_t size = e.s.k.rows * e.s.kv_heads * e.s.dim;
    float* to = e.part + int64_t(part) * 2 * size + ((p.k0 + key) * e.s.kv_heads + head) * e.s.dim;
    const int h = lane_again() >> 5;
#pragma unroll
    for (int b = 0; b < T::kBlocks; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int col = 32 * b + 8 * g + 4 * h;
        if (col >= e.s.dim) continue;
        *reinterpret_cast<f32x4*>(to + col) = f32x4{w.dk[b][4 * g], w.dk[b][4 * g + 1], w.dk[b][4 * g + 2], w.dk[b][4 * g + 3]};
        *reinterpret_cast<f32x4*>(to + size + col) = f32x4{w.dv[b][4 * g], w.dv[b][4 * g + 1], w.dv[b][4 * g + 2], w.dv[b][4 * g + 3]};
      }
    return;
  }
  // zeros, not a factor of 0: a key of zeros weighs exp(-lse), which may be infinite or NaN
  const uint32_t keep = used ? ~0u : 0u;
  store_columns<D>(w.dk, e.s.scale, e.dk.p + (p.k0 + key) * e.dk.row + head * e.dk.head, real, e.s.dim, keep);
  store_columns<D>(w.dv, 1.0f, e.dv.p + (p.k0 + key) * e.dv.row + head * e.dv.head, real, e.s.dim, keep);
}

// The shares' sums of dk and dv, in order: a block per tile of 128 keys, head and quarter of its values, which it reads all at once.
constexpr int kJoinParts = 4;
__global__ __launch_bounds__(256) void attention_dkv_join_kernel(BwdArgs a) {
  const Shape& s = a.s;
  const int64_t id = a.first + blockIdx.x, rest = id / kJoinParts;
  const int quarter = int(id % kJoinParts), head = int(rest % s.kv_heads);
  Part p;
  if (!locate<false>(s, rest / s.kv_heads, 128, 1, p)) return;
  const int shares = row_tiles(a, p, p.tile * 128).shares;
  if (shares == 1) return;
  const int64_t size = s.k.rows * s.kv_heads * s.dim;
  const int pieces = s.dim / 4, last = s.fill ? p.k_slot : p.k_len;
  constexpr int kEach = 128 * (kAttentionDim / 4) / kJoinParts / 256;
  f32x4 dk[kEach], dv[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int i = (quarter * kEach + j) * 256 + int(threadIdx.x);
    const int key = p.tile * 128 + i / pieces, col = i % pieces * 4;
    dk[j] = dv[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (i >= 128 * pieces || key >= p.k_len) continue;
    const float* from = a.part + ((p.k0 + key) * s.kv_heads + head) * s.dim + col;
    for (int n = 0; n < shares; ++n) {
      dk[j] += *reinterpret_cast<const f32x4*>(from + 2 * n * size);
      dv[j] += *reinterpret_cast<const f32x4*>(from + (2 * n + 1) * size);
    }
  }
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int i = (quarter * kEach + j) * 256 + int(threadIdx.x);
    const int key = p.tile * 128 + i / pieces, col = i % pieces * 4;
    if (i >= 128 * pieces || key >= last) continue;
    const u32x2 wk = {pack_bf16x2(dk[j][0] * s.scale, dk[j][1] * s.scale), pack_bf16x2(dk[j][2] * s.scale, dk[j][3] * s.scale)};
    const u32x2 wv = {pack_bf16x2(dv[j][0], dv[j][1]), pack_bf16x2(dv[j][2], dv[j][3])};
    *reinterpret_cast<u32x2*>(a.dk.p + (p.k0 + key) * a.dk.row + head * a.dk.head + col) = wk;
    *reinterpret_cast<u32x2*>(a.dv.p + (p.k0 + key) * a.dv.row + head * a.dv.head + col) = wv;
  }
}

// How the packed rows that see a key tile are shared out, where the key tiles give too few blocks for the places on the device:
// fewer than 2 to a place for sequences of different lengths, 5 to 4 places where causal tiles of one length even each other out,
// fewer than places else. A share has half the tiles that a place would have on average, if all sequences were of one length; at
// most as many shares as fill the places, but 2 where the tiles nearly do, their sums at most 256 MiB. A longer sequence among
// short ones is split by the kernel, which knows the lengths, but where the average is a quarter of a share or less. Backward, us, causal unless said: 4096 tokens of 8 heads on 1 230 (one share
// 1276, 2 707, 32 248); 16384 tokens of the same 2150 (64 shares 1948); 1024 tokens of 32 on 8 86 (16 shares 106); 8192 tokens of 8 on 8 (512
// blocks) 560 (one share 597), not causal 866 in one (907 in 2), 12288 tokens (768) 1041 in one (1094); 16384 of 32 on 8 (1024): dk and dv 3926 in
// one (4757: shares read different rows). Packed sequences of 1 to 2048, 32 on 8 (552): 473 (one share 528, 4 560), of 1 to 4048 (800) 1110 (1220).
static void row_shares(const AttentionPlan& a, int cus, int& shares, int& share) {
  const Shape s = shape_of(a);
  const int64_t places = 2 * cus, tiles = tiles_of(s.k, a.batch, false, 1, 128), blocks = tiles * a.kv_heads;
  // row tiles that a key can have: a sequence's, or all where only the device knows the lengths
  const int64_t rows = ((a.q_starts ? a.q_rows : a.q_rows / a.batch) * s.group + kRows - 1) / kRows;
  const int64_t average = (a.q_rows / a.batch * s.group + kRows - 1) / kRows, bytes = a.k_rows * a.kv_heads * a.dim * 8;
  shares = share = 1;
  if (blocks == 0 || bytes == 0 || rows == 0) return;
  share = int(std::max<int64_t>(8, tiles * average * a.kv_heads / (a.causal ? 4 : 2) / places));
  const int64_t enough = a.q_starts || a.k_starts ? 2 * places : a.causal ? places * 5 / 4 : places;
  if (blocks >= enough || (a.q_starts && 4 * average <= share)) return;
  const int64_t most = std::max<int64_t>(2, places / blocks);
  shares = int(std::max<int64_t>(1, std::min<int64_t>({most, (rows + share - 1) / share, (int64_t(256) << 20) / bytes})));
}

template <int D>
hipError_t launch_bwd(const BwdArgs& f, int dev, hipStream_t st) {
  static std::atomic<uint64_t> done_q{0}, done_kv{0};
  constexpr int kBytesQ = 4 * kKeys * D * 2, kBytesKv = (4 * kRows + 128) * D * 2 + 2 * kRows * 8;
  hipError_t e = allow_lds(reinterpret_cast<const void*>(attention_dq_kernel<D>), kBytesQ, dev, done_q);
  if (e == hipSuccess) e = allow_lds(reinterpret_cast<const void*>(attention_dkv_kernel<D>), kBytesKv, dev, done_kv);
  if (e != hipSuccess) return e;
  BwdArgs g = f;
  e = in_parts(tiles_of(f.s.q, f.s.batch, f.s.fill, f.s.group, 128) * f.s.kv_heads, most_blocks(256), [&](int64_t first, int64_t count) {
    g.first = first;
    g.per_xcd = blocks_per_xcd(g.s, count);
    attention_dq_kernel<D><<<uint32_t(count), 256, kBytesQ, st>>>(g);
  });
  if (e != hipSuccess) return e;
  const int64_t tiles = tiles_of(f.s.k, f.s.batch, f.s.fill, 1, 128) * f.s.kv_heads;
  e = in_parts(tiles * f.shares, most_blocks(256), [&](int64_t first, int64_t count) {
    g.first = first;
    g.per_xcd = blocks_per_xcd(g.s, count);
    attention_dkv_kernel<D><<<uint32_t(count), 256, kBytesKv, st>>>(g);
  });
  if (e != hipSuccess || f.shares == 1) return e;
  return in_parts(tiles * kJoinParts, most_blocks(256), [&](int64_t first, int64_t count) {
    g.first = first;
    attention_dkv_join_kernel<<<uint32_t(count), 256, 0, st>>>(g);
  });
}

}  // namespace attn

namespace {
size_t stats_bytes(const AttentionPlan& a) { return (size_t(a.q_rows) * size_t(a.heads) * 8 + 15) / 16 * 16; }
}  // namespace

size_t attention_bwd_workspace(const AttentionPlan& a) {
  int dev = 0, cus = 256;
  if (current_device(dev, cus) != hipSuccess) cus = 256;
  int shares, share;
  attn::row_shares(a, cus, shares, share);
  return stats_bytes(a) + (shares > 1 ? size_t(shares) * size_t(a.k_rows) * size_t(a.kv_heads) * size_t(a.dim) * 8 : 0);
}

hipError_t launch_attention_bwd(const AttentionPlan& a, const HeadsView& d_o, const HeadsView& q, const HeadsView& k, const HeadsView& v,
                                const HeadsView& o, const float* lse, const HeadsView& dq, const HeadsView& dk, const HeadsView& dv,
                                void* workspace, hipStream_t st) {
  int dev, cus;
  const hipError_t e = current_device(dev, cus);
  if (e != hipSuccess) return e;
  attn::BwdArgs f{};
  f.s = attn::shape_of(a);
  f.q = attn::heads_of(q);
  f.k = attn::heads_of(k);
  f.v = attn::heads_of(v);
  f.o = attn::heads_of(o);
  f.d_o = attn::heads_of(d_o);
  f.dq = attn::heads_of(dq);
  f.dk = attn::heads_of(dk);
  f.dv = attn::heads_of(dv);
  f.lse = lse;
  f.stats = static_cast<float*>(workspace);
  f.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + stats_bytes(a));
  attn::row_shares(a, cus, f.shares, f.share);
  return a.dim <= 64 ? attn::launch_bwd<64>(f, dev, st) : attn::launch_bwd<128>(f, dev, st);
}

}  // namespace lmbp
