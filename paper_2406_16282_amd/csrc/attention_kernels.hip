// Attention forward for gfx950: o = softmax(scale q k^T) v over the keys that each query sees, and the
// logarithm of each row's sum, in one pass over the keys with a running maximum and sum.
//
// Two products of 64 keys' tiles with an exponential between them: the matrix units bound it for long rows, memory for few.
// P is rounded to bf16 once, as the second product's operand; the sum takes it unrounded. A block has 128 packed rows (the heads that
// share a key head side by side, so that K and V are read once for them), 32 to a wave, two blocks to a CU: 16384 tokens of 32 heads on 8,
// dim 128, causal, 2.09 ms (1053 TFLOP/s; matrix units 52% of the cycles at the power limit's 1.9 GHz; no LDS conflicts), 2.24 with the
// LDS reads where the compiler puts them. 4 sequences of 2048, 32 heads: 183 us. What did not help: a third slot of tiles for narrow
// heads (31.0 us for 30.4 at 64 images), keys asked into L2 ahead of their turn (4 to 7% slower).
#include "attention_device.hpp"

#include <algorithm>
#include <type_traits>

namespace lmbp {
namespace attn {

struct FwdArgs {
  Shape s;
  Heads q, k, v, o;
  float* lse;        // [rows][heads]
  float* part;       // splits > 1: [splits][rows * heads][dim], unnormalised
  float* stats;      // splits > 1: [splits][rows * heads][2]: running maximum (log2), sum; kNoKeys where the row sees none of the share
  int splits;
  int64_t first;     // block number of this launch's first block
  uint32_t per_xcd;
};

constexpr int kKeys = 64;      // keys to a tile
// A row's running maximum may stay this much (log2) behind its largest score, so that sums are seldom rescaled: exponentials up to 2^8
// lose nothing in fp32 or bf16. 16384 tokens 2064 us, without 2156.
constexpr float kSlack = 8.0f;

constexpr float kNoKeys = -1.0f;   // no sum: one of 0 has keys whose scores are all -inf

// One wave's 32 rows over keys in LDS.
template <int D>
struct Rows {
  using T = Tile<D>;
  bf16x8 q[T::kSteps];
  f32x16 o[T::kBlocks];
  float top, sum;   // running maximum of the scaled scores in log2, this lane's part of the sum
  int limit;        // keys below it are seen by this lane's row

  __device__ inline void clear() {
#pragma unroll
    for (int b = 0; b < T::kBlocks; ++b) o[b] = f32x16{};
    top = kLowest;
    sum = 0.0f;
  }

  // Scores of 32 kB keys, the tile's from `first` on: a lane has its row's, 16 of each 32 keys. Operands are read two steps
  // ahead: left to itself the compiler reads each just before its MFMA and waits for LDS every time.
  template <int kB>
  __device__ inline void scores(f32x16 (&x)[kB], const uint16_t* K, const Reader<D>& rd, int first) const {
    constexpr int kS = T::kSteps, kAhead = 2;
    bf16x8 k[kS][kB];
    auto read = [&](int s) {
#pragma unroll
      for (int b = 0; b < kB; ++b) k[s][b] = rd.rows(K, first + 32 * b, s);
    };
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < kAhead; ++s) read(s);
#pragma unroll
    for (int b = 0; b < kB; ++b) x[b] = f32x16{};
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      if (s + kAhead < kS) read(s + kAhead);
#pragma unroll
      for (int b = 0; b < kB; ++b) x[b] = mfma(k[s][b], q[s], x[b]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // The running maximum behind these scores.
  template <int kB>
  __device__ inline void follow(const f32x16 (&x)[kB], float c) {
    float most = x[0][0];
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) most = fmaxf(most, x[b][i]);
    most = column_max(most) * c;
    const bool behind = most > top + kSlack;   // each row by itself: its results do not depend on its neighbours'
    if (__any(behind)) {
      const float now = behind ? most : top, f = exp2_fast(top - now);
      top = now;
      sum *= f;
#pragma unroll
      for (int b = 0; b < T::kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] *= f;
    }
  }
  __device__ inline void weight(f32x16& x, int i, float c) {
    const float p = exp2_fast(__builtin_fmaf(x[i], c, -top));
    sum += p;
    x[i] = p;
  }
  // 32 kB keys that the whole block sees. Half of the exponentials stand between the MFMAs of the other half's sums.
  template <int kB>
  __device__ inline void whole(const uint16_t* K, const uint16_t* V, const Reader<D>& rd, float c) {
    constexpr int kN = 2 * kB * T::kBlocks, kAhead = 3;   // MFMAs of the sums
    constexpr int kFirst = 8 * kB;                          // exponentials in front of them
    f32x16 x[kB];
    bf16x8 v[kN];
    scores<kB>(x, K, rd, 0);
    follow<kB>(x, c);
    auto read = [&](int n) { v[n] = rd.across(V, 16 * (n / T::kBlocks), n % T::kBlocks); };
#pragma unroll
    for (int n = 0; n < kAhead; ++n) read(n);
#pragma unroll
    for (int i = 0; i < kFirst; ++i) weight(x[i / 16], i % 16, c);
    bf16x8 p = pack8(x[0], 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      const int t = n / T::kBlocks;
      if (n % T::kBlocks == 0 && n > 0) p = pack8(x[t / 2], 8 * (t % 2));
      o[n % T::kBlocks] = mfma(v[n], p, o[n % T::kBlocks]);
      if (n + kAhead < kN) read(n + kAhead);
      if (n < kN / 2) {
#pragma unroll
        for (int i = kFirst + n * kFirst * 2 / kN; i < kFirst + (n + 1) * kFirst * 2 / kN; ++i) weight(x[i / 16], i % 16, c);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // 32 keys from key0 on, the tile's from `first` on, of which a row sees those below its limit. GUARD: V may hold
  // infinities and NaN.
  template <bool GUARD>
  __device__ inline void masked(const uint16_t* K, const uint16_t* V, const Reader<D>& rd, int first, int key0, float c) {
    f32x16 x[1];
    scores<1>(x, K, rd, first);
    const int left = limit - key0 - 4 * ((threadIdx.x >> 5) & 1);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (8 * (i / 4) + i % 4 >= left) x[0][i] = -__builtin_inff();
    follow<1>(x, c);
#pragma unroll
    for (int i = 0; i < 16; ++i) weight(x[0], i, c);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8 p = pack8(x[0], 8 * t);
      if constexpr (GUARD) {
        add_guarded<false>(o, V, rd, first + 16 * t, p, seen_of(key0 + 16 * t, 0, limit));
      } else {
#pragma unroll
        for (int b = 0; b < T::kBlocks; ++b) o[b] = mfma(rd.across(V, first + 16 * t, b), p, o[b]);
      }
    }
  }
};

// A block of 4 waves: 128 packed rows of one key head, 32 to a wave, against all (or a share of) the keys that they see.
template <int D>
__global__ __launch_bounds__(256, 2) void attention_fwd_kernel(FwdArgs a) {
  using T = Tile<D>;
  constexpr int kTile = kKeys * D;   // elements
  extern __shared__ __attribute__((aligned(16))) uint16_t lds[];   // two slots of K and V
  __shared__ int flags[2];
  if (threadIdx.x < 2) flags[threadIdx.x] = 0;   // a barrier follows in any case
  const Shape& s = a.s;
  const int64_t id = block_number(a.first, a.per_xcd);
  const int head = int(id % s.kv_heads);
  const int64_t rest = id / s.kv_heads;
  const int split = int(rest % a.splits);
  Part p;
  if (!locate<true>(s, rest / a.splits, 128, s.group, p)) return;
  const int wave = wave_in_block(), lane = threadIdx.x & (kWave - 1);
  const int tile = s.causal ? p.tiles - 1 - p.tile : p.tile;   // the longest first
  const uint32_t rows = uint32_t(p.q_len) * uint32_t(s.group);
  const uint32_t row = uint32_t(tile) * 128 + wave * 32 + (lane & 31);
  const bool real = row < rows;
  uint32_t token, member;
  split_row(s, real ? row : 0, token, member);

  // keys seen by a row: this lane's, the block's first (whole tiles need no mask) and last
  auto seen = [&](uint32_t r) {
    if (!s.causal) return p.k_len;
    const uint32_t last = r < rows ? r : rows - 1;
    const int n = int(last / uint32_t(s.group)) + 1 + p.k_len - p.q_len;
    return n < 0 ? 0 : n < p.k_len ? n : p.k_len;
  };
  Rows<D> w;
  w.clear();
  w.limit = real ? seen(row) : 0;
  const int all = (uniform(seen(uint32_t(tile) * 128 + 127)) + kKeys - 1) / kKeys;
  const int share = (all + a.splits - 1) / a.splits;
  const int begin = split * share, end = begin + share < all ? begin + share : all;
  const int whole = uniform(seen(uint32_t(tile) * 128)) / kKeys;
  const int wave_max = uniform(seen(uint32_t(tile) * 128 + wave * 32 + 31));

  const int64_t q_head = int64_t(head) * s.group + member;
  load_rows<D>(w.q, real ? a.q.p + (p.q0 + token) * a.q.row + q_head * a.q.head : nullptr, s.dim);

  const Loader<D, kKeys, 4> ld(wave, s.dim);
  const Reader<D> rd;
  const uint32_t lds0 = lds_addr(lds);
  const uint32_t k_pitch = uint32_t(a.k.row * 2), v_pitch = uint32_t(a.v.row * 2);
  const uint64_t kb = reinterpret_cast<uint64_t>(a.k.p + p.k0 * a.k.row + head * a.k.head);
  const uint64_t vb = reinterpret_cast<uint64_t>(a.v.p + p.k0 * a.v.row + head * a.v.head);
  auto fetch = [&](int t, int slot) {
    const int left = p.k_len - t * kKeys;
    ld.load(kb + uint64_t(t) * kKeys * k_pitch, k_pitch, left, lds0 + slot * 4 * kTile);
    ld.load(vb + uint64_t(t) * kKeys * v_pitch, v_pitch, left, lds0 + slot * 4 * kTile + 2 * kTile);
  };
  const float c = s.scale * kLog2e;
  if (begin < end) fetch(begin, begin & 1);
  int t = begin;
  auto next = [&]() {   // tile t has landed
    wait_and_meet();
    if (t + 1 < end) fetch(t + 1, (t + 1) & 1);
  };
  auto k_of = [&]() { return lds + (t & 1) * 2 * kTile; };
  for (const int last = whole < end ? whole : end; t < last; ++t) {
    next();
    w.template whole<kKeys / 32>(k_of(), k_of() + kTile, rd, c);
  }
  auto masked = [&](auto guard) {
#pragma unroll 1
    for (int f = 0; f < kKeys && t * kKeys + f < wave_max; f += 32)
      w.template masked<decltype(guard)::value>(k_of(), k_of() + kTile, rd, f, t * kKeys + f, c);
  };
  bool odd = false;
  for (; t < end; ++t) {
    next();
    odd = tile_is_odd<D, kKeys>(k_of() + kTile, flags, t & 1);
    if (odd) break;
    masked(std::false_type{});
  }
  for (; t < end; ++t) {
    if (!odd) next();
    odd = false;
    masked(std::true_type{});
  }
  wait_all();   // no load into LDS outlives the block
  const auto& e = late_args<FwdArgs>();
  const float sum = column_sum(w.sum);
  const int64_t o_head = int64_t(head) * e.s.group + member, out_row = (p.q0 + token) * e.s.heads + o_head;
  if (e.splits > 1 && p.b < e.s.batch) {
    if (!real) return;
    float* to = e.part + (int64_t(split) * e.s.q.rows * e.s.heads + out_row) * e.s.dim;
    const int h = lane >> 5;
    if (begin < end) {
#pragma unroll
      for (int b = 0; b < T::kBlocks; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int col = 32 * b + 8 * g + 4 * h;
          if (col < e.s.dim) *reinterpret_cast<f32x4*>(to + col) = f32x4{w.o[b][4 * g], w.o[b][4 * g + 1], w.o[b][4 * g + 2], w.o[b][4 * g + 3]};
        }
    }
    if (h == 0) {
      float* st = e.stats + (int64_t(split) * e.s.q.rows * e.s.heads + out_row) * 2;
      st[0] = w.top;
      st[1] = begin < end && begin * kKeys < w.limit ? sum : kNoKeys;
    }
    return;
  }
  if (split > 0) return;
  uint16_t* o = e.o.p + (p.q0 + token) * e.o.row + o_head * e.o.head;
  store_columns<D>(w.o, w.limit > 0 ? 1.0f / sum : 0.0f, o, real, e.s.dim);
  if (real && lane < 32) e.lse[out_row] = w.limit > 0 ? (w.top + __builtin_amdgcn_logf(sum)) * kLn2 : -__builtin_inff();
}

// Few rows, many keys: a block of kFewWaves waves has 32 packed rows and a share of their keys; each wave walks keys of its own
// through two slots of its own, with no barrier, and the block's waves join at the end. Memory is what it waits
// for: 16 KB to a wave are on their way while 16 KB are multiplied, 64 KB to a CU. The kernel alone: 16 sequences of 1 to 4096 keys, 32 heads:
// 90 us (5.1 TB/s); one of 65537 keys, 8 key heads: 50 (5.4), with one wave to a block 62, with four 54.
constexpr int kFewWaves = 2, kFewTiles = 4;   // at least so many tiles of keys to a wave, where rows' keys are shared out
template <int D>
constexpr int kFewKeys = 4096 / D;   // keys to a wave's tile: 8 KB of K, 8 of V
template <int D>
constexpr int kFewLds = kFewWaves * 32768;

template <int D>
__global__ __launch_bounds__(kFewWaves * 64) void attention_few_kernel(FwdArgs a) {
  constexpr int kT = kFewKeys<D>, kTile = kT * D;
  constexpr int kPitch = D + 4;   // floats from row to row of a wave's sums: 16 rows on distinct banks
  extern __shared__ __attribute__((aligned(16))) uint16_t lds[];
  __shared__ float tops[kFewWaves][32], sums[kFewWaves][32], norm[32];
  const Shape& s = a.s;
  const int64_t id = a.first + blockIdx.x;
  const int head = int(id % s.kv_heads);
  const int64_t rest = id / s.kv_heads;
  const int split = int(rest % a.splits);
  Part p;
  if (!locate<true>(s, rest / a.splits, 32, s.group, p)) return;
  const int wave = wave_in_block(), lane = threadIdx.x & (kWave - 1), h = lane >> 5, in = lane & 31;
  const uint32_t rows = uint32_t(p.q_len) * uint32_t(s.group), row0 = uint32_t(p.tile) * 32;
  const bool real = row0 + in < rows;
  uint32_t token, member;
  split_row(s, real ? row0 + in : 0, token, member);
  auto seen = [&](uint32_t r) {
    if (!s.causal) return p.k_len;
    const uint32_t last = r < rows ? r : rows - 1;
    const int n = int(last / uint32_t(s.group)) + 1 + p.k_len - p.q_len;
    return n < 0 ? 0 : n < p.k_len ? n : p.k_len;
  };
  Rows<D> w;
  w.clear();
  w.limit = real ? seen(row0 + in) : 0;
  const int most = uniform(seen(row0 + 31));
  const int all = (most + kT - 1) / kT, whole = uniform(seen(row0)) / kT;
  const int even = (all + a.splits - 1) / a.splits, share = even > kFewTiles * kFewWaves ? even : kFewTiles * kFewWaves;
  const int begin = split * share, end = begin + share < all ? begin + share : all;
  const Loader<D, kT, 1> ld(0, s.dim);
  const Reader<D> rd;
  uint16_t* mine = lds + wave * 16384;
  const uint32_t at = lds_addr(mine), k_pitch = uint32_t(a.k.row * 2), v_pitch = uint32_t(a.v.row * 2);
  const uint64_t kb = reinterpret_cast<uint64_t>(a.k.p + p.k0 * a.k.row + head * a.k.head);
  const uint64_t vb = reinterpret_cast<uint64_t>(a.v.p + p.k0 * a.v.row + head * a.v.head);
  auto fetch = [&](int t, int slot) {   // past the share: zeros, so that the count of loads on their way stays the same
    const int left = t < end ? p.k_len - t * kT : 0;
    const int64_t from = t < end ? int64_t(t) * kT : 0;
    ld.load(kb + uint64_t(from) * k_pitch, k_pitch, left, at + slot * 16384);
    ld.load(vb + uint64_t(from) * v_pitch, v_pitch, left, at + slot * 16384 + 8192);
  };
  const float c = s.scale * kLog2e;
  const int64_t q_head = int64_t(head) * s.group + member;
  if (begin < end) {
    load_rows<D>(w.q, real ? a.q.p + (p.q0 + token) * a.q.row + q_head * a.q.head : nullptr, s.dim);
    int t = begin + wave, slot = 0;
    fetch(t, 0);
    auto next = [&]() {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot to be filled has been read
      fetch(t + kFewWaves, slot ^ 1);
      asm volatile("s_waitcnt vmcnt(16)" ::: "memory");    // all but those loads have landed
      const uint16_t* K = mine + slot * 8192;
      slot ^= 1;
      return K;
    };
    for (; t < end && t < whole; t += kFewWaves) {
      const uint16_t* K = next();
      w.template whole<kT / 32>(K, K + kTile, rd, c);
    }
    for (; t < end; t += kFewWaves) {
      const uint16_t* K = next();
#pragma unroll 1
      for (int f = 0; f < kT && t * kT + f < most; f += 32) w.template masked<true>(K, K + kTile, rd, f, t * kT + f, c);
    }
  }
  wait_all();
  w.sum = column_sum(w.sum);
  if (h == 0) {
    tops[wave][in] = w.top;
    sums[wave][in] = w.sum;
  }
  __syncthreads();
  float top = kLowest, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kFewWaves; ++i) top = fmaxf(top, tops[i][in]);
#pragma unroll
  for (int i = 0; i < kFewWaves; ++i) sum = __builtin_fmaf(sums[i][in], exp2_fast(tops[i][in] - top), sum);
  const float f = exp2_fast(w.top - top);
  float* part = reinterpret_cast<float*>(lds);
  static_assert(kFewWaves * 32 * kPitch * 4 <= kFewLds<D>, "the sums fit");
  float* own = part + (wave * 32 + in) * kPitch;
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4*>(own + 32 * b + 8 * g + 4 * h) =
          f32x4{w.o[b][4 * g] * f, w.o[b][4 * g + 1] * f, w.o[b][4 * g + 2] * f, w.o[b][4 * g + 3] * f};
  const auto& e = late_args<FwdArgs>();
  const int64_t o_head = int64_t(head) * e.s.group + member, out_row = (p.q0 + token) * e.s.heads + o_head;
  const bool joined = e.splits > 1 && p.b < e.s.batch;   // by the next kernel
  if (!joined && split > 0) return;
  if (real && wave == 0 && h == 0) {
    if (joined) {
      float* st = e.stats + (int64_t(split) * e.s.q.rows * e.s.heads + out_row) * 2;
      st[0] = top;
      st[1] = begin < end && begin * kT < w.limit ? sum : kNoKeys;
    } else {
      e.lse[out_row] = w.limit > 0 ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -__builtin_inff();
      norm[in] = w.limit > 0 ? 1.0f / sum : 0.0f;
    }
  }
  __syncthreads();
  if (joined && begin >= end) return;
  for (int i = threadIdx.x; i < 32 * (D / 4); i += kFewWaves * 64) {
    const int r = i / (D / 4), col = i % (D / 4) * 4;
    if (row0 + r >= rows || col >= e.s.dim) continue;
    f32x4 v = *reinterpret_cast<const f32x4*>(part + r * kPitch + col);
#pragma unroll
    for (int j = 1; j < kFewWaves; ++j) v += *reinterpret_cast<const f32x4*>(part + (j * 32 + r) * kPitch + col);
    uint32_t tok, mem;
    split_row(e.s.group, e.s.inv_group, row0 + r, tok, mem);
    const int64_t hd = int64_t(head) * e.s.group + mem;
    if (joined) {
      *reinterpret_cast<f32x4*>(e.part + (int64_t(split) * e.s.q.rows * e.s.heads + (p.q0 + tok) * e.s.heads + hd) * e.s.dim + col) = v;
    } else {
      const float n = norm[r];
      const u32x2 out = {pack_bf16x2(v[0] * n, v[1] * n), pack_bf16x2(v[2] * n, v[3] * n)};
      *reinterpret_cast<u32x2*>(e.o.p + (p.q0 + tok) * e.o.row + hd * e.o.head + col) = out;
    }
  }
}

// The shares' results of each row: a block per row. Its waves take the shares in turn, lanes two columns each.
__global__ __launch_bounds__(256) void attention_join_kernel(FwdArgs a) {
  __shared__ float lds[3][2 * kWave];
  const Shape& s = a.s;
  const int64_t row = a.first + blockIdx.x, count = s.q.rows * s.heads, token = row / s.heads;
  if (s.q.starts != nullptr && token >= s.q.starts[s.batch]) return;   // a row of no sequence
  const int lane = threadIdx.x & (kWave - 1), wave = wave_in_block();
  // lane i has share i's maximum and sum; a share without keys counts nothing, one whose scores are all -inf weighs 0
  float m = kLowest, l = kNoKeys;
  if (lane < a.splits) {
    m = a.stats[(lane * count + row) * 2];
    l = a.stats[(lane * count + row) * 2 + 1];
  }
  const bool none = l == kNoKeys;
  float top = m;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
  const float f = none ? -1.0f : exp2_fast(m - top), sum = wave_sum(none ? 0.0f : l * f);
  const bool any = __any(!none);
  const int col = 2 * lane < s.dim ? 2 * lane : 0;
  float v[2] = {0.0f, 0.0f};
  constexpr int kAtOnce = 4;
  for (int base = wave; base < a.splits; base += 4 * kAtOnce) {
    f32x2 x[kAtOnce];
    float g[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {   // a share without keys has written no sums: they are read, and not used
      const int i = base + 4 * j < a.splits ? base + 4 * j : base;
      x[j] = *reinterpret_cast<const f32x2*>(a.part + (i * count + row) * s.dim + col);
      g[j] = base + 4 * j < a.splits ? __shfl(f, i, kWave) : -1.0f;
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) v[e] = g[j] < 0.0f ? v[e] : __builtin_fmaf(x[j][e], g[j], v[e]);
  }
  if (wave > 0) {
    lds[wave - 1][lane] = v[0];
    lds[wave - 1][kWave + lane] = v[1];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    v[0] += lds[i][lane];
    v[1] += lds[i][kWave + lane];
  }
  const float n = any ? 1.0f / sum : 0.0f;
  uint16_t* o = a.o.p + token * a.o.row + (row - token * s.heads) * a.o.head;
  if (2 * lane < s.dim) *reinterpret_cast<uint32_t*>(o + 2 * lane) = pack_bf16x2(v[0] * n, v[1] * n);
  if (lane == 0) a.lse[row] = any ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -__builtin_inff();
}

// How a call is taken: blocks of 32 packed rows (few) or of 128, and the shares of the keys. Both kernels of a call, in a graph: one token of
// 16 sequences of 1 to 4096 keys, 32 heads: few 96 us (one share 104), 128 rows to a block 103 to 137; 64 sequences of 1000 keys 183 and 198; 4
// rows of 8 key heads each of 8 sequences of 500 keys 14 and 14; 8 queries of 16 sequences of 200 keys, 32 heads on 8, 11.3 and 8.7, so short
// sequences do not take it.
struct FwdForm {
  bool few;
  int splits;
};
static FwdForm fwd_form(const AttentionPlan& a, int cus) {
  const Shape s = shape_of(a);
  const int64_t keys = a.k_rows / a.batch;
  FwdForm f;
  f.few = a.q_rows * s.group <= 32 * a.batch && keys >= 512;
  const int64_t blocks = tiles_of(s.q, a.batch, false, s.group, f.few ? 32 : 128) * a.kv_heads;
  // Keys to a share: 4 tiles of each wave (few) or of the block, where blocks are to fill the device; 4 times as many where shares of few
  // queries' keys only even out sequences of different lengths (the device alone knows them). 256 queries and 16384 keys of 8 heads 37 us
  // (one share 364); 16 sequences of 2000 keys, 32 heads, one token in one share 95 (7 shares 112), 32 tokens 98 (158), and the sequences
  // of 1 to 4096 keys in 4 shares 96 (2: 106, 5: 92, 8: 95).
  const int64_t least = f.few ? kFewTiles * kFewWaves * (s.dim <= 64 ? kFewKeys<64> : kFewKeys<128>) : 4 * kKeys;
  const int64_t filling = std::min(blocks == 0 ? 1 : 2 * int64_t(cus) / blocks, keys / least);
  const int64_t evening = f.few && blocks > 0 ? std::min(8 * int64_t(cus) / blocks, keys / (4 * least)) : 1;
  f.splits = int(std::max<int64_t>(1, std::min<int64_t>(std::max(filling, evening), kWave)));
  return f;
}

template <int D>
hipError_t launch_fwd(FwdArgs f, bool few, int dev, hipStream_t st) {
  static std::atomic<uint64_t> done{0}, done_few{0};
  constexpr int kBytes = 4 * kKeys * D * 2;
  hipError_t e = few ? allow_lds(reinterpret_cast<const void*>(attention_few_kernel<D>), kFewLds<D>, dev, done_few)
                     : allow_lds(reinterpret_cast<const void*>(attention_fwd_kernel<D>), kBytes, dev, done);
  if (e != hipSuccess) return e;
  const int threads = few ? kFewWaves * 64 : 256;
  const int64_t blocks = tiles_of(f.s.q, f.s.batch, f.s.fill, f.s.group, few ? 32 : 128) * f.s.kv_heads * f.splits;
  return in_parts(blocks, most_blocks(threads), [&](int64_t first, int64_t count) {
    FwdArgs g = f;
    g.first = first;
    g.per_xcd = blocks_per_xcd(g.s, count);
    if (few) attention_few_kernel<D><<<uint32_t(count), threads, kFewLds<D>, st>>>(g);
    else attention_fwd_kernel<D><<<uint32_t(count), threads, kBytes, st>>>(g);
  });
}

}  // namespace attn

namespace {
int cus_or_default(int& dev) {
  int cus;
  return current_device(dev, cus) == hipSuccess ? cus : 256;
}
}  // namespace

size_t attention_fwd_workspace(const AttentionPlan& a) {
  int dev = 0;
  const int splits = attn::fwd_form(a, cus_or_default(dev)).splits;
  return splits > 1 ? size_t(splits) * size_t(a.q_rows) * size_t(a.heads) * size_t(a.dim + 2) * 4 : 0;
}

hipError_t launch_attention_fwd(const AttentionPlan& a, const HeadsView& q, const HeadsView& k, const HeadsView& v, const HeadsView& o,
                                float* lse, void* workspace, hipStream_t st) {
  int dev, cus;
  hipError_t e = current_device(dev, cus);
  if (e != hipSuccess) return e;
  attn::FwdArgs f{};
  f.s = attn::shape_of(a);
  f.q = attn::heads_of(q);
  f.k = attn::heads_of(k);
  f.v = attn::heads_of(v);
  f.o = attn::heads_of(o);
  f.lse = lse;
  const attn::FwdForm form = attn::fwd_form(a, cus);
  f.splits = form.splits;
  f.part = static_cast<float*>(workspace);
  f.stats = f.part + int64_t(f.splits) * a.q_rows * a.heads * a.dim;
  e = a.dim <= 64 ? attn::launch_fwd<64>(f, form.few, dev, st) : attn::launch_fwd<128>(f, form.few, dev, st);
  if (e != hipSuccess || f.splits == 1) return e;
  return in_parts(a.q_rows * a.heads, most_blocks(256), [&](int64_t first, int64_t count) {
    attn::FwdArgs g = f;
    g.first = first;
    attn::attention_join_kernel<<<uint32_t(count), 256, 0, st>>>(g);
  });
}

}  // namespace lmbp
