// Attention forward for gfx950: o = softmax(scale q k^T) v over the keys that each query sees, and the
// logarithm of each row's sum.
#include "attention_device.hpp"

#include <algorithm>

namespace lmbp {
namespace attn {

struct FwdArgs {
  Shape s;
  Heads q, k, v, o;
  float* lse;        // [rows][heads]
  float* part;       // splits > 1: [splits][rows * heads][dim], unnormalised
  float* stats;      // splits > 1: [splits][rows * heads][2]: running maximum (log2), sum
  int splits;
  int64_t first;     // block number of this launch's first block
};

constexpr int kKeys = 64;      // keys to a tile
constexpr float kSlack = 8.0f;  // a row's running maximum may stay this much (log2) behind its largest score

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

  // Keys key0 .. + 32 B - 1, the tile's from `first` on.
  template <bool MASKED, int kB>
  __device__ inline void step(const uint16_t* K, const uint16_t* V, const Reader<D>& rd, int first, int key0, float c) {
    f32x16 x[kB];
#pragma unroll
    for (int b = 0; b < kB; ++b) x[b] = f32x16{};
#pragma unroll
    for (int s = 0; s < T::kSteps; ++s)
#pragma unroll
      for (int b = 0; b < kB; ++b) x[b] = mfma(rd.rows(K, first + 32 * b, s), q[s], x[b]);
    const int h = (threadIdx.x >> 5) & 1;
    if constexpr (MASKED) {
      const int left = limit - key0 - 4 * h;
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * b + 8 * (i / 4) + i % 4 >= left) x[b][i] = -__builtin_inff();
    }
    float most = x[0][0];
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) most = fmaxf(most, x[b][i]);
    most = fmaxf(most, other_half(most)) * c;
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
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[b][i] = exp2_fast(__builtin_fmaf(x[b][i], c, -top));
        sum += x[b][i];
      }
#pragma unroll
    for (int t = 0; t < 2 * kB; ++t) {
      const bf16x8 p = pack8(x[t / 2], 8 * (t % 2));
      if constexpr (MASKED) {
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
  const Shape& s = a.s;
  const int64_t id = a.first + blockIdx.x;
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
  if (begin < end) fetch(begin, 0);
  int t = begin;
  auto next = [&]() {   // the tile in LDS
    const int slot = (t - begin) & 1;
    wait_and_meet();
    if (t + 1 < end) fetch(t + 1, slot ^ 1);
    return lds + slot * 2 * kTile;
  };
  for (; t < end && t < whole; ++t) {
    const uint16_t* K = next();
    w.template step<false, kKeys / 32>(K, K + kTile, rd, 0, t * kKeys, c);
  }
  for (; t < end; ++t) {
    const uint16_t* K = next();
#pragma unroll 1
    for (int f = 0; f < kKeys && t * kKeys + f < wave_max; f += 32) w.template step<true, 1>(K, K + kTile, rd, f, t * kKeys + f, c);
  }
  wait_all();   // no load into LDS outlives the block
  const auto& e = late_args<FwdArgs>();
  const float sum = w.sum + other_half(w.sum);
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
      st[1] = sum;
    }
    return;
  }
  if (split > 0) return;
  uint16_t* o = e.o.p + (p.q0 + token) * e.o.row + o_head * e.o.head;
  store_columns<D>(w.o, w.limit > 0 ? 1.0f / sum : 0.0f, o, real, e.s.dim);
  if (real && lane < 32) e.lse[out_row] = w.limit > 0 ? (w.top + __builtin_amdgcn_logf(sum)) * kLn2 : -__builtin_inff();
}

// The shares' results of each row: a wave per row, its columns over the lanes.
__global__ __launch_bounds__(256) void attention_join_kernel(FwdArgs a) {
  const Shape& s = a.s;
  const int64_t row = a.first + int64_t(blockIdx.x) * 4 + wave_in_block();
  const int64_t count = s.q.rows * s.heads;
  if (row >= count) return;
  const int64_t token = row / s.heads;
  if (s.q.starts != nullptr && token >= s.q.starts[s.batch]) return;   // a row of no sequence
  const int lane = threadIdx.x & (kWave - 1);
  float top = kLowest;
  for (int i = 0; i < a.splits; ++i) top = fmaxf(top, a.stats[(i * count + row) * 2]);
  float sum = 0.0f, v[2] = {0.0f, 0.0f};
  bool any = false;
  for (int i = 0; i < a.splits; ++i) {
    const float m = a.stats[(i * count + row) * 2], l = a.stats[(i * count + row) * 2 + 1];
    if (l == 0.0f && m == kLowest) continue;   // no key in this share
    any = true;
    const float f = exp2_fast(m - top);
    sum = __builtin_fmaf(l, f, sum);
    const float* from = a.part + (i * count + row) * s.dim;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (2 * lane + e < s.dim) v[e] = __builtin_fmaf(from[2 * lane + e], f, v[e]);
  }
  const float f = any ? 1.0f / sum : 0.0f;
  uint16_t* o = a.o.p + token * a.o.row + (row - token * s.heads) * a.o.head;
  if (2 * lane < s.dim) *reinterpret_cast<uint32_t*>(o + 2 * lane) = pack_bf16x2(v[0] * f, v[1] * f);
  if (lane == 0) a.lse[row] = any ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -__builtin_inff();
}

// Shares of the keys: where the rows give fewer blocks than the device takes at once, each at least 4 tiles.
static int key_shares(const AttentionPlan& a, int cus) {
  const Shape s = shape_of(a);
  const int64_t blocks = tiles_of(s.q, a.batch, false, s.group, 128) * a.kv_heads;
  const int64_t keys = a.k_rows / a.batch;
  if (blocks == 0) return 1;
  return int(std::max<int64_t>(1, std::min<int64_t>({2 * cus / blocks, keys / (4 * kKeys), 64})));
}

template <int D>
hipError_t launch_fwd(FwdArgs f, int dev, hipStream_t st) {
  static std::atomic<uint64_t> done{0};
  constexpr int kBytes = 4 * kKeys * D * 2;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(attention_fwd_kernel<D>), kBytes, dev, done);
  if (e != hipSuccess) return e;
  const int64_t blocks = tiles_of(f.s.q, f.s.batch, f.s.fill, f.s.group, 128) * f.s.kv_heads * f.splits;
  return in_parts(blocks, most_blocks(256), [&](int64_t first, int64_t count) {
    FwdArgs g = f;
    g.first = first;
    attention_fwd_kernel<D><<<uint32_t(count), 256, kBytes, st>>>(g);
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
  const int splits = attn::key_shares(a, cus_or_default(dev));
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
  f.splits = attn::key_shares(a, cus);
  f.part = static_cast<float*>(workspace);
  f.stats = f.part + int64_t(f.splits) * a.q_rows * a.heads * a.dim;
  e = a.dim <= 64 ? attn::launch_fwd<64>(f, dev, st) : attn::launch_fwd<128>(f, dev, st);
  if (e != hipSuccess || f.splits == 1) return e;
  return in_parts((a.q_rows * a.heads + 3) / 4, most_blocks(256), [&](int64_t first, int64_t count) {
    attn::FwdArgs g = f;
    g.first = first * 4;
    attn::attention_join_kernel<<<uint32_t(count), 256, 0, st>>>(g);
  });
}

}  // namespace lmbp
