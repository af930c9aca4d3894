// Attention backward for gfx950. With P = exp(scale q k^T - lse), D = rowsum(do o), dS = P (do v^T - D):
//
//   dq = scale dS k,  dk = scale dS^T q,  dv = P^T do
//
// Two kernels, each forming the scores again: dq per rows (which also writes each row's lse and D for the other),
// dk and dv per keys. One kernel for all three would have to add dq up with atomics, whose order changes results.
#include "attention_device.hpp"

#include <algorithm>

namespace lmbp {
namespace attn {

struct BwdArgs {
  Shape s;
  Heads q, k, v, o, d_o, dq, dk, dv;
  const float* lse;   // [rows][heads]
  float* stats;       // [kv_heads][rows * group][2]: lse in log2, D
  float* part;        // shares > 1: [shares][2][rows of k][kv_heads][dim]: dk, dv
  int shares;
  int64_t first;      // block number of this launch's first block
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

  // 32 keys, the tile's from `first` on.
  template <bool MASKED>
  __device__ inline void step(const uint16_t* K, const uint16_t* V, Reader<D>& rd, int first, int key0, float c) {
    f32x16 x = f32x16{}, y = f32x16{};
    rd.refresh();
#pragma unroll
    for (int s = 0; s < T::kSteps; ++s) {
      x = mfma(rd.rows(K, first, s), q[s], x);
      y = mfma(rd.rows(V, first, s), d_o[s], y);
    }
    __builtin_amdgcn_sched_barrier(0);
    const int left = limit - key0 - 4 * ((threadIdx.x >> 5) & 1);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      x[i] = exp2_fast(__builtin_fmaf(x[i], c, -lse)) * (y[i] - share);
      if constexpr (MASKED) x[i] = 8 * (i / 4) + i % 4 < left ? x[i] : 0.0f;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8 ds = pack8(x, 8 * t);
      if constexpr (MASKED) {
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
  const Shape& s = a.s;
  const int64_t id = a.first + blockIdx.x;
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
  w.share = sum + other_half(sum);
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
    for (int f = 0; f < kKeys; f += 32) w.template step<false>(K, K + kTile, rd, f, t * kKeys + f, c);
  }
  for (; t < end; ++t) {
    const uint16_t* K = next();
#pragma unroll 1
    for (int f = 0; f < kKeys && t * kKeys + f < wave_max; f += 32) w.template step<true>(K, K + kTile, rd, f, t * kKeys + f, c);
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
  int from;   // packed rows from it on see this lane's key

  // 32 packed rows from row0 on, with their lse and D. V: the block's values, this wave's from row `mine` on.
  template <bool MASKED>
  __device__ inline void step(const uint16_t* Q, const uint16_t* O, const uint16_t* V, int mine, const float* stats, Reader<D>& rd, int row0, float c) {
    f32x16 x = f32x16{}, y = f32x16{};
    rd.refresh();
#pragma unroll
    for (int s = 0; s < T::kSteps; ++s) {
      x = mfma(rd.rows(Q, 0, s), k[s], x);
      y = mfma(rd.rows(O, 0, s), rd.rows(V, mine, s), y);
    }
    __builtin_amdgcn_sched_barrier(0);
    const int h = (threadIdx.x >> 5) & 1;
    const int skip = from - row0 - 4 * h;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4* st = reinterpret_cast<const f32x4*>(stats + (8 * g + 4 * h) * 2);
      const f32x4 lo = st[0], hi = st[1];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 4 * g + e;
        const float lse = e < 2 ? lo[2 * e] : hi[2 * e - 4], share = e < 2 ? lo[2 * e + 1] : hi[2 * e - 3];
        x[i] = exp2_fast(__builtin_fmaf(x[i], c, -lse));
        y[i] = x[i] * (y[i] - share);
        if constexpr (MASKED) {
          const bool sees = 8 * g + e >= skip;
          x[i] = sees ? x[i] : 0.0f;
          y[i] = sees ? y[i] : 0.0f;
        }
      }
    }
    const bf16x8 p[2] = {pack8(x, 0), pack8(x, 8)}, ds[2] = {pack8(y, 0), pack8(y, 8)};
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (MASKED) {
#pragma unroll 1
      for (int t = 0; t < 2; ++t) {
        const bf16x8 see = seen_of(row0 + 16 * t, from, 0x7fffffff);
        add_guarded<false, D>(dv, O, rd, 16 * t, t == 0 ? p[0] : p[1], see);
        add_guarded<true, D>(dk, Q, rd, 16 * t, t == 0 ? ds[0] : ds[1], see);
      }
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int b = 0; b < T::kBlocks; ++b) {
          dv[b] = mfma(rd.across(O, 16 * t, b), p[t], dv[b]);
          dk[b] = mfma(rd.across(Q, 16 * t, b), ds[t], dk[b]);
        }
    }
  }
};

// A block of 4 waves: 128 keys of one head, 32 to a wave, against all (or a share of) the packed rows that see them.
template <int D>
__global__ __launch_bounds__(256, 2) void attention_dkv_kernel(BwdArgs a) {
  using T = Tile<D>;
  constexpr int kTile = kRows * D;
  extern __shared__ __attribute__((aligned(16))) uint16_t lds[];   // two slots of Q and dO, V, two slots of the rows' values
  const uint16_t* V = lds + 4 * kTile;
  float* stats = reinterpret_cast<float*>(lds + 4 * kTile + 128 * D);
  const Shape& s = a.s;
  const int64_t id = a.first + blockIdx.x;
  const int head = int(id % s.kv_heads);
  const int64_t rest = id / s.kv_heads;
  const int part = int(rest % a.shares);
  Part p;
  if (!locate<false>(s, rest / a.shares, 128, 1, p)) return;
  const int wave = wave_in_block(), lane = threadIdx.x & (kWave - 1);
  const int key_b = p.tile * 128, key_w = key_b + wave * 32, key = key_w + (lane & 31);
  const bool used = key < p.k_len;
  const int rows = p.q_len * s.group, off = p.k_len - p.q_len;
  auto first_row = [&](int j) { return s.causal && j > off ? (j - off) * s.group : 0; };   // that sees key j
  Keys<D> w;
#pragma unroll
  for (int b = 0; b < T::kBlocks; ++b) w.dk[b] = w.dv[b] = f32x16{};
  w.from = first_row(key);
  load_rows<D>(w.k, used ? a.k.p + (p.k0 + key) * a.k.row + head * a.k.head : nullptr, s.dim);
  const int masked = uniform((first_row(key_b + 127) + kRows - 1) / kRows);   // tiles from it on need no mask

  const int lowest = key_b < p.k_len ? first_row(key_b) / kRows : 0;
  const int all = key_b < p.k_len && lowest * kRows < rows ? (rows + kRows - 1) / kRows - lowest : 0;   // tiles
  const int each = (all + a.shares - 1) / a.shares;
  const int begin = uniform(lowest + part * each);
  const int end = uniform(lowest + (part * each + each < all ? part * each + each : all));

  const Loader<D, kRows, 4> ld(wave, s.dim);
  Reader<D> rd;
  const uint32_t lds0 = lds_addr(lds);
  const int64_t q_head0 = int64_t(head) * s.group;
  const uint64_t qb = reinterpret_cast<uint64_t>(a.q.p + p.q0 * a.q.row + q_head0 * a.q.head);
  const uint64_t ob = reinterpret_cast<uint64_t>(a.d_o.p + p.q0 * a.d_o.row + q_head0 * a.d_o.head);
  const uint64_t sb = reinterpret_cast<uint64_t>(a.stats + (int64_t(head) * s.q.rows + p.q0) * s.group * 2);
  auto fetch = [&](int t, int slot) {
    const uint32_t row0 = uint32_t(t) * kRows;
    ld.load_packed(s, qb, a.q.row * 2, uint32_t(a.q.head * 2), row0, uint32_t(rows), lds0 + slot * 4 * kTile);
    ld.load_packed(s, ob, a.d_o.row * 2, uint32_t(a.d_o.head * 2), row0, uint32_t(rows), lds0 + slot * 4 * kTile + 2 * kTile);
    if (wave == 0)
      load_lds4_asm(rsrc_words(sb + uint64_t(row0) * 8, kAllRecords), lds0 + 8 * kTile + 256 * D + slot * kRows * 8,
                    int(row0) + lane / 2 < rows ? uint32_t(lane) * 4 : kOutOfRange);
  };
  const float c = s.scale * kLog2e;
  if (begin < end) {
    const Loader<D, 128, 4> lv(wave, s.dim);
    lv.load(reinterpret_cast<uint64_t>(a.v.p + (p.k0 + key_b) * a.v.row + head * a.v.head), uint32_t(a.v.row * 2), p.k_len - key_b,
            lds0 + 8 * kTile);
    fetch(begin, 0);
  }
  int t = begin;
  auto next = [&]() {   // the tile in LDS
    const int slot = (t - begin) & 1;
    wait_and_meet();
    if (t + 1 < end) fetch(t + 1, slot ^ 1);
    return slot;
  };
  for (; t < end && t < masked; ++t) {
    const int slot = next();
    const uint16_t* Q = lds + slot * 2 * kTile;
    w.template step<true>(Q, Q + kTile, V, wave * 32, stats + slot * kRows * 2, rd, t * kRows, c);
  }
  for (; t < end; ++t) {
    const int slot = next();
    const uint16_t* Q = lds + slot * 2 * kTile;
    w.template step<false>(Q, Q + kTile, V, wave * 32, stats + slot * kRows * 2, rd, t * kRows, c);
  }
  wait_all();   // no load into LDS outlives the block
  const auto& e = late_args<BwdArgs>();
  // keys that are not in use get zeros where the rows of no sequence do
  const bool real = key < (e.s.fill ? p.k_slot : p.k_len);
  if (e.shares > 1) {
    if (key >= p.k_len) return;   // the sum takes them as zeros
    const int64_t size = e.s.k.rows * e.s.kv_heads * e.s.dim;
    float* to = e.part + int64_t(part) * 2 * size + ((p.k0 + key) * e.s.kv_heads + head) * e.s.dim;
    const int h = lane >> 5;
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
  store_columns<D>(w.dk, used ? e.s.scale : 0.0f, e.dk.p + (p.k0 + key) * e.dk.row + head * e.dk.head, real, e.s.dim);
  store_columns<D>(w.dv, used ? 1.0f : 0.0f, e.dv.p + (p.k0 + key) * e.dv.row + head * e.dv.head, real, e.s.dim);
}

// The shares' sums of dk and dv, in order: a block per tile of 128 keys and head.
__global__ __launch_bounds__(256) void attention_dkv_join_kernel(BwdArgs a) {
  const Shape& s = a.s;
  const int64_t id = a.first + blockIdx.x;
  const int head = int(id % s.kv_heads);
  Part p;
  if (!locate<false>(s, id / s.kv_heads, 128, 1, p)) return;
  const int64_t size = s.k.rows * s.kv_heads * s.dim;
  const int pieces = s.dim / 4;
  for (int i = threadIdx.x; i < 128 * pieces; i += 256) {
    const int key = p.tile * 128 + i / pieces, col = i % pieces * 4;
    if (key >= (s.fill ? p.k_slot : p.k_len)) break;
    f32x4 dk = {0.0f, 0.0f, 0.0f, 0.0f}, dv = dk;
    if (key < p.k_len) {
      const float* from = a.part + ((p.k0 + key) * s.kv_heads + head) * s.dim + col;
      for (int n = 0; n < a.shares; ++n) {
        dk += *reinterpret_cast<const f32x4*>(from + 2 * n * size);
        dv += *reinterpret_cast<const f32x4*>(from + (2 * n + 1) * size);
      }
    }
    const u32x2 wk = {pack_bf16x2(dk[0] * s.scale, dk[1] * s.scale), pack_bf16x2(dk[2] * s.scale, dk[3] * s.scale)};
    const u32x2 wv = {pack_bf16x2(dv[0], dv[1]), pack_bf16x2(dv[2], dv[3])};
    *reinterpret_cast<u32x2*>(a.dk.p + (p.k0 + key) * a.dk.row + head * a.dk.head + col) = wk;
    *reinterpret_cast<u32x2*>(a.dv.p + (p.k0 + key) * a.dv.row + head * a.dv.head + col) = wv;
  }
}

// Shares of the packed rows that a key's sums are split into: where the keys give fewer blocks than the device takes
// at once, each at least 8 tiles, their sums at most 256 MiB.
static int row_shares(const AttentionPlan& a, int cus) {
  const Shape s = shape_of(a);
  const int64_t blocks = tiles_of(s.k, a.batch, false, 1, 128) * a.kv_heads;
  const int64_t rows = a.q_rows / a.batch * s.group, bytes = a.k_rows * a.kv_heads * a.dim * 8;
  if (blocks == 0 || bytes == 0) return 1;
  return int(std::max<int64_t>(1, std::min<int64_t>({2 * cus / blocks, rows / (8 * kRows), (int64_t(256) << 20) / bytes})));
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
    attention_dq_kernel<D><<<uint32_t(count), 256, kBytesQ, st>>>(g);
  });
  if (e != hipSuccess) return e;
  const int64_t tiles = tiles_of(f.s.k, f.s.batch, f.s.fill, 1, 128) * f.s.kv_heads;
  e = in_parts(tiles * f.shares, most_blocks(256), [&](int64_t first, int64_t count) {
    g.first = first;
    attention_dkv_kernel<D><<<uint32_t(count), 256, kBytesKv, st>>>(g);
  });
  if (e != hipSuccess || f.shares == 1) return e;
  return in_parts(tiles, most_blocks(256), [&](int64_t first, int64_t count) {
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
  const int shares = attn::row_shares(a, cus);
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
  f.shares = attn::row_shares(a, cus);
  return a.dim <= 64 ? attn::launch_bwd<64>(f, dev, st) : attn::launch_bwd<128>(f, dev, st);
}

}  // namespace lmbp
