// Pieces that the attention kernels share (gfx950): the tiles in LDS, how a block finds its sequence,
// operand fragments, products that keep masked rows out of each other.
//
// Layout of the products. All of them are 32 x 32 x 16 MFMAs whose column is one row of the block's own
// side (a query in the forward and dq, a key in dk / dv): lane l holds column l % 32, and of the 16 values
// of a result the rows 8 (i / 4) + 4 (l / 32) + i % 4. As B operand of the next product the same lane needs 8
// consecutive k of its column; k is only summed over, so slot j of half h = l / 32 is taken to be row 8 (j / 4) +
// 4 h + j % 4 of 16: a result, rounded and packed, IS the next B operand, with nothing moved between
// lanes. The A operand of that product lies across memory and is read with the transposing LDS read (of 16
// lanes, lane q passes the address of columns 4 (q % 4) .. + 3 of row q / 4 and lane i gets the 4 rows of column i),
// two of them for the rows 4 h .. + 3 and 8 + 4 h .. + 3.
#pragma once

#include "lmbp_device.hpp"
#include "lmbp_launch.hpp"
#include "tile_device.hpp"

#include <atomic>

namespace lmbp {
namespace attn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
using lin::kOutOfRange;
using lin::lds_addr;
using lin::load_lds16_asm;
using lin::rsrc_words;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr float kLowest = -3.0e38f;   // start of a running maximum: below every score, and finite
constexpr uint32_t kAllRecords = 0x7fffffffu;   // rows that do not exist are passed as kOutOfRange

__device__ inline f32x16 mfma(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline s16x4 read_tr(const uint16_t* p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p)); }
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// The lane, as a value of its own: what is derived from it takes no register before.
__device__ inline int lane_again() {
  int v = threadIdx.x & (kWave - 1);
  asm volatile("" : "+v"(v));
  return v;
}
// The largest, and the sum, of the values of a column's two lanes.
__device__ inline float column_max(float v) {
  const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float column_sum(float v) {
  const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ inline int64_t uniform(int64_t v) {
  return int64_t(uint64_t(uint32_t(uniform(int(v)))) | uint64_t(uint32_t(uniform(int(v >> 32)))) << 32);
}

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// As load_lds16_asm, 4 bytes to a lane.
__device__ inline void load_lds4_asm(const u32x4& r, uint32_t dst, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds"
               :: "s"(dst), "v"(offset), "s"(r) : "memory", "m0");
}
#pragma clang diagnostic pop
// All of this wave's loads into LDS have landed and its reads are done, and then all waves'.
__device__ inline void wait_all() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
__device__ inline void wait_and_meet() {
  wait_all();
  asm volatile("s_barrier" ::: "memory");
}

// Heads of one tensor: element strides from row to row and from head to head; columns lie together.
struct Heads {
  uint16_t* p;
  int64_t row, head;
};

// Where the sequences of one side lie: given starts (packed), or all of one length.
struct Seqs {
  const int32_t* starts;   // batch + 1, or null
  int64_t rows;            // of the whole tensor
  int64_t each;            // rows of a sequence where starts is null
};

struct Shape {
  Seqs q, k;
  const int32_t* k_lens;   // keys in use of each sequence, or null
  int batch, heads, kv_heads, group, dim, causal, fill;
  uint32_t inv_group;      // floor(2^32 / group), 2^32 - 1 for 1
  float scale;
};

// r / group and the rest, for r < 2^31.
__device__ inline void split_row(uint32_t group, uint32_t inv_group, uint32_t r, uint32_t& token, uint32_t& member) {
  uint32_t t = __umulhi(r, inv_group);
  uint32_t m = r - t * group;
  if (m >= group) {
    m -= group;
    ++t;
  }
  token = t;
  member = m;
}
__device__ inline void split_row(const Shape& s, uint32_t r, uint32_t& token, uint32_t& member) {
  split_row(uint32_t(s.group), s.inv_group, r, token, member);
}

// Rows [first, first + len) of sequence b; b = batch: the rows behind the last one. Starts that do not
// ascend or leave the tensor give wrong results, never an access outside it.
__device__ inline void rows_of(const Seqs& s, int batch, int b, int64_t& first, int64_t& len) {
  if (s.starts == nullptr) {
    first = int64_t(b) * s.each;
    len = b < batch ? s.each : s.rows - first;
    return;
  }
  int64_t lo = b == 0 ? 0 : s.starts[b];
  lo = lo < 0 ? 0 : lo > s.rows ? s.rows : lo;
  int64_t hi = b < batch ? s.starts[b + 1] : s.rows;
  hi = hi < lo ? lo : hi > s.rows ? s.rows : hi;
  first = lo;
  len = hi - lo;
}

// The kernel's arguments, read again from memory: what only the end of a kernel needs takes no registers before it.
#define LMBP_CONSTANT __attribute__((address_space(4)))
template <class A>
__device__ inline const LMBP_CONSTANT A& late_args() {
  uint64_t p = uint64_t(__builtin_amdgcn_kernarg_segment_ptr());
  asm volatile("" : "+s"(p));
  return *(const LMBP_CONSTANT A*)(p);
}

// One block's part: tile `tile` of sequence b (b = batch: rows of no sequence).
struct Part {
  int b, tile, tiles;
  int64_t q0, k0;     // first rows
  int q_len, k_len;   // k_len: keys in use
  int k_slot;         // keys up to the next sequence
};

// A block's number where each XCD gets a run of per_xcd blocks (0: no such runs).
__device__ inline int64_t block_number(int64_t first, uint32_t per_xcd) {
  const uint32_t b = blockIdx.x;
  return first + (b < per_xcd * kXcds ? (b % kXcds) * per_xcd + b / kXcds : b);
}

// The t-th tile of causal sequences of different lengths, those that see (or are seen by) most first: by their distance from
// their sequence's lightest tile. 10 sequences of 1 to 2048 tokens, 8 key heads of 4 query heads, dim 128: the gradients of keys and
// values 276 us, in the sequences' order 337, the forward pass 155 and 166. A wave's lanes hold a sequence each.
template <bool QUERIES>
__device__ inline bool heaviest_first(const Shape& s, int64_t t, int per, int times, int& b, Part& p) {
  const Seqs& side = QUERIES ? s.q : s.k;
  const int lane = threadIdx.x & (kWave - 1), all = s.batch + (s.fill ? 1 : 0);
  int64_t first, len = 0;
  if (lane < all) rows_of(side, s.batch, lane, first, len);
  const int n = int((len * times + per - 1) / per);
  if (!__any(n > 1)) {   // a tile to a sequence
    const uint64_t real = __ballot(n > 0);
    if (t >= __popcll(real)) return false;
    b = __builtin_ctzll(__ballot(n > 0 && __popcll(real & ((uint64_t(1) << lane) - 1)) == int(t)));
    p.tiles = 1;
    p.tile = 0;
    return true;
  }
  // How many tiles are at a distance of at least `from`; the largest distance with more than t of them.
  auto tiles_from = [&](int from) {
    int count = 0;
    for (int i = 0; i < all; ++i) {
      const int over = __builtin_amdgcn_readlane(n, i) - from;
      count += over > 0 ? over : 0;
    }
    return count;
  };
  const int64_t most = (side.rows * times + per - 1) / per;
  int step = 1, low = 0, count = 0, at = 0;
  while (int64_t(step) * kWave <= most) step *= kWave;
  for (; step > 0; step /= kWave) {   // each lane tries a distance
    count = tiles_from(low + lane * step);
    at = __popcll(__ballot(count > t)) - 1;
    if (at < 0) return false;
    low += at * step;
  }
  const uint64_t there = __ballot(n > low);   // the sequences that have a tile at this distance, in order
  const int rank = int(t) - uniform(__shfl(count, at, kWave)) + __popcll(there);
  b = __builtin_ctzll(__ballot(n > low && __popcll(there & ((uint64_t(1) << lane) - 1)) == rank));
  p.tiles = uniform(__shfl(n, b, kWave));
  p.tile = p.tiles - 1 - low;
  return true;
}

// The t-th tile of `per` rows, a row of the side counting `times` times. false: there is none.
template <bool QUERIES>
__device__ inline bool locate(const Shape& s, int64_t t, int per, int times, Part& p) {
  const Seqs& side = QUERIES ? s.q : s.k;
  int b = 0;
  if (side.starts == nullptr) {
    const int64_t tiles = (side.each * times + per - 1) / per;
    if (t >= tiles * s.batch) return false;
    b = int(t / tiles);
    p.tile = int(t - b * tiles);
    p.tiles = int(tiles);
  } else if (s.causal && s.batch + (s.fill ? 1 : 0) <= kWave) {
    if (!heaviest_first<QUERIES>(s, t, per, times, b, p)) return false;
  } else {
    // 8 sequences to a lane, 512 to a wave, at a time. 4000 sequences of 8 tokens, 2 key heads: 242 us forward
    // (side by side 74), with one to a lane and 64-bit lengths 555.
    constexpr int kEach = 8;
    const int lane = threadIdx.x & (kWave - 1);
    const int all = s.batch + (s.fill ? 1 : 0);
    bool found = false;
    for (int base = 0; base < all; base += kWave * kEach) {
      int n[kEach], own = 0;
      // where sequence i starts, as rows_of() has it
      auto start_of = [&](int i) {
        const int at = side.starts[i < s.batch ? i : s.batch], rows = int(side.rows);
        return i > s.batch ? rows : i == 0 || at < 0 ? 0 : at < rows ? at : rows;
      };
      const int i0 = base + lane * kEach;
      int here = start_of(i0);
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int next = start_of(i0 + j + 1), len = next > here && i0 + j < all ? next - here : 0;
        n[j] = int((uint32_t(len) * uint32_t(times) + uint32_t(per - 1)) / uint32_t(per));
        own += n[j];
        here = next;
      }
      int sum = own;
#pragma unroll
      for (int off = 1; off < kWave; off <<= 1) {
        const int up = __shfl_up(sum, off, kWave);
        if (lane >= off) sum += up;
      }
      const int total = uniform(__shfl(sum, kWave - 1, kWave));
      if (t < total) {
        const int at = __builtin_ctzll(__ballot(sum > int(t)));
        int left = int(t) - uniform(__shfl(sum - own, at, kWave)), j = 0;
        p.tiles = uniform(__shfl(n[0], at, kWave));
#pragma unroll
        for (int i = 1; i < kEach; ++i) {
          if (j == i - 1 && left >= p.tiles) {
            left -= p.tiles;
            p.tiles = uniform(__shfl(n[i], at, kWave));
            j = i;
          }
        }
        b = base + at * kEach + j;
        p.tile = left;
        found = true;
        break;
      }
      t -= total;
    }
    if (!found) return false;
  }
  b = uniform(b);
  p.b = b;
  p.tile = uniform(p.tile);
  p.tiles = uniform(p.tiles);
  int64_t len, klen = 0;
  rows_of(s.q, s.batch, b, p.q0, len);
  p.q0 = uniform(p.q0);
  p.q_len = uniform(int(len));
  rows_of(s.k, s.batch, b, p.k0, klen);
  p.k0 = uniform(p.k0);
  p.k_slot = uniform(int(klen));
  if (b == s.batch) {
    klen = 0;
  } else if (s.k_lens != nullptr) {
    const int64_t used = s.k_lens[b];
    klen = used < 0 ? 0 : used < klen ? used : klen;
  }
  p.k_len = uniform(int(klen));
  if (QUERIES && b == s.batch) p.k_slot = 0;
  if (!QUERIES && b == s.batch) p.q_len = 0;
  return true;
}

// A tile of rows in LDS: D columns of 2 bytes, in pieces of 16 bytes. Piece c of row r is stored at c ^ swizzle(r): 16 rows
// of a row-wise read (16 bytes to a lane, 4 cycles) fall on distinct banks, and so do the 64 bytes of each of four rows that
// a transposing read takes at once (8 bytes to a lane, 2 cycles; with rows 1 apart 32 bytes apart, as smaller tiles
// of 16 columns want them, it took 4).
template <int D>
struct Tile {
  static constexpr int kPieces = D / 8;
  static constexpr int kSteps = D / 16;    // of 16 columns
  static constexpr int kBlocks = D / 32;   // of 32 columns
  static constexpr int kRowsPerLoad = 64 / kPieces;
  static constexpr __device__ int swizzle(int r) {
    if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
    else return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  }
  // Element offset of piece c of row r.
  static __device__ inline int at(int r, int c) { return r * D + (c ^ swizzle(r)) * 8; }
};

// Reads of fragments: this lane's element offsets within a tile. The pieces are stored under an exclusive or, so the
// other columns are at an exclusive or of the first ones' offset.
template <int D>
struct Reader {
  using T = Tile<D>;
  int row, col;
  __device__ inline Reader() {
    const int lane = threadIdx.x & (kWave - 1);
    const int h = lane >> 5, r = lane & 31, q = lane & 15, right = (lane >> 4) & 1;
    row = T::at(r, h);
    col = T::at(4 * h + q / 4, 2 * right + (q % 4) / 2) + (q % 2) * 4;
  }
  // The offsets derived from here on are formed again, not held in registers over a loop.
  __device__ inline void refresh() { asm volatile("" : "+v"(row), "+v"(col)); }
  // A operand, rows first .. first + 31 (first a multiple of 32): columns 16 s + 8 h .. of row l % 32.
  __device__ inline bf16x8 rows(const uint16_t* tile, int first, int s) const {
    return *reinterpret_cast<const bf16x8*>(tile + first * D + (row ^ (16 * s)));
  }
  // A operand across: rows first .. first + 15 (first a multiple of 16) of column 32 b + l % 32.
  __device__ inline bf16x8 across(const uint16_t* tile, int first, int b) const {
    const s16x4 lo = read_tr(tile + first * D + (col ^ (32 * b)));
    const s16x4 hi = read_tr(tile + (first + 8) * D + (col ^ (32 * b) ^ (T::swizzle(8) * 8)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// Loads of a tile of ROWS rows by WAVES waves, straight into LDS: rows of a tensor one behind the other
// (keys), or packed rows (token, head of the group). The swizzle is linear in the bits of the row.
template <int D, int ROWS, int WAVES>
struct Loader {
  using T = Tile<D>;
  static constexpr int kLoads = ROWS / T::kRowsPerLoad / WAVES;   // of each wave
  static constexpr int kStep = T::kRowsPerLoad * WAVES;           // rows from one load of a wave to its next
  static_assert(kLoads >= 1 && kLoads * kStep == ROWS, "rows to a wave");
  int first, piece, dim;   // this lane's row and piece of its first load
  uint32_t at;             // where the wave's first load goes
  __device__ inline Loader(int wave, int dim_) : dim(dim_), at(uint32_t(wave) * 1024) {
    const int lane = threadIdx.x & (kWave - 1);
    first = wave * T::kRowsPerLoad + lane / T::kPieces;
    piece = (lane % T::kPieces) ^ T::swizzle(first);
  }
  // Rows at `base` of which `left` exist, `pitch` bytes apart.
  __device__ inline void load(uint64_t base, uint32_t pitch, int left, uint32_t dst) const {
    const u32x4 r = rsrc_words(base, kAllRecords);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = first + j * kStep, c = piece ^ T::swizzle(j * kStep);
      const uint32_t off = uint32_t(row) * pitch + uint32_t(c) * 16;
      load_lds16_asm(r, dst + at + j * WAVES * 1024, row < left && c * 8 < dim ? off : kOutOfRange);
    }
  }
  // This lane's byte offsets of packed rows row0 .., from the token of row0 on.
  __device__ inline void packed(const Shape& s, uint32_t pitch, uint32_t head, uint32_t row0, uint32_t (&off)[kLoads]) const {
    uint32_t t0, m0;
    split_row(s, row0, t0, m0);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int c = piece ^ T::swizzle(j * kStep);
      uint32_t t, m;
      split_row(s, row0 + first + j * kStep, t, m);
      off[j] = c * 8 < dim ? (t - t0) * pitch + m * head + uint32_t(c) * 16 : kOutOfRange;
    }
  }
  // Rows at those offsets from `base`, of which `left` exist.
  __device__ inline void load_at(uint64_t base, const uint32_t (&off)[kLoads], int left, uint32_t dst) const {
    const u32x4 r = rsrc_words(base, kAllRecords);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load_lds16_asm(r, dst + at + j * WAVES * 1024, first + j * kStep < left ? off[j] : kOutOfRange);
  }
};

// Eight results of a column, rounded: the B operand of the next product.
__device__ inline bf16x8 pack8(const f32x16& v, int first) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(v[first + 2 * i], v[first + 2 * i + 1]);
  return __builtin_bit_cast(bf16x8, w);
}

// 1 (bf16) for those of this lane's 8 of 16 rows n0 .. that lie in [lo, hi): what its column sees.
__device__ inline bf16x8 seen_of(int n0, int lo, int hi) {
  const int h = (threadIdx.x >> 5) & 1;
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = n0 + 8 * (i / 2) + 4 * h + 2 * (i % 2);
    w[i] = (n >= lo && n < hi ? 0x3f80u : 0u) | (n + 1 >= lo && n + 1 < hi ? 0x3f800000u : 0u);
  }
  return __builtin_bit_cast(bf16x8, w);
}

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// Whether a tile of ROWS rows in LDS holds an infinity or NaN: the same for the whole block of 4 waves, which meets here. Two
// flags, cleared before; once one is set the caller asks no more.
template <int D, int ROWS>
__device__ inline bool tile_is_odd(const uint16_t* tile, int* flags, int which) {
  u16x2 most = {0, 0};
#pragma unroll
  for (int i = 0; i < ROWS * D / 2048; ++i) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(tile + (i * 256 + threadIdx.x) * 8);
#pragma unroll
    for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w[j] & 0x7fff7fffu));
  }
  if (most[0] >= 0x7f80 || most[1] >= 0x7f80) flags[which] = 1;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  asm volatile("s_barrier" ::: "memory");
  return uniform(*const_cast<volatile int*>(flags + which)) != 0;
}

// Whether a wave's fragments hold an infinity or NaN.
template <int N>
__device__ inline bool any_odd(const bf16x8 (&f)[N]) {
  u16x2 most = {0, 0};
#pragma unroll
  for (int s = 0; s < N; ++s) {
    const u32x4 w = __builtin_bit_cast(u32x4, f[s]);
#pragma unroll
    for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w[j] & 0x7fff7fffu));
  }
  return __any(most[0] >= 0x7f80 || most[1] >= 0x7f80);
}

// acc += tile^T p for 16 rows of the tile of which a column sees those of `see`, and the others, where p is 0, may
// hold anything. Infinities and NaN are looked for first; where there are any they are taken out of the product and go to
// the columns that see them, counted by a product with ones. NANS: an infinity too makes NaN.
template <bool NANS, int D>
__device__ inline void add_guarded(f32x16 (&acc)[D / 32], const uint16_t* tile, const Reader<D>& rd, int first, const bf16x8& p,
                                   const bf16x8& see) {
#pragma unroll
  for (int b = 0; b < D / 32; ++b) {
    __builtin_amdgcn_sched_barrier(0);   // one block of columns at a time: registers
    const u32x4 f = __builtin_bit_cast(u32x4, rd.across(tile, first, b));
    u16x2 most = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, f[i] & 0x7fff7fffu));
    const bool bad = __any(most[0] >= 0x7f80 || most[1] >= 0x7f80);
    u32x4 w = f;
    if (bad) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] &= ((f[i] & 0x7f80u) == 0x7f80u ? 0xffff0000u : ~0u) & ((f[i] & 0x7f800000u) == 0x7f800000u ? 0xffffu : ~0u);
    }
    acc[b] = mfma(__builtin_bit_cast(bf16x8, w), p, acc[b]);
    if (bad) {
      u32x4 odd;   // +inf 1, -inf 2^8, NaN 2^16: sums of 16 say which there are
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t part[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t v = (f[i] >> (16 * e)) & 0xffffu;
          const uint32_t kind = NANS ? 0x4780u : v == 0x7f80u ? 0x3f80u : v == 0xff80u ? 0x4380u : 0x4780u;
          part[e] = (v & 0x7f80u) == 0x7f80u ? kind : 0u;
        }
        odd[i] = part[0] | (part[1] << 16);
      }
      const f32x16 n = mfma(__builtin_bit_cast(bf16x8, odd), see, f32x16{});
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int k = int(n[i]);
        const float v = k < 0x100 ? __builtin_inff() : k < 0x10000 && (k & 0xff) == 0 ? -__builtin_inff() : __builtin_nanf("");
        acc[b][i] += k == 0 ? 0.0f : v;
      }
    }
  }
}

// Stores 32 rows' results times f, rounded: lane l has row l % 32; the halves exchange pieces, so that each lane
// stores 16 bytes at a time. keep: the bits of a row's values that are stored, all or none.
template <int D>
__device__ inline void store_columns(const f32x16 (&v)[D / 32], float f, uint16_t* row, bool real, int dim, uint32_t keep = ~0u) {
  const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      u32x4 out;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t lo = pack_bf16x2(v[b][8 * u + 2 * i] * f, v[b][8 * u + 2 * i + 1] * f);
        const uint32_t hi = pack_bf16x2(v[b][8 * u + 4 + 2 * i] * f, v[b][8 * u + 4 + 2 * i + 1] * f);
        const u32x2 both = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(lo, hi, false, false));
        out[i] = both[0];
        out[2 + i] = both[1];
      }
      const int col = 32 * b + 16 * u + 8 * h;
      if (real && col < dim) *reinterpret_cast<u32x4*>(row + col) = out & keep;
    }
}

// 8 columns of fragments of row `row` (null: zeros).
template <int D>
__device__ inline void load_rows(bf16x8 (&f)[D / 16], const uint16_t* row, int dim) {
  const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    u32x4 w = {0u, 0u, 0u, 0u};
    if (row != nullptr && 16 * s + 8 * h < dim) w = *reinterpret_cast<const u32x4*>(row + 16 * s + 8 * h);
    f[s] = __builtin_bit_cast(bf16x8, w);
  }
}

// Host side.
inline Heads heads_of(const HeadsView& v) { return Heads{static_cast<uint16_t*>(v.p), v.row, v.head}; }
inline Shape shape_of(const AttentionPlan& a) {
  Shape s{};
  s.q = Seqs{a.q_starts, a.q_rows, a.q_starts ? 0 : a.q_rows / a.batch};
  s.k = Seqs{a.k_starts, a.k_rows, a.k_starts ? 0 : a.k_rows / a.batch};
  s.k_lens = a.k_lens;
  s.batch = int(a.batch);
  s.heads = int(a.heads);
  s.kv_heads = int(a.kv_heads);
  s.group = int(a.heads / a.kv_heads);
  s.dim = int(a.dim);
  s.causal = a.causal;
  s.fill = a.fill;
  s.inv_group = s.group == 1 ? 0xffffffffu : uint32_t((uint64_t(1) << 32) / uint64_t(s.group));
  s.scale = a.scale;
  return s;
}
// Consecutive blocks go to the XCDs in turn: with a multiple of 8 key heads all tiles of a head come to one XCD, whose L2 keeps what
// they share. With others each XCD gets a run of blocks, where these have about the same work: 64 images of 197 tokens, 12 heads of
// 64, take 28 us forward and 35 and 35 backward so, 31, 37 and 38 with blocks in turn.
inline uint32_t blocks_per_xcd(const Shape& s, int64_t blocks) {
  const bool alike = s.q.starts == nullptr && s.k.starts == nullptr && (!s.causal || s.batch % kXcds == 0);
  return alike && s.kv_heads % kXcds != 0 ? uint32_t(blocks / kXcds) : 0;
}
// The most tiles of `per` rows that a side has, a row counting `times` times.
inline int64_t tiles_of(const Seqs& s, int64_t batch, bool fill, int64_t times, int64_t per) {
  if (s.starts == nullptr) return (s.each * times + per - 1) / per * batch;
  return s.rows * times / per + batch + (fill ? 1 : 0);
}
// Dynamic LDS beyond 64 KB has to be asked for, once per kernel and device.
inline hipError_t allow_lds(const void* kernel, int bytes, int dev, std::atomic<uint64_t>& done) {
  const uint64_t bit = uint64_t(1) << dev;
  if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

}  // namespace attn
}  // namespace lmbp
