// Pieces of the tiled matrix products whose operands go straight from memory into LDS (gfx950):
// buffer resources, the loads, the order of tiles, scheduling groups.
#pragma once

#include "lmbp_device.hpp"
#include "lmbp_launch.hpp"

namespace lmbp {
namespace lin {

typedef __attribute__((address_space(3))) void lds_void;

constexpr int kGroupM = 8;
constexpr uint32_t kBufferGDword3 = 0x00020000;  // raw 32-bit buffer, gfx9 family
constexpr uint32_t kOutOfRange = 0x80000000u;    // beyond any resource's range: reads 0

// The grid of tiles: sizes, tiles per XCD, and floor(2^32 / tiles_n).
struct TileMap {
  uint32_t tiles_m, tiles_n, tiles, per_xcd, inv_n;
};

// The target builtins below are wrapped in device functions: used directly in the body of
// a kernel template, they make the host-side instantiation fail silently and the launch
// stub is never emitted.

// A raw buffer resource over `bytes` bytes at `base` (reads beyond return zeros).
__device__ inline __amdgpu_buffer_rsrc_t make_rsrc(const void* base, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, int(bytes), kBufferGDword3);
}
// 16 or 4 bytes per lane from the buffer into LDS at `dst` + lane * 16 or 4 (dst wave-uniform).
// CPOL: cache policy bits of the instruction (nt = 2).
template <int CPOL = 0>
__device__ inline void load_lds16(__amdgpu_buffer_rsrc_t r, void* dst, uint32_t offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)dst, 16, offset, 0, 0, CPOL);
}
__device__ inline void load_lds4(__amdgpu_buffer_rsrc_t r, void* dst, uint32_t offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)dst, 4, offset, 0, 0, 0);
}

// A buffer resource as its four words.
__device__ inline u32x4 rsrc_words(uint64_t base, uint32_t bytes) {
  return u32x4{uint32_t(base), uint32_t(base >> 32) & 0xffffu, bytes, kBufferGDword3};
}
// The same load as load_lds16, written as asm, for kernels that read LDS with transposing reads:
// of the builtin the compiler knows that it writes LDS, and it waits for all of them before
// every such read. `dst`: LDS address (lds_addr). The waits are the kernel's own. The wait states
// cover a resource whose registers a VALU operation has just written (5, with the move).
// The compiler reserves m0 for itself and warns that it cannot keep a value there across
// the asm; the clobber is to say just that, so that it never counts on one.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void load_lds16_asm(const u32x4& r, uint32_t dst, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(dst), "v"(offset), "s"(r) : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ inline uint32_t lds_addr(const void* p) { return uint32_t(uintptr_t((const lds_void*)p)); }

// Scheduling groups for MF MFMAs, with VM buffer loads and then DS LDS reads spread over
// the first half of them (so the reads have landed before the next wait).
template <int MF, int VM, int DS, int I = 0>
__device__ inline void spread() {
  if constexpr (I < MF) {
    constexpr int W = MF / 2 < 1 ? 1 : MF / 2;
    constexpr int T = VM + DS;
    constexpr int lo = I < W ? T * I / W : T, hi = I < W ? T * (I + 1) / W : T;
    constexpr int vm = (hi < VM ? hi : VM) - (lo < VM ? lo : VM);
    constexpr int ds = (hi - lo) - vm;
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                  // one MFMA
    if constexpr (vm > 0) __builtin_amdgcn_sched_group_barrier(0x020, vm, 0);  // buffer loads
    if constexpr (ds > 0) __builtin_amdgcn_sched_group_barrier(0x100, ds, 0);  // LDS reads
    spread<MF, VM, DS, I + 1>();
  }
}

// Tile coordinates of the t-th tile: XCD by XCD (consecutive blocks go to the 8 XCDs in turn),
// in groups of kGroupM row tiles. tiles_n is divided by with a host-made reciprocal
// (floor(2^32 / tiles_n), at most one short of the quotient for t < 2^30) instead of an integer
// division.
__device__ inline void tile_of(uint32_t t, const TileMap& m, uint32_t& tm, uint32_t& tn) {
  const uint32_t id = (t < m.per_xcd * kXcds) ? (t % kXcds) * m.per_xcd + t / kXcds : t;
  const uint32_t id8 = id / kGroupM;
  uint32_t group = __umulhi(id8, m.inv_n);
  uint32_t in = id8 - group * m.tiles_n;
  while (in >= m.tiles_n) {
    in -= m.tiles_n;
    ++group;
  }
  const uint32_t first_m = group * kGroupM, r = in * kGroupM + id % kGroupM;
  const uint32_t left = m.tiles_m - first_m;
  if (left >= uint32_t(kGroupM)) {
    tm = first_m + r % kGroupM;
    tn = r / kGroupM;
  } else {   // the last, smaller group of row tiles
    tm = first_m + r % left;
    tn = r / left;
  }
}

}  // namespace lin
}  // namespace lmbp
