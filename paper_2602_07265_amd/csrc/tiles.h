// What the kernels of groups of rows share: bf16 matrix operands in LDS, loaded without registers in
// between, and the finding of a workgroup's group and rows.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "wave.h"

namespace xs {
namespace {

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
using GlobalPtr = const __attribute__((address_space(1))) void*;
using LdsPtr = __attribute__((address_space(3))) void*;
using LdsQuad = __attribute__((address_space(3))) i16x4*;

constexpr int kBlock = 64;     // of the reduction

__device__ const uint4 kZeros[1] = {{0, 0, 0, 0}};

__device__ __forceinline__ uint16_t to_bf16(float v) {
  uint32_t b = __float_as_uint(v);
  if ((b & 0x7FFFFFFFu) > 0x7F800000u) return 0x7FC0u;
  b += 0x7FFFu + ((b >> 16) & 1u);   // round to nearest even
  return (uint16_t)(b >> 16);
}
__device__ __forceinline__ uint32_t to_bf16x2(float lo, float hi) {
  return to_bf16(lo) | (uint32_t)to_bf16(hi) << 16;
}

__device__ __forceinline__ void to_lds(const uint16_t* src, uint16_t* dst) {
  __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)dst, 16, 0, 0);
}
// All but this wave's last N loads are done, and those of the workgroup's other waves too; nor does
// any wave still read LDS.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Group e's rows; what the offsets say is kept inside the buffers.
__device__ __forceinline__ void group_rows(const int32_t* offsets, int e, int P, int& lo, int& hi) {
  lo = min(max(offsets[e], 0), P);
  hi = max(lo, min(offsets[e + 1], P));
}

// A row tile: its group, first row and rows; tiles are counted over the groups in turn, and the
// columns' tiles within them, near ones to the same XCD.
struct Place {
  int e, first, live, column;
};
// The place of this workgroup among `columns` column tiles of every row tile of `tile` rows; false
// where there is none for it (the grid is an upper bound).  Every wave finds it for itself: lane
// l counts the tiles of groups l S .. l S + S - 1.
__device__ __forceinline__ bool find_place(const int32_t* offsets, int E, int P, int tile, int columns,
                                           Place& p) {
  const int lane = threadIdx.x & 63;
  const int span = (E + 63) / 64;
  int mine = 0;
  for (int i = 0; i < span; ++i) {
    const int e = lane * span + i;
    if (e >= E) break;
    int lo, hi;
    group_rows(offsets, e, P, lo, hi);
    mine += (hi - lo + tile - 1) / tile;
  }
  const int upto = wave_scan(mine);
  const int tiles = __builtin_amdgcn_readlane(upto, 63);
  // workgroups go to the eight XCDs in turn: each gets a run of tiles
  const long all = (long)tiles * columns;
  const int per = (int)((all + 7) / 8);
  const int idx = blockIdx.x >> 3, xcd = blockIdx.x & 7;
  const long at = (long)xcd * per + idx;
  if (idx >= per || at >= all) return false;
  // four row tiles next to each other, column after column
  constexpr int kDeep = 4;
  const int band = (int)(at / ((long)kDeep * columns));
  const int deep = min(kDeep, tiles - band * kDeep);
  const int rest = (int)(at - (long)band * kDeep * columns);
  const int want = band * kDeep + rest % deep;
  p.column = rest / deep;
  const int holder = __builtin_ctzll(__ballot(upto > want));
  int left = want - __builtin_amdgcn_readlane(upto - mine, holder);
  for (int e = holder * span; e < E; ++e) {
    int lo, hi;
    group_rows(offsets, e, P, lo, hi);
    const int n = (hi - lo + tile - 1) / tile;
    if (left < n) {
      p.e = e;
      p.first = lo + left * tile;
      p.live = min(tile, hi - p.first);
      return true;
    }
    left -= n;
  }
  return false;
}

// One operand's tile of `kRows` rows or columns of the output, kThreads loading it.
//   along  LDS [kRows][64]: row R's 16-byte piece c lies at c ^ swap(R)
//   across LDS [64][kRows]: the 16 columns u of reduction q lie at u ^ swap(q)
template <bool kAcross, bool kSpread, int kRows, int kThreads>
struct Operand {
  static constexpr int kLoads = kRows * 8 / kThreads;
  static constexpr int kPieces = kAcross ? kRows / 8 : 8;       // of an LDS row
  static constexpr int kStep = kThreads / kPieces;              // LDS rows of a load
  static_assert(kRows * 8 % kThreads == 0, "whole loads");
  // kSpread: the instruction's 16 rows lie 8 a + 4 m + b, a, b < 4, apart (see tile_kernel)
  __device__ static __forceinline__ int swap(int R) {
    if constexpr (!kAcross) return kSpread ? (R >> 1 & 1) | (R >> 3 & 3) << 1 : R >> 1 & 7;
    if constexpr (kRows >= 128) return (R & 3) | (R >> 3 & 1) << 2;
    if constexpr (kRows == 64) return (R >> 1 & 1) | (R >> 3 & 1) << 1;
    return kRows == 32 ? R >> 3 & 1 : 0;
  }
  const uint16_t* base;
  long ld;
  int end;                     // of the reduction
  uint32_t off[kLoads];        // along: of the lane's rows; across: of its columns
  int piece, row;

  // rows `live` of them from `base`, `ld` elements apart (along); or columns from `base`
  __device__ __forceinline__ void init(const uint16_t* b, long l, int live, int reduction, int tid) {
    base = b;
    ld = l;
    end = reduction;
    row = tid / kPieces;
    const int slot = tid % kPieces;
    if constexpr (kAcross) {
      piece = 0;
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        off[j] = min(8 * (slot ^ swap(j * kStep + row) << 1), live - 8);
    } else {
      piece = 8 * (slot ^ swap(row));
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        off[j] = (uint32_t)(min(j * kStep + row, live - 1) * ld);
    }
  }
  __device__ __forceinline__ void load(int block, uint16_t* lds, int j, int wave) const {
    const int k0 = block * kBlock;
    const uint16_t* src;
    if constexpr (kAcross) {
      const int q = k0 + j * kStep + row;
      src = base + (long)q * ld + off[j];
      if (q >= end) src = reinterpret_cast<const uint16_t*>(kZeros);
    } else {
      src = base + off[j] + k0 + piece;
      if (k0 + piece >= end) src = reinterpret_cast<const uint16_t*>(kZeros);
    }
    to_lds(src, lds + j * kThreads * 8 + wave * 512);
  }
  // The instruction's operand: lane (n, g) holds reductions 32 s + 8 g .. + 7 of row (along) R,
  // or of column c0 + n (across).
  __device__ static __forceinline__ bf16x8 read_along(const uint16_t* lds, int R, int s, int g) {
    return *reinterpret_cast<const bf16x8*>(lds + R * kBlock + 8 * ((4 * s + g) ^ swap(R)));
  }
  __device__ static __forceinline__ bf16x8 read_across(const uint16_t* lds, int c0, int s, int n,
                                                       int g) {
    const int q = 32 * s + 8 * g + (n >> 2);
    const uint16_t* const p = lds + q * kRows + 16 * ((c0 >> 4) ^ swap(q)) + 4 * (n & 3);
    const uint16_t* const p4 = lds + (q + 4) * kRows + 16 * ((c0 >> 4) ^ swap(q + 4)) + 4 * (n & 3);
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)p);
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)p4);
    typedef short i16x8 __attribute__((ext_vector_type(8)));
    const i16x8 both = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(bf16x8, both);
  }
};

}  // namespace
}  // namespace xs
