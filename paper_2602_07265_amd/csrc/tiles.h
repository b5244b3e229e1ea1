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
constexpr uint32_t kPast = 1u << 31;   // bytes that no buffer of a load has

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

// Workgroups go to the eight XCDs in turn.  For `n` pieces of work of which neighbours share operands:
// workgroup i's piece, such that every XCD gets a run of them; -1 where there is none for it.
__device__ __forceinline__ long piece_of(int i, long n) {
  const long per = (n + 7) / 8, at = (i & 7) * per + (i >> 3);
  return (i >> 3) < per && at < n ? at : -1;
}

// Row tiles of `tile` rows, counted over the groups in turn.  Every wave counts them for itself: lane
// l those of groups l span .. l span + span - 1.
struct RowTiles {
  int span, mine, upto;        // groups of a lane; their tiles; those and all before
  int total;
};
__device__ __forceinline__ RowTiles count_row_tiles(const int32_t* offsets, int E, int P, int tile) {
  const int lane = threadIdx.x & 63;
  RowTiles c;
  c.span = (E + 63) / 64;
  c.mine = 0;
  for (int i = 0; i < c.span; ++i) {
    const int e = lane * c.span + i;
    if (e >= E) break;
    int lo, hi;
    group_rows(offsets, e, P, lo, hi);
    c.mine += (hi - lo + tile - 1) / tile;
  }
  c.upto = wave_scan(c.mine);
  c.total = __builtin_amdgcn_readlane(c.upto, 63);
  return c;
}

// A tile of the output: its group, first row, rows, and column tile.
struct Place {
  int e, first, live, column;
};
// The at-th of c.total * columns tiles: four row tiles next to each other, column after column.
__device__ __forceinline__ bool place_of(const int32_t* offsets, int E, int P, int tile, int columns,
                                         const RowTiles& c, long at, Place& p) {
  constexpr int kDeep = 4;
  const int band = (int)(at / ((long)kDeep * columns));
  const int deep = min(kDeep, c.total - band * kDeep);
  const int rest = (int)(at - (long)band * kDeep * columns);
  const int want = band * kDeep + rest % deep;
  p.column = rest / deep;
  const int holder = __builtin_ctzll(__ballot(c.upto > want));
  int left = want - __builtin_amdgcn_readlane(c.upto - c.mine, holder);
  for (int e = holder * c.span; e < E; ++e) {
    int lo, hi;
    group_rows(offsets, e, P, lo, hi);
    const int n = (hi - lo + tile - 1) / tile;
    if (left < n) {
      p.e = __builtin_amdgcn_readfirstlane(e);
      p.first = __builtin_amdgcn_readfirstlane(lo + left * tile);
      p.live = __builtin_amdgcn_readfirstlane(min(tile, hi - p.first));
      p.column = __builtin_amdgcn_readfirstlane(p.column);
      return true;
    }
    left -= n;
  }
  return false;
}
// The tile of workgroup i, of `columns` column tiles of every row tile of `tile` rows; false where
// there is none for it (the grid is an upper bound).
__device__ __forceinline__ bool find_place(const int32_t* offsets, int E, int P, int tile, int columns,
                                           int i, Place& p) {
  const RowTiles c = count_row_tiles(offsets, E, P, tile);
  const long at = piece_of(i, (long)c.total * columns);
  return at >= 0 && place_of(offsets, E, P, tile, columns, c, at, p);
}

// One operand's tile of `kRows` rows or columns of the output, kThreads loading it.
//   along  LDS [kRows][64]: row R's 16-byte piece c lies at c ^ swap(R)
//   across LDS [kB][kRows]: the 16 columns u of reduction q lie at u ^ swap(q)
template <bool kAcross, bool kSpread, int kRows, int kThreads, int kB = kBlock>
struct Operand {
  static_assert(kAcross || kB == kBlock, "rows of 128 bytes");
  static constexpr int kLoads = kRows * kB / 8 / kThreads;
  static constexpr int kPieces = kAcross ? kRows / 8 : 8;       // of an LDS row
  static constexpr int kStep = kThreads / kPieces;              // LDS rows of a load
  static_assert(kRows * kB / 8 % kThreads == 0, "whole loads");
  // kSpread: the instruction's 16 rows lie 8 a + 4 m + b, a, b < 4, apart (see tile_kernel)
  __device__ static __forceinline__ int swap(int R) {
    if constexpr (!kAcross) return kSpread ? (R >> 1 & 1) | (R >> 3 & 3) << 1 : R >> 1 & 7;
    if constexpr (kRows >= 128) return (R & 3) | (R >> 3 & 1) << 2;
    if constexpr (kRows == 64) return (R >> 1 & 1) | (R >> 3 & 1) << 1;
    return kRows == 32 ? R >> 3 & 1 : 0;
  }
  static_assert(kAcross || kStep % 32 == 0, "along, the places in a load's rows are every load's");

  const uint16_t* base;
  long ld;
  int live;                    // rows (along) or columns (across) from base on; none: zeros
  int end;                     // of the reduction
  int at;                      // the lane's first reduction of a block (along)
  uint32_t off[kAcross ? kLoads : 1];   // the lane's, from a block's (along: a load's) start, bytes

  // The column (across) of this lane's place in the LDS rows of load j.
  __device__ static __forceinline__ int column(int tid, int j) {
    return 8 * (tid % kPieces ^ swap(j * kStep + tid / kPieces) << 1);
  }
  // `live` rows (along) or columns (across) from b on, rows l elements apart
  __device__ __forceinline__ void init(const uint16_t* b, long l, int n, int reduction, int tid) {
    base = b;
    ld = l;
    live = n;
    end = reduction;
    const int row = tid / kPieces;
    at = 8 * (tid % kPieces ^ swap(row));
#pragma unroll
    for (int j = 0; j < (kAcross ? kLoads : 1); ++j)
      off[j] = 2 * ((uint32_t)((j * kStep + row) * l) + (kAcross ? column(tid, j) : at));
  }
  // Load j of a block.  Buffer loads give zeros for what lies past the buffer that they are told of:
  // it ends with the last live row's last value.  (Across, columns past the live ones bring the next
  // row's values, to columns of the output that are not there.)
  __device__ __forceinline__ void load(int block, uint16_t* lds, int j, int wave) const {
    const int k = block * kB;
    const uint16_t* from;
    int elements, ahead = 0;
    uint32_t o;
    if constexpr (kAcross) {
      from = base + k * ld;
      elements = live > 0 && end > k ? (min(end - k, kB) - 1) * (int)ld + live : 0;
      o = off[j];
    } else {
      const int rows = live - j * kStep;
      from = base + j * kStep * ld;
      elements = rows > 0 ? (min(rows, kStep) - 1) * (int)ld + end : 0;
      ahead = 2 * k;
      o = at < end - k ? off[0] : kPast;               // (a row's end is no buffer's)
    }
    const auto buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(from), 0,
                                                          2 * elements, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        buffer, (LdsPtr)(lds + j * kThreads * 8 + wave * 512), 16, o, ahead, 0, 0);
  }
  // The instruction's operand: lane (n, g) holds reductions 32 s + 8 g .. + 7 of row (along) R,
  // or of column c0 + n (across).
  __device__ static __forceinline__ bf16x8 read_along(const uint16_t* lds, int R, int s, int g) {
    return *reinterpret_cast<const bf16x8*>(lds + R * kBlock + 8 * ((4 * s + g) ^ swap(R)));
  }
  // (a lane's place in tile u of 16 columns; what a step of four reductions adds is the same for all)
  __device__ static __forceinline__ int across(int u, int n, int g) {
    const int q = 8 * g + (n >> 2);
    return q * kRows + 16 * (u ^ swap(q)) + 4 * (n & 3);
  }
  __device__ static __forceinline__ bf16x8 read_across(const uint16_t* lds, int place, int s) {
    const uint16_t* const p = lds + place + 32 * s * kRows;
    const uint16_t* const p4 = p + 4 * kRows;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)p);
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)p4);
    typedef short i16x8 __attribute__((ext_vector_type(8)));
    const i16x8 both = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(bf16x8, both);
  }
};

}  // namespace
}  // namespace xs
