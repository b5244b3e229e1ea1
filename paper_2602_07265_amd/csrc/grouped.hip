// Products of groups of rows, one matrix W_e [n, k] for the rows p of each group e:
//   forward     y_p  = W_e x_p
//   gradient    dx_p = W_e^T dy_p,    dW_e = sum over its rows of dy_p x_p^T
// bf16 operands, exact products, fp32 sums, one rounding.
//
// A workgroup computes a tile [BB output rows, BA output columns] from two operands in LDS, blocks of
// kB of the reduction at a time.  The output's columns are the matrix instruction's rows (A), the
// output's rows its columns (B), so a lane's four results are neighbours in a row of the output
// (dW's the other way round, see store).  An operand lies either along the reduction (rows of x,
// dy, and of W going forward) or across it (W in dx, both operands of dW); what lies across is
// read from LDS by transposing loads, four reductions of one column in each.  Loads go straight
// to LDS, 16 bytes a lane; 16-byte pieces are swapped within a row so that the reads of the
// instruction's operands hit all banks; each load's buffer ends with the group's last value, so that
// past it (another group's values, infinities too) zeros arrive.
//
// Few rows are bound by the weights' stream (8 rows of 8 (1536, 2048) experts, 50 MB: 10.8 us again and
// again, out of the Infinity Cache, 14.3 us out of memory, where eight calls read 400 MB), many by the
// matrix cores (turns_kernel), dW of many small groups by its stores.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "groups.h"
#include "tiles.h"

namespace xs {
namespace {

enum Kind { kForward, kGradX, kGradW };

constexpr int kUnits = 256;             // compute units of the GPU
constexpr int kTileQuads = 256 * 256 / 4;
// Tiles a unit from which none is split.  Rows of one group by (8192, 4096): 8448, 4.1 rounds, 426 us,
// 460 where none is split from 4 on; 33024, 16.1 rounds, 1611, 1584 if they were; by (8192, 1024) 66000
// rows, 32.3 rounds, 984, and 992.
constexpr int kSplitRounds = 16;

struct Product {
  const int32_t* offsets;
  int E, P;
  int columns;                 // of the output
  int out_rows;                // kGradW: of dW_e
  int reduction;               // kForward, kGradX
  const uint16_t* a;           // W, W, x
  const uint16_t* b;           // x, dy, dy
  long lda, ldb;
  uint16_t* out;               // kForward, kGradX
  long ldo;
  void* dw;
  int dw_fp32, accumulate;
  int column_tiles, row_tiles; // row_tiles: kGradW
  floatx4* sums;               // of parts of tiles (kUnits of 256 x 256), or null: none is split
};

// Where a workgroup's tile lies, and its operands.
struct Tile {
  int e, first, live, c0, reduction;
  int rows_left;               // of the output from the tile's first on, as its operand has them
  int part;                    // of the workspace, which takes its sums; -1: the output does
  const uint16_t *a, *b;       // the tile's first column's (row's) values
  long lda, ldb;
};

// Tiles that are worked on whole: one for every compute unit as often as that goes.  Of the rest
// every tile's reduction is split in so many parts that they are one for every unit again, or in as
// many as have kLeastBlocks blocks each (reduction: the rows of a group on average where it is they).
struct Shares {
  long whole;
  int rest, parts;
};
// With at least 4 blocks 8192 rows of 4 groups by (2312, 1032) take 72.9 us, 62.8 with 8; with 16 8192 rows
// of one by (4104, 1032) 91.7, 89.7 with 8; 22 other products of 300 to 8192 rows take the same, within 1.2 %.
constexpr int kLeastBlocks = 8;
__host__ __device__ inline Shares shares_of(long tiles, int reduction) {
  Shares s{tiles, 0, 1};
  const int rest = (int)(tiles % kUnits);
  if (rest == 0) return s;
  const int by_units = kUnits / rest, by_blocks = reduction / (kBlock * kLeastBlocks);
  const int parts = by_units < by_blocks ? by_units : by_blocks;
  if (parts < 2) return s;
  s.whole = tiles - rest;
  s.rest = rest;
  s.parts = parts;
  return s;
}
template <Kind kKind>
__device__ __forceinline__ int common_reduction(const Product& p) {
  return kKind == kGradW ? p.P / p.E : p.reduction;
}

template <Kind kKind, int BA, int BB>
__device__ __forceinline__ bool tile_at(const Product& p, const RowTiles& c, long at, Tile& t) {
  if constexpr (kKind == kGradW) {
    const int per = p.column_tiles * p.row_tiles;
    t.e = (int)(at / per);
    const int in = (int)(at % per);
    t.first = in / p.column_tiles * BB;                // row of dW_e
    t.c0 = in % p.column_tiles * BA;
    t.rows_left = p.out_rows - t.first;
    t.live = min(BB, t.rows_left);
    int lo, hi;
    group_rows(p.offsets, t.e, p.P, lo, hi);
    lo = __builtin_amdgcn_readfirstlane(lo);
    t.reduction = __builtin_amdgcn_readfirstlane(hi) - lo;
    t.a = p.a + (size_t)lo * p.lda + t.c0;
    t.b = p.b + (size_t)lo * p.ldb + t.first;
    t.lda = p.lda;
  } else {
    Place q;
    if (!place_of(p.offsets, p.E, p.P, BB, p.column_tiles, c, at, q)) return false;
    t.e = q.e;
    t.first = q.first;
    t.rows_left = t.live = q.live;
    t.c0 = q.column * BA;
    t.reduction = p.reduction;
    const size_t group = (size_t)t.e * p.columns * p.reduction;
    t.a = kKind == kForward ? p.a + group + (size_t)t.c0 * p.reduction : p.a + group + t.c0;
    t.lda = kKind == kForward ? p.reduction : p.columns;
    t.b = p.b + (size_t)t.first * p.ldb;
  }
  t.ldb = p.ldb;
  t.part = -1;
  return true;
}
// Part `part` of `parts` of a tile's reduction, in whole blocks of kB.
template <Kind kKind, int kB>
__device__ __forceinline__ void take_part(Tile& t, int part, int parts) {
  const int blocks = (t.reduction + kB - 1) / kB;
  const int from = (int)((long)blocks * part / parts) * kB;
  const int upto = (int)((long)blocks * (part + 1) / parts) * kB;
  t.reduction = min(upto, t.reduction) - from;
  t.a += kKind == kForward ? from : from * t.lda;
  t.b += kKind == kGradW ? from * t.ldb : from;
}
template <Kind kKind, int BB>
__device__ __forceinline__ long count_tiles(const Product& p, RowTiles& c) {
  if constexpr (kKind == kGradW) return (long)p.E * p.column_tiles * p.row_tiles;
  c = count_row_tiles(p.offsets, p.E, p.P, BB);
  return (long)c.total * p.column_tiles;
}
// This workgroup's tile, or the part of it; false where there is none for it.
template <Kind kKind, int BA, int BB>
__device__ __forceinline__ bool find_tile(const Product& p, Tile& t) {
  RowTiles c;
  const long tiles = count_tiles<kKind, BB>(p, c);
  const Shares s = p.sums ? shares_of(tiles, common_reduction<kKind>(p)) : Shares{tiles, 0, 1};
  const int i = blockIdx.x;
  const long whole = (s.whole + 7) / 8 * 8;            // (kUnits times something, or all)
  if (i < whole) {
    const long at = kKind == kGradW ? (i < s.whole ? i : -1) : piece_of(i, s.whole);
    return at >= 0 && tile_at<kKind, BA, BB>(p, c, at, t);
  }
  const long at = piece_of(i - (int)whole, (long)s.rest * s.parts);
  if (at < 0 || !tile_at<kKind, BA, BB>(p, c, s.whole + at / s.parts, t)) return false;
  take_part<kKind, kBlock>(t, (int)(at % s.parts), s.parts);
  t.part = (int)at;
  return true;
}

// One product of operands; dW's the other way round, so that a lane's results are a column's.
template <Kind kKind>
__device__ __forceinline__ floatx4 multiply_add(const bf16x8& a, const bf16x8& b, const floatx4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(kKind == kGradW ? b : a, kKind == kGradW ? a : b, c, 0,
                                                 0, 0);
}

// The results of 16 output rows from r0 on and MA column tiles from column c on.  Lane (n, g) holds
// columns 4 g .. 4 g + 3 of each tile in row n; kSpread: of the pairs that tile_kernel deals; kGradW:
// rows 4 g .. 4 g + 3 of column n, so that 16 lanes store 64 neighbouring bytes and not 16 of each of 16
// rows (dW of 128 groups of 256 rows by (1536, 2048): 471 us, 558 the other way, of which 273 are the
// stores alone; 64 of 64 rows by (2048, 1536): 158 us, 191.  y and dx took no less time so).  In bf16
// the two take 482 and 176 us.  Added to dW they take 1546 and 766: a lane's values are read, added and
// stored one after the other; one group of 8192 rows by (4096, 4096) 248, 226 if it is not added.
template <Kind kKind, bool kSpread, int MA>
__device__ __forceinline__ void store(const Product& a, const Tile& t, int r0, int c, int n, int g,
                                      const floatx4 (&v)[MA]) {
  if constexpr (kKind == kGradW) {
    const size_t first = ((size_t)t.e * a.out_rows + t.first + r0 + 4 * g) * a.columns;
    const int live = t.live - r0 - 4 * g;
    if (a.dw_fp32) {
      auto rows = [&](auto accumulate) {               // (one question, not one for each value)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float* const out = static_cast<float*>(a.dw) + first + (size_t)j * a.columns;
#pragma unroll
          for (int m = 0; m < MA; ++m) {
            const int at = c + 16 * m + n;
            if (j < live && at < a.columns) out[at] = accumulate ? out[at] + v[m][j] : v[m][j];
          }
        }
      };
      if (a.accumulate)
        rows(std::true_type());
      else
        rows(std::false_type());
    } else {
      const bool odd = n & 1;                          // two columns of rows j (even lanes), j + 1 (odd)
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        const int row = j + odd;
        uint16_t* const out = static_cast<uint16_t*>(a.dw) + first + (size_t)row * a.columns;
#pragma unroll
        for (int m = 0; m < MA; ++m) {
          const int at = c + 16 * m + (n & ~1);
          const float mine = odd ? v[m][j + 1] : v[m][j], other = odd ? v[m][j] : v[m][j + 1];
          const float next = __int_as_float(
              __builtin_amdgcn_mov_dpp(__float_as_int(other), 0xB1, 0xF, 0xF, true));  // lane n ^ 1's
          if (row < live && at < a.columns)
            *reinterpret_cast<uint32_t*>(out + at) = to_bf16x2(odd ? next : mine, odd ? mine : next);
        }
      }
    }
  } else {
    const int r = r0 + n;
    if (r >= t.live) return;
    uint16_t* const out = a.out + (size_t)(t.first + r) * a.ldo;
    if constexpr (kSpread) {
#pragma unroll
      for (int m = 0; m < MA; m += 2) {
        const int at = c + 16 * m + 8 * g;
        if (at >= a.columns) continue;
        *reinterpret_cast<uint4*>(out + at) =
            make_uint4(to_bf16x2(v[m][0], v[m][1]), to_bf16x2(v[m][2], v[m][3]),
                       to_bf16x2(v[m + 1][0], v[m + 1][1]), to_bf16x2(v[m + 1][2], v[m + 1][3]));
      }
    } else {
#pragma unroll
      for (int m = 0; m < MA; ++m) {
        const int at = c + 16 * m + 4 * g;
        if (at < a.columns)
          *reinterpret_cast<uint2*>(out + at) =
              make_uint2(to_bf16x2(v[m][0], v[m][1]), to_bf16x2(v[m][2], v[m][3]));
      }
    }
  }
}

// BA columns by BB rows; WA waves along the columns by WB along the rows; kGroups such groups of waves,
// each with a part of the reduction and buffers of its own, whose sums meet in LDS.
template <Kind kKind, int BA, int BB, int WA, int WB, int kStages, int kB, int kGroups>
__global__ __launch_bounds__(64 * WA * WB * kGroups) void tile_kernel(Product a) {
  constexpr bool kAcrossA = kKind != kForward, kAcrossB = kKind == kGradW;
  constexpr int kThreads = 64 * WA * WB;
  constexpr int MA = BA / WA / 16, MB = BB / WB / 16;
  // Going forward the columns of two neighbouring A tiles are dealt so that a lane's eight results
  // are neighbours: row i = 4 a + b of tile m is column 8 a + 4 (m % 2) + b of the pair.
  constexpr bool kSpread = !kAcrossA && MA % 2 == 0;
  using OpA = Operand<kAcrossA, kSpread, BA, kThreads, kB>;
  using OpB = Operand<kAcrossB, false, BB, kThreads, kB>;
  constexpr int kLoads = OpA::kLoads + OpB::kLoads;
  constexpr int kStage = (BA + BB) * kB;
  extern __shared__ __attribute__((aligned(16))) uint16_t lds_of_all[];
  const int tid = threadIdx.x % kThreads, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
  uint16_t* const lds = lds_of_all + group * kStages * kStage;
  const int wa = wave % WA, wb = wave / WA;
  const int n = lane & 15, g = lane >> 4;

  Tile tile;
  if (!find_tile<kKind, BA, BB>(a, tile)) return;     // (its parts are turns_kernel's alone)
  // (every group takes as many steps, for they meet at the barriers)
  const int blocks = ((tile.reduction + kB - 1) / kB + kGroups - 1) / kGroups;
  if constexpr (kGroups > 1) take_part<kKind, kB>(tile, group, kGroups);
  const int reduction = tile.reduction;
  OpA oa;
  OpB ob;
  oa.init(tile.a, tile.lda, a.columns - tile.c0, reduction, tid);
  ob.init(tile.b, tile.ldb, tile.rows_left, reduction, tid);

  floatx4 acc[MA][MB];
#pragma unroll
  for (int m = 0; m < MA; ++m)
#pragma unroll
    for (int t = 0; t < MB; ++t) acc[m][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

  auto load = [&](int b, uint16_t* stage, int i) {
    if (i < OpA::kLoads)
      oa.load(b, stage, i < OpA::kLoads ? i : 0, wave);
    else
      ob.load(b, stage + BA * kB, i < OpA::kLoads ? 0 : i - OpA::kLoads, wave);
  };
  auto step = [&](int b, const uint16_t* __restrict__ stage, uint16_t* __restrict__ next) {
    const uint16_t* const sa = stage;
    const uint16_t* const sb = stage + BA * kB;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(b + kStages - 1, next, i);
#pragma unroll
    for (int s = 0; s < kB / 32; ++s) {
      bf16x8 fa[MA], fb[MB];
#pragma unroll
      for (int m = 0; m < MA; ++m) {
        if constexpr (kAcrossA) {
          fa[m] = OpA::read_across(sa, OpA::across(wa * MA + m, n, g), s);
        } else {
          const int R = kSpread ? wa * MA * 16 + m / 2 * 32 + 8 * (n >> 2) + 4 * (m & 1) + (n & 3)
                                : (wa * MA + m) * 16 + n;
          fa[m] = OpA::read_along(sa, R, s, g);
        }
      }
#pragma unroll
      for (int t = 0; t < MB; ++t) {
        if constexpr (kAcrossB)
          fb[t] = OpB::read_across(sb, OpB::across(wb * MB + t, n, g), s);
        else
          fb[t] = OpB::read_along(sb, (wb * MB + t) * 16 + n, s, g);
      }
#pragma unroll
      for (int t = 0; t < MB; ++t)
#pragma unroll
        for (int m = 0; m < MA; ++m)
          acc[m][t] = multiply_add<kKind>(fa[m], fb[t], acc[m][t]);
    }
  };
  if (blocks > 0) {
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load(s, lds + s * kStage, i);
    int cur = 0;                                       // the buffer of block b
    for (int b = 0; b < blocks; ++b) {
      wait_loads<kLoads*(kStages - 2)>();
      step(b, lds + cur * kStage, lds + (cur == 0 ? kStages - 1 : cur - 1) * kStage);
      cur = cur + 1 == kStages ? 0 : cur + 1;
    }
    wait_loads<0>();
  }

  if constexpr (kGroups > 1) {
    floatx4* const sums = reinterpret_cast<floatx4*>(lds_of_all) + tid;
    if (group > 0)
#pragma unroll
      for (int i = 0; i < MA * MB; ++i)
        sums[((group - 1) * MA * MB + i) * kThreads] = acc[i / MB][i % MB];
    __syncthreads();
    if (group > 0) return;
    for (int q = 0; q < kGroups - 1; ++q)
#pragma unroll
      for (int i = 0; i < MA * MB; ++i)
        acc[i / MB][i % MB] += sums[(q * MA * MB + i) * kThreads];
  }
#pragma unroll
  for (int t = 0; t < MB; ++t) {
    floatx4 v[MA];
#pragma unroll
    for (int m = 0; m < MA; ++m) v[m] = acc[m][t];
    store<kKind, kSpread>(a, tile, wb * MB * 16 + 16 * t, tile.c0 + wa * MA * 16, n, g, v);
  }
}

// Tiles of 256 x 256, eight waves of 128 columns by 64 rows, in two groups that take turns: while one
// works through the matrix instructions of a quarter of its block, the other reads the operands of its
// next quarter from LDS and starts loads.  Either operand has two halves of 128 rows (columns); a
// wave has 64 columns and 32 rows of each.  A half is loaded for the block after the next as soon
// as both groups have read it, so that two buffers hold almost two blocks of loads in flight.
//
// Bound by the matrix cores: 4096 rows of one group by (4096, 4096) take 101 us (1.36 PFLOP/s; a large
// library product 1.43), dx 113 (1.22), dW 124 (1.11).  In tiles of 128 x 128, two workgroups a unit,
// whose waves read an operand from LDS twice as often for a product, the first took 150.
template <Kind kKind>
__global__ __launch_bounds__(512, 2) void turns_kernel(Product a) {
  constexpr bool kAcrossA = kKind != kForward, kAcrossB = kKind == kGradW;
  constexpr bool kSpread = !kAcrossA;
  using OpA = Operand<kAcrossA, kSpread, 128, 512>;
  using OpB = Operand<kAcrossB, false, 128, 512>;
  constexpr int kHalf = 128 * kBlock;                  // elements of a half
  constexpr int kStage = 4 * kHalf;                    // A's halves, B's halves
  extern __shared__ __attribute__((aligned(16))) uint16_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wa = wave & 1, wb = wave >> 1;
  const int n = lane & 15, g = lane >> 4;
  Tile tile;
  if (!find_tile<kKind, 256, 256>(a, tile)) return;
  const int reduction = tile.reduction;
  OpA oa[2];
  OpB ob[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    oa[h].init(tile.a + 128 * h * (kAcrossA ? 1 : tile.lda), tile.lda, a.columns - tile.c0 - 128 * h,
               reduction, tid);
    ob[h].init(tile.b + 128 * h * (kAcrossB ? 1 : tile.ldb), tile.ldb, tile.rows_left - 128 * h,
               reduction, tid);
  }
  const int blocks = (reduction + kBlock - 1) / kBlock;
  floatx4 acc[2][2][2][4];                             // A's half, B's half, row tile, column tile
#pragma unroll
  for (int i = 0; i < 2 * 2 * 2 * 4; ++i)
    acc[i >> 4][i >> 3 & 1][i >> 2 & 1][i & 3] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  bf16x8 fa[2][2][4], fb[2][2][2];                     // half, 32 of the block, tile

  int place_a[4], place_b[2];                          // of what lies across the reduction
#pragma unroll
  for (int m = 0; m < 4; ++m) place_a[m] = OpA::across(wa * 4 + m, n, g);
#pragma unroll
  for (int t = 0; t < 2; ++t) place_b[t] = OpB::across(wb * 2 + t, n, g);
  auto read_a = [&](int h, int s, const uint16_t* __restrict__ from) {
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      if constexpr (kAcrossA)
        fa[h][s][m] = OpA::read_across(from, place_a[m], s);
      else
        fa[h][s][m] = OpA::read_along(
            from, wa * 64 + m / 2 * 32 + 8 * (n >> 2) + 4 * (m & 1) + (n & 3), s, g);
    }
  };
  auto read_b = [&](int h, const uint16_t* __restrict__ from) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if constexpr (kAcrossB)
          fb[h][s][t] = OpB::read_across(from, place_b[t], s);
        else
          fb[h][s][t] = OpB::read_along(from, wb * 32 + 16 * t + n, s, g);
      }
  };
  auto load_a = [&](int b, int h, uint16_t* __restrict__ to) {
    oa[h].load(b, to, 0, wave);
    oa[h].load(b, to, 1, wave);
  };
  auto load_b = [&](int b, int h, uint16_t* __restrict__ to) {
    ob[h].load(b, to, 0, wave);
    ob[h].load(b, to, 1, wave);
  };
  // The end of a quarter's reads: they are done, and all but N loads; then the other group's turn.
  auto meet = [&](auto loads) {
    constexpr int N = decltype(loads)::value;
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (N >= 0)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N >= 0 ? N : 0) : "memory");
    else
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto multiply = [&](int ha, int hb) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int m = 0; m < 4; ++m)
          acc[ha][hb][t][m] =
              multiply_add<kKind>(fa[ha][s][m], fb[hb][s][t], acc[ha][hb][t][m]);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  std::integral_constant<int, -1> reads;
  std::integral_constant<int, 6> six;
  std::integral_constant<int, 8> eight;
  std::integral_constant<int, 12> twelve;
  // One block, a quarter of its products a turn: what a turn reads was loaded two blocks ago, and what
  // all have read by then is loaded for the block after the next.
  auto block = [&](int b, uint16_t* __restrict__ here, uint16_t* __restrict__ other) {
    read_b(0, here + 2 * kHalf);
    read_a(0, 1, here);
    meet(reads);
    multiply(0, 0);
    read_b(1, here + 3 * kHalf);
    read_a(1, 0, here + kHalf);
    __builtin_amdgcn_sched_barrier(0);
    load_a(b + 2, 0, here);
    meet(reads);
    multiply(0, 1);
    read_a(1, 1, here + kHalf);
    __builtin_amdgcn_sched_barrier(0);
    load_b(b + 2, 0, here + 2 * kHalf);
    load_b(b + 2, 1, here + 3 * kHalf);
    meet(twelve);                                      // the next block's first half of A is there
    multiply(1, 1);
    read_a(0, 0, other);
    __builtin_amdgcn_sched_barrier(0);
    load_a(b + 2, 1, here + kHalf);
    meet(eight);                                       // and the rest of it
    multiply(1, 0);
  };
  // The same without the second half of B, which holds no rows: two turns (the three products
  // of 554 rows of 12 groups by (2104, 9304) take 196 us, without it 257).
  auto half_block = [&](int b, uint16_t* __restrict__ here, uint16_t* __restrict__ other) {
    read_b(0, here + 2 * kHalf);
    read_a(0, 0, here);
    read_a(0, 1, here);
    __builtin_amdgcn_sched_barrier(0);
    load_a(b + 1, 1, other + kHalf);
    meet(six);                                         // this block's second half of A is there
    multiply(0, 0);
    read_a(1, 0, here + kHalf);
    read_a(1, 1, here + kHalf);
    __builtin_amdgcn_sched_barrier(0);
    load_a(b + 2, 0, here);
    load_b(b + 2, 0, here + 2 * kHalf);
    meet(six);                                         // and the next one's other halves
    multiply(1, 0);
  };
  if (blocks > 0 && tile.live <= 128) {
    load_a(0, 0, lds);
    load_b(0, 0, lds + 2 * kHalf);
    load_a(0, 1, lds + kHalf);
    load_a(1, 0, lds + kStage);
    load_b(1, 0, lds + kStage + 2 * kHalf);
    meet(six);
    if (wave >= 4) meet(reads);                        // the second group comes a turn later
#pragma unroll 1
    for (int b = 0; b < blocks; ++b) {
      const int here = (b & 1) * kStage;
      half_block(b, lds + here, lds + (kStage - here));
    }
    if (wave < 4) meet(reads);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load outlives the workgroup's LDS
  } else if (blocks > 0) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      load_a(b, 0, lds + b * kStage);
      load_b(b, 0, lds + b * kStage + 2 * kHalf);
      load_b(b, 1, lds + b * kStage + 3 * kHalf);
      load_a(b, 1, lds + b * kStage + kHalf);
    }
    meet(eight);
    read_a(0, 0, lds);
    if (wave >= 4) meet(reads);                        // the second group comes a turn later
#pragma unroll 1
    for (int b = 0; b < blocks; ++b) {
      const int here = (b & 1) * kStage;
      block(b, lds + here, lds + (kStage - here));
    }
    if (wave < 4) meet(reads);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load outlives the workgroup's LDS
  }
  if (tile.part >= 0) {
    floatx4* const to = a.sums + (size_t)tile.part * kTileQuads + tid;
#pragma unroll
    for (int i = 0; i < 32; ++i) to[i * 512] = acc[i >> 4][i >> 3 & 1][i >> 2 & 1][i & 3];
    return;
  }
#pragma unroll
  for (int hb = 0; hb < 2; ++hb)
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int ha = 0; ha < 2; ++ha)
        store<kKind, kSpread>(a, tile, hb * 128 + wb * 32 + 16 * t, tile.c0 + ha * 128 + wa * 64, n, g,
                              acc[ha][hb][t]);
}

// The parts of the tiles that turns_kernel splits, summed in order and stored: workgroup (quarter,
// tile), the threads' values as in that kernel.
template <Kind kKind>
__global__ __launch_bounds__(512) void join_kernel(Product a) {
  constexpr bool kSpread = kKind == kForward;
  RowTiles c;
  const long tiles = count_tiles<kKind, 256>(a, c);
  const Shares s = shares_of(tiles, common_reduction<kKind>(a));
  Tile tile;
  if ((int)blockIdx.y >= s.rest || !tile_at<kKind, 256, 256>(a, c, s.whole + blockIdx.y, tile)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wa = wave & 1, wb = wave >> 1, hb = blockIdx.x >> 1, t = blockIdx.x & 1;
  const floatx4* from = a.sums + (size_t)blockIdx.y * s.parts * kTileQuads + tid;
#pragma unroll
  for (int ha = 0; ha < 2; ++ha) {
    floatx4 v[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) v[m] = from[(16 * ha + 8 * hb + 4 * t + m) * 512];
    for (int p = 1; p < s.parts; ++p)
#pragma unroll
      for (int m = 0; m < 4; ++m)
        v[m] += from[(size_t)p * kTileQuads + (16 * ha + 8 * hb + 4 * t + m) * 512];
    store<kKind, kSpread>(a, tile, hb * 128 + wb * 32 + 16 * t, tile.c0 + ha * 128 + wa * 64, lane & 15,
                          lane >> 4, v);
  }
}

// The most tiles of BA x BB that there can be.
template <Kind kKind, int BA, int BB>
long most_tiles(Product& a) {
  a.column_tiles = (a.columns + BA - 1) / BA;
  a.row_tiles = (a.out_rows + BB - 1) / BB;
  if (kKind == kGradW) return (long)a.E * a.column_tiles * a.row_tiles;
  const long some = a.P < a.E ? a.P : a.E;             // at most one partly filled tile a group
  return (some + (a.P - some) / BB) * a.column_tiles;
}

template <typename F>
hipError_t launch(const Product& a, F kernel, long grid, int threads, int bytes,
                  hipStream_t stream) {
  if (bytes > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  grid = (grid + 7) / 8 * 8;
  if (grid * threads > 0xFFFFFFFFl) return hipErrorInvalidConfiguration;
  kernel<<<(unsigned)grid, threads, bytes, stream>>>(a);
  return hipGetLastError();
}

template <Kind kKind, int BA, int BB, int WA, int WB, int kStages, int kB = kBlock, int kGroups = 1>
hipError_t launch_tile(Product a, hipStream_t stream) {
  constexpr int kBytes = kGroups * kStages * (BA + BB) * kB * 2;
  static_assert((kGroups - 1) * BA * BB * 4 <= kBytes, "the groups' sums");
  static_assert(kBytes <= 160 * 1024, "LDS of a compute unit");
  a.sums = nullptr;
  const long tiles = most_tiles<kKind, BA, BB>(a);
  return launch(a, tile_kernel<kKind, BA, BB, WA, WB, kStages, kB, kGroups>, tiles,
                64 * WA * WB * kGroups, kBytes, stream);
}

template <Kind kKind>
hipError_t launch_turns(Product a, hipStream_t stream) {
  const long tiles = most_tiles<kKind, 256, 256>(a);
  if (tiles > kSplitRounds * kUnits) a.sums = nullptr; // (the last round is a small part)
  const long more = a.sums ? kUnits : 0;               // parts in place of the rest
  const hipError_t e =
      launch(a, turns_kernel<kKind>, tiles + more, 512, 2 * 512 * kBlock * 2, stream);
  if (e != hipSuccess || !a.sums) return e;
  const long rest = tiles < kUnits ? tiles : kUnits - 1;
  join_kernel<kKind><<<dim3(4, (unsigned)rest), 512, 0, stream>>>(a);
  return hipGetLastError();
}

// The forms of a product: its tile, and what it costs in microseconds: 64 of the reduction, `few` with
// little else on the GPU, `full` for each tile that every compute unit has to work on, and `out`, what a
// tile takes besides (finding its rows, the first loads, the stores).  Measured over 1 to 256 groups of
// 1 to 16384 rows by ten shapes of 72 to 10304; there the rule's choice took 3.5 % (forward), 4.7 % (dx)
// and 2.1 % (dW) longer than the fastest form on average, and within 10 % of it in 160 of 184, 147 of
// 178 and 299 of 325.
// Both sides, in the forms' order without the first: 64 rows of one group by (4096, 4096) 15.7, 18.5,
// 23.7 and 70 us (29.7 split); 1024 rows 73, 53, 43 and 76 (53); 4096 rows 285, 195, 154 and 97 (99);
// 512 rows in each of 8 groups 349, 268, 220 and 172 (149).  The first against the second: one row by
// (256, 10304) 22.7 and 32 us.  dW of 256 rows in each of 64 groups by (7592, 344) 425, 353, 280 and
// 293 us; of 4096 rows in each of 4 by (512, 4096) 90, 86, 158 and 109.
enum Units { kShared, kAlone, kSplit };  // tiles of a unit: several, one, one and the last round split
struct Form {
  int columns, rows;
  float few, full, out;
  Units units;
  hipError_t (*launch)(Product, hipStream_t);
};
const Form kForwardForms[] = {
    {64, 32, 0.122f, 0.145f, 1.2f, kShared, launch_tile<kForward, 64, 32, 4, 1, 3, 64, 2>},
    {64, 32, 0.185f, 0.13f, 0.6f, kShared, launch_tile<kForward, 64, 32, 4, 1, 4>},
    {64, 64, 0.23f, 0.19f, 0.65f, kShared, launch_tile<kForward, 64, 64, 2, 2, 3>},
    {128, 64, 0.30f, 0.32f, 1.4f, kShared, launch_tile<kForward, 128, 64, 2, 2, 3>},
    {256, 256, 1.07f, 1.4f, 9.0f, kSplit, launch_turns<kForward>},
};
const Form kGradXForms[] = {
    {64, 32, 0.155f, 0.15f, 1.2f, kShared, launch_tile<kGradX, 64, 32, 4, 1, 3, 64, 2>},
    {64, 32, 0.225f, 0.13f, 0.6f, kShared, launch_tile<kGradX, 64, 32, 4, 1, 4>},
    {64, 64, 0.25f, 0.19f, 0.7f, kShared, launch_tile<kGradX, 64, 64, 2, 2, 3>},
    {128, 64, 0.38f, 0.31f, 1.4f, kShared, launch_tile<kGradX, 128, 64, 2, 2, 3>},
    {256, 256, 1.30f, 1.55f, 12.0f, kSplit, launch_turns<kGradX>},
};
const Form kGradWForms[] = {
    {128, 64, 0.46f, 0.41f, 1.4f, kShared, launch_tile<kGradW, 128, 64, 2, 2, 3, 32>},
    {128, 128, 0.92f, 0.51f, 3.1f, kShared, launch_tile<kGradW, 128, 128, 2, 2, 3, 32>},
    {256, 256, 2.53f, 1.48f, 12.5f, kAlone, launch_tile<kGradW, 256, 256, 2, 4, 4, 32>},
    {256, 256, 0.77f, 1.33f, 20.4f, kSplit, launch_turns<kGradW>},
};

float form_cost(const Form& f, float out, float tiles, int reduction) {
  const float blocks = (float)((reduction + kBlock - 1) / kBlock);
  if (f.units == kShared) {
    const float round = tiles / kUnits, full = blocks * f.full + out;
    float some = blocks * f.few;
    if (full > some) some += (full - some) * (round < 1 ? round : 1);
    return full * round > some ? full * round : some;
  }
  Shares s{(long)(tiles + 0.999f), 0, 1};
  if (f.units == kSplit) s = shares_of(s.whole, reduction);
  const long rounds = (s.whole + kUnits - 1) / kUnits;
  const int left = (int)(s.whole - (rounds - 1) * kUnits);       // tiles of the last whole round
  float cost = rounds * (blocks * f.full + out);
  if (rounds > 0) cost -= (blocks * (f.full - f.few) + out) * (1.0f - (float)left / kUnits);
  if (s.rest == 0) return cost;
  const int more = s.rest * s.parts;                   // parts, each written and read again
  return cost + blocks * (f.few + (f.full - f.few) * more / kUnits) / s.parts + 4.0f + 0.1f * more;
}

template <int N>
const Form& form_for(const Form (&forms)[N], const Product& a, int groups, int reduction) {
  int best = 0;
  float least = 0;
  for (int i = 0; i < N; ++i) {
    const Form& f = forms[i];
    if (f.units == kSplit && a.P < kTurnsRows) continue;
    const int columns = (a.columns + f.columns - 1) / f.columns;
    // the rows of dW, or of groups: their last tile is half full on average (one's size is known);
    // turns_kernel works on that in halves
    const float mean = (float)a.P / groups, last = f.units == kSplit ? 0.25f : 0.5f;
    const float rows = a.out_rows ? (float)((a.out_rows + f.rows - 1) / f.rows)
                       : groups == 1 ? (float)((a.P + f.rows - 1) / f.rows)
                       : mean > 1 ? mean / f.rows + last : 1.0f;
    // of dW's tiles, much of which is their stores, the part that is there
    const float cover =
        a.out_rows ? (float)a.columns * a.out_rows / ((float)columns * f.columns * rows * f.rows) : 1.0f;
    const float cost =
        form_cost(f, f.out * cover, (float)groups * columns * (rows > 1 ? rows : 1.0f), reduction);
    if (i == 0 || cost < least) {
      best = i;
      least = cost;
    }
  }
  return forms[best];
}

Product product_of(const GroupedArgs& g) {
  Product a{};
  a.offsets = g.offsets;
  a.E = g.E;
  a.P = g.P;
  a.out = g.out;
  a.ldo = g.ldo;
  a.sums = reinterpret_cast<floatx4*>(g.sums);
  return a;
}

template <int N>
hipError_t launch_rows(const Form (&forms)[N], const Product& a, hipStream_t stream) {
  const int groups = a.P < a.E ? a.P : a.E;
  return form_for(forms, a, groups, a.reduction).launch(a, stream);
}

}  // namespace

hipError_t launch_grouped_linear(const GroupedArgs& g, hipStream_t stream) {
  Product a = product_of(g);
  a.columns = g.n;
  a.reduction = g.k;
  a.a = g.w;
  a.b = g.x;
  a.ldb = g.ldx;
  return launch_rows(kForwardForms, a, stream);
}

hipError_t launch_grouped_backward_x(const GroupedArgs& g, hipStream_t stream) {
  Product a = product_of(g);
  a.columns = g.k;
  a.reduction = g.n;
  a.a = g.w;
  a.b = g.dy;
  a.ldb = g.lddy;
  return launch_rows(kGradXForms, a, stream);
}

hipError_t launch_grouped_backward_w(const GroupedArgs& g, hipStream_t stream) {
  Product a = product_of(g);
  a.columns = g.k;
  a.out_rows = g.n;
  a.a = g.x;
  a.lda = g.ldx;
  a.b = g.dy;
  a.ldb = g.lddy;
  a.dw = g.dw;
  a.dw_fp32 = g.dw_fp32;
  a.accumulate = g.accumulate;
  const int mean = a.P / a.E;
  return form_for(kGradWForms, a, a.E, mean > 0 ? mean : 1).launch(a, stream);
}

}  // namespace xs
