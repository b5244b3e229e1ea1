// Products of groups of rows, one matrix W_e [n, k] for the rows p of each group e:
//   forward     y_p  = W_e x_p
//   gradient    dx_p = W_e^T dy_p,    dW_e = sum over its rows of dy_p x_p^T
// bf16 operands, exact products, fp32 sums, one rounding.
//
// One kernel computes a tile [BB output rows, BA output columns] from two operands in LDS, blocks
// of 64 of the reduction at a time.  The output's columns are the matrix instruction's rows (A),
// the output's rows its columns (B), so a lane's four results are neighbours in a row of the
// output.  An operand lies either along the reduction (rows of x, dy, and of W going forward) or
// across it (W in dx, both operands of dW); what lies across is read from LDS by transposing
// loads, four reductions of one column in each.  Loads go straight to LDS, 16 bytes a lane; 16-byte
// pieces are swapped within a row so that the reads of the instruction's operands hit
// all banks; past the reduction's end they take zeros from a row of zeros, so that what lies there
// (another group's values, infinities too) has no part.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "groups.h"
#include "tiles.h"

namespace xs {
namespace {

enum Kind { kForward, kGradX, kGradW };

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
};

template <Kind kKind, int BA, int BB, int WA, int WB, int kStages>
__global__ __launch_bounds__(64 * WA * WB) void tile_kernel(Product a) {
  constexpr bool kAcrossA = kKind != kForward, kAcrossB = kKind == kGradW;
  constexpr int kThreads = 64 * WA * WB;
  constexpr int MA = BA / WA / 16, MB = BB / WB / 16;
  // Going forward the columns of two neighbouring A tiles are dealt so that a lane's eight results
  // are neighbours: row i = 4 a + b of tile m is column 8 a + 4 (m % 2) + b of the pair.
  constexpr bool kSpread = !kAcrossA && MA % 2 == 0;
  using OpA = Operand<kAcrossA, kSpread, BA, kThreads>;
  using OpB = Operand<kAcrossB, false, BB, kThreads>;
  constexpr int kLoads = OpA::kLoads + OpB::kLoads;
  constexpr int kStage = (BA + BB) * kBlock;
  extern __shared__ __attribute__((aligned(16))) uint16_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wa = wave % WA, wb = wave / WA;
  const int n = lane & 15, g = lane >> 4;

  int e, first, live, c0, reduction;
  if constexpr (kKind == kGradW) {
    const int per = a.column_tiles * a.row_tiles;
    e = blockIdx.x / per;
    const int at = blockIdx.x % per;
    first = at / a.column_tiles * BB;                  // row of dW_e
    c0 = at % a.column_tiles * BA;
    live = min(BB, a.out_rows - first);
  } else {
    Place p;
    if (!find_place(a.offsets, a.E, a.P, BB, a.column_tiles, p)) return;
    e = __builtin_amdgcn_readfirstlane(p.e);
    first = __builtin_amdgcn_readfirstlane(p.first);
    live = __builtin_amdgcn_readfirstlane(p.live);
    c0 = __builtin_amdgcn_readfirstlane(p.column) * BA;
  }
  OpA oa;
  OpB ob;
  const int live_columns = min(BA, a.columns - c0);
  if constexpr (kKind == kForward) {
    reduction = a.reduction;
    oa.init(a.a + ((size_t)e * a.columns + c0) * reduction, reduction, live_columns, reduction, tid);
    ob.init(a.b + (size_t)first * a.ldb, a.ldb, live, reduction, tid);
  } else if constexpr (kKind == kGradX) {
    reduction = a.reduction;
    oa.init(a.a + (size_t)e * a.columns * reduction + c0, a.columns, live_columns, reduction, tid);
    ob.init(a.b + (size_t)first * a.ldb, a.ldb, live, reduction, tid);
  } else {
    int lo, hi;
    group_rows(a.offsets, e, a.P, lo, hi);
    lo = __builtin_amdgcn_readfirstlane(lo);
    reduction = __builtin_amdgcn_readfirstlane(hi) - lo;
    oa.init(a.a + (size_t)lo * a.lda + c0, a.lda, live_columns, reduction, tid);
    ob.init(a.b + (size_t)lo * a.ldb + first, a.ldb, live, reduction, tid);
  }
  const int blocks = (reduction + kBlock - 1) / kBlock;

  floatx4 acc[MA][MB];
#pragma unroll
  for (int m = 0; m < MA; ++m)
#pragma unroll
    for (int t = 0; t < MB; ++t) acc[m][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

  auto load = [&](int b, uint16_t* stage, int i) {
    if (i < OpA::kLoads)
      oa.load(b, stage, i < OpA::kLoads ? i : 0, wave);
    else
      ob.load(b, stage + BA * kBlock, i < OpA::kLoads ? 0 : i - OpA::kLoads, wave);
  };
  auto step = [&](int b, const uint16_t* __restrict__ stage, uint16_t* __restrict__ next) {
    const uint16_t* const sa = stage;
    const uint16_t* const sb = stage + BA * kBlock;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(b + kStages - 1, next, i);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8 fa[MA], fb[MB];
#pragma unroll
      for (int m = 0; m < MA; ++m) {
        if constexpr (kAcrossA) {
          fa[m] = OpA::read_across(sa, (wa * MA + m) * 16, s, n, g);
        } else {
          const int R = kSpread ? wa * MA * 16 + m / 2 * 32 + 8 * (n >> 2) + 4 * (m & 1) + (n & 3)
                                : (wa * MA + m) * 16 + n;
          fa[m] = OpA::read_along(sa, R, s, g);
        }
      }
#pragma unroll
      for (int t = 0; t < MB; ++t) {
        if constexpr (kAcrossB)
          fb[t] = OpB::read_across(sb, (wb * MB + t) * 16, s, n, g);
        else
          fb[t] = OpB::read_along(sb, (wb * MB + t) * 16 + n, s, g);
      }
#pragma unroll
      for (int t = 0; t < MB; ++t)
#pragma unroll
        for (int m = 0; m < MA; ++m)
          acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[m], fb[t], acc[m][t], 0, 0, 0);
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

  // lane (n, g) holds columns 4 g .. 4 g + 3 of column tile m, in row n of row tile t
#pragma unroll
  for (int t = 0; t < MB; ++t) {
    const int r = wb * MB * 16 + 16 * t + n;
    if (r >= live) continue;
    if constexpr (kKind == kGradW) {
      const size_t row = ((size_t)e * a.out_rows + first + r) * a.columns;
#pragma unroll
      for (int m = 0; m < MA; ++m) {
        const int c = c0 + (wa * MA + m) * 16 + 4 * g;
        if (c >= a.columns) continue;                  // (columns come in eights)
        if (a.dw_fp32) {
          floatx4* const out = reinterpret_cast<floatx4*>(static_cast<float*>(a.dw) + row + c);
          *out = a.accumulate ? *out + acc[m][t] : acc[m][t];
        } else {
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.dw) + row + c) =
              make_uint2(to_bf16x2(acc[m][t][0], acc[m][t][1]),
                         to_bf16x2(acc[m][t][2], acc[m][t][3]));
        }
      }
    } else {
      uint16_t* const out = a.out + (size_t)(first + r) * a.ldo;
      if constexpr (kSpread) {
#pragma unroll
        for (int m = 0; m < MA; m += 2) {
          const int c = c0 + wa * MA * 16 + m / 2 * 32 + 8 * g;
          if (c >= a.columns) continue;
          *reinterpret_cast<uint4*>(out + c) =
              make_uint4(to_bf16x2(acc[m][t][0], acc[m][t][1]), to_bf16x2(acc[m][t][2], acc[m][t][3]),
                         to_bf16x2(acc[m + 1][t][0], acc[m + 1][t][1]),
                         to_bf16x2(acc[m + 1][t][2], acc[m + 1][t][3]));
        }
      } else {
#pragma unroll
        for (int m = 0; m < MA; ++m) {
          const int c = c0 + (wa * MA + m) * 16 + 4 * g;
          if (c >= a.columns) continue;
          *reinterpret_cast<uint2*>(out + c) = make_uint2(to_bf16x2(acc[m][t][0], acc[m][t][1]),
                                                          to_bf16x2(acc[m][t][2], acc[m][t][3]));
        }
      }
    }
  }
}

template <Kind kKind, int BA, int BB, int WA, int WB, int kStages>
hipError_t launch_tile(Product a, hipStream_t stream) {
  constexpr int kBytes = kStages * (BA + BB) * kBlock * 2;
  static_assert(kBytes <= 160 * 1024, "LDS of a compute unit");
  const auto kernel = tile_kernel<kKind, BA, BB, WA, WB, kStages>;
  if (kBytes > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != hipSuccess) return e;
  }
  a.column_tiles = (a.columns + BA - 1) / BA;
  a.row_tiles = (a.out_rows + BB - 1) / BB;
  long grid;
  if (kKind == kGradW) {
    grid = (long)a.E * a.column_tiles * a.row_tiles;
  } else {
    const long some = a.P < a.E ? a.P : a.E;           // at most one partly filled tile a group
    grid = ((some + (a.P - some) / BB) * a.column_tiles + 7) / 8 * 8;
  }
  if (grid * 64 * WA * WB > 0xFFFFFFFFl) return hipErrorInvalidConfiguration;
  kernel<<<(unsigned)grid, 64 * WA * WB, kBytes, stream>>>(a);
  return hipGetLastError();
}

Product product_of(const GroupedArgs& g) {
  Product a{};
  a.offsets = g.offsets;
  a.E = g.E;
  a.P = g.P;
  a.out = g.out;
  a.ldo = g.ldo;
  return a;
}

}  // namespace

hipError_t launch_grouped_linear(const GroupedArgs& g, hipStream_t stream) {
  Product a = product_of(g);
  a.columns = g.n;
  a.reduction = g.k;
  a.a = g.w;
  a.b = g.x;
  a.ldb = g.ldx;
  const int mean = g.P / (g.P < g.E ? g.P : g.E);
  if (mean <= 24) return launch_tile<kForward, 64, 32, 4, 1, 4>(a, stream);
  if (mean <= 160) return launch_tile<kForward, 128, 128, 2, 2, 2>(a, stream);
  return launch_tile<kForward, 256, 256, 2, 4, 2>(a, stream);
}

hipError_t launch_grouped_backward_x(const GroupedArgs& g, hipStream_t stream) {
  Product a = product_of(g);
  a.columns = g.k;
  a.reduction = g.n;
  a.a = g.w;
  a.b = g.dy;
  a.ldb = g.lddy;
  const int mean = g.P / (g.P < g.E ? g.P : g.E);
  if (mean <= 24) return launch_tile<kGradX, 64, 32, 4, 1, 4>(a, stream);
  if (mean <= 160) return launch_tile<kGradX, 128, 128, 2, 2, 2>(a, stream);
  return launch_tile<kGradX, 256, 256, 2, 4, 2>(a, stream);
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
  return launch_tile<kGradW, 128, 128, 2, 2, 2>(a, stream);
}

}  // namespace xs
