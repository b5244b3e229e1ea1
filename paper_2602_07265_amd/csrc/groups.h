// Launchers of the pairs' expert order (order.hip), the moves of rows into it and back (move.hip),
// the products of groups of rows (grouped.hip) and the low-rank adapters (adapters.hip), and
// the workspace layouts of those that need one.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "internal.h"

namespace xs {

constexpr int kMaxGroupSize = 1 << 20;   // every size of these calls, and T * k
constexpr int kMaxRank = 128;            // of an adapter

// ---------------------------------------------------------------------------- order

struct OrderArgs {
  const int32_t* ids;          // [pairs]
  int pairs, E;
  int32_t* offsets;            // [E + 1]
  int32_t* rows;               // [pairs]
  int32_t* pair_of;            // [pairs]
  int32_t* counts;             // [order_parts(pairs), E], unused by one workgroup
};
constexpr int kOrderOne = 4096;     // pairs that one workgroup sorts by itself
constexpr int kOrderMost = 8192;    // and can
constexpr int kOrderParts = 64;     // workgroups where there are several, as far as that goes
inline int order_part(int pairs) {
  int part = 1024;                  // pairs of a workgroup
  while (part < kOrderMost && pairs > kOrderParts * part) part *= 2;
  return part;
}
inline int order_parts(int pairs) {
  return pairs <= kOrderOne ? 0 : (pairs + order_part(pairs) - 1) / order_part(pairs);
}
// (the counts of as many parts as fewer pairs may have)
inline size_t order_bytes(int pairs, int E) {
  if (pairs <= kOrderOne) return 0;
  const int parts = order_parts(pairs);
  return align256(sizeof(int32_t) * size_t(parts > kOrderParts ? parts : kOrderParts) * E);
}
// A matrix [rows, cols] of each expert with pairs -> [cols, rows].
struct Transposed {
  const uint16_t* in;
  uint16_t* out;
  int rows, cols;
};
hipError_t launch_order(const OrderArgs& a, hipStream_t stream);
// The order and, beside it where it is one launch, both transposed.
hipError_t launch_order_and_transpose(const OrderArgs& a, const Transposed& first,
                                      const Transposed& second, hipStream_t stream);

// ---------------------------------------------------------------------------- moves

struct MoveArgs {
  int fp32;                    // 0: bf16 elements
  int T, k, d;
  const int32_t* rows;         // [T, k]
  const void* token;           // [T, d] x, dy
  long ld_token;
  const void* row;             // [T k, d] rows read
  long ld_row;
  const float* w;              // [T, k], or null: 1
  void* out_token;             // [T, d]
  long ld_out_token;
  void* out_row;               // [T k, d]
  long ld_out_row;
  float* dw;                   // [T, k]
};
hipError_t launch_dispatch(const MoveArgs& a, hipStream_t stream);
hipError_t launch_combine(const MoveArgs& a, hipStream_t stream);
hipError_t launch_combine_backward(const MoveArgs& a, hipStream_t stream);

// ---------------------------------------------------------------------------- products

// Rows from which the products may take 256 x 256 tiles, which keep the sums of split ones in the
// workspace: at most one part for each of 256 compute units.
constexpr int kTurnsRows = 256;
inline size_t grouped_bytes(int P) { return P < kTurnsRows ? 0 : size_t(256) * 256 * 256 * 4; }

struct GroupedArgs {
  int P, E, n, k;
  const int32_t* offsets;      // [E + 1]
  const uint16_t* x;           // [P, k]
  long ldx;
  const uint16_t* dy;          // [P, n]
  long lddy;
  const uint16_t* w;           // [E, n, k]
  uint16_t* out;               // y [P, n] or dx [P, k]
  long ldo;
  void* dw;                    // [E, n, k], bf16 or fp32
  int dw_fp32, accumulate;
  float* sums;                 // grouped_bytes(P) of them, or null
};
hipError_t launch_grouped_linear(const GroupedArgs& a, hipStream_t stream);
hipError_t launch_grouped_backward_x(const GroupedArgs& a, hipStream_t stream);
hipError_t launch_grouped_backward_w(const GroupedArgs& a, hipStream_t stream);

// ---------------------------------------------------------------------------- adapters

// Whether an adapters call goes token by token, without an order: by what both ways take in microseconds,
// each token's factors at 9 TB/s from the caches against an order and, for each tile, chains over d.
// Measured with 8 adapters at 48 to 256 tokens; with 1 and with 64 of them, at 32 to 256 tokens, the choice was
// the faster one of all 20 sizes too.  n = d = 4096: rank 16 8.4 us of 128 tokens, 16.6 in
// order; rank 64 13.5 of 96, 24.8, and 29.4 of 256, 25.5; rank 128 12.9 of 48. n = 8192, d = 512, rank 64:
// 16.9 of 96, 14.0.
constexpr int kAdapterFew = 256;
inline bool few_tokens(int T, int r, int n, int d) {
  const float one_by_one = 4.0f + float(T) * r * (float(n) + d) / 4.4e6f;
  const float in_order = 9.0f + d * (1.4f + r / 40.0f) * 1e-3f + float(r) * n / 2.5e6f;
  return T <= kAdapterFew && one_by_one <= in_order;
}
// Such a call in one launch, whose workgroups (of 1024 columns of a token) each make the token's h for
// themselves, or in two, whose first has a wave for each value.  A workgroup has 16 waves: up to 16
// ranks are a row of A each, as in two launches; more rows come one after the other, which the launch
// saved (1.4 us) pays for while rows are short; from 56 ranks on the rows of B that were not loaded ahead
// cost more than it.  With more than a workgroup a compute unit A is read too often.  One launch and
// two, us, of 840 sizes with 8 adapters.  One token, n = 4096: rank 16, d = 4096 4.8, 6.1, d = 8192
// 6.7, 8.3; rank 24, d = 2048 4.2, 4.9, d = 4096 6.8, 6.3; rank 32, d = 1024 4.3, 4.6, d = 2048 5.2,
// 4.9; rank 40, d = 2048 5.4, 5.0; rank 48, d = 512 4.3, 4.6; rank 64, d = 256 7.3, 5.1, d = 4096
// 14.8, 6.8.  Rank 16, n = 4096: 32 tokens of d = 4096 5.0, 6.3; 128 of d = 2048 6.0, 6.6, of d = 8192
// 12.2, 10.4.
inline bool in_one_launch(int T, int r, int n, int d) {
  const long groups = long(T) * ((n + 1023) / 1024), values = long(r) * d;   // of A, a workgroup
  return (r <= 16 || (r <= 48 && values < 1 << 16)) && (groups <= 256 || groups * values <= 1 << 24);
}
// Values of a row of h: the ranks of the kernels' instances, which have 1, 2, 4 or 8 tiles of 16.
inline int padded_rank(int r) { return r <= 16 ? 16 : r <= 32 ? 32 : r <= 64 ? 64 : 128; }

// Parts that the rows of an adapter are summed in for its factors' gradients: as many as make two
// workgroups for every compute unit, of 256 rows or more on average, for their sums take a launch
// (2094 tokens of 26 adapters of rank 120, n = 192, d = 376: 36.8 us in 2 parts, 32.4 in one; 5482 of 2,
// rank 72, n = 2704, d = 4584: 132 in 4, 153 in 2).
constexpr int kGradColumns = 128;      // columns of x or dy of a workgroup
inline int adapter_splits(int T, int L, int n, int d) {
  const long groups = long(L) * ((n + kGradColumns - 1) / kGradColumns +
                                 (d + kGradColumns - 1) / kGradColumns);
  const long want = 511 / groups, most = T / (256l * L);
  const long n_parts = want < most ? want : most;
  return n_parts < 1 ? 1 : int(n_parts);
}

struct AdaptersLayout {
  size_t offsets, rows, tokens;  // the tokens in adapters' order
  size_t counts;                 // of the sort
  size_t h, dh;                  // bf16 [T, 3, padded_rank]: A x and s B^T dy, as three parts that sum up
  size_t at, bt;                 // [L, d, r] and [L, r, n]: the factors transposed (backward)
  size_t part;                   // fp32 [splits, L (n + d) r] where splits > 1 (backward)
  size_t total;
};
inline AdaptersLayout adapters_layout(int T, int L, int r, int n, int d, bool backward) {
  AdaptersLayout A{};
  size_t o = 0;
  A.offsets = o; o += align256(sizeof(int32_t) * (size_t(L) + 1));
  A.rows = o;    o += align256(sizeof(int32_t) * size_t(T));
  A.tokens = o;  o += align256(sizeof(int32_t) * size_t(T));
  A.counts = o;  o += order_bytes(T, L);
  A.h = o;       o += align256(6 * size_t(T) * padded_rank(r));
  A.dh = o;
  A.at = A.bt = A.part = o;
  if (backward) {
    o += align256(6 * size_t(T) * padded_rank(r));
    A.at = o;    o += align256(2 * size_t(L) * d * r);
    A.bt = o;    o += align256(2 * size_t(L) * n * r);
    A.part = o;
    // (of any number of tokens up to T: the parts grow with them)
    const int splits = adapter_splits(T, L, n, d);
    if (splits > 1) o += align256(4 * size_t(splits) * L * r * (size_t(n) + d));
  }
  A.total = o > 0 ? o : 256;
  return A;
}

struct AdaptersArgs {
  int T, L, r, n, d;
  const uint16_t* x;           // [T, d]
  long ldx;
  const uint16_t* a;           // [L, r, d]
  const uint16_t* b;           // [L, n, r]
  const int32_t* ids;          // [T]
  const float* scales;         // [L], or null: 1
  const uint16_t* base;        // [T, n] or, backward, [T, d]; or null: 0
  long ld_base;
  uint16_t* out;               // [T, n] or, backward, [T, d]
  long ld_out;
  const uint16_t* dy;          // [T, n] (backward)
  long lddy;
  float* da;                   // [L, r, d] (backward)
  float* db;                   // [L, n, r]
  int32_t *offsets, *rows, *tokens, *counts;
  uint16_t *h, *dh, *at, *bt;
  float* part;
  int splits;
};
hipError_t launch_adapters(const AdaptersArgs& a, hipStream_t stream);
hipError_t launch_adapters_backward(const AdaptersArgs& a, hipStream_t stream);

}  // namespace xs
