// Launchers of the routing by scores (gate.hip) and of the FP8 products with a scale for each
// block of 128 (blocks.hip), and the workspace layout of the latter.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "internal.h"

namespace xs {

constexpr int kMaxGateGroups = 64;
constexpr int kMaxBlockSize = 1 << 20;   // every size of the block calls
constexpr int kQuantBlock = 128;         // inputs (and weight rows) that share a scale

inline int quant_blocks(int n) { return (n + kQuantBlock - 1) / kQuantBlock; }

struct GateArgs {
  const void* logits;
  int bf16;                    // 0: fp32 logits
  int T, N, k;
  long ld;
  const float* bias;           // nullable [N]
  int sigmoid;                 // 0: softmax
  int G, top_groups, top2;
  int renormalize;
  float scale;
  int32_t* ids;                // [T, k], written by the forward pass
  float* w;
  const float* dw;             // backward: [T, k]
  float* dlogits;              // [T, N]
  int vec, vec_bias, vec_out;  // aligned for wide loads and stores (set by the launch)
};

hipError_t launch_gate(const GateArgs& a, hipStream_t stream);
hipError_t launch_gate_backward(const GateArgs& a, hipStream_t stream);

// x [rows, cols] bf16 -> codes and scales; block_rows 1 or 128.
hipError_t launch_block_quantize(const uint16_t* x, int rows, int cols, long ld, int block_rows,
                                 uint8_t* q, float* scales, hipStream_t stream);


struct BlockLinearLayout {
  size_t xq;                   // uint8 [T, k]  codes of x
  size_t xs;                   // fp32 [T, ceil(k / 128)]
  size_t total;
};
inline BlockLinearLayout block_linear_layout(int T, int k) {
  BlockLinearLayout L{};
  size_t o = 0;
  L.xq = o; o += align256(size_t(T) * k);
  L.xs = o; o += align256(sizeof(float) * size_t(T) * quant_blocks(k));
  L.total = o > 0 ? o : 256;
  return L;
}

// Whether a product quantises x in every workgroup, a launch less (launch_block_linear with x
// given): up to 16 rows of 16384 values in all.  One row of 2048 by 7168 takes 5.3 us so, 6.9 in
// two launches; 4 rows of 4096 by 4096 8.6 and 8.9; 8 of 2048 by 7168 7.0 and 7.6, by 14336 11.5
// and 10.7; past the limit 16 of 2048 by 7168 9.0 and 8.3, 4 of 7168 by 7168 16.3 and 14.6.
inline bool block_linear_small(int T, int k) { return T <= 16 && long(T) * k <= 16384; }

struct BlockLinearArgs {
  int T, n, k;
  const uint16_t* x;           // bf16 rows, of block_linear_small sizes; or null, with
  long ldx;
  const uint8_t* xq;
  const float* xs;
  const uint8_t* wq;
  const float* wscale;
  uint16_t* y;
  long ldy;
};
hipError_t launch_block_linear(const BlockLinearArgs& a, hipStream_t stream);

// Tiles of the (token, expert) pairs in expert order: at most one partly filled tile for each
// expert with a pair, the rest full.
inline int pair_tiles(int pairs, int E, int tile_rows) {
  const int some = pairs < E ? pairs : E;
  return some + (pairs - some) / tile_rows;
}

// The forms of the experts' two products, by the rows of an expert on average if as many experts
// as can be have a pair.  From 12 rows on tiles of 128 tokens cost no more than narrower ones
// (their empty 32s are skipped) and read the weights of nearly every expert once; below, tiles
// of 32 have less to load.  The tiled form wants a workgroup for most compute units: four tokens
// of 64 (1024, 256) experts have 32 in gate/up and take 9 us in it, 6 in the few-row form; down
// of two (4096, 14336) experts has 32, 53 against 21 us; eight of them with 16 rows 128, 105 in
// the form of 256 x 128 against 85 in that of 128 x 64.  One token's pairs, where their hidden
// rows are short enough for every workgroup to quantise them, take two launches of their own
// (one of eight (2048, 768) experts 34.7 -> 15.4 us a call).
constexpr int kFewMean = 16;    // gate/up in the few-row form: rows of an expert at most
constexpr int kFewGroups = 96;  // and fewer workgroups than this in the tiled one
constexpr int kLeastTile = 16;  // the least rows of a tile of any plan
// Gate/up in bf16 instructions (blocks.hip says what for) up to 32 rows an expert: 96 tokens of
// two of eight (4096, 14336) experts take 322 us a call so and 316 in FP8 ones, 512 of eight of 256
// (7168, 2048) 2018 and 2051, 200 of eight of 128 (2048, 768) 144 and 142; past it the
// instructions show: 1000 of those 208 and 195, 777 of the first 656 and 484, one (4096, 4096)
// expert's 512 96 and 68.
struct BlockExpertsPlan {
  bool one;                    // one token: the launches without tiles
  bool few_up, few_down;       // few workgroups: gate/up in the few-row form; down in that or 128 x 64
  int wide;                    // tokens of the tiled form's tiles
  bool bf16_up;                // gate/up in bf16 instructions
  int up_rows, down_rows;      // rows of a tile of either product
};
inline bool one_token_form(int k, int d, int f) {   // (their rows in LDS: 38 KB at most)
  return long(k) * f <= 32768 && d <= 16384;
}
inline BlockExpertsPlan block_experts_plan(int T, int k, int E, int d, int f) {
  BlockExpertsPlan p{};
  const int pairs = T > 0 ? T * k : k;
  const int expect = pairs < E ? pairs : E, mean = pairs / expect;
  p.one = T == 1 && one_token_form(k, d, f);
  p.wide = mean >= 12 ? 128 : 32;
  p.bf16_up = mean <= 32;
  const long spans = (mean + p.wide - 1) / p.wide;
  p.few_up = mean <= kFewMean && long(expect) * quant_blocks(f) < kFewGroups;
  p.few_down = long(expect) * spans * ((d + 255) / 256) < 192;
  p.up_rows = p.few_up ? kLeastTile : p.wide;
  p.down_rows = !p.few_down ? p.wide : mean <= 8 ? kLeastTile : 64;
  return p;
}

struct BlockExpertsLayout {
  size_t xq, xs;               // as BlockLinearLayout, of x [T, d]
  size_t counts;               // int32 [3]: pairs, tiles of gate/up, tiles of down
  size_t perm;                 // int32 [T * k] pair (t * k + r) of each row in expert order
  size_t up_tiles;             // int4 [pair_tiles] {expert, first row, rows, 0} of gate/up
  size_t down_tiles;           // and of down
  size_t h;                    // fp32 [hidden_tokens * k, f] hidden rows in expert order, where a
                               //      plan quantises them after gate/up
  size_t hq, hs;               // their codes [T * k, f] and scales [T * k, ceil(f / 128)]
  size_t o;                    // fp32 [T * k, d] the pairs' outputs, by pair
  size_t total;
};
// The most tokens, of up to T, whose plan quantises the hidden rows after gate/up (as those of all
// smaller numbers do, but for one token's own form).
inline int hidden_tokens(int T, int k, int E, int d, int f) {
  const int blocks = quant_blocks(f);
  const int pairs = long(E) * blocks < kFewGroups ? (kFewMean + 1) * E - 1   // by the mean
                                                  : (kFewGroups - 1) / blocks;  // by the grid
  const int one = one_token_form(k, d, f) ? 1 : 0, n = pairs / k > one ? pairs / k : one;
  return n < T ? n : T;
}
// A workspace for T tokens serves any smaller number too: no region shrinks as T grows, whatever the
// plans (the tiles are counted in the least rows a plan gives them).
inline BlockExpertsLayout block_experts_layout(int T, int k, int E, int d, int f) {
  BlockExpertsLayout L{};
  const size_t rows = size_t(T) * k;
  size_t o = 0;
  L.xq = o;     o += align256(size_t(T) * d);
  L.xs = o;     o += align256(sizeof(float) * size_t(T) * quant_blocks(d));
  L.counts = o; o += 256;
  L.perm = o;   o += align256(sizeof(int32_t) * rows);
  const size_t tiles = align256(16 * size_t(pair_tiles(int(rows), E, kLeastTile)));
  L.up_tiles = o;   o += tiles;
  L.down_tiles = o; o += tiles;
  L.h = o;      o += align256(sizeof(float) * size_t(hidden_tokens(T, k, E, d, f)) * k * f);
  L.hq = o;     o += align256(rows * f);
  L.hs = o;     o += align256(sizeof(float) * rows * quant_blocks(f));
  L.o = o;      o += align256(sizeof(float) * rows * d);
  L.total = o;
  return L;
}

struct BlockExpertsArgs {
  int T, k, E, d, f;
  const uint16_t* x;
  long ldx;
  const int32_t* ids;
  const float* w;
  const uint8_t *w1, *w3, *w2;
  const float *s1, *s3, *s2;
  uint16_t* y;
  long ldy;
  uint8_t* xq;
  float* xs;
  int32_t* counts;
  int32_t* perm;
  int4* up_tiles;
  int4* down_tiles;
  float* h;
  uint8_t* hq;
  float* hs;
  float* o;
};
hipError_t launch_block_experts(const BlockExpertsArgs& a, hipStream_t stream);

}  // namespace xs
