// FP8 products with a scale for each block of 128: the quantiser, y = x W^T, and the routed
// SwiGLU experts of given (token, expert, weight) triples.
//
// A product over K runs in blocks of 128 inputs, one v_mfma_f32_16x16x128_f8f6f4 for each
// 16 x 16 tile and block: the instruction's sum starts at zero and enters the fp32 accumulator
// times the token's scale and the weight block's.  Weights are the instruction's rows (A),
// tokens its columns (B), so a lane's four results are one token's and share one factor.  Lane
// (n, g), n = lane % 16 and g = lane / 16, feeds row n of either operand with its bytes 16 g ..
// and 64 + 16 g .. of the block: each load instruction reads 64 neighbouring bytes of 16 rows,
// and as both operands permute the 128 inputs alike, the sum is unchanged.
//
// The instruction aligns the products of eight neighbouring inputs to their largest and keeps
// about 13 bits below it: 1.4e-5 of the result's RMS on Gaussian data, against 1.7e-3 of the
// final rounding to bf16.  Gate/up is another matter: its results are quantised again, and an
// error that moves a hidden value across the middle of two codes moves it by a whole step.  In FP8
// instructions 16 tokens of eight (2048, 768) experts were off by 3.6e-3, one expert's 16 tokens
// by 3.2e-3, where exact sums give 1.7e-3.  So gate/up runs in bf16 instructions of the decoded
// codes (exact products, fp32 sums) wherever that hides behind the weights' stream (bf16_up in the
// plan), and in FP8 ones where the instructions bound it; there the error is 1.8e-3 to 2.8e-3, the
// more the fewer values a call has.
//
// With the four multiply-adds that enter a result, an instruction takes 37 cycles of its matrix
// core, 32 without (3.6 and 4.4 PFLOP/s over the whole GPU when nothing else is done).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "blocks.h"
#include "wave.h"

namespace xs {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ floatx4 mfma128(const i32x8& a, const i32x8& b) {
  const floatx4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  // formats 0, 0: E4M3 both; scale operands 0: the unscaled instruction
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, zero, 0, 0, 0, 0, 0, 0);
}

// Eight codes as bf16, exactly (a value has four significant bits).
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t a, uint32_t b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true)};
  return bf16x8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
}

// A lane's codes of a block as the operands of four bf16 instructions.
struct Wide {
  bf16x8 v[4];
};
__device__ __forceinline__ Wide widen(const i32x8& c) {
  return {{codes_to_bf16(c[0], c[1]), codes_to_bf16(c[2], c[3]), codes_to_bf16(c[4], c[5]),
           codes_to_bf16(c[6], c[7])}};
}
// The block's products in bf16 instructions: exact products, summed in fp32.
__device__ __forceinline__ floatx4 mfma128(const Wide& a, const Wide& b) {
  floatx4 t = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int u = 0; u < 4; ++u)
    t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[u], b.v[u], t, 0, 0, 0);
  return t;
}

__device__ __forceinline__ uint16_t to_bf16(float v) {
  uint32_t b = __float_as_uint(v);
  if ((b & 0x7FFFFFFFu) > 0x7F800000u) return 0x7FC0u;
  b += 0x7FFFu + ((b >> 16) & 1u);   // round to nearest even
  return (uint16_t)(b >> 16);
}

// ---------------------------------------------------------------------------- quantiser

constexpr float kMaxCode = 448.0f;               // largest E4M3 value
constexpr float kTiny = 448.0f * 0x1p-126f;      // least maximum a scale is made from

// What a block's values are quantised with.  code = rne(448 x / a) wants the quotient of a bf16
// x correctly rounded, so that it gives the code of exact arithmetic even where the quotient lies
// on the middle of two codes.  With r = 1 / a to a rounding or so, q = t r and one step q + (t -
// q a) r do it: the step's own error is about 2^-23 roundings of q, and t / a of a t of 11 bits
// and an a of 8 is no nearer than 2^-9 to where the rounding turns.  All operands are scaled by
// `pre` out of the ranges where they would overflow or lose bits.  The scale a / 448 is correctly
// rounded for every a by the same step, 1 / 448 being so.
struct Quantum {
  float a, r, pre, scale;
  bool finite;
};
__device__ __forceinline__ Quantum quantum(uint32_t abs_bits) {
  constexpr float kInverse = 1.0f / kMaxCode;
  Quantum z;
  const float a = fmaxf(__uint_as_float(abs_bits), kTiny);
  z.finite = abs_bits < 0x7F800000u;
  const float s = a * kInverse;
  z.scale = z.finite ? __builtin_fmaf(__builtin_fmaf(-s, kMaxCode, a), kInverse, s)
                     : __uint_as_float(abs_bits);
  const float by = a > 0x1p100f ? 0x1p-64f : (a < 0x1p-60f ? 0x1p64f : 1.0f);
  z.a = a * by;
  const float r = __builtin_amdgcn_rcpf(z.a);
  z.r = __builtin_fmaf(__builtin_fmaf(-z.a, r, 1.0f), r, r);
  z.pre = kMaxCode * by;
  return z;
}
__device__ __forceinline__ float quotient(const Quantum& z, float x) {
  const float t = x * z.pre;
  const float q = t * z.r;
  return __builtin_fmaf(__builtin_fmaf(-q, z.a, t), z.r, q);   // |x| <= a: at most 448
}
// The codes of four values, first in the low byte.
__device__ __forceinline__ uint32_t codes4(const Quantum& z, const float* x) {
  if (!z.finite) {   // scale inf or NaN: codes are 0, or NaN for what is not finite
    uint32_t c = 0;
    for (int i = 0; i < 4; ++i)
      if (!(__builtin_fabsf(x[i]) < INFINITY)) c |= 0x7Fu << (8 * i);
    return c;
  }
  int v = 0;
  v = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(z, x[0]), quotient(z, x[1]), v, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(z, x[2]), quotient(z, x[3]), v, true);
  return (uint32_t)v;
}

// Largest bit pattern of |x| (NaN above inf above the finite values).
__device__ __forceinline__ uint32_t abs_max8(const float (&x)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  return m;
}

// The largest of 16 neighbouring lanes' values, in all of them.
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, dpp<0xB1, 0xF, 0u>(v));
  v = max(v, dpp<0x4E, 0xF, 0u>(v));
  v = max(v, dpp<0x141, 0xF, 0u>(v));
  return max(v, dpp<0x140, 0xF, 0u>(v));
}

__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0];
  const float4 b = reinterpret_cast<const float4*>(p)[1];
  x[0] = a.x;
  x[1] = a.y;
  x[2] = a.z;
  x[3] = a.w;
  x[4] = b.x;
  x[5] = b.y;
  x[6] = b.z;
  x[7] = b.w;
}

// Blocks of 1 x 128: 16 lanes a block, eight neighbouring values a lane; this thread's 16 lanes
// take every `step`-th block from `i` on.
template <typename In>
__device__ __forceinline__ void quantize_rows(const In* x, long rows, int cols, long ld, uint8_t* q,
                                              float* scales, long i, long step) {
  const int nb = (cols + kQuantBlock - 1) / kQuantBlock;
  const int l = threadIdx.x & 15;
  for (; i < rows * nb; i += step) {
    const long r = i / nb;
    const int b = (int)(i - r * nb), c = b * kQuantBlock + 8 * l;
    const bool in = c < cols;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (in) load8(x + r * ld + c, v);
    const Quantum z = quantum(max16(abs_max8(v)));
    if (in)
      *reinterpret_cast<uint2*>(q + r * cols + c) = make_uint2(codes4(z, v), codes4(z, v + 4));
    if (l == 0) scales[i] = z.scale;
  }
}

// Bound by memory: 4000 x 7168 in 17.0 us, 5.1 TB/s of reads and writes (a large copy: 4.9); wide
// loads and stores, several blocks in flight a thread row.  `live`: nullable count of rows on
// the device, at most `rows`.
template <typename In>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const In* x, int rows, int cols,
                                                            long ld, uint8_t* q, float* scales,
                                                            const int32_t* live) {
  quantize_rows(x, live ? *live : rows, cols, ld, q, scales,
                (long)blockIdx.x * 16 + (threadIdx.x >> 4), (long)gridDim.x * 16);
}

// Blocks of 128 x 128: one workgroup a block, 64 values a thread (row threadIdx / 16 + 16 i), which
// stay in registers between the maximum and the codes: one read.  14336 x 4096 in 34 us, the
// rate of a large copy.
__global__ __launch_bounds__(256) void quantize_tile_kernel(const uint16_t* x, int rows, int cols,
                                                            long ld, uint8_t* q, float* scales) {
  __shared__ uint32_t part[4];
  const int c = blockIdx.x * kQuantBlock + 8 * (threadIdx.x & 15);
  const long r0 = (long)blockIdx.y * kQuantBlock + (threadIdx.x >> 4);
  float v[8][8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    if (c < cols && r0 + 16 * i < rows) load8(x + (r0 + 16 * i) * ld + c, v[i]);
    m = max(m, abs_max8(v[i]));
  }
#pragma unroll
  for (int s = 1; s < 64; s *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, s));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  m = max(max(part[0], part[1]), max(part[2], part[3]));
  const Quantum z = quantum(m);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c < cols && r0 + 16 * i < rows)
      *reinterpret_cast<uint2*>(q + (r0 + 16 * i) * cols + c) =
          make_uint2(codes4(z, v[i]), codes4(z, v[i] + 4));
  if (threadIdx.x == 0) scales[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = z.scale;
}

template <typename In>
hipError_t launch_quantize_rows(const In* x, long rows, int cols, long ld, uint8_t* q, float* scales,
                         const int32_t* live, hipStream_t stream) {
  const long groups = (rows * quant_blocks(cols) + 15) / 16;
  const int grid = (int)(groups < 16384 ? groups : 16384);
  quantize_rows_kernel<In>
      <<<grid, 256, 0, stream>>>(x, (int)rows, cols, ld, q, scales, live);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------- products

constexpr int kUnits = 256;    // compute units of the GPU

enum Kind { kLinear, kGateUp, kDown };

struct Product {
  const uint8_t* xq;           // token rows: codes [., K] and scales [., blocks of K]
  const float* xs;
  const uint8_t* w1;           // weights [E, N, K] and scales [E, blocks of N, blocks of K]
  const uint8_t* w3;           // kGateUp: the up projection
  const float* s1;
  const float* s3;
  int N, K;
  int rows;                    // kLinear: token rows
  int k;                       // pairs of a token
  const int4* tiles;           // kGateUp, kDown: {expert, first row, rows, 0}
  const int32_t* n_tiles;      // how many of them there are
  const int32_t* perm;         // pair of each row in expert order
  float* out;                  // kGateUp: h [row, N]; kDown: o [pair, N]
  uint8_t* hq;                 // kGateUp of the tiled kernel: the codes and scales of h
  float* hs;
  uint16_t* y;                 // kLinear
  long ldy;
};

typedef const __attribute__((address_space(4))) float* ScalarPtr;   // read by scalar loads

// Products with few token rows: a workgroup's share is 16 MR weight rows (kGateUp: half of W1,
// half of W3, in bf16 instructions) times a tile of 16 NT tokens.  Its KW waves take the blocks of K in turn, so that
// no wave reads what another does and no barrier stands in the loop; the weights go from
// memory straight into the instruction's operands, the next block's loads in flight under
// this one's instructions.  The waves' sums meet in LDS at the end, added in wave order.
// Bound by the weights' stream, and below a few MB by its latency: 16 x 7168 x 2048 takes 5.9 us
// (2.5 TB/s), 45 x 1367 x 2720 5.5; more waves over K (8, 16) measured equal or slower.
template <Kind kKind, int MR, int NT, int KW>
__global__ __launch_bounds__(64 * KW, 2) void product_kernel(Product a) {
  constexpr int kRows = 16 * NT;
  constexpr int MW = kKind == kGateUp ? MR / 2 : MR;    // tiles of one matrix
  constexpr int LD = 16 * MR + 4;
  static_assert(kKind != kGateUp || MR % 2 == 0, "W1 and W3 tiles in pairs");
  __shared__ float red[KW][kRows][LD];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int N = a.N, K = a.K;
  const int nb = (K + kQuantBlock - 1) / kQuantBlock, nbN = (N + kQuantBlock - 1) / kQuantBlock;
  int first, live;
  const uint8_t *w1 = a.w1, *w3 = a.w3;
  const float *s1 = a.s1, *s3 = a.s3;
  if constexpr (kKind == kLinear) {
    first = blockIdx.y * kRows;
    live = min(kRows, a.rows - first);
  } else {
    if ((int)blockIdx.y >= *a.n_tiles) return;
    const int4 t = a.tiles[blockIdx.y];
    first = t.y;
    live = t.z;
    const int e = __builtin_amdgcn_readfirstlane(t.x);
    w1 += (size_t)e * N * K;
    s1 += (size_t)e * nbN * nb;
    if constexpr (kKind == kGateUp) {
      w3 += (size_t)e * N * K;
      s3 += (size_t)e * nbN * nb;
    }
  }
  const int n0 = blockIdx.x * 16 * MW;
  // rows past the end repeat the last one; their results are not stored
  const uint8_t* wrow[MR];
#pragma unroll
  for (int m = 0; m < MR; ++m) {
    const int r = min(n0 + 16 * (m % MW) + n, N - 1);
    wrow[m] = (m < MW ? w1 : w3) + (size_t)r * K;
  }
  const ScalarPtr f1 = (ScalarPtr)(s1 + (size_t)(n0 / kQuantBlock) * nb);
  const ScalarPtr f3 = kKind == kGateUp ? (ScalarPtr)(s3 + (size_t)(n0 / kQuantBlock) * nb) : f1;
  const uint8_t* xrow[NT];
  const float* srow[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int p = first + min(16 * t + n, live - 1);
    const int r = kKind == kGateUp ? a.perm[p] / a.k : p;
    xrow[t] = a.xq + (size_t)r * K;
    srow[t] = a.xs + (size_t)r * nb;
  }
  floatx4 acc[MR][NT];
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[m][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

  struct Block {
    i32x4 w[MR][2], x[NT][2];
    float sx[NT], f1, f3;
  };
  // Pieces past the row's end read its last one.
  auto load = [&](Block& r, int b) {
    const int lo = min(b * kQuantBlock + 16 * g, K - 16);
    const int hi = min(b * kQuantBlock + 64 + 16 * g, K - 16);
#pragma unroll
    for (int m = 0; m < MR; ++m) {
      r.w[m][0] = *reinterpret_cast<const i32x4*>(wrow[m] + lo);
      r.w[m][1] = *reinterpret_cast<const i32x4*>(wrow[m] + hi);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      r.x[t][0] = *reinterpret_cast<const i32x4*>(xrow[t] + lo);
      r.x[t][1] = *reinterpret_cast<const i32x4*>(xrow[t] + hi);
      r.sx[t] = srow[t][b];
    }
    r.f1 = f1[b];
    if constexpr (kKind == kGateUp) r.f3 = f3[b];
  };
  auto add = [&](const Block& r, int b) {
    // where the rows end inside this block, what was read past them is not theirs
    const int lo = b * kQuantBlock + 16 * g < K ? -1 : 0;
    const int hi = b * kQuantBlock + 64 + 16 * g < K ? -1 : 0;
    auto whole = [&](const i32x4 (&v)[2]) {
      return __builtin_shufflevector(v[0] & lo, v[1] & hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    using Operand = std::conditional_t<kKind == kGateUp, Wide, i32x8>;
    auto operand = [&](const i32x8& c) -> Operand {
      if constexpr (kKind == kGateUp)
        return widen(c);
      else
        return c;
    };
    Operand w[MR];
#pragma unroll
    for (int m = 0; m < MR; ++m) w[m] = operand(whole(r.w[m]));
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const Operand x = operand(whole(r.x[t]));
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        const floatx4 v = mfma128(w[m], x);
        const float s = r.sx[t] * (m < MW ? r.f1 : r.f3);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][t][i] = __builtin_fmaf(v[i], s, acc[m][t][i]);
      }
    }
  };
  Block u, v;
  int b = wave;
  if (b < nb) load(u, b);
  while (b < nb) {                                      // (no loads past the last block)
    if (b + KW >= nb) {
      add(u, b);
      break;
    }
    load(v, b + KW);
    __builtin_amdgcn_sched_barrier(0);                  // loads stay above the instructions
    add(u, b);
    b += KW;
    if (b + KW >= nb) {
      add(v, b);
      break;
    }
    load(u, b + KW);
    __builtin_amdgcn_sched_barrier(0);
    add(v, b);
    b += KW;
  }
  // lane (n, g) holds rows 4 g .. 4 g + 3 of weight tile m for token n of tile t
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int m = 0; m < MR; ++m)
      *reinterpret_cast<floatx4*>(&red[wave][16 * t + n][16 * m + 4 * g]) = acc[m][t];
  __syncthreads();
  for (int i = threadIdx.x; i < live * 16 * MW; i += 64 * KW) {
    const int t = i / (16 * MW), c = i - t * 16 * MW;
    if (n0 + c >= N) continue;
    auto sum = [&](int col) {
      float s = red[0][t][col];
#pragma unroll
      for (int w = 1; w < KW; ++w) s += red[w][t][col];
      return s;
    };
    const float v = sum(c);
    if constexpr (kKind == kLinear) {
      a.y[(size_t)(first + t) * a.ldy + n0 + c] = to_bf16(v);
    } else if constexpr (kKind == kGateUp) {
      a.out[(size_t)(first + t) * N + n0 + c] = v / (1.0f + expf(-v)) * sum(16 * MW + c);
    } else {
      a.out[(size_t)a.perm[first + t] * N + n0 + c] = v;
    }
  }
}

// Products with many token rows: BW weight rows (kGateUp: BW / 2 rows of W1 and the same of
// W3) times BT tokens a workgroup, both operands through LDS in kStages buffers of one block
// of K each, filled straight from global memory (no registers between).  The workgroup's waves
// are WW along the weight rows by WT along the tokens, MW x TT instruction tiles each; a
// block's results enter the accumulators while the next tile's instructions run.  kBf16: in
// bf16 instructions.
//
// LDS rows are the 128 bytes of a block.  Row r keeps its 16-byte piece c at place
// c ^ ((r >> 1) & 7): the sixteen rows of an operand read then lie in sixteen different
// places modulo 256 bytes.  The loads write LDS in lane order, so the lanes take their
// source pieces in that order.
//
// Few tokens an expert: bound by HBM, 228 us for the 1.41 GB of 48 experts' W1 and W3 (6.2 TB/s)
// and 128 us for W2 (5.5).  64 tokens an expert over 256 of them: 1.43 ms (5.3 TB/s; the
// experts past 128 tokens read their weights again) and 0.86 ms, of which the fp32 outputs'
// stores are 0.12.  4000 x 4096 x 7168 in 256 x 256 tiles: 117 us, 2.0 PFLOP/s, at a clock that
// falls to 1.5-2.0 GHz; the loads alone would take 88 us, the instructions and reads of LDS
// alone 108.  Tried without gain: tiles ordered for the eight L2 caches, prefetching into
// them, persistent workgroups that load the next tile's operands before they store, 16 waves,
// reading the next block's operands under this one's instructions, asking whether a block is left
// to load (1000 x 4096 x 7168 44 -> 48 us).
typedef const __attribute__((address_space(1))) void* GlobalPtr;
typedef __attribute__((address_space(3))) void* LdsPtr;

__device__ __forceinline__ void to_lds16(const uint8_t* src, uint8_t* dst) {
  __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)dst, 16, 0, 0);
}
__device__ __forceinline__ void to_lds4(const float* src, float* dst) {
  __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)dst, 4, 0, 0);
}
// All but this wave's last N loads are done, and those of the workgroup's other waves too.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");   // no read of LDS moves above the barrier
}

constexpr int kScaleBlocks = 4;

// LDS of the tiled kernel: kStages blocks of both operands, then two buffers of the scales of
// kScaleBlocks blocks: the tokens' [BT][kScaleBlocks] and, one load's 64 floats, the weights'
// [2][kScaleBlocks] (kGateUp: W1's and W3's; else the first 128 rows' and the next ones').
template <int BW, int BT, int kStages>
struct TileLds {
  static constexpr int kStage = (BW + BT) * kQuantBlock;
  static constexpr int kScales = kStages * kStage;
  static constexpr int kTokenFloats = BT * kScaleBlocks;
  static constexpr int kScaleBytes = (kTokenFloats + 64) * 4;
  static constexpr int kBytes = kScales + 2 * kScaleBytes;
};

template <Kind kKind, int BW, int BT, int WW, int WT, int kStages, bool kBf16>
__global__ __launch_bounds__(64 * WW * WT) void tile_kernel(Product a) {
  using L = TileLds<BW, BT, kStages>;
  constexpr int kThreads = 64 * WW * WT;
  constexpr int MW = BW / WW / 16, TT = BT / WT / 16;
  constexpr int kRows = kThreads / 8;                       // rows of one load of the workgroup
  constexpr int LW = BW / kRows, LT = BT >= kRows ? BT / kRows : 1;
  constexpr int kLoads = LW + LT;                           // of a wave and stage
  constexpr int kScaleLoads = BT / 16 > WW * WT ? BT / 16 / (WW * WT) : 1;   // and chunk of scales
  constexpr int kCols = kKind == kGateUp ? BW / 2 : BW;    // output columns of a workgroup
  // token tiles worked on together; where a workgroup's tokens may be few, the rest is skipped
  constexpr int kGroup = kBf16 ? 1 : BT >= 256 || TT < 2 ? TT : 2;
  static_assert(TT % kGroup == 0, "whole groups");
  constexpr int kLead = kStages > 3 ? kStages - 2 : 1;
  static_assert(kLead <= kScaleBlocks, "two buffers of scales");
  static_assert(kKind != kGateUp || MW % 2 == 0, "W1 and W3 tiles in pairs");
  static_assert(kKind == kGateUp || !kBf16, "the only product whose results are quantised");
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ww = wave % WW, wt = wave / WW;
  const int n = lane & 15, g = lane >> 4;
  const int N = a.N, K = a.K;
  const int nb = (K + kQuantBlock - 1) / kQuantBlock, nbN = (N + kQuantBlock - 1) / kQuantBlock;
  int first, live;
  const uint8_t *w1 = a.w1, *w3 = a.w3;
  const float *s1 = a.s1, *s3 = a.s3;
  if constexpr (kKind == kLinear) {
    first = blockIdx.y * BT;
    live = min(BT, a.rows - first);
  } else {
    if ((int)blockIdx.y >= *a.n_tiles) return;
    const int4 t = a.tiles[blockIdx.y];
    first = t.y;
    live = t.z;
    const int e = __builtin_amdgcn_readfirstlane(t.x);
    w1 += (size_t)e * N * K;
    s1 += (size_t)e * nbN * nb;
    if constexpr (kKind == kGateUp) {
      w3 += (size_t)e * N * K;
      s3 += (size_t)e * nbN * nb;
    }
  }
  const int n0 = blockIdx.x * kCols;
  // LDS row R of the weights: tile (R / 16) % MW of wave R / (16 MW) along the weight rows
  // (offsets from the tile's first row fit 32 bits: 256 rows of at most 2^20 bytes)
  const uint8_t *const wbase1 = w1 + (size_t)n0 * K, *const wbase3 = w3 + (size_t)n0 * K;
  uint32_t woff[LW];
  const int piece = 16 * ((lane & 7) ^ (((tid >> 3) >> 1) & 7));
#pragma unroll
  for (int j = 0; j < LW; ++j) {
    const int R = j * kRows + (tid >> 3);
    const int unit = kKind == kGateUp
                         ? R / (16 * MW) * (8 * MW) + R / 16 % MW % (MW / 2) * 16 + R % 16
                         : R;
    woff[j] = (uint32_t)min(unit, N - 1 - n0) * (uint32_t)K;
  }
  // whether load j is of W3 is the wave's to know: its eight rows lie in one tile
  auto of_w3 = [&](int j) { return kKind == kGateUp && (j * kRows + wave * 8) / 16 % MW >= MW / 2; };
  const uint8_t* const xbase = kKind == kGateUp ? a.xq : a.xq + (size_t)first * K;
  size_t xoff[LT];
#pragma unroll
  for (int j = 0; j < LT; ++j) {
    const int p = min((j * kRows + (tid >> 3)) % BT, live - 1);
    xoff[j] = kKind == kGateUp ? (size_t)(a.perm[first + p] / a.k) * K
                               : (size_t)((uint32_t)p * (uint32_t)K);
  }
  // lane l of a load of scales takes block l % 4 of token l / 4
  const float* ssrc[kScaleLoads];
  uint32_t sdst[kScaleLoads];
#pragma unroll
  for (int j = 0; j < kScaleLoads; ++j) {
    const int t0 = ((wave + j * WW * WT) * 16) % BT;
    const int p = first + min(t0 + lane / kScaleBlocks, live - 1);
    const int r = kKind == kGateUp ? a.perm[p] / a.k : p;
    ssrc[j] = a.xs + (size_t)r * nb;
    sdst[j] = L::kScales + t0 * kScaleBlocks * 4;
  }
  // the i-th of a wave's loads of block b (what lies past the row's end: its last piece)
  auto load = [&](int b, uint8_t* stage, int i) {
    const uint32_t at = (uint32_t)min(b * kQuantBlock + piece, K - 16);
    if (i < LW)
      to_lds16((of_w3(i) ? wbase3 : wbase1) + (woff[i < LW ? i : 0] + at),
               stage + (i * kRows + wave * 8) * kQuantBlock);
    else
      to_lds16(xbase + (xoff[i < LW ? 0 : i - LW] + at),
               stage + (BW + ((i - LW) * kRows + wave * 8) % BT) * kQuantBlock);
  };
  const int n_block = n0 / kQuantBlock;
  const float* const fsrc =
      kKind == kGateUp ? (lane / kScaleBlocks % 2 ? s3 : s1) + (size_t)n_block * nb
                       : s1 + (size_t)min(n_block + lane / kScaleBlocks % 2, nbN - 1) * nb;
  auto load_scales = [&](int b) {          // of blocks b .. b + 3, b a multiple of four
    const int at = min(b + lane % kScaleBlocks, nb - 1);
    const int buffer = (b / kScaleBlocks & 1) * L::kScaleBytes;
#pragma unroll
    for (int j = 0; j < kScaleLoads; ++j)
      to_lds4(ssrc[j] + at, reinterpret_cast<float*>(lds + sdst[j] + buffer));
    to_lds4(fsrc + at,
            reinterpret_cast<float*>(lds + L::kScales + buffer) + L::kTokenFloats);
  };
  // first output column of the wave; its weight rows lie in one block of 128 (of each matrix)
  const int u0 = n0 + ww * (kKind == kGateUp ? 8 * MW : 16 * MW);
  const int nt = (live - wt * 16 * TT + 15) / 16;      // live tiles of this wave, at most TT
  floatx4 acc[MW][TT];
#pragma unroll
  for (int m = 0; m < MW; ++m)
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[m][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

  const int swz = (n >> 1) & 7;
  const int lo = 16 * (g ^ swz), hi = 16 * ((4 + g) ^ swz);
  auto operand = [&](const uint8_t* row) {
    const int4 u = *reinterpret_cast<const int4*>(row + lo);
    const int4 v = *reinterpret_cast<const int4*>(row + hi);
    return i32x8{u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
  };
  load_scales(0);
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s)
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(min(s, nb - 1), lds + s * L::kStage, i);
  // Block b from its buffer while a later block's loads fill another.  The order is written
  // out and held: the loads go between the matrix instructions (at the step's start, all waves
  // at once, they would hold up the reads of LDS), a token tile's operand is read while the
  // tile before it is worked on, and an instruction's result enters its accumulator two
  // instructions later.  The pointers are declared apart: without that every read of LDS
  // would wait for every load in flight.
  auto step = [&](int b, const uint8_t* __restrict__ stage, const float* __restrict__ scales,
                  uint8_t* __restrict__ next) {
    const int ahead = min(b + kStages - 1, nb - 1);    // (past the end: block nb - 1 again)
    const uint8_t* const wl = stage + (ww * 16 * MW + n) * kQuantBlock;
    const uint8_t* const xl = stage + (BW + wt * 16 * TT + n) * kQuantBlock;
    const float* const sl = scales + (wt * 16 * TT + n) * kScaleBlocks + b % kScaleBlocks;
    const float* const fl = scales + L::kTokenFloats + b % kScaleBlocks;
    // The loads before instruction i: spread over the step, or with two buffers, where the last
    // has the rest of this step alone to arrive in, one at every second instruction
    // (4000 x 4096 x 7168 in 256 x 256 tiles 136-143 -> 125-133 us).
    auto load_share = [&](int i) {
      constexpr int kTotal = MW * TT;
      if constexpr (kStages == 2 && kTotal >= 2 * kLoads) {
        if (i % 2 == 0 && i / 2 < kLoads) load(ahead, next, i / 2);
      } else {
#pragma unroll
        for (int l = (i * kLoads + kTotal - 1) / kTotal; l * kTotal < (i + 1) * kLoads; ++l)
          load(ahead, next, l);
      }
    };
    if constexpr (kBf16) {
      Wide w[MW];
#pragma unroll
      for (int m = 0; m < MW; ++m) w[m] = widen(operand(wl + 16 * m * kQuantBlock));
      const float fw[2] = {fl[0], fl[kScaleBlocks]};
      __builtin_amdgcn_sched_barrier(0);               // the scales' loads are older than these
#pragma unroll
      for (int t = 0; t < TT; ++t) {
#pragma unroll
        for (int i = t * MW; i < (t + 1) * MW; ++i) load_share(i);
        if (t >= nt) continue;                         // no tokens here
        const Wide x = widen(operand(xl + 16 * t * kQuantBlock));
        const float sx = sl[16 * t * kScaleBlocks];
#pragma unroll
        for (int m = 0; m < MW; ++m) {
          const floatx4 v = mfma128(w[m], x);
#pragma unroll
          for (int c = 0; c < 4; ++c)
            acc[m][t][c] = __builtin_fmaf(v[c], sx * fw[m >= MW / 2], acc[m][t][c]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      return;
    }
    i32x8 w[MW], x[2];
    float sx[TT];
    x[0] = operand(xl);
#pragma unroll
    for (int m = 0; m < MW; ++m) w[m] = operand(wl + 16 * m * kQuantBlock);
    const float fw1 = kKind == kGateUp ? fl[0] : fl[(u0 / kQuantBlock - n_block) * kScaleBlocks];
    const float fw3 = kKind == kGateUp ? fl[kScaleBlocks] : fw1;
#pragma unroll
    for (int t = 0; t < TT; ++t) sx[t] = sl[16 * t * kScaleBlocks];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t0 = 0; t0 < TT; t0 += kGroup) {
      if (kGroup < TT && t0 >= nt) {                   // no tokens here: the loads alone
#pragma unroll
        for (int i = t0 * MW; i < (t0 + kGroup) * MW; ++i) load_share(i);
        continue;
      }
      floatx4 v[3];
      auto enter = [&](int i) {
        const int t = t0 + i / MW, m = i % MW;
        const float s = sx[t] * (kKind == kGateUp && m >= MW / 2 ? fw3 : fw1);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          acc[m][t][c] = __builtin_fmaf(v[i % 3][c], s, acc[m][t][c]);
      };
#pragma unroll
      for (int i = 0; i < kGroup * MW; ++i) {
        const int t = t0 + i / MW, m = i % MW, at = t0 * MW + i;
        if (m == 0 && t + 1 < TT) x[(t + 1) & 1] = operand(xl + 16 * (t + 1) * kQuantBlock);
        load_share(at);
        v[i % 3] = mfma128(w[m], x[t & 1]);
        if (i >= 2) enter(i - 2);
        __builtin_amdgcn_sched_barrier(0);
      }
      enter(kGroup * MW - 2);
      enter(kGroup * MW - 1);
    }
  };
  int cur = 0;                                         // the buffer of block b
  for (int b = 0; b < nb; ++b) {
    // The loads of this block are done; those of the kStages - 2 after it may be in flight.
    // A chunk of scales is loaded kLead steps before its first block, so that it is older than
    // any load that may be in flight then; its buffer was last read the step before, or earlier.
    wait_loads<kLoads*(kStages - 2)>();
    if (b == nb - 1 && K % kQuantBlock != 0) {         // the rows end inside this block
      uint8_t* const mine = lds + cur * L::kStage + wave * 8 * kQuantBlock + 16 * lane;
      if (b * kQuantBlock + piece >= K) {
#pragma unroll
        for (int i = 0; i < LW; ++i)
          *reinterpret_cast<i32x4*>(mine + i * kRows * kQuantBlock) = i32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < LT; ++i)
          *reinterpret_cast<i32x4*>(lds + cur * L::kStage + 16 * lane +
                                    (BW + (i * kRows + wave * 8) % BT) * kQuantBlock) =
              i32x4{0, 0, 0, 0};
      }
      __syncthreads();
    }
    if ((b + kLead) % kScaleBlocks == 0 && b + kLead < nb) load_scales(b + kLead);
    step(b, lds + cur * L::kStage,
         reinterpret_cast<const float*>(lds + L::kScales +
                                        (b / kScaleBlocks & 1) * L::kScaleBytes),
         lds + (cur == 0 ? kStages - 1 : cur - 1) * L::kStage);
    cur = cur + 1 == kStages ? 0 : cur + 1;
  }
  wait_loads<0>();                                     // LDS is free

  // lane (n, g) holds units 4 g .. 4 g + 3 of weight tile m for token n of tile t
  if constexpr (kKind == kGateUp) {
    constexpr int MH = MW / 2;
    uint32_t* const part = reinterpret_cast<uint32_t*>(lds);   // [WW][BT] maxima
    static_assert(kCols == kQuantBlock, "a workgroup holds one block of the hidden row");
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      uint32_t m = 0;
#pragma unroll
      for (int u = 0; u < MH; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = acc[u][t][i];
          const float h = v / (1.0f + expf(-v)) * acc[MH + u][t][i];
          const int c = u0 + 16 * u + 4 * g + i;
          acc[u][t][i] = c < N ? h : 0.0f;
          m = max(m, __float_as_uint(acc[u][t][i]) & 0x7FFFFFFFu);
        }
      m = max(m, (uint32_t)__shfl_xor((int)m, 16));
      m = max(m, (uint32_t)__shfl_xor((int)m, 32));
      if (g == 0) part[ww * BT + wt * 16 * TT + 16 * t + n] = m;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int tok = wt * 16 * TT + 16 * t + n;
      uint32_t m = 0;
#pragma unroll
      for (int w = 0; w < WW; ++w) m = max(m, part[w * BT + tok]);
      if (tok >= live) continue;
      const Quantum z = quantum(m);
      const size_t row = first + tok;
#pragma unroll
      for (int u = 0; u < MH; ++u) {
        const int c = u0 + 16 * u + 4 * g;
        const float v[4] = {acc[u][t][0], acc[u][t][1], acc[u][t][2], acc[u][t][3]};
        if (c < N) *reinterpret_cast<uint32_t*>(a.hq + row * N + c) = codes4(z, v);
      }
      if (ww == 0 && g == 0) a.hs[row * nbN + n0 / kQuantBlock] = z.scale;
    }
  } else {
    const bool whole = kKind == kDown || (a.ldy % 4 == 0 && ((uintptr_t)a.y & 7) == 0);
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int tok = wt * 16 * TT + 16 * t + n;
      if (tok >= live) continue;
      const size_t row = kKind == kDown ? a.perm[first + tok] : first + tok;
#pragma unroll
      for (int m = 0; m < MW; ++m) {
        const int c = u0 + 16 * m + 4 * g;
        if constexpr (kKind == kDown) {
          if (c < N) *reinterpret_cast<floatx4*>(a.out + row * N + c) = acc[m][t];
        } else if (whole && c + 3 < N) {
          const uint32_t p0 = to_bf16(acc[m][t][0]) | (uint32_t)to_bf16(acc[m][t][1]) << 16;
          const uint32_t p1 = to_bf16(acc[m][t][2]) | (uint32_t)to_bf16(acc[m][t][3]) << 16;
          *reinterpret_cast<uint2*>(a.y + row * a.ldy + c) = make_uint2(p0, p1);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (c + i < N) a.y[row * a.ldy + c + i] = to_bf16(acc[m][t][i]);
        }
      }
    }
  }
}

template <Kind kKind, int BW, int BT, int WW, int WT, int kStages, bool kBf16 = false>
hipError_t launch_tile(const Product& a, int tiles, hipStream_t stream) {
  constexpr int kBytes = TileLds<BW, BT, kStages>::kBytes;
  static_assert(kBytes <= 160 * 1024, "LDS of a compute unit");
  const auto kernel = tile_kernel<kKind, BW, BT, WW, WT, kStages, kBf16>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, kBytes);
  if (e != hipSuccess) return e;
  const int cols = kKind == kGateUp ? BW / 2 : BW;
  kernel<<<dim3((a.N + cols - 1) / cols, tiles), 64 * WW * WT, kBytes, stream>>>(a);
  return hipGetLastError();
}

template <Kind kKind, int MR, int NT, int KW>
hipError_t launch_product(const Product& a, int tiles, hipStream_t stream) {
  const int cols = 16 * (kKind == kGateUp ? MR / 2 : MR);
  product_kernel<kKind, MR, NT, KW>
      <<<dim3((a.N + cols - 1) / cols, tiles), 64 * KW, 0, stream>>>(a);
  return hipGetLastError();
}

// The forms of y = x W^T: weight rows and tokens of a workgroup, and what a block of 128 inputs
// costs in microseconds: `few` with little else on the GPU, `full` for each workgroup that every
// one of the 256 compute units has to run (several at a time where LDS holds them: what a
// further one adds).  Measured over 7 batches of 24 to 1200 tokens by 7 shapes of 576 to
// 14336 rows and 512 to 7168 inputs; a launch takes about 2.5 us more.  The choice came within
// 10 % of the best form (of 13 measured) on 42 of the 49, within 20 % on all.
struct LinearForm {
  int rows, tokens;
  float few, full;
  hipError_t (*launch)(const Product&, int, hipStream_t);
};
const LinearForm kLinearForms[] = {
    {16, 16, 0.12f, 0.136f, launch_product<kLinear, 1, 1, 4>},
    {32, 16, 0.19f, 0.195f, launch_product<kLinear, 2, 1, 4>},
    {16, 32, 0.21f, 0.22f, launch_product<kLinear, 1, 2, 4>},
    {32, 32, 0.235f, 0.24f, launch_product<kLinear, 2, 2, 4>},
    {64, 32, 0.245f, 0.165f, launch_tile<kLinear, 64, 32, 2, 2, 4>},
    {64, 64, 0.32f, 0.23f, launch_tile<kLinear, 64, 64, 2, 2, 3>},
    {128, 64, 0.40f, 0.43f, launch_tile<kLinear, 128, 64, 4, 2, 5>},
    {128, 128, 0.58f, 0.67f, launch_tile<kLinear, 128, 128, 2, 4, 4>},
    {128, 256, 0.90f, 1.1f, launch_tile<kLinear, 128, 256, 2, 4, 3>},
    {256, 256, 1.57f, 2.15f, launch_tile<kLinear, 256, 256, 2, 4, 2>},
};
float form_cost(const LinearForm& f, int T, int n) {
  const long groups = long((n + f.rows - 1) / f.rows) * ((T + f.tokens - 1) / f.tokens);
  if (groups <= kUnits) return f.few + (f.full > f.few ? f.full - f.few : 0.0f) * groups / kUnits;
  const float full = f.full * float((groups + kUnits - 1) / kUnits);
  return full > f.few ? full : f.few;
}

// ---------------------------------------------------------------------------- one token

// Products whose token rows are few enough to be quantised by every workgroup for itself, into
// LDS: a linear product of up to 16 short rows, and the two products of one token's experts, so
// that these calls are one launch and two.  The waves take the blocks of K in turn as in
// product_kernel.
//   kLinear  x rows [T, K] bf16; 16 MR WR weight rows a workgroup.
//   kGateUp  the one token's x; workgroup (., r) the expert of pair r: h[r] = silu(W1 x) (W3 x),
//            in bf16 instructions.
//   kDown    all pairs' h rows [k, K]; y = sum_r w_r W2_{id_r} q(h_r), the pairs one after the
//            other in every wave, no outputs of single pairs in between.
// A workgroup has WR shares of 16 MR weight rows, of KW waves each, whose sums meet in
// product_kernel's order.
// Bound by the weights' latency and stream: 1 x 7168 x 2048 in 5.3 us; eight (2048, 768) experts'
// 25 MB and 13 MB in 15.8 us together.  The first weights are under way while the rows are
// quantised (gate/up 9.7 -> 8.9 us; two blocks of them: both products 17.6 -> 19.6), and nothing is
// loaded past the last block (17.6 -> 16.3).
struct Small {
  const uint16_t* x;           // kLinear, kGateUp
  long ldx;
  const float* hin;            // kDown
  int T, N, K;
  const uint8_t *w1, *w3;
  const float *s1, *s3;
  const int32_t* ids;          // [k]
  const float* w;
  int k, E;
  float* h;                    // kGateUp: [k, N]
  uint16_t* y;                 // kLinear [T, N], kDown [N]
  long ldy;
};

constexpr int kSmallPairs = kMaxTopK;
// Bytes of a row in LDS, of codes or (kGateUp) bf16: whole blocks, rows 16 bytes past a multiple
// of 128 apart.
template <Kind kKind>
__host__ __device__ inline int small_pitch(int K) {
  return (K + kQuantBlock - 1) / kQuantBlock * kQuantBlock * (kKind == kGateUp ? 2 : 1) + 16;
}

template <Kind kKind, int MR, int KW, int WR>
__global__ __launch_bounds__(64 * KW * WR, 2) void small_kernel(Small a) {
  constexpr int kRows = kKind == kLinear ? 16 : 1;
  constexpr int MW = kKind == kGateUp ? MR / 2 : MR;
  constexpr int LD = 16 * MR + 4;
  constexpr int kCols = 16 * MW;           // output columns of a wave
  static_assert(kQuantBlock % kCols == 0, "they share the weights' scales");
  __shared__ float red[KW * WR][kRows][LD];
  __shared__ int expert[kSmallPairs];
  __shared__ int pair[kSmallPairs];
  extern __shared__ __attribute__((aligned(16))) uint8_t codes[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int N = a.N, K = a.K;
  const int nb = (K + kQuantBlock - 1) / kQuantBlock, nbN = (N + kQuantBlock - 1) / kQuantBlock;
  const int pitch = small_pitch<kKind>(K);
  const int n0 = blockIdx.x * kCols * WR, nw = n0 + wave / KW * kCols;   // the wave's first
  int e0 = 0, pairs = 1;                   // kGateUp's expert; pairs that the workgroup adds up
  if constexpr (kKind == kGateUp) {
    e0 = __builtin_amdgcn_readfirstlane(a.ids[blockIdx.y]);
    if (e0 < 0 || e0 >= a.E) return;
  }
  if constexpr (kKind == kDown) {
    const int id = lane < a.k ? a.ids[lane] : -1;
    const uint64_t live = __ballot(id >= 0 && id < a.E);
    pairs = __popcll(live);
    const int at = __popcll(live & ((1ull << lane) - 1));
    if (wave == 0 && ((live >> lane) & 1)) {
      expert[at] = id;
      pair[at] = lane;
    }
    __syncthreads();
  }
  const int rows = kKind == kLinear ? a.T : pairs;
  float* const scales = reinterpret_cast<float*>(codes + (size_t)rows * pitch);   // [rows][nb]

  // rows past the end repeat the last one; their results are not stored
  size_t wrow[MW];
#pragma unroll
  for (int m = 0; m < MW; ++m) wrow[m] = (size_t)min(nw + 16 * m + n, N - 1) * K;
  floatx4 acc[MR];
#pragma unroll
  for (int m = 0; m < MR; ++m) acc[m] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  struct Block {
    i32x4 w[MR][2];
    float f1, f3;
  };
  struct Item {                            // block b of pair q
    int q, b;
  };
  auto next = [&](Item i) {
    i.b += KW;
    while (i.b >= nb && i.q + 1 < pairs) {
      i.b -= nb;
      ++i.q;
    }
    return i;
  };
  // Pieces past the row's end, and blocks past the last, read the last one.
  auto load = [&](Block& r, Item i) {
    const int b = min(i.b, nb - 1);
    const int e = kKind == kDown ? __builtin_amdgcn_readfirstlane(expert[i.q]) : e0;
    const int lo = min(b * kQuantBlock + 16 * g, K - 16);
    const int hi = min(b * kQuantBlock + 64 + 16 * g, K - 16);
    const size_t s = ((size_t)e * nbN + min(nw / kQuantBlock, nbN - 1)) * nb + b;
    r.f1 = a.s1[s];
    if constexpr (kKind == kGateUp) r.f3 = a.s3[s];
#pragma unroll
    for (int m = 0; m < MR; ++m) {
      const uint8_t* const p = (m < MW ? a.w1 : a.w3) + (size_t)e * N * K + wrow[m % MW];
      r.w[m][0] = *reinterpret_cast<const i32x4*>(p + lo);
      r.w[m][1] = *reinterpret_cast<const i32x4*>(p + hi);
    }
  };
  auto add = [&](const Block& r, Item i) {
    const int row = kKind == kLinear ? min(n, a.T - 1) : i.q;
    const int at = i.b * kQuantBlock + 16 * g;
    const float sx = scales[row * nb + i.b];
    // where the rows end inside this block, what was read past them is not theirs
    const int lo = at < K ? -1 : 0, hi = at + 64 < K ? -1 : 0;
    bf16x8 xb[4];                          // kGateUp: inputs 0, 8, 64 and 72 of the lane's on
    i32x8 xc;
    if constexpr (kKind == kGateUp) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        xb[u] = *reinterpret_cast<const bf16x8*>(codes + 2 * (at + u / 2 * 64 + u % 2 * 8));
    } else {
      const uint8_t* const p = codes + row * pitch + at;
      xc = __builtin_shufflevector(*reinterpret_cast<const i32x4*>(p),
                                   *reinterpret_cast<const i32x4*>(p + 64), 0, 1, 2, 3, 4, 5, 6, 7);
    }
#pragma unroll
    for (int m = 0; m < MR; ++m) {
      const i32x8 w = __builtin_shufflevector(r.w[m][0] & lo, r.w[m][1] & hi, 0, 1, 2, 3, 4, 5, 6,
                                              7);
      floatx4 t = {0.0f, 0.0f, 0.0f, 0.0f};
      if constexpr (kKind == kGateUp) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
          t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16(w[2 * u], w[2 * u + 1]), xb[u],
                                                      t, 0, 0, 0);
      } else {
        t = mfma128(w, xc);
      }
      const float s = sx * (m < MW ? r.f1 : r.f3);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[m][j] = __builtin_fmaf(t[j], s, acc[m][j]);
    }
  };
  Block u, v;
  Item i{0, wave % KW};
  while (i.b >= nb && i.q + 1 < pairs) {                // (fewer blocks than waves)
    i.b -= nb;
    ++i.q;
  }
  if (pairs > 0) load(u, i);                            // under way while the rows are quantised

  {                                                     // 16 lanes a block, as in quantize_rows
    constexpr int kStep = 4 * KW * WR;
    const int row_step = kStep / nb, block_step = kStep - row_step * nb;
    int r = (tid >> 4) / nb, b = (tid >> 4) - r * nb;
    while (r < rows) {
      const int c = b * kQuantBlock + 8 * (tid & 15);
      float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (c < K) {
        if constexpr (kKind == kDown)
          load8(a.hin + (size_t)pair[r] * K + c, v);
        else
          load8(a.x + (size_t)r * a.ldx + c, v);
      }
      const Quantum z = quantum(max16(abs_max8(v)));
      const uint32_t c0 = codes4(z, v), c1 = codes4(z, v + 4);
      if constexpr (kKind == kGateUp)
        *reinterpret_cast<bf16x8*>(codes + r * pitch + 2 * c) = codes_to_bf16(c0, c1);
      else
        *reinterpret_cast<uint2*>(codes + r * pitch + c) = make_uint2(c0, c1);
      if ((tid & 15) == 0) scales[r * nb + b] = z.scale * (kKind == kDown ? a.w[pair[r]] : 1.0f);
      r += row_step;
      if ((b += block_step) >= nb) {
        b -= nb;
        ++r;
      }
    }
  }
  __syncthreads();
  if (pairs > 0) {
    while (i.b < nb) {
      const Item j = next(i);
      if (j.b >= nb) {                                  // (no loads past the last block)
        add(u, i);
        break;
      }
      load(v, j);
      __builtin_amdgcn_sched_barrier(0);
      add(u, i);
      i = next(j);
      if (i.b >= nb) {
        add(v, j);
        break;
      }
      load(u, i);
      __builtin_amdgcn_sched_barrier(0);
      add(v, j);
    }
  }
#pragma unroll
  for (int m = 0; m < MR; ++m)
    if (n < kRows) *reinterpret_cast<floatx4*>(&red[wave][n][16 * m + 4 * g]) = acc[m];
  __syncthreads();
  const int live = kKind == kLinear ? a.T : 1;
  for (int i = tid; i < live * kCols * WR; i += 64 * KW * WR) {
    const int t = i / (kCols * WR), c = i - t * kCols * WR;
    if (n0 + c >= N) continue;
    auto sum = [&](int more) {
      const int w0 = c / kCols * KW, col = c % kCols + more;
      float s = red[w0][t][col];
#pragma unroll
      for (int w = 1; w < KW; ++w) s += red[w0 + w][t][col];
      return s;
    };
    const float v = sum(0);
    if constexpr (kKind == kGateUp)
      a.h[(size_t)blockIdx.y * N + n0 + c] = v / (1.0f + expf(-v)) * sum(kCols);
    else
      a.y[(size_t)t * a.ldy + n0 + c] = to_bf16(v);
  }
}

template <Kind kKind, int MR, int KW, int WR>
hipError_t launch_small(const Small& a, int rows, int groups, hipStream_t stream) {
  const int cols = 16 * (kKind == kGateUp ? MR / 2 : MR) * WR;
  small_kernel<kKind, MR, KW, WR><<<dim3((a.N + cols - 1) / cols, groups), 64 * KW * WR,
                                   rows * (small_pitch<kKind>(a.K) + 4 * quant_blocks(a.K)),
                                   stream>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------- experts

// What the products of the experts need: x quantised, and the pairs in expert order.  The first E
// workgroups are an expert's each, over all ids; the rest take the blocks of x.  An expert's
// counts the pairs of every expert (in LDS) and, wave by wave, its own; its rows begin after those of the
// experts before it, its tiles of either product likewise, and its pairs are listed in
// ascending order.  No atomics but those counts, so every call lists them alike.  4.8 us for 32
// tokens of 7168 and 256 experts, 20 us for 2048 (the E passes over 16384 ids).
struct Prepare {
  const uint16_t* x;
  int T, d;
  long ldx;
  uint8_t* xq;
  float* xs;
  const int32_t* ids;
  int pairs, E, up_rows, down_rows;
  int32_t* counts;
  int32_t* perm;
  int4* up_tiles;
  int4* down_tiles;
};
__global__ __launch_bounds__(1024) void prepare_kernel(Prepare a) {
  if ((int)blockIdx.x >= a.E) {
    quantize_rows(a.x, a.T, a.d, a.ldx, a.xq, a.xs,
                  (long)(blockIdx.x - a.E) * 64 + (threadIdx.x >> 4),
                  (long)(gridDim.x - a.E) * 64);
    return;
  }
  const int32_t* const ids = a.ids;
  const int pairs = a.pairs, E = a.E;
  __shared__ int count[kMaxExperts];
  __shared__ int mine[16];
  __shared__ int sums[3][16];
  const int e = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  count[tid] = 0;
  __syncthreads();
  // each wave a contiguous part of the pairs
  const int part = ((pairs + 16 * 64 - 1) / (16 * 64)) * 64;
  const int from = min(pairs, wave * part), to = min(pairs, from + part);
  int own = 0;
  for (int i = from; i < to; i += 64) {
    const int id = i + lane < to ? ids[i + lane] : -1;
    if (id >= 0 && id < E) atomicAdd(&count[id], 1);
    own += __popcll(__ballot(id == e));
  }
  if (lane == 0) mine[wave] = own;
  __syncthreads();
  // rows and tiles of the experts before e
  auto tiles_of = [](int rows, int tile) { return (rows + tile - 1) / tile; };
  const int c = tid < e ? count[tid] : 0;
  int before[3] = {c, tiles_of(c, a.up_rows), tiles_of(c, a.down_rows)};
#pragma unroll
  for (int i = 0; i < 3; ++i) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2) before[i] += __shfl_xor(before[i], s);
    if (lane == 0) sums[i][wave] = before[i];
  }
  __syncthreads();
  int row0 = 0, up0 = 0, down0 = 0, at = 0;
  for (int w = 0; w < 16; ++w) {
    row0 += sums[0][w];
    up0 += sums[1][w];
    down0 += sums[2][w];
    if (w < wave) at += mine[w];
  }
  const int n = count[e];
  if (e == E - 1 && tid == 0) {
    a.counts[0] = row0 + n;
    a.counts[1] = up0 + tiles_of(n, a.up_rows);
    a.counts[2] = down0 + tiles_of(n, a.down_rows);
  }
  for (int i = tid * a.up_rows; i < n; i += 1024 * a.up_rows)
    a.up_tiles[up0 + i / a.up_rows] = make_int4(e, row0 + i, min(a.up_rows, n - i), 0);
  for (int i = tid * a.down_rows; i < n; i += 1024 * a.down_rows)
    a.down_tiles[down0 + i / a.down_rows] = make_int4(e, row0 + i, min(a.down_rows, n - i), 0);
  for (int i = from; i < to; i += 64) {
    const bool hit = i + lane < to && ids[i + lane] == e;
    const uint64_t hits = __ballot(hit);
    if (hit) a.perm[row0 + at + __popcll(hits & ((1ull << lane) - 1))] = i + lane;
    at += __popcll(hits);
  }
}

// y_i = sum_r w_ir o[i k + r], rank order, eight columns a thread.  The pairs' outputs stay fp32:
// rounded to bf16 their error (1.6 times the final rounding's) would show in y.  Bound by
// reading them: 2048 tokens of 8 x 7168 in 100 us, 5.0 TB/s.
__global__ __launch_bounds__(256) void combine_kernel(const float* o, const int32_t* ids,
                                                      const float* w, int k, int E, int d,
                                                      uint16_t* y, long ldy) {
  const int t = blockIdx.x, c = 8 * (blockIdx.y * 256 + threadIdx.x);
  if (c >= d) return;
  float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int r = 0; r < k; ++r) {
    const long p = (long)t * k + r;
    const int e = ids[p];
    if (e < 0 || e >= E) continue;
    float v[8];
    load8(o + p * d + c, v);
    const float wr = w[p];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = __builtin_fmaf(wr, v[i], s[i]);
  }
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = to_bf16(s[2 * i]) | (uint32_t)to_bf16(s[2 * i + 1]) << 16;
  *reinterpret_cast<uint4*>(y + t * ldy + c) = make_uint4(b[0], b[1], b[2], b[3]);
}

}  // namespace

hipError_t launch_block_quantize(const uint16_t* x, int rows, int cols, long ld, int block_rows,
                                 uint8_t* q, float* scales, hipStream_t stream) {
  if (block_rows == 1)
    return launch_quantize_rows(x, rows, cols, ld, q, scales, nullptr, stream);
  quantize_tile_kernel<<<dim3(quant_blocks(cols), quant_blocks(rows)), 256, 0, stream>>>(
      x, rows, cols, ld, q, scales);
  return hipGetLastError();
}

hipError_t launch_block_linear(const BlockLinearArgs& a, hipStream_t stream) {
  Product p{};
  p.xq = a.xq;
  p.xs = a.xs;
  p.w1 = a.wq;
  p.s1 = a.wscale;
  p.N = a.n;
  p.K = a.k;
  p.rows = a.T;
  p.y = a.y;
  p.ldy = a.ldy;
  if (a.x) {
    Small s{};
    s.x = a.x;
    s.ldx = a.ldx;
    s.T = a.T;
    s.N = a.n;
    s.K = a.k;
    s.w1 = a.wq;
    s.s1 = a.wscale;
    s.y = a.y;
    s.ldy = a.ldy;
    // Twice the waves a workgroup, which share the quantisation, where as many workgroups remain
    // as there are compute units or nearly: one row of 2048 by 7168 5.5 -> 5.3 us, by 2048 4.1 ->
    // 4.8; of 7168 by 14336 24.3 -> 22.6, by 1536 8.0 -> 9.7; 4 rows of 4096 by 4096 9.8 -> 8.6.
    // (Four times: one row of 4096 by 24576 22.4 -> 24.9, 8 of 2048 by 32768 17.6 -> 15.9.)
    if (a.n >= 4096) return launch_small<kLinear, 1, 4, 2>(s, a.T, 1, stream);
    return launch_small<kLinear, 1, 4, 1>(s, a.T, 1, stream);
  }
  const LinearForm* best = &kLinearForms[0];
  for (const LinearForm& f : kLinearForms)
    if (form_cost(f, a.T, a.n) < form_cost(*best, a.T, a.n)) best = &f;
  return best->launch(p, (a.T + best->tokens - 1) / best->tokens, stream);
}

hipError_t launch_block_experts(const BlockExpertsArgs& a, hipStream_t stream) {
  const int pairs = a.T * a.k;
  const BlockExpertsPlan plan = block_experts_plan(a.T, a.k, a.E, a.d, a.f);
  if (plan.one) {
    Small s{};
    s.x = a.x;
    s.T = 1;
    s.N = a.f;
    s.K = a.d;
    s.w1 = a.w1;
    s.w3 = a.w3;
    s.s1 = a.s1;
    s.s3 = a.s3;
    s.ids = a.ids;
    s.w = a.w;
    s.k = a.k;
    s.E = a.E;
    s.h = a.h;
    const hipError_t e = launch_small<kGateUp, 2, 8, 1>(s, 1, a.k, stream);
    if (e != hipSuccess) return e;
    s.hin = a.h;
    s.N = a.d;
    s.K = a.f;
    s.w1 = a.w2;
    s.s1 = a.s2;
    s.y = a.y;
    return launch_small<kDown, 1, 8, 1>(s, a.k, 1, stream);
  }
  const long groups = (long(a.T) * quant_blocks(a.d) + 63) / 64;
  prepare_kernel<<<int(a.E + (groups < 4096 ? groups : 4096)), 1024, 0, stream>>>(
      {a.x, a.T, a.d, a.ldx, a.xq, a.xs, a.ids, pairs, a.E, plan.up_rows, plan.down_rows, a.counts,
       a.perm, a.up_tiles, a.down_tiles});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  Product p{};
  p.xq = a.xq;
  p.xs = a.xs;
  p.w1 = a.w1;
  p.w3 = a.w3;
  p.s1 = a.s1;
  p.s3 = a.s3;
  p.N = a.f;
  p.K = a.d;
  p.k = a.k;
  p.tiles = a.up_tiles;
  p.n_tiles = a.counts + 1;
  p.perm = a.perm;
  p.out = a.h;
  p.hq = a.hq;
  p.hs = a.hs;
  const int up = pair_tiles(pairs, a.E, plan.up_rows);
  const int down = pair_tiles(pairs, a.E, plan.down_rows);
  if (plan.few_up) {
    if ((e = launch_product<kGateUp, 2, 1, 4>(p, up, stream)) != hipSuccess) return e;
    e = launch_quantize_rows(a.h, pairs, a.f, a.f, a.hq, a.hs, a.counts, stream);
  } else {
    e = plan.wide == 32  ? launch_tile<kGateUp, 256, 32, 8, 1, 4, true>(p, up, stream)
        : plan.bf16_up ? launch_tile<kGateUp, 256, 128, 4, 2, 3, true>(p, up, stream)
                       : launch_tile<kGateUp, 256, 128, 4, 2, 3>(p, up, stream);
  }
  if (e != hipSuccess) return e;
  p.xq = a.hq;
  p.xs = a.hs;
  p.w1 = a.w2;
  p.s1 = a.s2;
  p.N = a.d;
  p.K = a.f;
  p.tiles = a.down_tiles;
  p.n_tiles = a.counts + 2;
  p.out = a.o;
  if (plan.few_down)
    e = plan.down_rows == 16 ? launch_product<kDown, 2, 1, 4>(p, down, stream)
                             : launch_tile<kDown, 128, 64, 4, 2, 5>(p, down, stream);
  else
    e = plan.wide == 32 ? launch_tile<kDown, 256, 32, 8, 1, 4>(p, down, stream)
                   : launch_tile<kDown, 256, 128, 4, 2, 3>(p, down, stream);
  if (e != hipSuccess) return e;
  combine_kernel<<<dim3(a.T, (a.d / 8 + 255) / 256), 256, 0, stream>>>(a.o, a.ids, a.w, a.k, a.E,
                                                                     a.d, a.y, a.ldy);
  return hipGetLastError();
}

}  // namespace xs
