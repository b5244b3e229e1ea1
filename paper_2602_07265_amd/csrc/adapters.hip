// Low-rank adapters of many requests beside a shared projection, and their gradients.
//   y_t = base_t + s_e B_e A_e x_t          e the adapter of token t, A_e [r, d], B_e [n, r]
//   dh_t = s_e B_e^T dy_t,  dx_t = base_t + A_e^T dh_t,
//   dA_e = sum over its tokens of dh_t x_t^T,  dB_e = s_e sum of dy_t h_t^T,  h_t = A_e x_t
//
// Every product has one short side, r, so all are bound by reading and writing rows of d and n
// values.  Few tokens (few_tokens) are worked on one by one: a wave for each value of h, then a
// lane for each of y.  More are put in adapters' order first, and tiles of tokens of one adapter
// go through the matrix instructions.  h and dh are held as sums of three bf16 values (24 bits), so
// that the products with them are as exact as those of fp32 values; y and dx, which are rounded
// to bf16, take two of the three.  Going backward the factors are transposed first (order.hip), which
// are small beside the rows, and dh and dx are the two forward products on them.
//
// 4000 tokens of 5 adapters of rank 16, n = d = 4096: h 12.6 us (33 MB, 2.6 TB/s: 251 workgroups, each a
// chain of loads), y 13.8 (66 MB, 4.8 TB/s), h and dh in one launch 19.9 (3.3 TB/s), the factors'
// gradients 16.5 (4.0 TB/s), the order, with the transposed factors beside it or without, 5.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "groups.h"
#include "tiles.h"

namespace xs {
namespace {

__device__ __forceinline__ float value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ void values8(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 to_bf16x8(const float (&x)[8]) {
  return make_uint4(to_bf16x2(x[0], x[1]), to_bf16x2(x[2], x[3]), to_bf16x2(x[4], x[5]),
                    to_bf16x2(x[6], x[7]));
}

// ---------------------------------------------------------------------------- few tokens

// h[t, j] = A_e[j] . x_t, a wave each.
__global__ __launch_bounds__(256) void few_shrink_kernel(AdaptersArgs a, float* h) {
  const int lane = threadIdx.x & 63;
  const int t = blockIdx.y, j = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int e = a.ids[t];
  if ((unsigned)e >= (unsigned)a.L || j >= a.r) return;
  const uint16_t* const x = a.x + (size_t)t * a.ldx;
  const uint16_t* const w = a.a + ((size_t)e * a.r + j) * a.d;
  float sum = 0.0f;
#pragma unroll 8
  for (int c = 8 * lane; c < a.d; c += 512) {
    float p[8], q[8];
    values8(*reinterpret_cast<const uint4*>(x + c), p);
    values8(*reinterpret_cast<const uint4*>(w + c), q);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(p[i], q[i], sum);
  }
  sum = wave_sum(sum);
  if (lane == 0) h[(size_t)t * a.r + j] = sum;
}

// y[t, c] = base + s B_e[c] . h_t, a lane each.
__global__ __launch_bounds__(256) void few_expand_kernel(AdaptersArgs a, const float* h) {
  __shared__ float hs[kMaxRank];
  const int t = blockIdx.y, c = blockIdx.x * 256 + threadIdx.x;
  const int e = a.ids[t];
  const bool live = (unsigned)e < (unsigned)a.L;
  if (live && (int)threadIdx.x < a.r) hs[threadIdx.x] = h[(size_t)t * a.r + threadIdx.x];
  __syncthreads();
  if (c >= a.n) return;
  float y = 0.0f;
  if (live) {
    const uint16_t* const w = a.b + ((size_t)e * a.n + c) * a.r;
#pragma unroll 4
    for (int j = 0; j < a.r; j += 8) {
      float q[8];
      values8(*reinterpret_cast<const uint4*>(w + j), q);
#pragma unroll
      for (int i = 0; i < 8; ++i) y = __builtin_fmaf(q[i], hs[j + i], y);
    }
    if (a.scales) y *= a.scales[e];
  }
  if (a.base) {
    const float b = value(a.base[(size_t)t * a.ld_base + c]);
    y = live ? y + b : b;
  }
  a.out[(size_t)t * a.ld_out + c] = to_bf16(y);
}

// Both in one launch (in_one_launch): workgroup (1024 columns, t) makes token t's h for itself, a wave a
// value at a time, while the first values of B_e are under way.
__global__ __launch_bounds__(1024) void few_kernel(AdaptersArgs a) {
  constexpr int kAhead = 4;                            // of eight values of a row of B_e
  __shared__ float hs[kMaxRank];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.y, c = blockIdx.x * 1024 + threadIdx.x;
  const int e = a.ids[t];
  const bool live = (unsigned)e < (unsigned)a.L;       // (the same for the whole workgroup)
  const uint16_t* const row = a.b + ((size_t)(live ? e : 0) * a.n + min(c, a.n - 1)) * a.r;
  uint4 ahead[kAhead];
  float base = 0.0f, scale = 1.0f;
  if (a.base && c < a.n) base = value(a.base[(size_t)t * a.ld_base + c]);
  if (live) {
    if (a.scales) scale = a.scales[e];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      ahead[i] = *reinterpret_cast<const uint4*>(row + (8 * i < a.r ? 8 * i : 0));
    const uint16_t* const x = a.x + (size_t)t * a.ldx;
    for (int j = wave; j < a.r; j += 16) {
      const uint16_t* const w = a.a + ((size_t)e * a.r + j) * a.d;
      float sum = 0.0f;
#pragma unroll 8
      for (int k = 8 * lane; k < a.d; k += 512) {
        float p[8], q[8];
        values8(*reinterpret_cast<const uint4*>(x + k), p);
        values8(*reinterpret_cast<const uint4*>(w + k), q);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(p[i], q[i], sum);
      }
      sum = wave_sum(sum);
      if (lane == 0) hs[j] = sum;
    }
  }
  __syncthreads();
  if (c >= a.n) return;
  float y = 0.0f;
  if (live) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (8 * i >= a.r) break;
      float q[8];
      values8(ahead[i], q);
#pragma unroll
      for (int u = 0; u < 8; ++u) y = __builtin_fmaf(q[u], hs[8 * i + u], y);
    }
    for (int j = 8 * kAhead; j < a.r; j += 8) {
      float q[8];
      values8(*reinterpret_cast<const uint4*>(row + j), q);
#pragma unroll
      for (int u = 0; u < 8; ++u) y = __builtin_fmaf(q[u], hs[j + u], y);
    }
  }
  a.out[(size_t)t * a.ld_out + c] = to_bf16(live ? __builtin_fmaf(scale, y, base) : base);
}

// ---------------------------------------------------------------------------- many tokens

// Eight elements of a row from k on, or zeros in their place (the load of the row's first goes on).
__device__ __forceinline__ uint4 load8(const uint16_t* row, int k, bool in) {
  const uint4 v = *reinterpret_cast<const uint4*>(row + (in ? k : 0));
  return make_uint4(in ? v.x : 0, in ? v.y : 0, in ? v.z : 0, in ? v.w : 0);
}

// Two values, each as three bf16 values that sum up to it (to 24 bits); infinities and NaN as one.
struct Split {
  uint32_t p0, p1, p2;
};
__device__ __forceinline__ Split split3(float lo, float hi) {
  Split s;
  s.p0 = to_bf16x2(lo, hi);
  const float lo0 = __uint_as_float(s.p0 << 16), hi0 = __uint_as_float(s.p0 & 0xFFFF0000u);
  lo = fabsf(lo0) < __builtin_inff() ? lo - lo0 : 0.0f;
  hi = fabsf(hi0) < __builtin_inff() ? hi - hi0 : 0.0f;
  s.p1 = to_bf16x2(lo, hi);
  s.p2 = to_bf16x2(lo - __uint_as_float(s.p1 << 16), hi - __uint_as_float(s.p1 & 0xFFFF0000u));
  return s;
}

struct Shrink {
  const uint16_t* x;           // [T, K]
  long ldx;
  int K;
  const uint16_t* w;           // [L, r, K]
  const float* scales;         // [L], or null
  uint16_t* h;                 // [T, 3, 16 JT]
};
struct Tokens {                // in adapters' order
  const int32_t* offsets;
  const int32_t* tokens;
  int L, T, r;
};

// Four values of h of one token, ranks `rank` on, as its three parts; past the rank zeros.
template <int JT>
__device__ __forceinline__ void store_h(uint16_t* row, int rank, int r, const floatx4& v, float s) {
  const Split a = split3(rank < r ? v[0] * s : 0.0f, rank + 1 < r ? v[1] * s : 0.0f);
  const Split b = split3(rank + 2 < r ? v[2] * s : 0.0f, rank + 3 < r ? v[3] * s : 0.0f);
  *reinterpret_cast<uint2*>(row + rank) = make_uint2(a.p0, b.p0);
  *reinterpret_cast<uint2*>(row + 16 * JT + rank) = make_uint2(a.p1, b.p1);
  *reinterpret_cast<uint2*>(row + 32 * JT + rank) = make_uint2(a.p2, b.p2);
}

template <int JT, int BB>
struct ShrinkLds {
  static constexpr int kStages = JT == 4 ? 8 : 5;
  static constexpr int kStage = (16 * JT + BB) * kBlock;              // elements
};

// h of 16 MT tokens of one adapter: the waves take blocks of 64 of the reduction in turn, kAhead of
// them at a time, operands straight from memory, and their sums meet in LDS.  The first `groups`
// workgroups have one product's tiles, the others another's (x and A, dy and B transposed).
template <int MT, int JT>
__global__ __launch_bounds__(512) void shrink_kernel(Tokens o, Shrink first_a, Shrink second,
                                                     int groups) {
  static_assert(JT <= 2, "ranks past 32 are shrink_tile_kernel's");
  constexpr int kWaves = 8, kAhead = JT == 1 ? 4 : 2;
  extern __shared__ floatx4 sums[];                    // [kWaves][MT JT][64]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  const bool is_first = (int)blockIdx.x < groups;
  const Shrink a = is_first ? first_a : second;
  Place p;
  if (!find_place(o.offsets, o.L, o.T, 16 * MT, 1, is_first ? blockIdx.x : blockIdx.x - groups, p))
    return;
  const int e = p.e, first = p.first, live = p.live;
  const uint16_t* x[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t)
    x[t] = a.x + (size_t)o.tokens[first + min(16 * t + n, live - 1)] * a.ldx;
  const uint16_t* w[JT];
#pragma unroll
  for (int j = 0; j < JT; ++j)
    w[j] = a.w + ((size_t)e * o.r + min(16 * j + n, o.r - 1)) * a.K;
  floatx4 acc[JT][MT];
#pragma unroll
  for (int j = 0; j < JT; ++j)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[j][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int k0 = 64 * kAhead * wave; k0 < a.K; k0 += 64 * kAhead * kWaves) {
    uint4 fx[2 * kAhead][MT], fw[2 * kAhead][JT];
#pragma unroll
    for (int s = 0; s < 2 * kAhead; ++s) {
      const int k = k0 + 32 * s + 8 * g;
      const bool in = k < a.K;
#pragma unroll
      for (int t = 0; t < MT; ++t) fx[s][t] = load8(x[t], k, in);
#pragma unroll
      for (int j = 0; j < JT; ++j) fw[s][j] = load8(w[j], k, in);
    }
#pragma unroll
    for (int s = 0; s < 2 * kAhead; ++s)
#pragma unroll
      for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int t = 0; t < MT; ++t)
          acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8, fw[s][j]), __builtin_bit_cast(bf16x8, fx[s][t]), acc[j][t],
              0, 0, 0);
  }
#pragma unroll
  for (int j = 0; j < JT; ++j)
#pragma unroll
    for (int t = 0; t < MT; ++t) sums[(wave * MT * JT + j * MT + t) * 64 + lane] = acc[j][t];
  __syncthreads();
  const float s = a.scales ? a.scales[e] : 1.0f;
  for (int i = wave; i < MT * JT; i += kWaves) {
    const int j = i / MT, t = i % MT;
    floatx4 v = sums[i * 64 + lane];
#pragma unroll
    for (int q = 1; q < kWaves; ++q) v += sums[(q * MT * JT + i) * 64 + lane];
    if (16 * t + n >= live) continue;
    store_h<JT>(a.h + (size_t)(first + 16 * t + n) * (48 * JT), 16 * j + 4 * g, o.r, v, s);
  }
}

// The same for ranks past 32, where the factor is what is read most: BB tokens, both operands through
// LDS, deep in flight; two waves along the ranks by two along the tokens.
template <int JT, int BB>
__global__ __launch_bounds__(256) void shrink_tile_kernel(Tokens o, Shrink first_a, Shrink second,
                                                          int groups) {
  constexpr int kThreads = 256, BA = 16 * JT, MA = JT / 2, MB = BB / 32;
  constexpr int kStages = ShrinkLds<JT, BB>::kStages, kStage = ShrinkLds<JT, BB>::kStage;
  using OpA = Operand<false, false, BA, kThreads>;
  using OpB = Operand<false, false, BB, kThreads>;
  extern __shared__ __attribute__((aligned(16))) uint16_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const bool is_first = (int)blockIdx.x < groups;
  const Shrink a = is_first ? first_a : second;
  Place p;
  if (!find_place(o.offsets, o.L, o.T, BB, 1, is_first ? blockIdx.x : blockIdx.x - groups, p)) return;
  OpA oa;
  oa.init(a.w + (size_t)p.e * o.r * a.K, a.K, o.r, a.K, tid);
  const int at = 8 * (tid % 8 ^ OpB::swap(tid / 8));   // the piece of a block that the lane brings
  const uint16_t* x[OpB::kLoads];
#pragma unroll
  for (int j = 0; j < OpB::kLoads; ++j)
    x[j] = a.x + at +
           (size_t)o.tokens[p.first + min(j * OpB::kStep + tid / 8, p.live - 1)] * a.ldx;
  const int wa = wave & 1, wb = wave >> 1;
  const int blocks = (a.K + kBlock - 1) / kBlock;
  auto load = [&](int b, uint16_t* stage) {
#pragma unroll
    for (int j = 0; j < OpA::kLoads; ++j) oa.load(b, stage, j, wave);
#pragma unroll
    for (int j = 0; j < OpB::kLoads; ++j)
      to_lds(b * kBlock + at < a.K ? x[j] + b * kBlock : reinterpret_cast<const uint16_t*>(kZeros),
             stage + BA * kBlock + j * kThreads * 8 + wave * 512);
  };
  floatx4 acc[MA][MB];
#pragma unroll
  for (int m = 0; m < MA; ++m)
#pragma unroll
    for (int t = 0; t < MB; ++t) acc[m][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  auto step = [&](int b, const uint16_t* __restrict__ stage, uint16_t* __restrict__ next) {
    load(b + kStages - 1, next);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8 fa[MA], fb[MB];
#pragma unroll
      for (int m = 0; m < MA; ++m) fa[m] = OpA::read_along(stage, (wa * MA + m) * 16 + n, s, g);
#pragma unroll
      for (int t = 0; t < MB; ++t)
        fb[t] = OpB::read_along(stage + BA * kBlock, (wb * MB + t) * 16 + n, s, g);
#pragma unroll
      for (int m = 0; m < MA; ++m)
#pragma unroll
        for (int t = 0; t < MB; ++t)
          acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[m], fb[t], acc[m][t], 0, 0, 0);
    }
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) load(s, lds + s * kStage);
  int cur = 0;                                         // the buffer of block b
  for (int b = 0; b < blocks; ++b) {
    wait_loads<(OpA::kLoads + OpB::kLoads) * (kStages - 2)>();
    step(b, lds + cur * kStage, lds + (cur == 0 ? kStages - 1 : cur - 1) * kStage);
    cur = cur + 1 == kStages ? 0 : cur + 1;
  }
  wait_loads<0>();
  const float scale = a.scales ? a.scales[p.e] : 1.0f;
#pragma unroll
  for (int t = 0; t < MB; ++t) {
    const int at_row = (wb * MB + t) * 16 + n;
    if (at_row >= p.live) continue;
    uint16_t* const row = a.h + (size_t)(p.first + at_row) * (48 * JT);
#pragma unroll
    for (int m = 0; m < MA; ++m)
      store_h<JT>(row, (wa * MA + m) * 16 + 4 * g, o.r, acc[m][t], scale);
  }
}

struct Expand {
  const int32_t* rows;         // [T]
  int N;
  const uint16_t* h;           // [T, 3, 16 JT]
  const uint16_t* w;           // [L, N, r]
  const float* scales;         // [L], or null
  const uint16_t* base;        // [T, N], or null
  long ld_base;
  uint16_t* out;
  long ld_out;
  int columns;                 // of a workgroup, a multiple of 128 (set by the launch)
};
constexpr int kRestTokens = 64;        // (lanes) of a workgroup that looks for tokens without an adapter

// Tokens without an adapter, of kRestTokens from the first on: out = base, or zeros.
__device__ __forceinline__ void copy_rest(const Expand& a, int T, int first) {
  const int lane = threadIdx.x & 63;
  const bool dead = first + lane < T && a.rows[min(first + lane, T - 1)] < 0;
  for (uint64_t left = __ballot(dead); left; left &= left - 1) {   // (every wave sees the same)
    const size_t t = first + __builtin_ctzll(left);
    for (int c = 8 * threadIdx.x; c < a.N; c += 8 * 256) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (a.base) v = *reinterpret_cast<const uint4*>(a.base + t * a.ld_base + c);
      *reinterpret_cast<uint4*>(a.out + t * a.ld_out + c) = v;
    }
  }
}

// out of 16 MT tokens of one adapter and a.columns columns: each wave takes 32 of these at a time,
// dealt so that a lane's eight results are neighbours.  Workgroups from `groups` on look after the
// tokens without an adapter.
template <int MT, int JT>
__global__ __launch_bounds__(256) void expand_kernel(Tokens o, Expand a, int groups) {
  static_assert(JT <= 2, "ranks past 32 are expand_tile_kernel's");
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  if ((int)blockIdx.x >= groups) {
    copy_rest(a, o.T, (blockIdx.x - groups) * kRestTokens);
    return;
  }
  Place p;
  const int columns = (a.N + a.columns - 1) / a.columns;
  if (!find_place(o.offsets, o.L, o.T, 16 * MT, columns, blockIdx.x, p)) return;
  const int e = p.e, first = p.first, live = p.live;
  const int c0 = p.column * a.columns;
  long token[MT];
  bf16x8 fh[MT][JT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int row = first + min(16 * t + n, live - 1);
    token[t] = o.tokens[row];
#pragma unroll
    for (int s = 0; s < JT; ++s)
      fh[t][s] = *reinterpret_cast<const bf16x8*>(a.h + (size_t)row * (48 * JT) + 32 * s + 8 * g);
  }
  const float scale = a.scales ? a.scales[e] : 1.0f;
  const uint16_t* const w = a.w + (size_t)e * a.N * o.r;
  const int end = min(c0 + a.columns, a.N);
  // W's rows go with both parts of h: with 16 ranks the parts lie in one operand, with 32 in two
  uint4 fw[2], base[MT];
  auto fetch = [&](int c) {                            // under way while the columns before are stored
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      base[t] = make_uint4(0, 0, 0, 0);
      if (a.base && 16 * t + n < live && c + 8 * g < a.N)
        base[t] = *reinterpret_cast<const uint4*>(a.base + token[t] * a.ld_base + c + 8 * g);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int col = min(c + 8 * (n >> 2) + 4 * m + (n & 3), a.N - 1);
      const int j = 8 * g % (16 * JT);
      fw[m] = load8(w + (size_t)col * o.r, j, j < o.r);
    }
  };
  if (c0 + 32 * wave < end) fetch(c0 + 32 * wave);
  for (int c = c0 + 32 * wave; c < end; c += 128) {
    const int to = c + 8 * g;
    uint4 here[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) here[t] = base[t];
    floatx4 acc[2][MT];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        acc[m][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        const bf16x8 v = __builtin_bit_cast(bf16x8, fw[m]);
        acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, fh[t][0], acc[m][t], 0, 0, 0);
        if constexpr (JT > 1)
          acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, fh[t][1], acc[m][t], 0, 0, 0);
      }
    if (c + 128 < end) fetch(c + 128);
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      if (16 * t + n >= live || to >= a.N) continue;
      float v[8];
      values8(here[t], v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf(scale, acc[i / 4][t][i % 4], v[i]);
      *reinterpret_cast<uint4*>(a.out + token[t] * a.ld_out + to) = to_bf16x8(v);
    }
  }
}

// The same for ranks past 32: 64 tokens and 128 columns, W's rows and both parts of h's whole in LDS,
// loaded at once while base is read.
constexpr int kExpandTokens = 64, kExpandTile = 128;
template <int JT>
struct ExpandLds {
  static constexpr int kBlocks = JT / 4;               // of 64 ranks
  static constexpr int kW = kExpandTile * kBlock, kH = kExpandTokens * kBlock;   // elements of each
  static constexpr int kBytes = kBlocks * (kW + 2 * kH) * 2;
};
template <int JT>
__global__ __launch_bounds__(256) void expand_tile_kernel(Tokens o, Expand a, int groups) {
  using Lds = ExpandLds<JT>;
  constexpr int kThreads = 256, MA = 4, MB = 2;        // waves of 64 columns by 32 tokens
  using OpA = Operand<false, true, kExpandTile, kThreads>;
  using OpB = Operand<false, false, kExpandTokens, kThreads>;
  extern __shared__ __attribute__((aligned(16))) uint16_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wa = wave & 1, wb = wave >> 1;
  const int n = lane & 15, g = lane >> 4;
  if ((int)blockIdx.x >= groups) {
    copy_rest(a, o.T, (blockIdx.x - groups) * kRestTokens);
    return;
  }
  Place p;
  const int columns = (a.N + kExpandTile - 1) / kExpandTile;
  if (!find_place(o.offsets, o.L, o.T, kExpandTokens, columns, blockIdx.x, p)) return;
  const int c0 = p.column * kExpandTile;
  OpA oa;
  OpB ob[2];
  oa.init(a.w + ((size_t)p.e * a.N + c0) * o.r, o.r, a.N - c0, o.r, tid);
#pragma unroll
  for (int q = 0; q < 2; ++q)
    ob[q].init(a.h + (size_t)p.first * (48 * JT) + q * 16 * JT, 48 * JT, p.live, 16 * JT, tid);
  uint16_t* const hl = lds + Lds::kBlocks * Lds::kW;
#pragma unroll
  for (int b = 0; b < Lds::kBlocks; ++b) {
#pragma unroll
    for (int j = 0; j < OpA::kLoads; ++j) oa.load(b, lds + b * Lds::kW, j, wave);
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int j = 0; j < OpB::kLoads; ++j)
        ob[q].load(b, hl + (2 * b + q) * Lds::kH, j, wave);
  }
  long token[MB];
  uint4 base[MB][MA / 2];
#pragma unroll
  for (int t = 0; t < MB; ++t) {
    const int row = wb * 32 + 16 * t + n;
    token[t] = o.tokens[p.first + min(row, p.live - 1)];
#pragma unroll
    for (int m = 0; m < MA / 2; ++m) {
      const int to = c0 + wa * 64 + 32 * m + 8 * g;
      base[t][m] = make_uint4(0, 0, 0, 0);
      if (a.base && row < p.live && to < a.N)
        base[t][m] = *reinterpret_cast<const uint4*>(a.base + token[t] * a.ld_base + to);
    }
  }
  const float scale = a.scales ? a.scales[p.e] : 1.0f;
  wait_loads<0>();
  floatx4 acc[MA][MB];
#pragma unroll
  for (int m = 0; m < MA; ++m)
#pragma unroll
    for (int t = 0; t < MB; ++t) acc[m][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int b = 0; b < Lds::kBlocks; ++b)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8 fa[MA];
#pragma unroll
      for (int m = 0; m < MA; ++m)
        fa[m] = OpA::read_along(lds + b * Lds::kW,
                                wa * 64 + m / 2 * 32 + 8 * (n >> 2) + 4 * (m & 1) + (n & 3), s, g);
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int t = 0; t < MB; ++t) {
          const bf16x8 fb = OpB::read_along(hl + (2 * b + q) * Lds::kH, wb * 32 + 16 * t + n, s, g);
#pragma unroll
          for (int m = 0; m < MA; ++m)
            acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[m], fb, acc[m][t], 0, 0, 0);
        }
    }
#pragma unroll
  for (int t = 0; t < MB; ++t) {
    if (wb * 32 + 16 * t + n >= p.live) continue;
#pragma unroll
    for (int m = 0; m < MA / 2; ++m) {
      const int to = c0 + wa * 64 + 32 * m + 8 * g;
      if (to >= a.N) continue;
      float v[8];
      values8(base[t][m], v);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        v[i] = __builtin_fmaf(scale, acc[2 * m + i / 4][t][i % 4], v[i]);
      *reinterpret_cast<uint4*>(a.out + token[t] * a.ld_out + to) = to_bf16x8(v);
    }
  }
}

struct Factors {
  const int32_t* offsets;
  const int32_t* tokens;
  int L, T, r, n, d, splits;
  const uint16_t *x, *dy;
  long ldx, lddy;
  const uint16_t *h, *dh;      // [T, 3, 16 JT]
  const float* scales;
  float *da, *db;              // [L, r, d] and [L, n, r]; where splits > 1 a part's of the workspace
};

constexpr int kChunk = 2048;           // tokens whose indexes lie in LDS
// LDS of factors_kernel: blocks of kB tokens, so many that loads are long under way.
template <int JT>
struct FactorsLds {
  static constexpr int kB = JT <= 2 ? 64 : 32;
  static constexpr int kStages = JT == 1 || JT == 4 ? 3 : 2;           // two workgroups a unit
  static constexpr int kStage = kB * (kGradColumns + 48 * JT);        // elements
  static constexpr int kBytes = kStages * kStage * 2 + kChunk * 4;
};

// The gradients of kGradColumns columns of a factor's long side: dA from x and dh, dB from dy and
// h, both operands across the reduction, which runs over the adapter's tokens in blocks of kB.
// Workgroup (column tile: dA's, then dB's; part of the tokens; adapter).
template <int JT>
__global__ __launch_bounds__(256) void factors_kernel(Factors a) {
  using Lds = FactorsLds<JT>;
  constexpr int kThreads = 256, kRank = 16 * JT, kB = Lds::kB, kStages = Lds::kStages;
  using Wide = Operand<true, false, kGradColumns, kThreads, kB>;
  using Rank = Operand<true, false, kRank, kB * kRank / 8, kB>;        // each part of h
  constexpr int kPartPieces = kB * kRank / 8, kPieces = 3 * kPartPieces;   // 16 bytes each
  constexpr int kHLoads = (kPieces + kThreads - 1) / kThreads;
  constexpr int kLoads = Wide::kLoads + kPieces / kThreads;    // of a wave and block, at least
  static_assert(kPieces % 64 == 0 && kChunk % kB == 0, "whole waves and blocks");
  extern __shared__ __attribute__((aligned(16))) uint16_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int tiles_a = (a.d + kGradColumns - 1) / kGradColumns;
  const bool is_a = (int)blockIdx.x < tiles_a;
  const int c0 = (is_a ? blockIdx.x : blockIdx.x - tiles_a) * kGradColumns;
  const int width = is_a ? a.d : a.n;
  const int e = blockIdx.z;
  int lo, hi;
  group_rows(a.offsets, e, a.T, lo, hi);
  {  // this part of the adapter's tokens, in whole blocks
    const int blocks = (hi - lo + kB - 1) / kB;
    const int from = (int)((long)blocks * blockIdx.y / a.splits) * kB;
    const int upto = (int)((long)blocks * (blockIdx.y + 1) / a.splits) * kB;
    hi = min(hi, lo + upto);
    lo += from;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  const int rows = __builtin_amdgcn_readfirstlane(hi) - lo;
  const uint16_t* const wide = is_a ? a.x : a.dy;
  const long ld = is_a ? a.ldx : a.lddy;
  const uint16_t* const skinny = is_a ? a.dh : a.h;
  const uint16_t* const zeros = reinterpret_cast<const uint16_t*>(kZeros);

  int32_t* const tokens = reinterpret_cast<int32_t*>(lds + kStages * Lds::kStage);   // of a chunk
  const int column = min(Wide::column(tid, 0), width - c0 - 8);
  static_assert(Wide::kStep % 16 == 0, "one column for every load");
  int first = 0, here = 0;     // the chunk's first row, its rows
  // block b of the chunk: the wide rows, then LDS [3][kB][kRank] of h's
  auto load = [&](int b, uint16_t* stage) {
#pragma unroll
    for (int j = 0; j < Wide::kLoads; ++j) {
      const int q = b * kB + j * Wide::kStep + tid / Wide::kPieces;
      const size_t at = (size_t)tokens[min(q, here - 1)] * ld;
      to_lds(q < here ? wide + c0 + column + at : zeros, stage + j * kThreads * 8 + wave * 512);
    }
    uint16_t* const hl = stage + kB * kGradColumns;
#pragma unroll
    for (int j = 0; j < kHLoads; ++j) {
      if (kPieces % kThreads != 0 && j * kThreads + wave * 64 >= kPieces) break;   // (whole waves)
      const int i = j * kThreads + tid;
      const int part = i / kPartPieces, in = i % kPartPieces;
      const int q = in / (kRank / 8), slot = in % (kRank / 8);
      const int c = 8 * (slot ^ Rank::swap(q) << 1);
      const int row = b * kB + q;
      to_lds(row < here ? skinny + (size_t)(lo + first + row) * (3 * kRank) + part * kRank + c : zeros,
             hl + (j * kThreads + wave * 64) * 8);
    }
  };
  constexpr int kTiles = kGradColumns / 16 / 4;        // column tiles of a wave
  floatx4 acc[kTiles][JT];
#pragma unroll
  for (int m = 0; m < kTiles; ++m)
#pragma unroll
    for (int j = 0; j < JT; ++j) acc[m][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  auto step = [&](auto of_a, int b, const uint16_t* __restrict__ stage, uint16_t* __restrict__ next) {
    load(b + kStages - 1, next);
#pragma unroll
    for (int s = 0; s < kB / 32; ++s) {
      bf16x8 fw[kTiles];
#pragma unroll
      for (int m = 0; m < kTiles; ++m)
        fw[m] = Wide::read_across(stage, Wide::across(wave * kTiles + m, n, g), s);
#pragma unroll
      for (int part = 0; part < 3; ++part) {
        const uint16_t* const hl = stage + kB * kGradColumns + part * kB * kRank;
#pragma unroll
        for (int j = 0; j < JT; ++j) {
          const bf16x8 fh = Rank::read_across(hl, Rank::across(j, n, g), s);
#pragma unroll
          for (int m = 0; m < kTiles; ++m)
            acc[m][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                of_a ? fw[m] : fh, of_a ? fh : fw[m], acc[m][j], 0, 0, 0);
        }
      }
    }
  };
  auto run = [&](auto of_a) {                          // (one question, not one for each product)
    for (first = 0; first < rows; first += kChunk) {
      here = min(kChunk, rows - first);
      for (int i = tid; i < here; i += kThreads) tokens[i] = a.tokens[lo + first + i];
      __syncthreads();
#pragma unroll
      for (int s = 0; s < kStages - 1; ++s) load(s, lds + s * Lds::kStage);
      const int blocks = (here + kB - 1) / kB;
      int cur = 0;                                     // the buffer of block b
      for (int b = 0; b < blocks; ++b) {
        wait_loads<kLoads*(kStages - 2)>();
        step(of_a, b, lds + cur * Lds::kStage,
             lds + (cur == 0 ? kStages - 1 : cur - 1) * Lds::kStage);
        cur = cur + 1 == kStages ? 0 : cur + 1;
      }
      wait_loads<0>();
    }
  };
  if (is_a)
    run(std::true_type());
  else
    run(std::false_type());
  const size_t plane = (size_t)blockIdx.y * a.L * a.r * ((size_t)a.n + a.d);
  const float scale = is_a || !a.scales ? 1.0f : a.scales[e];   // (dh has its own in it)
#pragma unroll
  for (int m = 0; m < kTiles; ++m)
#pragma unroll
    for (int j = 0; j < JT; ++j) {
      const int wide0 = c0 + (wave * kTiles + m) * 16;
      if (is_a) {                                      // lane: rank n, columns 4 g ..
        const int rank = 16 * j + n, c = wide0 + 4 * g;
        if (rank < a.r && c < a.d)
          *reinterpret_cast<floatx4*>(a.da + plane + ((size_t)e * a.r + rank) * a.d + c) = acc[m][j];
      } else {                                         // lane: column n, ranks 4 g ..
        const int rank = 16 * j + 4 * g, c = wide0 + n;
        if (rank < a.r && c < a.n)
          *reinterpret_cast<floatx4*>(a.db + plane + ((size_t)e * a.n + c) * a.r + rank) =
              acc[m][j] * scale;
      }
    }
}

// The parts of the factors' gradients, [splits][da's, then db's values], in order.
__global__ __launch_bounds__(256) void sum_parts_kernel(const float* part, int splits, size_t na,
                                                        size_t nb, float* da, float* db) {
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= na + nb) return;
  floatx4 v = *reinterpret_cast<const floatx4*>(part + i);
  for (int s = 1; s < splits; ++s)
    v += *reinterpret_cast<const floatx4*>(part + (size_t)s * (na + nb) + i);
  *reinterpret_cast<floatx4*>(i < na ? da + i : db + (i - na)) = v;
}

template <typename F>
hipError_t by_rank(int r, F launch) {
  if (r <= 16) return launch(std::integral_constant<int, 1>());
  if (r <= 32) return launch(std::integral_constant<int, 2>());
  if (r <= 64) return launch(std::integral_constant<int, 4>());
  return launch(std::integral_constant<int, 8>());
}

// Row tiles of `tile` tokens at most, for the eight XCDs.
long most_tiles(int T, int L, int tile, long columns) {
  const long some = T < L ? T : L;
  return ((some + (T - some) / tile) * columns + 7) / 8 * 8;
}

template <typename K>
hipError_t allow_lds(K kernel, int bytes) {
  if (bytes <= 64 * 1024) return hipSuccess;
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                             hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <int JT, int BB>
hipError_t launch_shrink_tile(const Tokens& o, const Shrink& a, const Shrink* b, hipStream_t stream) {
  constexpr int kBytes = ShrinkLds<JT, BB>::kStages * ShrinkLds<JT, BB>::kStage * 2;
  static_assert(kBytes <= 160 * 1024, "LDS of a compute unit");
  const auto kernel = shrink_tile_kernel<JT, BB>;
  const hipError_t e = allow_lds(kernel, kBytes);
  if (e != hipSuccess) return e;
  const int groups = (int)most_tiles(o.T, o.L, BB, 1);
  kernel<<<b ? 2 * groups : groups, 256, kBytes, stream>>>(o, a, b ? *b : a, groups);
  return hipGetLastError();
}

// One product, or two in one launch.  Tiles of 32 tokens take less for a block (0.27 us against 0.39
// at 72 ranks), as long as every tile has a compute unit of its own.
hipError_t launch_shrink(const Tokens& o, const Shrink& a, const Shrink* b, hipStream_t stream) {
  return by_rank(o.r, [&](auto j) {
    constexpr int JT = decltype(j)::value;
    if constexpr (JT >= 4) {
      if (most_tiles(o.T, o.L, 32, 1) <= 256) return launch_shrink_tile<JT, 32>(o, a, b, stream);
      return launch_shrink_tile<JT, 64>(o, a, b, stream);
    } else {
      constexpr int kBytes = 8 * JT * 64 * 16;
      const int groups = (int)most_tiles(o.T, o.L, 16, 1);
      shrink_kernel<1, JT>
          <<<b ? 2 * groups : groups, 512, kBytes, stream>>>(o, a, b ? *b : a, groups);
      return hipGetLastError();
    }
  });
}

// Workgroups of expand_kernel: enough for every compute unit, each with columns enough to make up for
// its start (finding its tokens and reading their h).
constexpr int kExpandGroups = 1024, kExpandMost = 2048;

hipError_t launch_expand(const Tokens& o, const Expand& args, hipStream_t stream) {
  const long rest = args.out == args.base ? 0 : (o.T + kRestTokens - 1) / kRestTokens;
  return by_rank(o.r, [&](auto j) {
    constexpr int JT = decltype(j)::value;
    if constexpr (JT >= 4) {
      const auto kernel = expand_tile_kernel<JT>;
      const hipError_t e = allow_lds(kernel, ExpandLds<JT>::kBytes);
      if (e != hipSuccess) return e;
      const long columns = (args.N + kExpandTile - 1) / kExpandTile;
      const long groups = most_tiles(o.T, o.L, kExpandTokens, columns);
      if ((groups + rest) * 256 > 0xFFFFFFFFl) return hipErrorInvalidConfiguration;
      kernel<<<(unsigned)(groups + rest), 256, ExpandLds<JT>::kBytes, stream>>>(o, args,
                                                                               (int)groups);
    } else {
      constexpr int MT = 2;
      Expand x = args;
      const long tiles = most_tiles(o.T, o.L, 16 * MT, 1);
      const long share = tiles * x.N / kExpandGroups / 128 * 128;
      x.columns = (int)(share < 128 ? 128 : share < kExpandMost ? share : kExpandMost);
      const long groups = most_tiles(o.T, o.L, 16 * MT, (x.N + x.columns - 1) / x.columns);
      if ((groups + rest) * 256 > 0xFFFFFFFFl) return hipErrorInvalidConfiguration;
      expand_kernel<MT, JT><<<(unsigned)(groups + rest), 256, 0, stream>>>(o, x, (int)groups);
    }
    return hipGetLastError();
  });
}

hipError_t launch_factors(const Factors& f, hipStream_t stream) {
  return by_rank(f.r, [&](auto j) {
    constexpr int JT = decltype(j)::value;
    constexpr int kBytes = FactorsLds<JT>::kBytes;
    static_assert(kBytes <= 160 * 1024, "LDS of a compute unit");
    const auto kernel = factors_kernel<JT>;
    const hipError_t e = allow_lds(kernel, kBytes);
    if (e != hipSuccess) return e;
    const int tiles = (f.n + kGradColumns - 1) / kGradColumns +
                      (f.d + kGradColumns - 1) / kGradColumns;
    kernel<<<dim3(tiles, f.splits, f.L), 256, kBytes, stream>>>(f);
    return hipGetLastError();
  });
}

OrderArgs order_of(const AdaptersArgs& a) {
  return {a.ids, a.T, a.L, a.offsets, a.rows, a.tokens, a.counts};
}

}  // namespace

hipError_t launch_adapters(const AdaptersArgs& a, hipStream_t stream) {
  if (few_tokens(a.T, a.r, a.n, a.d)) {
    if (in_one_launch(a.T, a.r, a.n, a.d)) {
      few_kernel<<<dim3((a.n + 1023) / 1024, a.T), 1024, 0, stream>>>(a);
      return hipGetLastError();
    }
    float* const h = reinterpret_cast<float*>(a.h);    // (fp32 [T, r] in the place of three parts)
    few_shrink_kernel<<<dim3((a.r + 3) / 4, a.T), 256, 0, stream>>>(a, h);
    few_expand_kernel<<<dim3((a.n + 255) / 256, a.T), 256, 0, stream>>>(a, h);
    return hipGetLastError();
  }
  hipError_t e = launch_order(order_of(a), stream);
  if (e != hipSuccess) return e;
  const Tokens o{a.offsets, a.tokens, a.L, a.T, a.r};
  if ((e = launch_shrink(o, {a.x, a.ldx, a.d, a.a, nullptr, a.h}, nullptr, stream)) != hipSuccess)
    return e;
  return launch_expand(
      o, {a.rows, a.n, a.h, a.b, a.scales, a.base, a.ld_base, a.out, a.ld_out, 0}, stream);
}

hipError_t launch_adapters_backward(const AdaptersArgs& a, hipStream_t stream) {
  hipError_t e = launch_order_and_transpose(order_of(a), {a.a, a.at, a.r, a.d}, {a.b, a.bt, a.n, a.r},
                                            stream);
  if (e != hipSuccess) return e;
  if (a.T > 0) {
    const Tokens o{a.offsets, a.tokens, a.L, a.T, a.r};
    const Shrink g{a.dy, a.lddy, a.n, a.bt, a.scales, a.dh};
    if ((e = launch_shrink(o, {a.x, a.ldx, a.d, a.a, nullptr, a.h}, &g, stream)) != hipSuccess)
      return e;
    e = launch_expand(o, {a.rows, a.d, a.dh, a.at, nullptr, a.base, a.ld_base, a.out, a.ld_out, 0},
                      stream);
    if (e != hipSuccess) return e;
  }
  const size_t na = (size_t)a.L * a.r * a.d, nb = (size_t)a.L * a.r * a.n;
  const bool parts = a.splits > 1;
  const Factors f{a.offsets, a.tokens, a.L, a.T, a.r, a.n, a.d, a.splits, a.x, a.dy, a.ldx, a.lddy,
                  a.h, a.dh, a.scales, parts ? a.part : a.da, parts ? a.part + na : a.db};
  if ((e = launch_factors(f, stream)) != hipSuccess) return e;
  if (parts)
    sum_parts_kernel<<<(unsigned)((na + nb) / 4 / 256 + 1), 256, 0, stream>>>(a.part, a.splits, na,
                                                                             nb, a.da, a.db);
  return hipGetLastError();
}

}  // namespace xs
