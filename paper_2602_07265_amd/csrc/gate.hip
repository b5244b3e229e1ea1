// Routing by scores, bias and groups (xshare_gate) and the gradient of its logits.
//
// One wave holds one token's N <= 64 Q experts, expert j = lane + 64 q in register q.  The
// choice compares order-preserving integer keys (ord of c, 0: not available): k rounds of a
// wave-wide maximum, the lowest index among its holders.  Group scores come from a copy of
// the keys in LDS, one lane for each group.
//
// Compiled with -ffp-contract=off: every step of a score is one fp32 operation.
#pragma clang fp contract(off)

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "blocks.h"

namespace xs {
namespace {

constexpr int kWaves = 4;   // tokens of a workgroup
// Weights are divided by no less than this: sigmoid scores that all underflow give weights
// (and a gradient) of zero, not NaN.
constexpr float kLeastSum = 0x1p-126f;

__device__ __forceinline__ uint32_t ord(float h) {
  const uint32_t b = __float_as_uint(h);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float unord(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}

template <typename T>
__device__ __forceinline__ T wave_all(T v, T (*op)(T, T)) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) v = op(v, __shfl_xor(v, m));
  return v;
}
__device__ __forceinline__ uint32_t max_u(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t min_u(uint32_t a, uint32_t b) { return a < b ? a : b; }
__device__ __forceinline__ float max_f(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float add_f(float a, float b) { return a + b; }

// Logit j of a row; + 0.0 makes -0.0 equal to +0.0.
__device__ __forceinline__ float logit(const GateArgs& a, const void* row, int j) {
  const float h = a.bf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(row)[j] << 16)
                         : static_cast<const float*>(row)[j];
  return h + 0.0f;
}
__device__ __forceinline__ const void* logits_row(const GateArgs& a, int t) {
  return static_cast<const char*>(a.logits) + (size_t)t * a.ld * (a.bf16 ? 2 : 4);
}

// The score of logit h; m and z: the row's maximum and sum of exponentials (softmax).
__device__ __forceinline__ float score(const GateArgs& a, float h, float m, float z) {
  return a.sigmoid ? 1.0f / (1.0f + expf(-h)) : expf(h - m) / z;
}

// The row's logits in registers (-inf past N) and, for softmax, its maximum and sum.
template <int Q>
__device__ __forceinline__ void load_row(const GateArgs& a, const void* row, int lane,
                                         float (&h)[Q], float& m, float& z) {
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int j = lane + 64 * q;
    h[q] = j < a.N ? logit(a, row, j) : -INFINITY;
  }
  m = z = 0.0f;
  if (a.sigmoid) return;
  m = h[0];
#pragma unroll
  for (int q = 1; q < Q; ++q) m = fmaxf(m, h[q]);
  m = wave_all<float>(m, max_f);
#pragma unroll
  for (int q = 0; q < Q; ++q) z += expf(h[q] - m);
  z = wave_all<float>(z, add_f);
}

template <int Q>
__global__ __launch_bounds__(64 * kWaves) void gate_kernel(GateArgs a) {
  __shared__ uint32_t keys[kWaves][64 * Q];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.x * kWaves + wave;
  if (t >= a.T) return;
  const void* const row = logits_row(a, t);
  float h[Q], m, z;
  load_row<Q>(a, row, lane, h, m, z);
  const bool grouped = a.top_groups < a.G;
  uint32_t key[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int j = lane + 64 * q;
    key[q] = j < a.N ? ord(a.bias ? score(a, h[q], m, z) + a.bias[j] : h[q]) : 0u;
  }
  if (grouped) {
    const int size = a.N / a.G;
    // what a group's score is made of: the keys, or the scores where the key is the logit
    uint32_t* const mine = keys[wave];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = lane + 64 * q;
      if (j < a.N) mine[j] = a.top2 && !a.bias ? ord(score(a, h[q], m, z)) : key[q];
    }
    uint32_t g = 0u;
    if (lane < a.G) {
      uint32_t b1 = 0u, b2 = 0u;
      for (int i = 0; i < size; ++i) {
        const uint32_t v = mine[lane * size + i];
        b2 = max_u(b2, min_u(b1, v));
        b1 = max_u(b1, v);
      }
      g = a.top2 ? ord((unord(b1) + unord(b2)) + 0.0f) : b1;
    }
    // the groups that at least top_groups others beat are out
    int beaten = 0;
    for (int o = 0; o < a.G; ++o) {
      const uint32_t v = __shfl(g, o);
      beaten += v > g || (v == g && o < lane);
    }
    const uint64_t keep = __ballot(lane < a.G && beaten < a.top_groups);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = lane + 64 * q;
      if (j < a.N && !((keep >> (j / size)) & 1)) key[q] = 0u;
    }
  }
  int id = 0;   // lane r: the expert of rank r
  for (int r = 0; r < a.k; ++r) {
    uint32_t best = 0u, at = 0xFFFFFFFFu;
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (key[q] > best) {
        best = key[q];
        at = lane + 64 * q;
      }
    const uint32_t top = wave_all<uint32_t>(best, max_u);
    const uint32_t j = wave_all<uint32_t>(best == top ? at : 0xFFFFFFFFu, min_u);
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (j == (uint32_t)(lane + 64 * q)) key[q] = 0u;
    if (lane == r) id = (int)min_u(j, a.N - 1);   // finite logits always leave an expert
  }
  float w = lane < a.k ? score(a, logit(a, row, id), m, z) : 0.0f;
  if (a.renormalize) w /= fmaxf(wave_all<float>(w, add_f), kLeastSum);
  if (lane < a.k) {
    a.ids[(size_t)t * a.k + lane] = id;
    a.w[(size_t)t * a.k + lane] = w * a.scale;
  }
}

// dlogits of a row: the chosen experts' terms in an LDS row, written out whole.
template <int Q>
__global__ __launch_bounds__(64 * kWaves) void gate_backward_kernel(GateArgs a) {
  __shared__ float rows[kWaves][64 * Q];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.x * kWaves + wave;
  if (t >= a.T) return;
  const void* const row = logits_row(a, t);
  float* const mine = rows[wave];
  float h[Q], m, z;
  load_row<Q>(a, row, lane, h, m, z);
  int id = lane < a.k ? a.ids[(size_t)t * a.k + lane] : -1;
  if (id < 0 || id >= a.N) id = -1;
  const float s = id >= 0 ? score(a, logit(a, row, id), m, z) : 0.0f;
  float ds = id >= 0 ? a.scale * a.dw[(size_t)t * a.k + lane] : 0.0f;
  if (a.renormalize) {
    const float total = wave_all<float>(s, add_f);
    const float mean = wave_all<float>(ds * s, add_f) / total;
    ds = id >= 0 && total >= kLeastSum ? (ds - mean) / total : 0.0f;
  }
  // softmax's common term, sum of ds s, which renormalised weights make zero
  const float dot = a.sigmoid || a.renormalize ? 0.0f : wave_all<float>(ds * s, add_f);
#pragma unroll
  for (int q = 0; q < Q; ++q) mine[lane + 64 * q] = 0.0f;
  if (id >= 0) mine[id] = ds;
  float* const out = a.dlogits + (size_t)t * a.N;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int j = lane + 64 * q;
    if (j >= a.N) continue;
    const float sj = score(a, h[q], m, z), dj = mine[j];
    out[j] = a.sigmoid ? dj * sj * (1.0f - sj) : sj * (dj - dot);
  }
}

template <typename F>
hipError_t by_width(int N, F launch) {
  if (N <= 64) return launch(std::integral_constant<int, 1>());
  if (N <= 128) return launch(std::integral_constant<int, 2>());
  if (N <= 256) return launch(std::integral_constant<int, 4>());
  if (N <= 512) return launch(std::integral_constant<int, 8>());
  return launch(std::integral_constant<int, 16>());
}

}  // namespace

hipError_t launch_gate(const GateArgs& a, hipStream_t stream) {
  return by_width(a.N, [&](auto q) {
    gate_kernel<decltype(q)::value>
        <<<(a.T + kWaves - 1) / kWaves, 64 * kWaves, 0, stream>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_gate_backward(const GateArgs& a, hipStream_t stream) {
  return by_width(a.N, [&](auto q) {
    gate_backward_kernel<decltype(q)::value>
        <<<(a.T + kWaves - 1) / kWaves, 64 * kWaves, 0, stream>>>(a);
    return hipGetLastError();
  });
}

}  // namespace xs
