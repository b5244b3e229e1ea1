// Routing by scores, bias and groups (xshare_gate) and the gradient of its logits.
//
// One wave holds one token's N <= 64 Q experts, expert j = Q lane + q in register q, so that a
// lower lane holds lower experts.  The choice compares order-preserving integer keys (ord of c,
// 0: not available): k rounds of a wave-wide maximum (six DPP steps), whose first holder is the
// lowest lane of a ballot.  A group of experts that fills whole lanes, a power of two of them,
// has its score reduced among those lanes; other groups go over a copy of the keys in LDS, one
// lane for each group.
//
// A call reads T N logits and writes T k pairs, 9 MB at T = 8192, N = 256, about 2 us of
// memory time; the instructions of the rounds and scores bound it there (10.4 us in groups of 32,
// k = 8), the launch and the rounds' chain at T = 1 (4.2 us).  With reductions through LDS
// instead of DPP it took 19.5 and 7.5 us.
//
// Compiled with -ffp-contract=off: every step of a score is one fp32 operation.
#pragma clang fp contract(off)

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "blocks.h"
#include "wave.h"

namespace xs {
namespace {

constexpr int kWaves = 4;   // tokens of a workgroup
// Weights are divided by no less than this: sigmoid scores that all underflow give weights
// (and a gradient) of zero, not NaN.
constexpr float kLeastSum = 0x1p-126f;
// Logits up to this mask their expert: -inf, and the lowest finite values of bf16 (which programs
// put in fp32 logits too) and of fp32.
constexpr float kMask = -0x1.FEp127f;

__device__ __forceinline__ float from_bf16(uint32_t b) { return __uint_as_float(b << 16); }

// What a lane wrote to the wave's part of LDS before this, its other lanes read after it (the wave's
// LDS operations are done in order; the compiler keeps that order here).
__device__ __forceinline__ void lanes_meet() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Logit j of a row; + 0.0 makes -0.0 equal to +0.0.
__device__ __forceinline__ float logit(const GateArgs& a, const void* row, int j) {
  const float h = a.bf16 ? from_bf16(static_cast<const uint16_t*>(row)[j])
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

// d score / d logit of a sigmoid, s (1 - s): the subtraction would leave nothing of 1 - s from a
// logit of 17 on.
__device__ __forceinline__ float sigmoid_slope(float h) {
  const float e = expf(-fabsf(h));
  return e / ((1.0f + e) * (1.0f + e));
}

// The lane's logits (-inf past N) and, for softmax, the row's maximum and sum.  a.vec: the rows
// are aligned for loads of Q logits at once, and N is a multiple of Q.
template <int Q>
__device__ __forceinline__ void load_row(const GateArgs& a, const void* row, int lane,
                                         float (&h)[Q], float& m, float& z) {
  const int j0 = Q * lane;
  if (Q > 1 && a.vec) {
#pragma unroll
    for (int q = 0; q < Q; ++q) h[q] = -INFINITY;
    if (j0 < a.N) {
      if (a.bf16) {
        const uint32_t* const p = reinterpret_cast<const uint32_t*>(
            static_cast<const uint16_t*>(row) + j0);
#pragma unroll
        for (int q = 0; q < Q / 2; ++q) {
          const uint32_t v = p[q];
          h[2 * q] = __uint_as_float(v << 16) + 0.0f;
          h[2 * q + 1] = __uint_as_float(v & 0xFFFF0000u) + 0.0f;
        }
      } else {
        const float2* const p =
            reinterpret_cast<const float2*>(static_cast<const float*>(row) + j0);
#pragma unroll
        for (int q = 0; q < Q / 2; ++q) {
          const float2 v = p[q];
          h[2 * q] = v.x + 0.0f;
          h[2 * q + 1] = v.y + 0.0f;
        }
      }
    }
  } else {
#pragma unroll
    for (int q = 0; q < Q; ++q) h[q] = j0 + q < a.N ? logit(a, row, j0 + q) : -INFINITY;
  }
  m = z = 0.0f;
  if (a.sigmoid) return;
  m = h[0];
#pragma unroll
  for (int q = 1; q < Q; ++q) m = fmaxf(m, h[q]);
  m = wave_fmax(m);
  m = m <= kMask ? 0.0f : m;             // a row of masked experts: every score 0
#pragma unroll
  for (int q = 0; q < Q; ++q) z += expf(h[q] - m);
  z = fmaxf(wave_sum(z), kLeastSum);
}

// The lane's biases (0 past N and where there are none), under way while the row is loaded.
template <int Q>
__device__ __forceinline__ void load_bias(const GateArgs& a, int lane, float (&b)[Q]) {
  const int j0 = Q * lane;
#pragma unroll
  for (int q = 0; q < Q; ++q) b[q] = 0.0f;
  if (!a.bias) return;
  if (Q > 1 && a.vec_bias) {
    if (j0 < a.N) {
#pragma unroll
      for (int q = 0; q < Q; q += 2) {
        const float2 v = *reinterpret_cast<const float2*>(a.bias + j0 + q);
        b[q] = v.x;
        b[q + (Q > 1)] = v.y;
      }
    }
  } else {
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (j0 + q < a.N) b[q] = a.bias[j0 + q];
  }
}

// The two best of a group, from its parts' (0: no live expert).
struct Top2 {
  uint32_t b1, b2;
  __device__ __forceinline__ void add(uint32_t v) {
    b2 = max(b2, min(b1, v));
    b1 = max(b1, v);
  }
  __device__ __forceinline__ void add(const Top2& o) {
    b2 = max(min(b1, o.b1), max(b2, o.b2));
    b1 = max(b1, o.b1);
  }
  // The sum of the live ones of two; 0, behind every other group, where there is none.
  __device__ __forceinline__ uint32_t score(bool top2) const {
    if (!top2 || b2 == 0u) return b1;
    return ord((unord(b1) + unord(b2)) + 0.0f);
  }
};

// Clears the keys of the experts outside the top_groups best groups.  base: what a group's score
// is made of, where it is not the keys.
template <int Q>
__device__ __forceinline__ void limit_groups(const GateArgs& a, int lane, uint32_t* copy,
                                             const uint32_t (&base)[Q], uint32_t (&key)[Q]) {
  const int size = a.N / a.G, span = size / Q;      // lanes of a group
  const bool lanes = span * Q == size && (span & (span - 1)) == 0;
  Top2 top{0u, 0u};
  if (lanes) {
#pragma unroll
    for (int q = 0; q < Q; ++q) top.add(base[q]);
    for (int s = 1; s < span; s *= 2) {
      Top2 o;
      o.b1 = (uint32_t)__shfl_xor((int)top.b1, s);
      o.b2 = (uint32_t)__shfl_xor((int)top.b2, s);
      top.add(o);
    }
  } else {
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (Q * lane + q < a.N) copy[Q * lane + q] = base[q];
    lanes_meet();
    if (lane < a.G)
      for (int i = 0; i < size; ++i) top.add(copy[lane * size + i]);
  }
  const uint32_t mine = top.score(a.top2);
  const int group = lanes ? lane / span : lane;
  int beaten = 0;                                   // groups ahead of this one
  for (int o = 0; o < a.G; ++o) {
    const uint32_t v = (uint32_t)__builtin_amdgcn_readlane((int)mine, lanes ? o * span : o);
    beaten += v > mine || (v == mine && o < group);
  }
  if (lanes) {
#pragma unroll
    for (int q = 0; q < Q; ++q) key[q] = beaten < a.top_groups ? key[q] : 0u;
  } else {
    const uint64_t keep = __ballot(lane < a.G && beaten < a.top_groups);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = Q * lane + q;
      if (j < a.N && !((keep >> (j / size)) & 1)) key[q] = 0u;
    }
  }
}

template <int Q>
__global__ __launch_bounds__(64 * kWaves) void gate_kernel(GateArgs a) {
  __shared__ uint32_t copies[kWaves][64 * Q];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.x * kWaves + wave;
  if (t >= a.T) return;
  const void* const row = logits_row(a, t);
  float h[Q], b[Q], m, z;
  load_bias<Q>(a, lane, b);
  load_row<Q>(a, row, lane, h, m, z);
  const bool grouped = a.top_groups < a.G;
  uint32_t key[Q], base[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int j = Q * lane + q;
    key[q] = base[q] = 0u;
    if (j >= a.N) continue;
    const bool plain = !a.bias && !(grouped && a.top2);
    const float s = plain ? 0.0f : score(a, h[q], m, z);
    const float c = a.bias ? s + b[q] : h[q];
    const bool masked = h[q] <= kMask;
    key[q] = ord(masked ? h[q] : c);                 // below any score plus a finite bias
    // (in a sum of two a masked expert has no part: live ones may add up to less than 0)
    base[q] = !a.top2 ? key[q] : masked ? 0u : ord(a.bias ? c : s);
  }
  if (grouped) limit_groups<Q>(a, lane, copies[wave], base, key);
  int id = 0;   // lane r: the expert of rank r
  for (int r = 0; r < a.k; ++r) {
    uint32_t best = key[0];
    int at = 0;
#pragma unroll
    for (int q = 1; q < Q; ++q) {
      at = key[q] > best ? q : at;
      best = max(best, key[q]);
    }
    const uint32_t top = wave_max(best);
    const int holder = __builtin_ctzll(__ballot(best == top));
    const int q0 = __builtin_amdgcn_readlane(at, holder);
    const int j = min(Q * holder + q0, a.N - 1);   // (finite logits always leave an expert)
#pragma unroll
    for (int q = 0; q < Q; ++q) key[q] = lane == holder && q == q0 ? 0u : key[q];
    id = lane == r ? j : id;
  }
  float w = lane < a.k ? score(a, logit(a, row, id), m, z) : 0.0f;
  if (a.renormalize) w /= fmaxf(wave_sum(w), kLeastSum);
  if (lane < a.k) {
    a.ids[(size_t)t * a.k + lane] = id;
    a.w[(size_t)t * a.k + lane] = w * a.scale;
  }
}

// dlogits of a row: the chosen experts' terms in an LDS row, written out whole.  T = 4099, N = 128
// from bf16 logits: 4.3 us for 3.4 MB.
template <int Q>
__global__ __launch_bounds__(64 * kWaves) void gate_backward_kernel(GateArgs a) {
  __shared__ float rows[kWaves][64 * Q];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.x * kWaves + wave;
  if (t >= a.T) return;
  const void* const row = logits_row(a, t);
  float* const mine = rows[wave];
#pragma unroll
  for (int q = 0; q < Q; ++q) mine[Q * lane + q] = 0.0f;
  int id = lane < a.k ? a.ids[(size_t)t * a.k + lane] : -1;
  if (id < 0 || id >= a.N) id = -1;
  float h[Q], m, z;
  load_row<Q>(a, row, lane, h, m, z);
  const float s = id >= 0 ? score(a, logit(a, row, id), m, z) : 0.0f;
  float ds = id >= 0 ? a.scale * a.dw[(size_t)t * a.k + lane] : 0.0f;
  if (a.renormalize) {
    const float total = wave_sum(s);
    const float mean = wave_sum(ds * s) / total;
    ds = id >= 0 && total >= kLeastSum ? (ds - mean) / total : 0.0f;
  }
  // softmax's common term, sum of ds s, which renormalised weights make zero
  const float dot = a.sigmoid || a.renormalize ? 0.0f : wave_sum(ds * s);
  float sj[Q];                             // scores; their slopes where they are sigmoids
#pragma unroll
  for (int q = 0; q < Q; ++q) sj[q] = a.sigmoid ? sigmoid_slope(h[q]) : score(a, h[q], m, z);
  lanes_meet();
  if (id >= 0) mine[id] = ds;
  lanes_meet();
  float* const out = a.dlogits + (size_t)t * a.N + Q * lane;
  float d[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const float dj = mine[Q * lane + q];
    d[q] = a.sigmoid ? dj * sj[q] : sj[q] * (dj - dot);
  }
  if (Q > 1 && a.vec_out) {
    if (Q * lane < a.N)
#pragma unroll
      for (int q = 0; q < Q; q += 2)
        *reinterpret_cast<float2*>(out + q) = make_float2(d[q], d[q + (Q > 1)]);
  } else {
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (Q * lane + q < a.N) out[q] = d[q];
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

// Whether rows of `size`-byte elements, `ld` apart, can be read Q elements at once in pairs.
bool pairs_aligned(const void* p, long ld, int N, int Q, int size) {
  return N % Q == 0 && ld % 2 == 0 && reinterpret_cast<uintptr_t>(p) % (2 * size) == 0;
}

}  // namespace

hipError_t launch_gate(const GateArgs& args, hipStream_t stream) {
  return by_width(args.N, [&](auto q) {
    constexpr int Q = decltype(q)::value;
    GateArgs a = args;
    a.vec = pairs_aligned(a.logits, a.ld, a.N, Q, a.bf16 ? 2 : 4);
    a.vec_bias = pairs_aligned(a.bias, a.N, a.N, Q, 4);
    gate_kernel<Q><<<(a.T + kWaves - 1) / kWaves, 64 * kWaves, 0, stream>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_gate_backward(const GateArgs& args, hipStream_t stream) {
  return by_width(args.N, [&](auto q) {
    constexpr int Q = decltype(q)::value;
    GateArgs a = args;
    a.vec = pairs_aligned(a.logits, a.ld, a.N, Q, a.bf16 ? 2 : 4);
    a.vec_out = pairs_aligned(a.dlogits, a.N, a.N, Q, 4);
    gate_backward_kernel<Q><<<(a.T + kWaves - 1) / kWaves, 64 * kWaves, 0, stream>>>(a);
    return hipGetLastError();
  });
}

}  // namespace xs
