// Tokens to their pairs' rows and back: dispatch (and its gradient), combine (and its gradients).
//
// rows[t, r] is the row of pair (t, r), or no row at all.  Dispatch reads a token once and writes its
// rows; combine reads a token's rows, sums them in rank order in fp32, weighted, and rounds once
// (the gradient of dispatch is the same without weights); combine's gradient takes a wave for each
// pair: dR = w dy and dw = <dy, R> in one pass over both.  All are bound by memory: 4099 tokens of 2048
// bf16 values, 4 of 8 pairs of each with a row, take 18 us each way (84 MB, 4.7 TB/s) and 26 back
// through combine (151 MB, 5.8 TB/s).
//
// Rows of any length and alignment are moved 16 bytes at a time: the GPU's vector loads and stores
// need no more than the element's alignment (AnyVec says so to the compiler).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "groups.h"
#include "tiles.h"

namespace xs {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ void put(uint16_t& to, float v) { to = to_bf16(v); }
__device__ __forceinline__ void put(float& to, float v) { to = v; }

// 16 bytes of elements at any of their own alignments.
template <typename E>
struct AnyVec {
  static constexpr int kN = 16 / sizeof(E);
  struct __attribute__((packed, aligned(sizeof(E)))) Packed {
    uint32_t w[4];
  };
  union {
    uint32_t w[4];
    E v[kN];
  };
  // elements at p, `n` of them live (the rest stay as they are)
  __device__ __forceinline__ void load(const E* p, int n) {
    if (n >= kN) {
      const Packed q = *reinterpret_cast<const Packed*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = q.w[i];
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] = i < n ? p[i] : E(0);
    }
  }
  __device__ __forceinline__ void store(E* p, int n) const {
    if (n >= kN) {
      Packed q;
#pragma unroll
      for (int i = 0; i < 4; ++i) q.w[i] = w[i];
      *reinterpret_cast<Packed*>(p) = q;
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i)
        if (i < n) p[i] = v[i];
    }
  }
};

template <typename E>
__device__ __forceinline__ const E* row_of(const void* p, long ld, long r) {
  return static_cast<const E*>(p) + r * ld;
}
template <typename E>
__device__ __forceinline__ E* row_of(void* p, long ld, long r) {
  return static_cast<E*>(p) + r * ld;
}

// A row index as it is used: -1 where it is none of the buffer's.
__device__ __forceinline__ int checked(const MoveArgs& a, int row) {
  return (unsigned)row < (unsigned)(a.T * a.k) ? row : -1;
}

// Workgroup (t, chunk): kThreads vectors of token t, to each of its rows.
template <typename E>
__global__ __launch_bounds__(kThreads) void dispatch_kernel(MoveArgs a) {
  using V = AnyVec<E>;
  const int t = blockIdx.x;
  const int c = (blockIdx.y * kThreads + threadIdx.x) * V::kN;
  const int n = a.d - c;
  if (n <= 0) return;
  V x;
  x.load(row_of<E>(a.token, a.ld_token, t) + c, n);
  const int32_t* const rows = a.rows + (size_t)t * a.k;
  for (int r = 0; r < a.k; ++r) {
    const int row = checked(a, rows[r]);
    if (row >= 0) x.store(row_of<E>(a.out_row, a.ld_out_row, row) + c, n);
  }
}

// Workgroup (t, chunk): kThreads vectors of token t's sum.
template <typename E>
__global__ __launch_bounds__(kThreads) void combine_kernel(MoveArgs a) {
  using V = AnyVec<E>;
  const int t = blockIdx.x;
  const int c = (blockIdx.y * kThreads + threadIdx.x) * V::kN;
  const int n = a.d - c;
  if (n <= 0) return;
  float sum[V::kN];
#pragma unroll
  for (int i = 0; i < V::kN; ++i) sum[i] = 0.0f;
  const size_t at = (size_t)t * a.k;
#pragma unroll 4
  for (int r = 0; r < a.k; ++r) {
    const int row = checked(a, a.rows[at + r]);
    if (row < 0) continue;
    const float w = a.w ? a.w[at + r] : 1.0f;
    V v;
    v.load(row_of<E>(a.row, a.ld_row, row) + c, n);
#pragma unroll
    for (int i = 0; i < V::kN; ++i) sum[i] = __builtin_fmaf(w, value(v.v[i]), sum[i]);
  }
  V y;
#pragma unroll
  for (int i = 0; i < V::kN; ++i) put(y.v[i], sum[i]);
  y.store(row_of<E>(a.out_token, a.ld_out_token, t) + c, n);
}

// One wave a pair: dR = w dy, rounded once, and dw = <dy, R> in fp32.
template <typename E>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(MoveArgs a) {
  using V = AnyVec<E>;
  const int lane = threadIdx.x & 63;
  const int p = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (p >= a.T * a.k) return;
  const int row = checked(a, a.rows[p]);
  if (row < 0) {
    if (lane == 0) a.dw[p] = 0.0f;
    return;
  }
  const float w = a.w[p];
  const E* const dy = row_of<E>(a.token, a.ld_token, p / a.k);
  const E* const src = row_of<E>(a.row, a.ld_row, row);
  E* const out = row_of<E>(a.out_row, a.ld_out_row, row);
  float dot = 0.0f;
  for (int c = lane * V::kN; c < a.d; c += 64 * V::kN) {
    const int n = a.d - c;
    V g, v, o;
    g.load(dy + c, n);
    v.load(src + c, n);
#pragma unroll
    for (int i = 0; i < V::kN; ++i) {
      const float x = value(g.v[i]);
      dot = __builtin_fmaf(x, value(v.v[i]), dot);
      put(o.v[i], w * x);
    }
    o.store(out + c, n);
  }
  dot = wave_sum(dot);
  if (lane == 0) a.dw[p] = dot;
}

template <typename F>
hipError_t by_type(int fp32, F launch) {
  if (fp32)
    launch(float());
  else
    launch(uint16_t());
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dispatch(const MoveArgs& a, hipStream_t stream) {
  return by_type(a.fp32, [&](auto e) {
    using E = decltype(e);
    const int chunk = kThreads * AnyVec<E>::kN;
    dispatch_kernel<E><<<dim3(a.T, (a.d + chunk - 1) / chunk), kThreads, 0, stream>>>(a);
  });
}

hipError_t launch_combine(const MoveArgs& a, hipStream_t stream) {
  return by_type(a.fp32, [&](auto e) {
    using E = decltype(e);
    const int chunk = kThreads * AnyVec<E>::kN;
    combine_kernel<E><<<dim3(a.T, (a.d + chunk - 1) / chunk), kThreads, 0, stream>>>(a);
  });
}

hipError_t launch_combine_backward(const MoveArgs& a, hipStream_t stream) {
  return by_type(a.fp32, [&](auto e) {
    using E = decltype(e);
    const int waves = kThreads / 64;
    combine_backward_kernel<E><<<(a.T * a.k + waves - 1) / waves, kThreads, 0, stream>>>(a);
  });
}

}  // namespace xs
