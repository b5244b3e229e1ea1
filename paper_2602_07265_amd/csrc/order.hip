// The (token, rank) pairs of a routing in expert order: sorted by expert, ties by pair.
//
// A stable counting sort: the row of a pair is the number of pairs of lower experts plus the number
// of earlier pairs of its own.  A wave takes a run of consecutive pairs, 64 at a time; the
// lanes that hold the same expert find each other by one ballot for each bit of the id, so that
// a lane's place among them is a count of lower lanes and nothing depends on the order of
// atomics.  One workgroup sorts up to kOrderOne pairs in one launch; more go in two: the counts
// of each workgroup's part, then every workgroup sums the parts before its own.  Both sides at 4096
// pairs of 128 experts: 6.9 and 6.6 us (which need a workspace); at 8192 of 256: 12.0 and 6.4.
//
// A call reads and writes 12 bytes a pair, 1.6 MB at 131072 pairs: the launches and the waves'
// chains over their runs bound it.  32768 pairs of 256 experts take 7.5 us, 131072 10.0 and 2^20 22
// (0.6 TB/s).  In parts of 4096 pairs, of which a wave has four steps: 10.1, 10.8 and 23; of 2048
// pairs 2^20 take 32, for each workgroup sums the counts of all 512.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "groups.h"
#include "wave.h"

namespace xs {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// What a lane wrote to the wave's part of LDS before this, its other lanes read after it (the wave's
// LDS operations are done in order; the compiler keeps that order here).
__device__ __forceinline__ void lanes_meet() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The lanes whose key (of `bits` bits) is this lane's.
__device__ __forceinline__ uint64_t same_key(int key, int bits) {
  uint64_t m = ~0ull;
  for (int b = 0; b < bits; ++b) {
    const bool one = (key >> b) & 1;
    const uint64_t s = __ballot(one);
    m &= one ? s : ~s;
  }
  return m;
}

__device__ __forceinline__ int lower_lanes(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32),
                                   __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

__device__ __forceinline__ int key_of(const OrderArgs& a, int i, int end) {
  const int id = i < end ? a.ids[i] : -1;
  return (unsigned)id < (unsigned)a.E ? id : a.E;      // E: no expert
}

// The run of consecutive pairs of a wave among those that its workgroup sorts, and each pair's place
// among its expert's in the run, of which it keeps the counts.
template <int kSteps>                                  // of 64 pairs, at most
struct Run {
  int first, last;
  int key[kSteps], rank[kSteps];

  __device__ __forceinline__ Run(int begin, int end, int wave) {
    const int step = ((end - begin + kWaves - 1) / kWaves + 63) / 64 * 64;
    first = min(begin + wave * step, end);
    last = min(first + step, end);
  }
  // counts [E]: the wave's own
  __device__ __forceinline__ void count(const OrderArgs& a, int* counts, int bits, int lane) {
    for (int e = lane; e < a.E; e += 64) counts[e] = 0;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) key[s] = key_of(a, first + 64 * s + lane, last);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      if (first + 64 * s >= last) break;
      lanes_meet();                                    // a step reads what the last one wrote
      const uint64_t same = same_key(key[s], bits);
      const int lower = lower_lanes(same);
      const bool live = key[s] < a.E;
      const int before = live ? counts[key[s]] : 0;
      rank[s] = before + lower;
      lanes_meet();                                    // all lanes read before one writes
      if (live && lower == 0) counts[key[s]] = before + __popcll(same);
    }
  }
  // next [E]: the row of the run's first pair of each expert
  __device__ __forceinline__ void place(const OrderArgs& a, const int* next, int lane) const {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int p = first + 64 * s + lane;
      if (p >= last) break;
      const int row = key[s] < a.E ? next[key[s]] + rank[s] : -1;
      a.rows[p] = row;
      if (row >= 0) a.pair_of[row] = p;
    }
  }
};

// Exclusive sum of v over the threads of the workgroup; `total` the sum of all.
__device__ __forceinline__ int block_scan(int v, int* part, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int upto = wave_scan(v);
  if (lane == 63) part[wave] = upto;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += w < wave ? part[w] : 0;
    total += part[w];
  }
  __syncthreads();
  return before + upto - v;
}

// Both matrices of expert e, kThreads threads a workgroup; a thread takes eight rows of a column.
struct Transposes {
  Transposed first, second;
  int groups, groups_first;    // workgroups of an expert, those of its first matrix
};
int transpose_groups(const Transposed& m) {
  return (int)(((size_t)m.rows / 8 * m.cols + kThreads - 1) / kThreads);
}
__device__ __forceinline__ void transpose(const Transposes& t, int e, int group) {
  const bool first = group < t.groups_first;
  const Transposed m = first ? t.first : t.second;
  const size_t i = (size_t)(first ? group : group - t.groups_first) * kThreads + threadIdx.x;
  const int c = (int)(i % m.cols), r = (int)(i / m.cols) * 8;
  if (r >= m.rows) return;
  const size_t at = (size_t)e * m.rows * m.cols;
  uint32_t v[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = m.in[at + (size_t)(r + q) * m.cols + c];
  *reinterpret_cast<uint4*>(m.out + at + (size_t)c * m.rows + r) =
      make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}
__global__ __launch_bounds__(kThreads) void transpose_kernel(Transposes t, const int32_t* offsets) {
  const int e = blockIdx.y;
  if (offsets[e] < offsets[e + 1]) transpose(t, e, blockIdx.x);
}

// The whole sort (kParts false), or the second launch of two: part blockIdx.x of the pairs, whose
// counts[part][e] the first launch wrote.
template <bool kParts>
__global__ __launch_bounds__(kThreads) void order_kernel(OrderArgs a, int part_size, int bits,
                                                         Transposes beside) {
  extern __shared__ int lds[];                         // [kWaves][E] and [kWaves]
  if (!kParts && blockIdx.x > 0) {                     // (an expert's pairs are not known yet)
    const int e = (blockIdx.x - 1) / beside.groups;
    int has = 0;
    for (int i = threadIdx.x; i < a.pairs; i += kThreads) has |= a.ids[i] == e;
    if (__syncthreads_or(has)) transpose(beside, e, (blockIdx.x - 1) % beside.groups);
    return;
  }
  int* const part = lds + kWaves * a.E;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int begin = kParts ? blockIdx.x * part_size : 0;
  const int end = kParts ? min(begin + part_size, a.pairs) : a.pairs;
  Run<(kParts ? kOrderMost : kOrderOne) / kThreads> run(begin, end, wave);
  int* const mine = lds + wave * a.E;
  run.count(a, mine, bits, lane);
  // thread e: expert e's pairs in all parts and in those before this one
  int all = 0, before = 0;
  if (kParts && tid < a.E) {
    const int parts = gridDim.x;
#pragma unroll 8
    for (int b = 0; b < parts; ++b) {
      const int c = a.counts[(size_t)b * a.E + tid];
      all += c;
      before += b < (int)blockIdx.x ? c : 0;
    }
  }
  __syncthreads();
  if (!kParts && tid < a.E)
    for (int w = 0; w < kWaves; ++w) all += lds[w * a.E + tid];
  int total;
  const int first = block_scan(tid < a.E ? all : 0, part, total);
  if (tid < a.E) {
    int at = first + before;
    for (int w = 0; w < kWaves; ++w) {
      const int c = lds[w * a.E + tid];
      lds[w * a.E + tid] = at;
      at += c;
    }
    if (!kParts || blockIdx.x == 0) a.offsets[tid] = first;
  }
  if (tid == 0 && (!kParts || blockIdx.x == 0)) a.offsets[a.E] = total;
  __syncthreads();
  run.place(a, mine, lane);
  // rows past the last expert's hold no pair
  for (int p = max(total, begin) + tid; p < end; p += kThreads) a.pair_of[p] = -1;
}

__global__ __launch_bounds__(kThreads) void order_count_kernel(OrderArgs a, int part_size) {
  extern __shared__ int lds[];                         // [E]
  const int begin = blockIdx.x * part_size, end = min(begin + part_size, a.pairs);
  for (int e = threadIdx.x; e < a.E; e += kThreads) lds[e] = 0;
  __syncthreads();
  for (int i = begin + threadIdx.x; i < end; i += kThreads) {
    const int key = key_of(a, i, end);
    if (key < a.E) atomicAdd(&lds[key], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kThreads)
    a.counts[(size_t)blockIdx.x * a.E + e] = lds[e];
}

hipError_t run(const OrderArgs& a, const Transposes& beside, hipStream_t stream) {
  int bits = 1;
  while ((1 << bits) <= a.E) ++bits;                   // keys 0 .. E
  const size_t lds = sizeof(int) * (size_t(kWaves) * a.E + kWaves);
  const int parts = order_parts(a.pairs), part = order_part(a.pairs);
  const auto kernel = parts ? order_kernel<true> : order_kernel<false>;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  if (parts)
    order_count_kernel<<<parts, kThreads, sizeof(int) * a.E, stream>>>(a, part);
  const unsigned grid = parts ? parts : 1 + a.E * beside.groups;
  kernel<<<grid, kThreads, lds, stream>>>(a, part, bits, beside);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_order(const OrderArgs& a, hipStream_t stream) {
  return run(a, Transposes{}, stream);
}

// Every workgroup beside the sort looks through the ids for its expert, up to kOrderOne of them: a launch
// less, as long as the workgroups are so few that they take no longer than the sort (adapters' gradients
// of 4000 tokens, 5 of rank 16, n = d = 4096: 55.7 us, 58.0 in two launches; of 13 tokens 35 and 41 with
// the forward call; 1024 workgroups, 1000 tokens of 64 adapters, 56.4 and 58.2; 2048 of 128 91.8 and 94.3;
// 4096 of 256 162.1 and 159.7).
constexpr int kMostBeside = 1024;
hipError_t launch_order_and_transpose(const OrderArgs& a, const Transposed& first,
                                      const Transposed& second, hipStream_t stream) {
  Transposes t{first, second, 0, transpose_groups(first)};
  const int groups = t.groups_first + transpose_groups(second);
  const bool beside = a.pairs > 0 && order_parts(a.pairs) == 0 && (long)a.E * groups <= kMostBeside;
  if (beside) t.groups = groups;
  const hipError_t e = run(a, t, stream);
  if (e != hipSuccess || beside || a.pairs == 0) return e;
  transpose_kernel<<<dim3(groups, a.E), kThreads, 0, stream>>>(t, a.offsets);
  return hipGetLastError();
}

}  // namespace xs
