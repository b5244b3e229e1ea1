// Wave-wide reductions and ordered keys of the kernels that rank experts.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace xs {
namespace {

// Order-preserving map of finite fp32 values to uint32 (> 0); 0 marks "no value".
__device__ __forceinline__ uint32_t ord(float h) {
  const uint32_t b = __float_as_uint(h);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float unord(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}

// One DPP step of a reduction: the value of the lane that Ctrl names, or the reduction's
// identity in rows outside RowMask.  With the identity as the "old" operand the compiler
// folds the move into the reducing instruction (one v_max_u32_dpp / v_min_u32_dpp per step
// instead of two moves and the max).
template <int Ctrl, int RowMask, uint32_t Identity>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)Identity, (int)v, Ctrl, RowMask, 0xF, false);
}

// Wave-wide max / min of a uint32 with DPP (quad swaps, row mirrors, row broadcasts);
// lane 63 ends with the result, which is returned to every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, dpp<0xB1, 0xF, 0u>(v));   // quad_perm [1,0,3,2]
  v = max(v, dpp<0x4E, 0xF, 0u>(v));   // quad_perm [2,3,0,1]
  v = max(v, dpp<0x141, 0xF, 0u>(v));  // row_half_mirror
  v = max(v, dpp<0x140, 0xF, 0u>(v));  // row_mirror
  v = max(v, dpp<0x142, 0xA, 0u>(v));  // row_bcast:15
  v = max(v, dpp<0x143, 0xC, 0u>(v));  // row_bcast:31
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ uint32_t wave_min(uint32_t v) {
  constexpr uint32_t kId = 0xFFFFFFFFu;
  v = min(v, dpp<0xB1, 0xF, kId>(v));
  v = min(v, dpp<0x4E, 0xF, kId>(v));
  v = min(v, dpp<0x141, 0xF, kId>(v));
  v = min(v, dpp<0x140, 0xF, kId>(v));
  v = min(v, dpp<0x142, 0xA, kId>(v));
  v = min(v, dpp<0x143, 0xC, kId>(v));
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ int wave_scan(int v) {
  v += (int)dpp<0x111, 0xF, 0u>((uint32_t)v);   // row_shr:1
  v += (int)dpp<0x112, 0xF, 0u>((uint32_t)v);
  v += (int)dpp<0x114, 0xF, 0u>((uint32_t)v);
  v += (int)dpp<0x118, 0xF, 0u>((uint32_t)v);
  v += (int)dpp<0x142, 0xA, 0u>((uint32_t)v);   // row_bcast:15
  v += (int)dpp<0x143, 0xC, 0u>((uint32_t)v);   // row_bcast:31
  return v;
}

// Wave-wide sum and maximum of a float, in the same steps.
template <int Ctrl, int RowMask>
__device__ __forceinline__ float dpp_or(float old, float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(v), Ctrl,
                                                    RowMask, 0xF, false));
}
template <typename Op>
__device__ __forceinline__ float wave_reduce(float v, float identity, Op op) {
  v = op(v, dpp_or<0xB1, 0xF>(identity, v));
  v = op(v, dpp_or<0x4E, 0xF>(identity, v));
  v = op(v, dpp_or<0x141, 0xF>(identity, v));
  v = op(v, dpp_or<0x140, 0xF>(identity, v));
  v = op(v, dpp_or<0x142, 0xA>(identity, v));
  v = op(v, dpp_or<0x143, 0xC>(identity, v));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_reduce(v, 0.0f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_fmax(float v) {
  return wave_reduce(v, -__builtin_inff(), [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace
}  // namespace xs
