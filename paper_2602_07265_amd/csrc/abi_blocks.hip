// Host side of the C ABI's routing by scores and FP8 block products (include/xshare.h):
// argument checks (before any HIP call), workspace carving and launches.  No allocation, no
// synchronisation.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "blocks.h"
#include "xshare.h"

namespace {

using xs::kMaxBlockSize;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

template <typename P>
P* at(void* ws, size_t off) {
  return reinterpret_cast<P*>(static_cast<char*>(ws) + off);
}

// The checks of both directions; `groups` those of the choice too.
xshare_status check_gate(int32_t dtype, int32_t T, int64_t ld, const xshare_gate_params* p,
                         bool groups) {
  if (!p) return XSHARE_EINVAL;
  const int N = p->n_experts, k = p->top_k, G = p->n_groups;
  if (T < 0 || N < 1 || k < 1 || k > N || ld < N) return XSHARE_EINVAL;
  if (dtype != XSHARE_F32 && dtype != XSHARE_BF16) return XSHARE_EINVAL;
  if (p->score != XSHARE_GATE_SOFTMAX && p->score != XSHARE_GATE_SIGMOID) return XSHARE_EINVAL;
  if (!std::isfinite(p->scale)) return XSHARE_EINVAL;
  if (groups) {
    if (G < 1 || N % G != 0 || p->top_groups < 1 || p->top_groups > G) return XSHARE_EINVAL;
    if (k > p->top_groups * (N / G)) return XSHARE_EINVAL;
    if (p->group_score != XSHARE_GROUP_MAX && p->group_score != XSHARE_GROUP_TOP2)
      return XSHARE_EINVAL;
    if (p->top_groups < G && p->group_score == XSHARE_GROUP_TOP2 && N / G < 2)
      return XSHARE_EINVAL;
  }
  if (N > xs::kMaxExperts || k > xs::kMaxTopK || T > kMaxBlockSize) return XSHARE_EUNSUPPORTED;
  if (groups && p->top_groups < G && G > xs::kMaxGateGroups) return XSHARE_EUNSUPPORTED;
  return XSHARE_OK;
}

xs::GateArgs gate_args(const void* logits, int32_t dtype, int32_t T, int64_t ld,
                       const xshare_gate_params* p) {
  xs::GateArgs a{};
  a.logits = logits;
  a.bf16 = dtype == XSHARE_BF16;
  a.T = T;
  a.N = p->n_experts;
  a.k = p->top_k;
  a.ld = ld;
  a.sigmoid = p->score == XSHARE_GATE_SIGMOID;
  a.renormalize = p->renormalize != 0;
  a.scale = p->scale;
  return a;
}

// Sizes of a [rows, cols] operand in 128-blocks along cols.
xshare_status check_size(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1 || cols % 16 != 0) return XSHARE_EINVAL;
  return rows > kMaxBlockSize || cols > kMaxBlockSize ? XSHARE_EUNSUPPORTED : XSHARE_OK;
}

bool valid_x(const void* x, int64_t ld, int64_t cols) {
  return x && aligned16(x) && ld >= cols && ld % 8 == 0;
}

xshare_status check_experts(int32_t T, int32_t k, int32_t E, int32_t d, int32_t f) {
  if (T < 0 || k < 1 || E < 1 || d < 1 || f < 1 || d % 16 != 0 || f % 16 != 0)
    return XSHARE_EINVAL;
  if (E > xs::kMaxExperts || k > xs::kMaxTopK || d > kMaxBlockSize || f > kMaxBlockSize ||
      T > kMaxBlockSize || int64_t(T) * k > kMaxBlockSize)
    return XSHARE_EUNSUPPORTED;
  return XSHARE_OK;
}

xshare_status status_of(hipError_t e) { return e == hipSuccess ? XSHARE_OK : XSHARE_EHIP; }

}  // namespace

extern "C" {

xshare_status xshare_gate(const void* logits, int32_t dtype, int32_t T, int64_t ld,
                          const float* bias, const xshare_gate_params* params, int32_t* ids,
                          float* w, hipStream_t stream) {
  const xshare_status st = check_gate(dtype, T, ld, params, true);
  if (st != XSHARE_OK || T == 0) return st;
  if (!logits || !ids || !w) return XSHARE_EINVAL;
  xs::GateArgs a = gate_args(logits, dtype, T, ld, params);
  a.bias = bias;
  a.G = params->n_groups;
  a.top_groups = params->top_groups;
  a.top2 = params->group_score == XSHARE_GROUP_TOP2;
  a.ids = ids;
  a.w = w;
  return status_of(xs::launch_gate(a, stream));
}

xshare_status xshare_gate_backward(const void* logits, int32_t dtype, int32_t T, int64_t ld,
                                   const xshare_gate_params* params, const int32_t* ids,
                                   const float* dw, float* dlogits, hipStream_t stream) {
  const xshare_status st = check_gate(dtype, T, ld, params, false);
  if (st != XSHARE_OK || T == 0) return st;
  if (!logits || !ids || !dw || !dlogits) return XSHARE_EINVAL;
  xs::GateArgs a = gate_args(logits, dtype, T, ld, params);
  a.ids = const_cast<int32_t*>(ids);
  a.dw = dw;
  a.dlogits = dlogits;
  return status_of(xs::launch_gate_backward(a, stream));
}

xshare_status xshare_block_quantize(const uint16_t* x, int32_t rows, int32_t cols, int64_t ld,
                                    int32_t block_rows, uint8_t* q, float* scales,
                                    hipStream_t stream) {
  if (block_rows != 1 && block_rows != xs::kQuantBlock) return XSHARE_EINVAL;
  const xshare_status st = check_size(rows, cols);
  if (st != XSHARE_OK || rows == 0) return st;
  if (!valid_x(x, ld, cols) || !q || !aligned16(q) || !scales || !aligned4(scales))
    return XSHARE_EINVAL;
  return status_of(
      xs::launch_block_quantize(x, rows, cols, ld, block_rows, q, scales, stream));
}

size_t xshare_block_linear_workspace_bytes(int32_t T, int32_t n, int32_t k) {
  if (check_size(T, k) != XSHARE_OK || n < 1 || n > kMaxBlockSize) return 0;
  return xs::block_linear_layout(T, k).total;
}

xshare_status xshare_block_linear(const uint16_t* x, int64_t ldx, const uint8_t* xq,
                                  const float* xs, int32_t T, int32_t n, int32_t k,
                                  const uint8_t* wq, const float* wscale, uint16_t* y,
                                  int64_t ldy, void* ws, size_t ws_bytes, hipStream_t stream) {
  const xshare_status st = check_size(T, k);
  if (st == XSHARE_EINVAL || n < 1 || ldy < n) return XSHARE_EINVAL;
  if (st != XSHARE_OK || n > kMaxBlockSize) return XSHARE_EUNSUPPORTED;
  if (T == 0) return XSHARE_OK;
  if (!wq || !aligned16(wq) || !wscale || !aligned4(wscale) || !y) return XSHARE_EINVAL;
  if (x ? (xq || xs || !valid_x(x, ldx, k)) : (!xq || !xs || !aligned16(xq) || !aligned4(xs)))
    return XSHARE_EINVAL;
  xs::BlockLinearArgs a{T, n, k, nullptr, 0, xq, xs, wq, wscale, y, ldy};
  if (x) {
    const xs::BlockLinearLayout L = xs::block_linear_layout(T, k);
    if (!ws || ws_bytes < L.total) return XSHARE_EWORKSPACE;
    if (!aligned16(ws)) return XSHARE_EINVAL;
    if (xs::block_linear_small(T, k)) {
      a.x = x;
      a.ldx = ldx;
    } else {
      uint8_t* const q = at<uint8_t>(ws, L.xq);
      float* const s = at<float>(ws, L.xs);
      if (xs::launch_block_quantize(x, T, k, ldx, 1, q, s, stream) != hipSuccess)
        return XSHARE_EHIP;
      a.xq = q;
      a.xs = s;
    }
  }
  return status_of(xs::launch_block_linear(a, stream));
}

size_t xshare_block_experts_workspace_bytes(int32_t T, int32_t top_k, int32_t n_experts,
                                            int32_t d, int32_t f) {
  if (check_experts(T, top_k, n_experts, d, f) != XSHARE_OK) return 0;
  return xs::block_experts_layout(T, top_k, n_experts, d, f).total;
}

xshare_status xshare_block_experts(const xshare_block_experts_args* p) {
  if (!p || p->struct_size != sizeof(xshare_block_experts_args)) return XSHARE_EINVAL;
  const xshare_status st = check_experts(p->T, p->top_k, p->n_experts, p->d, p->f);
  if (st != XSHARE_OK || p->T == 0) return st;
  if (!valid_x(p->x, p->ldx, p->d) || !p->ids || !p->w || !p->y || !aligned16(p->y) ||
      p->ldy < p->d || p->ldy % 8 != 0)
    return XSHARE_EINVAL;
  if (!p->w1 || !p->w3 || !p->w2 || !p->w1_scale || !p->w3_scale || !p->w2_scale ||
      !aligned16(p->w1) || !aligned16(p->w3) || !aligned16(p->w2) || !aligned4(p->w1_scale) ||
      !aligned4(p->w3_scale) || !aligned4(p->w2_scale))
    return XSHARE_EINVAL;
  const xs::BlockExpertsLayout L =
      xs::block_experts_layout(p->T, p->top_k, p->n_experts, p->d, p->f);
  if (!p->ws || p->ws_bytes < L.total) return XSHARE_EWORKSPACE;
  if (!aligned16(p->ws)) return XSHARE_EINVAL;
  xs::BlockExpertsArgs a{};
  a.T = p->T;
  a.k = p->top_k;
  a.E = p->n_experts;
  a.d = p->d;
  a.f = p->f;
  a.x = p->x;
  a.ldx = p->ldx;
  a.ids = p->ids;
  a.w = p->w;
  a.w1 = p->w1;
  a.w3 = p->w3;
  a.w2 = p->w2;
  a.s1 = p->w1_scale;
  a.s3 = p->w3_scale;
  a.s2 = p->w2_scale;
  a.y = p->y;
  a.ldy = p->ldy;
  a.xq = at<uint8_t>(p->ws, L.xq);
  a.xs = at<float>(p->ws, L.xs);
  a.counts = at<int32_t>(p->ws, L.counts);
  a.perm = at<int32_t>(p->ws, L.perm);
  a.up_tiles = at<int4>(p->ws, L.up_tiles);
  a.down_tiles = at<int4>(p->ws, L.down_tiles);
  a.h = at<float>(p->ws, L.h);
  a.hq = at<uint8_t>(p->ws, L.hq);
  a.hs = at<float>(p->ws, L.hs);
  a.o = at<float>(p->ws, L.o);
  return status_of(xs::launch_block_experts(a, p->stream));
}

}  // extern "C"
