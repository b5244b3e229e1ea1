// Host side of the C ABI's expert order, moves, products of groups of rows and adapters
// (include/xshare.h): argument checks (before any HIP call), workspace carving and launches.  No
// allocation, no synchronisation.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "groups.h"
#include "xshare.h"

namespace {

using xs::kMaxGroupSize;

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

template <typename P>
P* at(void* ws, size_t off) {
  return reinterpret_cast<P*>(static_cast<char*>(ws) + off);
}

xshare_status status_of(hipError_t e) {
  return e == hipSuccess ? XSHARE_OK
         : e == hipErrorInvalidConfiguration ? XSHARE_EUNSUPPORTED : XSHARE_EHIP;
}

xshare_status check_pairs(int32_t T, int32_t k) {
  if (T < 0 || k < 1) return XSHARE_EINVAL;
  return T > kMaxGroupSize || k > xs::kMaxTopK || int64_t(T) * k > kMaxGroupSize
             ? XSHARE_EUNSUPPORTED : XSHARE_OK;
}

xshare_status check_order(int32_t T, int32_t k, int32_t E) {
  const xshare_status st = check_pairs(T, k);
  if (st == XSHARE_EINVAL || E < 1) return XSHARE_EINVAL;
  return st != XSHARE_OK || E > xs::kMaxExperts ? XSHARE_EUNSUPPORTED : XSHARE_OK;
}

xshare_status check_move(int32_t dtype, int32_t T, int32_t k, int32_t d) {
  if (dtype != XSHARE_F32 && dtype != XSHARE_BF16) return XSHARE_EINVAL;
  const xshare_status st = check_pairs(T, k);
  if (st == XSHARE_EINVAL || d < 1) return XSHARE_EINVAL;
  return st != XSHARE_OK || d > kMaxGroupSize ? XSHARE_EUNSUPPORTED : XSHARE_OK;
}

// A matrix of `cols` elements of `dtype` a row, at any of their alignments.
bool valid_rows(const void* p, int32_t dtype, int64_t ld, int32_t cols) {
  return p && aligned(p, dtype == XSHARE_F32 ? 4 : 2) && ld >= cols;
}

// A bf16 matrix read or written 16 bytes at a time.
bool valid_matrix(const void* p, int64_t ld, int32_t cols) {
  return p && aligned(p, 16) && ld >= cols && ld % 8 == 0;
}

// A matrix of rows, as a call is given it.
struct Rows {
  const void* p;
  int64_t ld;
  int64_t rows;
  int32_t cols;
};
// Whether two matrices of elements of `size` bytes share memory.  Columns of one buffer that lie side
// by side do not.  (Rows that lie differently far apart are taken to meet where the matrices' memory
// does; a single row has no distance of its own.)
bool overlap(const Rows& a, const Rows& b, uint64_t size) {
  if (!a.p || !b.p || a.rows == 0 || b.rows == 0) return false;
  const uint64_t p = reinterpret_cast<uintptr_t>(a.p), q = reinterpret_cast<uintptr_t>(b.p);
  const uint64_t bytes_p = (uint64_t(a.rows - 1) * uint64_t(a.ld) + a.cols) * size;
  const uint64_t bytes_q = (uint64_t(b.rows - 1) * uint64_t(b.ld) + b.cols) * size;
  if (p + bytes_p <= q || q + bytes_q <= p) return false;
  if (a.rows == 1 && b.rows == 1) return true;
  if (a.rows > 1 && b.rows > 1 && a.ld != b.ld) return true;
  const uint64_t row = uint64_t(a.rows > 1 ? a.ld : b.ld) * size;
  // b's first column from a's on, within a row
  const uint64_t apart = p <= q ? (q - p) % row : (row - (p - q) % row) % row;
  return apart < a.cols * size || apart + b.cols * size > row;
}
bool same(const Rows& a, const Rows& b) { return a.p == b.p && (a.ld == b.ld || a.rows == 1); }
uint64_t bytes_of(int32_t dtype) { return dtype == XSHARE_F32 ? 4 : 2; }

xs::MoveArgs move_args(int32_t dtype, int32_t T, int32_t k, int32_t d, const int32_t* rows) {
  xs::MoveArgs a{};
  a.fp32 = dtype == XSHARE_F32;
  a.T = T;
  a.k = k;
  a.d = d;
  a.rows = rows;
  return a;
}

xshare_status check_grouped(int32_t P, int32_t E, int32_t n, int32_t k) {
  if (P < 0 || E < 1 || n < 1 || k < 1 || n % 8 != 0 || k % 8 != 0) return XSHARE_EINVAL;
  return P > kMaxGroupSize || E > xs::kMaxExperts || n > kMaxGroupSize || k > kMaxGroupSize
             ? XSHARE_EUNSUPPORTED : XSHARE_OK;
}

// Rows further apart than this would not fit the kernels' 32-bit offsets within a tile.
constexpr int64_t kMaxRowStride = 1 << 22;

xshare_status check_sums(int32_t P, const void* ws, size_t ws_bytes) {
  const size_t need = xs::grouped_bytes(P);
  if (need > 0 && (!ws || ws_bytes < need)) return XSHARE_EWORKSPACE;
  return need > 0 && !aligned(ws, 16) ? XSHARE_EINVAL : XSHARE_OK;
}

xs::GroupedArgs grouped_args(int32_t P, int32_t E, int32_t n, int32_t k, const int32_t* offsets,
                             void* ws) {
  xs::GroupedArgs a{};
  a.sums = xs::grouped_bytes(P) > 0 ? at<float>(ws, 0) : nullptr;
  a.P = P;
  a.E = E;
  a.n = n;
  a.k = k;
  a.offsets = offsets;
  return a;
}

xshare_status check_adapters(int32_t T, int32_t L, int32_t r, int32_t n, int32_t d) {
  if (T < 0 || L < 1 || r < 1 || n < 1 || d < 1 || r % 8 != 0 || n % 8 != 0 || d % 8 != 0)
    return XSHARE_EINVAL;
  return T > kMaxGroupSize || L > xs::kMaxExperts || r > xs::kMaxRank || n > kMaxGroupSize ||
                 d > kMaxGroupSize
             ? XSHARE_EUNSUPPORTED : XSHARE_OK;
}

xshare_status run_adapters(const xshare_adapters_args* p, bool backward) {
  if (!p || p->struct_size != sizeof(xshare_adapters_args)) return XSHARE_EINVAL;
  const xshare_status st = check_adapters(p->T, p->n_adapters, p->rank, p->n, p->d);
  if (st != XSHARE_OK || (p->T == 0 && !backward)) return st;
  const int32_t cols = backward ? p->d : p->n;
  if (!p->a || !p->b || !aligned(p->a, 16) || !aligned(p->b, 16) || !aligned(p->scales, 4))
    return XSHARE_EINVAL;
  if (p->T > 0) {
    if (!valid_matrix(p->x, p->ldx, p->d) || !p->ids || !aligned(p->ids, 4) ||
        !valid_matrix(p->out, p->ld_out, cols))
      return XSHARE_EINVAL;
    if (p->base && !valid_matrix(p->base, p->ld_base, cols)) return XSHARE_EINVAL;
    if (backward && !valid_matrix(p->dy, p->lddy, p->n)) return XSHARE_EINVAL;
  }
  if (backward && (!p->da || !p->db || !aligned(p->da, 16) || !aligned(p->db, 16)))
    return XSHARE_EINVAL;
  const xs::AdaptersLayout A =
      xs::adapters_layout(p->T, p->n_adapters, p->rank, p->n, p->d, backward);
  if (!p->ws || p->ws_bytes < A.total) return XSHARE_EWORKSPACE;
  if (!aligned(p->ws, 16)) return XSHARE_EINVAL;
  // (some workgroups write out while others read x; the factors' gradients read x and dy after it)
  const Rows out{p->out, p->ld_out, p->T, cols}, base{p->base, p->ld_base, p->T, cols};
  if (overlap(out, {p->x, p->ldx, p->T, p->d}, 2) || (!same(out, base) && overlap(out, base, 2)) ||
      (backward && overlap(out, {p->dy, p->lddy, p->T, p->n}, 2)))
    return XSHARE_EINVAL;
  xs::AdaptersArgs a{};
  a.T = p->T;
  a.L = p->n_adapters;
  a.r = p->rank;
  a.n = p->n;
  a.d = p->d;
  a.x = p->x;
  a.ldx = p->ldx;
  a.a = p->a;
  a.b = p->b;
  a.ids = p->ids;
  a.scales = p->scales;
  a.base = p->base;
  a.ld_base = p->ld_base;
  a.out = p->out;
  a.ld_out = p->ld_out;
  a.dy = p->dy;
  a.lddy = p->lddy;
  a.da = p->da;
  a.db = p->db;
  a.offsets = at<int32_t>(p->ws, A.offsets);
  a.rows = at<int32_t>(p->ws, A.rows);
  a.tokens = at<int32_t>(p->ws, A.tokens);
  a.counts = at<int32_t>(p->ws, A.counts);
  a.h = at<uint16_t>(p->ws, A.h);
  a.dh = at<uint16_t>(p->ws, A.dh);
  a.at = at<uint16_t>(p->ws, A.at);
  a.bt = at<uint16_t>(p->ws, A.bt);
  a.part = at<float>(p->ws, A.part);
  a.splits = xs::adapter_splits(p->T, p->n_adapters, p->n, p->d);
  return status_of(backward ? xs::launch_adapters_backward(a, p->stream)
                            : xs::launch_adapters(a, p->stream));
}

}  // namespace

extern "C" {

size_t xshare_expert_order_workspace_bytes(int32_t T, int32_t top_k, int32_t n_experts) {
  if (check_order(T, top_k, n_experts) != XSHARE_OK) return 0;
  return xs::order_bytes(T * top_k, n_experts);
}

xshare_status xshare_expert_order(const int32_t* ids, int32_t T, int32_t top_k, int32_t n_experts,
                                  int32_t* offsets, int32_t* rows, int32_t* pairs, void* ws,
                                  size_t ws_bytes, hipStream_t stream) {
  const xshare_status st = check_order(T, top_k, n_experts);
  if (st != XSHARE_OK) return st;
  if (!offsets || !aligned(offsets, 4)) return XSHARE_EINVAL;
  if (T > 0 && (!ids || !rows || !pairs || !aligned(ids, 4) || !aligned(rows, 4) ||
                !aligned(pairs, 4)))
    return XSHARE_EINVAL;
  const size_t need = xs::order_bytes(T * top_k, n_experts);
  if (need > 0 && (!ws || ws_bytes < need)) return XSHARE_EWORKSPACE;
  if (need > 0 && !aligned(ws, 16)) return XSHARE_EINVAL;
  const xs::OrderArgs a{ids, T * top_k, n_experts, offsets, rows, pairs,
                        static_cast<int32_t*>(ws)};
  return status_of(xs::launch_order(a, stream));
}

xshare_status xshare_dispatch(const void* x, int64_t ldx, int32_t dtype, int32_t T, int32_t top_k,
                              int32_t d, const int32_t* rows, void* out, int64_t ld_out,
                              hipStream_t stream) {
  const xshare_status st = check_move(dtype, T, top_k, d);
  if (st != XSHARE_OK || T == 0) return st;
  if (!valid_rows(x, dtype, ldx, d) || !valid_rows(out, dtype, ld_out, d) || !rows ||
      !aligned(rows, 4))
    return XSHARE_EINVAL;
  if (overlap({x, ldx, T, d}, {out, ld_out, int64_t(T) * top_k, d}, bytes_of(dtype)))
    return XSHARE_EINVAL;
  xs::MoveArgs a = move_args(dtype, T, top_k, d, rows);
  a.token = x;
  a.ld_token = ldx;
  a.out_row = out;
  a.ld_out_row = ld_out;
  return status_of(xs::launch_dispatch(a, stream));
}

xshare_status xshare_combine(const void* src, int64_t ld_src, int32_t dtype, int32_t T,
                             int32_t top_k, int32_t d, const int32_t* rows, const float* w, void* y,
                             int64_t ldy, hipStream_t stream) {
  const xshare_status st = check_move(dtype, T, top_k, d);
  if (st != XSHARE_OK || T == 0) return st;
  if (!valid_rows(src, dtype, ld_src, d) || !valid_rows(y, dtype, ldy, d) || !rows ||
      !aligned(rows, 4) || !aligned(w, 4))
    return XSHARE_EINVAL;
  if (overlap({src, ld_src, int64_t(T) * top_k, d}, {y, ldy, T, d}, bytes_of(dtype)))
    return XSHARE_EINVAL;
  xs::MoveArgs a = move_args(dtype, T, top_k, d, rows);
  a.row = src;
  a.ld_row = ld_src;
  a.w = w;
  a.out_token = y;
  a.ld_out_token = ldy;
  return status_of(xs::launch_combine(a, stream));
}

xshare_status xshare_combine_backward(const void* dy, int64_t lddy, const void* src, int64_t ld_src,
                                      int32_t dtype, int32_t T, int32_t top_k, int32_t d,
                                      const int32_t* rows, const float* w, void* dsrc,
                                      int64_t ld_dsrc, float* dw, hipStream_t stream) {
  const xshare_status st = check_move(dtype, T, top_k, d);
  if (st != XSHARE_OK || T == 0) return st;
  if (!valid_rows(dy, dtype, lddy, d) || !valid_rows(src, dtype, ld_src, d) ||
      !valid_rows(dsrc, dtype, ld_dsrc, d) || !rows || !aligned(rows, 4) || !w || !aligned(w, 4) ||
      !dw || !aligned(dw, 4))
    return XSHARE_EINVAL;
  const Rows out{dsrc, ld_dsrc, int64_t(T) * top_k, d}, from{src, ld_src, out.rows, d};
  if (overlap({dy, lddy, T, d}, out, bytes_of(dtype)) ||
      (!same(from, out) && overlap(from, out, bytes_of(dtype))))
    return XSHARE_EINVAL;
  xs::MoveArgs a = move_args(dtype, T, top_k, d, rows);
  a.token = dy;
  a.ld_token = lddy;
  a.row = src;
  a.ld_row = ld_src;
  a.w = w;
  a.out_row = dsrc;
  a.ld_out_row = ld_dsrc;
  a.dw = dw;
  return status_of(xs::launch_combine_backward(a, stream));
}

xshare_status xshare_grouped_linear(const uint16_t* x, int64_t ldx, const uint16_t* w,
                                    const int32_t* offsets, int32_t P, int32_t n_groups, int32_t n,
                                    int32_t k, uint16_t* y, int64_t ldy, void* ws,
                                    size_t ws_bytes, hipStream_t stream) {
  const xshare_status st = check_grouped(P, n_groups, n, k);
  if (st != XSHARE_OK || P == 0) return st;
  if (!valid_matrix(x, ldx, k) || !w || !aligned(w, 16) || !offsets || !aligned(offsets, 4) ||
      !valid_matrix(y, ldy, n))
    return XSHARE_EINVAL;
  if (ldx > kMaxRowStride) return XSHARE_EUNSUPPORTED;
  if (const xshare_status bad = check_sums(P, ws, ws_bytes)) return bad;
  if (overlap({x, ldx, P, k}, {y, ldy, P, n}, 2)) return XSHARE_EINVAL;
  xs::GroupedArgs a = grouped_args(P, n_groups, n, k, offsets, ws);
  a.x = x;
  a.ldx = ldx;
  a.w = w;
  a.out = y;
  a.ldo = ldy;
  return status_of(xs::launch_grouped_linear(a, stream));
}

xshare_status xshare_grouped_linear_backward_x(const uint16_t* dy, int64_t lddy, const uint16_t* w,
                                               const int32_t* offsets, int32_t P, int32_t n_groups,
                                               int32_t n, int32_t k, uint16_t* dx, int64_t lddx,
                                               void* ws, size_t ws_bytes, hipStream_t stream) {
  const xshare_status st = check_grouped(P, n_groups, n, k);
  if (st != XSHARE_OK || P == 0) return st;
  if (!valid_matrix(dy, lddy, n) || !w || !aligned(w, 16) || !offsets || !aligned(offsets, 4) ||
      !valid_matrix(dx, lddx, k))
    return XSHARE_EINVAL;
  if (lddy > kMaxRowStride) return XSHARE_EUNSUPPORTED;
  if (const xshare_status bad = check_sums(P, ws, ws_bytes)) return bad;
  if (overlap({dy, lddy, P, n}, {dx, lddx, P, k}, 2)) return XSHARE_EINVAL;
  xs::GroupedArgs a = grouped_args(P, n_groups, n, k, offsets, ws);
  a.dy = dy;
  a.lddy = lddy;
  a.w = w;
  a.out = dx;
  a.ldo = lddx;
  return status_of(xs::launch_grouped_backward_x(a, stream));
}

xshare_status xshare_grouped_linear_backward_w(const uint16_t* dy, int64_t lddy, const uint16_t* x,
                                               int64_t ldx, const int32_t* offsets, int32_t P,
                                               int32_t n_groups, int32_t n, int32_t k, void* dw,
                                               int32_t dw_dtype, int32_t accumulate, void* ws,
                                               size_t ws_bytes, hipStream_t stream) {
  if (dw_dtype != XSHARE_F32 && dw_dtype != XSHARE_BF16) return XSHARE_EINVAL;
  const xshare_status st = check_grouped(P, n_groups, n, k);
  if (st != XSHARE_OK) return st;
  if (!offsets || !aligned(offsets, 4) || !dw || !aligned(dw, 16)) return XSHARE_EINVAL;
  if (P > 0 && (!valid_matrix(dy, lddy, n) || !valid_matrix(x, ldx, k))) return XSHARE_EINVAL;
  if ((accumulate && dw_dtype != XSHARE_F32) || lddy > kMaxRowStride || ldx > kMaxRowStride)
    return XSHARE_EUNSUPPORTED;
  if (const xshare_status bad = check_sums(P, ws, ws_bytes)) return bad;
  xs::GroupedArgs a = grouped_args(P, n_groups, n, k, offsets, ws);
  a.dy = dy;
  a.lddy = lddy;
  a.x = x;
  a.ldx = ldx;
  a.dw = dw;
  a.dw_fp32 = dw_dtype == XSHARE_F32;
  a.accumulate = accumulate != 0;
  return status_of(xs::launch_grouped_backward_w(a, stream));
}

size_t xshare_grouped_linear_workspace_bytes(int32_t P, int32_t n_groups, int32_t n, int32_t k) {
  return check_grouped(P, n_groups, n, k) == XSHARE_OK ? xs::grouped_bytes(P) : 0;
}

size_t xshare_adapters_workspace_bytes(int32_t T, int32_t n_adapters, int32_t rank, int32_t n,
                                       int32_t d, int32_t backward) {
  if (check_adapters(T, n_adapters, rank, n, d) != XSHARE_OK) return 0;
  return xs::adapters_layout(T, n_adapters, rank, n, d, backward != 0).total;
}

xshare_status xshare_adapters(const xshare_adapters_args* args) { return run_adapters(args, false); }

xshare_status xshare_adapters_backward(const xshare_adapters_args* args) {
  return run_adapters(args, true);
}

}  // extern "C"
