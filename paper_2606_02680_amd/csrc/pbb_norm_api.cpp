// C ABI of the per-head norms with rotation (declared in include/pbb.h): argument validation and launch.
// Every check runs on the host before anything is enqueued, so a failing call launches nothing and
// writes nothing.  No exception crosses the ABI.

#include "pbb.h"

#include <hip/hip_runtime.h>

#include "pbb_checks.h"
#include "pbb_norm_internal.h"

namespace {

using namespace pbb_checks;

pbb_status_t check_norm(const pbb_norm_t* norm, const pbb_rope_t* rope, int32_t head_dim, int32_t n,
                        int32_t hq, int32_t hkv, int32_t dtype) {
  if (norm == nullptr) return PBB_ERR_NULL;
  if (!known_dtype(dtype)) return PBB_ERR_DTYPE;
  if (head_dim != 64 && head_dim != 128) return PBB_ERR_SHAPE;
  if (!eps_ok(norm->eps)) return PBB_ERR_SHAPE;
  if (rope != nullptr) {
    const pbb_status_t st = check_rope(rope, head_dim);
    if (st != PBB_OK) return st;
  }
  if (n < 0 || n > kMaxTokens || hq < 1 || hkv < 0 || (int64_t)hq * head_dim > (1 << 24) ||
      (int64_t)hkv * head_dim > (1 << 24))
    return PBB_ERR_SHAPE;
  return PBB_OK;
}

// Rows that a call reads and writes in place share their strides.
bool in_place_ok(const void* x, int64_t xs, const void* out, int64_t os) { return out != x || os == xs; }

// Two sums of head_dim floats, where both are wanted, are written by different workgroups.
bool sums_apart(const float* a, const float* b, int32_t head_dim) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a == nullptr || b == nullptr || (x < y ? y - x : x - y) >= (uintptr_t)head_dim * sizeof(float);
}

pbb::NormArgs norm_args(const pbb_norm_t* norm, const pbb_rope_t* rope, double sign, int32_t n, int32_t hq,
                        int32_t hkv, const int32_t* positions) {
  pbb::NormArgs a{};
  a.part[0].heads = hq;
  a.part[1].heads = hkv;
  a.part[0].weight = norm->q_weight;
  a.part[1].weight = norm->k_weight;
  a.positions = positions;
  a.n = n;
  a.turn = rope != nullptr ? 1 : 0;
  a.eps = norm->eps;
  a.rope = rope_args(rope, sign);
  return a;
}

size_t backward_bytes(int32_t head_dim, int32_t n, int32_t hq, int32_t hkv, int32_t dtype) {
  const int row_bytes = (int)(head_dim * elem_bytes(dtype)), rows = 64 / (row_bytes / 32), all = hq + hkv;
  const int blocks = pbb::norm_grad_blocks(n, hq, all, rows, row_bytes) +
                     pbb::norm_grad_blocks(n, hkv, all, rows, row_bytes);
  return (size_t)blocks * head_dim * sizeof(float);
}

}  // namespace

extern "C" {

pbb_status_t pbb_norm_rotate(const pbb_norm_t* norm, const pbb_rope_t* rope, int32_t head_dim,
                             int32_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads,
                             const int32_t* positions, const void* q, int64_t q_stride, void* q_out,
                             int64_t q_out_stride, const void* k, int64_t k_stride, void* k_out,
                             int64_t k_out_stride, int32_t dtype, void* stream) {
  const pbb_status_t st = check_norm(norm, rope, head_dim, n_tokens, n_q_heads, n_kv_heads, dtype);
  if (st != PBB_OK) return st;
  const int64_t u = elem_bytes(dtype);
  const bool keys = n_kv_heads > 0;
  if (!stride_ok(q_stride, n_q_heads, head_dim, u) || !stride_ok(q_out_stride, n_q_heads, head_dim, u) ||
      (keys && (!stride_ok(k_stride, n_kv_heads, head_dim, u) ||
                !stride_ok(k_out_stride, n_kv_heads, head_dim, u))))
    return PBB_ERR_SHAPE;
  if (n_tokens == 0) return PBB_OK;   // (tensors of no tokens may have no address)
  if (!in_place_ok(q, q_stride, q_out, q_out_stride) ||
      (keys && !in_place_ok(k, k_stride, k_out, k_out_stride)))
    return PBB_ERR_SHAPE;
  if (!q || !q_out || (keys && (!k || !k_out)) || (rope != nullptr && !positions)) return PBB_ERR_NULL;
  if (!aligned(positions, 4) || !aligned(q, 16) || !aligned(q_out, 16) || !aligned(norm->q_weight, 16) ||
      (keys && (!aligned(k, 16) || !aligned(k_out, 16) || !aligned(norm->k_weight, 16))))
    return PBB_ERR_ALIGN;
  pbb::NormArgs a = norm_args(norm, rope, 1.0, n_tokens, n_q_heads, n_kv_heads, positions);
  a.part[0].x = q, a.part[0].x_stride = q_stride * u;
  a.part[0].out = q_out, a.part[0].out_stride = q_out_stride * u;
  a.part[1].x = k, a.part[1].x_stride = k_stride * u;
  a.part[1].out = k_out, a.part[1].out_stride = k_out_stride * u;
  const hipError_t e = pbb::launch_norm_rotate(a, head_dim, dtype == PBB_DTYPE_F32,
                                               reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? PBB_OK : PBB_ERR_LAUNCH;
}

pbb_status_t pbb_norm_workspace_bytes(int32_t head_dim, int32_t n_tokens, int32_t n_q_heads,
                                      int32_t n_kv_heads, int32_t dtype, size_t* bytes) {
  if (bytes == nullptr) return PBB_ERR_NULL;
  const pbb_norm_t norm = {1.0f, nullptr, nullptr};
  const pbb_status_t st = check_norm(&norm, nullptr, head_dim, n_tokens, n_q_heads, n_kv_heads, dtype);
  if (st != PBB_OK) return st;
  *bytes = backward_bytes(head_dim, n_tokens, n_q_heads, n_kv_heads, dtype);
  return PBB_OK;
}

pbb_status_t pbb_norm_rotate_backward(const pbb_norm_t* norm, const pbb_rope_t* rope, int32_t head_dim,
                                      int32_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads,
                                      const int32_t* positions, const void* q, int64_t q_stride,
                                      const void* q_grad, int64_t q_grad_stride, void* dq,
                                      int64_t dq_stride, const void* k, int64_t k_stride,
                                      const void* k_grad, int64_t k_grad_stride, void* dk,
                                      int64_t dk_stride, float* dq_weight, float* dk_weight,
                                      int32_t dtype, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  const pbb_status_t st = check_norm(norm, rope, head_dim, n_tokens, n_q_heads, n_kv_heads, dtype);
  if (st != PBB_OK) return st;
  const int64_t u = elem_bytes(dtype);
  const bool keys = n_kv_heads > 0;
  for (int64_t s : {q_stride, q_grad_stride, dq_stride})
    if (!stride_ok(s, n_q_heads, head_dim, u)) return PBB_ERR_SHAPE;
  if (keys)
    for (int64_t s : {k_stride, k_grad_stride, dk_stride})
      if (!stride_ok(s, n_kv_heads, head_dim, u)) return PBB_ERR_SHAPE;
  // (no tokens, or no heads of a kind: the weight's gradient is zero, and has to be written)
  const bool sums = dq_weight != nullptr || dk_weight != nullptr;
  if (n_tokens == 0 && !sums) return PBB_OK;
  if (!sums_apart(dq_weight, dk_weight, head_dim)) return PBB_ERR_SHAPE;
  if (!aligned(dq_weight, 4) || !aligned(dk_weight, 4)) return PBB_ERR_ALIGN;
  if (n_tokens > 0) {
    if (!in_place_ok(q, q_stride, dq, dq_stride) || !in_place_ok(q_grad, q_grad_stride, dq, dq_stride) ||
        (keys && (!in_place_ok(k, k_stride, dk, dk_stride) ||
                  !in_place_ok(k_grad, k_grad_stride, dk, dk_stride))))
      return PBB_ERR_SHAPE;
    if (!q || !q_grad || !dq || (keys && (!k || !k_grad || !dk)) || (rope != nullptr && !positions))
      return PBB_ERR_NULL;
    if (!aligned(positions, 4) || !aligned(q, 16) || !aligned(q_grad, 16) || !aligned(dq, 16) ||
        !aligned(norm->q_weight, 16) ||
        (keys && (!aligned(k, 16) || !aligned(k_grad, 16) || !aligned(dk, 16) ||
                  !aligned(norm->k_weight, 16))))
      return PBB_ERR_ALIGN;
    if (dq_weight != nullptr || (keys && dk_weight != nullptr)) {
      const size_t need = backward_bytes(head_dim, n_tokens, n_q_heads, n_kv_heads, dtype);
      if (workspace == nullptr || workspace_bytes < need) return PBB_ERR_WORKSPACE;
      if (!aligned(workspace, 16)) return PBB_ERR_ALIGN;
    }
  }
  pbb::NormArgs a = norm_args(norm, rope, -1.0, n_tokens, n_q_heads, n_kv_heads, positions);
  a.part[0].x = q, a.part[0].x_stride = q_stride * u;
  a.part[0].grad = q_grad, a.part[0].grad_stride = q_grad_stride * u;
  a.part[0].out = dq, a.part[0].out_stride = dq_stride * u;
  a.part[0].dweight = dq_weight;
  a.part[1].x = k, a.part[1].x_stride = k_stride * u;
  a.part[1].grad = k_grad, a.part[1].grad_stride = k_grad_stride * u;
  a.part[1].out = dk, a.part[1].out_stride = dk_stride * u;
  a.part[1].dweight = dk_weight;
  a.partials = static_cast<float*>(workspace);
  const hipError_t e = pbb::launch_norm_rotate_backward(a, head_dim, dtype == PBB_DTYPE_F32,
                                                        reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? PBB_OK : PBB_ERR_LAUNCH;
}

}  // extern "C"
