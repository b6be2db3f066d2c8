// C ABI of the rotation and paged-cache operators (declared in include/pbb.h): argument
// validation and launch.  Every check runs on the host before anything is enqueued, so a failing
// call launches nothing and writes nothing.  No exception crosses the ABI.

#include "pbb.h"

#include <hip/hip_runtime.h>

#include "pbb_checks.h"

namespace {

using namespace pbb_checks;

static_assert(PBB_PAGED_COUNTER_BYTES == pbb::kPagedCounterBytes, "counter block");
static_assert((2 * pbb::kPagedMaxPieces + pbb::kPagedMaxPieces / 8 + pbb::kPagedMaxPieces) * 4 <=
                  (int)pbb::kPagedCounterBytes,
              "a counter per partial state (2 more per head, of at most kPagedMaxPieces / 2 heads)");

// The rules of a descriptor's attention kernels.
auto kind_of(const pbb_paged_desc_t* d) {
  return [d](bool narrow) { return pbb::paged_kind(d->dtype == PBB_DTYPE_F32, narrow, d->head_dim); };
}

}  // namespace

extern "C" {

pbb_status_t pbb_rope_init(pbb_rope_t* rope, int32_t head_dim, double base, int32_t n_axes,
                           const uint8_t* axis) {
  if (rope == nullptr) return PBB_ERR_NULL;
  if (head_dim != 64 && head_dim != 128) return PBB_ERR_SHAPE;
  if (!(base > 1.0) || !std::isfinite(base)) return PBB_ERR_SHAPE;
  if (n_axes < 1 || n_axes > PBB_MAX_AXES) return PBB_ERR_SHAPE;
  if (axis != nullptr)
    for (int c = 0; c < head_dim / 2; ++c)
      if (axis[c] >= n_axes) return PBB_ERR_SHAPE;
  const double two_pi = 6.283185307179586476925286766559;
  rope->head_dim = head_dim;
  rope->n_axes = n_axes;
  for (int c = 0; c < 64; ++c) {
    const bool used = c < head_dim / 2;
    rope->turns[c] = used ? std::pow(base, -2.0 * (double)c / (double)head_dim) / two_pi : 0.0;
    rope->axis[c] = used && axis != nullptr ? axis[c] : 0;
  }
  return PBB_OK;
}

pbb_status_t pbb_rotate(const pbb_rope_t* rope, int32_t n_tokens, int32_t n_heads,
                        const int32_t* positions, const void* x, int64_t x_stride, void* out,
                        int64_t out_stride, int32_t inverse, int32_t dtype, void* stream) {
  if (rope == nullptr) return PBB_ERR_NULL;
  if (!known_dtype(dtype)) return PBB_ERR_DTYPE;
  if (rope->head_dim != 64 && rope->head_dim != 128) return PBB_ERR_SHAPE;
  const pbb_status_t st = check_rope(rope, rope->head_dim);
  if (st != PBB_OK) return st;
  if (n_tokens < 0 || n_tokens > kMaxTokens || n_heads < 1 ||
      (int64_t)n_heads * rope->head_dim > (1 << 24))
    return PBB_ERR_SHAPE;
  const int64_t u = elem_bytes(dtype);
  if (!stride_ok(x_stride, n_heads, rope->head_dim, u) ||
      !stride_ok(out_stride, n_heads, rope->head_dim, u))
    return PBB_ERR_SHAPE;
  if (n_tokens == 0) return PBB_OK;   // (tensors of no tokens may have no address)
  if (out == x && out_stride != x_stride) return PBB_ERR_SHAPE;
  if (!positions || !x || !out) return PBB_ERR_NULL;
  if (!aligned(positions, 4) || !aligned(x, 16) || !aligned(out, 16)) return PBB_ERR_ALIGN;
  pbb::RotateArgs a;
  a.x = x;
  a.out = out;
  a.positions = positions;
  a.x_stride = x_stride * u;
  a.out_stride = out_stride * u;
  a.n = n_tokens;
  a.heads = n_heads;
  a.rope = rope_args(rope, inverse != 0 ? -1.0 : 1.0);
  const hipError_t e = pbb::launch_rotate(a, rope->head_dim, dtype == PBB_DTYPE_F32,
                                          reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? PBB_OK : PBB_ERR_LAUNCH;
}

pbb_status_t pbb_paged_append(const pbb_paged_desc_t* desc, int32_t n_tokens, const int32_t* pos,
                              const int32_t* q_start, const int32_t* table,
                              const pbb_rope_t* rope, const int32_t* rope_pos, const void* q,
                              int64_t q_stride, void* q_out, const void* k, int64_t k_stride,
                              const void* v, int64_t v_stride, void* k_pages, void* v_pages,
                              void* stream) {
  const pbb_status_t st = check_paged(desc, n_tokens);
  if (st != PBB_OK) return st;
  if (q_start == nullptr && n_tokens % desc->batch != 0) return PBB_ERR_SHAPE;
  if (rope != nullptr) {
    const pbb_status_t rs = check_rope(rope, desc->head_dim);
    if (rs != PBB_OK) return rs;
    if (rope_pos == nullptr && rope->n_axes != 1) return PBB_ERR_SHAPE;
  }
  const int64_t u = elem_bytes(desc->dtype);
  if (!stride_ok(k_stride, desc->n_kv_heads, desc->head_dim, u) ||
      !stride_ok(v_stride, desc->n_kv_heads, desc->head_dim, u) ||
      (q != nullptr && !stride_ok(q_stride, desc->n_q_heads, desc->head_dim, u)))
    return PBB_ERR_SHAPE;
  if (n_tokens == 0) return PBB_OK;
  if (q != nullptr && q_out == q && q_stride != (int64_t)desc->n_q_heads * desc->head_dim)
    return PBB_ERR_SHAPE;
  if (!pos || !table || !k || !v || !k_pages || !v_pages) return PBB_ERR_NULL;
  if ((q == nullptr) != (q_out == nullptr)) return PBB_ERR_NULL;
  if (!aligned(pos, 4) || !aligned(q_start, 4) || !aligned(table, 4) || !aligned(rope_pos, 4) ||
      !aligned(q, 16) || !aligned(q_out, 16) || !aligned(k, 16) || !aligned(v, 16) ||
      !aligned(k_pages, 16) || !aligned(v_pages, 16))
    return PBB_ERR_ALIGN;
  pbb::AppendArgs a;
  a.pos = pos;
  a.q_start = q_start;
  a.table = table;
  a.rope_pos = rope != nullptr ? rope_pos : nullptr;
  a.q = q;
  a.q_out = q_out;
  a.k = k;
  a.v = v;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.q_stride = q_stride * u;
  a.k_stride = k_stride * u;
  a.v_stride = v_stride * u;
  a.n = n_tokens;
  a.batch = desc->batch;
  a.uniform = q_start != nullptr ? -1 : n_tokens / desc->batch;
  a.by_uniform = pbb::FastDiv::make(a.uniform > 0 ? (uint32_t)a.uniform : 1u);
  a.hq = desc->n_q_heads;
  a.hkv = desc->n_kv_heads;
  a.turn = rope != nullptr ? 1 : 0;
  a.shape = shape_of(desc);
  a.rope = rope_args(rope, 1.0);
  const hipError_t e = pbb::launch_paged_append(a, desc->head_dim, desc->dtype == PBB_DTYPE_F32,
                                                reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? PBB_OK : PBB_ERR_LAUNCH;
}

pbb_status_t pbb_paged_workspace_bytes(const pbb_paged_desc_t* desc, int32_t n_tokens,
                                       size_t* bytes) {
  if (desc == nullptr || bytes == nullptr) return PBB_ERR_NULL;
  const pbb_status_t st = check_paged(desc, n_tokens);
  if (st != PBB_OK) return st;
  *bytes = workspace_of(desc, shape_of(desc), kind_of(desc)).bytes;
  return PBB_OK;
}

pbb_status_t pbb_paged_attention(const pbb_paged_desc_t* desc, int32_t n_tokens,
                                 const int32_t* pos, const int32_t* q_start, const int32_t* table,
                                 const void* q, int64_t q_stride, const void* k_pages,
                                 const void* v_pages, void* out, float* lse, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  const pbb_status_t st = check_paged(desc, n_tokens);
  if (st != PBB_OK) return st;
  if (q_start == nullptr && n_tokens % desc->batch != 0) return PBB_ERR_SHAPE;
  const int64_t u = elem_bytes(desc->dtype);
  if (!stride_ok(q_stride, desc->n_q_heads, desc->head_dim, u)) return PBB_ERR_SHAPE;
  if (n_tokens == 0) return PBB_OK;
  pbb::PagedArgs a;
  a.shape = shape_of(desc);
  a.plan = plan_of(desc, a.shape, n_tokens, q_start != nullptr, kind_of(desc));
  if ((uint64_t)a.plan.tiles * (uint64_t)desc->n_kv_heads > kMaxTiles) return PBB_ERR_SHAPE;
  if (!pos || !table || !q || !k_pages || !v_pages || !out) return PBB_ERR_NULL;
  if (!aligned(pos, 4) || !aligned(q_start, 4) || !aligned(table, 4) || !aligned(q, 16) ||
      !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(out, 16) || !aligned(lse, 4))
    return PBB_ERR_ALIGN;
  const Workspace ws = workspace_of(desc, a.shape, kind_of(desc));
  const size_t need = workspace_need(desc, a.plan, ws);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return PBB_ERR_WORKSPACE;
  if (need > 0 && !aligned(workspace, 16)) return PBB_ERR_ALIGN;
  take_workspace(a, need, ws, workspace);
  a.pos = pos;
  a.q_start = q_start;
  a.table = table;
  a.q = q;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.out = out;
  a.lse = lse;
  a.q_stride = q_stride * u;
  a.n = n_tokens;
  a.batch = desc->batch;
  a.hq = desc->n_q_heads;
  a.hkv = desc->n_kv_heads;
  a.group = desc->n_q_heads / desc->n_kv_heads;
  a.scale_log2 = scale_log2(desc);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  hipError_t e = a.plan.planned ? pbb::launch_paged_plan(a, s) : hipSuccess;
  if (e == hipSuccess)
    e = desc->dtype == PBB_DTYPE_F32 ? pbb::launch_paged_f32(a, desc->head_dim, s)
                                     : pbb::launch_paged_bf16(a, desc->head_dim, s);
  return e == hipSuccess ? PBB_OK : PBB_ERR_LAUNCH;
}

}  // extern "C"
