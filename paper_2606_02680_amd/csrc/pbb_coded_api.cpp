// C ABI of the 8-bit paged cache (declared in include/pbb.h): argument validation and launch.  Every check
// runs on the host before anything is enqueued, so a failing call launches nothing and writes nothing.
// No exception crosses the ABI.

#include "pbb.h"

#include <hip/hip_runtime.h>

#include "pbb_checks.h"
#include "pbb_norm_internal.h"

namespace {

using namespace pbb_checks;

pbb_status_t check_coded(const pbb_paged_desc_t* d, int32_t n) {
  const pbb_status_t st = check_paged(d, n);
  return st != PBB_OK ? st : d->dtype == PBB_DTYPE_BF16 ? PBB_OK : PBB_ERR_DTYPE;
}

auto kind_of(const pbb_paged_desc_t* d) {
  return [d](bool narrow) { return pbb::coded_kind(narrow, d->head_dim, (int64_t)d->batch * d->n_kv_heads); };
}

bool cache_given(const void* kp, const void* vp, const void* ks, const void* vs) { return kp && vp && ks && vs; }
bool cache_aligned(const void* kp, const void* vp, const void* ks, const void* vs) {
  return aligned(kp, 16) && aligned(vp, 16) && aligned(ks, 16) && aligned(vs, 16);
}

}  // namespace

extern "C" {

pbb_status_t pbb_coded_append(const pbb_paged_desc_t* desc, int32_t n_tokens, const int32_t* pos,
                              const int32_t* q_start, const int32_t* table, const pbb_norm_t* norm,
                              const pbb_rope_t* rope, const int32_t* rope_pos, const void* q,
                              int64_t q_stride, void* q_out, const void* k, int64_t k_stride,
                              const void* v, int64_t v_stride, void* k_pages, void* v_pages,
                              uint8_t* k_scales, uint8_t* v_scales, void* stream) {
  const pbb_status_t st = check_coded(desc, n_tokens);
  if (st != PBB_OK) return st;
  if (q_start == nullptr && n_tokens % desc->batch != 0) return PBB_ERR_SHAPE;
  if (norm != nullptr && !eps_ok(norm->eps)) return PBB_ERR_SHAPE;
  if (rope != nullptr) {
    const pbb_status_t rs = check_rope(rope, desc->head_dim);
    if (rs != PBB_OK) return rs;
    if (rope_pos == nullptr && rope->n_axes != 1) return PBB_ERR_SHAPE;
  }
  if (!stride_ok(k_stride, desc->n_kv_heads, desc->head_dim, 2) ||
      !stride_ok(v_stride, desc->n_kv_heads, desc->head_dim, 2) ||
      (q != nullptr && !stride_ok(q_stride, desc->n_q_heads, desc->head_dim, 2)))
    return PBB_ERR_SHAPE;
  if (n_tokens == 0) return PBB_OK;
  if (q != nullptr && q_out == q && q_stride != (int64_t)desc->n_q_heads * desc->head_dim)
    return PBB_ERR_SHAPE;
  if (!pos || !table || !k || !v || !cache_given(k_pages, v_pages, k_scales, v_scales)) return PBB_ERR_NULL;
  if ((q == nullptr) != (q_out == nullptr)) return PBB_ERR_NULL;
  if (!aligned(pos, 4) || !aligned(q_start, 4) || !aligned(table, 4) || !aligned(rope_pos, 4) ||
      !aligned(q, 16) || !aligned(q_out, 16) || !aligned(k, 16) || !aligned(v, 16) ||
      !cache_aligned(k_pages, v_pages, k_scales, v_scales) ||
      (norm != nullptr && (!aligned(norm->q_weight, 16) || !aligned(norm->k_weight, 16))))
    return PBB_ERR_ALIGN;
  pbb::CodedAppendArgs a{};
  a.pos = pos;
  a.q_start = q_start;
  a.table = table;
  a.rope_pos = rope != nullptr ? rope_pos : nullptr;
  a.q = q;
  a.q_out = q_out;
  a.k = k;
  a.v = v;
  a.q_weight = norm != nullptr ? norm->q_weight : nullptr;
  a.k_weight = norm != nullptr ? norm->k_weight : nullptr;
  a.k_pages = static_cast<uint8_t*>(k_pages);
  a.v_pages = static_cast<uint8_t*>(v_pages);
  a.k_scales = k_scales;
  a.v_scales = v_scales;
  a.q_stride = q_stride * 2;
  a.k_stride = k_stride * 2;
  a.v_stride = v_stride * 2;
  a.n = n_tokens;
  a.batch = desc->batch;
  a.uniform = q_start != nullptr ? -1 : n_tokens / desc->batch;
  a.by_uniform = pbb::FastDiv::make(a.uniform > 0 ? (uint32_t)a.uniform : 1u);
  a.hq = desc->n_q_heads;
  a.hkv = desc->n_kv_heads;
  a.turn = rope != nullptr ? 1 : 0;
  a.norm = norm != nullptr ? 1 : 0;
  a.eps = norm != nullptr ? norm->eps : 0.0f;
  a.shape = shape_of(desc);
  a.rope = rope_args(rope, 1.0);
  const hipError_t e = pbb::launch_coded_append(a, desc->head_dim, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? PBB_OK : PBB_ERR_LAUNCH;
}

pbb_status_t pbb_coded_read(const pbb_paged_desc_t* desc, int32_t n_tokens, const int32_t* pos,
                            const int32_t* q_start, const int32_t* table, const void* k_pages,
                            const void* v_pages, const uint8_t* k_scales, const uint8_t* v_scales, void* k,
                            void* v, void* stream) {
  const pbb_status_t st = check_coded(desc, n_tokens);
  if (st != PBB_OK) return st;
  if (q_start == nullptr && n_tokens % desc->batch != 0) return PBB_ERR_SHAPE;
  if (n_tokens == 0) return PBB_OK;
  if (!pos || !table || !k || !v || !cache_given(k_pages, v_pages, k_scales, v_scales)) return PBB_ERR_NULL;
  if (!aligned(pos, 4) || !aligned(q_start, 4) || !aligned(table, 4) || !aligned(k, 16) || !aligned(v, 16) ||
      !cache_aligned(k_pages, v_pages, k_scales, v_scales))
    return PBB_ERR_ALIGN;
  pbb::CodedReadArgs a{};
  a.pos = pos;
  a.q_start = q_start;
  a.table = table;
  a.k_pages = static_cast<const uint8_t*>(k_pages);
  a.v_pages = static_cast<const uint8_t*>(v_pages);
  a.k_scales = k_scales;
  a.v_scales = v_scales;
  a.k = k;
  a.v = v;
  a.n = n_tokens;
  a.batch = desc->batch;
  a.uniform = q_start != nullptr ? -1 : n_tokens / desc->batch;
  a.by_uniform = pbb::FastDiv::make(a.uniform > 0 ? (uint32_t)a.uniform : 1u);
  a.hkv = desc->n_kv_heads;
  a.shape = shape_of(desc);
  const hipError_t e = pbb::launch_coded_read(a, desc->head_dim, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? PBB_OK : PBB_ERR_LAUNCH;
}

pbb_status_t pbb_coded_workspace_bytes(const pbb_paged_desc_t* desc, int32_t n_tokens, size_t* bytes) {
  if (desc == nullptr || bytes == nullptr) return PBB_ERR_NULL;
  const pbb_status_t st = check_coded(desc, n_tokens);
  if (st != PBB_OK) return st;
  *bytes = workspace_of(desc, shape_of(desc), kind_of(desc)).bytes;
  return PBB_OK;
}

pbb_status_t pbb_coded_attention(const pbb_paged_desc_t* desc, int32_t n_tokens, const int32_t* pos,
                                 const int32_t* q_start, const int32_t* table, const void* q,
                                 int64_t q_stride, const void* k_pages, const void* v_pages,
                                 const uint8_t* k_scales, const uint8_t* v_scales, void* out, float* lse,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  const pbb_status_t st = check_coded(desc, n_tokens);
  if (st != PBB_OK) return st;
  if (q_start == nullptr && n_tokens % desc->batch != 0) return PBB_ERR_SHAPE;
  if (!stride_ok(q_stride, desc->n_q_heads, desc->head_dim, 2)) return PBB_ERR_SHAPE;
  if (n_tokens == 0) return PBB_OK;
  pbb::CodedArgs a8{};
  pbb::PagedArgs& a = a8.p;
  a.shape = shape_of(desc);
  a.plan = plan_of(desc, a.shape, n_tokens, q_start != nullptr, kind_of(desc));
  if ((uint64_t)a.plan.tiles * (uint64_t)desc->n_kv_heads > kMaxTiles) return PBB_ERR_SHAPE;
  if (!pos || !table || !q || !cache_given(k_pages, v_pages, k_scales, v_scales) || !out) return PBB_ERR_NULL;
  if (!aligned(pos, 4) || !aligned(q_start, 4) || !aligned(table, 4) || !aligned(q, 16) ||
      !cache_aligned(k_pages, v_pages, k_scales, v_scales) || !aligned(out, 16) || !aligned(lse, 4))
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
  a8.k_scales = k_scales;
  a8.v_scales = v_scales;
  a.out = out;
  a.lse = lse;
  a.q_stride = q_stride * 2;
  a.n = n_tokens;
  a.batch = desc->batch;
  a.hq = desc->n_q_heads;
  a.hkv = desc->n_kv_heads;
  a.group = desc->n_q_heads / desc->n_kv_heads;
  a.scale_log2 = scale_log2(desc);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  hipError_t e = a.plan.planned ? pbb::launch_paged_plan(a, s) : hipSuccess;
  if (e == hipSuccess) e = pbb::launch_coded_attention(a8, desc->head_dim, s);
  return e == hipSuccess ? PBB_OK : PBB_ERR_LAUNCH;
}

}  // extern "C"
