// Argument checks and launch plans that the C-ABI layers of the row and paged-cache operators share.
#pragma once

#include "pbb.h"

#include <cmath>
#include <cstdint>

#include "pbb_paged_internal.h"

namespace pbb_checks {

constexpr int32_t kMaxTokens = 1 << 30;
constexpr int32_t kMaxCapacity = 1 << 30;
constexpr int32_t kMaxBatch = 1 << 24;
// Tiles of an attention call in all heads.  With the pieces (some 2176) and one workgroup per head (at
// most 2^18) more, a launch of 256 threads each stays below 2^32 threads.
constexpr uint64_t kMaxTiles = 1u << 23;
constexpr int32_t kMaxPage = 1 << 20;   // (a page's rows under one KV head lie within 32-bit byte offsets)

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline int64_t elem_bytes(int32_t dtype) { return dtype == PBB_DTYPE_F32 ? 4 : 2; }

inline bool known_dtype(int32_t dtype) { return dtype == PBB_DTYPE_F32 || dtype == PBB_DTYPE_BF16; }

inline pbb_status_t check_rope(const pbb_rope_t* r, int32_t head_dim) {
  if (r->head_dim != head_dim) return PBB_ERR_SHAPE;
  if (r->n_axes < 1 || r->n_axes > PBB_MAX_AXES) return PBB_ERR_SHAPE;
  for (int c = 0; c < head_dim / 2; ++c)   // (below 2^992 no position's turns pass the largest double)
    if (r->axis[c] >= r->n_axes || !(std::fabs(r->turns[c]) < 0x1p992)) return PBB_ERR_SHAPE;
  return PBB_OK;
}

inline pbb::RopeArgs rope_args(const pbb_rope_t* r, double sign) {
  pbb::RopeArgs a;
  for (int c = 0; c < 64; ++c) {
    const bool used = r != nullptr && c < r->head_dim / 2;
    a.turns[c] = used ? sign * r->turns[c] : 0.0;
    a.axis[c] = used ? r->axis[c] : 0;
  }
  return a;
}

// Token stride of rows [n][heads][d] in elements: room for a token's rows, whole 16-byte pieces,
// and no byte offset beyond 2^62.
inline bool stride_ok(int64_t stride, int64_t heads, int64_t d, int64_t u) {
  return stride >= heads * d && (stride * u) % 16 == 0 && stride < (int64_t(1) << 28);
}

// A norm's eps: above 0 (rows of zeros stay zeros) and finite.
inline bool eps_ok(float eps) { return eps > 0.0f && std::isfinite(eps); }

inline pbb_status_t check_paged(const pbb_paged_desc_t* d, int32_t n) {
  if (d == nullptr) return PBB_ERR_NULL;
  if (!known_dtype(d->dtype)) return PBB_ERR_DTYPE;
  if (d->batch < 1 || d->batch > kMaxBatch || d->n_kv_heads < 1 || d->n_q_heads < 1) return PBB_ERR_SHAPE;
  if (d->n_q_heads % d->n_kv_heads != 0) return PBB_ERR_SHAPE;
  if (d->n_q_heads / d->n_kv_heads > pbb::kMaxGroup) return PBB_ERR_SHAPE;
  if (d->head_dim != 64 && d->head_dim != 128) return PBB_ERR_SHAPE;
  if ((int64_t)d->n_q_heads * d->head_dim > (1 << 24)) return PBB_ERR_SHAPE;
  if (d->page_size < 16 || d->page_size > kMaxPage || d->page_size % 16 != 0) return PBB_ERR_SHAPE;
  if (d->n_pages < 1 || d->table_width < 1) return PBB_ERR_SHAPE;
  if ((int64_t)d->page_size * d->table_width > kMaxCapacity) return PBB_ERR_SHAPE;
  if (d->block < 0 || d->block % 2 != 0 || d->window < 0 || (d->block > 0 && d->window > 0))
    return PBB_ERR_SHAPE;
  if (n < 0 || n > kMaxTokens) return PBB_ERR_SHAPE;
  if ((int64_t)d->batch * d->table_width >= (int64_t(1) << 40) ||
      (int64_t)d->n_q_heads * n >= (int64_t(1) << 40))
    return PBB_ERR_SHAPE;
  return PBB_OK;
}

inline pbb::PagedShape shape_of(const pbb_paged_desc_t* d) {
  return pbb::PagedShape::make(d->page_size, d->n_pages, d->table_width, d->block, d->window);
}

// The plan of an attention call, `kind(narrow)` the rules of its kernels.
template <typename K>
pbb::PagedPlan plan_of(const pbb_paged_desc_t* d, const pbb::PagedShape& s, int32_t n, bool ragged, K&& kind) {
  const int group = d->n_q_heads / d->n_kv_heads;
  const bool narrow = pbb::PagedPlan::is_narrow(d->batch, group, n, ragged);
  return pbb::PagedPlan::make(s, kind(narrow), d->batch, d->n_kv_heads, group, n, ragged);
}

inline size_t states_of(const pbb_paged_desc_t* d, const pbb::PagedPlan& p) {
  return (size_t)p.slots * d->n_kv_heads * pbb::paged_state_bytes(p.cols, d->head_dim);
}

// What any call may need: calls of few columns per sequence are all planned alike, of the others one of
// a single token needs most (which of them a call is, its q_start decides).  So the size depends on the
// descriptor alone.
struct Workspace {   // counters, `states` bytes of partial states, the sequences' summary
  size_t bytes, states;
};
template <typename K>
Workspace workspace_of(const pbb_paged_desc_t* d, const pbb::PagedShape& s, K&& kind) {
  const int group = d->n_q_heads / d->n_kv_heads;
  const size_t narrow = states_of(
      d, pbb::PagedPlan::make(s, kind(true), d->batch, d->n_kv_heads, group, d->batch, false));
  const size_t wide = states_of(
      d, pbb::PagedPlan::make(s, kind(false), d->batch, d->n_kv_heads, group, 1, true));
  Workspace w;
  w.states = narrow > wide ? narrow : wide;
  const int scanned = w.states > 0 ? pbb::kPagedScan : pbb::kPagedScanUncut;   // (PagedPlan::planned)
  const size_t bytes = w.states + (d->batch > scanned ? (size_t)pbb::paged_rounds_bytes(d->batch) : 0);
  w.bytes = bytes > 0 ? pbb::kPagedCounterBytes + bytes : 0;
  return w;
}

// What an attention call needs of its workspace, and the parts of one.
inline size_t workspace_need(const pbb_paged_desc_t* d, const pbb::PagedPlan& p, const Workspace& w) {
  const size_t own = w.states + (p.planned ? (size_t)pbb::paged_rounds_bytes(d->batch) : 0);
  return own > 0 ? pbb::kPagedCounterBytes + own : 0;
}
inline void take_workspace(pbb::PagedArgs& a, size_t need, const Workspace& w, void* workspace) {
  unsigned char* const p = need > 0 ? static_cast<unsigned char*>(workspace) : nullptr;
  a.counters = reinterpret_cast<uint32_t*>(p);
  a.states = p != nullptr ? reinterpret_cast<float*>(p + pbb::kPagedCounterBytes) : nullptr;
  a.rounds = p != nullptr ? reinterpret_cast<uint32_t*>(p + pbb::kPagedCounterBytes + w.states) : nullptr;
}

inline float scale_log2(const pbb_paged_desc_t* d) {
  const float scale = d->scale > 0.0f ? d->scale : (float)(1.0 / std::sqrt((double)d->head_dim));
  return (float)((double)scale * 1.4426950408889634);  // log2(e)
}

}  // namespace pbb_checks
