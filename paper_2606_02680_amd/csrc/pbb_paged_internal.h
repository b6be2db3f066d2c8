// Internal interface between the C-ABI layer (pbb_paged_api.cpp) and the HIP kernels of the rotation
// and paged-cache operators (pbb_rotary.hip, pbb_paged.hip, pbb_paged_f32.hip).  Not installed; not part
// of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "pbb_internal.h"
#include "pbb_paged_index.h"

namespace pbb {

// Rotary rates of a launch (pbb_rope_t, checked).
struct RopeArgs {
  double turns[64];
  uint8_t axis[64];
};

// Rotation of rows, validated on the host; n >= 1.  Strides in bytes.
struct RotateArgs {
  const void* x;
  void* out;
  const int32_t* positions;   // [axes][n]
  int64_t x_stride, out_stride;
  int32_t n;
  int32_t heads;
  int32_t run;                // heads per grid row (this and the next two set by the launcher)
  int32_t tokens_per_wave;
  FastDiv by_heads;
  RopeArgs rope;              // negative rates turn backwards
};

// Append to a paged cache, validated on the host; n >= 1.  Strides in bytes.
struct AppendArgs {
  const int32_t* pos;
  const int32_t* q_start;     // null with uniform >= 0
  const int32_t* table;
  const int32_t* rope_pos;    // null: the cache position
  const void* q;              // null: no queries
  void* q_out;
  const void* k;
  const void* v;
  void* k_pages;
  void* v_pages;
  int64_t q_stride, k_stride, v_stride;
  int32_t n;
  int32_t batch;
  int32_t uniform;            // tokens of every sequence, -1: q_start says
  int32_t hq;
  int32_t hkv;
  int32_t run;                // rows per grid row (set by the launcher)
  int32_t turn;               // 1: rope applies
  FastDiv by_uniform;
  PagedShape shape;
  RopeArgs rope;
};

// Attention over a paged cache, validated on the host; n >= 1.
struct PagedArgs {
  const int32_t* pos;
  const int32_t* q_start;     // null with plan.uniform >= 0
  const int32_t* table;
  const void* q;              // rows [n][hq][d], tokens q_stride bytes apart
  const void* k_pages;        // [n_pages][hkv][page_size][d]
  const void* v_pages;
  void* out;                  // [n][hq][d]
  float* lse;                 // optional [hq][n]
  uint32_t* counters;         // per partial state of a head, zero between launches
  float* states;              // partial states of cut walks
  uint32_t* rounds;           // the sequences' summary (plan.planned)
  int64_t q_stride;
  int32_t n;
  int32_t batch;
  int32_t hq;
  int32_t hkv;
  int32_t group;
  float scale_log2;
  PagedShape shape;
  PagedPlan plan;
};

// Kinds of paged attention kernels.
constexpr int kPagedCols = 128, kPagedStep = 32;          // bf16
constexpr int kPagedColsF32 = 64, kPagedStepF32 = 16;     // fp32
inline PagedKind paged_kind(bool f32, bool narrow, int head_dim) {
  // Few columns.  One round is one workgroup per CU at d = 128 (32/8 heads: one sequence of 32000 28.0
  // us, 33.2 with half as many again; eight of up to 8000 30.7 / 34.3; tiles and pieces over one round
  // 37), two at d = 64, and two of the fp32 kernel's register-bound ones.  Shares of 64 steps and more
  // are cut by the second rule: 2048 pieces (192 sequences of up to 32768: 1875, 1934 with 1024) of 64
  // steps (256 of up to 600: 71; pieces of 8: 115), in fp32 32 of 16 keys (256 of up to 2000, 16/2
  // heads: 125 / 134 with 64).
  if (f32 && narrow) return PagedKind{kPagedNarrowCols, kPagedStepF32, 512, 8, 2048, 32};
  if (narrow) return PagedKind{kPagedNarrowCols, kPagedStep, head_dim == 64 ? 512 : 256, 8, 2048, 64};
  // Many columns: two workgroups per CU are a round, and shares of 32 steps and more come under the
  // second rule, since states are large (one sequence of 26 tokens behind 9900, 16/2 heads: 25.7 us, 38.5
  // with pieces of 32 steps; 128 tokens behind 16000, 32/8 heads: 57 with 32, 69 with 64).
  if (f32) return PagedKind{kPagedColsF32, kPagedStepF32, 512, 8, 2048, 32};
  return PagedKind{kPagedCols, kPagedStep, 512, 8, 1024, 32};
}
constexpr size_t kPagedCounterBytes = 65536;

// Bytes of one partial state: an unnormalised output, a reference and a sum per column.
constexpr size_t paged_state_bytes(int cols, int head_dim) {
  return (size_t)cols * (size_t)(head_dim + 2) * 4;
}

// Rotary rows, paged append, attention over a paged cache; head_dim 64 or 128.
hipError_t launch_rotate(const RotateArgs& a, int32_t head_dim, bool f32, hipStream_t stream);
hipError_t launch_paged_append(const AppendArgs& a, int32_t head_dim, bool f32, hipStream_t stream);
hipError_t launch_paged_plan(const PagedArgs& a, hipStream_t stream);   // (before either of these two)
hipError_t launch_paged_bf16(const PagedArgs& a, int32_t head_dim, hipStream_t stream);
hipError_t launch_paged_f32(const PagedArgs& a, int32_t head_dim, hipStream_t stream);

}  // namespace pbb
