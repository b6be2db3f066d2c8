// Internal interface between the C-ABI layer (pbb_api.cpp) and the HIP kernels
// (pbb_kernels.hip).  Not installed; not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "pbb_paged_index.h"

namespace pbb {

enum SupportMode : int32_t { kSupportPBB = 0, kSupportSWA = 1 };

constexpr int32_t kMaxGroup = 16;         // query heads per KV head held by one MFMA tile
constexpr int64_t kSplitMaxUnits = 64;    // bf16 decode launches with at most this many units split
constexpr int64_t kSplitMaxWays = 8;      // workgroups per unit of a split launch, at most
// bf16 decode launches with at most this many units over rings of at most this many slots
// prefetch the whole ring (one 32-slot chunk per wave of a 4-wave workgroup) at entry.
constexpr int32_t kWholeRingMaxUnits = 256;
constexpr int32_t kWholeRingMaxSlots = 128;
constexpr int kWholeRingWaves = 4;        // waves per workgroup of those launches

// Every decode workspace starts with a counter block of this size (one counter per unit of a
// split launch, at most kSplitMaxUnits), whatever the descriptor, so that one workspace,
// zero-filled once, serves split launches of every descriptor it is large enough for.
constexpr size_t kCounterBytes = 256;
static_assert(kCounterBytes >= (size_t)kSplitMaxUnits * 4, "counter block");

// Largest workspace a decode launch can need: the counter block, then the partial states of
// kSplitMaxUnits units (kSplitMaxWays splits x kMaxGroup heads x (head_dim 128 + maximum +
// sum) floats each) -- 4,260,096 bytes.  The allocation-free entry point keeps one buffer of
// this size per device.
constexpr size_t kNoAllocScratchBytes =
    kCounterBytes + (size_t)kSplitMaxUnits * kSplitMaxWays * kMaxGroup * (128 + 2) * 4;

// Everything a decode kernel needs, validated on the host before launch.
struct DecodeArgs {
  const int32_t* pos;
  int32_t* pos_next;   // optional: receives pos + 1 (pos itself for pos < 0); never aliases pos
  const void* q;
  const void* k_new;
  const void* v_new;
  void* k_ring;
  void* v_ring;
  void* out;
  int32_t batch;
  int32_t hq;
  int32_t hkv;
  int32_t group;       // query heads per KV head, 1..16
  int32_t slots;       // ring slots per (sequence, KV head)
  int32_t block;       // PBB block size B
  int32_t window;      // SWA window W
  int32_t mode;        // SupportMode
  float scale_log2;    // softmax scale times log2(e)
  int32_t rope;        // 1: rotate q and the new key by their position (rotary embedding)
  // Split of each unit's key steps over `splits` workgroups (1: none).  With splits > 1 the
  // workgroups of a unit leave partial states (unnormalised output, maximum and sum per head)
  // in ws_part and count in counters[unit]; the last to arrive merges them (Eq.(lse)) and
  // resets the counter to 0.
  int32_t splits;
  uint32_t* counters;  // [batch * hkv], zero between launches
  // [batch * hkv][splits] states: outputs [group][head_dim], then (maximum, sum) [group]
  float* ws_part;
  // Turns per position of rotary channel pair c (angle / 2 pi), c < head_dim / 2.
  double rope_turns[64];
};

// Prefill of prompts at positions 0..n-1, validated on the host before launch.
struct PrefillArgs {
  const void* q;       // [batch][n][hq][d]
  const void* k;       // [batch][n][hkv][d]
  const void* v;
  void* out;           // [batch][n][hq][d]
  float* lse;          // optional [batch][hq][n]
  void* k_ring;        // optional [batch][hkv][slots][d]
  void* v_ring;
  int32_t batch;
  int32_t n;
  int32_t hq;
  int32_t hkv;
  int32_t group;
  int32_t mode;        // SupportMode
  int32_t block;
  int32_t window;
  int32_t slots;
  float scale_log2;
};

// Backward of the prefill attention (gradients of q, k, v), validated on the host.
struct BackwardArgs {
  const void* q;       // [batch][n][hq][d]
  const void* k;       // [batch][n][hkv][d]
  const void* v;
  const void* out;     // forward output [batch][n][hq][d]
  const void* dout;    // upstream gradient [batch][n][hq][d]
  const float* lse;    // forward log-partitions (natural log) [batch][hq][n]
  void* dq;            // [batch][n][hq][d]
  void* dk;            // [batch][n][hkv][d]
  void* dv;
  float* ws;           // workspace [batch][hq][2][n]: lse * log2(e), then dout . out
  int32_t batch;
  int32_t n;
  int32_t hq;
  int32_t hkv;
  int32_t group;
  int32_t mode;        // SupportMode
  int32_t block;
  int32_t window;
  float scale;         // softmax scale
  float scale_log2;    // scale times log2(e)
};

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
  // Many columns: states are large, pieces of fewer than 32 steps cost more than they gain (512 tokens
  // of four prompts 28.7 us, 50 with 16; 128 tokens behind 16000 57, 69 with 64 steps).
  if (f32) return PagedKind{kPagedColsF32, kPagedStepF32, 0, 0, 2048, 32};
  return PagedKind{kPagedCols, kPagedStep, 0, 0, 1024, 32};
}
constexpr size_t kPagedCounterBytes = 65536;

// Bytes of one partial state: an unnormalised output, a reference and a sum per column.
constexpr size_t paged_state_bytes(int cols, int head_dim) {
  return (size_t)cols * (size_t)(head_dim + 2) * 4;
}

hipError_t launch_ring_zero(void* k_ring, void* v_ring, size_t bytes_per_tensor,
                            hipStream_t stream);

hipError_t launch_ring_fill(const int32_t* pos, const void* k_src, const void* v_src,
                            void* k_ring, void* v_ring, int32_t batch, int32_t hkv,
                            int32_t src_len, int32_t slots, int32_t row_bytes,
                            hipStream_t stream);

// bf16 decode on matrix cores; head_dim 64 or 128.
hipError_t launch_decode_bf16(const DecodeArgs& a, int32_t head_dim, hipStream_t stream);

// bf16 prefill on matrix cores; head_dim 64 or 128; n >= 1.
hipError_t launch_prefill_bf16(const PrefillArgs& a, int32_t head_dim, hipStream_t stream);

// bf16 backward on matrix cores: dq (with delta), then dk/dv; head_dim 64 or 128; n >= 1.
hipError_t launch_backward_bf16(const BackwardArgs& a, int32_t head_dim, hipStream_t stream);

// fp32 decode, on matrix cores (one query head per KV head: on vector ALUs); head_dim 64 or 128.
hipError_t launch_decode_f32(const DecodeArgs& a, int32_t head_dim, hipStream_t stream);

// Rotary rows, paged append, attention over a paged cache; head_dim 64 or 128.
hipError_t launch_rotate(const RotateArgs& a, int32_t head_dim, bool f32, hipStream_t stream);
hipError_t launch_paged_append(const AppendArgs& a, int32_t head_dim, bool f32, hipStream_t stream);
hipError_t launch_paged_bf16(const PagedArgs& a, int32_t head_dim, hipStream_t stream);
hipError_t launch_paged_f32(const PagedArgs& a, int32_t head_dim, hipStream_t stream);

// The library-held decode workspace of the current device (kNoAllocScratchBytes bytes): its
// device address, resolved once per device, whose first call also clears the counter block
// with a fill kernel on `stream`.  Allocates nothing.
hipError_t noalloc_scratch(void** ptr, hipStream_t stream);

}  // namespace pbb
