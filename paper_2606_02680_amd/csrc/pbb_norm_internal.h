// Internal interface between the C-ABI layer (pbb_norm_api.cpp, pbb_coded_api.cpp) and the HIP kernels of
// the norms with rotation (pbb_norm.hip) and of the 8-bit paged cache (pbb_coded_rows.hip,
// pbb_coded.hip).  Not installed; not part of the public ABI.
#pragma once

#include "pbb_paged_internal.h"

namespace pbb {

// Rows of one kind (queries or keys) of a norm call.  Strides in bytes.
struct NormPart {
  const void* x;
  const void* grad;      // backward: the gradient of the rotated rows
  void* out;             // forward: the rotated rows; backward: the gradient of x
  const void* weight;    // [head_dim], null: ones
  float* dweight;        // backward, optional: [head_dim]
  int64_t x_stride, grad_stride, out_stride;
  int32_t heads;         // 0: no rows of this kind
  // set by the launcher
  int32_t run;           // heads of a unit of work, and units per group of tokens
  int32_t tokens_per_wave;
  int32_t units;
  int32_t blocks;        // workgroups
  FastDiv by_heads, by_runs;
};

// Norm and rotation of rows, validated on the host; n >= 1 (backward: >= 0).
struct NormArgs {
  NormPart part[2];            // queries, keys
  const int32_t* positions;    // [axes][n]
  float* partials;             // backward: partial sums of the weights' gradients
  int32_t n;
  int32_t turn;                // 1: rope applies
  float eps;
  RopeArgs rope;               // negative rates turn backwards
};

// Workgroups of a backward launch, both kinds together, at most (each writes one partial sum of a weight's
// gradient), and the bytes that one should move at least.
// (2 x 16384 tokens of 32/8 heads, d 128: 198 us with 4096 or 8192, 216 with 2048; 5041 tokens of 16/4 heads,
// d 64, fp32: 19.9 us with 64 KiB, 21.7 with 48; 5000 of 12/2 heads, bf16: 14 to 15, 17.8 without a least.)
constexpr int kNormBlocks = 4096, kNormLeastBytes = 65536, kNormFew = 512;
constexpr int kNormThreads = 256;

// Tokens that a wave of `rows` rows at a time takes together, and a backward launch's workgroups of a
// kind of `heads` of `all` heads: as many units of work to each, no more than the share of kNormBlocks, and
// where there are more than kNormFew none that moves less than kNormLeastBytes.
inline int norm_tokens_per_wave(int heads, int rows) { return heads < rows ? rows / heads : 1; }
inline int norm_grad_blocks(int n, int heads, int all, int rows, int row_bytes) {
  if (heads == 0 || n == 0) return 0;
  const int64_t per = (int64_t)(kNormThreads / 64) * norm_tokens_per_wave(heads, rows);
  const int64_t units = (n + per - 1) / per;
  const int64_t share = (int64_t)kNormBlocks * heads / all > 1 ? (int64_t)kNormBlocks * heads / all : 1;
  const int64_t bytes = 3 * per * heads * row_bytes;   // of a unit
  const int64_t least = (kNormLeastBytes + bytes - 1) / bytes, few = (units + kNormFew - 1) / kNormFew;
  int64_t each = (units + share - 1) / share;
  const int64_t more = least < few ? least : few;
  if (each < more) each = more;
  return (int)((units + each - 1) / each);
}

// Rows of the 8-bit paged cache, validated on the host; n >= 1.  Strides in bytes.
struct CodedAppendArgs {
  const int32_t* pos;
  const int32_t* q_start;     // null with uniform >= 0
  const int32_t* table;
  const int32_t* rope_pos;    // null: the cache position
  const void* q;              // null: no queries
  void* q_out;
  const void* k;
  const void* v;
  const void* q_weight;       // null: ones
  const void* k_weight;
  uint8_t* k_pages;           // [n_pages][hkv][page_size][d] codes
  uint8_t* v_pages;
  uint8_t* k_scales;          // [n_pages][hkv][page_size] scale bytes
  uint8_t* v_scales;
  int64_t q_stride, k_stride, v_stride;
  int32_t n;
  int32_t batch;
  int32_t uniform;            // tokens of every sequence, -1: q_start says
  int32_t hq;
  int32_t hkv;
  int32_t turn;               // 1: rope applies
  int32_t norm;               // 1: the norms apply
  float eps;
  int32_t run;                // rows per grid row (this and the next two set by the launcher)
  int32_t tokens_per_wave;
  FastDiv by_rows;
  FastDiv by_uniform;
  PagedShape shape;
  RopeArgs rope;
};

struct CodedReadArgs {
  const int32_t* pos;
  const int32_t* q_start;
  const int32_t* table;
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const uint8_t* k_scales;
  const uint8_t* v_scales;
  void* k;                    // [n][hkv][d]
  void* v;
  int32_t n;
  int32_t batch;
  int32_t uniform;
  int32_t hkv;
  int32_t run;                // (this and the next two set by the launcher)
  int32_t tokens_per_wave;
  FastDiv by_rows;
  FastDiv by_uniform;
  PagedShape shape;
};

// Attention over an 8-bit paged cache, validated on the host; n >= 1.  p.k_pages and p.v_pages hold codes.
struct CodedArgs {
  PagedArgs p;
  const uint8_t* k_scales;
  const uint8_t* v_scales;
};

// Kinds of attention kernels over it: those of the bf16 cache (paged_kind has the reasons), but for two
// rules.  Few columns: a step takes half the bytes, so that walks are cut into longer pieces where there are
// many (256 tokens of 8 KV heads over PBB supports of up to 2048: 138 us, 156 with 64 steps; 64 tokens of 2
// KV heads over up to 30000: 53, 58 with 128).  Many columns: 1280 pieces (nine chunks of 100 to 3000 over up
// to 20000, 16/2 heads: 1267 us, 1336 with 1024; four of 512: 180 and 188; two chunks and 128 tokens: 198 and
// 203, 211 with 1536).
inline PagedKind coded_kind(bool narrow, int head_dim, int64_t units) {
  PagedKind k = paged_kind(false, narrow, head_dim);
  if (narrow && units >= 1024) k.many_least = 96;   // sequences times KV heads
  if (!narrow) k.pieces = 1280;
  return k;
}

hipError_t launch_norm_rotate(const NormArgs& a, int32_t head_dim, bool f32, hipStream_t stream);
hipError_t launch_norm_rotate_backward(const NormArgs& a, int32_t head_dim, bool f32, hipStream_t stream);
hipError_t launch_coded_append(const CodedAppendArgs& a, int32_t head_dim, hipStream_t stream);
hipError_t launch_coded_read(const CodedReadArgs& a, int32_t head_dim, hipStream_t stream);
hipError_t launch_coded_attention(const CodedArgs& a, int32_t head_dim, hipStream_t stream);

}  // namespace pbb
