// Attention over an 8-bit paged KV cache on gfx950 (MI355X): single tokens, chunks, or a mixture.
//
// The work, its split and its masks are those of pbb_paged.hip; what differs is how rows enter the products.
// A cached row is D e4m3 codes and a scale byte (a power of two).
//
// Codes become bf16 values, exactly (two per instruction, the row's power of two with them), and the products
// run on v_mfma_f32_16x16x32_bf16: queries are not quantised.  Chunks: once per workgroup, on the way from
// registers into the LDS tiles.  Few columns: each wave its own rows, on the way from its LDS stages into
// the products (values after the transposed read, their powers of two multiplied into the weights).
// v_mfma_scale_f32_16x16x128_f8f6f4 takes codes and scale bytes as they are, and twice as many of them, so
// that two products with queries in two e4m3 parts (which hold a bf16 exactly) cost one of these; but it
// aligns products of eight to some 18 bits of their largest: log-partitions were off by up to 3e-4.
//
// Bound: few columns HBM, with (D + 1) bytes per key row; many columns the matrix and vector work of a step.

#include <type_traits>

#include "pbb_norm_internal.h"
#include "pbb_coded_device.h"
#include "pbb_paged_device.h"

namespace pbb {
namespace {

constexpr int kWaves = 4;
constexpr int kGroups = 2;             // 16-column groups of a wave
static_assert(kPagedCols == 16 * kGroups * kWaves && kPagedStep == 32, "tile");

// Wave priorities: where several waves of a SIMD could issue, those in their products go first (their chain of
// matrix instructions is what a step waits for), value products before score products, whose conversions run
// along.  Five chunks 1407 -> 1360 us, four of 2000 to 4000 under a window of 4096 765 -> 735, D 64 287 ->
// 272.  Few-column walks in such a launch go with score products, but for the issue of their loads: above all
// but value products throughout, 130 sequences with two chunks took 184 us instead of 198, but 140 with
// twelve short chunks, whose long walks then starve, 427 instead of 400; below them all the time, 64-channel
// mixtures 158 instead of 146.  (300 with six chunks, D 64: 157, 151 without priorities.)
constexpr int kNoPriority = 0, kScorePriority = 1, kValuePriority = 2;

// ------------------------------------------------------------------------------------------
// LDS tiles of codes: blocks of 8 rows (8 D bytes), in lines of 128 bytes that hold 8 pieces of 16 bytes:
// at D = 128 line r is row r, at D = 64 line r holds rows r and r + 4.  A piece lies in slot
// piece ^ (2 line mod 8) of its line, so that the row reads and the transposed reads spread over the banks
// (see tile_row in pbb_device.h).
template <int D>
__device__ __forceinline__ constexpr uint32_t code_at(int r, int piece) {
  const int line = D == 128 ? r & 7 : r & 3;
  const int slot = (D == 128 ? piece : ((r >> 2) & 1) * 4 + piece) ^ ((2 * (D == 128 ? line >> 1 : line)) & 7);
  return (uint32_t)((r >> 3) * 8 * D + line * 128 + slot * 16);
}
// Byte offset, within the 8-row blocks, of what lane `lane` of a DMA instruction loads (16 bytes; at D =
// 128 the instruction fills one block, at D = 64 two).
template <int D>
__device__ __forceinline__ uint32_t code_source(int lane) {
  const int block = D == 128 ? 0 : lane >> 5;
  const int line = D == 128 ? lane >> 3 : (lane >> 3) & 3;
  const int piece = (lane & 7) ^ ((2 * (D == 128 ? line >> 1 : line)) & 7);
  const int row = D == 128 ? line : line + 4 * (piece >> 2);
  return (uint32_t)((8 * block + row) * D + (D == 128 ? piece : piece & 3) * 16);
}

// The bytes of a word of codes that are NaN, as 0xFF.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  const uint32_t m = (((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7;
  return m * 0xFFu;
}

// ------------------------------------------------------------------------------------------
// Few columns: tiles of at most 16 (single tokens, short drafts).  The 16-key halves of the piece's steps
// are dealt to the waves one by one, each with LDS stages of its own (keys, values, scale bytes of a
// half), so that nothing but the merge of the waves at the end waits for another wave.  Bound: HBM.  192
// tokens over 256 to 32768, 32/8 heads, D 128 (6.75 GB): 1055 to 1065 us, 6.4 TB/s, where streaming reads reach
// 6.5 (of the bf16 cache's twice the bytes: 2008 us); two or four stages, or four waves per SIMD: the same.
template <int D>
struct Narrow {
  static constexpr int STAGES = D == 128 ? 3 : 4;
  static constexpr int TILE = 16 * D;                  // a half's codes of K or V
  static constexpr int STAGE = 2 * TILE + 256;         // and 16 scale bytes each, in the last 256
  static constexpr int LDS = kWaves * STAGES * STAGE;
  static constexpr int OPS = 2 * (TILE / 1024) + 1;    // DMA instructions of a half
};

template <int D, bool IN_PLACE>
__device__ __forceinline__ void narrow_walk(const CodedArgs& a8, const PagedItem& it, int g,
                                            unsigned char* smem) {
  typedef Narrow<D> L;
  const PagedArgs& a = a8.p;
  constexpr int NW = kWaves;
  constexpr int S = L::STAGES;
  constexpr int NB = D / 16;
  constexpr int NC = D / 32;            // 32-channel chunks: a transposed read each
  constexpr int KK = D / 32;            // 32-channel slices of the score contraction
  constexpr int P = D / 64;             // pieces of a key's codes that a lane reads
  constexpr int COLS = kPagedNarrowCols;
  static_assert(NarrowOut<uint16_t, D, NW>::LDS <= L::LDS, "the waves' states fit their stages");

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15;
  const int j4 = lane >> 4;
  const int G = a.group;
  const PagedPlan& pl = a.plan;
  const PagedShape& sh = a.shape;
  const int tokens = it.c.count;
  const int64_t row0 = it.c.row0;
  const int cols = tokens * G;
  const NarrowOut<uint16_t, D, NW> result{a, it, g, cols};
  if (it.c.pos < 0) {
    result.skip(tid);
    return;
  }

  // Halves [h0, h1) of the piece (half h: keys 16 h .. 16 h + 15).
  const int t0 = it.c.pos;
  const int t_last = t0 + tokens - 1;
  const int s_first = sh.support_lo(t0) >> 5;
  const int last_key = min(t_last, sh.capacity - 1);
  const int nsteps = max(0, (last_key >> 5) - s_first + 1);
  int h0 = 2 * s_first, h1 = min(2 * (s_first + nsteps), (last_key >> 4) + 1);
  if (it.ways > 1) {
    h1 = min(h1, 2 * (s_first + (int)((int64_t)(it.piece + 1) * nsteps / it.ways)));
    h0 = 2 * (s_first + (int)((int64_t)it.piece * nsteps / it.ways));
  }
  if (h1 <= h0) h0 = h1 = 0;   // (positions past the table: 16 h would pass 2^31)

  // A half's rows in the pool, from its page entry, which is read through the scalar cache ahead of the
  // half's loads; halves without a page read page 0.
  const int32_t* const table = a.table + (size_t)it.b * sh.width;
  struct Entry { int id, slot; };
  auto fetch = [&](int h) -> Entry {   // (halves past the walk read the last entry, for nothing)
    const int i = min(sh.by_page.div(16 * h), sh.width - 1);
    return Entry{scalar_word(table, i), 16 * h - i * sh.page_size};
  };
  auto row_of = [&](const Entry& e) -> uint64_t {
    return ((uint64_t)(sh.is_page(e.id) ? (uint32_t)e.id : 0u) * (uint32_t)a.hkv + (uint32_t)g) *
               (uint32_t)sh.page_size + (uint32_t)e.slot;
  };
  unsigned char* const wbuf = smem + wave * S * L::STAGE;
  const uint32_t src = code_source<D>(lane);
  const uint8_t* const scales = (lane & 4 ? a8.v_scales : a8.k_scales) + 4 * (lane & 3);
  uint32_t gone = 0;   // whether the halves' keys have no page, the youngest issued lowest
  auto issue = [&](const Entry& e, int stage) {   // (codes non-temporal: read once in a call)
    gone |= sh.is_page(e.id) ? 0u : 1u;
    const uint64_t row = row_of(e);
    unsigned char* lds = wbuf + stage * L::STAGE;
    const unsigned char* k = (const unsigned char*)a.k_pages + row * D;
    const unsigned char* v = (const unsigned char*)a.v_pages + row * D;
#pragma unroll
    for (int y = 0; y < L::TILE / 1024; ++y)
      __builtin_amdgcn_global_load_lds((const void*)(k + 1024 * y + src),
                                       (__attribute__((address_space(3))) void*)(lds + 1024 * y), 16, 0,
                                       kCachePolicyNT);
#pragma unroll
    for (int y = 0; y < L::TILE / 1024; ++y)
      __builtin_amdgcn_global_load_lds((const void*)(v + 1024 * y + src),
                                       (__attribute__((address_space(3))) void*)(lds + L::TILE + 1024 * y), 16,
                                       0, kCachePolicyNT);
    __builtin_amdgcn_global_load_lds((const void*)(scales + row),
                                     (__attribute__((address_space(3))) void*)(lds + 2 * L::TILE), 4, 0, 0);
  };
  int h = h0 + wave;
  // this lane's column (past the tile's: the last token's row, a zero query, no key seen)
  const int cp = min(pl.by_group.div(c16), tokens - 1);
  const bool valid = c16 < cols;
  const int tcol = valid ? t0 + cp : -1;
  const int lo_c = sh.support_lo(t0 + cp);
  bf16x8 qB[KK];   // slice 2 i + x: channels 16 (j4 + 4 i) + 8 x .. + 7
  {
    const unsigned char* qrow = (const unsigned char*)a.q + (row0 + cp) * a.q_stride +
                                (int64_t)(g * G + (valid ? c16 - cp * G : 0)) * (D * 2) + 32 * j4;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const u32x4 w = *(const u32x4*)(qrow + 128 * (kk >> 1) + 16 * (kk & 1));
      qB[kk] = __builtin_bit_cast(bf16x8, valid ? w : u32x4{0u, 0u, 0u, 0u});
    }
  }
  Entry after = {0, 0};
  if (h < h1) {
#pragma unroll
    for (int s = 0; s < S - 1; ++s) {
      gone <<= 1;
      if (h + s * NW < h1) issue(fetch(h + s * NW), s);
    }
    after = fetch(min(h + (S - 1) * NW, h1 - 1));
  }

  // LDS byte addresses of this lane's reads in stage 0
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)wbuf;
  uint32_t ra[P], va[NC];
#pragma unroll
  for (int i = 0; i < P; ++i) ra[i] = base + code_at<D>(c16, j4 + 4 * i);
#pragma unroll
  for (int nc = 0; nc < NC; ++nc)   // (a transposed read takes pairs of channels as its elements)
    va[nc] = base + L::TILE + code_at<D>(4 * j4 + (c16 >> 2), 2 * nc + ((c16 & 3) >> 1)) + ((c16 & 1) << 3);
  const uint32_t ks = base + 2 * L::TILE + (uint32_t)c16, vs = base + 2 * L::TILE + 16 + 4 * (uint32_t)j4;
  const __attribute__((address_space(3))) unsigned char* lds0 = nullptr;
  // the run [ua, ub) of halves whose keys all lie in every column's support
  const int ua = (sh.support_lo(t_last) + 15) >> 4;
  const int ub = (t0 + 1) >> 4;

  float m = valid ? kNoScore : 0.0f, lsum = 0.0f;
  f32x4 acc[NB];   // [2 nc + parity][e]: channel 32 nc + 8 j4 + 2 e + parity
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) acc[nb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const float sc = a.scale_log2;
  bool odd = false;

  int stage = 0;
  for (; h < h1; h += NW) {
    // the half S - 1 ahead goes over the stage that the last half has left
    if constexpr (!IN_PLACE) __builtin_amdgcn_s_setprio(kNoPriority);
    gone <<= 1;
    if (h + (S - 1) * NW < h1) issue(after, stage == 0 ? S - 1 : stage - 1);
    after = fetch(min(h + S * NW, h1 - 1));
    __builtin_amdgcn_sched_barrier(0);
    wait_groups<S - 1, L::OPS>(min(S - 1, (h1 - 1 - h) / NW));
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!IN_PLACE) __builtin_amdgcn_s_setprio(kScorePriority);
    const uint32_t sb = (uint32_t)(stage * L::STAGE);
    stage = stage == S - 1 ? 0 : stage + 1;
    const bool none = (gone >> (S - 1)) & 1u;
    u32x4 keys[P];
#pragma unroll
    for (int i = 0; i < P; ++i) keys[i] = *(const __attribute__((address_space(3))) u32x4*)(lds0 + ra[i] + sb);
    const float key_unit = __uint_as_float((uint32_t)*(lds0 + ks + sb) << 23);
    const uint32_t value_scales = *(const __attribute__((address_space(3))) uint32_t*)(lds0 + vs + sb);
    u32x2 vr[NC];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) vr[nc] = tr_read<0>(va[nc] + sb);
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const uint32_t x = keys[kk >> 1][2 * (kk & 1)], y = keys[kk >> 1][2 * (kk & 1) + 1];
      const u32x4 w = {values2<false>(x, key_unit), values2<true>(x, key_unit), values2<false>(y, key_unit),
                       values2<true>(y, key_unit)};
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), qB[kk], s, 0, 0, 0);
    }
    const bool masked = h < ua || h >= ub || none;
    const int k0 = 16 * h + 4 * j4;
    if (masked) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s[e] = e >= lo_c - k0 && e <= tcol - k0 && !none ? s[e] : kNegInf;
    }
    float p[4], ps;
    auto weights = [&]() {
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = fast_exp2(__builtin_fmaf(s[e], sc, -m));
      ps = (p[0] + p[1]) + (p[2] + p[3]);
      return !(ps <= kWeightCap);
    };
    auto column_max = [&]() {
      return max_xor16_32(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))) * sc;
    };
    if (h == h0 + wave) m = fmaxf(m, column_max());
    if (__builtin_amdgcn_ballot_w64(weights()) != 0) {
      const float cand = column_max();
      // (only the columns whose own weights ask for it: none depends on its neighbours' data)
      const bool grow = cand > m && max_xor16_32(ps) > kWeightCap;
      const float alpha = grow ? fast_exp2(m - cand) : 1.0f;
      m = grow ? cand : m;
      lsum *= alpha;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) acc[nb] *= alpha;
      weights();
    }
    lsum += ps;
    // Weights times their values' powers of two (exact), as two bf16 parts, the upper one cut off, the lower
    // one rounded: 2^-15 of a weight is lost.  One product contracts both with the same values, since 16
    // keys would fill half of its 32 slots.
    u32x2 high, low;
    float w[4], rest[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float unit = __uint_as_float((e == 0 ? value_scales << 23 : value_scales >> (8 * e) << 23) & 0x7F800000u);
      w[e] = p[e] * unit;
      if (masked) w[e] = s[e] == kNegInf ? 0.0f : w[e];   // (a scale byte outside the support may be 255)
      rest[e] = w[e] - __uint_as_float(__float_as_uint(w[e]) & 0xFFFF0000u);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      high[e] = __builtin_amdgcn_perm(__float_as_uint(w[2 * e + 1]), __float_as_uint(w[2 * e]), 0x07060302u);
      low[e] = pack_bf16(rest[2 * e], rest[2 * e + 1]);
    }
    const bf16x8 weight = join_chunks(high, low);
    if constexpr (D == 128)
      asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(vr[0]), "+v"(vr[1]), "+v"(vr[2]), "+v"(vr[3]));
    else
      asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(vr[0]), "+v"(vr[1]));
    if (masked) {
      uint32_t any = 0;
#pragma unroll
      for (int nc = 0; nc < NC; ++nc) any |= nan_bytes(vr[nc][0]) | nan_bytes(vr[nc][1]);
      if (__builtin_amdgcn_ballot_w64(any != 0) != 0) {
        odd = true;
#pragma unroll
        for (int nc = 0; nc < NC; ++nc)
#pragma unroll
          for (int e = 0; e < 2; ++e) vr[nc][e] &= ~nan_bytes(vr[nc][e]);
      }
    }
    // keys 4 j4 .. + 3 of the even, then of the odd channel of this lane's pair
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const u32x2 r = vr[nb >> 1];
      const uint32_t c = __builtin_amdgcn_perm(r[1], r[0], nb & 1 ? 0x07050301u : 0x06040200u);
      const u32x2 v = {values2<false>(c, 1.0f), values2<true>(c, 1.0f)};
      acc[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join_chunks(v, v), weight, acc[nb], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  if (odd) {   // the NaN of masked halves, straight from the pages, into the columns that see their keys
    for (h = h0 + wave; h < h1; h += NW) {
      const Entry e = fetch(h);
      if (!sh.is_page(e.id) || (h >= ua && h < ub)) continue;
      const unsigned char* row = (const unsigned char*)a.v_pages + row_of(e) * D + 8 * j4;
      for (int key = 16 * h; key < 16 * h + 16; ++key, row += D) {
        const bool sees = key >= lo_c && key <= tcol;
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
          const u32x2 c = *(const u32x2*)(row + 32 * nc);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (sees && (nan_bytes(c[i >> 2]) >> (8 * (i & 3)) & 1u))
              acc[2 * nc + (i & 1)][i >> 1] = __builtin_nanf("");
        }
      }
    }
  }

  lsum = sum_xor16_32(lsum);
  __syncthreads();   // every wave is done with its stages
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
    const f32x4 x = acc[2 * nc], y = acc[2 * nc + 1];
    float* o = result.outputs(smem) + (wave * COLS + c16) * D + 32 * nc + 8 * j4;
    *(f32x4*)o = f32x4{x[0], y[0], x[1], y[1]};
    *(f32x4*)(o + 4) = f32x4{x[2], y[2], x[3], y[3]};
  }
  if (j4 == 0) {
    result.references(smem)[wave * COLS + c16] = m;
    result.sums(smem)[wave * COLS + c16] = lsum;
  }
  result.template finish<IN_PLACE, IN_PLACE ? COLS : kPagedCols>(tid, smem, 16 * h0, 16 * h1 - 1);
}

// ------------------------------------------------------------------------------------------
// Many columns.  Each wave takes 8 of a step's key rows and 8 of its value rows into registers, two steps
// ahead, their scale bytes through the scalar cache, and converts them into the bf16 tiles of the step after
// the one that it works on, under the score products of that one.  The rest of a step is the bf16 kernel's,
// so both give the same bits from the same values.
//
// Bound: a step's matrix instructions (128 x 32 x D twice, a SIMD's matrix core 0.39 busy) and the softmax and
// conversions beside them (its vector ALUs 0.6: an exponential takes four times as long as other
// instructions), with the barrier's and the chain's waits between.  Five chunks of 300 to 2048 tokens over up
// to 30 thousand, 32/8 heads, D 128: 1360 us (943 TFLOP/s; the bf16 cache's kernel, which moves its rows by
// DMA and converts nothing, 1321).  Measured there, without the priorities (1412): rows two steps ahead as DMA
// of codes into LDS stages and converted from there, which takes no registers, 1568; a branch around the
// conversions of a last step, so that none run under the products, 1470; scale bytes by vector loads and the
// table by 64-bit addresses, 1456.
template <int D>
struct Wide {
  static constexpr int TILE = 64 * D;               // 32 rows in bf16
  static constexpr int STAGE = 2 * TILE;            // keys, then values
  static constexpr int LDS = 2 * STAGE;
  static constexpr int ALL = LDS > Narrow<D>::LDS ? LDS : Narrow<D>::LDS;
};

// The transposed operands of 32 of a tile's channels, 32 PART .. + 31, as read_chunks has them; wait_part: until
// at most N LDS reads issued after them are on their way.
template <int D, int OFF, int PART>
__device__ __forceinline__ void read_part(u32x2 (&dst)[4], const uint32_t (&ta)[4], uint32_t sb) {
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    constexpr int AT = OFF + (PART >> 1) * kTileLine;
    dst[2 * x] = tr_read<AT>(ta[2 * (PART & 1) + x] + sb);
    dst[2 * x + 1] = tr_read<AT + 32 * D>(ta[2 * (PART & 1) + x] + sb);
  }
}
template <int N>
__device__ __forceinline__ void wait_part(u32x2 (&v)[4]) {
  asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]) : "i"(N));
}

// Table entry i >= 0, through the scalar cache, by a 32-bit byte offset (a width is at most 2^26; the 64-bit
// sum costs scalar registers and instructions in every step).
__device__ __forceinline__ int entry(const int32_t* table, int i) {
  typedef const __attribute__((address_space(4))) char* Bytes;
  return *(const __attribute__((address_space(4))) int32_t*)((Bytes)(const void*)table + (uint32_t)i * 4u);
}

// Eight bytes that the launch does not write, through the scalar cache.
__device__ __forceinline__ uint64_t scalar_long(const uint8_t* p) {
  return *(const __attribute__((address_space(4))) uint64_t*)(const void*)p;
}

template <int D, int OCC>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(OCC)))
void coded_kernel(CodedArgs a8) {
  typedef Wide<D> L;
  const PagedArgs& a = a8.p;
  constexpr int NW = kWaves;
  constexpr int QC = kGroups;
  constexpr int NB = D / 16;
  constexpr int ROWB = D * 2;           // bytes of a query or output row, and of a bf16 value row
  constexpr int KK = D / 32;            // 32-channel slices of the score contraction
  __shared__ __align__(1024) unsigned char smem[L::ALL];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15;
  const int j4 = lane >> 4;
  const int G = a.group;
  const PagedPlan& pl = a.plan;
  const PagedShape& sh = a.shape;

  const int item = pl.by_hkv.div((int)blockIdx.x);
  const int g = (int)blockIdx.x - item * a.hkv;
  PagedItem it;
  if (!find_item<false>(a, item, lane, it)) return;
  if (it.c.count <= pl.narrow_tokens) {
    narrow_walk<D, false>(a8, it, g, smem);
    return;
  }
  const int p0 = it.tile * pl.tq;                               // the tile's tokens in the chunk
  const int tokens = min(pl.tq, it.c.count - p0);
  const int64_t row0 = (int64_t)it.c.row0 + p0;                 // packed row of the first one
  const int cols = tokens * G;

  if (it.c.pos < 0) {   // a skipped sequence, never cut: zeros, no log-partition
    for (int i = tid; i < cols * (ROWB / 16); i += NW * 64) {
      const int col = i / (ROWB / 16), pc = i - col * (ROWB / 16);
      const int cp = pl.by_group.div(col);
      *(u32x4*)((unsigned char*)a.out + ((row0 + cp) * a.hq + (int64_t)g * G + (col - cp * G)) * ROWB +
                pc * 16) = u32x4{0u, 0u, 0u, 0u};
    }
    if (a.lse != nullptr)
      for (int col = tid; col < cols; col += NW * 64) {
        const int cp = pl.by_group.div(col);
        a.lse[(int64_t)(g * G + col - cp * G) * a.n + row0 + cp] = kNegInf;
      }
    return;
  }

  const int t0 = it.c.pos + p0;
  const int t_last = t0 + tokens - 1;
  int s_first = sh.support_lo(t0) >> 5;
  int nsteps = max(0, (min(t_last, sh.capacity - 1) >> 5) - s_first + 1);
  if (nsteps == 0) s_first = 0;   // (all past the table: positions whose next steps pass 2^31)
  if (it.ways > 1) {
    const int lo = (int)((int64_t)it.piece * nsteps / it.ways);
    const int hi = (int)((int64_t)(it.piece + 1) * nsteps / it.ways);
    s_first += lo;
    nsteps = hi - lo;
  }

  // Loads of a step: wave w takes rows 8 w .. + 7 of its keys and values, which lie in one page.  An entry
  // that names no page reads page 0, and the half's keys are masked (`gone`, two bits per step, the
  // youngest lowest).
  const int32_t* const table = a.table + (size_t)it.b * sh.width;
  int next_key = s_first * 32;   // first key of the step to be issued next
  int id0 = 0, id1 = 0;          // its entries (the two halves')
  bool past = false;             // the second half lies past the table
  int slot = 0;                  // this wave's rows in their page
  auto fetch = [&]() {
    const int i0 = sh.by_page.div(next_key), i1 = sh.by_page.div(next_key + 16);
    id0 = entry(table, min(i0, sh.width - 1));
    id1 = entry(table, min(i1, sh.width - 1));
    past = i1 >= sh.width;
    slot = next_key + 8 * wave - (wave >= 2 ? i1 : i0) * sh.page_size;
  };
  uint32_t gone = 0;
  const uint64_t page_rows = (uint64_t)(uint32_t)a.hkv * (uint32_t)sh.page_size;
  const uint64_t head_row = (uint64_t)(uint32_t)g * (uint32_t)sh.page_size;
  u32x2 raw_k[D / 64], raw_v[D / 64];   // 8 codes of each line of the row
  uint64_t raw_ks = 0, raw_vs = 0;      // the 8 rows' scale bytes, through the scalar cache
  auto load = [&]() {   // the next step's rows: lane l takes 8 codes of each 64 of row l / 8
    const bool ok0 = sh.is_page(id0), ok1 = sh.is_page(id1) && !past;
    gone |= (ok0 ? 0u : 1u) | (ok1 ? 0u : 2u);
    const uint32_t id0s = ok0 ? (uint32_t)id0 : 0u, id1s = ok1 ? (uint32_t)id1 : 0u;
    const uint32_t id = wave >= 2 ? id1s : id0s;
    const uint64_t row = (uint64_t)id * page_rows + head_row + (uint32_t)slot;
    // (an offset that the compiler takes as new: else it keeps 64-bit addresses per lane)
    uint32_t at = D * ((uint32_t)lane >> 3) + 8 * ((uint32_t)lane & 7);
    asm volatile("" : "+v"(at));
    const unsigned char* const k = (const unsigned char*)a.k_pages + row * D;
    const unsigned char* const v = (const unsigned char*)a.v_pages + row * D;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      raw_k[i] = *(const u32x2*)(k + at + 64 * i);
      raw_v[i] = *(const u32x2*)(v + at + 64 * i);
    }
    raw_ks = scalar_long(a8.k_scales + row);
    raw_vs = scalar_long(a8.v_scales + row);
    next_key += 32;
  };
  // where this lane's values go in a tile: row 8 wave + lane / 8, piece lane mod 8 of each line (so that 16
  // lanes write 16 different pieces of a bank row)
  __attribute__((address_space(3))) unsigned char* lds0 = nullptr;
  uint32_t vw;
  {
    const int r = 8 * wave + (lane >> 3);
    vw = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem +
         (uint32_t)(tile_row<D>(r) + (((lane & 7) ^ tile_swz(r)) << 4));
  }
  auto convert = [&](int stage) {
    const uint32_t to = vw + (uint32_t)(stage * L::STAGE);
    auto put = [&](uint32_t at, const u32x2 (&raw)[D / 64], float unit) {
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const u32x4 x = {values2<false>(raw[i][0], unit), values2<true>(raw[i][0], unit),
                         values2<false>(raw[i][1], unit), values2<true>(raw[i][1], unit)};
        *(__attribute__((address_space(3))) u32x4*)(lds0 + at + kTileLine * i) = x;
      }
    };
    const uint32_t mine = (uint32_t)lane & 56u;   // this lane's row's byte of the 8
    put(to, raw_k, __uint_as_float((uint32_t)(raw_ks >> mine) << 23 & 0x7F800000u));
    put(to + L::TILE, raw_v, __uint_as_float((uint32_t)(raw_vs >> mine) << 23 & 0x7F800000u));
  };

  fetch();
  if (nsteps > 0) load();
  // This lane's query columns: column col -> token p0 + col / G, head g*G + col % G.  Columns past
  // the tile's tokens get zero queries and see no key of a masked step (tcol -1); they load the last
  // token's row, and nothing of them is stored.
  struct Column {
    int cp, head;   // token within the tile (the last one for columns past it), query head
    bool valid;
  };
  auto column = [&](int qc, int c) -> Column {
    const int col = (wave * QC + qc) * 16 + c;
    const int cp = pl.by_group.div(col);
    const int cu = min(cp, tokens - 1);
    return Column{cu, col - cp * G, cp == cu};
  };
  int tcol[QC];
  bf16x8 qB[QC][KK];
#pragma unroll
  for (int qc = 0; qc < QC; ++qc) {
    const Column x = column(qc, c16);
    tcol[qc] = x.valid ? t0 + x.cp : -1;
    const unsigned char* qrow = (const unsigned char*)a.q + (row0 + x.cp) * a.q_stride +
                                (int64_t)(g * G + x.head) * ROWB + 16 * j4;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const u32x4 w = *(const u32x4*)(qrow + 64 * kk);
      qB[qc][kk] = __builtin_bit_cast(bf16x8, x.valid ? w : u32x4{0u, 0u, 0u, 0u});
    }
  }
  fetch();
  if (nsteps > 0) convert(0);
  gone <<= 2;
  if (nsteps > 1) load();
  fetch();

  // LDS byte addresses of this lane's reads in stage 0 (tile_addresses; the V tile is TILE on).
  uint32_t ra[2], va[4];
  {
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    tile_addresses<D>(base, c16, j4, ra, va);
  }

  // The wave's own range of steps [wlo, whi] (its columns' positions tw_lo .. tw_hi), and the
  // run [ua, ub) of them whose keys all lie in every column's support (a(t) never decreases).
  const int w_first = pl.by_group.div(wave * 16 * QC);
  const int tw_lo = t0 + min(w_first, tokens - 1);
  const int tw_hi = t0 + min(pl.by_group.div(wave * 16 * QC + 16 * QC - 1), tokens - 1);
  const int wlo = w_first < tokens ? max(0, (sh.support_lo(tw_lo) >> 5) - s_first) : nsteps;
  const int whi = min(nsteps - 1, (tw_hi >> 5) - s_first);
  const int ua = ((sh.support_lo(tw_hi) + 31) >> 5) - s_first;
  const int ub = ((tw_lo + 1) >> 5) - s_first;

  // m starts at a finite floor below any score, so that a column whose keys are all masked so
  // far gets exp2(-inf - m) = 0 without a separate test; its first real maximum always moves m.
  // Columns past the tile's tokens score 0 against a reference of 0: they never move it.
  float m[QC], lsum[QC];
  f32x4 acc[QC][NB];
#pragma unroll
  for (int qc = 0; qc < QC; ++qc) {
    m[qc] = tcol[qc] >= 0 ? kNoScore : 0.0f;
    lsum[qc] = 0.0f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[qc][nb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  const float sc = a.scale_log2;
  bool odd = false;   // a masked step held an infinity or NaN

  // Begins step st: its tiles are whole (every wave has converted its rows of them, a step ago) and every
  // wave is done with step st - 1, whose stage step st + 1's rows take.
  auto begin_step = [&](int st) -> uint32_t {
    lds_barrier();
    return (uint32_t)((st & 1) * L::STAGE);
  };
  // The loads of step st + 2's rows.
  auto next_rows = [&](int st) {
    gone <<= 2;
    if (st + 2 < nsteps) load();
    fetch();
  };

  auto step = [&](int st, uint32_t sb, uint32_t dropped, bool masked) {
    f32x4 s0[QC], s1[QC];
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
      s0[qc] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      s1[qc] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    __builtin_amdgcn_s_setprio(kScorePriority);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const auto* kp = lds0 + ra[kk & 1] + sb + kTileLine * (kk >> 1);
      const bf16x8 ka = *(const __attribute__((address_space(3))) bf16x8*)(kp);
      const bf16x8 kb = *(const __attribute__((address_space(3))) bf16x8*)(kp + L::TILE / 2);
#pragma unroll
      for (int qc = 0; qc < QC; ++qc) {
        s0[qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qB[qc][kk], s0[qc], 0, 0, 0);
        s1[qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, qB[qc][kk], s1[qc], 0, 0, 0);
      }
    }
    // (step st + 1's rows, always: those of a step past the last go where nothing reads them, and without a
    // branch the conversions run under the products)
    convert((st + 1) & 1);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(kNoPriority);
    next_rows(st);
    __builtin_amdgcn_sched_barrier(0);
    // Element e of s0 is key k0 + 4 j4 + e of the lane's column, of s1 key k0 + 16 + 4 j4 + e.
    const int k0 = (s_first + st) * 32 + 4 * j4;
    if (masked) {
#pragma unroll
      for (int qc = 0; qc < QC; ++qc) {
        const int lo = sh.support_lo(tcol[qc]) - k0, hi = tcol[qc] - k0;   // (taken anew: registers)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s0[qc][e] = e >= lo && e <= hi && !(dropped & 1u) ? s0[qc][e] : kNegInf;
          s1[qc][e] = e + 16 >= lo && e + 16 <= hi && !(dropped & 2u) ? s1[qc][e] : kNegInf;
        }
      }
    }
    // The online softmax of the bf16 kernel: weights rounded to bf16 for the value products, as there (at most
    // 2^-8 of each: outputs are off by 2.3e-3 of their size, 1.7e-3 with the output's own rounding alone), their
    // sums in 32 bits.  A second value product with what the rounding leaves takes that error away and costs more
    // than memory or the chain of a step hide: five chunks 1344 -> 1892 us, four under a window of 4096 733 -> 1001,
    // D 64 273 -> 341, two short chunks beside 128 single tokens 202 -> 224.
    bf16x8 pB[QC];
    float ps[QC];
    auto weights = [&]() {
      bool over = false;
#pragma unroll
      for (int qc = 0; qc < QC; ++qc) {
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float pe =
              fast_exp2(__builtin_fmaf(e < 4 ? s0[qc][e] : s1[qc][e - 4], sc, -m[qc]));
          sum += pe;
          pB[qc][e] = (__bf16)pe;
        }
        ps[qc] = sum;
        over |= !(sum <= kWeightCap);
      }
      return over;
    };
    auto column_max = [&](int qc) {
      float mx = kNegInf;
#pragma unroll
      for (int e = 0; e < 8; ++e) mx = fmaxf(mx, e < 4 ? s0[qc][e] : s1[qc][e - 4]);
      return max_xor16_32(mx) * sc;
    };
    if (st == wlo) {
#pragma unroll
      for (int qc = 0; qc < QC; ++qc) m[qc] = fmaxf(m[qc], column_max(qc));
    }
    if (__builtin_amdgcn_ballot_w64(weights()) != 0) {
#pragma unroll
      for (int qc = 0; qc < QC; ++qc) {
        const float cand = column_max(qc);
        const bool grow = cand > m[qc] && max_xor16_32(ps[qc]) > kWeightCap;
        const float alpha = grow ? fast_exp2(m[qc] - cand) : 1.0f;
        m[qc] = grow ? cand : m[qc];
        lsum[qc] *= alpha;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[qc][nb] *= alpha;
      }
      weights();
    }
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) lsum[qc] += ps[qc];
    __builtin_amdgcn_s_setprio(kValuePriority);
    // 32 channels' values at a time, the next 32's on their way (five chunks 1366 us; 64 at a time, none on
    // their way, 1383; all at once, or the first ones' reads under the weights, spills into every step: 1429
    // and 1774)
    u32x2 vr[2][4];
    read_part<D, L::TILE, 0>(vr[0], va, sb);
    auto values_of = [&](auto part) {
      constexpr int H = decltype(part)::value;
      if constexpr (H + 1 < D / 32) read_part<D, L::TILE, H + 1>(vr[(H + 1) & 1], va, sb);
      u32x2 (&v)[4] = vr[H & 1];
      wait_part<H + 1 < D / 32 ? 4 : 0>(v);
      if (masked && __builtin_amdgcn_ballot_w64(any_special(v)) != 0) {
        odd = true;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) v[i][e] &= ~special_halves(v[i][e]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bf16x8 vt = join_chunks(v[2 * i], v[2 * i + 1]);
#pragma unroll
        for (int qc = 0; qc < QC; ++qc)
          acc[qc][2 * H + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pB[qc], acc[qc][2 * H + i], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    values_of(std::integral_constant<int, 0>{});
    values_of(std::integral_constant<int, 1>{});
    if constexpr (D == 128) {
      values_of(std::integral_constant<int, 2>{});
      values_of(std::integral_constant<int, 3>{});
    }
    __builtin_amdgcn_s_setprio(kNoPriority);
  };

  // (after next_rows(st), gone ends with the bits of step st + 2; before it, of step st + 1)
  int st = 0;
  for (; st < wlo && st < nsteps; ++st) begin_step(st), convert((st + 1) & 1), next_rows(st);
  for (; st <= whi; ++st) {
    const uint32_t sb = begin_step(st);
    const uint32_t dropped = (gone >> 2) & 3u;
    step(st, sb, dropped, st < ua || st >= ub || dropped != 0);
  }
  for (; st < nsteps; ++st) begin_step(st), convert((st + 1) & 1), next_rows(st);

  if (odd) {
    // The infinities and NaN of masked steps, straight from the pages: their weights are positive,
    // so each enters the columns that see its key as it is.
    for (st = wlo; st <= whi; ++st) {
      const int first = (s_first + st) * 32;
      const int e0 = sh.by_page.div(first), e1 = sh.by_page.div(first + 16);
      const bool whole = e1 < sh.width && sh.is_page(scalar_word(table, e0)) &&
                         sh.is_page(scalar_word(table, min(e1, sh.width - 1)));
      if (st >= ua && st < ub && whole) continue;
      for (int key = first; key < first + 32; ++key) {
        const int i = sh.by_page.div(key);
        const int id = i < sh.width ? scalar_word(table, min(i, sh.width - 1)) : -1;
        if (!sh.is_page(id)) continue;
        const uint64_t at = ((uint64_t)(uint32_t)id * (uint32_t)a.hkv + (uint32_t)g) * (uint32_t)sh.page_size +
                            (uint32_t)(key - i * sh.page_size);
        const float unit = __uint_as_float((uint32_t)a8.v_scales[at] << 23);
        const unsigned char* row = (const unsigned char*)a.v_pages + at * D + 4 * j4;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const uint32_t c = *(const uint32_t*)(row + 16 * nb);
          const uint32_t v[2] = {values2<false>(c, unit), values2<true>(c, unit)};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t x = e & 1 ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16;
            const float add = (x & 0x7F800000u) == 0x7F800000u ? __uint_as_float(x) : 0.0f;
#pragma unroll
            for (int qc = 0; qc < QC; ++qc)
              acc[qc][nb][e] += key >= sh.support_lo(tcol[qc]) && key <= tcol[qc] ? add : 0.0f;
          }
        }
      }
    }
  }

  // Output of a column: o = acc / l (bf16 RNE), lse = (m + log2 l) * ln 2.
#pragma unroll
  for (int qc = 0; qc < QC; ++qc) {
    lsum[qc] = sum_xor16_32(lsum[qc]);
    if (__builtin_expect(lsum[qc] == 0.0f, 0) &&
        any_page(sh, table, max(sh.support_lo(tcol[qc]), s_first * 32), min(tcol[qc], (s_first + nsteps) * 32 - 1)))
      m[qc] = kNoWeight;
  }
  if (it.ways == 1) {
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
      const float l = lsum[qc];
      const float inv = inverse_sum(m[qc], l);
      u32x4 w[NB / 2];
#pragma unroll
      for (int i = 0; i < NB / 2; ++i) w[i] = pair_blocks(acc[qc][2 * i], acc[qc][2 * i + 1], inv);
      const Column x = column(qc, c16);
      if (x.valid) {
        unsigned char* orow = (unsigned char*)a.out +
                              ((row0 + x.cp) * a.hq + (int64_t)(g * G + x.head)) * ROWB;
#pragma unroll
        for (int i = 0; i < NB / 2; ++i)
          *(u32x4*)(orow + 64 * i + 32 * (j4 & 1) + 16 * (j4 >> 1)) = w[i];
        if (a.lse != nullptr && j4 == 0)
          a.lse[(int64_t)(g * G + x.head) * a.n + row0 + x.cp] = log_partition(m[qc], l);
      }
    }
    return;
  }

  // A cut walk leaves the piece's state for the merge launch; the tile's states lie together.
  constexpr size_t STATE = paged_state_bytes(kPagedCols, D) / 4;
  float* const part =
      a.states + ((size_t)it.slot * a.hkv + (size_t)g * it.ways + it.piece) * STATE;
#pragma unroll
  for (int qc = 0; qc < QC; ++qc) {
    const float l = lsum[qc];
    const int col = (wave * QC + qc) * 16 + c16;
    if (col < cols) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) *(f32x4*)(part + col * D + 16 * nb + 4 * j4) = acc[qc][nb];
      if (j4 == 0) *(float2*)(part + kPagedCols * D + 2 * col) = make_float2(m[qc], l);
    }
  }
}

// Calls of at most 16 columns per sequence, and all that they need: the last piece of a cut walk to end
// merges them.  Workgroup i runs on compute die i mod 8, so an item's KV heads go to one die, one after the
// other: the scale bytes of a short page under all its heads share lines, which each die that reads one
// fetches by itself (192 tokens over up to 32768 in pages of 16: 1060 us, 1073 with a head to a die, where a
// request in eleven was for scale bytes; 256 over up to 2000: 106 and 112).
constexpr int kDies = 8;
template <int D>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(3)))
void coded_narrow_kernel(CodedArgs a8) {
  __shared__ __align__(1024) unsigned char smem[Narrow<D>::LDS];
  const PagedArgs& a = a8.p;
  const int lane = threadIdx.x & 63;
  const int turn = (int)(blockIdx.x / kDies), eight = a.plan.by_hkv.div(turn);
  const int item = eight * kDies + (int)(blockIdx.x % kDies);
  const int g = turn - eight * a.hkv;
  PagedItem it;
  if (!find_item<false>(a, item, lane, it)) return;
  narrow_walk<D, true>(a8, it, g, smem);
}

template <int D, int OCC>
hipError_t attention_t(const CodedArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)(a.p.plan.items() * a.p.hkv));
  if (a.p.plan.narrow) {
    const int64_t eights = (a.p.plan.items() + kDies - 1) / kDies;
    hipLaunchKernelGGL((coded_narrow_kernel<D>), dim3((unsigned)(eights * kDies * a.p.hkv)), dim3(kWaves * 64), 0,
                       stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((coded_kernel<D, OCC>), grid, dim3(kWaves * 64), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.p.plan.pieces == 0) return e;
  return launch_paged_merge<uint16_t, D, kPagedCols>(a.p, stream);
}

}  // namespace

hipError_t launch_coded_attention(const CodedArgs& a, int32_t head_dim, hipStream_t stream) {
  return head_dim == 64 ? attention_t<64, 4>(a, stream) : attention_t<128, 3>(a, stream);
}

}  // namespace pbb
