// bf16 attention over a paged KV cache on gfx950 (MI355X): chunks of new tokens, or single ones.
//
// A target at position t attends with one softmax over its support {a(t) .. t} (a(t) = 0, or that of
// the PBB or sliding-window layer), whose keys lie in pages of 16 n rows that a table names.
//
// Work unit: a tile of TQ = floor(128 / G) consecutive tokens of one sequence with the G query heads
// of a KV head, up to 128 query columns, position-major, head-minor; 32 columns per wave in two
// groups of 16.  The keys of the tile's walk stream through LDS in 32-key steps by LDS DMA, each
// loaded once per workgroup: wave w loads 16 rows of K or V, which lie in one page, so a step costs a
// wave one table entry, read through the scalar cache a step ahead.  S^T = K Q^T and O^T += V^T P^T on
// v_mfma_f32_16x16x32_bf16, with an online softmax whose reference moves lazily, as in the prefill.
// Long walks are cut into pieces (PagedPlan), which leave partial states (Eq.(lse)); a second launch
// merges those of wide tiles, the last piece to end those of single tokens.  Sequences of few columns go
// through narrow_walk, in the same launch.
//
// Bound: with many columns the matrix and vector work of a step at the clock that the card's power
// allows (16384 tokens, 32/8 heads, d 128: 1872 to 2240 us over the cards measured, 980 to 1175
// TFLOP/s, matrix cores 0.51 busy at 1.9 GHz); with few columns HBM (192 single tokens at up to 32768:
// 1876 us, 6.7 TB/s).
//
// Masks.  Steps with a key outside some column's support set its scores to -inf.  What such keys hold
// is unknown (rows never written, dropped pages), and 0 * inf or 0 * NaN would reach the products, so
// masked steps look whether any value that they read is infinite or NaN, and if so clear those; after
// the walk, a wave that met one adds them to the columns that see their keys (handling them on the
// spot costs registers that every step needs).

#include <type_traits>

#include "pbb_paged_device.h"

namespace pbb {
namespace {

constexpr int kPagedWaves = 4;
constexpr int kPagedGroups = 2;
static_assert(kPagedCols == 16 * kPagedGroups * kPagedWaves && kPagedStep == 32, "tile");
// LDS stages and waves per SIMD that the registers are budgeted for (see the prefill).
constexpr int kPagedStages128 = 3, kPagedOcc128 = 3;
constexpr int kPagedStages64 = 4, kPagedOcc64 = 4;

// Few columns: tiles of at most 16 (single tokens, short drafts).  The 16-key halves of the piece's
// steps are dealt to the waves one by one, each with LDS tiles of its own, so that nothing but the
// merge of the waves at the end waits for another wave.  A wave has three 16-row tiles: while it works
// on one, the two after it (K and V rows alternate) are in flight; a tile is loaded over as soon as it
// has been read.  The value products contract 16 keys with both parts of their weights.
// Bound: HBM, with 12 waves per CU, 8 KiB of each in flight.  (32-key steps with two buffers per wave
// take 64 KiB for two waves: 256 single tokens of up to 600 71 us, 67 so.)
template <int D>
constexpr int narrow_lds() { return kPagedWaves * 3 * 16 * D * 2; }

template <int D, bool IN_PLACE>
__device__ __forceinline__ void narrow_walk(const PagedArgs& a, const PagedItem& it, int g,
                                            unsigned char* smem) {
  constexpr int NW = kPagedWaves;
  constexpr int KK = D / 32;
  constexpr int NB = D / 16;
  constexpr int ROWB = D * 2;
  constexpr int TILE = 16 * ROWB;       // 16 rows of K or V
  constexpr int OPS = TILE / 1024;      // DMA instructions of a tile
  constexpr int COLS = kPagedNarrowCols;
  static_assert(NarrowOut<uint16_t, D, NW>::LDS <= narrow_lds<D>(), "the waves' states fit their tiles");

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

  // This lane's column (past the tile's: the last token's row, a zero query, no key seen).
  const int cp = min(pl.by_group.div(c16), tokens - 1);
  const bool valid = c16 < cols;
  const int tcol = valid ? t0 + cp : -1;
  const int lo_c = sh.support_lo(t0 + cp);
  bf16x8 qB[KK];
  {
    const unsigned char* qrow = (const unsigned char*)a.q + (row0 + cp) * a.q_stride +
                                (int64_t)(g * G + (valid ? c16 - cp * G : 0)) * ROWB + 16 * j4;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qB[kk] = *(const bf16x8*)(qrow + 64 * kk);
  }

  // A half's page entry through the scalar cache, a half before its loads.
  const int32_t* const table = a.table + (size_t)it.b * sh.width;
  const uint32_t page_bytes = (uint32_t)sh.page_size * ROWB;   // of one KV head
  const uint64_t page_stride = (uint64_t)page_bytes * (uint32_t)a.hkv;
  const unsigned char* const keys = (const unsigned char*)a.k_pages + (uint64_t)page_bytes * (uint32_t)g;
  const unsigned char* const values = (const unsigned char*)a.v_pages + (uint64_t)page_bytes * (uint32_t)g;
  struct Entry { int id; uint32_t slot; };
  auto fetch = [&](int h) -> Entry {   // (halves past the walk read the last entry, for nothing)
    const int i = min(sh.by_page.div(16 * h), sh.width - 1);
    return Entry{scalar_word(table, i), (uint32_t)(16 * h - i * sh.page_size) * ROWB};
  };
  auto offset = [&](const Entry& e) -> uint64_t {
    return (sh.is_page(e.id) ? (uint32_t)e.id : 0u) * page_stride + e.slot;
  };
  uint32_t doff[kDmaBlocks<D>];
  dma_offsets<D>(lane, ROWB, doff);
  unsigned char* const wbuf = smem + wave * 3 * TILE;
  auto load = [&](const unsigned char* src, int tile) {   // (non-temporal: read once in a call)
#pragma unroll
    for (int y = 0; y < OPS; ++y)
      __builtin_amdgcn_global_load_lds(
          (const void*)((y < kDmaBlocks<D> ? src : src + 8 * ROWB) + doff[y % kDmaBlocks<D>]),
          (__attribute__((address_space(3))) void*)(wbuf + tile + 1024 * y), 16, 0, kCachePolicyNT);
  };
  int h = h0 + wave;
  bool gone = false, next_gone = false;   // the half's, and the next one's, keys have no page
  uint64_t next_off = 0;
  Entry after = {0, 0};
  if (h < h1) {
    const Entry e0 = fetch(h), e1 = fetch(min(h + NW, h1 - 1));
    after = fetch(min(h + 2 * NW, h1 - 1));
    gone = !sh.is_page(e0.id);
    next_gone = !sh.is_page(e1.id);
    next_off = offset(e1);
    load(keys + offset(e0), 0);
    load(values + offset(e0), TILE);
    if (h + NW < h1) load(keys + next_off, 2 * TILE);
  }

  uint32_t ra[2], va[4];
  {
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)wbuf;
    tile_addresses<D>(base, c16, j4, ra, va);
  }
  const __attribute__((address_space(3))) unsigned char* lds0 = nullptr;
  // the run [ua, ub) of halves whose keys all lie in every column's support
  const int ua = (sh.support_lo(t_last) + 15) >> 4;
  const int ub = (t0 + 1) >> 4;

  float m = valid ? kNoScore : 0.0f, lsum = 0.0f;
  f32x4 acc[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) acc[nb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int kk = 0; kk < KK; ++kk)
    qB[kk] = __builtin_bit_cast(bf16x8, valid ? __builtin_bit_cast(u32x4, qB[kk]) : u32x4{0u, 0u, 0u, 0u});
  const float sc = a.scale_log2;
  bool odd = false;

  int kt = 0, vt = TILE, nt = 2 * TILE;   // tiles of this half's keys and values, of the next one's keys
  for (; h < h1; h += NW) {
    const int more = h + NW < h1 ? (h + 2 * NW < h1 ? 2 : 1) : 0;   // halves after this one (2: or more)
    // its keys have landed: its values and the next half's keys may be outstanding
    wait_groups<2, OPS>(more > 0 ? 2 : 1);
    __builtin_amdgcn_sched_barrier(0);
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    bf16x8 ka[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      ka[kk] = *(const __attribute__((address_space(3))) bf16x8*)(lds0 + ra[kk & 1] + kt +
                                                                   kTileLine * (kk >> 1));
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[kk], qB[kk], s, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    // (the keys have been read: the next half's values go over them)
    if (more > 0) load(values + next_off, kt);
    const bool masked = h < ua || h >= ub || gone;
    if (masked) {
      const int k0 = 16 * h + 4 * j4;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s[e] = e >= lo_c - k0 && e <= tcol - k0 && !gone ? s[e] : kNegInf;
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
      const bool grow = cand > m && max_xor16_32(ps) > kWeightCap;
      const float alpha = grow ? fast_exp2(m - cand) : 1.0f;
      m = grow ? cand : m;
      lsum *= alpha;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) acc[nb] *= alpha;
      weights();
    }
    lsum += ps;
    // The weights as two bf16 parts, the upper one cut off, the lower one rounded: 2^-15 of a weight is
    // lost.  One product contracts both with the same values, since 16 keys would fill half of its 32
    // slots; so it costs no more than weights rounded to one bf16 each would (192 single tokens 1878 us,
    // 1877 so; one token over 3000 9.9, 9.7; error against fp64 1.66e-3, the output's rounding, 2.34e-3
    // so).  No part of a weight above 0 is 0 or less, so that an infinite value stays one.
    u32x2 high, low;
    float rest[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      rest[e] = fmaxf(p[e] - __uint_as_float(__float_as_uint(p[e]) & 0xFFFF0000u), p[e] * 0x1p-24f);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      high[e] = __builtin_amdgcn_perm(__float_as_uint(p[2 * e + 1]), __float_as_uint(p[2 * e]), 0x07060302u);
      low[e] = pack_bf16(rest[2 * e], rest[2 * e + 1]);
    }
    const bf16x8 weight = join_chunks(high, low);
    // its values have landed: the next half's keys and values may be outstanding
    wait_groups<2, OPS>(more > 0 ? 2 : 0);
    __builtin_amdgcn_sched_barrier(0);
    u32x2 vr[NB];
    read_tile<D>(vr, va, (uint32_t)vt);
    wait_tile<D>(vr);
    if (masked && __builtin_amdgcn_ballot_w64(any_special(vr)) != 0) {
      odd = true;
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) vr[i][e] &= ~special_halves(vr[i][e]);
    }
    __builtin_amdgcn_sched_barrier(0);
    // (the values have been read: the keys of the half after next go over them)
    gone = next_gone;
    next_gone = !sh.is_page(after.id);
    next_off = offset(after);
    if (more > 1) load(keys + next_off, vt);
    after = fetch(min(h + 3 * NW, h1 - 1));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      acc[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join_chunks(vr[nb], vr[nb]), weight, acc[nb], 0, 0, 0);
    const int t = kt;
    kt = nt;
    nt = vt;
    vt = t;
  }
  if (odd) {   // (see paged_bf16_kernel)
    for (h = h0 + wave; h < h1; h += NW) {
      const Entry e = fetch(h);
      if (!sh.is_page(e.id) || (h >= ua && h < ub)) continue;
      const unsigned char* row = values + offset(e) + 8 * j4;
      for (int key = 16 * h; key < 16 * h + 16; ++key, row += ROWB) {
        const bool sees = key >= lo_c && key <= tcol;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const u32x2 w = *(const u32x2*)(row + 32 * nb);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t x = e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16;
            acc[nb][e] += sees && (x & 0x7F800000u) == 0x7F800000u ? __uint_as_float(x) : 0.0f;
          }
        }
      }
    }
  }

  lsum = sum_xor16_32(lsum);
  __syncthreads();   // every wave is done with its tiles
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
    *(f32x4*)(result.outputs(smem) + (wave * COLS + c16) * D + 16 * nb + 4 * j4) = acc[nb];
  if (j4 == 0) {
    result.references(smem)[wave * COLS + c16] = m;
    result.sums(smem)[wave * COLS + c16] = lsum;
  }
  result.template finish<IN_PLACE, IN_PLACE ? COLS : kPagedCols>(tid, smem, 16 * h0, 16 * h1 - 1);
}

template <int D, int ST, int OCC>
__global__ __launch_bounds__(kPagedWaves * 64) __attribute__((amdgpu_waves_per_eu(OCC)))
void paged_bf16_kernel(PagedArgs a) {
  constexpr int NW = kPagedWaves;
  constexpr int QC = kPagedGroups;
  constexpr int KK = D / 32;            // 32-channel slices of the score contraction
  constexpr int NB = D / 16;            // 16-channel blocks of the output
  constexpr int ROWB = D * 2;           // bytes of one K or V row
  constexpr int HALF = 16 * ROWB;       // 16 rows of a tile
  constexpr int TILE = 2 * HALF;
  constexpr int BUF = 2 * TILE;         // K tile, then V tile
  constexpr int STAGES = ST;
  static_assert(STAGES >= 3, "stages");
  static_assert(NW == 4, "one (tensor, 16-row half) of a step per wave");
  __shared__ __align__(1024) unsigned char smem[STAGES * BUF];

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
    static_assert(narrow_lds<D>() <= STAGES * BUF, "LDS");
    narrow_walk<D, false>(a, it, g, smem);
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
  int tcol[QC], lo_c[QC];
  bf16x8 qB[QC][KK];
#pragma unroll
  for (int qc = 0; qc < QC; ++qc) {
    const Column x = column(qc, c16);
    tcol[qc] = x.valid ? t0 + x.cp : -1;
    lo_c[qc] = sh.support_lo(t0 + x.cp);
    const unsigned char* qrow = (const unsigned char*)a.q + (row0 + x.cp) * a.q_stride +
                                (int64_t)(g * G + x.head) * ROWB + 16 * j4;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qB[qc][kk] = *(const bf16x8*)(qrow + 64 * kk);
  }

  // DMA of a step: wave w loads 16 rows (half w & 1) of K (w < 2) or V from the page that holds
  // them.  An entry that names no page reads page 0, and the half's keys are masked (`gone`, two
  // bits per step, the youngest lowest).
  const unsigned char* const pool = (const unsigned char*)(wave >= 2 ? a.v_pages : a.k_pages);
  const int32_t* const table = a.table + (size_t)it.b * sh.width;
  const uint32_t page_bytes = (uint32_t)sh.page_size * ROWB;   // of one KV head
  const uint64_t page_stride = (uint64_t)page_bytes * (uint32_t)a.hkv;
  const unsigned char* const heads = pool + (uint64_t)page_bytes * (uint32_t)g;
  int next_key = s_first * 32;   // first key of the step to be issued next
  int id0 = 0, id1 = 0;          // its entries (the two halves')
  bool past = false;             // the second half lies past the table
  uint32_t slot_b = 0;           // bytes from its page to this wave's half
  auto fetch = [&]() {
    const int i0 = sh.by_page.div(next_key), i1 = sh.by_page.div(next_key + 16);
    id0 = scalar_word(table, min(i0, sh.width - 1));
    id1 = scalar_word(table, min(i1, sh.width - 1));
    past = i1 >= sh.width;
    const int i = (wave & 1) ? i1 : i0;
    slot_b = (uint32_t)(next_key + 16 * (wave & 1) - i * sh.page_size) * ROWB;
  };
  uint32_t gone = 0;
  uint32_t doff[kDmaBlocks<D>];
  dma_offsets<D>(lane, ROWB, doff);
  auto issue = [&](int stage) {   // the next step
    const bool ok0 = sh.is_page(id0), ok1 = sh.is_page(id1) && !past;
    gone |= (ok0 ? 0u : 1u) | (ok1 ? 0u : 2u);
    const uint32_t id0s = ok0 ? (uint32_t)id0 : 0u, id1s = ok1 ? (uint32_t)id1 : 0u;
    const uint32_t id = (wave & 1) ? id1s : id0s;
    const unsigned char* src = heads + id * page_stride + slot_b;
    unsigned char* lds = smem + stage * BUF + wave * HALF;
#pragma unroll
    for (int y = 0; y < 2 * kDmaBlocks<D>; ++y)
      dma16(y < kDmaBlocks<D> ? src : src + 8 * ROWB, doff[y % kDmaBlocks<D>], lds + 1024 * y);
    next_key += 32;
  };
  fetch();

  // Steps 0 .. STAGES-2 go out first; step st then issues step st + STAGES - 1.
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) {
    gone <<= 2;
    if (s < nsteps) issue(s);
    fetch();
  }

  // LDS byte addresses of this lane's reads in stage 0 (tile_addresses; the V tile is TILE on).
  uint32_t ra[2], va[4];
  {
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    tile_addresses<D>(base, c16, j4, ra, va);
  }
  const __attribute__((address_space(3))) unsigned char* lds0 = nullptr;

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
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      qB[qc][kk] = __builtin_bit_cast(
          bf16x8, tcol[qc] >= 0 ? __builtin_bit_cast(u32x4, qB[qc][kk]) : u32x4{0u, 0u, 0u, 0u});
  }
  const float sc = a.scale_log2;

  bool odd = false;   // a masked step held an infinity or NaN
  int rstage = 0;
  constexpr int OPS = D / 32;           // DMA instructions of a wave per step

  // Begins step st: its tiles have landed; returns the stage offset.
  auto begin_step = [&](int st) -> uint32_t {
    // This wave's loads of step st have landed once at most the loads of the steps issued
    // after it (up to STAGES - 2) are outstanding; the barrier then covers every wave's loads,
    // and every wave is done with step st-1, whose stage the loads of step st+STAGES-1 reuse.
    wait_groups<STAGES - 2, OPS>(min(STAGES - 2, nsteps - 1 - st));
    lds_barrier();
    gone <<= 2;
    if (st + STAGES - 1 < nsteps) issue(rstage == 0 ? STAGES - 1 : rstage - 1);
    __builtin_amdgcn_sched_barrier(0);
    const uint32_t sb = (uint32_t)(rstage * BUF);
    rstage = rstage == STAGES - 1 ? 0 : rstage + 1;
    return sb;
  };

  auto step = [&](int st, uint32_t sb, uint32_t dropped, bool masked) {
    f32x4 s0[QC], s1[QC];
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
      s0[qc] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      s1[qc] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const auto* kp = lds0 + ra[kk & 1] + sb + kTileLine * (kk >> 1);
      const bf16x8 ka = *(const __attribute__((address_space(3))) bf16x8*)(kp);
      const bf16x8 kb = *(const __attribute__((address_space(3))) bf16x8*)(kp + HALF);
#pragma unroll
      for (int qc = 0; qc < QC; ++qc) {
        s0[qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qB[qc][kk], s0[qc], 0, 0, 0);
        s1[qc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, qB[qc][kk], s1[qc], 0, 0, 0);
      }
    }
    // The next step's entries, here so that no wait for LDS reads waits for them too.
    __builtin_amdgcn_sched_barrier(0);
    fetch();
    __builtin_amdgcn_sched_barrier(0);
    // Element e of s0 is key k0 + 4 j4 + e of the lane's column, of s1 key k0 + 16 + 4 j4 + e.
    const int k0 = (s_first + st) * 32 + 4 * j4;
    auto seen = [&](int qc, int e) -> bool {   // element e: 0..3 of s0, 4..7 of s1
      const int k = e < 4 ? e : e + 12;
      return k >= lo_c[qc] - k0 && k <= tcol[qc] - k0 && !(dropped & (e < 4 ? 1u : 2u));
    };
    if (masked) {
#pragma unroll
      for (int qc = 0; qc < QC; ++qc)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s0[qc][e] = seen(qc, e) ? s0[qc][e] : kNegInf;
          s1[qc][e] = seen(qc, 4 + e) ? s1[qc][e] : kNegInf;
        }
    }
    // Online softmax in log2 units with a lazily moved reference m (the log-sum-exp rescaling
    // of Eq.(lse)): the weights are taken against the current m, and m moves to the column
    // maxima (the accumulators rescaled, the weights taken again) only in a step where the
    // eight weights of some lane and column sum above 2^8 or to infinity.
    // The weights enter the products rounded to bf16, the sum in 32 bits: products of what the rounding
    // leaves would be half as much matrix work again and 10 more spilled registers (chunks 4.5 ms instead
    // of 2.65, a 16384-token prompt 2.94 instead of 1.89; error against fp64 1.66e-3 instead of 2.34e-3).
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
    // The wave's first step sets the reference before its weights (it would always move it);
    // its sums and accumulators are still zero.
    if (st == wlo) {
#pragma unroll
      for (int qc = 0; qc < QC; ++qc) m[qc] = fmaxf(m[qc], column_max(qc));
    }
    // V^T operand of O^T += V^T P^T: lane (c16, j4) needs channel 16nb + c16 of keys
    // 4j4..4j4+3 and 16+4j4..16+4j4+3 (the key order of P^T in the score layout): one transposed
    // read per half.
    u32x2 vr[2 * NB];
    if (__builtin_amdgcn_ballot_w64(weights()) != 0) {
#pragma unroll
      for (int qc = 0; qc < QC; ++qc) {
        const float cand = column_max(qc);
        // (only the columns whose own weights ask for it: none depends on its neighbours' data)
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
    read_chunks<D, TILE>(vr, va, sb);
    wait_chunks<D>(vr);
    if (masked && __builtin_amdgcn_ballot_w64(any_special(vr)) != 0) {
      odd = true;
#pragma unroll
      for (int i = 0; i < 2 * NB; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) vr[i][e] &= ~special_halves(vr[i][e]);
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const bf16x8 vt = join_chunks(vr[2 * nb], vr[2 * nb + 1]);
#pragma unroll
      for (int qc = 0; qc < QC; ++qc)
        acc[qc][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pB[qc], acc[qc][nb], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  int st = 0;
  for (; st < wlo && st < nsteps; ++st) begin_step(st), fetch();
  for (; st <= whi; ++st) {
    const uint32_t sb = begin_step(st);
    const uint32_t dropped = (gone >> (2 * (STAGES - 1))) & 3u;
    step(st, sb, dropped, st < ua || st >= ub || dropped != 0);
  }
  for (; st < nsteps; ++st) begin_step(st), fetch();

  if (odd) {
    // The infinities and NaN of masked steps, straight from the pages: their weights are positive,
    // so each enters the columns that see its key as it is.
    const unsigned char* const values = (const unsigned char*)a.v_pages + (uint64_t)page_bytes * (uint32_t)g;
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
        const unsigned char* row = values + (uint32_t)id * page_stride +
                                   (uint32_t)(key - i * sh.page_size) * ROWB + 8 * j4;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const u32x2 w = *(const u32x2*)(row + 32 * nb);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t h = e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16;
            const float add = (h & 0x7F800000u) == 0x7F800000u ? __uint_as_float(h) : 0.0f;
#pragma unroll
            for (int qc = 0; qc < QC; ++qc)
              acc[qc][nb][e] += key >= lo_c[qc] && key <= tcol[qc] ? add : 0.0f;
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
        any_page(sh, table, max(lo_c[qc], s_first * 32), min(tcol[qc], (s_first + nsteps) * 32 - 1)))
      m[qc] = kNoWeight;
  }
  if (it.ways == 1) {
#pragma unroll
    for (int qc = 0; qc < QC; ++qc) {
      const float l = lsum[qc];
      const float inv = inverse_sum(m[qc], l);
      u32x4 w[NB / 2];
#pragma unroll
      for (int q = 0; q < NB / 2; ++q) w[q] = pair_blocks(acc[qc][2 * q], acc[qc][2 * q + 1], inv);
      const Column x = column(qc, c16);
      if (x.valid) {
        unsigned char* orow = (unsigned char*)a.out +
                              ((row0 + x.cp) * a.hq + (int64_t)(g * G + x.head)) * ROWB;
#pragma unroll
        for (int q = 0; q < NB / 2; ++q)
          *(u32x4*)(orow + 64 * q + 32 * (j4 & 1) + 16 * (j4 >> 1)) = w[q];
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

// Calls of at most 16 columns per sequence (single tokens, short drafts), and all that they need: the
// last piece of a cut walk to end merges them.
template <int D>
__global__ __launch_bounds__(kPagedWaves * 64) __attribute__((amdgpu_waves_per_eu(3)))
void paged_narrow_kernel(PagedArgs a) {
  __shared__ __align__(1024) unsigned char smem[narrow_lds<D>()];
  const int lane = threadIdx.x & 63;
  const int item = a.plan.by_hkv.div((int)blockIdx.x);
  const int g = (int)blockIdx.x - item * a.hkv;
  PagedItem it;
  if (!find_item<false>(a, item, lane, it)) return;
  narrow_walk<D, true>(a, it, g, smem);
}

// The summary of a call of many sequences (PlanWord), one workgroup: the steps and tiles of all of
// them, which say how walks are cut, then the running sums over rounds of 64, a round to a wave.  Sums
// stop at 2^30, above any item (see kMostItems).
constexpr int kPlanWaves = 16;
__global__ __launch_bounds__(kPlanWaves * 64) void paged_plan_kernel(PagedArgs a) {
  constexpr int KINDS = 2 * kPlanRows;
  __shared__ float sm_steps[kPlanWaves];
  __shared__ uint32_t sm_tiles[kPlanWaves];
  __shared__ uint32_t sm_round[2][kPlanWaves][KINDS];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const PagedPlan& p = a.plan;
  float sum = 0.0f;
  uint32_t count = 0;
  for (int b = tid; b < a.batch; b += kPlanWaves * 64) {
    const Chunk c = chunk_at(a, b);
    const uint32_t nt = (uint32_t)p.tiles_of(c);
    sum = __builtin_fmaf((float)nt, (float)p.steps_of(a.shape, c), sum);
    count = count + nt < kMostItems ? count + nt : kMostItems;
  }
  const float steps_w = wave_scan(sum);
  const uint32_t tiles_w = wave_scan(count);
  if (lane == 63) {
    sm_steps[wave] = steps_w;
    sm_tiles[wave] = tiles_w < kMostItems ? tiles_w : kMostItems;
  }
  __syncthreads();
  float steps = 0.0f;
  uint32_t tiles = 0;
  for (int w = 0; w < kPlanWaves; ++w) steps += sm_steps[w], tiles += sm_tiles[w];
  const float per_share = per_share_of(p, steps, tiles);

  const int rounds = paged_rounds(a.batch);
  uint32_t before = 0;   // lane k < KINDS: the sum of row k / 2, kind k mod 2, of the rounds before r0
  for (int r0 = 0, buf = 0; r0 < rounds; r0 += kPlanWaves, buf ^= 1) {
    const int r = r0 + wave;
    const Chunk c = r < rounds ? chunk_at(a, 64 * r + lane) : Chunk{0, 0, 0};
#pragma unroll
    for (int narrow = 0; narrow < 2; ++narrow) {
      const Share s = share_of_chunk(a, c, narrow != 0, per_share);
      const uint32_t items = wave_scan(s.items), cut = wave_scan(s.cut), slots = wave_scan(s.slots);
      if (lane == 63) {
        sm_round[buf][wave][2 * kRowItems + narrow] = items;
        sm_round[buf][wave][2 * kRowCut + narrow] = cut;
        sm_round[buf][wave][2 * kRowSlots + narrow] = slots;
      }
    }
    __syncthreads();   // (the other buffer is written after every wave has passed the next one)
    if (lane < KINDS) {
      uint32_t upto = before;
      for (int w = 0; w < kPlanWaves; ++w) {
        const uint32_t own = sm_round[buf][w][lane];
        const uint32_t end = upto + own < (1u << 30) ? upto + own : 1u << 30;
        if (w == wave && r < rounds)
          plan_row(a, lane >> 1, lane & 1)[r] = (lane >> 1) == kRowSlots ? upto : end;
        upto = end;
      }
      before = upto;
    }
  }
  // (uniform calls have one kind, counted under both: only the first is searched)
  if (wave == 0) {
    if (lane == 0) a.rounds[kPlanShare] = __float_as_uint(per_share);
    if (lane == 2 * kRowItems) a.rounds[kPlanItems] = before;
    if (lane == 2 * kRowSlots) a.rounds[kPlanSlots] = before;
    if (lane == 2 * kRowCut) a.rounds[kPlanCut] = before;
  }
}

}  // namespace

hipError_t launch_paged_plan(const PagedArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(kPlanWaves * 64), 0, stream, a);
  return hipGetLastError();
}

namespace {

template <int D, int ST, int OCC>
hipError_t launch_paged_t(const PagedArgs& a, hipStream_t stream) {
  if (a.plan.narrow) {
    hipLaunchKernelGGL((paged_narrow_kernel<D>), dim3((unsigned)(a.plan.items() * a.hkv)),
                       dim3(kPagedWaves * 64), 0, stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((paged_bf16_kernel<D, ST, OCC>), dim3((unsigned)(a.plan.items() * a.hkv)),
                     dim3(kPagedWaves * 64), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.plan.pieces == 0) return e;
  return launch_paged_merge<uint16_t, D, kPagedCols>(a, stream);
}

}  // namespace

hipError_t launch_paged_bf16(const PagedArgs& a, int32_t head_dim, hipStream_t stream) {
  return head_dim == 64 ? launch_paged_t<64, kPagedStages64, kPagedOcc64>(a, stream)
                        : launch_paged_t<128, kPagedStages128, kPagedOcc128>(a, stream);
}

}  // namespace pbb
