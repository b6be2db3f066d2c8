// Device-side helpers shared by the paged attention kernels: which work a workgroup does, page
// addresses, and the merge of cut walks.
#pragma once

#include <type_traits>

#include "pbb_device.h"
#include "pbb_paged_internal.h"

namespace pbb {

// read_chunks and wait_chunks of a 16-row tile: dst[nb] holds rows 4j4 .. +3 of channel 16nb + c16.
template <int D>
__device__ __forceinline__ void read_tile(u32x2 (&dst)[D / 16], const uint32_t (&ta)[4], uint32_t sb) {
#pragma unroll
  for (int x = 0; x < 4; ++x) dst[x] = tr_read<0>(ta[x] + sb);
  if constexpr (D == 128) {
#pragma unroll
    for (int x = 0; x < 4; ++x) dst[4 + x] = tr_read<kTileLine>(ta[x] + sb);
  }
}
template <int D>
__device__ __forceinline__ void wait_tile(u32x2 (&v)[D / 16]) {
  if constexpr (D == 128)
    asm volatile("s_waitcnt lgkmcnt(0)"
                 : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]), "+v"(v[4]), "+v"(v[5]),
                   "+v"(v[6]), "+v"(v[7]));
  else
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]));
}

typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;

// Whether one of the bf16 values of an operand is infinite or NaN.
template <int N>
__device__ __forceinline__ bool any_special(const u32x2 (&v)[N]) {
  u16x2 top = {0, 0};
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e)
      top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, v[i][e] & 0x7FFF7FFFu));
  return top[0] >= 0x7F80 || top[1] >= 0x7F80;
}

// The halves of a word of two bf16 values that are infinite or NaN.
__device__ __forceinline__ uint32_t special_halves(uint32_t w) {
  return ((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) |
         ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
}

// Device-coherent store and load of two floats (8 bytes, aligned): agent-scope atomics, which on this
// chip go through to and come from the point where its compute dies meet, past their own caches.  A
// state published with these stores is complete for whoever reads it with these loads after a counter
// that was added to once the stores had been acknowledged (s_waitcnt vmcnt(0), then a barrier, then the
// add): the split decode steps merge by the same protocol, and their kernel says why it holds.
__device__ __forceinline__ void coherent_store2(float* p, float x, float y) {
  const uint64_t v = (uint64_t)__float_as_uint(x) | ((uint64_t)__float_as_uint(y) << 32);
  __hip_atomic_store((uint64_t*)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 coherent_load2(const float* p) {
  const uint64_t v = __hip_atomic_load((uint64_t*)const_cast<float*>(p), __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// Inclusive sums over the lanes of a wave (row shifts by 1, 2, 4, 8, then the sums of the rows
// before: on the VALU).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_zero(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += dpp_or_zero<0x111, 0xf>(x);
  x += dpp_or_zero<0x112, 0xf>(x);
  x += dpp_or_zero<0x114, 0xf>(x);
  x += dpp_or_zero<0x118, 0xf>(x);
  x += dpp_or_zero<0x142, 0xa>(x);
  x += dpp_or_zero<0x143, 0xc>(x);
  return x;
}
__device__ __forceinline__ float wave_scan(float x) {
  auto add = [](float v, uint32_t o) { return v + __uint_as_float(o); };
  x = add(x, dpp_or_zero<0x111, 0xf>(__float_as_uint(x)));
  x = add(x, dpp_or_zero<0x112, 0xf>(__float_as_uint(x)));
  x = add(x, dpp_or_zero<0x114, 0xf>(__float_as_uint(x)));
  x = add(x, dpp_or_zero<0x118, 0xf>(__float_as_uint(x)));
  x = add(x, dpp_or_zero<0x142, 0xa>(__float_as_uint(x)));
  x = add(x, dpp_or_zero<0x143, 0xc>(__float_as_uint(x)));
  return x;
}
__device__ __forceinline__ int lane_value(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// Starting reference of a running maximum (log2 units): finite and below any score; and that of a
// column which has seen keys, but only with scores of -inf: its sum is 0 like that of one without keys.
constexpr float kNoScore = -3.0e38f, kNoWeight = -2.9e38f;

// A 32-bit word that the launch does not write, through the scalar cache.
__device__ __forceinline__ int scalar_word(const int32_t* p, size_t i) {
  return ((const __attribute__((address_space(4))) int32_t*)(const void*)p)[i];
}

// What a workgroup does: piece `piece` of `ways` of the walk of tile `tile` of sequence b.
struct PagedItem {
  int b, tile, piece, ways;
  int slot;    // first partial state of the tile under a KV head (ways > 1)
  Chunk c;
};

// How many of the n entries of `ends`, which never fall, are at most x: every lane of the wave takes
// part, 64 entries are compared at a time.  (Entries that do fall still give a number of 0 .. n.)
template <typename T>
__device__ __forceinline__ int count_upto(const T* ends, int n, T x, int lane) {
  int lo = 0;
  while (n > 64) {   // the answer lies in lo .. lo + n
    const int stride = (n + 63) >> 6;
    const int i = (lane + 1) * stride - 1;
    const int k = __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < n && ends[lo + i] <= x)) * stride;
    lo += k < n ? k : n;
    n = stride < n - k ? stride : n > k ? n - k : 0;
  }
  return lo + __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < n && ends[lo + lane] <= x));
}

// Words of a planned call's summary (PagedPlan::planned), written by a launch before the attention's:
// 1 / C; the items, partial states and cut tiles of the sequences of more than kPagedNarrowCols columns
// (all sequences where every one brings the same number of tokens); and per round of 64 sequences
// the running sums of the two kinds of sequences: items and cut tiles at its end, states before it.
enum PlanWord { kPlanShare, kPlanItems, kPlanSlots, kPlanCut, kPlanRounds = 8 };
enum PlanRow { kRowItems, kRowCut, kRowSlots, kPlanRows };
__device__ __forceinline__ uint32_t* plan_row(const PagedArgs& a, int row, int narrow) {
  return a.rounds + kPlanRounds + (size_t)(2 * row + narrow) * (size_t)paged_rounds(a.batch);
}

__device__ __forceinline__ Chunk chunk_at(const PagedArgs& a, int b) {
  if (b >= a.batch) return Chunk{0, 0, 0};
  const bool ragged = a.plan.uniform < 0;
  return chunk_of(b, a.plan.uniform, ragged ? a.q_start[b] : 0, ragged ? a.q_start[b + 1] : 0, a.pos[b],
                  a.n);
}

// What a sequence's chunk counts for among those of its kind: items, cut tiles, partial states.
// (q_start entries out of order can name any number of tiles: no count passes kMostItems, which is
// more than any launch has, so that sums over a wave stay below 2^31.)
constexpr uint32_t kMostItems = 1u << 24;
struct Share {
  int tiles, ways;
  uint32_t items, cut, slots;
};
__device__ __forceinline__ Share share_of_chunk(const PagedArgs& a, const Chunk& c, bool narrow,
                                                float per_share) {
  const PagedPlan& p = a.plan;
  const bool mine = p.uniform >= 0 || (c.count <= p.narrow_tokens) == narrow;
  Share s;
  s.tiles = mine ? p.tiles_of(c) : 0;
  s.ways = p.pieces > 0 ? p.pieces_of(p.steps_of(a.shape, c), per_share) : 1;
  const uint32_t pieces = (uint32_t)s.tiles * (uint32_t)s.ways;
  s.items = pieces < kMostItems ? pieces : kMostItems;
  s.cut = s.ways > 1 ? (uint32_t)s.tiles : 0u;
  s.slots = s.ways > 1 ? pieces : 0u;
  return s;
}

// 1 / C of a call of these many steps and tiles.  (q_start entries out of order can name more tiles
// than the launch has room for: no walk is cut then, so that no merge takes the state of a piece that does
// not run.)
__device__ __forceinline__ float per_share_of(const PagedPlan& p, float steps, uint32_t tiles) {
  return p.pieces > 0 && tiles <= (uint32_t)p.tiles ? 1.0f / p.share_of(steps) : 0.0f;
}

// Item `item` of a KV head (false: there are not that many).  Items go sequence by sequence, those of
// more than kPagedNarrowCols columns first, whose pieces take longest (128 single tokens and chunks of
// 665 and 577: 249 us, 267 in the sequences' order, 303 with both kinds in turn, eight items of each);
// of one sequence, piece by piece from the last tile (the longest walk) to the first, so that workgroups
// running side by side read the same keys.  CUT: the items are the tiles whose walks are cut (piece 0).
//
// Every wave finds its item by itself: the counts of 64 sequences at a time, one to a lane, and sums
// over the lanes.  In small batches it does so from the first on; in others (PagedPlan::planned) a launch
// before this one has summed up the rounds of 64 (PlanWord), and the wave searches those for its round.
template <bool CUT>
__device__ __forceinline__ bool find_item(const PagedArgs& a, int item, int lane, PagedItem& it) {
  const PagedPlan& p = a.plan;
  if (!CUT && p.uniform >= 0 && p.pieces == 0) {   // nothing to search for
    const int tiles = p.tiles_of(Chunk{0, p.uniform, 0});
    it.b = tiles == 1 ? item : item / tiles;
    if (it.b >= a.batch) return false;
    it.c = chunk_of(it.b, p.uniform, 0, 0, scalar_word(a.pos, (size_t)it.b), a.n);
    it.ways = 1;
    it.piece = 0;
    it.tile = tiles - 1 - (item - it.b * tiles);
    it.slot = 0;   // (the last store here and below: else the compiler keeps fields in memory)
    return true;
  }
  float per_share = 0.0f;
  uint32_t base = 0, sbase = 0;
  // looks for the item among the sequences b0 .. b0 + 63 (this lane's chunk c) of a kind
  auto found = [&](int b0, const Chunk& c, bool narrow) -> bool {
    const Share s = share_of_chunk(a, c, narrow, per_share);
    const uint32_t count = CUT ? s.cut : s.items;
    const uint32_t upto = wave_scan(count), supto = p.pieces > 0 ? wave_scan(s.slots) : 0u;
    const uint32_t all = (uint32_t)lane_value((int)upto, 63);
    if ((uint32_t)item >= base + all) {
      base += all;
      sbase += (uint32_t)lane_value((int)supto, 63);
      return false;
    }
    const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64((uint32_t)item < base + upto));
    it.b = b0 + l;
    it.c.row0 = lane_value(c.row0, l);
    it.c.count = lane_value(c.count, l);
    it.c.pos = lane_value(c.pos, l);
    it.ways = lane_value(s.ways, l);
    const int tiles = lane_value(s.tiles, l);
    const int r = item - (int)(base + (uint32_t)lane_value((int)(upto - count), l));
    it.piece = r / tiles;
    it.tile = tiles - 1 - (r - it.piece * tiles);
    it.slot = (int)(sbase + (uint32_t)lane_value((int)(supto - s.slots), l)) + it.tile * it.ways;
    return true;
  };
  if (p.planned) {
    const int32_t* const words = (const int32_t*)a.rounds;
    per_share = __uint_as_float((uint32_t)scalar_word(words, kPlanShare));
    const uint32_t wide = (uint32_t)scalar_word(words, CUT ? kPlanCut : kPlanItems);
    const bool narrow = (uint32_t)item >= wide;
    if (narrow && p.uniform >= 0) return false;
    if (narrow) base = wide, sbase = (uint32_t)scalar_word(words, kPlanSlots);
    const uint32_t* const ends = plan_row(a, CUT ? kRowCut : kRowItems, narrow);
    const int round = count_upto(ends, paged_rounds(a.batch), (uint32_t)item - base, lane);
    if (round >= paged_rounds(a.batch)) return false;
    if (round > 0) base += (uint32_t)scalar_word((const int32_t*)ends, (size_t)(round - 1));
    sbase += (uint32_t)scalar_word((const int32_t*)plan_row(a, kRowSlots, narrow), (size_t)round);
    return found(64 * round, chunk_at(a, 64 * round + lane), narrow);
  }
  // the first 128 sequences' chunks, their loads in flight together
  constexpr int ROUNDS = 2;
  Chunk kept[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) kept[r] = chunk_at(a, 64 * r + lane);
  if (p.pieces > 0) {
    float sum = 0.0f;
    uint32_t count = 0;
    auto add = [&](const Chunk& c) {
      const uint32_t nt = (uint32_t)p.tiles_of(c);
      // (contracted by hand: the merge launch works out the same pieces from the same sum)
      sum = __builtin_fmaf((float)nt, (float)p.steps_of(a.shape, c), sum);
      count = count + nt < kMostItems ? count + nt : kMostItems;
    };
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      if (64 * r >= a.batch) break;
      add(kept[r]);
    }
    for (int b0 = 64 * ROUNDS; b0 < a.batch; b0 += 64) add(chunk_at(a, b0 + lane));
    const float steps =
        __uint_as_float((uint32_t)lane_value((int)__float_as_uint(wave_scan(sum)), 63));
    per_share = per_share_of(p, steps, (uint32_t)lane_value((int)wave_scan(count), 63));
  }
  auto search = [&](bool narrow) -> bool {
    if (found(0, kept[0], narrow)) return true;
    if (a.batch > 64 && found(64, kept[1], narrow)) return true;
    for (int b0 = 64 * ROUNDS; b0 < a.batch; b0 += 64)
      if (found(b0, chunk_at(a, b0 + lane), narrow)) return true;
    return false;
  };
  return search(false) || (p.uniform < 0 && search(true));
}

// Whether one of the positions first .. last has a page: what a column whose sum is 0 asks about its keys.
__device__ __forceinline__ bool any_page(const PagedShape& sh, const int32_t* table, int first, int last) {
  last = min(last, sh.capacity - 1);
  if (last < first) return false;
  const int end = sh.by_page.div(last);
  for (int i = sh.by_page.div(first); i <= end; i += 8) {
    bool any = false;
#pragma unroll
    for (int u = 0; u < 8; ++u) any |= sh.is_page(table[min(i + u, end)]);
    if (any) return true;
  }
  return false;
}

// Merges the `ways` partial states of a tile ([COLS][D] outputs, then (reference, sum) per column,
// `stride` floats apart) into rows of the output: store(column, channel, o, reference, l) takes 4 channels
// of a column, unnormalised, its reference (log2 units) and its sum, lse(column, reference, l) these two.
// Every thread sums 4 channels of a column, eight states' loads in flight at a time.
template <int D, int COLS, int THREADS, typename S, typename L>
__device__ __forceinline__ void merge_states(const float* s0, size_t stride, int ways, int cols,
                                             int tid, S&& store, L&& lse) {
  constexpr int Q = D / 4;
  constexpr int U = 8;
  for (int i = tid; i < cols * Q; i += THREADS) {
    const int col = i / Q, q = i - col * Q;
    float m = kNoScore, l = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int w0 = 0; w0 < ways; w0 += U) {
      float2 ml[U], x[U], y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float* s = s0 + (size_t)(w0 + u < ways ? w0 + u : w0) * stride;
        ml[u] = coherent_load2(s + COLS * D + 2 * col);
        x[u] = coherent_load2(s + col * D + 4 * q);
        y[u] = coherent_load2(s + col * D + 4 * q + 2);
      }
      float mx = m;
#pragma unroll
      for (int u = 0; u < U; ++u) mx = fmaxf(mx, ml[u].x);
      const float keep = fast_exp2(m - mx);
      l *= keep;
      o *= keep;
      m = mx;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (w0 + u < ways) {   // (a state taken with weight 0 would turn an infinity into NaN)
          const float wt = fast_exp2(ml[u].x - mx);
          l += wt * ml[u].y;
          o[0] += wt * x[u].x;
          o[1] += wt * x[u].y;
          o[2] += wt * y[u].x;
          o[3] += wt * y[u].y;
        }
      }
    }
    store(col, 4 * q, o, m, l);
    if (q == 0) lse(col, m, l);
  }
}

// 1 / l and the natural-log partition of a column with reference m and sum l.  An empty support has l 0
// and gets zeros and -inf; one whose scores are all -inf (kNoWeight) NaN, 0 / 0, and -inf.
__device__ __forceinline__ float inverse_sum(float m, float l) {
  return l != 0.0f ? 1.0f / l : m > kNoScore ? __builtin_nanf("") : 0.0f;
}
__device__ __forceinline__ float log_partition(float m, float l) {
  return l == 0.0f ? kNegInf : (m + __builtin_log2f(l)) * 0.69314718055994531f;
}

__device__ __forceinline__ void store4(uint16_t* p, f32x4 o, float scale) {
  *(u32x2*)p = u32x2{pack_bf16(o[0] * scale, o[1] * scale), pack_bf16(o[2] * scale, o[3] * scale)};
}
__device__ __forceinline__ void store4(float* p, f32x4 o, float scale) { *(f32x4*)p = o * scale; }

// What a workgroup of a few-column walk (at most kPagedNarrowCols columns: all of a sequence's tokens
// under a KV head, position-major, head-minor) does after its waves have walked, for both types.
template <typename T, int D, int NW>
struct NarrowOut {
  static constexpr int COLS = kPagedNarrowCols;
  static constexpr int LDS = NW * COLS * (D + 2) * 4 + 16;   // the waves' states, and a word
  const PagedArgs& a;
  const PagedItem& it;
  int g;
  int cols;

  __device__ __forceinline__ int64_t address(int col) const {   // output row of a column
    const int cp = a.plan.by_group.div(col);
    return ((int64_t)it.c.row0 + cp) * a.hq + (int64_t)(g * a.group + col - cp * a.group);
  }
  __device__ __forceinline__ int64_t lse_at(int col) const {
    const int cp = a.plan.by_group.div(col);
    return (int64_t)(g * a.group + col - cp * a.group) * a.n + it.c.row0 + cp;
  }

  // A skipped sequence (one step by PagedPlan::steps_of, so never cut): zeros, no log-partition.
  __device__ __forceinline__ void skip(int tid) const {
    constexpr int Q = D * (int)sizeof(T) / 16;
    for (int i = tid; i < cols * Q; i += NW * 64) {
      const int col = i / Q;
      *(u32x4*)((unsigned char*)((T*)a.out + address(col) * D) + (i - col * Q) * 16) = u32x4{0u, 0u, 0u, 0u};
    }
    if (a.lse != nullptr && tid < cols) a.lse[lse_at(tid)] = kNegInf;
  }

  // The waves' states in LDS: unnormalised outputs [NW][COLS][D], references and sums [NW][COLS].
  static __device__ __forceinline__ float* outputs(unsigned char* smem) { return (float*)smem; }
  static __device__ __forceinline__ float* references(unsigned char* smem) {
    return (float*)smem + NW * COLS * D;
  }
  static __device__ __forceinline__ float* sums(unsigned char* smem) {
    return references(smem) + NW * COLS;
  }

  // Merges the waves' states (Eq.(lse)), each thread 4 channels of a column, once every wave has
  // stored its own; they have walked positions first .. last.  A cut walk leaves the result as the
  // piece's state: IN_PLACE the last piece to end merges them, else a second launch does.
  template <bool IN_PLACE, int SCOLS>
  __device__ __forceinline__ void finish(int tid, unsigned char* smem, int first, int last) const {
    const float* const sm_acc = outputs(smem);
    const float* const sm_m = references(smem);
    const float* const sm_l = sums(smem);
    int* const last_one = (int*)(smem + LDS - 16);
    __syncthreads();
    constexpr size_t STATE = paged_state_bytes(SCOLS, D) / 4;
    const size_t unit = (size_t)it.slot * a.hkv + (size_t)g * it.ways;   // the tile's states lie together
    float* const part = a.states + (unit + it.piece) * STATE;
    for (int i = tid; i < cols * (D / 4); i += NW * 64) {
      const int col = i / (D / 4), q = i - col * (D / 4);
      float M = kNoScore;
#pragma unroll
      for (int w = 0; w < NW; ++w) M = fmaxf(M, sm_m[w * COLS + col]);
      float L = 0.0f;
      f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {   // (a wave that saw nothing holds zeros)
        const float wt = fast_exp2(sm_m[w * COLS + col] - M);
        L += wt * sm_l[w * COLS + col];
        o += wt * *(const f32x4*)(sm_acc + (w * COLS + col) * D + 4 * q);
      }
      if (__builtin_expect(L == 0.0f, 0)) {
        const int t = it.c.pos + a.plan.by_group.div(col);
        if (any_page(a.shape, a.table + (size_t)it.b * a.shape.width, max(first, a.shape.support_lo(t)),
                     min(last, t)))
          M = kNoWeight;
      }
      if (it.ways == 1) {
        store4((T*)a.out + address(col) * D + 4 * q, o, inverse_sum(M, L));
        if (a.lse != nullptr && q == 0) a.lse[lse_at(col)] = log_partition(M, L);
      } else if (IN_PLACE) {
        coherent_store2(part + col * D + 4 * q, o[0], o[1]);
        coherent_store2(part + col * D + 4 * q + 2, o[2], o[3]);
        if (q == 0) coherent_store2(part + SCOLS * D + 2 * col, M, L);
      } else {
        *(f32x4*)(part + col * D + 4 * q) = o;
        if (q == 0) *(float2*)(part + SCOLS * D + 2 * col) = make_float2(M, L);
      }
    }
    if (!IN_PLACE || it.ways == 1) return;
    // Whoever completes the count of the walk's pieces merges them (coherent_store2 says why this
    // orders).
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this wave's stores have completed
    __syncthreads();
    if (tid == 0) {
      const unsigned before = __hip_atomic_fetch_add(&a.counters[unit], 1u, __ATOMIC_RELAXED,
                                                     __HIP_MEMORY_SCOPE_AGENT);
      *last_one = before == (unsigned)(it.ways - 1);
      if (*last_one)
        __hip_atomic_store(&a.counters[unit], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!*last_one) return;
    merge_states<D, SCOLS, NW * 64>(
        a.states + unit * STATE, STATE, it.ways, cols, tid,
        [&](int col, int c, f32x4 o, float mref, float l) {
          store4((T*)a.out + address(col) * D + c, o, inverse_sum(mref, l));
        },
        [&](int col, float mref, float l) {
          if (a.lse != nullptr) a.lse[lse_at(col)] = log_partition(mref, l);
        });
  }
};

// Merges the states of cut walks, a launch of its own after the pieces': x = (cut tile, KV head), y =
// runs of 16 columns (in turn where the grid has fewer), four to a wave.  Lane l takes channels
// 64 i + 4 (l mod 16) .. +3 of column l / 16.
template <typename T, int D, int COLS>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedArgs a) {
  constexpr int NB = D / 64;
  constexpr int U = 8;   // states in flight
  constexpr size_t STATE = paged_state_bytes(COLS, D) / 4;
  const int lane = threadIdx.x & 63;
  const PagedPlan& pl = a.plan;
  const int item = pl.by_hkv.div((int)blockIdx.x);
  const int g = (int)blockIdx.x - item * a.hkv;
  PagedItem it;
  if (!find_item<true>(a, item, lane, it) || it.c.pos < 0) return;
  const int p0 = it.tile * pl.tq;
  const int cols = min(pl.tq, it.c.count - p0) * a.group;
  const float* s = a.states + ((size_t)it.slot * a.hkv + (size_t)g * it.ways) * STATE;
  for (int col = (int)blockIdx.y * 16 + (int)(threadIdx.x >> 4); col < cols; col += (int)gridDim.y * 16) {
    const float* so = s + col * D + 4 * (lane & 15);
    const float* sm = s + COLS * D + 2 * col;
    float m = kNoScore, l = 0.0f;
    f32x4 o[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto take = [&](auto states, int w0) {   // (a state read twice would need a weight of 0)
      constexpr int N = decltype(states)::value;
      float2 ml[N];
      f32x4 x[N][NB];
#pragma unroll
      for (int u = 0; u < N; ++u) {
        ml[u] = *(const float2*)(sm + (size_t)(w0 + u) * STATE);
#pragma unroll
        for (int i = 0; i < NB; ++i) x[u][i] = *(const f32x4*)(so + (size_t)(w0 + u) * STATE + 64 * i);
      }
      float mx = m;
#pragma unroll
      for (int u = 0; u < N; ++u) mx = fmaxf(mx, ml[u].x);
      const float keep = fast_exp2(m - mx);
      l *= keep;
#pragma unroll
      for (int i = 0; i < NB; ++i) o[i] *= keep;
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const float wt = fast_exp2(ml[u].x - mx);
        l += wt * ml[u].y;
#pragma unroll
        for (int i = 0; i < NB; ++i) o[i] += wt * x[u][i];
      }
      m = mx;
    };
    int w = 0;
    for (; w + U <= it.ways; w += U) take(std::integral_constant<int, U>{}, w);
    if (w + 4 <= it.ways) take(std::integral_constant<int, 4>{}, w), w += 4;
    if (w + 2 <= it.ways) take(std::integral_constant<int, 2>{}, w), w += 2;
    if (w < it.ways) take(std::integral_constant<int, 1>{}, w);
    const int cp = pl.by_group.div(col);
    const int64_t row = (int64_t)it.c.row0 + p0 + cp;
    const int head = g * a.group + col - cp * a.group;
    const float inv = inverse_sum(m, l);
    T* out = (T*)a.out + (row * a.hq + head) * D + 4 * (lane & 15);
#pragma unroll
    for (int i = 0; i < NB; ++i) store4(out + 64 * i, o[i], inv);
    if (a.lse != nullptr && (lane & 15) == 0) a.lse[(int64_t)head * a.n + row] = log_partition(m, l);
  }
}

// (At most some 2048 workgroups: a call that cuts nothing still has them look; 8768 took 15 us.)
template <typename T, int D, int COLS>
hipError_t launch_paged_merge(const PagedArgs& a, hipStream_t stream) {
  const int tiles = a.plan.cut_tiles() * a.hkv;
  const int runs = 2048 / tiles < 1 ? 1 : 2048 / tiles > COLS / 16 ? COLS / 16 : 2048 / tiles;
  hipLaunchKernelGGL((paged_merge_kernel<T, D, COLS>), dim3((unsigned)tiles, (unsigned)runs), dim3(256), 0,
                     stream, a);
  return hipGetLastError();
}

}  // namespace pbb
