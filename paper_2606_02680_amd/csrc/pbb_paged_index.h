// Index arithmetic of the paged-cache launches, usable on the host and in kernels (and by a plain
// C++ compiler: nothing here needs HIP).
#pragma once

#include <stdint.h>

#include "pbb_index.h"

namespace pbb {

enum PagedSupport : int32_t { kPagedFull = 0, kPagedPBB = 1, kPagedSWA = 2 };

// Rows and positions of one sequence's chunk in a packed call.
struct Chunk {
  int row0;    // first packed row
  int count;   // tokens (0: none)
  int pos;     // position of the first one; negative: the sequence is skipped
};

// A sequence's chunk from its q_start entries (or, uniform >= 0, that many tokens each) and pos,
// cut so that no row leaves [0, n_tokens) and no position passes 2^31 - 1.
PBB_HD Chunk chunk_of(int b, int uniform, int start, int end, int pos, int n_tokens) {
  Chunk c;
  if (uniform >= 0) {
    c.row0 = b * uniform;
    c.count = uniform;
  } else {
    const int s = start < 0 ? 0 : start > n_tokens ? n_tokens : start;
    const int e = end < s ? s : end > n_tokens ? n_tokens : end;
    c.row0 = s;
    c.count = e - s;
  }
  c.pos = pos > 0x7fffffff - n_tokens ? -1 : pos;
  return c;
}

// Everything a walk over a cache depends on, launch constants.
struct PagedShape {
  int page_size, n_pages, width;
  int capacity;          // width * page_size: positions from here on have no page
  int support;           // PagedSupport
  int half, window;      // PBB: half-block; sliding window
  FastDiv by_page, by_half;
  static PagedShape make(int page_size, int n_pages, int width, int block, int window) {
    PagedShape s;
    s.page_size = page_size;
    s.n_pages = n_pages;
    s.width = width;
    s.capacity = page_size * width;
    s.support = block > 0 ? kPagedPBB : window > 0 ? kPagedSWA : kPagedFull;
    s.half = block / 2;
    s.window = window;
    s.by_page = FastDiv::make((uint32_t)page_size);
    s.by_half = FastDiv::make((uint32_t)(block > 0 ? block / 2 : 1));
    return s;
  }
  // First source of the support of target t; never decreases in t.
  PBB_HD int support_lo(int t) const {
    const int lo = support == kPagedFull ? 0
                   : support == kPagedPBB ? half * (by_half.div(t) - 1)
                                          : t - window + 1;
    return lo > 0 ? lo : 0;
  }
  // A table entry, made safe to address with: 0 in place of one that names no page.
  PBB_HD bool is_page(int id) const { return (uint32_t)id < (uint32_t)n_pages; }
  // Keys that a run of `tokens` targets ending at position `last` can walk, at most.
  PBB_HD uint32_t max_keys(int last, int tokens) const {
    const uint32_t all = (uint32_t)(last < capacity ? last + 1 : capacity);
    const uint32_t span = (support == kPagedPBB ? 2u * (uint32_t)half : (uint32_t)window) + (uint32_t)tokens;
    return support != kPagedFull && span < all ? span : all;
  }
};

// How the walks of an attention call are spread over workgroups.
//
// A unit is a tile of `tq` tokens of one sequence under one KV head; its walk is a number of key
// steps.  With T the call's steps per KV head (tiles times the sequence's longest walk) and a
// budget of `pieces` workgroups per KV head, a sequence's walks are cut into P = ceil(steps / C)
// pieces each, C = max(least, T / pieces): so no piece is longer than an even share of the whole
// (a sequence far longer than the others does not hold the call up), there are at most
// tiles + pieces workgroups, and at most 2 x pieces of them belong to walks that are cut.  The
// kernels work this out by themselves, from positions that only the device knows.
//
// Calls of few columns per sequence (`narrow`: single tokens, short drafts) have kernels of their
// own.  Their states are small, and the last piece of a walk to end merges them; states of 128
// columns (66 KiB at d = 128) would keep one workgroup busy for 3 us each, so the others merge in a
// second launch, four waves per 16 columns.
constexpr int kPagedNarrowCols = 16;
constexpr int kPagedMaxPieces = 2048;   // budget of a call's KV heads together, at most

// Sequences that every workgroup looks through by itself for its item; calls of more are summed up by a
// launch of one workgroup before the attention's, since that search grows with the square of the batch
// (single tokens named by q_start, 16/2 heads, d 128, 100 cached each, walks that may be cut: 132 of them
// 22.2 us, 27.2 with every workgroup looking through all; 1024 41 / 120; 16384 434 / 10870).  Where every
// sequence brings the same number the search is one pass shorter (192 19.6 / 19.2, 224 19.7 / 21.7), and
// where no walk can be cut one more (256 21.8 / 19.6, 320 23.0 / 21.9, 512 26.2 / 30.9).
constexpr int kPagedScan = 128, kPagedScanEqual = 192, kPagedScanUncut = 384;
// Rounds of 64 sequences, and the bytes of their summary.
PBB_HD int paged_rounds(int batch) { return (batch + 63) >> 6; }
inline uint64_t paged_rounds_bytes(int batch) {
  return (32 + 24 * (uint64_t)paged_rounds(batch) + 15) / 16 * 16;
}

// Tile and cutting rules of a kind of kernel.  Where the even share of one round of the chip is short
// (below many_least), C is that share, at least few_least: T / (round - tiles), so that tiles and pieces
// together are no more than the round (half of the round, where the tiles alone are that many).  Else
// C = max(many_least, T / pieces): as many pieces as even out the end of the call, but none so short
// that its first loads and its merge cost more than that gains.
struct PagedKind {
  int cols;     // query columns of a tile
  int step;     // keys per step, 16 or 32
  int round;    // workgroups of one round, in all heads (0: always the second rule)
  int few_least;
  int pieces;   // in all heads
  int many_least;
};

struct PagedPlan {
  int cols;      // query columns of a tile
  int tq;        // tokens per tile
  int step, step_bits;   // keys per step, a power of two
  int pieces;    // pieces of cut walks per KV head, at most; 0: no walk is cut
  int few_least, many_least;
  float per_round, per_pieces;   // 1 / workgroups of a round, 1 / pieces, per KV head
  int uniform;   // tokens of every sequence, -1: q_start says
  int narrow;    // 1: at most kPagedNarrowCols columns per sequence
  int narrow_tokens;   // tokens of that many columns
  int planned;   // 1: a launch of its own sums up the sequences
  int tiles;     // tiles of a call, at most
  int slots;     // partial states per KV head, at most
  FastDiv by_hkv, by_tq, by_group;
  static bool is_narrow(int batch, int group, int n_tokens, bool ragged) {
    return !ragged && (int64_t)(n_tokens / batch) * group <= kPagedNarrowCols;
  }
  static PagedPlan make(const PagedShape& s, const PagedKind& k, int batch, int hkv, int group,
                        int n_tokens, bool ragged) {
    PagedPlan p;
    p.uniform = ragged ? -1 : n_tokens / batch;
    p.narrow = is_narrow(batch, group, n_tokens, ragged);
    p.narrow_tokens = kPagedNarrowCols / group;
    p.cols = k.cols;
    p.tq = p.cols / group;
    p.step = k.step;
    p.step_bits = k.step == 16 ? 4 : 5;
    p.by_hkv = FastDiv::make((uint32_t)hkv);
    p.by_tq = FastDiv::make((uint32_t)p.tq);
    p.by_group = FastDiv::make((uint32_t)group);
    // ceil(n / tq) of every sequence, summed: at most one more each than of all together
    p.tiles = ragged ? n_tokens / p.tq + (batch < n_tokens ? batch : n_tokens)
                     : batch * ((p.uniform + p.tq - 1) / p.tq);
    const int all = k.round / hkv, many = k.pieces / hkv;
    const int round = all - (p.tiles < all / 2 ? p.tiles : all / 2);
    p.few_least = round > 0 && k.few_least < k.many_least ? k.few_least : k.many_least;
    p.many_least = k.many_least;
    p.per_round = 1.0f / (float)(round > 0 ? round : 1);
    p.per_pieces = 1.0f / (float)(many > 0 ? many : 1);
    // (Walks of fewer than many_least steps are worth the merge launch only where there are few: 512
    // tokens of four prompts, 32/8 heads, 28.5 us, 33.2 with a launch that finds nothing to merge.)
    // Single tokens merge without one: there it is the search for a workgroup's item that a call without
    // cut walks is spared (256 of 100 keys, 16/2 heads: 20.5 us, 15.5 without it).
    const bool many_tiles = p.narrow ? p.tiles >= 4 * all : 4 * p.tiles >= all;
    const int worth = many_tiles ? k.many_least : p.few_least;
    p.pieces = longest_walk(s, k, p.tq) > worth && 2 * hkv <= kPagedMaxPieces
                   ? (round > many ? round : many) : 0;
    p.slots = p.pieces > 0 ? 2 * p.pieces + p.pieces / 8 + 2 : 0;
    p.planned = p.pieces > 0 ? batch > (ragged ? kPagedScan : kPagedScanEqual)
                             : ragged && batch > kPagedScanUncut;
    return p;
  }
  static int64_t longest_walk(const PagedShape& s, const PagedKind& k, int tq) {
    return (int64_t)((s.max_keys(s.capacity, tq) + k.step - 1) / k.step) + 1;
  }
  // Tiles of a chunk, and the longest walk of one of them in steps.
  PBB_HD int tiles_of(const Chunk& c) const { return c.count > 0 ? by_tq.div(c.count - 1) + 1 : 0; }
  PBB_HD int steps_of(const PagedShape& s, const Chunk& c) const {
    if (c.pos < 0 || c.count == 0) return 1;
    const uint32_t keys = s.max_keys(c.pos + c.count - 1, tq < c.count ? tq : c.count);
    return (int)((keys + (1u << step_bits) - 1) >> step_bits) + 1;
  }
  // Pieces of each of a sequence's walks, per_share = 1 / C (C the steps of a piece).
  PBB_HD int pieces_of(int steps, float per_share) const {
    if (pieces == 0) return 1;
    const int p = (int)__builtin_ceilf((float)steps * per_share);
    return p > 1 ? p : 1;
  }
  PBB_HD float share_of(float total) const {
    const float one = total * per_round, many = total * per_pieces;
    const float least = (float)many_least;
    if (few_least < many_least && one < least) return one > (float)few_least ? one : (float)few_least;
    return many > least ? many : least;
  }
  // Tiles per KV head whose walks are cut, at most (each is longer than an even share).
  int cut_tiles() const { return tiles < pieces + pieces / 16 + 1 ? tiles : pieces + pieces / 16 + 1; }
  // Workgroups per KV head, at most.
  int64_t items() const { return (int64_t)tiles + pieces + pieces / 16 + 1; }
};

}  // namespace pbb
