// Device-side helpers shared by the paged attention kernels: which work a workgroup does, page
// addresses, and the merge of cut walks.
#pragma once

#include "pbb_device.h"
#include "pbb_internal.h"

namespace pbb {

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

// Item `item` of a KV head (false: there are not that many).  Every wave finds it by itself, 64
// sequences at a time: their counts of pieces, and a sum over the lanes.  Items go sequence by
// sequence; of one sequence, piece by piece from the last tile (the longest walk) to the first, so
// that workgroups running side by side read the same keys.
__device__ __forceinline__ bool find_item(const PagedArgs& a, int item, int lane, PagedItem& it) {
  const PagedPlan& p = a.plan;
  auto chunk = [&](int b) -> Chunk {
    if (b >= a.batch) return Chunk{0, 0, 0};
    const bool ragged = p.uniform < 0;
    return chunk_of(b, p.uniform, ragged ? a.q_start[b] : 0, ragged ? a.q_start[b + 1] : 0, a.pos[b],
                    a.n);
  };
  const Chunk c0 = chunk(lane);
  float share = 1.0e30f;
  if (p.pieces > 0) {
    float total = 0.0f;
    uint32_t tiles = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
      const Chunk c = b0 == 0 ? c0 : chunk(b0 + lane);
      const int nt = p.tiles_of(c);
      total += __uint_as_float((uint32_t)lane_value(
          (int)__float_as_uint(wave_scan((float)nt * (float)p.steps_of(a.shape, c))), 63));
      tiles += (uint32_t)lane_value((int)wave_scan((uint32_t)nt), 63);
    }
    // (q_start entries out of order can name more tiles than the launch has room for: no walk is
    // cut then, so that no merge waits for a piece that does not run)
    if (tiles <= (uint32_t)p.tiles) share = p.share_of(total);
  }
  uint32_t base = 0, sbase = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const Chunk c = b0 == 0 ? c0 : chunk(b0 + lane);
    const int nt = p.tiles_of(c);
    const int ways = p.pieces_of(p.steps_of(a.shape, c), share);
    const uint32_t count = (uint32_t)nt * (uint32_t)ways;
    const uint32_t cut = ways > 1 ? count : 0u;
    const uint32_t upto = wave_scan(count), supto = wave_scan(cut);
    const uint32_t all = (uint32_t)lane_value((int)upto, 63);
    if ((uint32_t)item < base + all) {
      const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64((uint32_t)item < base + upto));
      it.b = b0 + l;
      it.c.row0 = lane_value(c.row0, l);
      it.c.count = lane_value(c.count, l);
      it.c.pos = lane_value(c.pos, l);
      it.ways = lane_value(ways, l);
      const int tiles = lane_value(nt, l);
      const int r = item - (int)(base + (uint32_t)lane_value((int)(upto - count), l));
      it.piece = r / tiles;
      it.tile = tiles - 1 - (r - it.piece * tiles);
      it.slot = (int)(sbase + (uint32_t)lane_value((int)(supto - cut), l)) + it.tile * it.ways;
      return true;
    }
    base += all;
    sbase += (uint32_t)lane_value((int)supto, 63);
  }
  return false;
}

// Merges the `ways` partial states of a tile ([COLS][D] outputs, then (reference, sum) per column,
// `stride` floats apart) into rows of the output: store(column, channel, x, y, z, w) takes 4
// channels of a column, lse(column, value) its log-partition in log2 units.  Every thread sums 4
// channels of a column, eight states' loads in flight at a time.
template <int D, int COLS, int THREADS, typename S, typename L>
__device__ __forceinline__ void merge_states(const float* s0, size_t stride, int ways, int cols,
                                             int tid, S&& store, L&& lse) {
  constexpr int Q = D / 4;
  constexpr int U = 8;
  for (int i = tid; i < cols * Q; i += THREADS) {
    const int col = i / Q, q = i - col * Q;
    float m = -3.0e38f, l = 0.0f;
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
    store(col, 4 * q, o, l);
    if (q == 0) lse(col, m, l);
  }
}

}  // namespace pbb
