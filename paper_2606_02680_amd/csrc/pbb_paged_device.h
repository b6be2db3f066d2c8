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
// sequence, those of more than kPagedNarrowCols columns first, whose pieces take longest (128 single
// tokens and chunks of 665 and 577: 249 us, 267 in the sequences' order, 303 with both kinds in turn,
// eight items of each); of one sequence, piece by piece from the last tile (the longest walk) to the
// first, so that workgroups running side by side read the same keys.  CUT: the items are the tiles
// whose walks are cut (piece 0).
template <bool CUT>
__device__ __forceinline__ bool find_item(const PagedArgs& a, int item, int lane, PagedItem& it) {
  const PagedPlan& p = a.plan;
  if (!CUT && p.uniform >= 0 && p.pieces == 0) {   // nothing to search for
    const int tiles = p.tiles_of(Chunk{0, p.uniform, 0});
    it.b = tiles == 1 ? item : item / tiles;
    if (it.b >= a.batch) return false;
    it.tile = tiles - 1 - (item - it.b * tiles);
    it.piece = 0;
    it.ways = 1;
    it.slot = 0;
    it.c = chunk_of(it.b, p.uniform, 0, 0, scalar_word(a.pos, (size_t)it.b), a.n);
    return true;
  }
  auto chunk = [&](int b) -> Chunk {
    if (b >= a.batch) return Chunk{0, 0, 0};
    const bool ragged = p.uniform < 0;
    return chunk_of(b, p.uniform, ragged ? a.q_start[b] : 0, ragged ? a.q_start[b + 1] : 0, a.pos[b],
                    a.n);
  };
  // the first 128 sequences' chunks, their loads in flight together
  constexpr int KEPT = 2;
  Chunk kept[KEPT];
#pragma unroll
  for (int r = 0; r < KEPT; ++r) kept[r] = chunk(64 * r + lane);
  auto round = [&](auto&& visit) {   // visit(first sequence, this lane's chunk): false ends it
#pragma unroll
    for (int r = 0; r < KEPT; ++r) {
      if (64 * r >= a.batch) return;
      if (!visit(64 * r, kept[r])) return;
    }
    for (int b0 = 64 * KEPT; b0 < a.batch; b0 += 64)
      if (!visit(b0, chunk(b0 + lane))) return;
  };
  float per_share = 0.0f;
  if (p.pieces > 0) {
    float sum = 0.0f;
    uint32_t count = 0;
    round([&](int, const Chunk& c) {
      const int nt = p.tiles_of(c);
      // (contracted by hand: the merge launch works out the same pieces from the same sum)
      sum = __builtin_fmaf((float)nt, (float)p.steps_of(a.shape, c), sum);
      count += (uint32_t)nt;
      return true;
    });
    const float total =
        __uint_as_float((uint32_t)lane_value((int)__float_as_uint(wave_scan(sum)), 63));
    const uint32_t tiles = (uint32_t)lane_value((int)wave_scan(count), 63);
    // (q_start entries out of order can name more tiles than the launch has room for: no walk is
    // cut then, so that no merge waits for a piece that does not run)
    if (tiles <= (uint32_t)p.tiles) per_share = 1.0f / p.share_of(total);
  }
  uint32_t base = 0, sbase = 0;
  bool found = false;
  auto search = [&](auto&& mine) {   // among the sequences that mine(tokens) takes
    round([&](int b0, const Chunk& c) {
      const int nt = mine(c.count) ? p.tiles_of(c) : 0;
      const int ways = p.pieces_of(p.steps_of(a.shape, c), per_share);
      const uint32_t pieces = (uint32_t)nt * (uint32_t)ways;
      const uint32_t cut = ways > 1 ? pieces : 0u;
      const uint32_t count = !CUT ? pieces : ways > 1 ? (uint32_t)nt : 0u;
      const uint32_t upto = wave_scan(count), supto = wave_scan(cut);
      const uint32_t all = (uint32_t)lane_value((int)upto, 63);
      if ((uint32_t)item >= base + all) {
        base += all;
        sbase += (uint32_t)lane_value((int)supto, 63);
        return true;
      }
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
      found = true;
      return false;
    });
  };
  if (p.uniform >= 0) {
    search([](int) { return true; });
  } else {
    search([&](int count) { return count > p.narrow_tokens; });
    if (!found) search([&](int count) { return count <= p.narrow_tokens; });
  }
  return found;
}

// Merges the `ways` partial states of a tile ([COLS][D] outputs, then (reference, sum) per column,
// `stride` floats apart) into rows of the output: store(column, channel, o, l) takes 4 channels of a
// column, unnormalised, and its sum, lse(column, reference, l) the reference (log2 units) and the sum.
// Every thread sums 4 channels of a column, eight states' loads in flight at a time.
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

// 1 / l and the natural-log partition of a column with reference m and sum l; an empty support has
// l 0 and gets zeros and -inf.
__device__ __forceinline__ float inverse_sum(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
__device__ __forceinline__ float log_partition(float m, float l) {
  return l == 0.0f ? kNegInf : (m + __builtin_log2f(l)) * 0.69314718055994531f;
}

__device__ __forceinline__ void store4(uint16_t* p, f32x4 o, float scale) {
  *(u32x2*)p = u32x2{pack_bf16(o[0] * scale, o[1] * scale), pack_bf16(o[2] * scale, o[3] * scale)};
}
__device__ __forceinline__ void store4(float* p, f32x4 o, float scale) { *(f32x4*)p = o * scale; }

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
    float m = -3.0e38f, l = 0.0f;
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
    const float inv = inverse_sum(l);
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
