// Rotary positions and the paged append on gfx950 (MI355X).
//
// Channels (c, c + d/2) of a row turn by the angle 2 pi turns[c] p, p the token's position on the
// pair's axis: (x cos - y sin, y cos + x sin); the transposed rotation, which gradients take, is
// the same with the angle negated.  The append does this to the new keys (and the chunk's queries)
// on their way into the pages, and copies the values.
//
// Bound: HBM (each row read once and written once).  A lane takes the 16-byte piece of channels
// c.. and its partner d/2 further on, of the rows of one token that are 64 / PC apart (PC pieces per
// half row), so a wave reads 64 / PC whole rows at once and works out its sines and cosines once for
// all rows of the token that it visits.

#include "pbb_device.h"
#include "pbb_paged_device.h"

namespace pbb {
namespace {

constexpr int kRotThreads = 256;
// A grid's x has fewer than 2^32 threads: groups of tokens beyond kGridX go on along z.
constexpr int kGridX = 1 << 23;
__device__ __forceinline__ int token_group() { return (int)(blockIdx.z * kGridX + blockIdx.x); }
dim3 token_grid(int64_t groups, int runs) {
  return dim3((unsigned)(groups < kGridX ? groups : kGridX), (unsigned)runs,
              (unsigned)((groups + kGridX - 1) / kGridX));
}
// Rows of more bytes than the last-level cache (256 MB) are read and written with the non-temporal
// hint: what is written first is gone before anything reads it (4 x 16384 tokens of 32 heads, d 128:
// 537 MB, 259 us with the 8 key heads' call, 239 to 241 with the hint, 5.6 TB/s; 16000 tokens, 131 MB: the
// next kernel finds them in the cache).
constexpr int64_t kStreamBytes = 256ll << 20;

template <typename T>
struct Piece;   // 16 bytes of a row as floats
template <>
struct Piece<uint16_t> {
  static constexpr int N = 8;
  typedef u32x4 raw;
  static __device__ __forceinline__ float get(raw r, int e) {
    return __uint_as_float(e & 1 ? r[e >> 1] & 0xFFFF0000u : r[e >> 1] << 16);
  }
  static __device__ __forceinline__ raw put(const float (&f)[N]) {
    return raw{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]),
               pack_bf16(f[6], f[7])};
  }
};
template <>
struct Piece<float> {
  static constexpr int N = 4;
  typedef u32x4 raw;
  static __device__ __forceinline__ float get(raw r, int e) { return __uint_as_float(r[e]); }
  static __device__ __forceinline__ raw put(const float (&f)[N]) {
    return raw{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
               __float_as_uint(f[3])};
  }
};

// cos and sin of `turns` whole turns.  The angle is reduced to half a turn either way in fp64.
// bf16: the hardware's sine and cosine (of turns; their error of a few 2^-22 is far below the
// rounding of the result); fp32: sincospif, whose last-bit error is of the order of the result's.
template <typename T>
__device__ __forceinline__ void cos_sin(double turns, float& cs, float& sn) {
  const float f = (float)(turns - __builtin_rint(turns));
  if constexpr (sizeof(T) == 2) {
    cs = __builtin_amdgcn_cosf(f);
    sn = __builtin_amdgcn_sinf(f);
  } else {
    sincospif(2.0f * f, &sn, &cs);
  }
}

// The sines and cosines of piece pc of a row (pairs pc N .. + N - 1) at a token's positions;
// position(axis) reads them.
template <typename T, typename F>
__device__ __forceinline__ void piece_turns(const RopeArgs& r, int pc, F&& position,
                                            float (&cs)[Piece<T>::N], float (&sn)[Piece<T>::N]) {
  constexpr int N = Piece<T>::N;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const int c = pc * N + e;
    cos_sin<T>((double)position(r.axis[c]) * r.turns[c], cs[e], sn[e]);
  }
}

template <typename T>
__device__ __forceinline__ void turn_pieces(u32x4& lo, u32x4& hi, const float (&cs)[Piece<T>::N],
                                            const float (&sn)[Piece<T>::N]) {
  constexpr int N = Piece<T>::N;
  float ox[N], oy[N];
#pragma unroll
  for (int e = 0; e < N; ++e)
    rope_turn(Piece<T>::get(lo, e), Piece<T>::get(hi, e), cs[e], sn[e], ox[e], oy[e]);
  lo = Piece<T>::put(ox);
  hi = Piece<T>::put(oy);
}

// Grid: x (and z) = groups of tokens / waves per workgroup, y = runs of a token's heads.  Where a token
// has fewer heads than a wave takes rows, a wave takes several tokens (2 heads, d 64, 16000 tokens with
// 12 query heads: 20.9 us for both calls with one token per wave, 15.9 with eight).
template <typename T, int D, bool NT>
__global__ __launch_bounds__(kRotThreads) void rotate_kernel(RotateArgs a) {
  constexpr int PC = D * (int)sizeof(T) / 32;   // pieces per half row
  constexpr int ROWS = 64 / PC;                 // rows of a wave at a time
  constexpr int ROWB = D * (int)sizeof(T);
  const int lane = threadIdx.x & 63;
  const int row = lane / PC;
  const int sub = a.tokens_per_wave > 1 ? a.by_heads.div(row) : 0;   // token within the wave's
  const int64_t wave = (int64_t)token_group() * (kRotThreads / 64) + (threadIdx.x >> 6);
  const int64_t tok = wave * a.tokens_per_wave + sub;
  if (tok >= a.n || sub >= a.tokens_per_wave) return;
  const int pc = lane % PC;
  float cs[Piece<T>::N], sn[Piece<T>::N];
  piece_turns<T>(a.rope, pc, [&](int axis) { return a.positions[(size_t)axis * a.n + tok]; }, cs, sn);
  const unsigned char* x = (const unsigned char*)a.x + tok * a.x_stride + pc * 16;
  unsigned char* o = (unsigned char*)a.out + tok * a.out_stride + pc * 16;
  const int h1 = min(a.heads, (int)(blockIdx.y + 1) * a.run);
  for (int h = blockIdx.y * a.run + row - sub * a.heads; h < h1; h += ROWS) {
    const unsigned char* p = x + (size_t)h * ROWB;
    unsigned char* w = o + (size_t)h * ROWB;
    if constexpr (NT) {
      u32x4 lo = __builtin_nontemporal_load((const u32x4*)p);
      u32x4 hi = __builtin_nontemporal_load((const u32x4*)(p + ROWB / 2));
      turn_pieces<T>(lo, hi, cs, sn);
      __builtin_nontemporal_store(lo, (u32x4*)w);
      __builtin_nontemporal_store(hi, (u32x4*)(w + ROWB / 2));
    } else {
      u32x4 lo = *(const u32x4*)p, hi = *(const u32x4*)(p + ROWB / 2);
      turn_pieces<T>(lo, hi, cs, sn);
      *(u32x4*)w = lo;
      *(u32x4*)(w + ROWB / 2) = hi;
    }
  }
}

// The sequence that packed row `tok` belongs to, or -1: the number of sequences whose rows end at or
// before it (every lane of the wave takes part; q_start never falls).
__device__ __forceinline__ int sequence_of(const int32_t* q_start, int batch, int tok, int lane) {
  const int b = count_upto(q_start + 1, batch, tok, lane);
  if (b >= batch) return -1;
  return __builtin_amdgcn_readfirstlane(q_start[b]) <= tok ? b : -1;
}

// Grid as rotate_kernel, over a token's query rows, key rows and value rows (in this order).
template <typename T, int D>
__global__ __launch_bounds__(kRotThreads) void paged_append_kernel(AppendArgs a) {
  constexpr int PC = D * (int)sizeof(T) / 32;
  constexpr int ROWS = 64 / PC;
  constexpr int ROWB = D * (int)sizeof(T);
  const int lane = threadIdx.x & 63;
  const int tok = __builtin_amdgcn_readfirstlane(
      (int)((uint32_t)token_group() * (kRotThreads / 64) + (threadIdx.x >> 6)));
  if (tok >= a.n) return;
  const int b = a.uniform >= 0 ? a.by_uniform.div(tok) : sequence_of(a.q_start, a.batch, tok, lane);
  if (b < 0) return;
  const Chunk c = chunk_of(b, a.uniform, a.uniform >= 0 ? 0 : a.q_start[b],
                           a.uniform >= 0 ? 0 : a.q_start[b + 1], a.pos[b], a.n);
  const bool skip = c.pos < 0;
  const int t = skip ? 0 : c.pos + (tok - c.row0);
  // the page row of position t (page -1: none, nothing is stored)
  int page = -1, slot = 0;
  if (!skip && t < a.shape.capacity) {
    const int i = a.shape.by_page.div(t);
    slot = t - i * a.shape.page_size;
    const int id = a.table[(size_t)b * a.shape.width + i];
    page = a.shape.is_page(id) ? id : -1;
  }
  const int pc = lane % PC;
  float cs[Piece<T>::N], sn[Piece<T>::N];
  if (a.turn)
    piece_turns<T>(a.rope, pc,
                   [&](int axis) {
                     return a.rope_pos != nullptr ? a.rope_pos[(size_t)axis * a.n + tok] : t;
                   },
                   cs, sn);
  const int hq = a.q != nullptr ? a.hq : 0;
  const int rows = hq + 2 * a.hkv;
  const int r1 = min(rows, (int)(blockIdx.y + 1) * a.run);
  // rows of a lane in flight (one: 49.5 us at 37 sequences' 9000 tokens, two 47, both with the inputs in the
  // last-level cache; 55 from memory)
  constexpr int AU = 2;
  const int64_t page_row = page < 0 ? 0 : (int64_t)page * a.hkv * a.shape.page_size + slot;
  for (int r0 = blockIdx.y * a.run + lane / PC; r0 < r1; r0 += AU * ROWS) {
    u32x4 lo[AU], hi[AU];
#pragma unroll
    for (int u = 0; u < AU; ++u) {
      const int r = min(r0 + u * ROWS, r1 - 1);
      const unsigned char* p =
          (r < hq ? (const unsigned char*)a.q + tok * a.q_stride + (size_t)r * ROWB
           : r < hq + a.hkv ? (const unsigned char*)a.k + tok * a.k_stride + (size_t)(r - hq) * ROWB
                            : (const unsigned char*)a.v + tok * a.v_stride +
                                  (size_t)(r - hq - a.hkv) * ROWB) + pc * 16;
      lo[u] = *(const u32x4*)p, hi[u] = *(const u32x4*)(p + ROWB / 2);
    }
#pragma unroll
    for (int u = 0; u < AU; ++u) {
      const int r = r0 + u * ROWS;
      if (r >= r1) break;
      if (a.turn && r < hq + a.hkv) turn_pieces<T>(lo[u], hi[u], cs, sn);
      unsigned char* w;
      if (r < hq) {
        if (skip) lo[u] = hi[u] = u32x4{0u, 0u, 0u, 0u};
        w = (unsigned char*)a.q_out + ((size_t)tok * hq + r) * ROWB;
      } else {
        if (page < 0) break;
        const bool key = r < hq + a.hkv;
        const int h = r - hq - (key ? 0 : a.hkv);
        w = (unsigned char*)(key ? a.k_pages : a.v_pages) +
            (size_t)(page_row + (int64_t)h * a.shape.page_size) * ROWB;
      }
      *(u32x4*)(w + pc * 16) = lo[u];
      *(u32x4*)(w + pc * 16 + ROWB / 2) = hi[u];
    }
  }
}

// Heads per workgroup row of the grid: all of a token's, unless the tokens alone leave the chip
// short of waves; then as few as a wave takes at once, and no more than 65535 runs (2000 tokens of 48
// rows: 11.5 us, 13.5 with a run per 8 rows; 256 tokens: 5.0 us so; inputs in the last-level cache).
int head_run(int tokens, int heads, int rows) {
  if (tokens >= 1024) return heads;
  const int least = (heads + 65534) / 65535;
  return rows > least ? rows : least;
}

template <typename T, int D>
hipError_t rotate_t(const RotateArgs& a0, hipStream_t stream) {
  constexpr int ROWS = 64 / (D * (int)sizeof(T) / 32), WAVES = kRotThreads / 64;
  RotateArgs a = a0;
  a.by_heads = FastDiv::make((uint32_t)a.heads);
  a.tokens_per_wave = a.heads < ROWS ? ROWS / a.heads : 1;
  a.run = a.heads < ROWS ? a.heads : head_run(a.n, a.heads, ROWS);
  const int per = WAVES * a.tokens_per_wave;
  const dim3 grid = token_grid(((int64_t)a.n + per - 1) / per, (a.heads + a.run - 1) / a.run);
  const int64_t bytes = (int64_t)a.n * a.heads * D * (int64_t)sizeof(T);
  if (bytes > kStreamBytes)
    hipLaunchKernelGGL((rotate_kernel<T, D, true>), grid, dim3(kRotThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((rotate_kernel<T, D, false>), grid, dim3(kRotThreads), 0, stream, a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t append_t(const AppendArgs& a0, hipStream_t stream) {
  AppendArgs a = a0;
  const int rows = (a.q != nullptr ? a.hq : 0) + 2 * a.hkv;
  a.run = head_run(a.n, rows, 64 / (D * (int)sizeof(T) / 32));
  const dim3 grid = token_grid((a.n + kRotThreads / 64 - 1) / (kRotThreads / 64),
                               (rows + a.run - 1) / a.run);
  hipLaunchKernelGGL((paged_append_kernel<T, D>), grid, dim3(kRotThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, int32_t head_dim, bool f32, hipStream_t stream) {
  if (f32) return head_dim == 64 ? rotate_t<float, 64>(a, stream) : rotate_t<float, 128>(a, stream);
  return head_dim == 64 ? rotate_t<uint16_t, 64>(a, stream) : rotate_t<uint16_t, 128>(a, stream);
}

hipError_t launch_paged_append(const AppendArgs& a, int32_t head_dim, bool f32, hipStream_t stream) {
  if (f32) return head_dim == 64 ? append_t<float, 64>(a, stream) : append_t<float, 128>(a, stream);
  return head_dim == 64 ? append_t<uint16_t, 64>(a, stream) : append_t<uint16_t, 128>(a, stream);
}

}  // namespace pbb
