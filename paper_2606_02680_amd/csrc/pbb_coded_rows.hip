// Appending to an 8-bit paged cache, and reading it back, on gfx950 (MI355X).
//
// The append takes a chunk's new keys through the norm and the rotation (pbb_norm.hip has the formulas) in
// fp64 and rounds once, to e4m3 codes under the row's power of two (pbb_coded_device.h); values are
// quantised as they come, queries go out as bf16 rows, by way of fp32.  Reading back is exact: a code times a power
// of two is a bf16 value.
//
// Bound: HBM (each row read once and written once), small calls by the launch.  Append: a lane takes 8
// channels and their partners d/2 further on, as in the rotation, and writes 8 codes of each half.  9070
// tokens of 32/8 heads, d 128, normed and turned: 43.0 us, 4.8 TB/s with its inputs in the last-level cache;
// 256 tokens: 6.8 us.

#include "pbb_norm_internal.h"
#include "pbb_coded_device.h"
#include "pbb_rows.h"

namespace pbb {
namespace {

// The sequence that packed row `tok` belongs to, or -1, where the lanes of a wave may have tokens of their
// own from `first` (the wave's lowest) to `last`.
__device__ __forceinline__ int lane_sequence(const int32_t* q_start, int batch, int tok, int first, int last,
                                             int lane) {
  int b = count_upto(q_start + 1, batch, first, lane);   // sequences that end at or before the first
  if (b < batch && __builtin_amdgcn_readfirstlane(q_start[b + 1]) <= last) {
    int lo = b, n = batch - b;   // the others of the wave: a search each
    while (n > 0) {
      const int half = n >> 1;
      const bool up = q_start[lo + half + 1] <= tok;
      lo = up ? lo + half + 1 : lo;
      n = up ? n - half - 1 : half;
    }
    b = lo;
  }
  return b < batch && q_start[b] <= tok ? b : -1;
}

// What a packed token is: its sequence (-1: none), position, and its row in the pool under KV head 0 (-1:
// no page holds its position); consecutive heads' rows are page_size apart.
struct Place {
  int b, t;
  bool skip;
  int64_t row;
};
template <typename A>
__device__ __forceinline__ Place place_of(const A& a, int tok, int first, int last, int lane) {
  Place p;
  p.b = a.uniform >= 0 ? a.by_uniform.div(tok) : lane_sequence(a.q_start, a.batch, tok, first, last, lane);
  p.t = 0;
  p.skip = true;
  p.row = -1;
  if (p.b < 0) return p;
  const Chunk c = chunk_of(p.b, a.uniform, a.uniform >= 0 ? 0 : a.q_start[p.b],
                           a.uniform >= 0 ? 0 : a.q_start[p.b + 1], a.pos[p.b], a.n);
  p.skip = c.pos < 0;
  p.t = p.skip ? 0 : c.pos + (tok - c.row0);
  if (!p.skip && p.t < a.shape.capacity) {
    const int i = a.shape.by_page.div(p.t);
    const int id = a.table[(size_t)p.b * a.shape.width + i];
    if (a.shape.is_page(id))
      p.row = (int64_t)id * a.hkv * a.shape.page_size + (p.t - i * a.shape.page_size);
  }
  return p;
}

template <int PC>
__device__ __forceinline__ uint32_t row_max(uint32_t x) {   // over the PC (4 or 8) adjacent lanes of a row
  auto step = [](uint32_t v, uint32_t o) { return v > o ? v : o; };
  x = step(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true));
  x = step(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true));
  if constexpr (PC >= 8) x = step(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true));
  return x;
}
template <int CTRL>
__device__ __forceinline__ double add_dpp64(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xf, 0xf, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xf, 0xf, true);
  return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int PC>
__device__ __forceinline__ double row_sum64(double x) {   // row_sum in fp64, PC 4 or 8
  x = add_dpp64<0x4E>(add_dpp64<0xB1>(x));
  if constexpr (PC >= 8) x = add_dpp64<0x141>(x);
  return x;
}

// To fp32: bits are cut off, and the last one is set where any of them was: what rounds the result once more, to
// fewer bits, gives what rounding x itself would.
__device__ __forceinline__ float to_odd(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t cut = (uint32_t)u & 0x1FFFFFFFu;   // (below fp32's 24 bits)
  const float f = (float)__builtin_bit_cast(double, u ^ cut);
  return __uint_as_float(__float_as_uint(f) | (cut < 1u ? cut : 1u));
}

// A key's piece through the norm and the rotation in fp64, so that its codes are those of the exact values
// (in fp32 one value in 400 thousand falls over a border between codes).  Appended and read back, 9070 tokens of
// 32/8 heads, d 128, take 57.7 us so, 55.5 with keys in fp32; 16000 of 12/2 heads, d 64, whose waves work on a
// token's queries, keys and values at once, 35.2 and 26.7; 256 of 32/8 8.7 and 7.7.  (fp32 first, and this for
// rows with a value near a border, of which there is one in a hundred: 59.0, 34.7, 10.3.)  Products with the
// weights are exact in fp32 (16 bits).
template <int PC, int D>
__device__ __forceinline__ void exact_key(const CodedAppendArgs& a, u32x4 wl, u32x4 wh, const double2* turns,
                                          float (&y)[8], float (&z)[8]) {
  typedef Piece<uint16_t> P;
  double r = 1.0;
  if (a.norm) {
    double ss = 0.0;
#pragma unroll
    for (int e = 0; e < P::N; ++e) {
      const double s = y[e], t = z[e];
      ss = __builtin_fma(s, s, __builtin_fma(t, t, ss));
    }
    const double v = __builtin_fma(row_sum64<PC>(ss), 1.0 / D, (double)a.eps);
    // 1 / sqrt(v) from fp32's by one of Newton's steps, v brought near 1 by a power of four
    const int k = __builtin_amdgcn_frexp_exp(v) >> 1;
    const double w = __builtin_ldexp(v, -2 * k);
    r = (double)(1.0f / __builtin_sqrtf((float)w));
    r = v < (double)INFINITY || v != v ? __builtin_ldexp(r * __builtin_fma(-0.5 * w * r, r, 1.5), -k) : 0.0;
  }
#pragma unroll
  for (int e = 0; e < P::N; ++e) {
    double s = y[e], t = z[e];
    if (a.norm) s = y[e] * P::get(wl, e), t = z[e] * P::get(wh, e);
    if (a.turn) {
      const double2 u = turns[e];
      const double x = __builtin_fma(s, u.x, -(t * u.y));
      t = __builtin_fma(t, u.x, s * u.y);
      s = x;
    }
    y[e] = to_odd(s * r), z[e] = to_odd(t * r);
    __builtin_amdgcn_sched_barrier(0);   // (a pair at a time: registers)
  }
}

// Grid: x (and z) = groups of tokens / waves per workgroup, y = runs of a token's query rows, key rows and
// value rows (in this order).
template <int D>
__global__ __launch_bounds__(kRotThreads) void coded_append_kernel(CodedAppendArgs a) {
  typedef uint16_t T;
  constexpr int N = Piece<T>::N;
  constexpr int ROWB = D * 2;
  constexpr int PC = ROWB / 32;
  constexpr int ROWS = 64 / PC;
  __shared__ __align__(16) double2 turns[kRotThreads / 64][ROWS * D / 4];   // (a token has two rows or more)
  const int lane = threadIdx.x & 63;
  const int tpw = a.tokens_per_wave;
  const int64_t first = ((int64_t)token_group() * (kRotThreads / 64) +
                         __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6))) * tpw;
  if (first >= a.n) return;
  const int hq = a.q != nullptr ? a.hq : 0;
  const int rows = hq + 2 * a.hkv;
  const int sub = tpw > 1 ? a.by_rows.div(lane / PC) : 0;
  const int last = min((int)first + tpw - 1, a.n - 1);
  const int tok = min((int)first + sub, last);
  const int pc = lane % PC;
  const int r1 = min(rows, (int)(blockIdx.y + 1) * a.run);
  int r = blockIdx.y * a.run + lane / PC - sub * rows;
  struct Pair { u32x4 lo, hi; };
  auto load = [&](int i) -> Pair {   // (rows past the last: the last)
    i = min(i, r1 - 1);
    const unsigned char* src =
        (i < hq ? (const unsigned char*)a.q + tok * a.q_stride + (size_t)i * ROWB
         : i < hq + a.hkv ? (const unsigned char*)a.k + tok * a.k_stride + (size_t)(i - hq) * ROWB
                          : (const unsigned char*)a.v + tok * a.v_stride + (size_t)(i - hq - a.hkv) * ROWB) + pc * 16;
    return Pair{*(const u32x4*)src, *(const u32x4*)(src + ROWB / 2)};
  };
  // the first rows and the weights go out before the search for the token's sequence and page
  Pair next = load(max(r, 0));
  auto weight = [&](const void* w) -> Pair {
    const unsigned char* p = (const unsigned char*)w + pc * 16;
    const u32x4 one = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    return w != nullptr ? Pair{*(const u32x4*)p, *(const u32x4*)(p + ROWB / 2)} : Pair{one, one};
  };
  const Pair wq = weight(a.q_weight), wk = weight(a.k_weight);
  const Place at = place_of(a, tok, (int)first, last, lane);
  float cs[N], sn[N];
  double2* const wave = turns[threadIdx.x >> 6];
  if (a.turn)
    wave_turns<T, D>(a.rope, lane, pc, sub, tpw, wave, [&](int axis, int j) {
      const int t = __shfl(at.t, j * rows * PC);   // (the first lane of token j)
      return a.rope_pos != nullptr ? a.rope_pos[(size_t)axis * a.n + min((int)first + j, last)] : t;
    }, cs, sn);
  if (at.b < 0 || sub >= tpw || first + sub >= a.n) return;
  const double2* const own = wave + sub * (D / 2) + pc * N;
  for (; r < r1; r += ROWS) {
    const bool query = r < hq, value = r >= hq + a.hkv;
    const u32x4 lo = next.lo, hi = next.hi;
    if (r + ROWS < r1) next = load(r + ROWS);
    float y[N], z[N];
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = Piece<T>::get(lo, e), z[e] = Piece<T>::get(hi, e);
    if (query) {
      if (a.norm) {
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) ss = __builtin_fmaf(y[e], y[e], __builtin_fmaf(z[e], z[e], ss));
        const float rs = 1.0f / __builtin_sqrtf(__builtin_fmaf(row_sum<PC>(ss), 1.0f / D, a.eps));
#pragma unroll
        for (int e = 0; e < N; ++e) {
          y[e] = y[e] * rs * Piece<T>::get(wq.lo, e);
          z[e] = z[e] * rs * Piece<T>::get(wq.hi, e);
        }
      }
      if (a.turn) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float s = y[e], t = z[e];
          rope_turn(s, t, cs[e], sn[e], y[e], z[e]);
        }
      }
      unsigned char* w = (unsigned char*)a.q_out + ((size_t)tok * hq + r) * ROWB + pc * 16;
      const u32x4 none = {0u, 0u, 0u, 0u};
      *(u32x4*)w = at.skip ? none : Piece<T>::put(y);
      *(u32x4*)(w + ROWB / 2) = at.skip ? none : Piece<T>::put(z);
      continue;
    }
    if (at.row < 0) break;   // (the rows after it are keys and values too)
    if (!value && (a.norm || a.turn)) exact_key<PC, D>(a, wk.lo, wk.hi, own, y, z);
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const uint32_t u = finite_bits(y[e]), v = finite_bits(z[e]);
      most = u > most ? u : most;
      most = v > most ? v : most;
    }
    const int ex = scale_exponent(row_max<PC>(most), kScaleHi);
    const float inv = power_of_two(-ex);
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] *= inv, z[e] *= inv;
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(ex == kScaleHi) != 0, 0)) {
#pragma unroll
      for (int e = 0; e < N; ++e) y[e] = cut_finite(y[e]), z[e] = cut_finite(z[e]);
    }
    const int h = r - hq - (value ? a.hkv : 0);
    const int64_t row = at.row + (int64_t)h * a.shape.page_size;
    uint8_t* w = (value ? a.v_pages : a.k_pages) + row * D + pc * 8;
    *(u32x2*)w = u32x2{codes4(y[0], y[1], y[2], y[3]), codes4(y[4], y[5], y[6], y[7])};
    *(u32x2*)(w + D / 2) = u32x2{codes4(z[0], z[1], z[2], z[3]), codes4(z[4], z[5], z[6], z[7])};
    if (pc == 0) (value ? a.v_scales : a.k_scales)[row] = (uint8_t)(ex + 127);
  }
}

// Grid as the append's, over a token's key rows and value rows: 8 lanes to a row, each 8 codes of every 64,
// so that a store's lanes write whole lines.  Six sequences of up to 32768 tokens, 8 heads, d 128 (748 MB): 140
// us, 5.3 TB/s; the 9070 tokens above 12.3 us.
constexpr int kReadRows = 8;
template <int D, bool NT>
__global__ __launch_bounds__(kRotThreads) void coded_read_kernel(CodedReadArgs a) {
  constexpr int ROWB = D * 2;
  constexpr int P = D / 64;
  constexpr int U = 2;   // rows of a lane in flight
  const int lane = threadIdx.x & 63;
  const int tpw = a.tokens_per_wave;
  const int64_t first = ((int64_t)token_group() * (kRotThreads / 64) +
                         __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6))) * tpw;
  if (first >= a.n) return;
  const int rows = 2 * a.hkv;
  const int sub = tpw > 1 ? a.by_rows.div(lane >> 3) : 0;
  const int last = min((int)first + tpw - 1, a.n - 1);
  const int tok = min((int)first + sub, last);
  const Place at = place_of(a, tok, (int)first, last, lane);
  if (at.b < 0 || sub >= tpw || first + sub >= a.n) return;
  const int pc = lane & 7;
  const int r1 = min(rows, (int)(blockIdx.y + 1) * a.run);
  for (int r0 = blockIdx.y * a.run + (lane >> 3) - sub * rows; r0 < r1; r0 += U * kReadRows) {
    u32x2 w[U][P];
    uint32_t scale[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = min(r0 + u * kReadRows, r1 - 1);
      const bool value = r >= a.hkv;
      const int64_t row = at.row + (int64_t)(r - (value ? a.hkv : 0)) * a.shape.page_size;
      const uint8_t* const c = (value ? a.v_pages : a.k_pages) + row * D + pc * 8;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        w[u][i] = u32x2{0u, 0u};
        if (at.row >= 0) {
          if constexpr (NT) w[u][i] = __builtin_nontemporal_load((const u32x2*)(c + 64 * i));
          else w[u][i] = *(const u32x2*)(c + 64 * i);
        }
      }
      scale[u] = at.row >= 0 ? (value ? a.v_scales : a.k_scales)[row] : 127u;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * kReadRows;
      if (r >= r1) break;
      const bool value = r >= a.hkv;
      const float unit = power_of_two((int)scale[u] - 127);
      unsigned char* const o = (unsigned char*)(value ? a.v : a.k) +
                               ((size_t)tok * a.hkv + (size_t)(r - (value ? a.hkv : 0))) * ROWB + pc * 16;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const u32x4 x = {values2<false>(w[u][i][0], unit), values2<true>(w[u][i][0], unit),
                         values2<false>(w[u][i][1], unit), values2<true>(w[u][i][1], unit)};
        if constexpr (NT) __builtin_nontemporal_store(x, (u32x4*)(o + 128 * i));
        else *(u32x4*)(o + 128 * i) = x;
      }
    }
  }
}

// Sets the launcher's fields; returns the grid.
template <typename A>
dim3 rows_grid(A& a, int rows, int per_pass) {
  constexpr int WAVES = kRotThreads / 64;
  a.tokens_per_wave = rows < per_pass ? per_pass / rows : 1;
  a.run = rows < per_pass ? rows : head_run(a.n, rows, per_pass);
  a.by_rows = FastDiv::make((uint32_t)rows);
  const int per = WAVES * a.tokens_per_wave;
  return token_grid(((int64_t)a.n + per - 1) / per, (rows + a.run - 1) / a.run);
}

template <int D>
hipError_t append_t(const CodedAppendArgs& a0, hipStream_t stream) {
  CodedAppendArgs a = a0;
  const dim3 grid = rows_grid(a, (a.q != nullptr ? a.hq : 0) + 2 * a.hkv, 64 / (D / 16));
  hipLaunchKernelGGL((coded_append_kernel<D>), grid, dim3(kRotThreads), 0, stream, a);
  return hipGetLastError();
}

template <int D>
hipError_t read_t(const CodedReadArgs& a0, hipStream_t stream) {
  CodedReadArgs a = a0;
  const dim3 grid = rows_grid(a, 2 * a.hkv, kReadRows);
  if ((int64_t)a.n * a.hkv * D * 4 > kStreamBytes)   // (of the rows written)
    hipLaunchKernelGGL((coded_read_kernel<D, true>), grid, dim3(kRotThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((coded_read_kernel<D, false>), grid, dim3(kRotThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_coded_append(const CodedAppendArgs& a, int32_t head_dim, hipStream_t stream) {
  return head_dim == 64 ? append_t<64>(a, stream) : append_t<128>(a, stream);
}

hipError_t launch_coded_read(const CodedReadArgs& a, int32_t head_dim, hipStream_t stream) {
  return head_dim == 64 ? read_t<64>(a, stream) : read_t<128>(a, stream);
}

}  // namespace pbb
