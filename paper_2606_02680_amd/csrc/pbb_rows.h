// Device-side helpers of the kernels that work on rows of tokens (rotation, norms, appends): the 16-byte
// pieces of a row, the sines and cosines of a token's positions, and the launches' grids.
#pragma once

#include "pbb_device.h"
#include "pbb_paged_device.h"

namespace pbb {

constexpr int kRotThreads = 256;
// A grid's x has fewer than 2^32 threads: groups of tokens beyond kGridX go on along z.
constexpr int kGridX = 1 << 23;
__device__ __forceinline__ int token_group() { return (int)(blockIdx.z * kGridX + blockIdx.x); }
inline dim3 token_grid(int64_t groups, int runs) {
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

// A constant of an fp64 sum, in scalar registers where it is used (else the compiler keeps all of a sum's in
// vector registers throughout the kernel).
__device__ __forceinline__ double scalar_constant(double x) {
  asm volatile("" : "+s"(x));
  return x;
}
// cos and sin of position * rate whole turns to some 2^-36: of what is left of the nearest quarter turn, an eighth
// of a turn either way, by their Taylor sums.  The whole turns come off the exact product (31 bits times 53: a
// rounded one would be off by half a turn and more at far positions and rates above 2^21), and twice, since
// those of a product above 2^53 leave what its rounding took.
__device__ __forceinline__ void cos_sin64(double position, double rate, double& cs, double& sn) {
  const double part = __builtin_fma(position, rate, -__builtin_rint(position * rate));
  const double f = part - __builtin_rint(part);
  const double quarter = __builtin_rint(4.0 * f);
  const double x = (f - 0.25 * quarter) * scalar_constant(6.283185307179586477), z = x * x;
  auto next = [&](double sum, double k) { return __builtin_fma(sum, z, scalar_constant(k)); };
  double s = __builtin_fma(z, scalar_constant(-1.0 / 39916800.0), scalar_constant(1.0 / 362880.0));
  s = next(next(next(s, -1.0 / 5040.0), 1.0 / 120.0), -1.0 / 6.0);
  s = __builtin_fma(s * z, x, x);
  double c = __builtin_fma(z, scalar_constant(1.0 / 479001600.0), scalar_constant(-1.0 / 3628800.0));
  c = next(next(next(c, 1.0 / 40320.0), -1.0 / 720.0), 1.0 / 24.0);
  c = __builtin_fma(__builtin_fma(c, z, -0.5), z, 1.0);
  const int q = (int)quarter & 3;
  const double a = q & 1 ? s : c, b = q & 1 ? c : s;
  cs = q == 1 || q == 2 ? -a : a;
  sn = q >= 2 ? -b : b;
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

// The same, rounded once from cos_sin64, for a wave that works on `tokens` tokens, this lane on the one with
// index `sub`: the lanes work out a pair each and take their pieces' from one another through LDS (`turns`:
// tokens * D / 2 of the wave's own, float2 or double2, which stay there).  position(axis, j): of token j.  All
// lanes take part.  (With piece_turns' sums, whose fp64 steps each row of the wave does again, 9070 tokens
// took 48.7 us to append, 40.0 shared; 4 x 16384 tokens 245 and 231 to norm.)
template <typename T, int D, typename V, typename F>
__device__ __forceinline__ void wave_turns(const RopeArgs& r, int lane, int pc, int sub, int tokens, V* turns,
                                           F&& position, float (&cs)[Piece<T>::N], float (&sn)[Piece<T>::N]) {
  constexpr int N = Piece<T>::N;
#pragma unroll 1
  for (int first = 0; first < tokens * (D / 2); first += 64) {
    // (lanes past the last pair do it again: position() may ask other lanes, which have to be there)
    const int i = min(first + lane, tokens * (D / 2) - 1), j = i / (D / 2), c = i % (D / 2);
    double cd, sd;
    cos_sin64((double)position(r.axis[c], j), r.turns[c], cd, sd);
    V t;
    t.x = cd, t.y = sd;
    turns[i] = t;
  }
  __builtin_amdgcn_wave_barrier();   // (a wave's LDS accesses keep their order)
  const V* const own = turns + min(sub, tokens - 1) * (D / 2) + pc * N;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const V u = own[e];
    cs[e] = (float)u.x, sn[e] = (float)u.y;
  }
  __builtin_amdgcn_wave_barrier();
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

// The sum over the PC (4, 8 or 16) adjacent lanes that hold a row, in all of them, bit for bit the same
// in each (partners' sums are added pairwise).
template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
template <int PC>
__device__ __forceinline__ float row_sum(float x) {
  x = add_dpp<0xB1>(x);                        // quad_perm: lane ^ 1
  x = add_dpp<0x4E>(x);                        // lane ^ 2
  if constexpr (PC >= 8) x = add_dpp<0x141>(x);   // row_half_mirror: the other quad of eight
  if constexpr (PC >= 16) x = add_dpp<0x140>(x);  // row_mirror: the other eight of sixteen
  return x;
}

// The sequence that packed row `tok` belongs to, or -1: the number of sequences whose rows end at or
// before it (every lane of the wave takes part; q_start never falls).
__device__ __forceinline__ int sequence_of(const int32_t* q_start, int batch, int tok, int lane) {
  const int b = count_upto(q_start + 1, batch, tok, lane);
  if (b >= batch) return -1;
  return __builtin_amdgcn_readfirstlane(q_start[b]) <= tok ? b : -1;
}

// Heads per workgroup row of the grid: all of a token's, unless the tokens alone leave the chip
// short of waves; then as few as a wave takes at once, and no more than 65535 runs (2000 tokens of 48
// rows: 11.5 us, 13.5 with a run per 8 rows; 256 tokens: 5.0 us so; inputs in the last-level cache).
inline int head_run(int tokens, int heads, int rows) {
  if (tokens >= 1024) return heads;
  const int least = (heads + 65534) / 65535;
  return rows > least ? rows : least;
}

}  // namespace pbb
