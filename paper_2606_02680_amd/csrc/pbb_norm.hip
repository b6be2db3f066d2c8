// Per-head norms with rotation, and their gradients, on gfx950 (MI355X).
//
// A row x of a query or key head becomes y = R(p) (x r w): r = 1 / sqrt(mean x^2 + eps), w the kind's
// weight, R the rotation of channel pairs (c, c + d/2) by the token's positions.  For a gradient dy of
// the result: g = R^T dy, dw = sum over rows of g x r, and with a = g w and s = mean(a x) r
//   dx = r (a - (x r) s).
// All in fp32, rounded once to the rows' type; weights' gradients stay fp32.
//
// Bound: HBM (forward: each row read and written once; backward: two rows read, one written).  A lane
// takes the 16-byte piece of channels c.. and its partner d/2 further on, as in the rotation, so PC
// lanes hold a row and its sums are taken over them on the VALU (row_sum).

#include "pbb_rows.h"
#include "pbb_norm_internal.h"

namespace pbb {
namespace {

// The sum over the 64 / PC lanes that hold the same piece of different rows, in all of them.
template <int PC>
__device__ __forceinline__ float piece_sum(float x) {
  if constexpr (PC <= 4) x = add_dpp<0x124>(x);   // row_ror: 4 lanes on of sixteen
  if constexpr (PC <= 8) x = add_dpp<0x128>(x);   // 8 lanes on
  return sum_xor16_32(x);
}

// A piece of a weight, as floats (null: ones).
template <typename T>
struct Weights {
  float lo[Piece<T>::N], hi[Piece<T>::N];
  __device__ __forceinline__ Weights(const void* w, int pc, int half_bytes) {
    u32x4 a, b;
    if (w != nullptr) {
      a = *(const u32x4*)((const unsigned char*)w + pc * 16);
      b = *(const u32x4*)((const unsigned char*)w + half_bytes + pc * 16);
    }
#pragma unroll
    for (int e = 0; e < Piece<T>::N; ++e) {
      lo[e] = w != nullptr ? Piece<T>::get(a, e) : 1.0f;
      hi[e] = w != nullptr ? Piece<T>::get(b, e) : 1.0f;
    }
  }
};

template <bool NT>
__device__ __forceinline__ u32x4 load16(const unsigned char* p) {
  if constexpr (NT) return __builtin_nontemporal_load((const u32x4*)p);
  else return *(const u32x4*)p;
}
template <bool NT>
__device__ __forceinline__ void store16(u32x4 v, unsigned char* p) {
  if constexpr (NT) __builtin_nontemporal_store(v, (u32x4*)p);
  else *(u32x4*)p = v;
}

// Workgroups 0 .. part[0].blocks - 1 take queries, the others keys.  A unit of work is a run of heads of
// the tokens of a workgroup's waves; where a kind has fewer heads than a wave takes rows, a wave takes
// several tokens.  Queries and keys in one launch: of small calls the launch is all (one token of 12/2 heads:
// 3.6 us).  4 x 16384 tokens of 32/8 heads, d 128, bf16: 235 us, 1.34 GB at 5.7 TB/s, past the 4.9 of a large
// copy by the non-temporal hint.
template <typename T, int D, bool NT>
__global__ __launch_bounds__(kNormThreads) void norm_rotate_kernel(NormArgs a) {
  constexpr int N = Piece<T>::N;
  constexpr int ROWB = D * (int)sizeof(T);
  constexpr int PC = ROWB / 32;
  constexpr int ROWS = 64 / PC;
  __shared__ __align__(16) float2 turns[kNormThreads / 64][ROWS * D / 2];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const bool keys = (int)blockIdx.x >= a.part[0].blocks;
  const NormPart& p = a.part[keys ? 1 : 0];
  const int block = (int)blockIdx.x - (keys ? a.part[0].blocks : 0);
  const int row = lane / PC, pc = lane % PC;
  const int sub = p.tokens_per_wave > 1 ? p.by_heads.div(row) : 0;
  const Weights<T> w(p.weight, pc, ROWB / 2);
  for (int u = block; u < p.units; u += p.blocks) {
    const int group = p.by_runs.div(u);
    const int first = (u - group * (int)p.by_runs.d) * p.run;
    const int64_t tok0 = ((int64_t)group * (kNormThreads / 64) + wave) * p.tokens_per_wave, tok = tok0 + sub;
    if (tok0 >= a.n) continue;
    float cs[N], sn[N];
    if (a.turn)   // (rounded once to fp32, in bf16 too, as in the 8-bit append, whose queries are these bit for bit)
      wave_turns<T, D>(a.rope, lane, pc, sub, p.tokens_per_wave, turns[wave], [&](int axis, int j) {
        return a.positions[(size_t)axis * a.n + min(tok0 + j, (int64_t)a.n - 1)];
      }, cs, sn);
    if (sub >= p.tokens_per_wave || tok >= a.n) continue;
    const unsigned char* x = (const unsigned char*)p.x + tok * p.x_stride + pc * 16;
    unsigned char* o = (unsigned char*)p.out + tok * p.out_stride + pc * 16;
    const int h1 = min(p.heads, first + p.run);
    for (int h = first + row - sub * p.heads; h < h1; h += ROWS) {
      const unsigned char* src = x + (size_t)h * ROWB;
      const u32x4 lo = load16<NT>(src), hi = load16<NT>(src + ROWB / 2);
      float f[N], g[N], ss = 0.0f;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        f[e] = Piece<T>::get(lo, e), g[e] = Piece<T>::get(hi, e);
        ss = __builtin_fmaf(f[e], f[e], __builtin_fmaf(g[e], g[e], ss));
      }
      const float r = 1.0f / __builtin_sqrtf(__builtin_fmaf(row_sum<PC>(ss), 1.0f / D, a.eps));
      float y[N], z[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float s = f[e] * r * w.lo[e], t = g[e] * r * w.hi[e];
        if (a.turn) rope_turn(s, t, cs[e], sn[e], y[e], z[e]);
        else y[e] = s, z[e] = t;
      }
      unsigned char* dst = o + (size_t)h * ROWB;
      store16<NT>(Piece<T>::put(y), dst);
      store16<NT>(Piece<T>::put(z), dst + ROWB / 2);
    }
  }
}

// Workgroups as in the forward kernel, all heads of a token to a wave.  Each sums its rows' part of the
// weight's gradient: lanes over their rows, then the lanes of a piece, then the waves, in an order that
// the shapes alone determine.  2 x 16384 tokens of 32/8 heads, d 128, bf16: 188 us, 1.01 GB at 5.4 TB/s, and
// 6.6 us for the sums of the workgroups' parts; 5041 of 16/4 heads, d 64, fp32: 15.6 and 3.8 us.
template <typename T, int D, bool NT>
__global__ __launch_bounds__(kNormThreads) void norm_rotate_backward_kernel(NormArgs a) {
  constexpr int N = Piece<T>::N;
  constexpr int ROWB = D * (int)sizeof(T);
  constexpr int PC = ROWB / 32;
  constexpr int ROWS = 64 / PC;
  constexpr int NW = kNormThreads / 64;
  __shared__ float sums[NW][D];
  __shared__ __align__(16) float2 turns[NW][ROWS * D / 2];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const bool keys = (int)blockIdx.x >= a.part[0].blocks;
  const NormPart& p = a.part[keys ? 1 : 0];
  const int block = (int)blockIdx.x - (keys ? a.part[0].blocks : 0);
  const int row = lane / PC, pc = lane % PC;
  const int sub = p.tokens_per_wave > 1 ? p.by_heads.div(row) : 0;
  const Weights<T> w(p.weight, pc, ROWB / 2);
  float dlo[N], dhi[N];
#pragma unroll
  for (int e = 0; e < N; ++e) dlo[e] = dhi[e] = 0.0f;
  struct Pair { u32x4 xl, xh, gl, gh; };   // a row's piece and its gradient's
  for (int u = block; u < p.units; u += p.blocks) {
    const int64_t tok0 = ((int64_t)u * NW + wave) * p.tokens_per_wave;
    if (tok0 >= a.n) continue;
    const int64_t tok = min(tok0 + min(sub, p.tokens_per_wave - 1), (int64_t)a.n - 1);
    const unsigned char* x = (const unsigned char*)p.x + tok * p.x_stride + pc * 16;
    const unsigned char* gr = (const unsigned char*)p.grad + tok * p.grad_stride + pc * 16;
    unsigned char* o = (unsigned char*)p.out + tok * p.out_stride + pc * 16;
    auto load = [&](int h) -> Pair {
      const size_t at = (size_t)h * ROWB;
      return Pair{load16<NT>(x + at), load16<NT>(x + at + ROWB / 2), load16<NT>(gr + at),
                  load16<NT>(gr + at + ROWB / 2)};
    };
    // (the first rows' loads go out before the positions', whose sines and cosines are a chain of their own)
    int h = row - sub * p.heads;
    Pair r0 = load(min(h, p.heads - 1));
    float cs[N], sn[N];
    if (a.turn)
      wave_turns<T, D>(a.rope, lane, pc, sub, p.tokens_per_wave, turns[wave], [&](int axis, int j) {
        return a.positions[(size_t)axis * a.n + min(tok0 + j, (int64_t)a.n - 1)];
      }, cs, sn);
    if (sub >= p.tokens_per_wave || tok0 + sub >= a.n) continue;
    for (; h < p.heads; h += ROWS) {
      const size_t at = (size_t)h * ROWB;
      const Pair v = r0;
      float f[N], g[N], y[N], z[N], ss = 0.0f, dot = 0.0f;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        f[e] = Piece<T>::get(v.xl, e), g[e] = Piece<T>::get(v.xh, e);
        const float s = Piece<T>::get(v.gl, e), t = Piece<T>::get(v.gh, e);
        if (a.turn) rope_turn(s, t, cs[e], sn[e], y[e], z[e]);
        else y[e] = s, z[e] = t;
        ss = __builtin_fmaf(f[e], f[e], __builtin_fmaf(g[e], g[e], ss));
        dot = __builtin_fmaf(y[e] * w.lo[e], f[e], __builtin_fmaf(z[e] * w.hi[e], g[e], dot));
      }
      const float r = 1.0f / __builtin_sqrtf(__builtin_fmaf(row_sum<PC>(ss), 1.0f / D, a.eps));
      const float s = row_sum<PC>(dot) * r * (1.0f / D);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float nl = f[e] * r, nh = g[e] * r;
        dlo[e] = __builtin_fmaf(y[e], nl, dlo[e]);
        dhi[e] = __builtin_fmaf(z[e], nh, dhi[e]);
        y[e] = r * __builtin_fmaf(-nl, s, y[e] * w.lo[e]);
        z[e] = r * __builtin_fmaf(-nh, s, z[e] * w.hi[e]);
      }
      if (h + ROWS < p.heads) r0 = load(h + ROWS);
      store16<NT>(Piece<T>::put(y), o + at);
      store16<NT>(Piece<T>::put(z), o + at + ROWB / 2);
    }
  }
  if (p.dweight == nullptr) return;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    dlo[e] = piece_sum<PC>(dlo[e]);
    dhi[e] = piece_sum<PC>(dhi[e]);
    if (row == 0) {
      sums[wave][pc * N + e] = dlo[e];
      sums[wave][D / 2 + pc * N + e] = dhi[e];
    }
  }
  __syncthreads();
  // (the only workgroup of its kind writes the result itself)
  float* const out = p.blocks == 1 ? p.dweight : a.partials + (size_t)blockIdx.x * D;
  for (int c = threadIdx.x; c < D; c += kNormThreads) {
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < NW; ++v) s += sums[v][c];
    out[c] = s;
  }
}

// Sums the workgroups' parts of the weights' gradients: four channels of a kind to a workgroup, whose
// threads take every 512th part (5000 tokens of 12/2 heads, d 64: 12.7 us with
// the gradients, 13.6 with 16 channels to a workgroup).
constexpr int kSumThreads = 512;
template <int D>
__global__ __launch_bounds__(kSumThreads) void norm_weight_sum_kernel(NormArgs a) {
  __shared__ f32x4 sums[kSumThreads / 64];
  const int kind = (int)blockIdx.x / (D / 4);
  const NormPart& p = a.part[kind];
  if (p.dweight == nullptr || p.blocks == 1) return;   // (0 of a call of no tokens or no heads: zeros)
  const int channel = ((int)blockIdx.x % (D / 4)) * 4;
  const float* parts = a.partials + (size_t)(kind ? a.part[0].blocks : 0) * D + channel;
  f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int i = threadIdx.x; i < p.blocks; i += kSumThreads) s += *(const f32x4*)(parts + (size_t)i * D);
#pragma unroll
  for (int e = 0; e < 4; ++e) s[e] = sum_xor16_32(row_sum<16>(s[e]));
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x >= 4) return;
  float t = 0.0f;
#pragma unroll
  for (int w = 0; w < kSumThreads / 64; ++w) t += sums[w][threadIdx.x];
  p.dweight[channel + threadIdx.x] = t;
}

template <typename T, int D>
struct Rows {
  static constexpr int ROWS = 64 / (D * (int)sizeof(T) / 32);
};

bool streams(const NormArgs& a, int rows_per_pass, int64_t row_bytes) {
  return (int64_t)a.n * (a.part[0].heads + a.part[1].heads) * row_bytes * rows_per_pass > 2 * kStreamBytes;
}

template <typename T, int D>
hipError_t forward_t(const NormArgs& a0, hipStream_t stream) {
  constexpr int ROWS = Rows<T, D>::ROWS, WAVES = kNormThreads / 64;
  NormArgs a = a0;
  for (NormPart& p : a.part) {
    if (p.heads == 0) {
      p.units = p.blocks = 0;
      continue;
    }
    p.tokens_per_wave = norm_tokens_per_wave(p.heads, ROWS);
    p.run = p.heads < ROWS ? p.heads : head_run(a.n, p.heads, ROWS);
    const int runs = (p.heads + p.run - 1) / p.run;
    const int64_t per = (int64_t)WAVES * p.tokens_per_wave;
    p.units = (int32_t)((a.n + per - 1) / per * runs);   // (runs > 1 with fewer than 1024 tokens only)
    p.blocks = p.units < kGridX / 2 ? p.units : kGridX / 2;
    p.by_heads = FastDiv::make((uint32_t)p.heads);
    p.by_runs = FastDiv::make((uint32_t)runs);
  }
  const dim3 grid((unsigned)(a.part[0].blocks + a.part[1].blocks));
  if (streams(a, 2, D * (int64_t)sizeof(T)))
    hipLaunchKernelGGL((norm_rotate_kernel<T, D, true>), grid, dim3(kNormThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((norm_rotate_kernel<T, D, false>), grid, dim3(kNormThreads), 0, stream, a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t backward_t(const NormArgs& a0, hipStream_t stream) {
  constexpr int ROWS = Rows<T, D>::ROWS, WAVES = kNormThreads / 64;
  NormArgs a = a0;
  bool more = false;
  for (NormPart& p : a.part) {
    if (p.heads == 0) {   // (no rows: its weight's gradient is zeros)
      p.units = p.blocks = 0;
      more |= p.dweight != nullptr;
      continue;
    }
    p.tokens_per_wave = norm_tokens_per_wave(p.heads, ROWS);
    const int64_t per = (int64_t)WAVES * p.tokens_per_wave;
    p.units = (int32_t)((a.n + per - 1) / per);
    p.blocks = norm_grad_blocks(a.n, p.heads, a.part[0].heads + a.part[1].heads, ROWS, D * (int)sizeof(T));
    p.by_heads = FastDiv::make((uint32_t)p.heads);
    more |= p.dweight != nullptr && p.blocks != 1;
  }
  const dim3 grid((unsigned)(a.part[0].blocks + a.part[1].blocks));
  if (a.n == 0)
    ;   // no rows, and the weights' gradients are zeros
  else if (streams(a, 3, D * (int64_t)sizeof(T)))
    hipLaunchKernelGGL((norm_rotate_backward_kernel<T, D, true>), grid, dim3(kNormThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((norm_rotate_backward_kernel<T, D, false>), grid, dim3(kNormThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !more) return e;
  hipLaunchKernelGGL((norm_weight_sum_kernel<D>), dim3(2 * D / 4), dim3(kSumThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rotate(const NormArgs& a, int32_t head_dim, bool f32, hipStream_t stream) {
  if (f32) return head_dim == 64 ? forward_t<float, 64>(a, stream) : forward_t<float, 128>(a, stream);
  return head_dim == 64 ? forward_t<uint16_t, 64>(a, stream) : forward_t<uint16_t, 128>(a, stream);
}

hipError_t launch_norm_rotate_backward(const NormArgs& a, int32_t head_dim, bool f32, hipStream_t stream) {
  if (f32) return head_dim == 64 ? backward_t<float, 64>(a, stream) : backward_t<float, 128>(a, stream);
  return head_dim == 64 ? backward_t<uint16_t, 64>(a, stream) : backward_t<uint16_t, 128>(a, stream);
}

}  // namespace pbb
