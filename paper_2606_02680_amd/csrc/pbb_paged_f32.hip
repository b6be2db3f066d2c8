// fp32 attention over a paged KV cache on gfx950 (MI355X): fp32 operands, weights and accumulation.
//
// The work unit is that of the bf16 kernel with tiles of floor(64 / G) tokens, 16 columns per wave,
// and 16-key steps, each within one page: LDS DMA, every wave a quarter of the step's K and V rows.
// Products on v_mfma_f32_16x16x4_f32 with the channel and key orders of the fp32 decode kernel:
//   scores  lane (c16, j4) of MFMA m contracts channel 16 (m / 4) + 4 j4 + m mod 4 of key row c16 (one
//           16-byte LDS read per four MFMAs); the result gives it keys 4 j4 .. +3 of column c16;
//   values  row r of output block nb is channel 64 (nb / 4) + 4 r + nb mod 4, MFMA (nb, m) contracts
//           key 4 j4 + m: the lane's own weight, and one 16-byte read of that key's row for four nb.
// Rounding: the matrix core rounds every product that it adds, so scores run in eight chains and a
// step's 16 keys enter the output as one partial sum.
// LDS: K pieces are stored at slot p ^ row (their readers walk rows, 512 or 256 bytes apart, which
// would share their banks); V pieces in order (their readers walk a row).

#include "pbb_paged_device.h"

namespace pbb {
namespace {

constexpr int kF32Waves = 4;
static_assert(kPagedColsF32 == 16 * kF32Waves && kPagedStepF32 == 16, "tile");
constexpr int kF32Stages = 3;

__device__ __forceinline__ bool is_special(float x) {
  return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u;
}

// Few columns: tiles of at most 16.  The 16-key steps of a piece are dealt to the waves one by one;
// a wave reads its rows straight into registers as operands (as the fp32 decode does: 64 contiguous
// bytes of each of 16 key rows, 256 of each of 4 value rows per 16-byte load), the next step's loads in
// flight while it computes.  Bound: HBM, by the register loads that 8 waves per CU hold in flight.
template <int D, bool IN_PLACE>
__device__ __forceinline__ void narrow_walk_f32(const PagedArgs& a, const PagedItem& it, int g,
                                                unsigned char* smem) {
  constexpr int NW = kF32Waves;
  constexpr int KM = D / 4;
  constexpr int E = D / 16;
  constexpr int KQ = KM / 4;    // 16-byte loads of a lane's key channels
  constexpr int VQ = E / 4;     // and of each of its four value rows
  constexpr int ROWB = D * 4;
  constexpr int COLS = kPagedNarrowCols;

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
  const NarrowOut<float, D, NW> result{a, it, g, cols};
  if (it.c.pos < 0) {
    result.skip(tid);
    return;
  }

  const int t0 = it.c.pos;
  const int t_last = t0 + tokens - 1;
  int s0 = sh.support_lo(t0) >> 4;
  int nsteps = max(0, (min(t_last, sh.capacity - 1) >> 4) - s0 + 1);
  if (nsteps == 0) s0 = 0;   // (all past the table: positions whose next steps pass 2^31)
  if (it.ways > 1) {
    const int lo = (int)((int64_t)it.piece * nsteps / it.ways);
    const int hi = (int)((int64_t)(it.piece + 1) * nsteps / it.ways);
    s0 += lo;
    nsteps = hi - lo;
  }
  const int s1 = s0 + nsteps;   // steps [s0, s1): keys 16 s .. +15

  const int cp = min(pl.by_group.div(c16), tokens - 1);
  const bool valid = c16 < cols;
  const int tcol = valid ? t0 + cp : -1;
  const int lo_c = sh.support_lo(t0 + cp);
  float qf[KM];
  {
    const float* qrow = (const float*)((const unsigned char*)a.q + (row0 + cp) * a.q_stride +
                                       (int64_t)(g * G + (valid ? c16 - cp * G : 0)) * ROWB) + 4 * j4;
#pragma unroll
    for (int x = 0; x < KM / 4; ++x) {
      const f32x4 v = *(const f32x4*)(qrow + 16 * x);
#pragma unroll
      for (int e = 0; e < 4; ++e) qf[4 * x + e] = valid ? v[e] * a.scale_log2 : 0.0f;
    }
  }

  const int32_t* const table = a.table + (size_t)it.b * sh.width;
  const uint32_t page_bytes = (uint32_t)sh.page_size * ROWB;   // of one KV head
  const uint64_t page_stride = (uint64_t)page_bytes * (uint32_t)a.hkv;
  const unsigned char* const keys = (const unsigned char*)a.k_pages + (uint64_t)page_bytes * (uint32_t)g;
  const unsigned char* const values = (const unsigned char*)a.v_pages + (uint64_t)page_bytes * (uint32_t)g;
  struct Entry { int id; uint32_t slot; };
  auto fetch = [&](int st) -> Entry {
    const int i = min(sh.by_page.div(16 * st), sh.width - 1);
    return Entry{scalar_word(table, i), (uint32_t)(16 * st - i * sh.page_size) * ROWB};
  };
  auto load = [&](const Entry& e, f32x4 (&kb)[KQ], f32x4 (&vb)[4][VQ]) __attribute__((always_inline)) {
    const uint64_t off = (sh.is_page(e.id) ? (uint32_t)e.id : 0u) * page_stride + e.slot;
    const unsigned char* kp = keys + off + (uint32_t)(c16 * ROWB + 16 * j4);
    const unsigned char* vp = values + off + (uint32_t)(4 * j4 * ROWB + 16 * c16);
#pragma unroll
    for (int q = 0; q < KQ; ++q) kb[q] = __builtin_nontemporal_load((const f32x4*)(kp + 64 * q));
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int q = 0; q < VQ; ++q)
        vb[k][q] = __builtin_nontemporal_load((const f32x4*)(vp + k * ROWB + 256 * q));
  };
  // steps whose keys all lie in every column's support
  const int ua = (sh.support_lo(t_last) + 15) >> 4;
  const int ub = (t0 + 1) >> 4;

  float m = valid ? kNoScore : 0.0f, lsum = 0.0f;
  f32x4 acc[E];
#pragma unroll
  for (int nb = 0; nb < E; ++nb) acc[nb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  bool first = true;

  auto compute = [&](int st, bool gone, const f32x4 (&kb)[KQ], const f32x4 (&vb)[4][VQ])
      __attribute__((always_inline)) {
    f32x4 sp[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) sp[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < KM; ++i)
      sp[i & 7] = __builtin_amdgcn_mfma_f32_16x16x4f32(kb[i >> 2][i & 3], qf[i], sp[i & 7], 0, 0, 0);
    f32x4 s = ((sp[0] + sp[1]) + (sp[2] + sp[3])) + ((sp[4] + sp[5]) + (sp[6] + sp[7]));
    const bool masked = st < ua || st >= ub || gone;
    const int k0 = 16 * st + 4 * j4;
    bool sees[4] = {true, true, true, true};
    if (masked) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sees[e] = e >= lo_c - k0 && e <= tcol - k0 && !gone;
        s[e] = sees[e] ? s[e] : kNegInf;
      }
    }
    const float mx = max_xor16_32(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])));
    const bool grow = mx > m + 8.0f || (first && mx > m);
    first = false;
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
      const float alpha = grow ? fast_exp2(m - mx) : 1.0f;
      m = grow ? mx : m;
      lsum *= alpha;
#pragma unroll
      for (int nb = 0; nb < E; ++nb) acc[nb] *= alpha;
    }
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = fast_exp2(s[e] - m);
    lsum += (p[0] + p[1]) + (p[2] + p[3]);
    bool odd = false;
    if (masked) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int q = 0; q < VQ; ++q)
#pragma unroll
          for (int x = 0; x < 4; ++x) odd |= is_special(vb[k][q][x]);
    }
    const bool apart = masked && __builtin_amdgcn_ballot_w64(odd) != 0;
#pragma unroll
    for (int nb = 0; nb < E; ++nb) {
      f32x4 part = {0.0f, 0.0f, 0.0f, 0.0f};
      if (!apart) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          part = __builtin_amdgcn_mfma_f32_16x16x4f32(vb[k][nb >> 2][nb & 3], p[k], part, 0, 0, 0);
      } else {   // infinities and NaN, counted for the columns that see their key
        f32x4 cu = {0.0f, 0.0f, 0.0f, 0.0f}, cd = cu;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float w = vb[k][nb >> 2][nb & 3], one = sees[k] ? 1.0f : 0.0f;
          const bool sp1 = is_special(w), nan = w != w;
          cu = __builtin_amdgcn_mfma_f32_16x16x4f32(sp1 && (nan || w > 0.0f) ? 1.0f : 0.0f, one, cu, 0, 0, 0);
          cd = __builtin_amdgcn_mfma_f32_16x16x4f32(sp1 && (nan || w < 0.0f) ? 1.0f : 0.0f, one, cd, 0, 0, 0);
          part = __builtin_amdgcn_mfma_f32_16x16x4f32(sp1 ? 0.0f : w, p[k], part, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          part[e] += (cu[e] > 0.0f ? -kNegInf : 0.0f) + (cd[e] > 0.0f ? kNegInf : 0.0f);
      }
      acc[nb] += part;
    }
  };

  f32x4 ka[KQ], kb[KQ], va[4][VQ], vb[4][VQ];
  int st = s0 + wave;
  if (st < s1) {
    Entry e0 = fetch(st), e1 = fetch(min(st + NW, s1 - 1));
    load(e0, ka, va);
    while (true) {
      const bool g0 = !sh.is_page(e0.id);
      if (st + NW < s1) load(e1, kb, vb);
      e0 = fetch(min(st + 2 * NW, s1 - 1));
      compute(st, g0, ka, va);
      st += NW;
      if (st >= s1) break;
      const bool g1 = !sh.is_page(e1.id);
      if (st + NW < s1) load(e0, ka, va);
      e1 = fetch(min(st + 2 * NW, s1 - 1));
      compute(st, g1, kb, vb);
      st += NW;
      if (st >= s1) break;
    }
  }

  lsum = sum_xor16_32(lsum);
#pragma unroll
  for (int y = 0; y < E / 4; ++y)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(f32x4*)(result.outputs(smem) + (wave * COLS + c16) * D + 64 * y + 16 * j4 + 4 * i) =
          f32x4{acc[4 * y][i], acc[4 * y + 1][i], acc[4 * y + 2][i], acc[4 * y + 3][i]};
  if (j4 == 0) {
    result.references(smem)[wave * COLS + c16] = m;
    result.sums(smem)[wave * COLS + c16] = lsum;
  }
  result.template finish<IN_PLACE, IN_PLACE ? COLS : kPagedColsF32>(tid, smem, 16 * s0, 16 * s1 - 1);
}

template <int D>
__global__ __launch_bounds__(kF32Waves * 64) __attribute__((amdgpu_waves_per_eu(2)))
void paged_narrow_f32_kernel(PagedArgs a) {
  __shared__ __align__(1024) unsigned char smem[NarrowOut<float, D, kF32Waves>::LDS];
  const int lane = threadIdx.x & 63;
  const int item = a.plan.by_hkv.div((int)blockIdx.x);
  const int g = (int)blockIdx.x - item * a.hkv;
  PagedItem it;
  if (!find_item<false>(a, item, lane, it)) return;
  narrow_walk_f32<D, true>(a, it, g, smem);
}

template <int D>
__global__ __launch_bounds__(kF32Waves * 64) __attribute__((amdgpu_waves_per_eu(2)))
void paged_f32_kernel(PagedArgs a) {
  constexpr int NW = kF32Waves;
  constexpr int KM = D / 4;             // MFMAs of a score tile
  constexpr int E = D / 16;             // output blocks
  constexpr int ROWB = D * 4;
  constexpr int PPR = D / 4;            // 16-byte pieces per row
  constexpr int RPB = 64 / PPR;         // rows per 1 KiB DMA
  constexpr int TILE = 16 * ROWB;
  constexpr int BUF = 2 * TILE;
  constexpr int STAGES = kF32Stages;
  constexpr int OPS = BUF / 1024 / NW;  // DMA instructions of a wave per step
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
    static_assert(sizeof(smem) >= NarrowOut<float, D, NW>::LDS - 16, "LDS");   // (no word: not merged here)
    narrow_walk_f32<D, false>(a, it, g, smem);
    return;
  }
  const int p0 = it.tile * pl.tq;
  const int tokens = min(pl.tq, it.c.count - p0);
  const int64_t row0 = (int64_t)it.c.row0 + p0;
  const int cols = tokens * G;
  auto address = [&](int col) -> int64_t {   // output row of a column
    const int cp = pl.by_group.div(col);
    return (row0 + cp) * a.hq + (int64_t)(g * G + col - cp * G);
  };
  auto lse_at = [&](int col) -> int64_t {
    const int cp = pl.by_group.div(col);
    return (int64_t)(g * G + col - cp * G) * a.n + row0 + cp;
  };

  if (it.c.pos < 0) {   // a skipped sequence, never cut: zeros, no log-partition
    for (int i = tid; i < cols * PPR; i += NW * 64) {
      const int col = i / PPR;
      *(f32x4*)((unsigned char*)a.out + address(col) * ROWB + (i - col * PPR) * 16) =
          f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    if (a.lse != nullptr)
      for (int col = tid; col < cols; col += NW * 64) a.lse[lse_at(col)] = kNegInf;
    return;
  }

  const int t0 = it.c.pos + p0;
  const int t_last = t0 + tokens - 1;
  int s_first = sh.support_lo(t0) >> 4;
  int nsteps = max(0, (min(t_last, sh.capacity - 1) >> 4) - s_first + 1);
  if (nsteps == 0) s_first = 0;   // (all past the table: positions whose next steps pass 2^31)
  if (it.ways > 1) {
    const int lo = (int)((int64_t)it.piece * nsteps / it.ways);
    const int hi = (int)((int64_t)(it.piece + 1) * nsteps / it.ways);
    s_first += lo;
    nsteps = hi - lo;
  }

  // This lane's column (past the tile's tokens: the last token's row, a zero query, no key seen).
  const int col = wave * 16 + c16;
  const int cp = min(pl.by_group.div(col), tokens - 1);
  const bool valid = col < cols;
  const int tcol = valid ? t0 + cp : -1;
  const int lo_c = sh.support_lo(t0 + cp);
  float qf[KM];
  {
    const float* qrow = (const float*)((const unsigned char*)a.q + (row0 + cp) * a.q_stride +
                                       (int64_t)(g * G + (valid ? col - cp * G : 0)) * ROWB) + 4 * j4;
#pragma unroll
    for (int x = 0; x < KM / 4; ++x) {
      const f32x4 v = *(const f32x4*)(qrow + 16 * x);
#pragma unroll
      for (int e = 0; e < 4; ++e) qf[4 * x + e] = valid ? v[e] * a.scale_log2 : 0.0f;
    }
  }

  // DMA: waves 0 and 1 load K, 2 and 3 V, eight rows each.  `gone`: one bit per step.
  const unsigned char* const pool = (const unsigned char*)(wave >= 2 ? a.v_pages : a.k_pages);
  const int32_t* const table = a.table + (size_t)it.b * sh.width;
  int next_key = s_first * 16;
  int id = 0;
  auto fetch = [&]() {
    const int i = sh.by_page.div(next_key);
    id = i < sh.width ? scalar_word(table, i) : -1;
  };
  uint32_t gone = 0;
  uint32_t doff[OPS];
#pragma unroll
  for (int y = 0; y < OPS; ++y) {
    const int r = 8 * (wave & 1) + y * RPB + lane / PPR;
    const int slot = lane % PPR;
    doff[y] = (uint32_t)(r * ROWB + (wave >= 2 ? slot : slot ^ r) * 16);
  }
  auto issue = [&](int stage) {
    gone |= sh.is_page(id) ? 0u : 1u;
    const int slot = next_key - sh.by_page.div(next_key) * sh.page_size;
    const unsigned char* src =
        pool + (((size_t)(sh.is_page(id) ? id : 0) * a.hkv + g) * sh.page_size + slot) * ROWB;
    unsigned char* lds = smem + stage * BUF + wave * (BUF / NW);
#pragma unroll
    for (int y = 0; y < OPS; ++y) dma16(src, doff[y], lds + 1024 * y);
    next_key += 16;
    fetch();
  };
  fetch();
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) {
    gone <<= 1;
    if (s < nsteps) issue(s);
  }

  // This lane's LDS bytes: K piece 4x + j4 of row c16 at ka[x mod 4] + 256 (x / 4); V piece
  // 16y + c16 of row 4 j4 + m at va + m ROWB + 256 y.
  const __attribute__((address_space(3))) unsigned char* const lds =
      (const __attribute__((address_space(3))) unsigned char*)smem;
  int ka[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) ka[x] = c16 * ROWB + (((4 * x + j4) ^ c16) << 4);
  const int va = TILE + 4 * j4 * ROWB + 16 * c16;

  const int w_first = pl.by_group.div(wave * 16);
  const int tw_lo = t0 + min(w_first, tokens - 1);
  const int tw_hi = t0 + min(pl.by_group.div(wave * 16 + 15), tokens - 1);
  const int wlo = w_first < tokens ? max(0, (sh.support_lo(tw_lo) >> 4) - s_first) : nsteps;
  const int whi = min(nsteps - 1, (tw_hi >> 4) - s_first);
  const int ua = ((sh.support_lo(tw_hi) + 15) >> 4) - s_first;
  const int ub = ((tw_lo + 1) >> 4) - s_first;

  float m = valid ? kNoScore : 0.0f, lsum = 0.0f;
  f32x4 acc[E];
#pragma unroll
  for (int nb = 0; nb < E; ++nb) acc[nb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  int rstage = 0;
  auto begin_step = [&](int st) -> int {
    wait_groups<STAGES - 2, OPS>(min(STAGES - 2, nsteps - 1 - st));
    lds_barrier();
    gone <<= 1;
    if (st + STAGES - 1 < nsteps) issue(rstage == 0 ? STAGES - 1 : rstage - 1);
    __builtin_amdgcn_sched_barrier(0);
    const int sb = rstage * BUF;
    rstage = rstage == STAGES - 1 ? 0 : rstage + 1;
    return sb;
  };

  auto step = [&](int st, int sb) {
    f32x4 sp[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) sp[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int x = 0; x < KM / 4; ++x) {
      const f32x4 k =
          *(const __attribute__((address_space(3))) f32x4*)(lds + sb + ka[x & 3] + 256 * (x >> 2));
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sp[(4 * x + e) & 7] =
            __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], qf[4 * x + e], sp[(4 * x + e) & 7], 0, 0, 0);
    }
    f32x4 s = ((sp[0] + sp[1]) + (sp[2] + sp[3])) + ((sp[4] + sp[5]) + (sp[6] + sp[7]));
    const bool dropped = (gone >> (STAGES - 1)) & 1u;
    const bool masked = st < ua || st >= ub || dropped;
    const int k0 = (s_first + st) * 16 + 4 * j4;
    auto seen = [&](int e) -> bool { return e >= lo_c - k0 && e <= tcol - k0 && !dropped; };
    if (masked) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = seen(e) ? s[e] : kNegInf;
    }
    const float mx = max_xor16_32(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])));
    // the reference moves where a maximum exceeds it by more than 8 (weights stay <= 2^8), and in
    // the wave's first step
    const bool grow = mx > m + 8.0f || (st == wlo && mx > m);
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
      const float alpha = grow ? fast_exp2(m - mx) : 1.0f;
      m = grow ? mx : m;
      lsum *= alpha;
#pragma unroll
      for (int nb = 0; nb < E; ++nb) acc[nb] *= alpha;
    }
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = fast_exp2(s[e] - m);
    lsum += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
    for (int y = 0; y < E / 4; ++y) {
      f32x4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        v[k] = *(const __attribute__((address_space(3))) f32x4*)(lds + sb + va + k * ROWB + 256 * y);
      bool odd = false;
      if (masked) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int x = 0; x < 4; ++x) odd |= is_special(v[k][x]);
      }
      if (masked && __builtin_amdgcn_ballot_w64(odd) != 0) {
        // Infinities and NaN: counted for the columns that see their key (as in the bf16 kernel).
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          f32x4 cu = {0.0f, 0.0f, 0.0f, 0.0f}, cd = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float w = v[k][x], one = seen(k) ? 1.0f : 0.0f;
            const bool sp1 = is_special(w), nan = w != w;
            const float up = sp1 && (nan || w > 0.0f) ? 1.0f : 0.0f;
            const float down = sp1 && (nan || w < 0.0f) ? 1.0f : 0.0f;
            cu = __builtin_amdgcn_mfma_f32_16x16x4f32(up, one, cu, 0, 0, 0);
            cd = __builtin_amdgcn_mfma_f32_16x16x4f32(down, one, cd, 0, 0, 0);
            v[k][x] = sp1 ? 0.0f : w;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[4 * y + x][e] += (cu[e] > 0.0f ? -kNegInf : 0.0f) + (cd[e] > 0.0f ? kNegInf : 0.0f);
        }
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        f32x4 part = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          part = __builtin_amdgcn_mfma_f32_16x16x4f32(v[k][x], p[k], part, 0, 0, 0);
        acc[4 * y + x] += part;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  int st = 0;
  for (; st < wlo && st < nsteps; ++st) begin_step(st);
  for (; st <= whi; ++st) {
    const int sb = begin_step(st);
    step(st, sb);
  }
  for (; st < nsteps; ++st) begin_step(st);

  // Lane (c16, j4) holds channels 64 y + 16 j4 + 4 i + x in acc[4 y + x][i].
  const float l = sum_xor16_32(lsum);
  if (__builtin_expect(l == 0.0f, 0) &&
      any_page(sh, table, max(lo_c, s_first * 16), min(tcol, (s_first + nsteps) * 16 - 1)))
    m = kNoWeight;
  if (it.ways == 1) {
    if (valid) {
      const float inv = inverse_sum(m, l);
      float* o = (float*)a.out + address(col) * D + 16 * j4;
#pragma unroll
      for (int y = 0; y < E / 4; ++y)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(f32x4*)(o + 64 * y + 4 * i) = f32x4{acc[4 * y][i] * inv, acc[4 * y + 1][i] * inv,
                                                acc[4 * y + 2][i] * inv, acc[4 * y + 3][i] * inv};
      if (a.lse != nullptr && j4 == 0) a.lse[lse_at(col)] = log_partition(m, l);
    }
    return;
  }

  constexpr size_t STATE = paged_state_bytes(kPagedColsF32, D) / 4;
  float* const part =
      a.states + ((size_t)it.slot * a.hkv + (size_t)g * it.ways + it.piece) * STATE;
  if (valid) {
#pragma unroll
    for (int y = 0; y < E / 4; ++y)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(part + col * D + 64 * y + 16 * j4 + 4 * i) =
            f32x4{acc[4 * y][i], acc[4 * y + 1][i], acc[4 * y + 2][i], acc[4 * y + 3][i]};
    if (j4 == 0) *(float2*)(part + kPagedColsF32 * D + 2 * col) = make_float2(m, l);
  }
}

}  // namespace

namespace {

template <int D>
hipError_t launch_paged_t(const PagedArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)(a.plan.items() * a.hkv));
  if (a.plan.narrow) {
    hipLaunchKernelGGL((paged_narrow_f32_kernel<D>), grid, dim3(kF32Waves * 64), 0, stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((paged_f32_kernel<D>), grid, dim3(kF32Waves * 64), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.plan.pieces == 0) return e;
  return launch_paged_merge<float, D, kPagedColsF32>(a, stream);
}

}  // namespace

hipError_t launch_paged_f32(const PagedArgs& a, int32_t head_dim, hipStream_t stream) {
  return head_dim == 64 ? launch_paged_t<64>(a, stream) : launch_paged_t<128>(a, stream);
}

}  // namespace pbb
