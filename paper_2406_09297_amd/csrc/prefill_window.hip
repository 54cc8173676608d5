// Causal prefill attention within a window, and over the first tokens, of one
// layer, for CDNA4 (gfx950, wave64, MFMA).  Rows, units and results as in
// prefill.hip: a token at position n attends the positions p <= n with
// p < sinks or p > n - window.
//
// A workgroup of four waves takes 64 NB consecutive query rows and visits the
// tiles of the first tokens, then those from the first row's window on to the
// last row's position; the tiles between are not read.  A wave skips the tiles
// that none of its rows attends and masks those that not all of them do: with
// w positions a row and t tokens a wave, about (w + t) / 32 tiles, of which
// the 2 + t / 16 at the window's two edges are masked.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "prefill.h"
#include "serve.h"
#include "tile.h"

namespace mlkv {

namespace {

// What one column (query row) attends: p <= n with p < sinks or p >= lo.
struct Reach {
  int n, lo;
  __device__ __forceinline__ bool has(int p, int sinks) const {
    return p <= n && (p < sinks || p >= lo);
  }
  // Bit e: position first + e (0 .. 7), from what remains up to each bound.
  __device__ __forceinline__ unsigned bits(int first, int sinks) const {
    return below(n + 1 - first) & (below(sinks - first) | ~below(lo - first));
  }
  __device__ __forceinline__ static unsigned below(int count) {  // bits 0 .. count - 1 of eight
    return (1u << min(max(count, 0), 8)) - 1;
  }
};

__device__ __forceinline__ bool not_finite(u16x8 x) {
  bool odd = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) odd |= (x[e] & 0x7F80) == 0x7F80;
  return odd;
}

// acc += V^T P^T token by token, each only into the columns that attend it: a
// value that is not finite times the weight 0 of another column would make that
// column NaN.  For the rare tiles that hold such values.
template <int D, int NB>
__device__ __forceinline__ void add_values_apart(WaveState<D> (&st)[NB], const Tile<D>& t,
                                                 const bf16x8 (&pf)[NB],
                                                 const Reach (&reach)[NB], int t0, int grp,
                                                 int sinks) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#pragma nounroll
  for (int u = 0; u < kTile; ++u) {
    u32x4 only;  // of an operand's eight tokens: token u
#pragma unroll
    for (int i = 0; i < 4; ++i)
      only[i] = u >> 1 == grp * 4 + i ? (u & 1 ? 0xFFFF0000u : 0xFFFFu) : 0u;
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const bf16x8 w = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, pf[c]) & only);
      const bool has = reach[c].has(t0 + u, sinks);
#pragma unroll
      for (int db = 0; db < Tile<D>::DB; ++db) {
        const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, t.v[db]) & only);
        const f32x4 add = mfma_bf16(v, w, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int i = 0; i < 4; ++i) st[c].acc[db][i] += has ? add[i] : 0.f;
      }
    }
  }
}

// One 32-token tile against the wave's NB blocks of 16 rows.  MASK: some row
// does not attend some position of it.
template <int D, int NB, bool MASK>
__device__ __forceinline__ void window_tile(WaveState<D> (&st)[NB], Tile<D>& t,
                                            const bf16x8 (&qf)[NB][Tile<D>::KK], int t0, int L,
                                            const Reach (&reach)[NB], int sinks, int grp,
                                            float scale_log2) {
  constexpr int KK = Tile<D>::KK, DB = Tile<D>::DB;
  float x[NB][8];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      s0 = mfma_bf16(as_bf16(t.k[0][kk]), qf[c][kk], s0);
      s1 = mfma_bf16(as_bf16(t.k[1][kk]), qf[c][kk], s1);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[c][i] = s0[i];
      x[c][4 + i] = s1[i];
    }
  }
  const int first = t0 + grp * 8;
  unsigned kept[NB];  // bit e: the row attends position first + e
  bool apart = false;
  if (MASK) {
    bool odd = false;
#pragma unroll
    for (int c = 0; c < NB; ++c) kept[c] = reach[c].bits(first, sinks);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
      for (int c = 0; c < NB; ++c) x[c][e] = (kept[c] >> e) & 1 ? x[c][e] : -INFINITY;
      if (first + e >= L) {  // slots not filled yet may hold anything
#pragma unroll
        for (int db = 0; db < DB; ++db) t.v[db][e] = 0;
      }
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) odd |= not_finite(t.v[db]);
    apart = __ballot(odd) != 0;
  }
  // The reference of a row's weights is moved only when a tile exceeds it by
  // more than kLazyRescale; a row that has attended nothing yet has -inf.
  bool over = false;
#pragma unroll
  for (int c = 0; c < NB; ++c) over |= max8(x[c]) * scale_log2 > st[c].m + kLazyRescale;
  if (__ballot(over)) {
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const float lmax = max8(x[c]);
      float cm = fmaxf(lmax, __shfl_xor(lmax, 16));
      cm = fmaxf(cm, __shfl_xor(cm, 32)) * scale_log2;
      const float m_new = cm > st[c].m + kLazyRescale ? cm : st[c].m;
      const float alpha = m_new == st[c].m ? 1.f : fast_exp2(st[c].m - m_new);
      st[c].m = m_new;
      st[c].den *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) st[c].acc[db] *= alpha;
    }
  }
  const u16x8 ones = {0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80};
  bf16x8 pf[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const float neg_m = -st[c].m;
    u16x8 pbits;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float y = fmaf(x[c][e], scale_log2, neg_m);
      // A masked score against a reference of -inf would be NaN.
      if (MASK) y = (kept[c] >> e) & 1 ? y : -INFINITY;
      pbits[e] = f32_to_bf16_bits(fast_exp2(y));
    }
    pf[c] = as_bf16(pbits);
    st[c].den = mfma_bf16(as_bf16(ones), pf[c], st[c].den);
  }
  if (MASK && apart) {
    add_values_apart<D, NB>(st, t, pf, reach, t0, grp, sinks);
    return;
  }
#pragma unroll
  for (int c = 0; c < NB; ++c)
#pragma unroll
    for (int db = 0; db < DB; ++db)
      st[c].acc[db] = mfma_bf16(as_bf16(t.v[db]), pf[c], st[c].acc[db]);
}

template <int D, int NB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2)))
void window_kernel(WindowPrefillParams p) {
  constexpr int KK = Tile<D>::KK, DB = Tile<D>::DB;
  constexpr int WAVE_ROWS = 16 * NB;
  __shared__ TileRing<D> rg;
  const int lane = threadIdx.x & 63;
  const int wave = threadIdx.x >> 6;
  const int col = lane & 15;
  const int grp = lane >> 4;
  const int unit = blockIdx.x;
  const int b = unit / p.n_groups;
  const int r = unit - b * p.n_groups;
  const int rows = p.T * p.G;
  const int blk = gridDim.y - 1 - blockIdx.y;
  const int wg_row0 = blk * 4 * WAVE_ROWS;  // < rows: the grid has no empty workgroup
  const int row0 = wg_row0 + wave * WAVE_ROWS;
  const bool active = row0 < rows;  // a wave past the end still stages tiles and syncs
  const int c0 = min(max(p.ctx[b], 0), p.S - 1);
  const int L = min(c0 + p.T, p.S);  // filled positions of the sequence
  // Position and window start of a row.
  auto reach_of = [&](int rho) {
    Reach at;
    at.n = min(c0 + min(rho, rows - 1) / p.G, p.S - 1);
    at.lo = p.window > 0 ? max(at.n - p.window + 1, 0) : 0;
    return at;
  };
  const Reach wg_first = reach_of(wg_row0), wg_last = reach_of(wg_row0 + 4 * WAVE_ROWS - 1);
  const Reach w_first = reach_of(row0), w_last = reach_of(row0 + WAVE_ROWS - 1);
  const int head = (min(p.sinks, wg_first.lo) + kTile - 1) / kTile;
  const int skip = max(wg_first.lo / kTile, head) - head;
  const int n_tiles = wg_last.n / kTile + 1 - skip;
  auto start_of = [&](int it) { return (it < head ? it : it + skip) * kTile; };

  const size_t seq = static_cast<size_t>(p.kv_begin + r) * p.B + b;
  const uint16_t* kbase = p.k + seq * p.S * D;
  const uint16_t* vbase = p.v + seq * p.S * D;
  rg.issue(0, kbase, vbase, start_of(0));  // every workgroup has at least one tile

  Reach reach[NB];
  bf16x8 qf[NB][KK];
  WaveState<D> st[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const int rho = row0 + 16 * c + col;
    const RowPlace at = row_place(p, rho, rows, b, 0, r, D);
    reach[c] = reach_of(rho);
    const uint16_t* qrow = p.q + at.offset + grp * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const u16x8 v = load16(qrow + kk * 32);
      const u16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
      qf[c][kk] = as_bf16(at.valid ? v : zero);
    }
    st[c].den = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int db = 0; db < DB; ++db) st[c].acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // Tile it sits in buffer it & 1: at the barrier this wave's direct loads have
  // landed, so every wave's part of tile it is there, and every wave is done
  // with tile it - 1, whose buffer then takes tile it + 1.
  for (int it = 0; it < n_tiles; ++it) {
    wait_loads();
    __syncthreads();
    if (it + 1 < n_tiles) rg.issue((it + 1) & 1, kbase, vbase, start_of(it + 1));
    const int t0 = start_of(it);
    // Some row of the wave attends some of it?  Every row all of it?
    if (!active || t0 > w_last.n || (t0 >= p.sinks && t0 + kTile <= w_first.lo)) continue;
    Tile<D> t;
    rg.read(t, it & 1, col, grp);
    if (t0 + kTile - 1 <= w_first.n && (t0 + kTile <= p.sinks || t0 >= w_last.lo))
      window_tile<D, NB, false>(st, t, qf, t0, L, reach, p.sinks, grp, p.scale_log2);
    else
      window_tile<D, NB, true>(st, t, qf, t0, L, reach, p.sinks, grp, p.scale_log2);
  }

  // Lane (col, grp) holds channels db*16 + 4*grp .. +3 of its row in each block.
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const RowPlace at = row_place(p, row0 + 16 * c + col, rows, b, 0, r, D);
    if (!at.valid) continue;
    const float inv = 1.f / st[c].den[0];
#pragma unroll
    for (int db = 0; db < DB; ++db)
      store4(p, at.offset + db * 16 + grp * 4, st[c].acc[db] * inv);
  }
}

}  // namespace

hipError_t launch_prefill_window(const WindowPrefillParams& p, int head_dim, hipStream_t stream,
                                 hipEvent_t start, hipEvent_t stop) {
  const int per_wg = prefill_rows_per_workgroup(head_dim);
  const int blocks = static_cast<int>((static_cast<long>(p.T) * p.G + per_wg - 1) / per_wg);
  const dim3 grid(p.B * p.n_groups, blocks);
  auto kernel = head_dim == 64 ? window_kernel<64, prefill_wave_blocks(64)>
                               : window_kernel<128, prefill_wave_blocks(128)>;
  if (start || stop)
    hipExtLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, start, stop, 0, p);
  else
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace mlkv
