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
//
// Tiles go to LDS once a workgroup by direct loads, three of 64 channels or two
// of 128 ahead of the one in use (bytes that leave 4 or 3 waves a SIMD); a wave
// takes two blocks of 16 rows, which share each operand read (us, one block /
// two, 2 sequences of 4096 tokens, 32 heads of 128 channels on 8, window 1024:
// 171 / 139; three do not fit the registers; 32x32x16 products 167 where these
// took 148).
//
// Bound by vector instructions, matrix products and the waits for LDS, which
// overlap only between waves, and by q and out at each workgroup's ends: of the 137 us of
// that call (119 GFLOP, 0.87 PFLOP/s; a large product reaches 1.38) the matrix
// cores are busy in 46 %, vector issue in 52 % (72 instructions beside 34
// products a tile), and reading q and writing out, 134 MB, takes 32 by itself,
// since workgroups of equal length reach their ends together.  8 sequences of
// 2000 tokens, 12 heads of 64 on one, window 256 (12 GFLOP, 53 MB): 28.3 us, of
// which 14 are the ends, in one and a half rounds of resident workgroups.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernels.h"
#include "prefill.h"
#include "serve.h"
#include "tile.h"
#include "weights.h"

namespace mlkv {

namespace {

// Four operands 1 KB apart in LDS.  Written out, since the compiler waits for
// every direct load on its way before it reads LDS; here the kernel's own waits
// and barriers say what has landed.
__device__ __forceinline__ void lds_read4(const uint16_t* at, u16x8 (&op)[4]) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint32_t off = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) uint16_t*)at));
  asm volatile(
      "ds_read_b128 %0, %4\n\t"
      "ds_read_b128 %1, %4 offset:%5\n\t"
      "ds_read_b128 %2, %4 offset:%6\n\t"
      "ds_read_b128 %3, %4 offset:%7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(op[0]), "=&v"(op[1]), "=&v"(op[2]), "=&v"(op[3])
      : "v"(off), "n"(1024), "n"(2 * 1024), "n"(3 * 1024)
      : "memory");
#endif
}

// A 32-token tile in LDS, staged and read as by TileRing.
template <int D>
struct TileBuffer {
  static constexpr int kLoads = 2 * (D / 64);  // of each wave, for a tile
  alignas(16) uint16_t k[kTile * D];
  alignas(16) uint16_t v[kTile * D];

  __device__ __forceinline__ void issue(const uint16_t* kbase, const uint16_t* vbase, int t0) {
    const unsigned lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned voff = (lane >> 2) * 64 + (((lane & 3) ^ vswz16(lane >> 2)) * 16);
#pragma unroll
    for (int u = 0; u < D / 64; ++u) {
      const int piece = u * 4 + wave;
      const size_t at = static_cast<size_t>(t0) * D * 2 + piece * 1024;
      load_lds16(reinterpret_cast<const char*>(kbase) + at, lane * 16, &k[piece * 512]);
      load_lds16(reinterpret_cast<const char*>(vbase) + at, voff, &v[piece * 512]);
    }
  }
  // Key operands of score block sb, k-steps 0 .. D/32 - 1; D = 64: both blocks
  // in one go (sb 0).
  __device__ __forceinline__ void read_k(u16x8 (&op)[4], int sb, int lane) const {
    lds_read4(&k[sb * 2048 + lane * 8], op);
  }
  // Value operands of the output blocks 4 n .. 4 n + 3.
  __device__ __forceinline__ void read_v(u16x8 (&op)[4], int n, int col, int grp) const {
    lds_read4(&v[(col * 4 + (grp ^ vswz16(col))) * 8 + n * 2048], op);  // channel 16 db + col
  }
};

// Wait until at most the loads of the `tiles` latest tiles (or of MOST, if
// fewer) are in flight; a wave has no other vector memory loads then.
template <int D, int MOST>
__device__ __forceinline__ void wait_tiles_but(int tiles) {
  constexpr int n = MOST * TileBuffer<D>::kLoads;  // vmcnt, the other counters left alone
  if (MOST == 0 || tiles >= MOST)
    __builtin_amdgcn_s_waitcnt((n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14));
  else if constexpr (MOST > 0)
    wait_tiles_but<D, MOST - 1>(tiles);
}

// A barrier of the workgroup without the waits that __syncthreads puts before
// it (for every direct load); memory operations stay on their side of it.
__device__ __forceinline__ void group_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Between writes to LDS and reads of them by other lanes of the wave, and before
// the place is written again: the hardware takes a wave's LDS operations in order,
// and the compiler, which sees one lane's addresses only, must not change it.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// What one column (query row) attends: p <= n with p < sinks or p >= lo.
struct Reach {
  int n, lo;
  __device__ __forceinline__ bool has(int p, int sinks) const {
    return p <= n && (p < sinks || p >= lo);
  }
  __device__ __forceinline__ static int below(int count) {  // bits 0 .. count - 1 of eight
    return (1 << min(max(count, 0), 8)) - 1;
  }
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Of eight values those whose bit is set, zero for the others.
__device__ __forceinline__ u16x8 keep_filled(u16x8 v, int filled) {
  u32x4 d = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = static_cast<uint32_t>((filled << (31 - 2 * i)) >> 31) & 0xFFFFu;
    const uint32_t hi = static_cast<uint32_t>((filled << (30 - 2 * i)) >> 31) & 0xFFFF0000u;
    d[i] &= lo | hi;
  }
  return __builtin_bit_cast(u16x8, d);
}

// acc += V^T P^T (output blocks 4 n .. 4 n + 3) token by token, each only into
// the columns that attend it: a value that is not finite times the weight 0 of
// another column would make that column NaN.
template <int D, int NB>
__device__ __forceinline__ void add_values_apart(WaveState<D> (&st)[NB], const u16x8 (&v)[4], int n,
                                                 const bf16x8 (&pf)[NB],
                                                 const Reach (&reach)[NB], int t0, int grp,
                                                 int sinks) {
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
      for (int j = 0; j < 4; ++j) {
        const bf16x8 one = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, v[j]) & only);
        const f32x4 add = mfma_bf16(one, w, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int i = 0; i < 4; ++i) st[c].acc[4 * n + j][i] += has ? add[i] : 0.f;
      }
    }
  }
}

// Scores of a tile for the wave's NB blocks of 16 rows: x[c][e] of token 8 grp + e.
template <int D, int NB>
__device__ __forceinline__ void window_scores(float (&x)[NB][8], const TileBuffer<D>* tile,
                                              const bf16x8 (&qf)[NB][Tile<D>::KK], int lane) {
  u16x8 k[4];
  if constexpr (D == 64) tile->read_k(k, 0, lane);
#pragma unroll
  for (int sb = 0; sb < 2; ++sb) {
    if constexpr (D == 128) tile->read_k(k, sb, lane);
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < Tile<D>::KK; ++kk)
        s = mfma_bf16(as_bf16(k[D == 64 ? 2 * sb + kk : kk]), qf[c][kk], s);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[c][4 * sb + i] = s[i];
    }
  }
}

// What a wave needs to know of its place.
template <int NB>
struct WindowWave {
  Reach reach[NB];         // of this lane's rows
  Reach first, last;       // of the wave's first and last row
  bool active;
  int col, grp, L, sinks;  // L: filled positions
  float scale_log2;
};

// The wave's rows take the tile at t0.
template <int D, int NB, bool APART>
__device__ __forceinline__ void window_step(WaveState<D> (&st)[NB],
                                            const TileBuffer<D>* tile, int t0,
                                            const bf16x8 (&qf)[NB][Tile<D>::KK],
                                            const WindowWave<NB>& w) {
  // Some row of the wave attends some of it?
  if (!w.active || t0 > w.last.n || (t0 >= w.sinks && t0 + kTile <= w.first.lo)) return;
  const int first = t0 + w.grp * 8;
  float x[NB][8];
  bf16x8 pf[NB];
  window_scores<D, NB>(x, tile, qf, w.grp * 16 + w.col);
  // Positions that some rows do not attend: behind the last one of a row, and
  // between the first tokens and a row's window.
  const bool ends = t0 + kTile - 1 > w.first.n;
  const bool starts = t0 + kTile > w.sinks && t0 < w.last.lo;
  if (ends) {
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const int left = w.reach[c].n + 1 - first;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[c][e] = e < left ? x[c][e] : -INFINITY;
    }
  }
  if (starts) {
    if (t0 >= w.sinks) {
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const int before = w.reach[c].lo - first;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] = e >= before ? x[c][e] : -INFINITY;
      }
    } else {
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const int before = w.reach[c].lo - first, early = w.sinks - first;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] = e >= before || e < early ? x[c][e] : -INFINITY;
      }
    }
  }
  weigh_rows<D, NB>(st, x, w.scale_log2, pf);
  const bool apart = APART && (ends || starts);
#pragma unroll
  for (int n = 0; n < Tile<D>::DB / 4; ++n) {
    u16x8 v[4];
    tile->read_v(v, n, w.col, w.grp);
    if (t0 + kTile > w.L) {  // slots not filled yet may hold anything
      int filled = Reach::below(w.L - first);
      asm volatile("" : "+v"(filled));  // here: the masks are 30 instructions of every tile else
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = keep_filled(v[i], filled);
    }
    if (apart) {
      add_values_apart<D, NB>(st, v, n, pf, w.reach, t0, w.grp, w.sinks);
    } else {
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          st[c].acc[4 * n + i] = mfma_bf16(as_bf16(v[i]), pf[c], st[c].acc[4 * n + i]);
    }
  }
}

// Chunk j (four channels) of a row of results staged in LDS; rows are permuted
// so that lanes on the same chunk of 16 rows meet all banks.
template <int D>
__device__ __forceinline__ f32x4* staged_chunk(float* staged, int row, int j) {
  return reinterpret_cast<f32x4*>(staged + row * D + ((j ^ row) & (D / 4 - 1)) * 4);
}

// Of 16 staged rows the first `count`, whole rows side by side: 16 bytes a lane
// (32 bytes of a row at a time straight from the accumulators: 4096 tokens on
// 2 sequences, 32 heads of 128 channels, windows of 64 / 1024 48 / 145 us, in
// whole rows 42 / 142).
template <int D, bool BF16, typename Offset>
__device__ __forceinline__ void store_rows(const WindowPrefillParams& p, float* staged, int count,
                                           int lane, Offset offset_of) {
  constexpr int LANES = BF16 ? D / 8 : D / 4;  // of a row
  const int j = lane % LANES;
#pragma unroll
  for (int r = 0; r < 16; r += 64 / LANES) {
    const int row = r + lane / LANES;
    if constexpr (BF16) {
      const f32x4 x = *staged_chunk<D>(staged, row, 2 * j);
      const f32x4 y = *staged_chunk<D>(staged, row, 2 * j + 1);
      u16x8 o;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o[i] = f32_to_bf16_bits(x[i]);
        o[4 + i] = f32_to_bf16_bits(y[i]);
      }
      if (row < count)
        *reinterpret_cast<u16x8*>(static_cast<uint16_t*>(p.out) + offset_of(row) + j * 8) = o;
    } else {
      const f32x4 x = *staged_chunk<D>(staged, row, j);
      if (row < count)
        *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + offset_of(row) + j * 4) = x;
    }
  }
}

template <int D, int NB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 3)))
void window_kernel(WindowPrefillParams p) {
  constexpr int KK = Tile<D>::KK, DB = Tile<D>::DB;
  constexpr int WAVE_ROWS = 16 * NB;
  constexpr int RING = D == 64 ? 4 : 3;  // tiles in LDS: one in use, the others on their way
  __shared__ TileBuffer<D> ring[RING];
  static_assert(sizeof(ring) >= 4 * 16 * D * sizeof(float));  // results of 16 rows a wave
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int unit = blockIdx.x;
  const int b = unit / p.n_groups;
  const int r = unit - b * p.n_groups;
  const int rows = p.T * p.G;
  const int blk = gridDim.y - 1 - blockIdx.y;
  const int wg_row0 = blk * 4 * WAVE_ROWS;  // < rows: the grid has no empty workgroup
  const int row0 = wg_row0 + wave * WAVE_ROWS;
  const int c0 = min(max(p.ctx[b], 0), p.S - 1);
  // Position and window start of a row.
  auto reach_of = [&](int rho) {
    Reach at;
    at.n = min(c0 + quotient(min(rho, rows - 1), p.G, p.inv_G), p.S - 1);
    at.lo = p.window > 0 ? max(at.n - p.window + 1, 0) : 0;
    return at;
  };
  // Its place in q and out: head r G + rho % G of token rho / G.
  auto offset_of = [&](int rho) {
    rho = min(rho, rows - 1);
    const int tok = quotient(rho, p.G, p.inv_G);
    return ((static_cast<size_t>(b) * p.T + tok) * p.h + r * p.G + (rho - tok * p.G)) * D;
  };
  const Reach wg_first = reach_of(wg_row0), wg_last = reach_of(wg_row0 + 4 * WAVE_ROWS - 1);
  WindowWave<NB> w;
  w.active = row0 < rows;  // a wave past the end still stages tiles and syncs
  w.first = reach_of(row0);
  w.last = reach_of(row0 + WAVE_ROWS - 1);
  w.col = lane & 15;
  w.grp = lane >> 4;
  w.L = min(c0 + p.T, p.S);
  w.sinks = p.sinks;
  w.scale_log2 = p.scale_log2;
  const int head = (min(p.sinks, wg_first.lo) + kTile - 1) / kTile;
  const int skip = max(wg_first.lo / kTile, head) - head;
  const int n_tiles = wg_last.n / kTile + 1 - skip;  // at least one
  auto start_of = [&](int it) { return (it < head ? it : it + skip) * kTile; };

  const size_t seq = static_cast<size_t>(p.kv_begin + r) * p.B + b;
  const uint16_t* kbase = p.k + seq * p.S * D;
  const uint16_t* vbase = p.v + seq * p.S * D;

  bf16x8 qf[NB][KK];
  WaveState<D> st[NB];
  auto pass = [&](auto apart) {
#pragma unroll
    for (int s = 0; s < RING - 1; ++s)
      if (s < n_tiles) ring[s].issue(kbase, vbase, start_of(s));
    if (!apart.value) {
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const int rho = row0 + 16 * c + w.col;
        w.reach[c] = reach_of(rho);
        const uint16_t* qrow = p.q + offset_of(rho) + w.grp * 8;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          const u16x8 v = load16(qrow + kk * 32);
          const u16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
          qf[c][kk] = as_bf16(rho < rows ? v : zero);
        }
      }
    }
#pragma unroll
    for (int c = 0; c < NB; ++c) clear_rows(st[c]);
    // Tile it sits in buffer it % RING.  At the barrier this wave's part of it
    // has landed (all but the loads of the tiles after it), so every wave's
    // has, and every wave is done with tile it - 1, whose buffer then takes
    // tile it + RING - 1.
    for (int it = 0; it < n_tiles; ++it) {
      if constexpr (apart.value)  // (spilled registers come and go there, too)
        wait_loads();
      else
        wait_tiles_but<D, RING - 2>(n_tiles - 1 - it);
      group_barrier();
      if (it + RING - 1 < n_tiles)
        ring[(it + RING - 1) % RING].issue(kbase, vbase, start_of(it + RING - 1));
      window_step<D, NB, apart.value>(st, &ring[it % RING], start_of(it), qf, w);
    }
    wait_loads();
    __syncthreads();
  };
  // A first pass takes the values as finite.  Where a result is not, a second
  // one adds the values of masked tiles token by token: a value that is not
  // finite must not reach rows that do not attend it (0 times it is NaN).
  pass(std::false_type{});
  bool odd = false;
#pragma unroll
  for (int c = 0; c < NB; ++c)
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) odd |= !(fabsf(st[c].acc[db][i]) < INFINITY);
  if (__syncthreads_or(odd)) pass(std::true_type{});

  // Lane (col, grp) holds channels db*16 + 4*grp .. +3 of its row in each block;
  // the ring, which nobody reads any more, turns that into whole rows.
  float* const staged = reinterpret_cast<float*>(ring) + wave * 16 * D;
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const float inv = 1.f / st[c].den[0];
#pragma unroll
    for (int db = 0; db < DB; ++db)
      *staged_chunk<D>(staged, w.col, db * 4 + w.grp) = st[c].acc[db] * inv;
    wave_lds_fence();
    if (p.out_bf16)
      store_rows<D, true>(p, staged, rows - (row0 + 16 * c), lane,
                          [&](int row) { return offset_of(row0 + 16 * c + row); });
    else
      store_rows<D, false>(p, staged, rows - (row0 + 16 * c), lane,
                           [&](int row) { return offset_of(row0 + 16 * c + row); });
    wave_lds_fence();
  }
}

}  // namespace

hipError_t launch_prefill_window(const WindowPrefillParams& p, int head_dim, hipStream_t stream,
                                 hipEvent_t start, hipEvent_t stop) {
  constexpr int per_wg = kWindowRows;
  const int blocks = static_cast<int>((static_cast<long>(p.T) * p.G + per_wg - 1) / per_wg);
  const dim3 grid(p.B * p.n_groups, blocks);
  auto kernel = head_dim == 64 ? window_kernel<64, kWindowRows / 64>
                               : window_kernel<128, kWindowRows / 64>;
  if (start || stop)
    hipExtLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, start, stop, 0, p);
  else
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace mlkv
