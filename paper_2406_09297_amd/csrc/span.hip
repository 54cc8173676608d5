// Decode attention over a window and the first tokens, for CDNA4 (gfx950,
// wave64, MFMA): one layer, one new token per sequence, from a bf16 cache or
// from the 4-bit cache (then also without a window).
//
//   o = softmax(q K^T / sqrt(D)) V over the positions p < L with p < sinks or
//   p >= L - window
//
// A unit is one (sequence, KV head); its attended tiles of 32 tokens are those
// of the first tokens, then those from the window's start on, numbered
// through, so tiles between them are neither read nor visited.  They are cut
// into runs of at most run_tiles, a workgroup each, whose waves take every
// W-th tile with one online softmax; the last run of a unit to finish merges
// its runs in run order.  The tile arithmetic is that of tile.h: S^T = K Q^T
// with the query rows as MFMA columns, O^T += V^T P^T.
//
// The 4-bit form makes bf16 operands of the codes in registers.  Keys: the
// conversion instruction takes the block's power of two along, exactly.  Values:
// an operand's eight codes are eight tokens of one channel, each with a scale
// of its own, so the scale goes to the other operand: the weights times 2^e of
// their token, one set per block of 32 channels, also exact (a power of two).
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "decode.h"
#include "qcache.h"
#include "serve.h"
#include "tile.h"

namespace mlkv {

namespace {

template <int D>
struct Codes {  // a wave's part of one record: 2 D bits a lane and its exponents
  static constexpr int N = D / 64;
  u32x4 k[N], v[N], ve[N];
  uint32_t ke[N];
};

template <int D>
__device__ __forceinline__ void load_codes(Codes<D>& t, const uint8_t* rec, int col, int grp) {
  const int lane = grp * 16 + col;
#pragma unroll
  for (int n = 0; n < D / 64; ++n) {
    t.k[n] = *reinterpret_cast<const u32x4*>(rec + n * 1024 + lane * 16);
    t.v[n] = *reinterpret_cast<const u32x4*>(rec + QTile<D>::kVCodes + n * 1024 + lane * 16);
    t.ve[n] = *reinterpret_cast<const u32x4*>(rec + QTile<D>::kVExps + grp * (D / 4) + n * 16);
    t.ke[n] = *reinterpret_cast<const uint32_t*>(rec + QTile<D>::kKExps + col * (D / 16) + n * 4);
  }
}

// What a unit attends: positions p < L with p < first or p >= lo, in tiles 0 ..
// head - 1 and from head + skip on.
struct Span {
  int L, lo, first, head, skip, tiles;
  __device__ __forceinline__ int tile(int it) const { return it < head ? it : it + skip; }
  __device__ __forceinline__ bool partial(int t0) const {
    return t0 + kTile > L || (t0 < lo && t0 + kTile > first);
  }
  __device__ __forceinline__ bool kept(int p) const { return p < L && (p < first || p >= lo); }
};
__device__ __forceinline__ Span span_of(int len, int max_len, int window, int sinks) {
  Span s;
  s.L = len < 0 ? 0 : len > max_len ? max_len : len;
  s.lo = window > 0 && s.L > window ? s.L - window : 0;
  s.first = sinks < s.lo ? sinks : s.lo;
  s.head = (s.first + kTile - 1) / kTile;
  const int from = max(s.lo / kTile, s.head);
  s.skip = from - s.head;
  s.tiles = (s.L + kTile - 1) / kTile - s.skip;
  return s;
}

// Scores of a tile (x: tokens 8 grp + e) to weights against the row's running
// maximum; a position that is not kept weighs nothing, whatever its score.
template <int D>
__device__ __forceinline__ void weigh(WaveState<D>& st, float (&x)[8], bool partial, unsigned kept,
                                      float scale_log2) {
  if (partial) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (kept >> e) & 1 ? x[e] : -INFINITY;
  }
  float tmax = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                     fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
  if (__ballot(tmax * scale_log2 > st.m)) {
    tmax = fmaxf(tmax, __shfl_xor(tmax, 16));
    tmax = fmaxf(tmax, __shfl_xor(tmax, 32));
    tmax *= scale_log2;
    const float m_new = tmax > st.m ? tmax : st.m;
    const float alpha = fast_exp2(st.m - m_new);  // 0 on the first tile, 1 if unchanged
    st.m = m_new;
    st.den *= alpha;
#pragma unroll
    for (int db = 0; db < Tile<D>::DB; ++db) st.acc[db] *= alpha;
  }
  const float neg_m = -st.m;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = fmaf(x[e], scale_log2, neg_m);
  if (partial) {  // -inf against a maximum of -inf is NaN; it counts only where kept
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (kept >> e) & 1 ? x[e] : -INFINITY;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = fast_exp2(x[e]);
}

__device__ __forceinline__ bf16x8 to_bf16(const float (&x)[8]) {
  u16x8 b;
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = f32_to_bf16_bits(x[e]);
  return as_bf16(b);
}

__device__ __forceinline__ unsigned kept_bits(const Span& s, int first) {
  unsigned kept = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) kept |= (s.kept(first + e) ? 1u : 0u) << e;
  return kept;
}

constexpr uint16_t kOne = 0x3F80;

template <int D, int NB>
__device__ __forceinline__ void span_tile(WaveState<D> (&st)[NB], Tile<D>& t,
                                          const bf16x8 (&qf)[NB][Tile<D>::KK], const Span& sp,
                                          int t0, int grp, float scale_log2) {
  constexpr int KK = Tile<D>::KK, DB = Tile<D>::DB;
  const bool partial = sp.partial(t0);
  unsigned kept = 0xFF;
  if (partial) {
    kept = kept_bits(sp, t0 + grp * 8);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!((kept >> e) & 1)) {
#pragma unroll
        for (int db = 0; db < DB; ++db) t.v[db][e] = 0;
      }
  }
  const u16x8 ones = {kOne, kOne, kOne, kOne, kOne, kOne, kOne, kOne};
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      s0 = mfma_bf16(as_bf16(t.k[0][kk]), qf[c][kk], s0);
      s1 = mfma_bf16(as_bf16(t.k[1][kk]), qf[c][kk], s1);
    }
    float x[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
    weigh<D>(st[c], x, partial, kept, scale_log2);
    const bf16x8 pf = to_bf16(x);
    // The denominator sums the same rounded weights: a row of ones times P^T.
    st[c].den = mfma_bf16(as_bf16(ones), pf, st[c].den);
#pragma unroll
    for (int db = 0; db < DB; ++db) st[c].acc[db] = mfma_bf16(as_bf16(t.v[db]), pf, st[c].acc[db]);
  }
}

template <int D, int NB>
__device__ __forceinline__ void span_tile(WaveState<D> (&st)[NB], Codes<D>& t,
                                          const bf16x8 (&qf)[NB][Tile<D>::KK], const Span& sp,
                                          int t0, int grp, float scale_log2) {
  constexpr int KK = Tile<D>::KK, DB = Tile<D>::DB;
  const bool partial = sp.partial(t0);
  unsigned kept = 0xFF;
  if (partial) kept = kept_bits(sp, t0 + grp * 8);
  const u16x8 ones = {kOne, kOne, kOne, kOne, kOne, kOne, kOne, kOne};
  f32x4 s[NB][2];
#pragma unroll
  for (int c = 0; c < NB; ++c) s[c][0] = s[c][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 2 * KK; ++i) {
    // The shifts leave neighbouring bytes in the sign and mantissa, which the
    // conversion does not read.
    const float scale = __builtin_bit_cast(
        float, i % 4 == 3 ? t.ke[i / 4] >> 1 : t.ke[i / 4] << (23 - 8 * (i % 4)));
    const bf16x8 k = as_bf16(dequantise8(t.k[i / 4][i % 4], scale));
#pragma unroll
    for (int c = 0; c < NB; ++c) s[c][i / KK] = mfma_bf16(k, qf[c][i % KK], s[c][i / KK]);
  }
  bf16x8 p[NB][KK];  // the weights times the value scales of each channel block
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    float x[8] = {s[c][0][0], s[c][0][1], s[c][0][2], s[c][0][3],
                  s[c][1][0], s[c][1][1], s[c][1][2], s[c][1][3]};
    weigh<D>(st[c], x, partial, kept, scale_log2);
    st[c].den = mfma_bf16(as_bf16(ones), to_bf16(x), st[c].den);
#pragma unroll
    for (int b = 0; b < KK; ++b) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t d = t.ve[b / 2][(b % 2) * 2 + e / 4];
        const uint32_t bits = (e % 4 == 3 ? d >> 1 : d << (23 - 8 * (e % 4))) & 0x7F800000u;
        float f = __builtin_bit_cast(float, bits);
        if (partial) f = (kept >> e) & 1 ? f : 0.f;
        y[e] = x[e] * f;
      }
      p[c][b] = to_bf16(y);
    }
  }
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    const bf16x8 v = as_bf16(dequantise8(t.v[db / 4][db % 4], 1.f));
#pragma unroll
    for (int c = 0; c < NB; ++c) st[c].acc[db] = mfma_bf16(v, p[c][db / 2], st[c].acc[db]);
  }
}

template <int D, int NB, int W>
struct alignas(16) SpanShared {
  float acc[W][16 * NB][D + 4];  // the waves' merge
  float m[W][16 * NB];
  float l[W][16 * NB];
  int last;
};

template <int D, int NB, int W, bool Q4>
__global__ __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(D == 64 && NB == 1 ? 4 : 2)))
void span_kernel(SpanParams p) {
  constexpr int KK = Tile<D>::KK, DB = Tile<D>::DB;
  constexpr int NT = W * 64;
  constexpr int D4 = D / 4;
  constexpr int PF = Q4 && D * NB < 256 ? 3 : 2;  // tiles in registers: one in use, the others on their way
  __shared__ SpanShared<D, NB, W> sm;
  const int lane = threadIdx.x & 63;
  const int wave = threadIdx.x >> 6;
  const int col = lane & 15;
  const int grp = lane >> 4;

  // Workgroups go round the eight XCDs: the chunks of one run, which read the
  // same tiles, are eight apart, so that they share an XCD's L2.
  const unsigned per8 = 8u * static_cast<unsigned>(p.chunks);
  const unsigned x8 = blockIdx.x / per8, xr = blockIdx.x - x8 * per8;
  const int chunk = static_cast<int>(xr >> 3);
  const unsigned item = x8 * 8 + (xr & 7);
  if (item >= p.items) return;
  const unsigned unit = item / static_cast<unsigned>(p.runs);
  const int j = static_cast<int>(item - unit * static_cast<unsigned>(p.runs));
  const int b = static_cast<int>(unit / static_cast<unsigned>(p.n_groups));
  const int r = static_cast<int>(unit - static_cast<unsigned>(b) * p.n_groups);
  const int row0 = chunk * p.chunk_rows;
  const int n_rows = min(p.chunk_rows, p.G - row0);

  const Span sp = span_of(p.lens[b], p.max_len, p.window, p.sinks);
  const int nb = min(max((sp.tiles + p.run_tiles - 1) / p.run_tiles, 1), p.runs);
  if (j >= nb) return;
  const int k0 = static_cast<int>(static_cast<long>(sp.tiles) * j / nb);
  const int k1 = static_cast<int>(static_cast<long>(sp.tiles) * (j + 1) / nb);

  const size_t seq = static_cast<size_t>(p.kv_begin + r) * p.B + b;
  const uint16_t* kbase = Q4 ? nullptr : p.k + seq * p.S * D;
  const uint16_t* vbase = Q4 ? nullptr : p.v + seq * p.S * D;
  const uint8_t* recs = Q4 ? p.q4 + seq * (p.S / kTile) * QTile<D>::kBytes : nullptr;
  auto load = [&](auto& t, int it) {
    const int tile = sp.tile(it);
    if constexpr (Q4)
      load_codes<D>(t, recs + static_cast<size_t>(tile) * QTile<D>::kBytes, col, grp);
    else
      load_tile<D>(t, kbase, vbase, tile * kTile, col, grp);
  };

  const size_t out_row = static_cast<size_t>(b) * p.h + r * p.G + row0;
  bf16x8 qf[NB][KK];
  WaveState<D> st[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const int rr = c * 16 + col;
    const uint16_t* qrow = p.q + (out_row + (rr < n_rows ? rr : 0)) * D + grp * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const u16x8 v = load16(qrow + kk * 32);
      const u16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
      qf[c][kk] = as_bf16(rr < n_rows ? v : zero);  // padded rows score zero
    }
    st[c].den = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int db = 0; db < DB; ++db) st[c].acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  int it = k0 + wave;
  if (it < k1) {
    // Requests past the run's end repeat its last tile, so that every path
    // through the loop has the same loads in flight.
    typename std::conditional<Q4, Codes<D>, Tile<D>>::type t[PF];
#pragma unroll
    for (int s = 0; s < PF - 1; ++s) load(t[s], min(it + s * W, k1 - 1));
    for (bool more = true; more;) {
#pragma unroll
      for (int s = 0; s < PF; ++s) {
        if (it >= k1) {
          more = false;
          break;
        }
        load(t[(s + PF - 1) % PF], min(it + (PF - 1) * W, k1 - 1));
        span_tile<D, NB>(st, t[s], qf, sp, sp.tile(it) * kTile, grp, p.scale_log2);
        it += W;
      }
    }
  }

  // Merge the waves through LDS; a unit of one run is finished here, another
  // leaves a partial per run.
  const size_t uc = static_cast<size_t>(unit) * p.chunks + chunk;
  const int part_floats = p.chunk_rows * D;  // one run's partial outputs, [row][channel]
  float* const unit_acc = nb > 1 ? p.part_acc + uc * p.runs * part_floats : nullptr;
  float* const unit_ml = nb > 1 ? p.part_ml + uc * p.runs * p.chunk_rows * 2 : nullptr;
  const __amdgpu_buffer_rsrc_t rsrc =
      device_rsrc(unit_acc, nb > 1 ? static_cast<uint32_t>(nb * part_floats * 4) : 0u);
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    if (grp == 0) {
      sm.m[wave][c * 16 + col] = st[c].m;
      sm.l[wave][c * 16 + col] = st[c].den[0];
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
      *reinterpret_cast<f32x4*>(&sm.acc[wave][c * 16 + col][db * 16 + grp * 4]) = st[c].acc[db];
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < n_rows * D4; idx += NT) {
    const int rr = idx / D4;
    const int d = (idx - rr * D4) * 4;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, sm.m[w][rr]);
    const float ref = merge_reference(M);
    float wsum = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = fast_exp2(sm.m[w][rr] - ref);
      wsum += f * sm.l[w][rr];
      o += f * *reinterpret_cast<const f32x4*>(&sm.acc[w][rr][d]);
    }
    if (nb == 1) {
      store4_as<D>(p.out, p.out_bf16, out_row + rr, d, normalize4(o, wsum));
    } else {
      store4_device(rsrc, (j * part_floats + rr * D + d) * 4, o);
      if (d == 0) {
        store_device(&unit_ml[(j * p.chunk_rows + rr) * 2 + 0], M);
        store_device(&unit_ml[(j * p.chunk_rows + rr) * 2 + 1], wsum);
      }
    }
  }
  if (nb == 1) return;

  // The last run of the unit to finish merges them in run order, so results
  // do not depend on which that is.  Every other run bumped the counter after
  // its partials completed: the device-scope loads below see them.
  wait_stores_complete();
  __syncthreads();
  if (threadIdx.x == 0)
    sm.last = __hip_atomic_fetch_add(&p.counters[uc], 1, __ATOMIC_RELAXED,
                                     __HIP_MEMORY_SCOPE_AGENT) == nb - 1;
  __syncthreads();
  if (!sm.last) return;
  constexpr int U = 8;  // runs whose partials are requested together
  for (int idx = threadIdx.x; idx < n_rows * D4; idx += NT) {
    const int rr = idx / D4;
    float M = -INFINITY, den = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < nb; s0 += U) {
      float m[U], w[U];
      f32x4 a[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        m[u] = -INFINITY;
        w[u] = 0.f;
        a[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (s0 + u < nb) {
          float* ml = &unit_ml[((s0 + u) * p.chunk_rows + rr) * 2];
          m[u] = load_device(ml);
          w[u] = load_device(ml + 1);
          a[u] = load4_device(rsrc, ((s0 + u) * part_floats + idx * 4) * 4);
        }
      }
      float bm = M;
#pragma unroll
      for (int u = 0; u < U; ++u) bm = fmaxf(bm, m[u]);
      const float ref = merge_reference(bm);
      const float sc = fast_exp2(M - ref);  // 0 while nothing is accumulated
      den *= sc;
      o *= sc;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float f = fast_exp2(m[u] - ref);
        den += f * w[u];
        o += f * a[u];
      }
      M = bm;
    }
    store4_as<D>(p.out, p.out_bf16, out_row + rr, (idx - rr * D4) * 4, normalize4(o, den));
  }
  if (threadIdx.x == 0)  // ready for the next call on this workspace
    __hip_atomic_store(&p.counters[uc], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int D, int NB>
hipError_t launch_span_t(const SpanParams& p, hipStream_t stream, hipEvent_t start,
                         hipEvent_t stop) {
  const dim3 grid((p.items + 7) / 8 * 8 * static_cast<unsigned>(p.chunks));
  auto kernel = p.q4 ? span_kernel<D, NB, kWaves, true> : span_kernel<D, NB, kWaves, false>;
  if (start)
    hipExtLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, start, stop, 0, p);
  else
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_span(const SpanParams& p, int head_dim, hipStream_t stream, hipEvent_t start,
                       hipEvent_t stop) {
  const bool two = p.chunk_rows > 16;
  if (head_dim == 64)
    return two ? launch_span_t<64, 2>(p, stream, start, stop)
               : launch_span_t<64, 1>(p, stream, start, stop);
  return two ? launch_span_t<128, 2>(p, stream, start, stop)
             : launch_span_t<128, 1>(p, stream, start, stop);
}

}  // namespace mlkv
