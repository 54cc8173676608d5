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
// their token, one set per block of 32 channels, rounded to bf16 as the
// denominator's weights are (a power of two changes no rounding, and with weights
// <= 2^-24 none of the format's 2^e overflows; products below 2^-126 lose bits).
//
// Bound by reading the cache.  A tile is read once, straight into the registers
// of the wave that needs it, 1 KB a load in operand order, so nothing passes
// through LDS and no wave waits for another before the merge.  Two tiles in
// registers, one in use and one on its way (three or four: no faster).  us, a
// streaming read reaches 6.5 TB/s:
//   64 sequences of 8192, 8 heads of 128 channels, 4 bits (573 MB)   98, 5.9 TB/s
//   8 sequences of 32768, 4 heads of 64, 4 bits (70 MB)            15.2, 4.6 TB/s
//   128 sequences of 512 .. 2047, one head of 64, 4 bits (11 MB)    7.7
//   48 bf16 windows of 1023, 8 heads of 128 channels (203 MB)      41.8, 4.9 TB/s
//   one sequence of 128                                             3.6
// The first issues vector instructions in 55 % of its cycles and has the matrix
// cores busy in 17 %: 210 instructions a tile, of which 32 unpack codes and 64
// scale and round weights.  The last is launch, lengths, one tile and the merge,
// one after the other; the ragged batch is that and its longest sequence.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "decode.h"
#include "qcache.h"
#include "serve.h"
#include "tile.h"
#include "weights.h"

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

// Of a partial tile, this lane's positions first .. first + 7: a bit for each
// that is attended, and the scores of the others to -inf (whatever they are).
template <int NB>
__device__ __forceinline__ unsigned mask_scores(float (&x)[NB][8], const Span& sp, int first) {
  unsigned kept = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool has = sp.kept(first + e);
    kept |= (has ? 1u : 0u) << e;
#pragma unroll
    for (int c = 0; c < NB; ++c) x[c][e] = has ? x[c][e] : -INFINITY;
  }
  return kept;
}

template <int D, int NB>
__device__ __forceinline__ void span_tile(WaveState<D> (&st)[NB], Tile<D>& t,
                                          const bf16x8 (&qf)[NB][Tile<D>::KK], const Span& sp,
                                          int t0, int grp, float scale_log2) {
  constexpr int KK = Tile<D>::KK, DB = Tile<D>::DB;
  float x[NB][8];
  bf16x8 pf[NB];
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
  if (sp.partial(t0)) {
    const unsigned kept = mask_scores<NB>(x, sp, t0 + grp * 8);
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // values that are not attended may be anything
      const uint32_t keep = ((kept >> (2 * i)) & 1 ? 0xFFFFu : 0u) |
                            ((kept >> (2 * i + 1)) & 1 ? 0xFFFF0000u : 0u);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        u32x4 v = __builtin_bit_cast(u32x4, t.v[db]);
        v[i] &= keep;
        t.v[db] = __builtin_bit_cast(u16x8, v);
      }
    }
  }
  weigh_rows<D, NB>(st, x, scale_log2, pf);
#pragma unroll
  for (int c = 0; c < NB; ++c)
#pragma unroll
    for (int db = 0; db < DB; ++db)
      st[c].acc[db] = mfma_bf16(as_bf16(t.v[db]), pf[c], st[c].acc[db]);
}

// Byte i of d as the exponent of a power of two, in one instruction (a shift
// of the selected byte), which the compiler makes two of for bytes 0 to 2.
template <int i>
__device__ __forceinline__ float byte_scale(uint32_t d) {
  uint32_t r = 0;
#if defined(__HIP_DEVICE_COMPILE__)
  const uint32_t shift = 23;
  if constexpr (i == 0)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD "
        "src1_sel:BYTE_0" : "=v"(r) : "v"(shift), "v"(d));
  if constexpr (i == 1)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD "
        "src1_sel:BYTE_1" : "=v"(r) : "v"(shift), "v"(d));
  if constexpr (i == 2)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD "
        "src1_sel:BYTE_2" : "=v"(r) : "v"(shift), "v"(d));
  if constexpr (i == 3)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD "
        "src1_sel:BYTE_3" : "=v"(r) : "v"(shift), "v"(d));
#endif
  return __builtin_bit_cast(float, r);
}

template <int D, int NB>
__device__ __forceinline__ void span_tile(WaveState<D> (&st)[NB], Codes<D>& t,
                                          const bf16x8 (&qf)[NB][Tile<D>::KK], const Span& sp,
                                          int t0, int grp, float scale_log2) {
  constexpr int KK = Tile<D>::KK;
  float x[NB][8];
  bf16x8 pf[NB];
  {
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
#pragma unroll
    for (int c = 0; c < NB; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[c][i] = s[c][0][i];
        x[c][4 + i] = s[c][1][i];
      }
  }
  if (sp.partial(t0)) {
    // Exponents that are not attended may be NaN: 0 times the weight 0 they get.
    const unsigned kept = mask_scores<NB>(x, sp, t0 + grp * 8);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t bits = (kept >> (4 * i)) & 15;
      const uint32_t keep = ((bits * 0x00204081u) & 0x01010101u) * 0xFFu;
#pragma unroll
      for (int b = 0; b < KK; ++b) t.ve[b / 2][(b % 2) * 2 + i] &= keep;
    }
  }
  weigh_rows<D, NB>(st, x, scale_log2, pf);
#pragma unroll
  for (int b = 0; b < KK; ++b) {  // blocks of 32 channels, two of the output each
    const uint32_t lo = t.ve[b / 2][(b % 2) * 2], hi = t.ve[b / 2][(b % 2) * 2 + 1];
    const float f[8] = {byte_scale<0>(lo), byte_scale<1>(lo), byte_scale<2>(lo),
                        byte_scale<3>(lo), byte_scale<0>(hi), byte_scale<1>(hi),
                        byte_scale<2>(hi), byte_scale<3>(hi)};
    const bf16x8 v0 = as_bf16(dequantise8(t.v[b / 2][(2 * b) % 4], 1.f));
    const bf16x8 v1 = as_bf16(dequantise8(t.v[b / 2][(2 * b) % 4 + 1], 1.f));
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      u16x8 w;
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = f32_to_bf16_bits(x[c][e] * f[e]);
      st[c].acc[2 * b] = mfma_bf16(v0, as_bf16(w), st[c].acc[2 * b]);
      st[c].acc[2 * b + 1] = mfma_bf16(v1, as_bf16(w), st[c].acc[2 * b + 1]);
    }
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
  constexpr int PF = 2;  // tiles in registers: one in use, one on its way
  __shared__ SpanShared<D, NB, W> sm;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
  const int each = sp.tiles / nb, more = sp.tiles - each * nb;  // the first `more` take one more
  const int k0 = j * each + min(j, more), k1 = k0 + each + (j < more ? 1 : 0);

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
    clear_rows(st[c]);
  }

  int it = k0 + wave;
  if (it < k1) {
    // Requests past the run's end repeat its last tile, so that every path
    // through the loop has the same loads in flight.
    typename std::conditional<Q4, Codes<D>, Tile<D>>::type t[PF];
#pragma unroll
    for (int s = 0; s < PF - 1; ++s) load(t[s], min(it + s * W, k1 - 1));
    for (bool left = true; left;) {
#pragma unroll
      for (int s = 0; s < PF; ++s) {
        if (it >= k1) {
          left = false;
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
  const int part_floats = p.chunk_rows * D;  // one partial's outputs, [row][channel]
  const int segments = (p.runs + kSpanSegment - 1) / kSpanSegment;
  const int slots = p.runs + segments;
  float* const unit_acc = nb > 1 ? p.part_acc + uc * slots * part_floats : nullptr;
  float* const unit_ml = nb > 1 ? p.part_ml + uc * slots * p.chunk_rows * 2 : nullptr;
  const __amdgpu_buffer_rsrc_t rsrc =
      device_rsrc(unit_acc, nb > 1 ? static_cast<uint32_t>(slots * part_floats * 4) : 0u);
  // Row rr, channels d .. d + 3 of partial `slot`, or of the output (slot -1).
  auto put = [&](int slot, int rr, int d, f32x4 o, float m, float den) {
    if (slot < 0) {
      // A row that attends nothing is zero; one whose scores are all -inf has a
      // denominator of zero too, and is NaN.
      f32x4 y = sp.L > 0 ? o * __builtin_amdgcn_rcpf(den) : f32x4{0.f, 0.f, 0.f, 0.f};
      // Held values are finite or NaN, and so are their sums (kLead): an infinite
      // one comes from an exponent byte of 255, which scales weights by inf here.
      if constexpr (Q4) y += o * 0.f;
      store4_as<D>(p.out, p.out_bf16, out_row + rr, d, y);
      return;
    }
    store4_device(rsrc, (slot * part_floats + rr * D + d) * 4, o);
    if (d == 0) {
      store_device(&unit_ml[(slot * p.chunk_rows + rr) * 2 + 0], m);
      store_device(&unit_ml[(slot * p.chunk_rows + rr) * 2 + 1], den);
    }
  };
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    if (grp == 0) {
      // A row of which this wave attended nothing has no reference.
      sm.m[wave][c * 16 + col] = st[c].den[0] == 0.f ? -INFINITY : st[c].m;
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
    put(nb == 1 ? -1 : j, rr, d, o, M, wsum);
  }
  if (nb == 1) return;

  // Merge the unit's runs in two steps, each in the order of the runs, so that
  // results do not depend on which workgroup is the last: the last of a
  // segment of kSpanSegment runs merges it (one round trip, the segments on
  // as many compute units), the last segment's merges the segments.
  int* const counters = p.counters + uc * (1 + segments);
  auto last_of = [&](int* counter, int count) -> bool {
    // Every other one bumped the counter after its partials completed: the
    // device-scope loads of the merge see them.
    wait_stores_complete();
    __syncthreads();
    if (threadIdx.x == 0) {
      sm.last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                count - 1;
      if (sm.last)  // ready for the next call on this workspace
        __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return sm.last;
  };
  auto merge = [&](int first, int count, int into) {
    for (int idx = threadIdx.x; idx < n_rows * D4; idx += NT) {
      const int rr = idx / D4;
      float M = -INFINITY, den = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      for (int s0 = 0; s0 < count; s0 += kSpanSegment) {
        float m[kSpanSegment], w[kSpanSegment];
        f32x4 a[kSpanSegment];
#pragma unroll
        for (int u = 0; u < kSpanSegment; ++u) {
          m[u] = -INFINITY;
          w[u] = 0.f;
          a[u] = f32x4{0.f, 0.f, 0.f, 0.f};
          if (s0 + u < count) {
            const int slot = first + s0 + u;
            float* ml = &unit_ml[(slot * p.chunk_rows + rr) * 2];
            m[u] = load_device(ml);
            w[u] = load_device(ml + 1);
            a[u] = load4_device(rsrc, (slot * part_floats + idx * 4) * 4);
          }
        }
        float bm = M;
#pragma unroll
        for (int u = 0; u < kSpanSegment; ++u) bm = fmaxf(bm, m[u]);
        const float ref = merge_reference(bm);
        const float sc = fast_exp2(M - ref);  // 0 while nothing is accumulated
        den *= sc;
        o *= sc;
#pragma unroll
        for (int u = 0; u < kSpanSegment; ++u) {
          const float f = fast_exp2(m[u] - ref);
          den += f * w[u];
          o += f * a[u];
        }
        M = bm;
      }
      put(into, rr, (idx - rr * D4) * 4, o, M, den);
    }
  };
  const int seg = j / kSpanSegment, n_seg = (nb + kSpanSegment - 1) / kSpanSegment;
  const int in_seg = min(kSpanSegment, nb - seg * kSpanSegment);
  if (!last_of(counters + 1 + seg, in_seg)) return;
  merge(seg * kSpanSegment, in_seg, n_seg == 1 ? -1 : p.runs + seg);
  if (n_seg == 1 || !last_of(counters, n_seg)) return;
  merge(p.runs, n_seg, -1);
}

template <int D, int NB, bool Q4>
hipError_t launch_span_t(const SpanParams& p, hipStream_t stream, hipEvent_t start,
                         hipEvent_t stop) {
  const dim3 grid((p.items + 7) / 8 * 8 * static_cast<unsigned>(p.chunks));
  const dim3 threads(64 * p.waves);
  auto kernel = p.waves == kWideWaves ? span_kernel<D, NB, kWideWaves, Q4>
                                      : span_kernel<D, NB, kWaves, Q4>;
  if (start)
    hipExtLaunchKernelGGL(kernel, grid, threads, 0, stream, start, stop, 0, p);
  else
    hipLaunchKernelGGL(kernel, grid, threads, 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_span(const SpanParams& p, int head_dim, hipStream_t stream, hipEvent_t start,
                       hipEvent_t stop) {
  const bool two = p.chunk_rows > 16;
  if (p.waves != kWaves && p.waves != kWideWaves) return hipErrorInvalidValue;
  if (p.chunk_rows > 16 * span_max_blocks(head_dim, p.q4)) return hipErrorInvalidValue;
  if (p.q4) {
    if (head_dim == 64)
      return two ? launch_span_t<64, 2, true>(p, stream, start, stop)
                 : launch_span_t<64, 1, true>(p, stream, start, stop);
    return two ? launch_span_t<128, 2, true>(p, stream, start, stop)
               : launch_span_t<128, 1, true>(p, stream, start, stop);
  }
  if (head_dim == 64)
    return two ? launch_span_t<64, 2, false>(p, stream, start, stop)
               : launch_span_t<64, 1, false>(p, stream, start, stop);
  return launch_span_t<128, 1, false>(p, stream, start, stop);
}

}  // namespace mlkv
