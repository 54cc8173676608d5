// Rows into and out of the caches for CDNA4 (gfx950, wave64): the 4-bit cache
// filled from bf16 rows and read back, and new tokens' queries and keys normed
// and rotated on their way to a cache of either kind.
//
//   store_kernel  new rows of KV heads -> cache; with NORM also queries
//   read_kernel   4-bit cache -> bf16 rows
//
// A workgroup takes the 32 slots of one tile of one (KV head, sequence); a
// thread eight channels of a token, the four threads of a 32-channel block
// side by side, so a block's largest magnitude takes two lane exchanges and a
// row's sum of squares three or four.  Values change from token-major to
// channel-major through LDS.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qcache.h"
#include "serve.h"
#include "tile.h"

namespace mlkv {

namespace {

constexpr int kStoreThreads = 256;
constexpr long kMaxStoreGrid = 1L << 20;  // workgroups; each takes every gridDim-th item

__device__ __forceinline__ float bf16_to_f32(uint16_t x) {
  return __builtin_bit_cast(float, static_cast<uint32_t>(x) << 16);
}

// Largest magnitude (bf16 pattern; anything not finite is above every finite
// one) of the 32 channels held by the four lanes of a block.
__device__ __forceinline__ int block_top(u16x8 x) {
  int top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, static_cast<int>(x[i] & 0x7FFF));
  top = max(top, __shfl_xor(top, 1));
  return max(top, __shfl_xor(top, 2));
}

// One row's eight channels from c0 on: divided by the row's root mean square
// and weighted (w not null), then rotated with cs[0 .. half) = (cos, sin) of
// the row's token, in fp32, rounded once to bf16.  All D / 8 lanes of a row
// take part.
template <int D>
__device__ __forceinline__ u16x8 norm_rotate(u16x8 raw, const uint16_t* w, float eps, int c0,
                                             int half, const float2* cs) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = bf16_to_f32(raw[i]);
  if (w) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
    for (int s = 1; s < D / 8; s *= 2) ss += __shfl_xor(ss, s);
    const float inv = 1.f / sqrtf(ss * (1.f / D) + eps);
    const u16x8 wv = load16(w + c0);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * inv * bf16_to_f32(wv[i]);
  }
  if (half) {
    const bool hi = c0 >= half;
    const int partner = static_cast<int>(threadIdx.x & 63) + (hi ? -half : half) / 8;
    const bool turned = c0 < 2 * half;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], partner & 63);
    if (turned) {
      const float2* t = cs + (hi ? c0 - half : c0);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        x[i] = hi ? fmaf(x[i], t[i].x, y[i] * t[i].y) : fmaf(x[i], t[i].x, -(y[i] * t[i].y));
    }
  }
  u16x8 out;
#pragma unroll
  for (int i = 0; i < 8; ++i) out[i] = f32_to_bf16_bits(x[i]);
  return out;
}

// cos and sin of pair j at position pos: the turns in 64 bits (a position of
// 2^31 leaves 20 bits and more of its fraction), of which only the fraction
// counts, then in 32.
__device__ __forceinline__ float2 cos_sin(long pos, double turns) {
  double r = static_cast<double>(pos) * turns;
  r -= rint(r);
  float s, c;
  sincospif(2.f * static_cast<float>(r), &s, &c);
  return make_float2(c, s);
}

template <int D>
struct StoreShared {
  union {
    uint32_t nib[kTile * D / 4];       // value codes, a byte each: [token][channel]
    uint16_t val[kTile][D];            // values: [token][channel]
  };
};

template <int D, bool Q4, bool NORM>
__global__ __launch_bounds__(kStoreThreads) void store_kernel(StoreParams p) {
  constexpr int C8 = D / 8;
  constexpr int ROWS = kStoreThreads / C8;  // token rows a pass of the workgroup takes
  constexpr int PASSES = kTile / ROWS;
  __shared__ StoreShared<D> sm;
  __shared__ float2 cs[NORM ? kTile * kMaxRopePairs : 1];
  const int c8 = threadIdx.x % C8, row = threadIdx.x / C8;
  const int c0 = c8 * 8;
  for (long item = blockIdx.x; item < p.store_items + (NORM ? p.q_items : 0); item += gridDim.x) {
    if (NORM && item >= p.store_items) {
      // Queries: q_tokens tokens of one sequence, all heads.
      const long i = item - p.store_items;
      const int per = (p.T + p.q_tokens - 1) / p.q_tokens;
      const int b = static_cast<int>(i / per), t0 = static_cast<int>(i % per) * p.q_tokens;
      const int n_tok = min(p.q_tokens, p.T - t0);
      const long pos0 = (p.starts ? p.starts[b] : 0) + static_cast<long>(t0);
      for (int j = threadIdx.x; j < n_tok * p.half; j += kStoreThreads) {
        const int tok = j / p.half, pair = j - tok * p.half;
        cs[j] = cos_sin(pos0 + tok, p.turns[pair]);
      }
      __syncthreads();
      const int rows = n_tok * p.h;
      for (int r0 = 0; r0 < rows; r0 += ROWS) {
        const int r = min(r0 + row, rows - 1);  // rows past the end repeat the last one
        const int tok = r / p.h, head = r - tok * p.h;
        const size_t bt = static_cast<size_t>(b) * p.T + t0 + tok;
        const u16x8 x = load16(p.q + bt * p.q_stride + head * D + c0);
        const u16x8 y = norm_rotate<D>(x, p.q_w, p.eps, c0, p.half, cs + tok * p.half);
        if (r0 + row < rows)
          *reinterpret_cast<u16x8*>(p.q_out + (bt * p.h + head) * D + c0) = y;
      }
      __syncthreads();
      continue;
    }
    const int tile = static_cast<int>(item % p.tiles);
    const long unit = item / p.tiles;
    const int c = static_cast<int>(unit % p.kv_count), b = static_cast<int>(unit / p.kv_count);
    const long start = p.starts ? p.starts[b] : 0;
    const long s0 = ((start >> 5) + tile) * kTile;  // the tile's first slot
    // Its slots that take a row.
    const long lo = max(max(start, s0), 0L), end = min(min(start + p.T, s0 + kTile),
                                                       static_cast<long>(p.S));
    if (lo >= end) continue;  // uniform over the workgroup
    const int u_lo = static_cast<int>(lo - s0), u_end = static_cast<int>(end - s0);
    const size_t seq = static_cast<size_t>(p.kv_begin + c) * p.B + b;
    uint8_t* const rec =
        Q4 ? p.q4 + (seq * (p.S / kTile) + s0 / kTile) * QTile<D>::kBytes : nullptr;
    if (NORM && p.half) {
      for (int j = threadIdx.x + u_lo * p.half; j < u_end * p.half; j += kStoreThreads) {
        const int u = j / p.half;
        cs[j] = cos_sin(s0 + u, p.turns[j - u * p.half]);
      }
      __syncthreads();
    }
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
      const int u = pass * ROWS + row;
      const bool live = u >= u_lo && u < u_end;
      u16x8 xk = {0, 0, 0, 0, 0, 0, 0, 0}, xv = xk;
      if (live) {
        const size_t src = static_cast<size_t>(c) * p.s_head + static_cast<size_t>(b) * p.s_seq +
                           static_cast<size_t>(s0 + u - start) * p.s_tok + c0;
        xk = load16(p.k_src + src);
        xv = load16(p.v_src + src);
      }
      if (NORM) xk = norm_rotate<D>(xk, p.k_w, p.eps, c0, p.half, cs + u * p.half);
      if (Q4) {
        const int ek = block_exp(block_top(xk)), ev = block_exp(block_top(xv));
        const uint32_t nv = quantise8(xv, ev);
        // Nibbles 0 .. 3 and 4 .. 7 to bytes.
        uint32_t lo4 = nv & 0xFFFF, hi4 = nv >> 16;
        lo4 = (lo4 | lo4 << 8) & 0x00FF00FF;
        hi4 = (hi4 | hi4 << 8) & 0x00FF00FF;
        sm.nib[(u * D + c0) / 4] = (lo4 | lo4 << 4) & 0x0F0F0F0F;
        sm.nib[(u * D + c0) / 4 + 1] = (hi4 | hi4 << 4) & 0x0F0F0F0F;
        if (live) {
          *reinterpret_cast<uint32_t*>(rec + QTile<D>::k_dword(u, c8)) = quantise8(xk, ek);
          if (c8 % 4 == 0) {
            rec[QTile<D>::k_exp(u, c8 / 4)] = static_cast<uint8_t>(ek);
            rec[QTile<D>::v_exp(u, c8 / 4)] = static_cast<uint8_t>(ev);
          }
        }
      } else {
        if (live)
          *reinterpret_cast<u16x8*>(p.k + (seq * p.S + s0) * D + kchunk<D>(u, c8) * 8) = xk;
        *reinterpret_cast<u16x8*>(&sm.val[u][c0]) = xv;
      }
    }
    __syncthreads();
    // Values, eight tokens of a channel at a time; tokens without a new row
    // keep what the slot holds.
    for (int i = threadIdx.x; i < 4 * D; i += kStoreThreads) {
      int d, g;
      if (Q4) {  // in the order of the record's dwords
        const int lane = (i >> 2) & 63;
        d = ((i >> 8) * 4 + (i & 3)) * 16 + (lane & 15);
        g = lane >> 4;
      } else {
        d = i >> 2;
        g = i & 3;
      }
      const int first = max(u_lo - 8 * g, 0), last = min(u_end - 8 * g, 8);
      if (first >= last) continue;
      if (Q4) {
        uint32_t* dst = reinterpret_cast<uint32_t*>(rec + QTile<D>::kVCodes) + i;
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          w |= static_cast<uint32_t>(reinterpret_cast<const uint8_t*>(sm.nib)[(8 * g + e) * D + d])
               << (4 * e);
        if (last - first < 8) {
          const uint32_t taken =
              (last == 8 ? ~0u : (1u << (4 * last)) - 1) & ~((1u << (4 * first)) - 1);
          w = (w & taken) | (*dst & ~taken);
        }
        *dst = w;
      } else {
        uint16_t* dst = p.v + (seq * p.S + s0) * D + d * kTile + 8 * g;
        u16x8 w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = sm.val[8 * g + e][d];
        if (last - first == 8) {
          *reinterpret_cast<u16x8*>(dst) = w;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e >= first && e < last) dst[e] = w[e];
        }
      }
    }
    __syncthreads();  // the next item reuses the LDS
  }
}

template <int D>
__global__ __launch_bounds__(kStoreThreads) void read_kernel(ReadParams p) {
  constexpr int C8 = D / 8;
  constexpr int ROWS = kStoreThreads / C8;
  __shared__ uint32_t codes[4 * D];  // the tile's value codes
  const int c8 = threadIdx.x % C8, row = threadIdx.x / C8;
  for (long item = blockIdx.x; item < p.items; item += gridDim.x) {
    const int tile = static_cast<int>(item % p.tiles);
    const long unit = item / p.tiles;
    const int b = static_cast<int>(unit % p.B), c = static_cast<int>(unit / p.B);
    const long start = p.starts ? p.starts[b] : 0;
    const long s0 = ((start >> 5) + tile) * kTile;
    const long lo = max(start, s0), end = min(start + p.T, s0 + kTile);
    if (lo >= end) continue;
    const bool held = s0 >= 0 && s0 < p.S;  // other slots read as zeros
    const size_t seq = static_cast<size_t>(p.kv_begin + c) * p.B + b;
    const uint8_t* rec = p.q4 + (seq * (p.S / kTile) + (held ? s0 / kTile : 0)) * QTile<D>::kBytes;
    if (held)
      for (int i = threadIdx.x; i < 4 * D; i += kStoreThreads)
        codes[i] = reinterpret_cast<const uint32_t*>(rec + QTile<D>::kVCodes)[i];
    __syncthreads();
    for (int u = row; u < kTile; u += ROWS) {
      if (s0 + u < lo || s0 + u >= end) continue;
      u16x8 xk = {0, 0, 0, 0, 0, 0, 0, 0}, xv = xk;
      if (held) {
        xk = dequantise8(*reinterpret_cast<const uint32_t*>(rec + QTile<D>::k_dword(u, c8)),
                         exp_scale(rec[QTile<D>::k_exp(u, c8 / 4)]));
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int d = c8 * 8 + e, db = d >> 4;
          const int at = (db >> 2) * 256 + ((u >> 3) * 16 + (d & 15)) * 4 + (db & 3);
          w |= ((codes[at] >> (4 * (u & 7))) & 15) << (4 * e);
        }
        xv = dequantise8(w, exp_scale(rec[QTile<D>::v_exp(u, c8 / 4)]));
      }
      const size_t dst = ((static_cast<size_t>(c) * p.B + b) * p.T +
                          static_cast<size_t>(s0 + u - start)) * D + c8 * 8;
      *reinterpret_cast<u16x8*>(p.k_rows + dst) = xk;
      *reinterpret_cast<u16x8*>(p.v_rows + dst) = xv;
    }
    __syncthreads();
  }
}

dim3 store_grid(long items) {
  return dim3(static_cast<unsigned>(items < kMaxStoreGrid ? items : kMaxStoreGrid));
}

}  // namespace

hipError_t launch_store(const StoreParams& p, int head_dim, bool norm, hipStream_t stream) {
  const dim3 grid = store_grid(p.store_items + (norm ? p.q_items : 0));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kStoreThreads), 0, stream, p);
    return hipGetLastError();
  };
  if (head_dim == 64) {
    if (norm) return p.q4 ? go(store_kernel<64, true, true>) : go(store_kernel<64, false, true>);
    return go(store_kernel<64, true, false>);
  }
  if (norm) return p.q4 ? go(store_kernel<128, true, true>) : go(store_kernel<128, false, true>);
  return go(store_kernel<128, true, false>);
}

hipError_t launch_qcache_read(const ReadParams& p, int head_dim, hipStream_t stream) {
  auto kernel = head_dim == 64 ? read_kernel<64> : read_kernel<128>;
  hipLaunchKernelGGL(kernel, store_grid(p.items), dim3(kStoreThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace mlkv
