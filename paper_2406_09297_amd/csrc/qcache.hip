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
//
// A block of 32 channels with largest magnitude a is held as codes c of e2m1
// (+-0, 0.5, 1, 1.5, 2, 3, 4, 6) times 2^e, e the least with a < 7 2^e: the top
// code's rounding range ends there, so each value is the nearest that its scale
// can hold and none saturates below 7 2^125; from there on (bf16's last eighth of
// a binade) values are held as 6 2^125, as 4 2^126 is no bf16 number.  A row x of a query or key becomes
// y = w x / sqrt(mean(x^2) + eps), its pairs (j, j + half) turned by pos
// times the pair's angle, in fp32 and rounded once.
//
// Bound by the bytes of rows and records in a large call and by one tile's
// chain of loads, LDS and stores in a small one: a tile a workgroup has many of
// those chains on every compute unit, and whole tiles are what lets a value
// dword (eight tokens of a channel) have one writer.  us:
//   64 sequences of 8256 rows of 8 heads of 128 channels (2.73 GB)  545, 5.0 TB/s
//   8 sequences of 2000 rows of 4 heads of 64 (20.7 MB)             5.8, 3.6 TB/s
//   one row of each of 128 sequences                                2.8
//   norm and rotation, bf16 cache, 8 sequences of 2000 rows, 12
//   query and 4 KV heads of 64 (82 MB)                             17.7, 4.6 TB/s
//   4 sequences of 2000, 32 and 8 heads of 128, all turned (197 MB) 47, 4.2 TB/s
//   one row of each of 64 sequences, the same heads               6.2
// (a copy of 0.5 to 4 GB reaches 4.6 to 5.3 TB/s, read and written).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qcache.h"
#include "serve.h"
#include "tile.h"

namespace mlkv {

namespace {

// A grid has fewer than 2^32 threads along x: more workgroups go along y.
constexpr unsigned kGridX = 1u << 23;
dim3 item_grid(unsigned items) {
  return items <= kGridX ? dim3(items) : dim3(kGridX, (items + kGridX - 1) / kGridX);
}
__device__ __forceinline__ unsigned item_of_block() { return blockIdx.y * kGridX + blockIdx.x; }

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

// Sums over the D / 8 lanes of a row, in every lane of it: within a quad, then
// with the other quad of eight and the other half of sixteen lanes (mirrored:
// what is equal in all lanes of a half may come from any of them).
template <int ctrl>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, 0xF, 0xF, true));
}
template <int D>
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<0xB1>(x);   // quad_perm 1 0 3 2
  x += dpp<0x4E>(x);   // quad_perm 2 3 0 1
  x += dpp<0x141>(x);  // row_half_mirror
  if (D == 128) x += dpp<0x140>(x);  // row_mirror
  return x;
}

// What a thread needs for its channels c0 .. c0 + 7 of every row: their norm
// weights and the lane that has the channels they are turned with (fetched from
// it after its norm; reading and norming them twice took a tenth longer).
template <int D>
struct Lane {
  int c0, partner;    // partner: first channel of the other eight
  int from;           // and the lane that has them, times 4
  bool normed, turned, hi;
  float w[8];
  __device__ __forceinline__ Lane(const uint16_t* weight, int c0_, int half) : c0(c0_) {
    turned = c0 < 2 * half;
    hi = c0 >= half;
    partner = !turned ? c0 : hi ? c0 - half : c0 + half;
    from = 4 * ((static_cast<int>(threadIdx.x) & 63 & ~(D / 8 - 1)) + partner / 8);
    normed = weight != nullptr;
    if (normed) {
      const u16x8 a = load16(weight + c0);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = bf16_to_f32(a[i]);
    }
  }
};

// Where a token's (cos, sin) of a pair stand in LDS: two pairs of each lane's
// eight side by side, then the next two, so that a row's lanes read 16 bytes
// each from neighbouring places (in the order of pairs, lanes are 64 bytes apart
// and meet each other's banks: one token on 256 sequences, 32 and 8 heads of
// 128 channels, all turned, 12.7 us; so, 11.0).
__device__ __forceinline__ int angle_place(int pair, int half) {
  return (pair >> 1 & 3) * (half / 4) + (pair >> 3) * 2 + (pair & 1);
}

// A row's eight channels: divided by the row's root mean square and weighted,
// then rotated with the angles at cs (those of the row's token) of the lane's
// pairs, in fp32, rounded once to bf16.  All D / 8 lanes of a row take part.
template <int D>
__device__ __forceinline__ u16x8 norm_rotate(const Lane<D>& ln, u16x8 raw, const StoreParams& p,
                                             const float2* cs) {
  const int half = p.half;
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = bf16_to_f32(raw[i]);
  if (ln.normed) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
    float mean = row_sum<D>(ss) * (1.f / D) + p.eps;
    // Squares, or an eps, that leave fp32 at either end: the same row times a power
    // of two (the quotient does not change).  A row's lanes take one side together.
    if (!(mean < INFINITY) || mean < 0x1p-90f) {
      const bool up = mean < 1.f;
      const float scale = up ? 0x1p80f : 0x1p-80f;
      ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= scale;
        ss = fmaf(x[i], x[i], ss);
      }
      mean = row_sum<D>(ss) * (1.f / D) + (up ? p.eps_up : p.eps_down);
    }
    const float inv = __builtin_amdgcn_rsqf(mean);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * inv * ln.w[i];
  }
  if (half) {
    float y[8];  // the channels that these are turned with, from their lane
#pragma unroll
    for (int i = 0; i < 8; ++i)
      y[i] = __builtin_bit_cast(
          float, __builtin_amdgcn_ds_bpermute(ln.from, __builtin_bit_cast(int, x[i])));
    if (ln.turned) {
      const float2* at = cs + angle_place(ln.hi ? ln.partner : ln.c0, half);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float4 t = *reinterpret_cast<const float4*>(at + i / 2 * (half / 4));
        x[i] = fmaf(x[i], t.x, ln.hi ? y[i] * t.y : -(y[i] * t.y));
        x[i + 1] = fmaf(x[i + 1], t.z, ln.hi ? y[i + 1] * t.w : -(y[i + 1] * t.w));
      }
    }
  }
  u16x8 out;
#pragma unroll
  for (int i = 0; i < 8; ++i) out[i] = f32_to_bf16_bits(x[i]);
  return out;
}

__device__ __forceinline__ double turns_of(const StoreParams& p, int j) {
  return p.coarse[j >> 3] * p.fine[j & 7];
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

// The angles are done with when the values come (one place for both: eight
// waves a SIMD instead of six with 128 channels, 11.0 -> 10.0 us for that token).
template <int D, bool NORM>
struct alignas(16) StoreShared {
  union {
    float2 cs[NORM ? kAngleTokens * (D / 2) : 1];
    uint32_t nib[kTile * D / 4];       // value codes, a byte each: [token][channel]
    // Values: [token][channel]; rows four elements longer, so that the lanes
    // that read four groups of eight tokens meet four sets of banks.
    uint16_t val[kTile][D + 4];
  };
};

// j / p.half for the j < kAngleTokens * kMaxRopePairs < 2^12 angles of a
// workgroup: the factor is above 2^20 / half by less than one, the product above
// j 2^20 / half by less than 2^12, under one part in half.
__device__ __forceinline__ int angle_token(const StoreParams& p, unsigned j) {
  return static_cast<int>(__umul24(j, p.inv_half) >> 20);
}

// Queries: p.q_rows consecutive rows (token by token, head by head), the lanes
// of a row side by side.  The first rows are requested ahead of the angles and
// the next ones ahead of the arithmetic.
template <int D>
__device__ __forceinline__ void norm_queries(const StoreParams& p, unsigned item, float2* cs) {
  constexpr int C8 = D / 8;
  constexpr int ROWS = kStoreThreads / C8;
  const unsigned total = static_cast<unsigned>(p.B) * p.T * p.h;
  const unsigned first = item * p.q_rows, end = min(first + p.q_rows, total);
  const Lane<D> ln(p.q_w, (threadIdx.x % C8) * 8, p.half);
  u16x8 raw;
  unsigned r = first + threadIdx.x / C8, tok, head;
  auto request = [&]() {
    const unsigned at = min(r, end - 1);  // rows past the end repeat the last one
    tok = quotient(at, p.h, p.inv_h);
    head = at - tok * p.h;
    const uint16_t* row = p.q + tok * p.q_stride + head * D;
    raw = load16(row + ln.c0);
  };
  request();
  const unsigned tok0 = first / static_cast<unsigned>(p.h);
  if (p.half) {
    const unsigned n_tok = (end - 1) / static_cast<unsigned>(p.h) + 1 - tok0;
    for (unsigned j = threadIdx.x; j < n_tok * p.half; j += kStoreThreads) {
      const unsigned i = angle_token(p, j), g = tok0 + i, b = g / static_cast<unsigned>(p.T);
      const int pair = j - i * p.half;
      cs[i * p.half + angle_place(pair, p.half)] =
          cos_sin(static_cast<long>(p.starts[b]) + (g - b * p.T), turns_of(p, pair));
    }
    __syncthreads();
  }
  for (unsigned r0 = first; r0 < end; r0 += ROWS) {
    const u16x8 x = raw;
    const unsigned row = r, t = tok, hd = head;
    r += ROWS;
    if (r0 + ROWS < end) request();
    const u16x8 out = norm_rotate<D>(ln, x, p, cs + (t - tok0) * p.half);
    if (row < end)
      *reinterpret_cast<u16x8*>(p.q_out + (static_cast<size_t>(t) * p.h + hd) * D + ln.c0) = out;
  }
}

template <int D, bool Q4, bool NORM>
__global__ __launch_bounds__(kStoreThreads) void store_kernel(StoreParams p) {
  constexpr int C8 = D / 8;
  constexpr int ROWS = kStoreThreads / C8;  // token rows a pass of the workgroup takes
  constexpr int PASSES = kTile / ROWS;
  __shared__ StoreShared<D, NORM> sm;
  float2* const cs = sm.cs;
  const unsigned item = item_of_block();
  if (item >= p.store_items) {
    if (NORM && item - p.store_items < p.q_items) norm_queries<D>(p, item - p.store_items, cs);
    return;
  }
  const unsigned unit = item / static_cast<unsigned>(p.tiles);
  const int tile = static_cast<int>(item - unit * p.tiles);
  const int b = static_cast<int>(unit / static_cast<unsigned>(p.kv_count));
  const int c = static_cast<int>(unit - static_cast<unsigned>(b) * p.kv_count);
  const int c8 = threadIdx.x % C8, row = threadIdx.x / C8;
  const int c0 = c8 * 8;
  const long start = p.starts ? p.starts[b] : 0;
  const long s0 = ((start >> 5) + tile) * kTile;  // the tile's first slot
  // Its slots that take a row.
  const long lo = max(max(start, s0), 0L);
  const long end = min(min(start + p.T, s0 + kTile), static_cast<long>(p.S));
  if (lo >= end) return;  // uniform over the workgroup
  const int u_lo = static_cast<int>(lo - s0), u_end = static_cast<int>(end - s0);
  const size_t seq = static_cast<size_t>(p.kv_begin + c) * p.B + b;
  uint8_t* const rec = Q4 ? p.q4 + (seq * (p.S / kTile) + s0 / kTile) * QTile<D>::kBytes : nullptr;
  const Lane<D> ln(NORM ? p.k_w : nullptr, c0, NORM ? p.half : 0);
  u16x8 xk[PASSES], xv[PASSES];
#pragma unroll
  for (int pass = 0; pass < PASSES; ++pass) {
    const int u = pass * ROWS + row;
    const u16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
    xk[pass] = xv[pass] = zero;
    if (u >= u_lo && u < u_end) {
      const size_t src = static_cast<size_t>(c) * p.s_head + static_cast<size_t>(b) * p.s_seq +
                         static_cast<size_t>(s0 + u - start) * p.s_tok;
      xk[pass] = load16(p.k_src + src + c0);
      xv[pass] = load16(p.v_src + src + c0);
    }
  }
  if (NORM && p.half) {
    for (int j = threadIdx.x + u_lo * p.half; j < u_end * p.half; j += kStoreThreads) {
      const int u = angle_token(p, j), pair = j - u * p.half;
      cs[u * p.half + angle_place(pair, p.half)] = cos_sin(s0 + u, turns_of(p, pair));
    }
    __syncthreads();
  }
#pragma unroll
  for (int pass = 0; pass < PASSES; ++pass) {
    const int u = pass * ROWS + row;
    u16x8 k = xk[pass];
    if (NORM) k = norm_rotate<D>(ln, k, p, cs + u * p.half);
    if (Q4) {
      const int e = block_exp(block_top(k));
      if (u >= u_lo && u < u_end) {
        *reinterpret_cast<uint32_t*>(rec + QTile<D>::k_dword(u, c8)) = quantise8(k, e);
        if (c8 % 4 == 0) rec[QTile<D>::k_exp(u, c8 / 4)] = static_cast<uint8_t>(e);
      }
    } else if (u >= u_lo && u < u_end) {
      *reinterpret_cast<u16x8*>(p.k + (seq * p.S + s0) * D + kchunk<D>(u, c8) * 8) = k;
    }
  }
  if (NORM && p.half) __syncthreads();  // the angles' place is the values'
#pragma unroll
  for (int pass = 0; pass < PASSES; ++pass) {
    const int u = pass * ROWS + row;
    const u16x8 v = xv[pass];
    if (Q4) {
      const int e = block_exp(block_top(v));
      const uint32_t nv = quantise8(v, e);
      // Nibbles 0 .. 3 and 4 .. 7 to bytes.
      uint32_t lo4 = nv & 0xFFFF, hi4 = nv >> 16;
      lo4 = (lo4 | lo4 << 8) & 0x00FF00FF;
      hi4 = (hi4 | hi4 << 8) & 0x00FF00FF;
      sm.nib[(u * D + c0) / 4] = (lo4 | lo4 << 4) & 0x0F0F0F0F;
      sm.nib[(u * D + c0) / 4 + 1] = (hi4 | hi4 << 4) & 0x0F0F0F0F;
      if (u >= u_lo && u < u_end && c8 % 4 == 0)
        rec[QTile<D>::v_exp(u, c8 / 4)] = static_cast<uint8_t>(e);
    } else {
      const uint4 d = __builtin_bit_cast(uint4, v);
      *reinterpret_cast<uint2*>(&sm.val[u][c0]) = make_uint2(d.x, d.y);
      *reinterpret_cast<uint2*>(&sm.val[u][c0 + 4]) = make_uint2(d.z, d.w);
    }
  }
  __syncthreads();
  // Values, eight tokens of a channel at a time; tokens without a new row keep
  // what the slot holds.
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
}

template <int D>
__global__ __launch_bounds__(kStoreThreads) void read_kernel(ReadParams p) {
  constexpr int C8 = D / 8;
  constexpr int ROWS = kStoreThreads / C8;
  __shared__ uint32_t codes[4 * D];  // the tile's value codes
  const int c8 = threadIdx.x % C8, row = threadIdx.x / C8;
  const unsigned item = item_of_block();
  if (item >= p.items) return;
  const unsigned unit = item / static_cast<unsigned>(p.tiles);
  const int tile = static_cast<int>(item - unit * p.tiles);
  const int c = static_cast<int>(unit / static_cast<unsigned>(p.B));
  const int b = static_cast<int>(unit - static_cast<unsigned>(c) * p.B);
  const long start = p.starts ? p.starts[b] : 0;
  const long s0 = ((start >> 5) + tile) * kTile;
  const long lo = max(start, s0), end = min(start + p.T, s0 + kTile);
  if (lo >= end) return;
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
}

}  // namespace

hipError_t launch_store(const StoreParams& p, int head_dim, bool norm, hipStream_t stream) {
  const dim3 grid = item_grid(p.store_items + (norm ? p.q_items : 0));
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
  hipLaunchKernelGGL(kernel, item_grid(p.items), dim3(kStoreThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace mlkv
