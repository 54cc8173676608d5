// Device helpers of the prefill kernels: where a query row stands, direct
// global-to-LDS loads, tiles staged by them, output stores.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "tile.h"

namespace mlkv {

// Wait until this wave's vector memory loads, the direct loads included,
// have landed (vmcnt(0); the other counters are left alone).
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8)); }

// 16 bytes of every lane from base + off (base wave-uniform) to LDS at the
// wave-uniform dst + 16 lane.
// (The host pass knows neither the builtin's size 16 nor LDS pointers, and a
// template that names them cannot be instantiated twice there.)
__device__ __forceinline__ void load_lds16(const char* base, unsigned off, uint16_t* dst) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds(static_cast<const void*>(base + off),
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
#endif
}

// Query row rho of unit (b, r): its token and its place in q and out
// (elements); rows past the end are not valid and stand at token 0.
struct RowPlace {
  size_t offset;
  int tok;
  bool valid;
};
__device__ __forceinline__ RowPlace row_place(const PrefillParams& p, int rho, int rows, int b,
                                              int group, int r, int D) {
  RowPlace at;
  const int R = p.layers * p.G;
  at.valid = rho < rows;
  at.tok = at.valid ? rho / R : 0;
  const int c = at.valid ? rho - at.tok * R : 0;
  const int layer = c / p.G;
  const int head = (r - group * p.kv_per_layer) * p.G + c - layer * p.G;
  at.offset = (((static_cast<size_t>(group * p.layers + layer) * p.B + b) * p.T + at.tok) * p.h +
               head) * D;
  return at;
}

// Four channels at element `off` of the output, fp32 or bf16.
__device__ __forceinline__ void store4(const PrefillParams& p, size_t off, f32x4 o) {
  if (p.out_bf16) {
    const uint32_t lo = f32_to_bf16_bits(o[0]) | (static_cast<uint32_t>(f32_to_bf16_bits(o[1])) << 16);
    const uint32_t hi = f32_to_bf16_bits(o[2]) | (static_cast<uint32_t>(f32_to_bf16_bits(o[3])) << 16);
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + off) = make_uint2(lo, hi);
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + off) = o;
  }
}

// Maximum of a lane's eight values.  Over multiply-add results (canonical
// floats) the compiler forms three-input maxima with no canonicalising maxes;
// being compiler-visible, the reads of matrix-core results also get the wait
// states the hardware requires after a matrix-core write.
__device__ __forceinline__ float max8(const float (&x)[8]) {
  return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
               fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
}

// A 32-token tile staged in LDS by direct global-to-LDS loads (lane l of a
// wave writes its 16 bytes at the wave-uniform LDS address + 16 l: no registers
// hold a tile in transit), double-buffered and shared by the workgroup's four
// waves.  Key chunks keep the plane's order, in which a wave's operand reads
// are contiguous; the value chunk of channel c and 8-token part p sits at slot
// 4 c + (p ^ vswz16(c)).  A 16-byte read serves the lanes 0-3, 12-15 and 20-27
// together, then 4-11, 16-19 and 28-31 (and the same in the upper half): with
// this order their sixteen slots are distinct modulo 16, and the conflict
// counter reads zero, where an order distinct over sixteen consecutive lanes
// lost a third of the LDS cycles (one layer of 32 heads of 128 channels, 200
// new tokens on 8000: 139 -> 123 us).
constexpr int kRing = 2;
__device__ __forceinline__ int vswz16(int c) { return ((c >> 3) & 1) * 3; }

template <int D>
struct TileRing {
  alignas(16) uint16_t k[kRing][kTile * D];
  alignas(16) uint16_t v[kRing][kTile * D];

  // Requests the tile at position t0 into buffer s: 2 D/64 loads per wave.
  __device__ __forceinline__ void issue(int s, const uint16_t* kbase, const uint16_t* vbase, int t0) {
    const unsigned lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned voff = (lane >> 2) * 64 + (((lane & 3) ^ vswz16(lane >> 2)) * 16);
#pragma unroll
    for (int u = 0; u < D / 64; ++u) {
      const int piece = u * 4 + wave;  // 1 KB pieces: sixteen channels of the value tile
      const size_t at = static_cast<size_t>(t0) * D * 2 + piece * 1024;
      load_lds16(reinterpret_cast<const char*>(kbase) + at, lane * 16, &k[s][piece * 512]);
      load_lds16(reinterpret_cast<const char*>(vbase) + at, voff, &v[s][piece * 512]);
    }
  }

  // A wave's MFMA operands of one tile from buffer s (the register layout of
  // load_tile: permuted key rows, V^T rows).
  __device__ __forceinline__ void read(Tile<D>& t, int s, int col, int grp) const {
    const int lane = grp * 16 + col;
#pragma unroll
    for (int sb = 0; sb < 2; ++sb)
#pragma unroll
      for (int kk = 0; kk < Tile<D>::KK; ++kk)
        t.k[sb][kk] = *reinterpret_cast<const u16x8*>(&k[s][((sb * Tile<D>::KK + kk) * 64 + lane) * 8]);
#pragma unroll
    for (int db = 0; db < Tile<D>::DB; ++db) {
      const int c = db * 16 + col;
      t.v[db] = *reinterpret_cast<const u16x8*>(&v[s][(c * 4 + (grp ^ vswz16(c))) * 8]);
    }
  }
};

}  // namespace mlkv
