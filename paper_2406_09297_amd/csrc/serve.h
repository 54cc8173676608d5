// Internal interface of the long-context serving operators: the 4-bit cache
// and its rows, attention over it or over a window, norm and rotation before
// the append.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "kernels.h"

namespace mlkv {

// The 4-bit cache: one record of 34 D bytes per (KV head, sequence, 32 tokens),
// in the order in which a wave's matrix operands take it.  A channel block is
// 32 channels of one token; KK = D / 32 of them make a row.
//   [0, 16 D)     key codes: 64 lanes x 16 bytes per piece; lane 16 g + r of the
//                 operand of score block sb and channel block kk holds channels
//                 32 kk + 8 g .. + 7 of token 8 (r / 4) + 4 sb + r % 4 in dword
//                 i % 4 of piece i / 4, i = sb KK + kk
//   [16 D, 32 D)  value codes: lane 16 g + r of output block db holds tokens
//                 8 g .. + 7 of channel 16 db + r in dword db % 4 of piece db / 4
//   [32 D, 33 D)  key exponents + 127, a byte each: [row r][sb][kk]
//   [33 D, 34 D)  value exponents + 127: [token / 8][channel block][token % 8]
constexpr int kQTileBytes(int head_dim) { return 34 * head_dim; }
// Exponents: the least holds no subnormal value, the largest overflows none;
// 255 marks a block with a value that is not finite: all of it is NaN.
constexpr int kQMinExp = 3, kQMaxExp = 252, kQNaN = 255;

// New rows into a cache: row (c, b, t) at src + c*s_head + b*s_seq + t*s_tok,
// D channels, to slot starts[b] + t (0 where starts is null) of KV head
// kv_begin + c; slots outside [0, S) are skipped.
struct StoreParams {
  const uint16_t *k_src, *v_src;
  size_t s_head, s_seq, s_tok;
  const int32_t* starts;
  uint8_t* q4;                // 4-bit cache, or null:
  uint16_t *k, *v;            // bf16 planes
  int B, T, S, kv_begin, kv_count;
  unsigned store_items;       // kv_count * B * tiles a sequence's rows may touch
  int tiles;
  // Norm and rotation of keys and queries (norm kernels only).
  const uint16_t *q_w, *k_w;  // [D] norm weights, or null: no norm
  const uint16_t* q;          // row (b, t) at q + (b*T + t)*q_stride: [h][D]
  uint16_t* q_out;            // [B][T][h][D]
  size_t q_stride;
  int h;
  unsigned q_rows, q_items;   // (token, head) rows of a query workgroup, and these workgroups
  uint32_t inv_h;             // (2^32 - 1) / h
  int half;                   // rotated channel pairs (0: none)
  unsigned inv_half;          // 2^20 / half, rounded up
  float eps, eps_up, eps_down;  // eps, and times 2^160 and 2^-160 (from 64 bits)
  // A position turns pair j by coarse[j / 8] * fine[j % 8] revolutions (64
  // products in the arguments cost 0.4 us a launch).
  double coarse[kMaxRopePairs / 8], fine[8];
};

struct ReadParams {
  const uint8_t* q4;
  uint16_t *k_rows, *v_rows;  // [kv_count][B][T][D]
  const int32_t* starts;      // row t of sequence b is slot starts[b] + t (null: t)
  int B, T, S, kv_begin, kv_count, tiles;
  unsigned items;
};

constexpr int kStoreThreads = 256;
constexpr int kAngleTokens = 33;  // whose sines a workgroup holds
hipError_t launch_store(const StoreParams& p, int head_dim, bool norm, hipStream_t stream);
hipError_t launch_qcache_read(const ReadParams& p, int head_dim, hipStream_t stream);

// Attention of one new token per sequence over a window and the first tokens:
// the token at position L_b - 1 attends positions p < L_b with p < sinks or
// p >= L_b - window (window 0: every position).  Unit u is (sequence u /
// n_groups, KV head kv_begin + u % n_groups); its G query rows in `chunks` of
// chunk_rows, its attended tiles in runs of at most run_tiles.
struct SpanParams {
  const uint16_t* q;   // [B][h][D]
  const uint16_t *k, *v;  // bf16 planes, or null:
  const uint8_t* q4;   // 4-bit cache
  const int32_t* lens; // [B]
  void* out;           // [B][h][D] fp32 or bf16
  // Of a unit's chunk, where it may have several runs: finished segments and
  // the finished runs of each (zero between calls); partials of the runs and
  // of the segments.
  int* counters;       // [units*chunks][1 + segments]
  float* part_acc;     // [units*chunks][runs + segments][chunk_rows][D]
  float* part_ml;      // [units*chunks][runs + segments][chunk_rows][2]
  int B, h, S;
  int kv_begin, n_groups, G;
  int chunks, chunk_rows, runs, run_tiles;
  int waves;           // of a workgroup: 4 or 8
  unsigned items;      // units * runs
  int max_len, window, sinks;
  int out_bf16;
  float scale_log2;    // log2(e) / sqrt(D)
};
// Most blocks of 16 query rows a wave takes: two share a tile's operands (us,
// two / one: 4-bit, 600 sequences of 3000 .. 4000 tokens, 32 heads of 128 on one
// KV head 76.6 / 84.1; bf16 of 64 channels, 900 windows of 2048, 91 / 98),
// except two of 128 channels beside bf16 tiles, which do not fit the registers
// (600 windows of 2048: 173 / 125; 64 of them 23.1 / 16.6).
constexpr int span_max_blocks(int head_dim, bool four_bits) {
  return head_dim == 128 && !four_bits ? 1 : 2;
}
constexpr int kSpanSegment = 8;    // runs merged by one workgroup
hipError_t launch_span(const SpanParams& p, int head_dim, hipStream_t stream, hipEvent_t start,
                       hipEvent_t stop);

// Causal prefill attention of one layer within a window: token t of sequence b
// stands at n = ctx[b] + t and attends positions p <= n with p < sinks or
// p > n - window.
constexpr int kWindowRows = 128;  // query rows of a workgroup
struct WindowPrefillParams : PrefillParams {
  int window, sinks;
  uint32_t inv_G;  // (2^32 - 1) / G
};
hipError_t launch_prefill_window(const WindowPrefillParams& p, int head_dim, hipStream_t stream,
                                 hipEvent_t start, hipEvent_t stop);

}  // namespace mlkv
