// C ABI of the long-context serving operators: the 4-bit cache, attention over
// it or within a window, norm and rotation before the append.  Every argument
// error is reported before any HIP call.
#include "mlkv.h"

#include <cfloat>
#include <cmath>

#include "host.h"
#include "serve.h"

using namespace mlkv::host;

namespace {

mlkv_status check_qcache(const mlkv_qcache* c) {
  if (!c) return fail(MLKV_ERR_INVALID_ARG, "cache is NULL");
  if (!c->data) return fail(MLKV_ERR_INVALID_ARG, "cache data must be non-NULL");
  if (!aligned16(c->data)) return fail(MLKV_ERR_ALIGNMENT, "cache data must be 16-byte aligned");
  if (c->batch <= 0 || c->capacity <= 0 || c->n_kv <= 0)
    return fail(MLKV_ERR_INVALID_ARG, "cache n_kv, batch and capacity must be positive");
  if (c->capacity % kTileTokens != 0)
    return fail(MLKV_ERR_CAPACITY, "cache capacity %d is not a multiple of 32", c->capacity);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(MLKV_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", c->head_dim);
  const double elems = 2.0 * c->n_kv * c->batch * static_cast<double>(c->capacity) * c->head_dim;
  if (elems > 9.0e18) return fail(MLKV_ERR_CAPACITY, "cache too large");
  return MLKV_OK;
}

mlkv_status check_qcache(const mlkv_qcache* c, const mlkv_map* map) {
  const mlkv_status s = check_qcache(c);
  if (s != MLKV_OK) return s;
  if (c->n_kv != map->n_kv)
    return fail(MLKV_ERR_INVALID_ARG, "cache has %d KV heads, map has %d", c->n_kv, map->n_kv);
  return MLKV_OK;
}

mlkv_status check_layer(const mlkv_map* map, int layer) {
  const mlkv_status s = check_map(map);
  if (s != MLKV_OK) return s;
  if (layer < 0 || layer >= map->l)
    return fail(MLKV_ERR_INVALID_ARG, "layer %d out of range", layer);
  return MLKV_OK;
}

mlkv_status check_tokens(int T, int capacity) {
  if (T < 0 || T > capacity)
    return fail(MLKV_ERR_CAPACITY, "T = %d new tokens: must be in [0, capacity %d]", T, capacity);
  return MLKV_OK;
}

mlkv_status check_new_rows(const void* k_new, const void* v_new, int row_stride, int owned,
                           int head_dim) {
  if (!k_new || !v_new) return fail(MLKV_ERR_INVALID_ARG, "k_new and v_new must be non-NULL");
  if (!aligned16(k_new) || !aligned16(v_new))
    return fail(MLKV_ERR_ALIGNMENT, "k_new and v_new must be 16-byte aligned");
  if (row_stride % 8 != 0 || row_stride < static_cast<long>(owned) * head_dim)
    return fail(MLKV_ERR_INVALID_ARG, "new_row_stride %d must be a multiple of 8 and >= %ld",
                row_stride, static_cast<long>(owned) * head_dim);
  return MLKV_OK;
}

mlkv_status check_window(int window, int sinks) {
  if (window < 0 || sinks < 0)
    return fail(MLKV_ERR_INVALID_ARG, "window %d and sinks %d must not be negative", window, sinks);
  return MLKV_OK;
}

// Tiles that T rows from any slot on may touch.
int touched_tiles(int T, bool from_zero) {
  const long first = from_zero ? 0 : kTileTokens - 1;
  return static_cast<int>((T + first + kTileTokens - 1) / kTileTokens);
}

mlkv_status check_blocks(int kv_count, int batch, int tiles) {
  if (static_cast<double>(kv_count) * batch * tiles > 2147483647.0)
    return fail(MLKV_ERR_CAPACITY, "more than 2^31 - 1 blocks of 32 tokens in one call");
  return MLKV_OK;
}

mlkv_status store_params(const mlkv_qcache* q4, const mlkv_cache* bf16, int T, int kv_begin,
                         int kv_count, const int32_t* starts, mlkv::StoreParams& p) {
  if (q4) {
    p.q4 = static_cast<uint8_t*>(q4->data);
    p.B = q4->batch;
    p.S = q4->capacity;
  } else {
    p.k = static_cast<uint16_t*>(bf16->k);
    p.v = static_cast<uint16_t*>(bf16->v);
    p.B = bf16->batch;
    p.S = bf16->capacity;
  }
  p.T = T;
  p.kv_begin = kv_begin;
  p.kv_count = kv_count;
  p.starts = starts;
  p.tiles = touched_tiles(T, !starts);
  const mlkv_status s = check_blocks(kv_count, p.B, p.tiles);
  if (s == MLKV_OK) p.store_items = static_cast<unsigned>(kv_count) * p.B * p.tiles;
  return s;
}

mlkv_status launch_store_checked(const mlkv::StoreParams& p, int head_dim, bool norm,
                                 hipStream_t stream) {
  const hipError_t err = mlkv::launch_store(p, head_dim, norm, stream);
  if (err != hipSuccess) return fail(MLKV_ERR_HIP, "append launch: %s", hipGetErrorString(err));
  return ok();
}

// Rows of heads [kv_begin, kv_begin + kv_count) of a 4-bit cache, in or out.
mlkv_status check_rows(const mlkv_qcache* cache, int kv_begin, int kv_count, const int32_t* starts,
                       int T) {
  mlkv_status s;
  if ((s = check_qcache(cache)) != MLKV_OK) return s;
  if (kv_begin < 0 || kv_count < 0 || kv_begin + static_cast<long>(kv_count) > cache->n_kv)
    return fail(MLKV_ERR_INVALID_ARG, "KV heads [%d, %d + %d) outside [0, %d)", kv_begin, kv_begin,
                kv_count, cache->n_kv);
  if ((s = check_tokens(T, cache->capacity)) != MLKV_OK) return s;
  if (!aligned4(starts)) return fail(MLKV_ERR_ALIGNMENT, "starts must be 4-byte aligned");
  return MLKV_OK;
}

mlkv_status check_row_buffers(const void* k_rows, const void* v_rows) {
  if (!k_rows || !v_rows) return fail(MLKV_ERR_INVALID_ARG, "k_rows and v_rows must be non-NULL");
  if (!aligned16(k_rows) || !aligned16(v_rows))
    return fail(MLKV_ERR_ALIGNMENT, "k_rows and v_rows must be 16-byte aligned");
  return MLKV_OK;
}

// How a layer's (sequence, KV head) units are cut (span.hip): `chunks` parts of
// the G query rows, runs of run_tiles tiles, at most `runs` of a unit.
// runs: as many as give every compute unit one workgroup of eight waves, of at
// least two tiles a wave (us, on 256 such workgroups / 512 / 1024 of four waves:
// 8 x 32768 tokens of four heads in 4 bits 16.0 / 17.8 / 19.1, 128 ragged
// sequences 8.1 / 8.7 / 10.4, 4 x 16000 tokens of two heads of 128 channels
// 11.8 / 14.9 / 15.0; runs of one tile a wave instead of two 7.0 -> 8.0 for two
// windows of 4096).  Where those workgroups, or the unsplit units, leave more
// than a seventh of their rounds of the compute units idle, long units are cut
// into up to kSpanFill workgroups of four waves a compute unit, of at least
// kSpanLongTiles tiles (us, cut / not, 4 bits: 300 units of 4000 .. 32000 tokens
// 81 / 129, 140 of 8000 .. 16000 30 / 43, 264 of 8000 34 / 45, 320 of 16000 with
// 128 channels 125 / 134; bf16, 288 windows of 4096 114 / 134; from 16 tiles on
// instead, 384 bf16 windows of 1023 take 45.6 for 41.9).  bf16 units that are no
// more than the compute units take only the first cut, into cus / units runs: those
// that it leaves whole reach the memory's rate as they are (160 windows of 4096
// cut / not: 68 / 63).  Grids of more workgroups than compute units
// take four waves, of which more are resident at once (48 x 8 windows of 1023,
// 128 channels, bf16 43.8 / 45.3).
struct SpanPlan {
  int chunks, chunk_rows, runs, run_tiles, waves;
  long units;
  size_t ml, need;  // offset of the (max, denominator) pairs, bytes in all; 0 without split runs
};
constexpr int kSpanMinTiles = 16, kSpanLongTiles = 32;
constexpr long kSpanFill = 6;

SpanPlan span_plan(const mlkv_map* map, int layer, int batch, int head_dim, bool four_bits,
                   int max_len, int window, int sinks) {
  SpanPlan pl{};
  const int G = map->group[layer];
  const int blocks = (G + 15) / 16;
  pl.units = static_cast<long>(batch) * map->kv_count[layer];
  const int most = mlkv::span_max_blocks(head_dim, four_bits);
  pl.chunks = (blocks + most - 1) / most;
  pl.chunk_rows = (G + pl.chunks - 1) / pl.chunks;
  int tiles = tiles_of(max_len < 1 ? 1 : max_len);
  if (window > 0) {  // both ends of the window and the first tokens' end inside a tile
    const long bound = tiles_of(window) + 1L + (sinks + static_cast<long>(kTileTokens) - 1) / kTileTokens;
    tiles = static_cast<int>(tiles < bound ? tiles : bound);
  }
  const long groups = pl.units * pl.chunks;
  const long cus = compute_units_or_fallback();
  long runs = cus / groups;
  const long longest = tiles / kSpanMinTiles;
  runs = runs < longest ? runs : longest;
  runs = runs < 1 ? 1 : runs;
  const long rounds = (groups * runs + cus - 1) / cus * cus;
  if (20 * groups * runs < 17 * rounds && (four_bits || groups > cus)) {
    long fill = kSpanFill * cus / groups;
    fill = fill < tiles / kSpanLongTiles ? fill : tiles / kSpanLongTiles;
    runs = runs > fill ? runs : fill;
  }
  pl.runs = static_cast<int>(runs);
  pl.run_tiles = (tiles + pl.runs - 1) / pl.runs;
  pl.waves = groups * pl.runs <= cus ? 8 : 4;
  if (pl.runs > 1) {
    const int segments = (pl.runs + mlkv::kSpanSegment - 1) / mlkv::kSpanSegment;
    const size_t part_rows = static_cast<size_t>(groups) * (pl.runs + segments) * pl.chunk_rows;
    pl.ml = kCounterSlots * sizeof(int32_t) + align_up(part_rows * head_dim * sizeof(float), 256);
    pl.need = pl.ml + part_rows * 2 * sizeof(float);
  }
  return pl;
}

mlkv_status span_attention(int layer, const void* q, const mlkv_cache* bf16, const mlkv_qcache* q4,
                           const mlkv_map* map, const int32_t* seq_lens, int window, int sinks,
                           void* out, mlkv_out_dtype out_dtype, int max_len_hint, void* workspace,
                           size_t workspace_bytes, hipStream_t stream) {
  const int B = q4 ? q4->batch : bf16->batch, S = q4 ? q4->capacity : bf16->capacity;
  const int D = q4 ? q4->head_dim : bf16->head_dim;
  if (!q || !seq_lens || !out)
    return fail(MLKV_ERR_INVALID_ARG, "q, seq_lens, out must be non-NULL");
  if (!aligned16(q) || !aligned16(out))
    return fail(MLKV_ERR_ALIGNMENT, "q and out must be 16-byte aligned");
  if (!aligned4(seq_lens)) return fail(MLKV_ERR_ALIGNMENT, "seq_lens must be 4-byte aligned");
  if (out_dtype != MLKV_OUT_F32 && out_dtype != MLKV_OUT_BF16)
    return fail(MLKV_ERR_INVALID_ARG, "bad out_dtype");
  mlkv_status s;
  if ((s = check_window(window, sinks)) != MLKV_OK) return s;
  if (max_len_hint > S)
    return fail(MLKV_ERR_CAPACITY, "max_len_hint %d above capacity %d", max_len_hint, S);
  const int max_len = max_len_hint <= 0 ? S : max_len_hint;
  window = window < S ? window : S;  // larger ones say the same
  sinks = sinks < S ? sinks : S;
  const SpanPlan pl = span_plan(map, layer, B, D, q4 != nullptr, max_len, window, sinks);
  // A grid has fewer than 2^32 threads.
  if (static_cast<double>(pl.units) * pl.runs * pl.chunks >= (1L << 24) - 8.0 * pl.chunks)
    return fail(MLKV_ERR_UNSUPPORTED, "%ld (sequence, KV head) units: more than one launch takes",
                pl.units);
  if (pl.need > 0 && (!workspace || workspace_bytes < pl.need))
    return fail(MLKV_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", pl.need,
                workspace ? workspace_bytes : 0);
  if (pl.need > 0 && !aligned16(workspace))
    return fail(MLKV_ERR_ALIGNMENT, "workspace not 16-byte aligned");
  if ((s = check_lengths_if_requested(seq_lens, B, 0, max_len, stream)) != MLKV_OK) return s;
  mlkv::SpanParams p{};
  p.q = static_cast<const uint16_t*>(q);
  if (q4) {
    p.q4 = static_cast<const uint8_t*>(q4->data);
  } else {
    p.k = static_cast<const uint16_t*>(bf16->k);
    p.v = static_cast<const uint16_t*>(bf16->v);
  }
  p.lens = seq_lens;
  p.out = out;
  if (pl.need > 0) {
    char* base = static_cast<char*>(workspace);
    p.counters = reinterpret_cast<int*>(base);
    p.part_acc = reinterpret_cast<float*>(base + kCounterSlots * sizeof(int32_t));
    p.part_ml = reinterpret_cast<float*>(base + pl.ml);
  }
  p.B = B;
  p.h = map->h;
  p.S = S;
  p.kv_begin = map->kv_begin[layer];
  p.n_groups = map->kv_count[layer];
  p.G = map->group[layer];
  p.chunks = pl.chunks;
  p.chunk_rows = pl.chunk_rows;
  p.runs = pl.runs;
  p.run_tiles = pl.run_tiles;
  p.waves = pl.waves;
  p.items = static_cast<unsigned>(pl.units * pl.runs);
  p.max_len = max_len;
  p.window = window;
  p.sinks = sinks;
  p.out_bf16 = out_dtype == MLKV_OUT_BF16 ? 1 : 0;
  p.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(D)));
  Profile& prof = g_profile;
  const bool timed = prof.on && prof.used < static_cast<int>(prof.start.size());
  const hipError_t err = mlkv::launch_span(p, D, stream, timed ? prof.start[prof.used] : nullptr,
                                           timed ? prof.stop[prof.used] : nullptr);
  if (err != hipSuccess) return fail(MLKV_ERR_HIP, "attention launch: %s", hipGetErrorString(err));
  if (timed) ++prof.used;
  return ok();
}

// A number not below 0 as fp32, inf where fp32 ends (a cast alone is undefined there).
float to_float(double x) { return x > FLT_MAX ? HUGE_VALF : static_cast<float>(x); }

// Passes of a query workgroup (below; us, 16000 tokens of 12 and 4 heads of 64
// channels, all turned, with 8 / 4 / 16 workgroups a compute unit 18.2 / 19.5 /
// 18.7; 8000 of 32 and 8 heads of 128 with at most 4 / 8 passes 45.8 / 47.5).
constexpr long kQueryGroupsPerCu = 8, kMaxQueryPasses = 4;

mlkv_status norm_rope_append(int layer, const mlkv_map* map, const mlkv_cache* bf16,
                             const mlkv_qcache* q4, const void* q, int q_row_stride,
                             const void* k_new, const void* v_new, int new_row_stride, int T,
                             const int32_t* ctx_lens, const mlkv_norm_rope* nr, void* q_out,
                             hipStream_t stream) {
  const int B = q4 ? q4->batch : bf16->batch, S = q4 ? q4->capacity : bf16->capacity;
  const int D = q4 ? q4->head_dim : bf16->head_dim, h = map->h, owned = map->own_count[layer];
  mlkv_status s;
  if ((s = check_tokens(T, S)) != MLKV_OK) return s;
  if (!nr) return fail(MLKV_ERR_INVALID_ARG, "norm_rope is NULL");
  if (nr->rotary_dims < 0 || nr->rotary_dims > D || nr->rotary_dims % 16 != 0)
    return fail(MLKV_ERR_UNSUPPORTED, "rotary_dims %d: a multiple of 16 in [0, head_dim] required",
                nr->rotary_dims);
  if (nr->rotary_dims > 0 && (!(nr->rotary_base > 0.0) || !std::isfinite(nr->rotary_base)))
    return fail(MLKV_ERR_INVALID_ARG, "rotary_base must be positive and finite");
  if (!(nr->eps >= 0.0) || !std::isfinite(nr->eps))
    return fail(MLKV_ERR_INVALID_ARG, "eps must be finite and not negative");
  if (!aligned16(nr->q_weight) || !aligned16(nr->k_weight))
    return fail(MLKV_ERR_ALIGNMENT, "norm weights must be 16-byte aligned");
  if (T == 0) return ok();
  if (!q || !q_out || !ctx_lens)
    return fail(MLKV_ERR_INVALID_ARG, "q, q_out and ctx_lens must be non-NULL");
  if (!aligned16(q) || !aligned16(q_out))
    return fail(MLKV_ERR_ALIGNMENT, "q and q_out must be 16-byte aligned");
  if (!aligned4(ctx_lens)) return fail(MLKV_ERR_ALIGNMENT, "ctx_lens must be 4-byte aligned");
  if (q_row_stride % 8 != 0 || q_row_stride < static_cast<long>(h) * D)
    return fail(MLKV_ERR_INVALID_ARG, "q_row_stride %d must be a multiple of 8 and >= %ld",
                q_row_stride, static_cast<long>(h) * D);
  if (owned > 0 && (s = check_new_rows(k_new, v_new, new_row_stride, owned, D)) != MLKV_OK) return s;
  if ((s = check_prefill_lengths_if_requested(ctx_lens, B, T, S, stream)) != MLKV_OK) return s;
  mlkv::StoreParams p{};
  if ((s = store_params(q4, bf16, T, owned > 0 ? map->own_begin[layer] : 0, owned, ctx_lens, p)) !=
      MLKV_OK)
    return s;
  p.k_src = static_cast<const uint16_t*>(k_new);
  p.v_src = static_cast<const uint16_t*>(v_new);
  p.s_head = D;
  p.s_tok = new_row_stride;
  p.s_seq = static_cast<size_t>(T) * new_row_stride;
  p.q_w = static_cast<const uint16_t*>(nr->q_weight);
  p.k_w = static_cast<const uint16_t*>(nr->k_weight);
  p.q = static_cast<const uint16_t*>(q);
  p.q_out = static_cast<uint16_t*>(q_out);
  p.q_stride = q_row_stride;
  p.h = h;
  // A query workgroup takes its rows in passes, more where there are workgroups
  // enough for every compute unit, of at most kAngleTokens tokens.
  const double rows = static_cast<double>(B) * T * h;
  if (rows > 2147483647.0)
    return fail(MLKV_ERR_UNSUPPORTED, "%.0f query rows: at most 2^31 - 1", rows);
  const long per_pass = mlkv::kStoreThreads / (D / 8), total = static_cast<long>(rows);
  const long most = (static_cast<long>(mlkv::kAngleTokens - 2) * h + 1) / per_pass;
  long passes = total / (per_pass * kQueryGroupsPerCu * compute_units_or_fallback());
  passes = passes < most ? passes : most;
  passes = passes < 1 ? 1 : passes > kMaxQueryPasses ? kMaxQueryPasses : passes;
  p.q_rows = static_cast<unsigned>(per_pass * passes);
  p.q_items = static_cast<unsigned>((total + p.q_rows - 1) / p.q_rows);
  if (static_cast<double>(p.store_items) + p.q_items > 2147483647.0)
    return fail(MLKV_ERR_CAPACITY, "more than 2^31 - 1 workgroups in one call");
  p.inv_h = 0xFFFFFFFFu / static_cast<uint32_t>(h);
  p.half = nr->rotary_dims / 2;
  p.inv_half = p.half ? ((1u << 20) + p.half - 1) / p.half : 0;
  p.eps = to_float(nr->eps);
  p.eps_up = to_float(nr->eps * 0x1p160);
  p.eps_down = to_float(nr->eps * 0x1p-160);
  // Revolutions base^(-2j / dims) / 2 pi, as the product of two powers each
  // (sixteen powers instead of up to 64, 3 us of a call).
  for (int j = 0; j < 8 && j < p.half; ++j)
    p.fine[j] = std::pow(nr->rotary_base, -2.0 * j / nr->rotary_dims);
  for (int j = 0; j < p.half; j += 8)
    p.coarse[j / 8] =
        std::pow(nr->rotary_base, -2.0 * j / nr->rotary_dims) * 0.15915494309189533577;
  return launch_store_checked(p, D, true, stream);
}

}  // namespace

extern "C" {

size_t mlkv_qcache_bytes(const mlkv_map* map, int batch, int capacity, int head_dim) {
  if (!map || batch <= 0 || capacity <= 0 || capacity % kTileTokens != 0 ||
      (head_dim != 64 && head_dim != 128))
    return 0;
  return static_cast<size_t>(map->n_kv) * batch * (capacity / kTileTokens) *
         mlkv::kQTileBytes(head_dim);
}

mlkv_status mlkv_qcache_append_rows(int layer, const mlkv_map* map, const mlkv_qcache* cache,
                                    const void* k_new, const void* v_new, int T,
                                    int new_row_stride, const int32_t* ctx_lens,
                                    hipStream_t stream) {
  mlkv_status s;
  if ((s = check_layer(map, layer)) != MLKV_OK) return s;
  if ((s = check_qcache(cache, map)) != MLKV_OK) return s;
  if ((s = check_tokens(T, cache->capacity)) != MLKV_OK) return s;
  const int owned = map->own_count[layer];
  if (owned == 0 || T == 0) return ok();
  if ((s = check_new_rows(k_new, v_new, new_row_stride, owned, cache->head_dim)) != MLKV_OK)
    return s;
  if (!ctx_lens) return fail(MLKV_ERR_INVALID_ARG, "ctx_lens must be non-NULL");
  if (!aligned4(ctx_lens)) return fail(MLKV_ERR_ALIGNMENT, "ctx_lens must be 4-byte aligned");
  if ((s = check_prefill_lengths_if_requested(ctx_lens, cache->batch, T, cache->capacity,
                                              stream)) != MLKV_OK)
    return s;
  mlkv::StoreParams p{};
  if ((s = store_params(cache, nullptr, T, map->own_begin[layer], owned, ctx_lens, p)) != MLKV_OK)
    return s;
  p.k_src = static_cast<const uint16_t*>(k_new);
  p.v_src = static_cast<const uint16_t*>(v_new);
  p.s_head = cache->head_dim;
  p.s_tok = new_row_stride;
  p.s_seq = static_cast<size_t>(T) * new_row_stride;
  return launch_store_checked(p, cache->head_dim, false, stream);
}

mlkv_status mlkv_qcache_write_rows(const mlkv_qcache* cache, int kv_begin, int kv_count,
                                   const int32_t* starts, int T, const void* k_rows,
                                   const void* v_rows, hipStream_t stream) {
  mlkv_status s;
  if ((s = check_rows(cache, kv_begin, kv_count, starts, T)) != MLKV_OK) return s;
  if (kv_count == 0 || T == 0) return ok();
  if ((s = check_row_buffers(k_rows, v_rows)) != MLKV_OK) return s;
  mlkv::StoreParams p{};
  if ((s = store_params(cache, nullptr, T, kv_begin, kv_count, starts, p)) != MLKV_OK) return s;
  p.k_src = static_cast<const uint16_t*>(k_rows);
  p.v_src = static_cast<const uint16_t*>(v_rows);
  p.s_tok = cache->head_dim;
  p.s_seq = p.s_tok * T;
  p.s_head = p.s_seq * cache->batch;
  return launch_store_checked(p, cache->head_dim, false, stream);
}

mlkv_status mlkv_qcache_read_rows(const mlkv_qcache* cache, int kv_begin, int kv_count,
                                  const int32_t* starts, int T, void* k_rows, void* v_rows,
                                  hipStream_t stream) {
  mlkv_status s;
  if ((s = check_rows(cache, kv_begin, kv_count, starts, T)) != MLKV_OK) return s;
  if (kv_count == 0 || T == 0) return ok();
  if ((s = check_row_buffers(k_rows, v_rows)) != MLKV_OK) return s;
  mlkv::ReadParams p{};
  p.q4 = static_cast<const uint8_t*>(cache->data);
  p.k_rows = static_cast<uint16_t*>(k_rows);
  p.v_rows = static_cast<uint16_t*>(v_rows);
  p.starts = starts;
  p.B = cache->batch;
  p.T = T;
  p.S = cache->capacity;
  p.kv_begin = kv_begin;
  p.kv_count = kv_count;
  p.tiles = touched_tiles(T, !starts);
  if ((s = check_blocks(kv_count, p.B, p.tiles)) != MLKV_OK) return s;
  p.items = static_cast<unsigned>(kv_count) * p.B * p.tiles;
  const hipError_t err = mlkv::launch_qcache_read(p, cache->head_dim, stream);
  if (err != hipSuccess) return fail(MLKV_ERR_HIP, "cache rows launch: %s", hipGetErrorString(err));
  return ok();
}

size_t mlkv_workspace_bytes_window(const mlkv_map* map, int batch, int capacity, int head_dim) {
  if (!map || batch <= 0 || capacity <= 0 || (head_dim != 64 && head_dim != 128)) return 0;
  // The most runs are those without a window at the capacity.
  size_t most = 0;
  for (int n = 0; n < map->l; ++n) {
    for (const bool four_bits : {false, true}) {
      const size_t need = span_plan(map, n, batch, head_dim, four_bits, capacity, 0, 0).need;
      most = need > most ? need : most;
    }
  }
  return most;
}

mlkv_status mlkv_qcache_decode_attention(int layer, const void* q, const mlkv_qcache* cache,
                                         const mlkv_map* map, const int32_t* seq_lens, int window,
                                         int sinks, void* out, mlkv_out_dtype out_dtype,
                                         int max_len_hint, void* workspace, size_t workspace_bytes,
                                         hipStream_t stream) {
  mlkv_status s;
  if ((s = check_layer(map, layer)) != MLKV_OK) return s;
  if ((s = check_qcache(cache, map)) != MLKV_OK) return s;
  return span_attention(layer, q, nullptr, cache, map, seq_lens, window, sinks, out, out_dtype,
                        max_len_hint, workspace, workspace_bytes, stream);
}

mlkv_status mlkv_decode_attention_window(int layer, const void* q, const mlkv_cache* cache,
                                         const mlkv_map* map, const int32_t* seq_lens, int window,
                                         int sinks, void* out, mlkv_out_dtype out_dtype,
                                         int max_len_hint, void* workspace, size_t workspace_bytes,
                                         hipStream_t stream) {
  mlkv_status s;
  if ((s = check_layer(map, layer)) != MLKV_OK) return s;
  if ((s = check_cache(cache, map)) != MLKV_OK) return s;
  return span_attention(layer, q, cache, nullptr, map, seq_lens, window, sinks, out, out_dtype,
                        max_len_hint, workspace, workspace_bytes, stream);
}

mlkv_status mlkv_prefill_attention_window(int layer, const void* q, const mlkv_cache* cache,
                                          const mlkv_map* map, const int32_t* ctx_lens, int T,
                                          int window, int sinks, void* out,
                                          mlkv_out_dtype out_dtype, hipStream_t stream) {
  mlkv_status s;
  if ((s = check_layer(map, layer)) != MLKV_OK) return s;
  if ((s = check_cache(cache, map)) != MLKV_OK) return s;
  if ((s = check_tokens(T, cache->capacity)) != MLKV_OK) return s;
  if ((s = check_window(window, sinks)) != MLKV_OK) return s;
  const int B = cache->batch, D = cache->head_dim, G = map->group[layer];
  const long per_wg = mlkv::kWindowRows;
  if ((static_cast<long>(T) * G + per_wg - 1) / per_wg > kMaxGridY)
    return fail(MLKV_ERR_UNSUPPORTED, "T * (query heads per KV head) = %ld rows: at most %ld",
                static_cast<long>(T) * G, kMaxGridY * per_wg);
  if (static_cast<long>(B) * map->kv_count[layer] >= mlkv::kMaxPrefillUnits)
    return fail(MLKV_ERR_UNSUPPORTED, "%ld (sequence, KV head) units: at most %ld",
                static_cast<long>(B) * map->kv_count[layer], mlkv::kMaxPrefillUnits - 1);
  if (out_dtype != MLKV_OUT_F32 && out_dtype != MLKV_OUT_BF16)
    return fail(MLKV_ERR_INVALID_ARG, "bad out_dtype");
  if (T == 0) return ok();
  if (!q || !ctx_lens || !out)
    return fail(MLKV_ERR_INVALID_ARG, "q, ctx_lens, out must be non-NULL");
  if (!aligned16(q) || !aligned16(out))
    return fail(MLKV_ERR_ALIGNMENT, "q and out must be 16-byte aligned");
  if (!aligned4(ctx_lens)) return fail(MLKV_ERR_ALIGNMENT, "ctx_lens must be 4-byte aligned");
  if ((s = check_prefill_lengths_if_requested(ctx_lens, B, T, cache->capacity, stream)) != MLKV_OK)
    return s;
  mlkv::WindowPrefillParams p{};
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(cache->k);
  p.v = static_cast<const uint16_t*>(cache->v);
  p.ctx = ctx_lens;
  p.out = out;
  p.B = B;
  p.T = T;
  p.h = map->h;
  p.S = cache->capacity;
  p.kv_begin = map->kv_begin[layer];
  p.G = G;
  p.n_groups = map->kv_count[layer];
  p.layers = 1;
  p.kv_per_layer = p.n_groups;
  p.out_bf16 = out_dtype == MLKV_OUT_BF16 ? 1 : 0;
  p.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(D)));
  p.window = window < p.S ? window : p.S;  // larger ones say the same
  p.sinks = sinks < p.S ? sinks : p.S;
  p.inv_G = 0xFFFFFFFFu / static_cast<uint32_t>(G);
  Profile& prof = g_profile;
  const bool timed = prof.on && prof.used < static_cast<int>(prof.start.size());
  const hipError_t err =
      mlkv::launch_prefill_window(p, D, stream, timed ? prof.start[prof.used] : nullptr,
                                  timed ? prof.stop[prof.used] : nullptr);
  if (err != hipSuccess) return fail(MLKV_ERR_HIP, "prefill launch: %s", hipGetErrorString(err));
  if (timed) ++prof.used;
  return ok();
}

mlkv_status mlkv_norm_rope_append(int layer, const mlkv_map* map, const mlkv_cache* cache,
                                  const void* q, int q_row_stride, const void* k_new,
                                  const void* v_new, int new_row_stride, int T,
                                  const int32_t* ctx_lens, const mlkv_norm_rope* norm_rope,
                                  void* q_out, hipStream_t stream) {
  mlkv_status s;
  if ((s = check_layer(map, layer)) != MLKV_OK) return s;
  if ((s = check_cache(cache, map)) != MLKV_OK) return s;
  return norm_rope_append(layer, map, cache, nullptr, q, q_row_stride, k_new, v_new,
                          new_row_stride, T, ctx_lens, norm_rope, q_out, stream);
}

mlkv_status mlkv_qcache_norm_rope_append(int layer, const mlkv_map* map, const mlkv_qcache* cache,
                                         const void* q, int q_row_stride, const void* k_new,
                                         const void* v_new, int new_row_stride, int T,
                                         const int32_t* ctx_lens, const mlkv_norm_rope* norm_rope,
                                         void* q_out, hipStream_t stream) {
  mlkv_status s;
  if ((s = check_layer(map, layer)) != MLKV_OK) return s;
  if ((s = check_qcache(cache, map)) != MLKV_OK) return s;
  return norm_rope_append(layer, map, nullptr, cache, q, q_row_stride, k_new, v_new,
                          new_row_stride, T, ctx_lens, norm_rope, q_out, stream);
}

}  // extern "C"
