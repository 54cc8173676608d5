// Drives the host code of the long-context operators over small and extreme
// arguments under sanitizers, and checks what each launch would be given
// against the arrays the kernels index with it.
#include <limits.h>
#include <math.h>
#include <stdio.h>
#include <string.h>

#include "mlkv.h"
#include "serve.h"

extern long serve_launches;
extern mlkv::SpanParams last_span;
extern mlkv::StoreParams last_store;
extern mlkv::ReadParams last_read;
extern mlkv::WindowPrefillParams last_window;
extern int last_head_dim;
extern bool last_norm;

static int failures = 0;
#define CHECK(x)                                                    \
  do {                                                              \
    if (!(x)) {                                                     \
      ++failures;                                                   \
      printf("%s:%d: %s (%s)\n", __FILE__, __LINE__, #x, mlkv_last_error()); \
    }                                                               \
  } while (0)

static void* P(size_t at = 0) { return reinterpret_cast<void*>(uintptr_t(1) << 20 | at); }

// What span_kernel indexes: units and runs on the grid, tiles of a run, and
// counters and partials inside the workspace.
static void check_span(size_t ws_bytes, int max_len, int window, int sinks) {
  const mlkv::SpanParams& p = last_span;
  const long units = static_cast<long>(p.B) * p.n_groups;
  CHECK(p.waves == 4 || p.waves == 8);
  CHECK(p.chunks >= 1 && static_cast<long>(p.chunks) * p.chunk_rows >= p.G);
  CHECK((p.chunks - 1L) * p.chunk_rows < p.G);
  CHECK(p.chunk_rows <= 16 * mlkv::span_max_blocks(last_head_dim, p.q4 != nullptr));
  CHECK(p.runs >= 1 && p.items == static_cast<unsigned>(units * p.runs));
  const double groups = (p.items + 7) / 8 * 8.0 * p.chunks;
  CHECK(groups * 64 * p.waves < 4294967296.0);
  CHECK(p.window >= 0 && p.window <= p.S && p.sinks >= 0 && p.sinks <= p.S);
  CHECK(p.max_len >= 1 && p.max_len <= p.S && (max_len <= 0 || p.max_len == max_len));
  // The runs of the longest span take all its tiles.
  long tiles = (p.max_len + 31L) / 32;
  if (window > 0) {
    const long cover = (window - 1L) / 32 + 2 + (sinks + 31L) / 32;
    tiles = tiles < cover ? tiles : cover;
  }
  CHECK(static_cast<long>(p.runs) * p.run_tiles >= tiles);
  if (p.runs > 1) {
    const long segments = (p.runs + mlkv::kSpanSegment - 1) / mlkv::kSpanSegment;
    const char* base = reinterpret_cast<const char*>(p.counters);
    const size_t rows = static_cast<size_t>(units) * p.chunks * (p.runs + segments) * p.chunk_rows;
    CHECK(units * p.chunks * (1 + segments) * 4 <= 262144);
    const char* acc = reinterpret_cast<const char*>(p.part_acc);
    const char* ml = reinterpret_cast<const char*>(p.part_ml);
    CHECK(acc >= base + 262144 && acc + rows * last_head_dim * 4 <= ml);
    CHECK(ml + rows * 8 <= base + ws_bytes);
    CHECK((p.runs + segments) * static_cast<size_t>(p.chunk_rows) * last_head_dim * 4 < (1u << 31));
  }
}

static void decode(int l, int h, int m, int g) {
  mlkv_map* map = nullptr;
  CHECK(mlkv_map_create_uniform(l, h, m, g, &map) == MLKV_OK);
  const int batches[] = {1, 3, 128, 300, 5000}, caps[] = {32, 640, 32768, INT_MAX / 64 * 32};
  for (int B : batches)
    for (int S : caps)
      for (int D : {64, 128}) {
        const size_t need = mlkv_workspace_bytes_window(map, B, S, D);
        const mlkv_qcache qc = {P(), m * g, B, S, D};
        const mlkv_cache c = {P(), P(), m * g, B, S, D};
        for (int hint : {0, 1, 31, S})
          for (int window : {0, 1, 31, 4096, INT_MAX})
            for (int sinks : {0, 5, INT_MAX}) {
              const long before = serve_launches;
              CHECK(mlkv_qcache_decode_attention(l - 1, P(), &qc, map, (int*)P(), window, sinks,
                                                 P(), MLKV_OUT_F32, hint, P(), need,
                                                 nullptr) == MLKV_OK);
              check_span(need, hint, window, sinks);
              CHECK(mlkv_decode_attention_window(l - 1, P(), &c, map, (int*)P(), window, sinks,
                                                 P(), MLKV_OUT_BF16, hint, P(), need,
                                                 nullptr) == MLKV_OK);
              check_span(need, hint, window, sinks);
              CHECK(serve_launches == before + 2);
            }
        if (need > 0)
          CHECK(mlkv_qcache_decode_attention(0, P(), &qc, map, (int*)P(), 0, 0, P(), MLKV_OUT_F32,
                                             0, P(), need - 1, nullptr) == MLKV_ERR_WORKSPACE);
      }
  mlkv_map_destroy(map);
}

static void rows(int h, int g) {
  mlkv_map* map = nullptr;
  CHECK(mlkv_map_create_uniform(2, h, 1, g, &map) == MLKV_OK);
  for (int B : {1, 7, 4096})
    for (int S : {32, 4096, 1 << 20})
      for (int D : {64, 128}) {
        const mlkv_qcache qc = {P(), g, B, S, D};
        const mlkv_cache c = {P(), P(), g, B, S, D};
        for (int T : {1, 2, 31, 32, 33, 4096, 1 << 20}) {
          if (T > S) continue;
          const double blocks = static_cast<double>(g) * B * ((T + 62) / 32);
          const mlkv_status fits = blocks > 2147483647.0 ? MLKV_ERR_CAPACITY : MLKV_OK;
          CHECK(mlkv_qcache_append_rows(0, map, &qc, P(), P(), T, g * D, (int*)P(), nullptr) == fits);
          if (fits == MLKV_OK)
            CHECK(last_store.store_items == static_cast<unsigned>(blocks) && !last_norm &&
                  last_store.tiles * 32 >= T + 31);
          if (static_cast<double>(g) * B * ((T + 31) / 32) <= 2147483647.0) {
            CHECK(mlkv_qcache_write_rows(&qc, 0, g, nullptr, T, P(), P(), nullptr) == MLKV_OK);
            CHECK(last_store.tiles == (T + 31) / 32);
            CHECK(mlkv_qcache_read_rows(&qc, 0, g, nullptr, T, P(), P(), nullptr) == MLKV_OK);
            CHECK(last_read.tiles == (T + 31) / 32);
          }
          const mlkv_norm_rope nr = {P(), nullptr, 1e-6, D, 1e4};
          const double q_rows = static_cast<double>(B) * T * h;
          for (int layer : {0, 1}) {
            const mlkv_status s = mlkv_norm_rope_append(layer, map, &c, P(), h * D, P(), P(), g * D,
                                                        T, (int*)P(), &nr, P(), nullptr);
            if (s != MLKV_OK) {
              CHECK(q_rows > 2147483647.0 || blocks > 2147483647.0 - q_rows);
              continue;
            }
            const mlkv::StoreParams& p = last_store;
            CHECK(last_norm && p.store_items == (layer == 0 ? static_cast<unsigned>(blocks) : 0u));
            CHECK(static_cast<double>(p.q_items) * p.q_rows >= q_rows &&
                  (p.q_items - 1.0) * p.q_rows < q_rows);
            // Tokens of a workgroup's rows: its angles fit.
            CHECK((p.q_rows - 1) / h + 2 <= static_cast<unsigned>(mlkv::kAngleTokens));
            CHECK(p.half == D / 2);
            for (int j = 0; j < p.half; ++j) {
              const double want = pow(1e4, -2.0 * j / D) / (2 * M_PI);
              CHECK(fabs(p.coarse[j / 8] * p.fine[j % 8] - want) <= 4e-16 * want);
            }
          }
          if (static_cast<long>(T) * (h / g) <= 65535L * 128) {
            CHECK(mlkv_prefill_attention_window(1, P(), &c, map, (int*)P(), T, INT_MAX, INT_MAX, P(),
                                                MLKV_OUT_F32, nullptr) == MLKV_OK);
            CHECK(last_window.window == S && last_window.sinks == S);
            // The kernel's division of a row by the group size.
            const long G = last_window.G;
            for (long n : {0L, 1L, G - 1, G, G + 1, T * G / 2, T * G - 1}) {
              const long q = static_cast<long>(static_cast<unsigned long>(n) * last_window.inv_G >> 32);
              CHECK((n - q * G >= G ? q + 1 : q) == n / G);
            }
          }
        }
      }
  mlkv_map_destroy(map);
}

int main() {
  decode(4, 12, 2, 1);
  decode(2, 140, 1, 2);
  decode(1, 33, 1, 33);
  decode(3, 32, 3, 8);
  rows(12, 1);
  rows(32, 8);
  rows(1, 1);
  rows(200, 1);
  printf("%ld launches, %d failure(s)\n", serve_launches, failures);
  return failures != 0;
}
