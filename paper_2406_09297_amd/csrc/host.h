// What the C-ABI sources share on the host: the map's structure, error
// reporting, argument checks and the launch timing.  Defined in mlkv.cpp.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <vector>

#include "mlkv.h"

struct mlkv_map {
  int l = 0, h = 0, n_kv = 0;
  std::vector<int32_t> kv_of;     // [l*h]
  std::vector<int32_t> owner_of;  // [n_kv]
  // per layer: the KV heads read form [kv_begin, kv_begin + kv_count), G = h / kv_count
  std::vector<int> kv_begin, kv_count, group;
  // per layer: the KV heads appended form [own_begin, own_begin + own_count)
  std::vector<int> own_begin, own_count;
  // > 0: the layers fall into groups of this many consecutive layers, each
  // reading the same number of KV heads, its own, which its first layer
  // appends (every uniform map): a decode step may take all layers at once.
  int layers_per_group = 0;
};

namespace mlkv {
namespace host {

// Records the message of the calling thread's last failure and returns s.
mlkv_status fail(mlkv_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
mlkv_status ok();  // clears it

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

constexpr int kTileTokens = 32;
inline int tiles_of(int len) { return (len + kTileTokens - 1) / kTileTokens; }

mlkv_status check_map(const mlkv_map* map);
mlkv_status check_cache(const mlkv_cache* c, const mlkv_map* map);
// MLKV_CHECK=1 (synchronizes): every lens[b] + offset in [0, limit]; every
// ctx[b] in [0, S - T].
mlkv_status check_lengths_if_requested(const int32_t* lens, int batch, int offset, int limit,
                                       hipStream_t stream);
mlkv_status check_prefill_lengths_if_requested(const int32_t* ctx, int batch, int T, int S,
                                               hipStream_t stream);

constexpr long kCounterSlots = 65536;  // arrival counters of a workspace
constexpr long kMaxGridY = 65535;
long compute_units_or_fallback();

// Event pairs around attention launches (mlkv_profile_*).
struct Profile {
  std::vector<hipEvent_t> start, stop;
  int used = 0;
  bool on = false;
};
extern thread_local Profile g_profile;

}  // namespace host
}  // namespace mlkv
