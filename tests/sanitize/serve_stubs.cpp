// Host stand-ins for the launches of the long-context operators (see
// kernel_stubs.cpp): each succeeds, is counted, and keeps its parameters.
#include "serve.h"

long serve_launches = 0;
mlkv::SpanParams last_span;
mlkv::StoreParams last_store;
mlkv::ReadParams last_read;
mlkv::WindowPrefillParams last_window;
int last_head_dim = 0;
bool last_norm = false;

namespace mlkv {

hipError_t launch_store(const StoreParams& p, int head_dim, bool norm, hipStream_t) {
  ++serve_launches;
  last_store = p;
  last_head_dim = head_dim;
  last_norm = norm;
  return hipSuccess;
}
hipError_t launch_qcache_read(const ReadParams& p, int head_dim, hipStream_t) {
  ++serve_launches;
  last_read = p;
  last_head_dim = head_dim;
  return hipSuccess;
}
hipError_t launch_span(const SpanParams& p, int head_dim, hipStream_t, hipEvent_t, hipEvent_t) {
  ++serve_launches;
  last_span = p;
  last_head_dim = head_dim;
  return hipSuccess;
}
hipError_t launch_prefill_window(const WindowPrefillParams& p, int head_dim, hipStream_t,
                                 hipEvent_t, hipEvent_t) {
  ++serve_launches;
  last_window = p;
  last_head_dim = head_dim;
  return hipSuccess;
}

}  // namespace mlkv
