// A stand-in for the kernels under csrc/cache.cpp, for CPU tests: it keeps what
// the host would have passed to the rotation's kernel.

#include "cache.h"
#include "host_error.h"

using namespace mesh_attn;

namespace {
RopeParams rope;
}

namespace mesh_attn {

namespace host {
ma_status_t fail(ma_status_t st, const char*, ...) { return st; }
ma_status_t ok() { return MA_OK; }
}  // namespace host

hipError_t launch_cache_tables(const TablesParams&, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_cache_append(const StoreParams&, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_cache_read(const LoadParams&, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_cache_fwd(const CacheFwdParams&, bool, void*, hipStream_t) {
  return hipSuccess;
}
size_t cache_fwd_workspace(const CacheDims&, int32_t, int64_t) { return 0; }
hipError_t launch_rope(const RopeParams& p, bool, hipStream_t) {
  rope = p;
  return hipSuccess;
}

}  // namespace mesh_attn

extern "C" {
const char* hipGetErrorString(hipError_t) { return "stub error"; }
void stub_turns(uint64_t* out) {
  for (int i = 0; i < kRopeMaxPairs; ++i) out[i] = rope.t.turn[i];
}
}
