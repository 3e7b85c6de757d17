// The attention kernel over an int8 cache.
#include "kv_attend.cuh"

namespace lc {
cudaError_t launch_attend_int8(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return launch_format<LACACHE_KV_INT8>(a, num_sms, st);
}
}  // namespace lc
