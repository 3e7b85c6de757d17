// The attention kernel over an f16 cache.
#include "kv_attend.cuh"

namespace lc {
cudaError_t launch_attend_f16(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return launch_format<LACACHE_KV_F16>(a, num_sms, st);
}
}  // namespace lc
