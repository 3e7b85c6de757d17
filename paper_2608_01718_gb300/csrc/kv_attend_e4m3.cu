// The attention kernel over an e4m3 cache.
#include "kv_attend.cuh"

namespace lc {
cudaError_t launch_attend_e4m3(const AttendArgs& a, int num_sms, cudaStream_t st) {
  return launch_format<LACACHE_KV_E4M3>(a, num_sms, st);
}
}  // namespace lc
